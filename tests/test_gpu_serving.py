"""The serving calls together (the example's loop), from several host threads, and
without allocating device memory."""
import importlib.util
import os
import threading

import pytest
import torch

from paper_2509_16686_gb300 import _lib

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("serve", os.path.join(ROOT, "examples", "serve.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("kw", [dict(), dict(document=64, sequences=1, steps=1, budget=2),
                                dict(document=4100, sequences=30, steps=130, budget=64)])
def test_example_agrees_with_the_dense_decode(gpu_lib, kw):
    """Both forms and the dense decode are within rel-L2 5e-3 of the exact result; the
    sparse one is the dense decode over the chosen pages, bit for bit."""
    shared, sparse, all_free, status = example().main(**kw)
    assert shared <= 1e-2 and sparse == 0.0 and all_free and status == 0


def states():
    """(call, outputs) of every serving call on a layer of its own."""
    serve = example()
    layer = serve.Layer(4, 200, 40, seed=5)
    layer.plan([1500, 700, 64, 3])
    for b, n in enumerate((1500, 700, 64, 3)):
        layer.prefill(b, n)
    layer.summarise()
    q = layer.tokens(4)[3]
    out = torch.zeros((4, 16, 128), dtype=torch.bfloat16, device="cuda")
    prefix, plen = layer.table[0, :24].contiguous(), layer.lens[:1].contiguous()
    own = layer.table[1:].contiguous()
    lens = layer.lens[1:].contiguous()
    ws = layer.bytes(max(_lib.eg_mla_decode_shared_workspace_size(layer.dims, 3, 1500),
                         _lib.eg_mla_decode_sparse_workspace_size(layer.dims, 4, 40, 6)))
    lens_out, free_out = torch.empty_like(layer.lens), torch.empty_like(layer.free_count)

    def shared(stream=None):
        _lib.eg_mla_decode_shared(layer.dims, q[1:], *layer.cache(), prefix, plen, 1500, own, lens, 1500, *layer.gate,
                                  layer.w_uk, layer.w_uv, out[1:], ws, dev_status=layer.status, stream=stream)

    def sparse(stream=None):
        _lib.eg_mla_decode_sparse(layer.dims, q, *layer.cache(), layer.table, layer.lens, 1500, layer.summary, 6, 1, 1,
                                  *layer.gate, layer.w_uk, layer.w_uv, out, ws, dev_status=layer.status, stream=stream)

    def summary(stream=None):
        _lib.eg_mla_page_summary(layer.dims, *layer.cache(), layer.table, layer.lens, 1500, *layer.gate, layer.summary,
                                 dev_status=layer.status, stream=stream)

    def plan(stream=None):
        _lib.eg_mla_page_plan(layer.new, layer.lens, lens_out, layer.table.clone(), layer.free, layer.free_count,
                              free_out, layer.cu, layer.positions, layer.slots, dev_status=layer.status, stream=stream)

    layer.new = torch.tensor([1, 1, 0, 500], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    return {"shared": (shared, out), "sparse": (sparse, out), "summary": (summary, layer.summary),
            "plan": (plan, layer.slots)}, layer


@pytest.mark.parametrize("name", ["shared", "sparse", "summary", "plan"])
def test_two_threads_leave_each_other_alone(gpu_lib, name):
    results = {}

    def work(k):
        torch.cuda.set_device(0)
        calls, layer = states()
        call, out = calls[name]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                call(stream)
        stream.synchronize()
        results[k] = (out.clone(), int(layer.status.item()))
        torch.cuda.synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    (a, sa), (b, sb) = results[0], results[1]
    assert sa == 0 and sb == 0 and torch.equal(a, b)


@pytest.mark.parametrize("name", ["shared", "sparse", "summary"])
def test_calls_allocate_nothing_and_can_be_captured(gpu_lib, name):
    calls, layer = states()
    call, out = calls[name]
    call()
    torch.cuda.synchronize()
    want = out.clone()
    before = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == before
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and int(layer.status.item()) == 0


def alternating(which, graph, rounds=60):
    """Two different problems in turn on one workspace and the same input tensors, which a
    copy on the stream rewrites before every call: each result is that of the problem
    alone, so no kernel of a call reads what the call before it left."""
    serve = example()
    layer = serve.Layer(9, 400, 100, seed=6)   # (the slots of 5331 tokens)
    layer.plan([1500, 700, 64, 3, 130, 1, 900, 33, 2000])
    for b, n in enumerate((1500, 700, 64, 3, 130, 1, 900, 33, 2000)):
        layer.prefill(b, n)
    layer.summarise()
    base_table, base_lens = layer.table.clone(), layer.lens.clone()
    qs = [layer.tokens(8)[3] for _ in range(2)]
    ws = layer.bytes(max(_lib.eg_mla_decode_shared_workspace_size(layer.dims, 8, 2000),
                         _lib.eg_mla_decode_sparse_workspace_size(layer.dims, 8, 100, 6)))
    out = torch.zeros((8, 16, 128), dtype=torch.bfloat16, device="cuda")
    q, table, lens = torch.empty_like(qs[0]), base_table[:8].clone(), base_lens[:8].clone()
    prefix, plen = layer.ints(32), layer.ints(1)
    order = [torch.arange(8, device="cuda"), torch.tensor([7, 3, 5, 1, 6, 2, 4, 0], device="cuda")]
    inputs = [(qs[k], base_table[order[k]].contiguous(), base_lens[order[k]].contiguous(),
               base_table[8 if k else 1, :32].contiguous(), base_lens[8 if k else 1:][:1].contiguous()) for k in range(2)]

    def call(k):
        for dst, src in zip((q, table, lens, prefix, plen), inputs[k]):
            dst.copy_(src)
        if which == "shared":
            _lib.eg_mla_decode_shared(layer.dims, q, *layer.cache(), prefix, plen, 2000, table, lens, 2000, *layer.gate,
                                      layer.w_uk, layer.w_uv, out, ws, dev_status=layer.status)
        else:
            _lib.eg_mla_decode_sparse(layer.dims, q, *layer.cache(), table, lens, 2000, layer.summary, 6, 1, 1,
                                      *layer.gate, layer.w_uk, layer.w_uv, out, ws, dev_status=layer.status)

    want = []
    for k in range(2):
        ws.fill_(255)
        call(k)
        torch.cuda.synchronize()
        want.append(out.clone())
    got = [torch.empty_like(out) for _ in range(rounds)]

    def run():
        for i in range(rounds):
            call(i % 2)
            got[i].copy_(out)

    if graph:   # back to back, without the host's pace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for _ in range(5):
            g.replay()
    else:
        run()
    torch.cuda.synchronize()
    assert int(layer.status.item()) == 0
    assert not torch.equal(want[0], want[1])
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 2]), i


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("which", ["shared", "sparse"])
def test_calls_in_turn_on_one_workspace(gpu_lib, which, graph):
    alternating(which, graph)


@pytest.mark.parametrize("kw", [dict(document=30, sequences=3, steps=5), dict(document=1, sequences=1, steps=70, budget=2),
                                dict(document=130, sequences=2, steps=1, budget=64)])
def test_example_with_a_short_document(gpu_lib, kw):
    shared, sparse, all_free, status = example().main(**kw)
    assert shared <= 1e-2 and sparse == 0.0 and all_free and status == 0
