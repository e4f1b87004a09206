"""The packed-token calls and every form of the decode in 8 bits on streams, in threads, captured and replayed: each
problem against the same problem alone, with inputs, lengths and shapes that differ from one to the other."""
import threading

import pytest
import torch

from paper_2509_16686_gb300 import _lib
from tests.test_gpu_tokens import Cache, append_case, decode_q8, ints, make, normal, offsets, quantised, status_word

pytestmark = pytest.mark.gpu

DECODES = [(256, "mul_ln"), (256, "add_ln"), (192, "mul_ln"), (192, "none"), (256, "none"), (512, "none")]
CALLS = ["rope", "append", "read", *DECODES]
# (few sequences end in the decode kernel's own combine at d_c up to 256, many in a kernel of its own)
LENS = [[700, 64, 3, 300], [40, 0, 2000, 129, 64, 5], [65] * 12, [1, 1500]]


class Problem:
    """One call on tensors of its own: run(stream), its output, and the output of a run alone."""

    def __init__(self, what, seed):
        self.status, lens = status_word(), LENS[seed % len(LENS)]
        if isinstance(what, tuple):
            d_c, gate = what
            _, dc = make(lens, d_c, gate, seed=seed)
            cache, _ = quantised(dc)
            dc.status = self.status
            self.out = torch.zeros_like(dc.out)
            self.run = lambda stream=None, workspace=None: decode_q8(dc, cache, self.out, stream, workspace)
            self.dc = dc
        else:
            firsts = [seed, 60, 0, 130, 7, 64, 1, 2, 3, 4, 5, 6][:len(lens)]
            dims, c, kr, ids, table, _, cache = append_case(lens, firsts, 256, "bf16", seed=seed)
            cu, pos, tab = ints(offsets(lens)), ints(firsts), ints(table)
            if what == "rope":
                q, rope = normal((sum(lens), 16, 192), "bf16", seed), _lib.make_rope()
                self.out = torch.zeros_like(q)
                self.run = lambda stream=None: _lib.eg_mla_rope(dims, rope, q, self.out, None, None, pos, cu, self.status, stream)
            elif what == "append":
                self.out = cache.c8
                self.run = lambda stream=None: _lib.eg_mla_append_latent_q8(dims, *cache.all(), c, kr, ids, tab, pos, cu,
                                                                            self.status, stream)
            else:
                _lib.eg_mla_append_latent_q8(dims, *cache.all(), c, kr, ids, tab, pos, cu)
                self.out = torch.zeros_like(c)
                self.run = lambda stream=None: _lib.eg_mla_read_latent_q8(dims, *cache.all(), tab, self.out, None, None, pos, cu,
                                                                          self.status, stream)
        self.clear()
        self.run()
        self.want = self.out.clone()
        torch.cuda.synchronize()

    def clear(self):
        self.out.fill_(0x33)

    def good(self, out=None):
        return torch.equal(self.out if out is None else out, self.want) and int(self.status) == 0


@pytest.mark.parametrize("what", CALLS)
def test_repeated_calls_give_the_same_bits(gpu_lib, what):
    for seed in range(4):
        p = Problem(what, seed)
        for _ in range(10):
            p.clear()
            p.run()
            assert p.good(), seed


@pytest.mark.parametrize("what", CALLS)
def test_a_stream_that_is_not_the_current_one(gpu_lib, what):
    stream = torch.cuda.Stream()
    for seed in range(2):
        p = Problem(what, seed)
        p.clear()
        torch.cuda.synchronize()
        p.run(stream)
        stream.synchronize()
        assert p.good()


@pytest.mark.parametrize("what", CALLS)
def test_threads_with_problems_of_their_own(gpu_lib, what):
    """Two threads on streams of their own, every one of twenty outputs against the problem alone."""
    problems, outs = [Problem(what, seed) for seed in range(2)], [[], []]
    assert problems[0].want.shape != problems[1].want.shape or not torch.equal(problems[0].want, problems[1].want)
    failures = []

    def work(k):
        try:
            torch.cuda.set_device(0)
            p, stream = problems[k], torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    p.clear()
                    p.run()
                    outs[k].append(p.out.clone())
            stream.synchronize()
        except Exception as e:   # (of a thread: for the assertion below)
            failures.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures
    for p, o in zip(problems, outs):
        assert len(o) == 20 and all(p.good(x) for x in o)


@pytest.mark.parametrize("what", CALLS)
def test_captured_and_replayed(gpu_lib, what):
    p = Problem(what, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for _ in range(3):
        p.clear()
        graph.replay()
        assert p.good()


@pytest.mark.parametrize("what", DECODES)
def test_two_captured_decodes_share_a_workspace(gpu_lib, what):
    """Replayed in turn on one stream, with no wait in between."""
    a, b = Problem(what, 0), Problem(what, 1)
    shared = max((a.dc.workspace, b.dc.workspace), key=lambda t: t.numel())
    graphs = []
    for p in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.run(workspace=shared)
        graphs.append(g)
    outs = []
    for _ in range(10):
        for p, g in zip((a, b), graphs):
            p.clear()
            g.replay()
            outs.append((p, p.out.clone()))
    assert all(p.good(x) for p, x in outs)


@pytest.mark.parametrize("what", DECODES)
def test_a_captured_decode_follows_its_inputs(gpu_lib, what):
    """Lengths, block table and queries that change in place between replays, up to the length that was captured."""
    p = Problem(what, 0)
    dc = p.dc
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    first = dc.seq_lens.clone()
    for lens in ([1, 64, 0, 65], [0, 0, 0, 0], [699, 1, 3, 300], first.tolist()):
        dc.seq_lens.copy_(ints(lens))
        dc.q.mul_(-1)
        p.clear()
        p.run()
        p.want = p.out.clone()
        p.clear()
        graph.replay()
        assert p.good(), lens


def test_a_step_captured_whole(gpu_lib):
    """Rope, append and decode of one graph, ungated, replayed over new tokens: the decode reads what the append of the
    same replay wrote."""
    d_c, B, steps = 512, 5, 6
    dims = _lib.make_dims(16, 128, 64, 128, d_c, 100, gate=False)
    w = [normal((16, 128, d_c), "bf16", 3 + i, d_c ** -0.5) for i in range(2)]
    table = ints([[B * j + i for j in range(3)] for i in range(B)])
    firsts = [0, 63, 100, 5, 126]
    rope = _lib.make_rope(layout="half")
    tokens = [dict(q=normal((B, 16, 192), "bf16", 10 * s), k=normal((B, 64), "bf16", 10 * s + 1),
                   c=normal((B, d_c), "bf16", 10 * s + 2, 0.5)) for s in range(steps)]
    ws = torch.empty(_lib.eg_mla_decode_workspace_size(dims, B), dtype=torch.uint8, device="cuda")

    def fresh():
        cache = Cache(3 * B, d_c, "bf16", ids=False)
        past = ints(offsets(firsts))
        _lib.eg_mla_append_latent_q8(dims, *cache.all(), normal((sum(firsts), d_c), "bf16", 1, 0.5),
                                     normal((sum(firsts), 64), "bf16", 2), None, table, None, past)
        return cache

    def step(cache, now, pos, lens, out, status):
        _lib.eg_mla_rope(dims, rope, now["q"], now["q"], now["k"], now["k"], pos, None, status)
        _lib.eg_mla_append_latent_q8(dims, *cache.all(), now["c"], now["k"], None, table, pos, None, status)
        _lib.eg_mla_decode_q8(dims, now["q"], *cache.all(), table, lens, 192, None, None, None, *w, out, ws, 0, status)

    results = []
    for captured in (False, True):
        cache, status = fresh(), status_word()
        pos, lens = ints(firsts), ints(firsts) + 1
        now = {n: torch.empty_like(t) for n, t in tokens[0].items()}
        out = torch.empty((B, 16, 128), dtype=torch.bfloat16, device="cuda")
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(cache, now, pos, lens, out, status)
        outs = []
        for t in tokens:
            for n in now:
                now[n].copy_(t[n])
            if captured:
                graph.replay()
            else:
                step(cache, now, pos, lens, out, status)
            outs.append(out.clone())
            pos += 1
            lens += 1
        assert int(status) == 0
        results.append((outs, cache))
    (a, ca), (b, cb) = results
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and not torch.equal(a[0], a[1])
    assert torch.equal(ca.c8, cb.c8) and torch.equal(ca.scale, cb.scale) and torch.equal(ca.kr, cb.kr)
