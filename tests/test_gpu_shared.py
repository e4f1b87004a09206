"""GPU parity of eg_mla_decode_shared (a decode step of sequences that share a
prefix) against the fp64 oracle, which sees every sequence as its own: the
prefix's tokens followed by its own.

Bound: the bf16 bound of the hot path, rel-L2 <= 5e-3 and max-abs <= 1e-2
max(1, |u|).  The path's roundings are those of eg_mla_decode: the prepared
queries, one rounding of the gated latent (here after its normalisation), the
softmax weights and the output."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import egmla_oracle as orc
from paper_2509_16686_gb300 import _lib, device, synth

pytestmark = pytest.mark.gpu


def check(got, ref, where=""):
    assert np.isfinite(got).all(), where
    worst = (np.abs(got - ref) / np.maximum(1.0, np.abs(ref))).max()
    rel = np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30)
    assert worst <= 1e-2 and rel <= 5e-3, f"{where}: max={worst:.3e} rel_l2={rel:.3e}"


def make(prefix, lens, d_c=256, gate_op="mul_ln", seed=3, dn=128, dv=128, vocab=700, change=None):
    """Sequence 0 of the case is the prefix, the others are the batch."""
    dims = synth.Dims(num_heads=16, d_nope=dn, d_rope=64, d_v=dv, d_c=d_c, page_size=64, vocab=vocab, dtype="bf16",
                      gate=gate_op != "none", gate_op=gate_op if gate_op != "none" else "mul_ln")
    case = synth.make_case("shared", dims, [prefix, *lens], seed=seed, latent_scale=0.5, layout="permuted",
                           affine_ln=True, extra_pages=3)
    if change is not None:
        change(case)
    return case


def reference(case):
    """The oracle on the same tokens as sequences of their own."""
    d, B = case.dims, case.batch - 1
    lens = [len(case.logical_ids[0]) + len(case.logical_ids[b + 1]) for b in range(B)]
    pages = max(1, max((n + 63) // 64 for n in lens))
    pools = [np.zeros((B * pages, 64, *a.shape[2:]), a.dtype) for a in (case.c_pool, case.kr_pool, case.id_pool)]
    rows = [p.reshape(B * pages * 64, *p.shape[2:]) for p in pools]
    for b, n in enumerate(lens):
        for row, logical in zip(rows, (case.logical_c, case.logical_kr, case.logical_ids)):
            row[b * pages * 64:b * pages * 64 + n] = np.concatenate([logical[0], logical[b + 1]])
    last = [max(n - 1, 0) + b * pages * 64 for b, n in enumerate(lens)]
    alone = dataclasses.replace(
        case, c_pool=pools[0], kr_pool=pools[1], id_pool=pools[2], seq_lens=np.array(lens, np.int32),
        block_table=np.arange(B * pages, dtype=np.int32).reshape(B, pages), q=case.q[1:], c_new=rows[0][last],
        kr_new=rows[1][last], ids_new=rows[2][last])
    return orc.decode_unabsorbed(alone)


class Shared:
    def __init__(self, case, splits=0, max_prefix=None):
        self.dc = dc = device.upload(case, num_splits=splits)
        dc.append()
        B = case.batch - 1
        self.prefix = int(case.seq_lens[0])
        self.max_prefix = self.prefix if max_prefix is None else max_prefix
        self.q = dc.q[1:].contiguous()
        self.table = dc.block_table[1:].contiguous()
        self.lens = dc.seq_lens[1:].contiguous()
        self.longest = int(case.seq_lens[1:].max())
        pages = (self.max_prefix + 63) // 64
        self.prefix_table = torch.full((max(pages, 1),), -1, dtype=torch.int32, device="cuda")
        here = min(pages, dc.block_table.shape[1])
        self.prefix_table[:here] = dc.block_table[0, :here]
        self.prefix_len = dc.seq_lens[:1].contiguous()
        self.out = torch.full((B, 16, case.dims.d_v), float("nan"), dtype=torch.bfloat16, device="cuda")
        n = _lib.eg_mla_decode_shared_workspace_size(dc.dims, B, self.max_prefix, splits)
        self.workspace = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # NaN in every format

    def run(self, stream=None):
        dc = self.dc
        _lib.eg_mla_decode_shared(dc.dims, self.q, dc.c_pool, dc.kr_pool, dc.id_pool, self.prefix_table,
                                  self.prefix_len, self.max_prefix, self.table, self.lens, self.longest,
                                  dc.gate_table, dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, self.out, self.workspace,
                                  dc.num_splits, dc.status, stream)
        torch.cuda.synchronize()
        return device.output_f64(self.out)


LENS = {1: (3,), 8: (1, 64, 65, 0, 7, 130, 2, 1), 9: (1, 1, 1, 1, 1, 1, 1, 1, 200), 17: (5, 0, 70) * 5 + (1, 128)}


@pytest.mark.parametrize("batch", sorted(LENS))
@pytest.mark.parametrize("prefix", [1, 63, 64, 65, 700])
@pytest.mark.parametrize("d_c", [192, 256])
def test_matches_the_sequences_alone(gpu_lib, d_c, prefix, batch):
    case = make(prefix, LENS[batch], d_c=d_c)
    s = Shared(case)
    got = s.run()
    assert s.dc.read_status() == 0
    check(got, reference(case))


@pytest.mark.parametrize("gate_op", ["none", "mul", "add_ln"])
@pytest.mark.parametrize("prefix", [64, 100, 385])
@pytest.mark.parametrize("d_c", [192, 256])
def test_every_gate_mode(gpu_lib, d_c, prefix, gate_op):
    case = make(prefix, (3, 0, 66), d_c=d_c, gate_op=gate_op)
    s = Shared(case)
    got = s.run()
    assert s.dc.read_status() == 0
    check(got, reference(case))


@pytest.mark.parametrize("gate_op", ["none", "mul_ln"])
def test_without_a_prefix_or_without_own_tokens(gpu_lib, gate_op):
    for prefix, lens, bound in ((0, (3, 0, 200), 0), (0, (3, 0, 200), 640), (300, (0, 0), 300), (0, (0, 0), 64)):
        case = make(prefix, lens, gate_op=gate_op)
        s = Shared(case, max_prefix=bound)
        got = s.run()
        assert s.dc.read_status() == 0
        check(got, reference(case), (prefix, lens))
        assert prefix or not got[[b for b, n in enumerate(lens) if n == 0]].any()


@pytest.mark.parametrize("splits", [1, 2, 7, 40])
def test_ranges_that_cross_row_tiles(gpu_lib, splits):
    """Few CTAs: their ranges of (row tile, page) units start and end inside row tiles."""
    case = make(900, (1, 20, 70) * 7)
    s = Shared(case, splits=splits, max_prefix=4000)
    got = s.run()
    assert s.dc.read_status() == 0
    check(got, reference(case))


@pytest.mark.parametrize("rising", [1.0, -1.0])
def test_maxima_that_move_from_page_to_page(gpu_lib, rising):
    """Scores that rise (fall) by more than the reference's slack with every page."""
    def change(case):
        e = np.full(64, 0.125, np.float32)
        kr = synth.bf16_bits_to_f32(case.logical_kr[0])
        n = len(kr)
        page = np.arange(n) // 64 if rising > 0 else (n - 1) // 64 - np.arange(n) // 64
        kr = synth.f32_to_bf16_bits(kr + 2.0 * page[:, None].astype(np.float32) * e)
        case.logical_kr[0][:] = kr
        for j in range(n - 1):
            case.kr_pool[case.block_table[0, j // 64], j % 64] = kr[j]
        case.kr_new[0] = kr[n - 1]
        q = synth.bf16_bits_to_f32(case.q)
        q[..., -64:] += 40.0 * e
        case.q[:] = synth.f32_to_bf16_bits(q)

    case = make(600, (2, 70, 1), change=change)
    for splits in (0, 1):
        s = Shared(case, splits=splits)
        got = s.run()
        assert s.dc.read_status() == 0
        check(got, reference(case), splits)


def test_other_head_dims(gpu_lib):
    case = make(333, (4, 90), dn=64, dv=72)
    s = Shared(case)
    got = s.run()
    assert s.dc.read_status() == 0
    check(got, reference(case))


def test_agrees_with_decode_over_a_joint_block_table(gpu_lib):
    """Whole prefix pages in front of every sequence's own in one block table: the
    same tokens for eg_mla_decode.  Both are within the bound of the exact result."""
    case = make(640, (5, 64, 100, 1) * 8)
    s = Shared(case)
    got = s.run()
    dc = s.dc
    table = torch.cat([s.prefix_table.expand(s.table.shape[0], -1), s.table], 1).contiguous()
    lens = s.lens + 640
    ws = torch.empty(_lib.eg_mla_decode_workspace_size(dc.dims, len(lens)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(s.out)
    _lib.eg_mla_decode(dc.dims, s.q, dc.c_pool, dc.kr_pool, dc.id_pool, table, lens, 640 + s.longest, dc.gate_table,
                       dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, out, ws, 0, dc.status)
    joint = device.output_f64(out)
    assert dc.read_status() == 0
    assert (np.abs(got - joint) <= 2e-2 * np.maximum(1.0, np.abs(joint))).all()
    assert np.linalg.norm(got - joint) <= 1e-2 * np.linalg.norm(joint)


def test_repeated_calls_and_another_stream_give_the_same_bits(gpu_lib):
    case = make(2000, (1, 20, 70) * 6)
    s = Shared(case)
    s.run()
    first = s.out.clone()
    stream = torch.cuda.Stream()
    for _ in range(3):
        s.out.fill_(float("nan"))
        torch.cuda.synchronize()
        s.run(stream)
        assert torch.equal(first.view(torch.int16), s.out.view(torch.int16))


def test_graph_replay_with_a_longer_prefix(gpu_lib):
    """Lengths are read on the device: a captured step serves a prefix that has grown."""
    case = make(500, (3, 80))
    s = Shared(case)
    s.prefix_len.fill_(130)
    s.run()
    graph = torch.cuda.CUDAGraph()
    dc = s.dc
    with torch.cuda.graph(graph):
        _lib.eg_mla_decode_shared(dc.dims, s.q, dc.c_pool, dc.kr_pool, dc.id_pool, s.prefix_table, s.prefix_len,
                                  s.max_prefix, s.table, s.lens, s.longest, dc.gate_table, dc.ln_gamma, dc.ln_beta,
                                  dc.w_uk, dc.w_uv, s.out, s.workspace, 0, dc.status)
    s.prefix_len.fill_(500)
    graph.replay()
    torch.cuda.synchronize()
    assert dc.read_status() == 0
    check(device.output_f64(s.out), reference(case))


@pytest.mark.parametrize("gate_op", ["none", "mul_ln"])
def test_bad_pages_ids_and_lengths_are_reported(gpu_lib, gate_op):
    for bad in ("page", "negative page", "length", "negative length", "id"):
        if bad == "id" and gate_op == "none":
            continue
        s = Shared(make(200, (3, 80), gate_op=gate_op))
        if bad == "page":
            s.prefix_table[1] = s.dc.c_pool.shape[0]
        elif bad == "negative page":
            s.prefix_table[3] = -5
        elif bad == "length":
            s.prefix_len.fill_(201)
        elif bad == "negative length":
            s.prefix_len.fill_(-1)
        else:
            s.dc.id_pool[int(s.prefix_table[1]), 5] = s.dc.dims.vocab
        s.run()
        assert s.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE, bad


@pytest.mark.parametrize("gate_op", ["none", "mul", "mul_ln"])
@pytest.mark.parametrize("d_c", [192, 256])
@pytest.mark.parametrize("prefix,splits", [(385, 0), (256, 3), (640, 4), (900, 0)])
def test_short_ranges_repeat_bit_for_bit(gpu_lib, prefix, splits, d_c, gate_op):
    """Ranges of a few pages, where a warp may be two pages ahead of another at a range's
    end: the same bits forty times."""
    case = make(prefix, (3, 0, 66), d_c=d_c, gate_op=gate_op)
    s = Shared(case, splits=splits)
    first = s.run()
    check(first, reference(case))
    for _ in range(40):
        assert np.array_equal(s.run(), first)
    assert s.dc.read_status() == 0


@pytest.mark.parametrize("gate_op", ["mul_ln", "add_ln", "mul", "none"])
@pytest.mark.parametrize("power", [10, 40, -10, -40])
def test_softmax_scales_and_queries_of_any_size(gpu_lib, power, gate_op):
    """A softmax scale 2^power times the usual one with queries 2^-power times theirs: every
    score stays as it is, and so does every bit of the result."""
    def scaled(by):
        def change(case):
            case.dims.softmax_scale = float(np.float32(192 ** -0.5)) * 2.0 ** by
            case.q[:] = synth.f32_to_bf16_bits(synth.bf16_bits_to_f32(case.q) * np.float32(2.0 ** -by))
        return make(300, (2, 70, 1), gate_op=gate_op, change=change)

    case = scaled(power)
    s, usual = Shared(case), Shared(scaled(0))
    got, want = s.run(), usual.run()
    assert s.dc.read_status() == 0
    check(got, reference(case))
    assert np.array_equal(got, want)


@pytest.mark.parametrize("gate_op", ["none", "mul_ln"])
@pytest.mark.parametrize("length", [1, -1, 2 ** 31 - 1])
def test_a_prefix_where_the_bound_is_zero_is_reported(gpu_lib, length, gate_op):
    case = make(0, (3, 0, 200), gate_op=gate_op)
    s = Shared(case, max_prefix=0)
    s.prefix_len.fill_(length)
    got = s.run()
    assert s.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE
    check(got, reference(case))   # taken as 0


def exact(case, q, prefix, table, lens):
    """The definition in 64 bits from the cached rows: `prefix` rows of the cache, then
    each sequence's own."""
    d = case.dims
    c, kr, ids = orc.appended_pools(case)
    rows = [torch.from_numpy(orc.widen(a, "bf16").reshape(-1, a.shape[-1])).cuda() for a in (c, kr)]
    if d.gate:
        g = torch.from_numpy(orc.widen(case.gate_table, "bf16")).cuda()[torch.from_numpy(ids.reshape(-1)).long().cuda().clamp(0, d.vocab - 1)]
        x = rows[0] + g if d.gate_op == "add_ln" else rows[0] * g
        if d.gate_op != "mul":
            x = x - x.mean(-1, keepdim=True)
            x = x / (x.square().mean(-1, keepdim=True) + d.ln_eps).sqrt()
            x = x * torch.from_numpy(case.ln_gamma).cuda().double() + torch.from_numpy(case.ln_beta).cuda().double()
        rows[0] = x
    w_uk, w_uv = (torch.from_numpy(orc.widen(w, "bf16")).cuda() for w in (case.w_uk, case.w_uv))
    q = q.double()
    qa = torch.cat([torch.einsum("bhd,hdc->bhc", q[..., :d.d_nope], w_uk), q[..., d.d_nope:]], -1)
    out = []
    for b, n in enumerate(lens):
        at = torch.cat([prefix, table[b, torch.arange(n) // 64].long().cpu() * 64 + torch.arange(n) % 64]).cuda()
        z = rows[0][at]
        p = (qa[b] @ torch.cat([z, rows[1][at]], -1).T * orc.softmax_scale(d)).softmax(-1)
        out.append(torch.einsum("hc,hdc->hd", p @ z, w_uv))
    return torch.stack(out).cpu().numpy()


@pytest.mark.parametrize("d_c,gate_op", [(192, "none"), (256, "mul_ln"), (256, "mul")])
@pytest.mark.parametrize("batch,prefix,splits", [(3, 600 * 64 - 17, 0), (3, 600 * 64, 400), (1, 300 * 64 + 1, 200),
                                                 (70, 310 * 64 - 1, 0), (70, 100 * 64 + 5, 1000)])
def test_long_prefixes_and_many_partials(gpu_lib, batch, prefix, splits, d_c, gate_op):
    """Prefixes of hundreds of pages (a few physical ones, many times), up to 300 partials
    of a sequence."""
    case = make(15 * 64, (100,) * 2, d_c=d_c, gate_op=gate_op)
    r = np.random.default_rng(prefix + batch)
    s = Shared(case)
    dc = s.dc
    pages = (prefix + 63) // 64
    held = s.prefix_table.cpu()
    prefix_table = held[torch.from_numpy(r.integers(0, 15, pages))]
    lens = [int(x) for x in r.integers(0, 130, batch)]
    table = held[torch.from_numpy(r.integers(0, 15, (batch, 3)))]
    gen = torch.Generator(device="cuda").manual_seed(batch)
    q = torch.randn((batch, 16, 192), generator=gen, device="cuda").bfloat16()
    out = torch.full((batch, 16, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((_lib.eg_mla_decode_shared_workspace_size(dc.dims, batch, prefix, splits),), 255,
                    dtype=torch.uint8, device="cuda")
    n = torch.tensor([prefix], dtype=torch.int32, device="cuda")
    _lib.eg_mla_decode_shared(dc.dims, q, dc.c_pool, dc.kr_pool, dc.id_pool, prefix_table.cuda(), n, prefix,
                              table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), 192, dc.gate_table,
                              dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, out, ws, splits, dc.status)
    torch.cuda.synchronize()
    assert dc.read_status() == 0
    at = torch.arange(prefix)
    check(device.output_f64(out), exact(case, q, prefix_table[at // 64].long() * 64 + at % 64, table, lens))


@pytest.mark.parametrize("gate_op", ["none", "mul_ln"])
def test_pages_past_32_bits_of_a_pool(gpu_lib, gate_op):
    """Pages whose elements and bytes lie past 2^31 and 2^32 in the latent pool: the same bits."""
    s = Shared(make(333, (4, 90, 0), gate_op=gate_op))
    dc = s.dc
    want, n = s.run(), dc.c_pool.shape[0]
    shift = 2 ** 31 // (64 * 256) + 1
    for pool in ("c_pool", "kr_pool", "id_pool"):
        small = getattr(dc, pool)
        big = torch.zeros((shift + n, *small.shape[1:]), dtype=small.dtype, device="cuda")
        big[shift:] = small
        setattr(dc, pool, big)
    s.prefix_table, s.table = s.prefix_table + shift, s.table + shift
    s.out.fill_(float("nan"))
    assert np.array_equal(s.run(), want)
    assert dc.read_status() == 0
