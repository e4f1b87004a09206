"""GPU parity of the page calls.

eg_mla_page_plan is whole numbers: every output equals a plain loop's over the
requests, word for word.

eg_mla_page_summary is fp32 against fp64: worst-case bound from its operations
(see summary_bound).

eg_mla_decode_sparse: the selection's scores are fp32 sums, so a page may stand in
for another only if their exact scores are within those sums' error bound; given
the selection, the result is bit for bit eg_mla_decode's over the selected block
table, and within the hot path's bounds of the oracle."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import egmla_oracle as orc
from paper_2509_16686_gb300 import _lib, device, synth

pytestmark = pytest.mark.gpu
P = 64


# ------------------------------------------------------------------ plan
def pages_of(n):
    return (n + P - 1) // P


def plan_reference(new, lens, table, stack, free, max_slots):
    """The definition, request by request."""
    table, stack, num_pages = table.copy(), stack.copy(), len(stack)
    width = table.shape[1]
    status = 0
    if not 0 <= free <= num_pages:
        free, status = 0, _lib.EG_MLA_ERR_OUT_OF_RANGE
    avail = free
    sane = [0 <= L <= width * P for L in lens]
    if not all(sane):
        status = _lib.EG_MLA_ERR_OUT_OF_RANGE
    for b, n in enumerate(new):
        if n < 0 and sane[b]:
            for page in table[b, :pages_of(lens[b])]:
                if avail < num_pages:
                    stack[avail] = page
                    avail += 1
    asked, cu, positions, lens_out, slots = 0, [0], [], [], []
    left = avail
    for b, n in enumerate(new):
        L, t = lens[b], 0
        if sane[b] and n > 0 and L + n <= width * P:
            need = pages_of(L + n) - pages_of(L)
            if need == 0 or asked + need <= avail:
                t = n
                for i in range(need):
                    left -= 1
                    table[b, pages_of(L) + i] = stack[left]
            asked += need
        if sane[b] and n > 0 and t == 0 and status == 0:
            status = _lib.EG_MLA_ERR_NO_PAGES
        lens_out.append(0 if sane[b] and n < 0 else L + t)
        positions.append(L if t > 0 else -1)
        cu.append(cu[-1] + t)
        for pos in range(L, L + t):
            page = table[b, pos // P]
            slots.append(page * P + pos % P if 0 <= page < num_pages else -1)
    slots = slots[:max_slots] + [-1] * (max_slots - len(slots))
    return dict(seq_lens=lens_out, table=table, stack=stack, free=[left], cu=cu, positions=positions,
                slots=slots), status


def dev(x):
    return torch.tensor(np.asarray(x, np.int32), dtype=torch.int32, device="cuda")


def run_plan(new, lens, table, stack, free, max_slots, in_place=False, stream=None):
    B = len(new)
    d = dict(new=dev(new), lens=dev(lens), table=dev(table).view(B, -1) if B else torch.zeros((0, 4), dtype=torch.int32, device="cuda"),
             stack=dev(stack), free=dev([free]), cu=dev([-9] * (B + 1)), positions=dev([-9] * B),
             slots=dev([-9] * max_slots) if max_slots else None, status=dev([0]))
    lens_out = d["lens"] if in_place else dev([-9] * B)
    free_out = d["free"] if in_place else dev([-9])
    torch.cuda.synchronize()
    _lib.eg_mla_page_plan(d["new"], d["lens"], lens_out, d["table"], d["stack"], d["free"], free_out, d["cu"],
                          d["positions"], d["slots"], dev_status=d["status"], stream=stream)
    torch.cuda.synchronize()
    got = dict(seq_lens=lens_out, table=d["table"], stack=d["stack"], free=free_out, cu=d["cu"],
               positions=d["positions"], slots=d["slots"])
    return {k: v.cpu().numpy() if v is not None else np.zeros(0, np.int32) for k, v in got.items()}, \
        int(d["status"].item())


def plan_case(seed, batch, longest, prompts=0.2, leaving=0.2, spare=0, width=None):
    """`spare`: free pages beyond what the requests need (negative: too few)."""
    r = np.random.default_rng(seed)
    lens = r.integers(0, longest + 1, batch)
    kind = r.random(batch)
    new = np.where(kind < prompts, r.integers(1, longest + 1, batch), np.where(kind < prompts + leaving, -1,
                                                                              r.integers(0, 3, batch)))
    width = width or max(1, int(pages_of(lens + np.maximum(new, 0)).max()) if batch else 1)
    lens = np.minimum(lens, width * P)
    have = pages_of(lens)
    need = int((pages_of(lens + np.maximum(new, 0)) - have).sum())
    free = max(0, need + spare)
    ids = r.permutation(int(have.sum()) + free + 7)
    table = np.full((batch, width), 123456789, np.int64)
    k = 0
    for b in range(batch):
        table[b, :have[b]] = ids[k:k + have[b]]
        k += have[b]
    stack = np.full(len(ids), 77, np.int64)
    stack[:free] = ids[k:k + free]
    return [int(x) for x in new], [int(x) for x in lens], table, stack, free


def assert_plan(got, want):
    for k, v in want.items():
        assert np.array_equal(got[k], np.asarray(v).reshape(got[k].shape)), k


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("spare", [50, 0, -3, -1000])
@pytest.mark.parametrize("batch,longest", [(1, 1), (1, 300), (3, 64), (33, 129), (512, 90), (513, 500), (1500, 70),
                                           (40, 5000)])
def test_plan_matches_the_loop(gpu_lib, batch, longest, spare, in_place):
    case = plan_case(batch + longest, batch, longest, spare=spare)
    slots = sum(max(n, 0) for n in case[0]) + 5
    want, status = plan_reference(*case, slots)
    got, st = run_plan(*case, slots, in_place=in_place)
    assert_plan(got, want)
    assert st == status


def test_plan_of_the_largest_batch_and_of_none(gpu_lib):
    case = plan_case(5, 16384, 100)
    slots = sum(max(n, 0) for n in case[0])
    want, status = plan_reference(*case, slots)
    got, st = run_plan(*case, slots)
    assert_plan(got, want)
    assert st == status
    got, st = run_plan([], [], np.zeros((0, 4)), [3, 2, 1], 2, 9)
    assert st == 0 and got["cu"].tolist() == [0] and got["free"].tolist() == [2] and got["slots"].tolist() == [-1] * 9


def test_plan_without_optional_outputs(gpu_lib):
    case = plan_case(8, 20, 200)
    want, _ = plan_reference(*case, 0)
    new, lens, table, stack, free = case
    t = [dev(new), dev(lens), dev(lens), dev(table), dev(stack), dev([free]), dev([0]), dev([0] * 21)]
    _lib.eg_mla_page_plan(*t)
    torch.cuda.synchronize()
    assert t[2].tolist() == want["seq_lens"] and t[7].tolist() == want["cu"]
    assert np.array_equal(t[3].cpu().numpy(), want["table"])


def test_plan_refuses_what_a_row_cannot_hold_and_serves_the_others(gpu_lib):
    # width 2: 128 tokens a row
    new, lens = [100, 1, 29, 1, 64], [100, 128, 99, 64, 64]
    table = np.array([[1, 2], [3, 4], [5, 6], [7, 0], [8, 0]])
    stack = np.array([10, 11, 12, 13] + [0] * 20)
    want, status = plan_reference(new, lens, table, stack, 4, 200)
    got, st = run_plan(new, lens, table, stack, 4, 200)
    assert_plan(got, want)
    assert st == status == _lib.EG_MLA_ERR_NO_PAGES
    assert got["cu"].tolist() == [0, 0, 0, 29, 30, 94]


def test_plan_reports_what_it_cannot_use(gpu_lib):
    bad = _lib.EG_MLA_ERR_OUT_OF_RANGE
    table = np.array([[1, 2], [3, 4]])
    stack = np.array([5, 6, 0, 0, 0, 0, 0, 0])

    def case(new=(1, 1), lens=(64, 65), table=table, stack=stack, free=2, slots=4):
        want, status = plan_reference(list(new), list(lens), table, stack, free, slots)
        got, st = run_plan(list(new), list(lens), table, stack, free, slots)
        assert_plan(got, want)
        return got, st, status

    assert case()[1] == 0
    for lens in ((-1, 65), (64, 129), (2 ** 31 - 1, 1), (-2 ** 31, 1)):   # lengths
        for new in ((1, 1), (-1, -1), (2 ** 31 - 1, -2 ** 31)):
            got, st, status = case(new=new, lens=lens)
            assert st == bad and status == bad
    for free in (-1, 9, 2 ** 31 - 1):                                     # the stack's height
        assert case(free=free)[1] == bad
    got, st, _ = case(stack=np.array([5, 99, 0, 0, 0, 0, 0, 0]))          # a page on the stack
    assert st == bad and -1 in got["slots"]
    got, st, _ = case(table=np.array([[1, 2], [3, -4]]))                  # a page in a row
    assert st == bad and got["slots"].tolist()[1] == -1
    assert case(new=(3, 3), slots=4)[1] == bad                            # too few slots
    # more pages back than the stack holds
    got, st, _ = case(new=(-1, -1), lens=(128, 128), stack=np.arange(5, 10), free=3)
    assert st == bad and got["free"].tolist() == [5]


def test_plan_gives_the_same_on_another_stream_and_in_a_graph(gpu_lib):
    case = plan_case(21, 700, 900, spare=-20)
    slots = sum(max(n, 0) for n in case[0])
    want, _ = plan_reference(*case, slots)
    for _ in range(3):
        got, _ = run_plan(*case, slots, stream=torch.cuda.Stream())
        assert_plan(got, want)


def test_plan_feeds_append_and_decode(gpu_lib):
    """A few steps of a serving loop whose tables all come from the plan, against the
    oracle on the sequences' own tokens."""
    dims = synth.dims_bf16(d_c=256, vocab=500)
    r = np.random.default_rng(4)
    src = synth.make_case("src", dims, [200, 130, 70], seed=8, latent_scale=0.5, affine_ln=True)
    B, num_pages = 3, 9
    d = device.upload(src)
    c_pool = torch.zeros((num_pages, P, 256), dtype=torch.bfloat16, device="cuda")
    kr_pool = torch.zeros((num_pages, P, 64), dtype=torch.bfloat16, device="cuda")
    id_pool = torch.zeros((num_pages, P), dtype=torch.int32, device="cuda")
    lens, table = dev([0] * B), torch.full((B, 4), -1, dtype=torch.int32, device="cuda")
    stack, free, cu, pos, status = dev(r.permutation(num_pages)), dev([num_pages]), dev([0] * 4), dev([0] * 3), dev([0])
    slots = dev([0] * 400)

    def logical(a, b, n):
        return device.to_device_array(np.ascontiguousarray(a[b][n]), "bf16", "cuda")

    start = [100, 129, 3]
    _lib.eg_mla_page_plan(dev(start), lens, lens, table, stack, free, free, cu, pos, slots, dev_status=status)
    rows = slots[:sum(start)].long()
    for pool, a in ((c_pool, src.logical_c), (kr_pool, src.logical_kr), (id_pool, src.logical_ids)):
        packed = torch.cat([logical(a, b, slice(0, n)) for b, n in enumerate(start)])
        pool.view(num_pages * P, *pool.shape[2:])[rows] = packed
    at = list(start)
    for step in range(40):
        grow = [1, 1 if step == 0 else 0, 1]
        _lib.eg_mla_page_plan(dev(grow), lens, lens, table, stack, free, free, cu, pos, slots[:8], dev_status=status)
        n = [min(x, len(src.logical_ids[b]) - 1) for b, x in enumerate(at)]
        _lib.eg_mla_append_latent(d.dims, c_pool, kr_pool, id_pool,
                                  torch.stack([logical(src.logical_c, b, n[b]) for b in range(B)]),
                                  torch.stack([logical(src.logical_kr, b, n[b]) for b in range(B)]),
                                  dev([src.logical_ids[b][n[b]] for b in range(B)]), table, pos, status)
        at = [x + g for x, g in zip(at, grow)]
    assert lens.tolist() == at and int(status.item()) == 0
    _lib.eg_mla_decode(d.dims, d.q, c_pool, kr_pool, id_pool, table, lens, 256, d.gate_table, d.ln_gamma, d.ln_beta,
                       d.w_uk, d.w_uv, d.out, d.workspace, 0, status)
    got = device.output_f64(d.out)
    case = dataclasses.replace(src, seq_lens=np.array(at, np.int32),
                               c_new=np.stack([src.logical_c[b][n - 1] for b, n in enumerate(at)]),
                               kr_new=np.stack([src.logical_kr[b][n - 1] for b, n in enumerate(at)]),
                               ids_new=np.array([src.logical_ids[b][n - 1] for b, n in enumerate(at)], np.int32))
    ref = orc.decode_unabsorbed(case)
    assert int(status.item()) == 0
    assert (np.abs(got - ref) <= 1e-2 * np.maximum(1, np.abs(ref))).all()
    assert np.linalg.norm(got - ref) <= 5e-3 * np.linalg.norm(ref)


# --------------------------------------------------------------- summaries
SHAPES = {
    "gate256": dict(dims=synth.dims_bf16(d_c=256, vocab=700)),
    "gate192": dict(dims=synth.dims_bf16(d_c=192, vocab=700)),
    "mul": dict(dims=synth.dims_bf16(d_c=256, vocab=700, gate_op="mul")),
    "add_ln": dict(dims=synth.dims_bf16(d_c=192, vocab=700, gate_op="add_ln")),
    "none512": dict(dims=synth.dims_bf16(d_c=512, vocab=700, gate=False)),
    "fp32_64": dict(dims=dataclasses.replace(synth.dims_tiny())),
    "fp32_132": dict(dims=synth.Dims(5, 24, 12, 40, 132, 64, 300, "fp32")),
    "fp32_512": dict(dims=synth.Dims(16, 64, 64, 64, 512, 64, 300, "fp32")),
    "fp32_none": dict(dims=synth.Dims(3, 32, 16, 32, 256, 64, 300, "fp32", gate=False)),
}


def make(name, lens, seed=17):
    dims = SHAPES[name]["dims"]
    return synth.make_case(name, dims, list(lens), seed=seed, latent_scale=0.5 if dims.dtype == "bf16" else 1.0,
                           layout="permuted", affine_ln=True, extra_pages=3)


def keys64(case, page):
    """[c~ ; k^R] of a page's rows in 64 bits, and c (gated, before the LayerNorm)."""
    d = case.dims
    c_pool, kr_pool, id_pool = orc.appended_pools(case)
    c, kr = orc.widen(c_pool[page], d.dtype), orc.widen(kr_pool[page], d.dtype)
    if not d.gate:
        return np.concatenate([c, kr], 1), c
    g = orc.widen(case.gate_table, d.dtype)[id_pool[page]]
    z = orc.gate_latents(c, g, case.ln_gamma.astype(np.float64), case.ln_beta.astype(np.float64), d.ln_eps, d.gate_op)
    return np.concatenate([z, kr], 1), (c + g if d.gate_op == "add_ln" else c * g)


def summary_bound(case, keys, x):
    """Worst case of the fp32 operations.  The row sums of the mean and variance err by
    at most d_c 2^-24 of their terms' magnitudes, so an element x - mu by d_c 2^-24 max|x|
    and 1/sigma by a relative d_c 2^-24 (with rsqrt and the roundings: d_c + 16);
    the sum over 64 rows by 64 2^-24 of its terms' magnitudes."""
    d, u = case.dims, 2.0 ** -24
    if d.gate and d.gate_op != "mul":
        ratio = (np.abs(x).max(1) / x.std(1)).max()
        top = np.abs(case.ln_gamma).max() * (np.abs(x - x.mean(1, keepdims=True)).max(1) / x.std(1)).max()
        lat = u * ((2 * d.d_c + 96) * (ratio * np.abs(case.ln_gamma).max() + top) + 4 * np.abs(case.ln_beta).max())
    else:
        lat = 80 * u * np.abs(x).max()
    rope = 80 * u * np.abs(keys[:, d.d_c:]).max()
    return np.concatenate([np.full(d.d_c, lat), np.full(d.d_rope, rope)])


class Pages:
    def __init__(self, case):
        self.case, self.dc = case, device.upload(case)
        self.dc.append()
        d = case.dims
        self.summary = torch.full((case.num_pages, d.d_c + d.d_rope), -77.0, device="cuda")
        self.longest = int(case.seq_lens.max())

    def summarise(self, new=None, max_new=0, lens=None, longest=None):
        dc = self.dc
        _lib.eg_mla_page_summary(dc.dims, dc.c_pool, dc.kr_pool, dc.id_pool, dc.block_table,
                                 dc.seq_lens if lens is None else lens, self.longest if longest is None else longest,
                                 dc.gate_table, dc.ln_gamma, dc.ln_beta, self.summary, new, max_new, dc.status)
        torch.cuda.synchronize()
        return self.summary.cpu().numpy().astype(np.float64)


def check_summary(p, got, new):
    case = p.case
    done = set()
    for b, L in enumerate(case.seq_lens):
        n = int(L) if new is None else min(max(int(new[b]), 0), int(L))
        for lp in range((int(L) - n) // P, int(L) // P):
            page = int(case.block_table[b, lp])
            keys, x = keys64(case, page)
            err = np.abs(got[page] - keys.mean(0))
            bound = summary_bound(case, keys, x)
            assert (err <= bound).all(), (b, lp, (err / bound).max())
            done.add(page)
    for page in range(case.num_pages):
        if page not in done:
            assert (got[page] == -77.0).all(), page
    return done


@pytest.mark.parametrize("name", sorted(SHAPES))
def test_summaries_of_all_full_pages(gpu_lib, name):
    p = Pages(make(name, (0, 1, 63, 64, 65, 200, 320)))
    got = p.summarise()
    assert p.dc.read_status() == 0
    assert len(check_summary(p, got, None)) == 1 + 1 + 3 + 5


@pytest.mark.parametrize("new", [(1,) * 7, (0, 1, -1, 65, 64, 2, 500), (500,) * 7])
def test_summaries_of_the_pages_that_new_tokens_complete(gpu_lib, new):
    p = Pages(make("gate256", (0, 64, 128, 65, 192, 193, 320)))
    t = dev(new)
    got = p.summarise(t, max(new))
    assert p.dc.read_status() == 0
    check_summary(p, got, new)


def test_summaries_report_bad_arguments_on_the_device(gpu_lib):
    def fresh():
        return Pages(make("gate256", (130, 320)))
    p = fresh()
    p.dc.block_table[1, 2] = p.case.num_pages
    p.summarise()
    assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE
    p = fresh()
    p.dc.id_pool[int(p.case.block_table[0, 1]), 7] = -1
    p.summarise()
    assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE
    for lens in ((-4, 320), (130, 321)):
        p = fresh()
        p.summarise(lens=dev(lens))
        assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE
    p = fresh()
    p.summarise(dev((1, 200)), 100)
    assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE


# ------------------------------------------------------------------ sparse
class Sparse(Pages):
    def run(self, budget, first=1, last=1, splits=0, selected=True, stream=None):
        case, dc = self.case, self.dc
        B = case.batch
        self.selected = torch.full((B, budget), -9, dtype=torch.int32, device="cuda") if selected else None
        n = _lib.eg_mla_decode_sparse_workspace_size(dc.dims, B, case.max_pages, budget, splits)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        dc.out.fill_(float("nan"))
        torch.cuda.synchronize()
        _lib.eg_mla_decode_sparse(dc.dims, dc.q, dc.c_pool, dc.kr_pool, dc.id_pool, dc.block_table, dc.seq_lens,
                                  self.longest, self.summary, budget, first, last, dc.gate_table, dc.ln_gamma,
                                  dc.ln_beta, dc.w_uk, dc.w_uv, dc.out, ws, self.selected, splits, dc.status, stream)
        torch.cuda.synchronize()
        return self.selected.cpu().numpy() if selected else None

    def chosen(self, sel):
        """The selection as a block table and lengths, and eg_mla_decode over it."""
        case, dc = self.case, self.dc
        np_ = [pages_of(int(L)) for L in case.seq_lens]
        table = np.zeros((case.batch, sel.shape[1]), np.int32)
        lens = np.zeros(case.batch, np.int32)
        for b in range(case.batch):
            k = int((sel[b] >= 0).sum())
            table[b, :k] = case.block_table[b, sel[b, :k]]
            lens[b] = int(case.seq_lens[b]) - (np_[b] - k) * P
        ws = torch.empty(_lib.eg_mla_decode_workspace_size(dc.dims, case.batch, dc.num_splits), dtype=torch.uint8,
                         device="cuda")
        out = torch.empty_like(dc.out)
        _lib.eg_mla_decode(dc.dims, dc.q, dc.c_pool, dc.kr_pool, dc.id_pool, dev(table).view(table.shape), dev(lens),
                           int(lens.max()), dc.gate_table, dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, out, ws,
                           dc.num_splits, dc.status)
        torch.cuda.synchronize()
        c, kr, ids = orc.appended_pools(case)
        last = [max(int(n) - 1, 0) for n in lens]
        at = [(int(table[b, j // P]), j % P) for b, j in enumerate(last)]
        alone = dataclasses.replace(case, block_table=table, seq_lens=lens, c_pool=c, kr_pool=kr, id_pool=ids,
                                    c_new=np.stack([c[a] for a in at]), kr_new=np.stack([kr[a] for a in at]),
                                    ids_new=np.array([ids[a] for a in at], np.int32))
        return out, orc.decode_unabsorbed(alone)


def scores64(case, summary, b):
    """Scores of a sequence's pages from the stored summaries in 64 bits, and the fp32 sums' error bound."""
    d = case.dims
    m = summary[case.block_table[b, :pages_of(int(case.seq_lens[b]))]]
    q = orc.widen(case.q[b], d.dtype)
    w = orc.widen(case.w_uk, d.dtype)
    qa = np.concatenate([np.einsum("hd,hdc->hc", q[:, :d.d_nope], w), q[:, d.d_nope:]], 1)
    mag = np.concatenate([np.einsum("hd,hdc->hc", np.abs(q[:, :d.d_nope]), np.abs(w)), np.abs(q[:, d.d_nope:])], 1)
    s = qa @ m.T * orc.softmax_scale(d)
    err = 2.0 ** -24 * (d.d_nope + d.d_c + d.d_rope + 8) * (mag @ np.abs(m).T).max(0) * orc.softmax_scale(d)
    return s.max(0), err


def check_selection(case, sel, summary, budget, first, last):
    for b, L in enumerate(case.seq_lens):
        n = pages_of(int(L))
        got = sel[b][sel[b] >= 0].tolist()
        if n <= budget:
            assert got == list(range(n)) and (sel[b, n:] == -1).all()
            continue
        assert len(got) == budget and got == sorted(set(got))
        assert got[:first] == list(range(first)) and got[budget - last:] == list(range(n - last, n))
        s, err = scores64(case, summary, b)
        taken = got[first:budget - last]
        left = [p for p in range(first, n - last) if p not in taken]
        for p in taken:
            assert (s[p] + err[p] >= s[left] - err[left]).all(), (b, p)


LENS = (0, 1, 64, 500, 640, 1999, 1283)


@pytest.mark.parametrize("name", sorted(SHAPES))
@pytest.mark.parametrize("budget,first,last", [(1, 0, 1), (3, 1, 2), (9, 1, 1), (20, 2, 3), (64, 1, 1)])
def test_sparse_decode(gpu_lib, name, budget, first, last):
    p = Sparse(make(name, LENS))
    summary = p.summarise()
    sel = p.run(budget, first, last)
    assert p.dc.read_status() == 0
    check_selection(p.case, sel, summary, budget, first, last)
    out, ref = p.chosen(sel)
    assert torch.equal(p.dc.out, out)
    got = device.output_f64(p.dc.out)
    rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    if p.case.dims.dtype == "fp32":
        assert rel <= 1e-5
    else:
        assert rel <= 5e-3 and (np.abs(got - ref) <= 1e-2 * np.maximum(1, np.abs(ref))).all()


def test_a_budget_for_every_page_is_the_dense_decode(gpu_lib):
    p = Sparse(make("gate256", LENS))
    p.summary.fill_(float("nan"))   # not read
    p.run(32, selected=False)
    sparse = p.dc.out.clone()
    dc = p.dc
    _lib.eg_mla_decode(dc.dims, dc.q, dc.c_pool, dc.kr_pool, dc.id_pool, dc.block_table, dc.seq_lens, p.longest,
                       dc.gate_table, dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, dc.out, dc.workspace, 0, dc.status)
    torch.cuda.synchronize()
    assert p.dc.read_status() == 0 and torch.equal(sparse, dc.out)


@pytest.mark.parametrize("name", ["gate256", "fp32_64"])
def test_equal_scores_infinities_and_no_numbers(gpu_lib, name):
    """Pages whose summaries are the same rank by position; an infinite score first
    (last if negative), one that is no number after every number."""
    p = Sparse(make(name, (64 * 40, 64 * 700 + 5)))
    r = np.random.default_rng(2)
    D = p.summary.shape[1]
    kinds = r.standard_normal((5, D)).astype(np.float32)
    case = p.case
    for b in range(2):
        n = pages_of(int(case.seq_lens[b]))
        what = r.integers(0, 5, n)
        p.summary[case.block_table[b, :n]] = torch.from_numpy(kinds[what]).cuda()
        s, err = scores64(case, p.summary.cpu().numpy().astype(np.float64), b)
        order = sorted(range(1, n - 1), key=lambda i: (-round(s[i], 4), i))
        for budget in (2, 3, 7, 19, 38):
            got = p.run(budget)[b].tolist()
            assert got == sorted([0, n - 1] + order[:budget - 2]), (b, budget)
    # page 5 of sequence 1 has no number, page 9 an infinite score of either sign per head, so the largest is +inf
    p.summary[int(case.block_table[1, 5])] = float("nan")
    p.summary[int(case.block_table[1, 9])] = 0.0
    p.summary[int(case.block_table[1, 9]), 0] = float("inf")
    n = pages_of(int(case.seq_lens[1]))
    assert 9 in p.run(3)[1].tolist()
    everything_but_one = p.run(n - 1)[1].tolist()
    assert 5 not in everything_but_one and len(set(everything_but_one)) == n - 1
    p.summary.fill_(float("nan"))   # nothing but no numbers: by position
    assert p.run(6)[1].tolist() == [0, 1, 2, 3, 4, n - 1]
    p.summary.fill_(0.0)            # +0 and -0 are equal
    p.summary[int(case.block_table[1, 3])] = -0.0
    assert p.run(6)[1].tolist() == [0, 1, 2, 3, 4, n - 1]


def test_sparse_repeats_bit_for_bit_and_runs_on_any_stream(gpu_lib):
    p = Sparse(make("gate192", LENS))
    p.summarise()
    sel = p.run(7)
    out = p.dc.out.clone()
    for splits in (0, 0):
        again = p.run(7, splits=splits, stream=torch.cuda.Stream())
        assert np.array_equal(sel, again) and torch.equal(out, p.dc.out)


def test_sparse_reports_bad_lengths_and_pages(gpu_lib):
    p = Sparse(make("gate256", LENS))
    p.summarise()
    p.dc.seq_lens[3] = p.longest + 1
    p.run(5)
    assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE
    p = Sparse(make("gate256", LENS))
    p.summarise()
    p.dc.block_table[5, 7] = -3
    p.run(5)
    assert p.dc.read_status() == _lib.EG_MLA_ERR_OUT_OF_RANGE


def test_plan_drops_what_the_stack_cannot_hold_whatever_the_sum(gpu_lib):
    """Stale lengths that give back nearly 2^31 pages to a stack of 200,000."""
    B, width, num_pages, free = 16384, 131071, 200000, 160000
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    table[0, :num_pages - free] = torch.arange(free, num_pages, dtype=torch.int32, device="cuda")
    stack = torch.arange(num_pages, dtype=torch.int32, device="cuda")
    stack[free:] = -1
    lens, new = dev([width * P] * (B - 1) + [0]), dev([-1] * (B - 1) + [1])
    assert (B - 1) * width + free > 2 ** 31 - 1
    lens_out, left, cu, pos, slots, status = dev([-9] * B), dev([-9]), dev([0] * (B + 1)), dev([0] * B), dev([0] * 2), dev([0])
    _lib.eg_mla_page_plan(new, lens, lens_out, table, stack, dev([free]), left, cu, pos, slots, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == _lib.EG_MLA_ERR_OUT_OF_RANGE
    assert left.tolist() == [num_pages - 1]
    assert stack.tolist() == list(range(num_pages))
    assert lens_out.tolist() == [0] * (B - 1) + [1] and int(cu[B].item()) == 1 and pos.tolist() == [-1] * (B - 1) + [0]
    assert int(table[B - 1, 0].item()) == num_pages - 1 and slots.tolist() == [(num_pages - 1) * P, -1]


@pytest.mark.parametrize("name", ["gate256", "none512", "fp32_64", "fp32_132", "fp32_none", "fp32_512"])
def test_a_page_without_a_number_comes_after_the_lowest_score(gpu_lib, name):
    """Whatever the number of heads: a page whose every head has no number ranks after one
    of minus infinity; heads without a number are left out where others have one."""
    p = Sparse(make(name, (64 * 20,)))
    d, n = p.case.dims, 20
    p.summary.fill_(0.0)
    p.dc.q[0, :, d.d_nope] = 1.0
    p.dc.q[0, :, d.d_nope + 1] = 1.0
    p.dc.q[0, 0, d.d_nope + 1] = 0.0
    page = [int(x) for x in p.case.block_table[0]]
    p.summary[page[5]] = float("nan")
    p.summary[page[9], d.d_c] = -float("inf")
    assert p.run(n - 1)[0].tolist() == [i for i in range(n) if i != 5]
    assert p.run(n - 2)[0].tolist() == [i for i in range(n) if i not in (5, 9)]
    # head 0 has 0 times infinity, the others infinity: the page is the best
    p.summary[page[12], d.d_c + 1] = float("inf")
    assert p.run(3)[0].tolist() == [0, 12, n - 1]


@pytest.mark.parametrize("name", ["gate256", "fp32_64"])
def test_a_score_that_underflows_equals_zero(gpu_lib, name):
    """Scores of +0 and of -0 (a small negative one times a small scale) are equal: by position."""
    case = make(name, (64 * 20,))
    case = dataclasses.replace(case, dims=dataclasses.replace(case.dims, softmax_scale=1e-30))
    p = Sparse(case)
    p.summary.fill_(0.0)
    p.dc.q[0, :, case.dims.d_nope] = 1.0
    p.summary[int(case.block_table[0, 3]), case.dims.d_c] = -1e-30
    assert p.run(6)[0].tolist() == [0, 1, 2, 3, 4, 19]


def test_plan_can_be_captured(gpu_lib):
    """A captured plan serves the lengths that its inputs hold at each replay."""
    cases = [plan_case(seed, 700, 900, spare=spare, width=30) for seed, spare in ((21, -20), (22, 5), (23, 0))]
    slots = max(sum(max(n, 0) for n in c[0]) for c in cases)
    most = max(len(c[3]) for c in cases)
    cases = [(*c[:3], np.concatenate([c[3], np.full(most - len(c[3]), 77)]), c[4]) for c in cases]
    new, lens, table, stack, free = (dev(x) for x in (*cases[0][:4], [0]))
    lens_out, left, cu, pos, at, status = dev([0] * 700), dev([0]), dev([0] * 701), dev([0] * 700), dev([0] * slots), dev([0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _lib.eg_mla_page_plan(new, lens, lens_out, table, stack, free, left, cu, pos, at, dev_status=status)
    for case in cases:
        for dst, src in zip((new, lens, table, stack, free, status), (*case[:4], [case[4]], [0])):
            dst.copy_(dev(src))
        graph.replay()
        torch.cuda.synchronize()
        want, st = plan_reference(*case, slots)
        got = dict(seq_lens=lens_out, table=table, stack=stack, free=left, cu=cu, positions=pos, slots=at)
        assert_plan({k: v.cpu().numpy() for k, v in got.items()}, want)
        assert int(status.item()) == st


class Wide(Sparse):
    """Long sequences over a few physical pages, whose summaries are drawn."""

    def __init__(self, name, lens, seed=1):
        small = make(name, (64 * 9, 64 * 6))
        super().__init__(small)
        d, r, B = small.dims, np.random.default_rng(seed), len(lens)
        held = small.block_table[:, :6].reshape(-1)
        q = r.standard_normal((B, d.num_heads, d.d_nope + d.d_rope)).astype(np.float32)
        self.case = dataclasses.replace(
            small, block_table=held[r.integers(0, len(held), (B, pages_of(max(lens))))].astype(np.int32),
            seq_lens=np.array(lens, np.int32), q=synth.f32_to_bf16_bits(q) if d.dtype == "bf16" else q)
        dc = self.dc
        dc.q = device.to_device_array(self.case.q, d.dtype, "cuda")
        dc.block_table, dc.seq_lens = dev(self.case.block_table).view(B, -1), dev(lens)
        dc.out = torch.empty((B, d.num_heads, d.d_v), dtype=dc.out.dtype, device="cuda")
        self.summary = torch.from_numpy(r.standard_normal((small.num_pages, d.d_c + d.d_rope)).astype(np.float32)).cuda()
        self.longest = max(lens)

    def check(self, budget, first, last, splits=0):
        """The selection; of pages with the same summary the first ones; the decode's bits."""
        case, dc = self.case, self.dc
        sel = self.run(budget, first, last, splits)
        assert dc.read_status() == 0
        check_selection(case, sel, self.summary.cpu().numpy().astype(np.float64), budget, first, last)
        for b, L in enumerate(case.seq_lens):
            n, taken = pages_of(int(L)), set(sel[b].tolist())
            if n <= budget:
                continue
            left = {}
            for i in range(first, n - last):
                page = int(case.block_table[b, i])
                if i not in taken:
                    left[page] = i
                else:
                    assert page not in left, (b, i, left[page])
        count = (sel >= 0).sum(1)
        table = np.where(sel >= 0, np.take_along_axis(case.block_table, np.maximum(sel, 0), 1), 0)
        lens = [int(L) - (pages_of(int(L)) - int(k)) * P for L, k in zip(case.seq_lens, count)]
        ws = torch.empty(_lib.eg_mla_decode_workspace_size(dc.dims, case.batch, splits), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(dc.out)
        _lib.eg_mla_decode(dc.dims, dc.q, dc.c_pool, dc.kr_pool, dc.id_pool, dev(table).view(table.shape), dev(lens),
                           max(lens), dc.gate_table, dc.ln_gamma, dc.ln_beta, dc.w_uk, dc.w_uv, out, ws, splits,
                           dc.status)
        torch.cuda.synchronize()
        assert dc.read_status() == 0 and torch.equal(out, dc.out)


@pytest.mark.parametrize("name", ["gate256", "none512", "fp32_132", "fp32_512"])
@pytest.mark.parametrize("budget,first,last", [(9, 1, 1), (64, 0, 2)])
def test_selection_in_several_rounds_and_blocks(gpu_lib, name, budget, first, last):
    """More groups of pages than blocks: 32 sequences of up to 512 pages (four rounds of a
    block, two where a row is read in two parts), and fewer, of 900 (two)."""
    r = np.random.default_rng(6)
    long = [int(x) for x in r.integers(400 * P, 512 * P, 31)] + [512 * P]
    Wide(name, long).check(budget, first, last)
    Wide(name, long[:20] + [7 * P, 70 * P + 1, 0, 140 * P - 3], seed=2).check(budget, first, last)
    Wide(name, [900 * P, 899 * P + 1, 200 * P, 13] * 3, seed=3).check(budget, first, last)


@pytest.mark.parametrize("name", ["gate192", "none512", "fp32_132"])
@pytest.mark.parametrize("budget", [20, 2100, 4250, 4600])
def test_selection_from_more_pages_than_shared_memory_holds(gpu_lib, name, budget):
    """More than 4,096 ranked pages, with equal scores on both sides of that number."""
    Wide(name, [4700 * P - 5, 4300 * P, 100 * P]).check(budget, 1, 2)


@pytest.mark.parametrize("name", ["gate192", "gate256", "none512", "fp32_64"])
@pytest.mark.parametrize("splits", [1, 3, 40, 300])
def test_sparse_decode_with_a_number_of_splits(gpu_lib, name, splits):
    Wide(name, [30 * P, 1, 41 * P - 7, 8 * P]).check(9, 1, 1, splits)


@pytest.mark.parametrize("name", ["gate256", "none512", "fp32_none"])
def test_pages_past_32_bits_of_a_pool(gpu_lib, name):
    """Pages whose elements and bytes lie past 2^31 and 2^32 in the latent pool: the same bits."""
    p = Sparse(make(name, LENS))
    dc, n = p.dc, p.case.num_pages
    summary = torch.from_numpy(p.summarise())
    sel = p.run(9, 1, 1)
    out = dc.out.clone()
    shift = 2 ** 31 // (P * p.case.dims.d_c) + 1
    for pool in ("c_pool", "kr_pool", "id_pool"):
        small = getattr(dc, pool)
        big = torch.zeros((shift + n, *small.shape[1:]), dtype=small.dtype, device="cuda")
        big[shift:] = small
        setattr(dc, pool, big)
    dc.block_table = dc.block_table + shift
    p.summary = torch.full((shift + n, p.summary.shape[1]), -77.0, device="cuda")
    assert torch.equal(torch.from_numpy(p.summarise()[shift:]), summary)
    assert np.array_equal(p.run(9, 1, 1), sel) and torch.equal(dc.out, out)
    assert dc.read_status() == 0
