"""Packed-token calls with offsets that do not begin at 0 or that decrease: reported, and no token in a wrong place.

One offset j of a good list is changed so that the list decreases.  A token lies in a sequence b with cu[b] <= k <
cu[b + 1], and is taken only if cu[b - 1] <= cu[b] and cu[b + 1] <= cu[b + 2] too: with b and b + 1 other than j that
is the good list's sequence, and with either of them j the list would not decrease.  So every output is the good
list's or as it was."""
import numpy as np
import pytest
import torch

from paper_2509_16686_gb300 import _lib
from tests.test_gpu_tokens import Cache, DT, RANGE, append_case, ints, normal, offsets, status_word

pytestmark = pytest.mark.gpu


def changed(cu, seed, count):
    """Copies of a good list with one offset below the one before it or above the one behind it."""
    r = np.random.default_rng(seed)
    lists = []
    while len(lists) < count:
        j, other = int(r.integers(0, len(cu))), list(cu)
        if r.integers(2) and j > 0 and cu[j - 1] > 0:
            other[j] = int(r.integers(max(0, cu[j - 1] - 9), cu[j - 1]))
        elif j > 0 and j < len(cu) - 1:
            other[j] = int(cu[j + 1] + r.integers(1, 100))
        elif j == 0:
            other[j] = -int(r.integers(1, 9))
        if other[0] < 0 or any(a > b for a, b in zip(other, other[1:])):
            lists.append(other)
    return lists


def case(batch, seed, dtype="bf16", most=5):
    r = np.random.default_rng(seed)
    lens = r.integers(1, most, batch)
    lens[r.integers(0, batch, max(1, batch // 8))] = 0
    firsts = r.integers(0, 130, batch)
    dims, c, kr, ids, table, rows, cache = append_case(list(lens), list(firsts), 64, dtype, seed=seed)
    return lens, firsts, dims, c, kr, ids, ints(table), cache


def either(got, good, before):
    """Every entry as in the good call or as it was."""
    return bool(((got == good) | (got == before)).all())


# (the last: the tokens' warps are fewer than the offsets' 32s)
@pytest.mark.parametrize("batch", [2, 5, 31, 32, 33, 64, 100, 1024, 1057, 3000])
def test_offsets_that_decrease(gpu_lib, batch):
    lens, firsts, dims, c, kr, ids, table, cache = case(batch, batch, most=3 if batch == 3000 else 5)
    good_cu, pos, T = offsets(lens), ints(firsts), int(sum(lens))
    good = cache.clone()
    _lib.eg_mla_append_latent_q8(dims, *good.all(), c, kr, ids, table, pos, ints(good_cu))
    rope_dims = _lib.make_dims(1, 0, 8, 128, 256, 100, dtype="fp32")
    q = normal((T, 1, 8), "fp32", batch)

    def read(cu, status):
        out = torch.full_like(c, 99), torch.full_like(kr, 99), torch.full_like(ids, -9)
        _lib.eg_mla_read_latent_q8(dims, *good.all(), table, *out, pos, cu, status)
        return out

    def rope(cu, status):
        out = torch.full_like(q, 99)
        _lib.eg_mla_rope(rope_dims, _lib.make_rope(), q, out, None, None, pos, cu, status)
        return (out,)

    want, want_rope = read(ints(good_cu), None), rope(ints(good_cu), None)
    for bad in changed(good_cu, batch, 24):
        cu = ints(bad)
        st = [status_word() for _ in range(3)]
        got = cache.clone()
        _lib.eg_mla_append_latent_q8(dims, *got.all(), c, kr, ids, table, pos, cu, st[0])
        assert [int(s) for s in st] == [RANGE, 0, 0], bad
        for g, w, b in zip(got.all(), good.all(), cache.all()):
            assert either(g, w, b), bad
        for k, (call, full) in enumerate(((read, want), (rope, want_rope))):
            outs = call(cu, st[1 + k])
            assert int(st[1 + k]) == RANGE, bad
            for g, w in zip(outs, full):
                assert either(g, w, torch.full_like(w, -9 if w.dtype == torch.int32 else 99)), bad


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad,kept", [
    ([0, 5, 2, 6], []),              # the first two sequences meet at the decrease, the third is beside it
    ([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], []),   # all tokens lie before the first sequence
    ([1, 2, 4, 6], [1, 2, 3, 4, 5]), # begins above 0: the token before it belongs to no sequence
    ([-2, 2, 4, 6], [2, 3, 4, 5]),   # begins below 0: the first sequence's tokens have no place
    ([0, 2, 4, 3], [0, 1])])         # the last offset
def test_offsets_of_a_few_sequences(gpu_lib, dtype, bad, kept):
    """Which rows are taken, where a list of three sequences can be told by eye."""
    T, dims = 6, _lib.make_dims(16, 128, 64, 128, 64, 1000, dtype=dtype)
    c, kr, ids = normal((T, 64), dtype, 1), normal((T, 64), dtype, 2), ints(range(10, 16))
    table, cache, st = ints([[0], [1], [2]]), Cache(3, 64, dtype), status_word()
    cu = ints(bad)
    _lib.eg_mla_append_latent_q8(dims, *cache.all(), c, kr, ids, table, None, cu, st)
    assert int(st) == RANGE
    where = {k: (b, k - bad[b]) for k in kept for b in range(3) if bad[b] <= k < bad[b + 1]}
    left = torch.full_like(cache.ids, -5)
    for k, (b, p) in where.items():
        left[b, p] = 10 + k
    assert torch.equal(cache.ids, left)
    st.zero_()
    out = torch.full((T,), -9, dtype=torch.int32, device="cuda")
    _lib.eg_mla_read_latent_q8(dims, *cache.all(), table, torch.empty_like(c), None, out, None, cu, st)
    assert int(st) == RANGE and out.tolist() == [10 + k if k in where else -9 for k in range(T)]
    st.zero_()
    rd = _lib.make_dims(2, 8, 16, 128, 256, 100, dtype=dtype)
    q = normal((T, 2, 24), dtype, 3)
    qo, alone = torch.full_like(q, 9), torch.empty_like(q)
    _lib.eg_mla_rope(rd, _lib.make_rope(), q, qo, None, None, None, cu, st)
    _lib.eg_mla_rope(rd, _lib.make_rope(), q, alone, None, None, ints([where.get(k, (0, 0))[1] for k in range(T)]))
    assert int(st) == RANGE
    for k in range(T):
        assert torch.equal(qo[k], alone[k]) if k in where else bool((qo[k] == 9).all())


@pytest.mark.parametrize("batch", [300, 5000, 70000])
def test_a_few_tokens_of_many_sequences(gpu_lib, batch):
    """The offsets take more warps than the tokens: all of them are looked at, whatever the call's tokens are."""
    lens = np.zeros(batch, np.int64)
    lens[[3, batch // 2, batch - 1]] = [1, 2, 1]
    dims = _lib.make_dims(16, 128, 64, 128, 64, 1000)
    rd = _lib.make_dims(1, 0, 8, 128, 256, 100, dtype="fp32")
    odd = _lib.make_dims(1, 1, 6, 128, 256, 100)
    c, kr, ids = normal((4, 64), "bf16", 1), normal((4, 64), "bf16", 2), ints([10, 11, 12, 13])
    table, cu = torch.zeros((batch, 1), dtype=torch.int32, device="cuda"), np.asarray(offsets(lens))
    for k, b in enumerate((3, batch // 2, batch - 1)):
        table[b, 0] = k
    want = torch.full((3, 64), -5, dtype=torch.int32, device="cuda")
    want[0, 0], want[1, 0], want[1, 1], want[2, 0] = 10, 11, 12, 13
    q, x = normal((4, 1, 8), "fp32", 3), normal((4, 1, 7), "bf16", 4)
    r = np.random.default_rng(batch)
    for j in [None, 1, 2, 32, 33, batch // 2 + 1, batch - 1, batch, *r.integers(1, batch + 1, 12)]:
        bad = cu.copy()
        if j is not None:
            bad[j] = -1 if r.integers(2) or j == batch else 9
        bad = ints(bad)
        cache, st = Cache(3, 64, "bf16"), [status_word() for _ in range(4)]
        _lib.eg_mla_append_latent_q8(dims, *cache.all(), c, kr, ids, table, None, bad, st[0])
        io = torch.full((4,), -9, dtype=torch.int32, device="cuda")
        full = Cache(3, 64, "bf16")
        full.ids.copy_(want)
        _lib.eg_mla_read_latent_q8(dims, *full.all(), table, torch.empty_like(c), None, io, None, bad, st[1])
        _lib.eg_mla_rope(rd, _lib.make_rope(), q, torch.empty_like(q), None, None, None, bad, st[2])
        _lib.eg_mla_rope(odd, _lib.make_rope(), x, torch.empty_like(x), None, None, None, bad, st[3])
        assert [int(s) for s in st] == [0 if j is None else RANGE] * 4, j
        if j is None:
            assert torch.equal(cache.ids, want) and io.tolist() == [10, 11, 12, 13]
        assert either(cache.ids, want, torch.full_like(want, -5)) and either(io, ids, torch.full_like(io, -9)), j


def test_good_offsets_report_nothing(gpu_lib):
    """Empty sequences at either end and in between, and tokens behind the last."""
    for lens in ([0, 0, 3], [3, 0, 0], [0] * 40 + [1, 0, 2] + [0] * 40, [1] * 64):
        T, st = sum(lens) + 2, status_word()
        dims, c, kr, ids, table, _, cache = append_case(lens + [2], [0] * len(lens) + [-1], 64, "bf16")
        table, cu = ints(table[:-1]), ints(offsets(lens))
        _lib.eg_mla_append_latent_q8(dims, *cache.all(), c, kr, ids, table, None, cu, st)
        io = torch.full((T,), -9, dtype=torch.int32, device="cuda")
        _lib.eg_mla_read_latent_q8(dims, *cache.all(), table, torch.empty_like(c), None, io, None, cu, st)
        assert torch.equal(io[:-2], ids[:-2]) and bool((io[-2:] == -9).all()) and int(st) == 0
