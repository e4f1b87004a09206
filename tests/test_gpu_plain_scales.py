"""The ungated decode on codes as they are cached (d_c 256 and 512), at the far ends of what its contract allows."""
import pytest
import torch

from tests.test_gpu_tokens import apart, decode_q8, make, quantised, reference64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("power", [90, 112, 118])
def test_large_scales_keep_scores_finite(gpu_lib, d_c, power):
    """Sequences of one token, and of one token many times over, have that token's values as their result whatever its
    score, which is finite: below 2^(9 + power) |q^| with queries of ordinary size."""
    _, dc = make([1, 64, 130, 1], d_c, "none")
    c = dc.c_pool.mul_(2.0 ** power)
    for b, n in enumerate(dc.seq_lens.tolist()):   # the sequence's first token throughout
        pages = dc.block_table[b, :-(-n // 64)].long()
        c[pages] = c[pages[0], 0].clone()
        dc.kr_pool[pages] = dc.kr_pool[pages[0], 0].clone()
    cache, back = quantised(dc)
    got, want = decode_q8(dc, cache), reference64(dc, back)
    assert dc.read_status() == 0 and bool(got.isfinite().all())
    assert apart(got * 2.0 ** -power, want * 2.0 ** -power) <= 5e-3


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("power", [-80, 80, 100, 108])
def test_queries_small_beside_large_scales(gpu_lib, d_c, power):
    """Latents of 2^power and queries of 2^-power: scores of ordinary size, from queries whose own scale lies as far
    from 1 as the latents'."""
    _, dc = make([200, 64, 130], d_c, "none")
    dc.c_pool.mul_(2.0 ** power)
    dc.q[..., :128] *= 2.0 ** -power
    cache, back = quantised(dc)
    got, want = decode_q8(dc, cache), reference64(dc, back)
    assert dc.read_status() == 0
    assert apart(got * 2.0 ** -power, want * 2.0 ** -power) <= 5e-3


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("power", [0, 100])
def test_queries_of_zero_and_mixed_sizes(gpu_lib, d_c, power):
    """A head of zeros weighs all tokens alike; heads of very different sizes have scales of their own."""
    _, dc = make([200, 1, 130], d_c, "none")
    dc.c_pool.mul_(2.0 ** power)
    dc.q[..., :128] *= 2.0 ** -power
    dc.q[:, 0] = 0
    dc.q[:, 1, :128] = 0
    dc.q[:, 2] *= 2.0 ** -12
    dc.q[:, 15] *= 2.0
    cache, back = quantised(dc)
    got, want = decode_q8(dc, cache), reference64(dc, back)
    assert dc.read_status() == 0
    for h in (0, 1, 2, 3, 15):
        assert apart(got[:, h] * 2.0 ** -power, want[:, h] * 2.0 ** -power) <= 5e-3, h
