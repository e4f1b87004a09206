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


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("drop", [3.0, 9.0, 12.0, 15.0, 17.0])
def test_small_weights_beside_one_whose_value_is_not_read(gpu_lib, d_c, drop):
    """One token has all but a share of the weight, and values in features that W_UV does not look at; the others'
    weights lie about e^-drop below it, spread, and make up the whole output.  (A bf16 weight is off by 2^-9 of itself at
    most, at any size: the bound is the one of ordinary weights.)"""
    _, dc = make([6000, 300], d_c, "none", vocab=100, splits=1)
    half = d_c // 2
    dc.c_pool[..., :half] = 0
    dc.w_uv[..., :half] = 0
    for b in range(2):
        page = int(dc.block_table[b, 0])
        dc.c_pool[page, 0, :half] = dc.c_pool[page, 0, half:]
        dc.c_pool[page, 0, half:] = 0
    # scores by the RoPE part alone
    dc.q.zero_()
    dc.q[..., 128] = 1.0
    g = torch.Generator(device="cuda").manual_seed(3)
    s = -drop + torch.randn(dc.kr_pool.shape[:2], generator=g, device="cuda") * 0.5
    dc.kr_pool.zero_()
    dc.kr_pool[..., 0] = (s * 192 ** 0.5).to(torch.bfloat16)
    for b in range(2):
        dc.kr_pool[int(dc.block_table[b, 0]), 0, 0] = 0
    cache, back = quantised(dc)
    got, want = decode_q8(dc, cache), reference64(dc, back)
    assert dc.read_status() == 0
    for b in range(2):
        assert apart(got[b], want[b]) <= 5e-3, b
