"""Refusals of the serving calls (page plan, summaries, sparse and shared decode) that
come before any launch, and their workspace sizes: no GPU is needed."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2509_16686_gb300 import _lib

FAKE = 0x10000   # 256-byte aligned, never dereferenced: validation fails first
ODD = 0x10008
INVALID, UNSUPPORTED, WORKSPACE = _lib.EG_MLA_ERR_INVALID_ARG, _lib.EG_MLA_ERR_UNSUPPORTED, _lib.EG_MLA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def dims(d_c=256, **kw):
    return _lib.make_dims(16, 128, 64, 128, d_c, 32000, **kw)


def f32(d_rope=16):
    return _lib.make_dims(4, 32, d_rope, 32, 64, 1000, dtype="fp32")


def call(fn, spec, **changed):
    args = dict(spec)
    for k, v in changed.items():
        assert k in args
        args[k] = v
    d = args.get("dims")
    return fn(*[ctypes.byref(v) if v is d and d is not None else v for v in args.values()])


SHARED = dict(dims=dims(), q=FAKE, c_pool=FAKE, krope_pool=FAKE, id_pool=FAKE, prefix_table=FAKE, prefix_len=FAKE,
              max_prefix_len=1000, block_table=FAKE, max_pages=4, seq_lens=FAKE, max_seq_len=256, batch=3, num_pages=8,
              gate_table=FAKE, gamma=None, beta=None, w_uk=FAKE, w_uv=FAKE, out=FAKE, splits=152, workspace=FAKE,
              bytes=1 << 30, status=None, stream=None)


def test_shared_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_decode_shared, SHARED, **kw)
    for name in ("q", "c_pool", "krope_pool", "id_pool", "prefix_table", "prefix_len", "block_table", "seq_lens",
                 "gate_table", "w_uk", "w_uv", "out"):
        assert rc(**{name: None}) == INVALID, name
    for name in ("q", "c_pool", "krope_pool", "gate_table", "w_uk", "w_uv"):
        assert rc(**{name: ODD}) == INVALID, name
    assert rc(dims=None) == INVALID
    assert rc(max_prefix_len=-1) == INVALID
    assert rc(batch=-1) == INVALID
    assert rc(max_seq_len=257) == INVALID
    assert rc(splits=-1) == INVALID
    assert rc(dims=dims(d_c=512, gate=False)) == UNSUPPORTED
    assert rc(dims=f32()) == UNSUPPORTED
    assert rc(max_prefix_len=2 ** 31 - 1, batch=2 ** 20) == UNSUPPORTED
    assert rc(workspace=None) == WORKSPACE
    assert rc(workspace=ODD) == WORKSPACE
    need = _lib.eg_mla_decode_shared_workspace_size(SHARED["dims"], 3, 1000, 152)
    assert rc(bytes=need - 1) == WORKSPACE


def test_shared_workspace_size():
    d = dims()
    size = _lib.eg_mla_decode_shared_workspace_size
    dec = _lib.eg_mla_decode_workspace_size(d, 64, 152)
    n = size(d, 64, 32768, 152)
    # the gated prefix and the partials of 152 CTAs and 8 row tiles of 128 rows
    assert n >= dec + 32768 * 512 + (152 + 8) * 128 * (256 + 2) * 4 and n % 256 == 0
    assert size(d, 64, 0, 152) < n
    # with the gate off the pool is read in place
    assert size(dims(gate=False), 64, 32768, 152) <= n - 32000 * 512
    raw = _lib.load().eg_mla_decode_shared_workspace_size
    assert raw(ctypes.byref(d), -1, 10, 152) == 0 and raw(ctypes.byref(d), 1, -1, 152) == 0
    assert raw(ctypes.byref(f32()), 1, 10, 152) == 0 and raw(None, 1, 10, 152) == 0
    with pytest.raises(_lib.EgMlaError):
        size(dims(d_c=512, gate=False), 1, 10, 152)


SPARSE = dict(dims=dims(), q=FAKE, c_pool=FAKE, krope_pool=FAKE, id_pool=FAKE, block_table=FAKE, max_pages=40,
              seq_lens=FAKE, max_seq_len=2560, batch=3, num_pages=99, summary=FAKE, budget=8, first=1, last=2,
              gate_table=FAKE, gamma=None, beta=None, w_uk=FAKE, w_uv=FAKE, out=FAKE, selected=None, splits=152,
              workspace=FAKE, bytes=1 << 30, status=None, stream=None)


def test_sparse_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_decode_sparse, SPARSE, **kw)
    for name in ("q", "c_pool", "krope_pool", "id_pool", "block_table", "seq_lens", "summary", "gate_table", "w_uk",
                 "w_uv", "out"):
        assert rc(**{name: None}) == INVALID, name
    for name in ("q", "c_pool", "krope_pool", "summary", "gate_table", "w_uk", "w_uv"):
        assert rc(**{name: ODD}) == INVALID, name
    for kw in (dict(first=-1), dict(last=0), dict(budget=2), dict(budget=0), dict(budget=-5),
               dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(max_seq_len=2561), dict(max_seq_len=-1), dict(batch=-1),
               dict(num_pages=0), dict(max_pages=0), dict(splits=-1), dict(dims=None)):
        assert rc(**kw) == INVALID, kw
    assert rc(dims=dims(d_c=320)) == UNSUPPORTED
    assert rc(dims=f32(d_rope=18)) == UNSUPPORTED
    need = _lib.eg_mla_decode_sparse_workspace_size(SPARSE["dims"], 3, 40, 8, 152)
    assert need >= _lib.eg_mla_decode_workspace_size(SPARSE["dims"], 3, 152) + 3 * (16 * 320 * 4 + 40 * 4 + 8 * 4)
    for kw in (dict(workspace=None), dict(workspace=ODD), dict(bytes=need - 1)):
        assert rc(**kw) == WORKSPACE, kw
    raw = lib.eg_mla_decode_sparse_workspace_size
    d = ctypes.byref(dims())
    assert raw(d, -1, 40, 8, 152) == 0 and raw(d, 3, 0, 8, 152) == 0 and raw(d, 3, 40, 0, 152) == 0


def test_sparse_decode_of_no_sequence_returns():
    """Nothing to do, whatever the bounds: in a process of its own, which a division by
    the number of blocks would end."""
    code = """
import ctypes
from paper_2509_16686_gb300 import _lib
lib, F = _lib.load(), 0x10000
for d in (_lib.make_dims(16, 128, 64, 128, 256, 32000), _lib.make_dims(16, 128, 64, 128, 512, 32000, gate=False),
          _lib.make_dims(4, 32, 16, 32, 64, 1000, dtype="fp32")):
    for pages in (1, 40, 100000):
        rc = lib.eg_mla_decode_sparse(ctypes.byref(d), F, F, F, F, F, pages, F, 64 * pages, 0, 99, F, 8, 1, 2, F, None,
                                      None, F, F, F, None, 152, F, 1 << 30, None, None)
        assert rc == 0, (pages, rc)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stderr)


SUMMARY = dict(dims=dims(), c_pool=FAKE, krope_pool=FAKE, id_pool=FAKE, block_table=FAKE, max_pages=40, seq_lens=FAKE,
               max_seq_len=2560, new_tokens=None, max_new=0, batch=3, num_pages=99, gate_table=FAKE, gamma=None,
               beta=None, summary=FAKE, status=None, stream=None)


def test_summary_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_page_summary, SUMMARY, **kw)
    for name in ("c_pool", "krope_pool", "id_pool", "block_table", "seq_lens", "gate_table", "summary"):
        assert rc(**{name: None}) == INVALID, name
    for name in ("c_pool", "krope_pool", "gate_table", "summary"):
        assert rc(**{name: ODD}) == INVALID, name
    for kw in (dict(dims=None), dict(batch=-1), dict(num_pages=0), dict(max_pages=0), dict(max_seq_len=-1),
               dict(max_seq_len=2561), dict(max_new=-1)):
        assert rc(**kw) == INVALID, kw
    assert rc(dims=f32(d_rope=18)) == UNSUPPORTED
    assert rc(max_pages=2 ** 24, max_seq_len=2 ** 30, batch=2 ** 10) == UNSUPPORTED
    # nothing to do: nothing is launched
    assert rc(batch=0) == 0 and rc(max_seq_len=0) == 0 and rc(new_tokens=FAKE, max_new=0) == 0


PLAN = dict(new_tokens=FAKE, seq_lens=FAKE, seq_lens_out=FAKE, block_table=FAKE, max_pages=4, batch=3, free_pages=FAKE,
            num_pages=99, free_count=FAKE, free_count_out=FAKE, cu_seqlens=FAKE, positions=None, slots=None,
            max_slots=0, status=None, stream=None)


def test_plan_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_page_plan, PLAN, **kw)
    for name in ("new_tokens", "seq_lens", "seq_lens_out", "block_table", "free_pages", "free_count", "free_count_out",
                 "cu_seqlens"):
        assert rc(**{name: None}) == INVALID, name
    for kw in (dict(batch=-1), dict(max_pages=0), dict(num_pages=0), dict(max_slots=-1)):
        assert rc(**kw) == INVALID, kw
    for kw in (dict(batch=16385), dict(num_pages=2 ** 25), dict(max_pages=2 ** 25),
               dict(batch=16384, max_pages=2 ** 18), dict(slots=FAKE, max_slots=2 ** 31 - 1)):
        assert rc(**kw) == UNSUPPORTED, kw


def test_lengths_within_a_page_of_32_bits_are_refused(lib):
    """The pages of such a length are not counted in 32 bits."""
    for most, rc in ((2 ** 31 - 1, UNSUPPORTED), (2 ** 31 - 63, UNSUPPORTED), (2 ** 31 - 64, WORKSPACE)):
        assert call(lib.eg_mla_decode_sparse, SPARSE, max_pages=2 ** 25, max_seq_len=most, bytes=1) == rc
        assert call(lib.eg_mla_decode_shared, SHARED, dims=dims(gate=False), max_prefix_len=most, bytes=1) == rc
        assert call(lib.eg_mla_decode_shared, SHARED, max_pages=2 ** 25, max_seq_len=most, bytes=1) == rc
    for most in (2 ** 31 - 1, 2 ** 31 - 63):
        assert call(lib.eg_mla_page_summary, SUMMARY, max_pages=2 ** 25, max_seq_len=most) == UNSUPPORTED


def test_no_pages_has_its_own_text(lib):
    assert b"page" in lib.eg_mla_status_string(_lib.EG_MLA_ERR_NO_PAGES)
    assert b"unknown" in lib.eg_mla_status_string(-9)


def test_binding_checks_shapes():
    import torch
    t = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="cu_seqlens"):
        _lib.eg_mla_page_plan(t, t, t, t.view(3, 1), t, t[:1], t[:1], t)
    with pytest.raises(ValueError, match="summary"):
        _lib.eg_mla_page_summary(dims(), torch.zeros(4, 64, 256), t, t, t.view(3, 1), t, 64, t, t, t,
                                 torch.zeros(4, 256))
    with pytest.raises(ValueError, match="prefix_table"):
        _lib.eg_mla_decode_shared(dims(), t, t, t, t, t, t, 193, t, t, 64, t, t, t, t, t, t, t)
