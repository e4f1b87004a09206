"""Refusals of eg_mla_rope and of the calls on a cache in 8 bits that come before any
launch, and what the binding checks: no GPU is needed."""
import ctypes
import os
import re

import pytest
import torch

from paper_2509_16686_gb300 import _lib

FAKE = 0x10000   # 256-byte aligned, never dereferenced: validation fails first
ODD = 0x10008
INVALID, UNSUPPORTED, WORKSPACE = _lib.EG_MLA_ERR_INVALID_ARG, _lib.EG_MLA_ERR_UNSUPPORTED, _lib.EG_MLA_ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def dims(d_c=256, d_nope=128, d_rope=64, heads=16, **kw):
    return _lib.make_dims(heads, d_nope, d_rope, 128, d_c, 32000, **kw)


def call(fn, spec, **changed):
    args = dict(spec)
    for k, v in changed.items():
        assert k in args
        args[k] = v
    return fn(*[ctypes.byref(v) if isinstance(v, ctypes.Structure) else v for v in args.values()])


ROPE = dict(dims=dims(), rope=_lib.make_rope(), q=FAKE, q_stride=16 * 192, q_out=FAKE, q_out_stride=16 * 192, k=FAKE,
            k_stride=64, k_out=FAKE, k_out_stride=64, cu=FAKE, positions=FAKE, batch=3, tokens=10, status=None,
            stream=None)


def test_rope_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_rope, ROPE, **kw)
    for kw in (dict(dims=None), dict(rope=None), dict(batch=-1), dict(tokens=-1), dict(q=None), dict(q_out=None),
               dict(k=None), dict(k_out=None), dict(q=None, q_out=None, k=None, k_out=None), dict(q_stride=16 * 192 - 1),
               dict(q_out_stride=16 * 192 - 1), dict(q_stride=16 * 192 + 8), dict(k_stride=63), dict(k_out_stride=63),
               dict(k_stride=72), dict(q=0x10001), dict(k_out=0x10001), dict(cu=None), dict(cu=None, batch=9),
               dict(cu=None, batch=10, positions=None), dict(dims=dims(heads=0)), dict(dims=dims(d_nope=-1)),
               dict(dims=dims(d_rope=0))):
        assert rc(**kw) == INVALID, kw
    d = dims()
    d.dtype = 2
    assert rc(dims=d) == INVALID
    for kw in (dict(dims=dims(d_rope=63)), dict(dims=dims(d_rope=258)), dict(dims=dims(heads=65535)),
               dict(dims=dims(heads=60000, d_nope=2 ** 20))):
        assert rc(**kw) == UNSUPPORTED, kw
    # nothing to do: nothing is launched
    assert rc(batch=0) == 0 and rc(tokens=0) == 0
    assert rc(batch=0, tokens=0, cu=None, positions=None) == 0


@pytest.mark.parametrize("kw", [
    dict(theta=NAN), dict(theta=INF), dict(theta=0.5), dict(scaling="linear", factor=0.5),
    dict(scaling="ntk", factor=NAN), dict(scaling="ntk", factor=INF), dict(scaling="linear", factor=0.0),
    dict(magnitude=NAN), dict(magnitude=INF), dict(scaling="yarn", factor=4.0),
    dict(scaling="yarn", factor=4.0, original_len=-5),
    dict(scaling="yarn", factor=4.0, original_len=4096, beta_fast=1.0, beta_slow=1.0),
    dict(scaling="yarn", factor=4.0, original_len=4096, beta_fast=INF),
    dict(scaling="yarn", factor=4.0, original_len=4096, beta_slow=NAN, beta_fast=NAN)])
def test_rope_scalings_refused(lib, kw):
    if kw.get("beta_fast") != kw.get("beta_fast"):   # NaN selects the defaults, as 0 does
        assert call(lib.eg_mla_rope, ROPE, rope=_lib.make_rope(**kw), tokens=0) == 0
        return
    assert call(lib.eg_mla_rope, ROPE, rope=_lib.make_rope(**kw), tokens=0) == INVALID


def test_rope_layouts_refused(lib):
    for field, value in (("layout", 2), ("layout", -1), ("scaling", 4), ("scaling", -1)):
        r = _lib.make_rope()
        setattr(r, field, value)
        assert call(lib.eg_mla_rope, ROPE, rope=r) == INVALID
    assert call(lib.eg_mla_rope, ROPE, rope=_lib.make_rope(scaling="ntk", factor=2.0), dims=dims(d_rope=2)) == INVALID
    with pytest.raises(KeyError):
        _lib.make_rope("rotated")


APPEND = dict(dims=dims(), c8=FAKE, scale=FAKE, kr_pool=FAKE, ids_pool=FAKE, c=FAKE, c_stride=256, kr=FAKE,
              kr_stride=64, ids=FAKE, cu=FAKE, positions=FAKE, table=FAKE, max_pages=4, batch=3, tokens=10,
              num_pages=8, status=None, stream=None)
READ = dict(dims=dims(), c8=FAKE, scale=FAKE, kr_pool=FAKE, ids_pool=FAKE, cu=FAKE, positions=None, table=FAKE,
            max_pages=4, c=FAKE, c_stride=256, kr=FAKE, kr_stride=64, ids=FAKE, batch=3, tokens=10, num_pages=8,
            status=None, stream=None)


@pytest.mark.parametrize("which", ["append", "read"])
def test_cache_refusals(lib, which):
    fn, spec = (lib.eg_mla_append_latent_q8, APPEND) if which == "append" else (lib.eg_mla_read_latent_q8, READ)

    def rc(**kw):
        return call(fn, spec, **kw)
    for name in ("c8", "scale", "kr_pool", "c", "table", "dims"):
        assert rc(**{name: None}) == INVALID, name
    for name in ("c8", "kr_pool", "c", "kr"):
        assert rc(**{name: ODD}) == INVALID, name
    for kw in (dict(batch=-1), dict(tokens=-1), dict(num_pages=0), dict(max_pages=0), dict(c_stride=255),
               dict(c_stride=260), dict(kr_stride=63), dict(kr_stride=68), dict(cu=None),
               dict(cu=None, batch=10, positions=None), dict(dims=dims(d_c=0)), dict(dims=dims(d_rope=0))):
        assert rc(**kw) == INVALID, kw
    if which == "append":
        assert rc(kr=None) == INVALID
    else:
        assert rc(ids_pool=None) == INVALID   # ids wanted that the cache does not hold
    for kw in (dict(dims=dims(page_size=32)), dict(dims=dims(d_c=200)), dict(dims=dims(d_c=528)),
               dict(dims=dims(d_rope=60)), dict(dims=dims(d_rope=264)), dict(dims=dims(d_rope=62, dtype="fp32")),
               dict(num_pages=2 ** 25)):
        assert rc(**kw) == UNSUPPORTED, kw
    assert rc(batch=0) == 0 and rc(tokens=0) == 0


DECODE = dict(dims=dims(), q=FAKE, c8=FAKE, scale=FAKE, kr_pool=FAKE, ids_pool=FAKE, table=FAKE, max_pages=40,
              seq_lens=FAKE, max_seq_len=2560, batch=3, num_pages=99, gate_table=FAKE, gamma=None, beta=None,
              w_uk=FAKE, w_uv=FAKE, out=FAKE, splits=152, workspace=FAKE, bytes=1 << 30, status=None, stream=None)


def test_decode_refusals(lib):
    def rc(**kw):
        return call(lib.eg_mla_decode_q8, DECODE, **kw)
    for name in ("q", "c8", "scale", "kr_pool", "ids_pool", "table", "seq_lens", "gate_table", "w_uk", "w_uv", "out",
                 "dims"):
        assert rc(**{name: None}) == INVALID, name
    for name in ("q", "c8", "scale", "kr_pool", "gate_table", "w_uk", "w_uv"):
        assert rc(**{name: ODD}) == INVALID, name
    for kw in (dict(batch=-1), dict(num_pages=0), dict(max_pages=0), dict(max_seq_len=-1), dict(max_seq_len=2561),
               dict(splits=-1)):
        assert rc(**kw) == INVALID, kw
    for kw in (dict(dims=dims(d_c=320)), dict(dims=dims(d_c=512)), dict(dims=dims(heads=8)),
               dict(dims=_lib.make_dims(4, 32, 16, 32, 68, 1000, dtype="fp32")), dict(num_pages=2 ** 25),
               dict(max_pages=2 ** 25, max_seq_len=2 ** 31 - 63)):
        assert rc(**kw) == UNSUPPORTED, kw
    need = _lib.eg_mla_decode_workspace_size(DECODE["dims"], 3, 152)
    for kw in (dict(workspace=None), dict(workspace=ODD), dict(bytes=need - 1)):
        assert rc(**kw) == WORKSPACE, kw
    assert rc(batch=0) == 0


def test_rope_struct_matches_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "egmla.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} eg_mla_rope_dims;", text).group(1)
    fields = re.findall(r"(int32_t|float)\s+(\w+);", body)
    kinds = {"int32_t": ctypes.c_int32, "float": ctypes.c_float}
    assert [(n, kinds[t]) for t, n in fields] == list(_lib.EgMlaRopeDims._fields_)


def test_binding_checks_shapes_and_types():
    """Every refusal comes before a pointer is taken, so CPU tensors show it."""
    d = dims()
    q, k = torch.zeros(3, 16, 192, dtype=torch.bfloat16), torch.zeros(3, 64, dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    rope = _lib.make_rope()
    with pytest.raises(ValueError, match="k_out"):
        _lib.eg_mla_rope(d, rope, None, None, k, None, pos)
    with pytest.raises(ValueError, match="q: shape"):
        _lib.eg_mla_rope(d, rope, q[:, :8], q, k, k, pos)
    with pytest.raises(ValueError, match="q: torch.bfloat16"):
        _lib.eg_mla_rope(d, rope, q.float(), q, k, k, pos)
    c8, scale = torch.zeros(4, 64, 256, dtype=torch.uint8), torch.zeros(4, 64)
    kr, ids = torch.zeros(4, 64, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.int32)
    table, c = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 256, dtype=torch.bfloat16)
    for name, args in (("c8_pool", (c8[:, :, :128], scale, kr, ids)), ("scale_pool", (c8, scale[:3], kr, ids)),
                       ("krope_pool", (c8, scale, kr[:, :32], ids)), ("id_pool", (c8, scale, kr, ids[:, :1])),
                       ("c8_pool", (c8.float(), scale, kr, ids)), ("scale_pool", (c8, scale.double(), kr, ids)),
                       ("krope_pool", (c8, scale, kr.float(), ids)), ("id_pool", (c8, scale, kr, ids.long()))):
        with pytest.raises(ValueError, match=name):
            _lib.eg_mla_append_latent_q8(d, *args, c, k, pos, table, pos)
        with pytest.raises(ValueError, match=name):
            _lib.eg_mla_read_latent_q8(d, *args, table, c, k, pos, pos)
        with pytest.raises(ValueError, match=name):
            _lib.eg_mla_decode_q8(d, q, *args, table, pos, 100, c, None, None, c, c, q, c)
    for name, bad in (("c_new", (c[:, :128], k, pos, table, pos)), ("krope_new", (c, k[:2], pos, table, pos)),
                      ("ids_new", (c, k, pos.long(), table, pos)), ("block_table", (c, k, pos, table[:2], pos)),
                      ("positions", (c, k, pos, table, pos[:2])), ("cu_seqlens", (c, k, pos, table, pos, pos.long()))):
        with pytest.raises(ValueError, match=name):
            _lib.eg_mla_append_latent_q8(d, c8, scale, kr, ids, *bad)
    with pytest.raises(ValueError, match="device"):
        _lib.eg_mla_append_latent_q8(d, c8, scale, kr, ids, c, k, pos, table, pos)
    with pytest.raises(ValueError, match="device"):
        _lib.eg_mla_decode_q8(d, q, c8, scale, kr, ids, table, pos, 100, c, None, None, c, c, q, c)
    with pytest.raises(ValueError, match="device"):
        _lib.eg_mla_rope(d, rope, q, q, k, k, pos)


def test_token_rows_are_dense_but_for_the_tokens():
    def rows(t, shape):
        return _lib._rows(t, shape, torch.float32, -1, "x")[1]   # (-1: the CPU)
    wide = torch.zeros(5, 100)
    assert rows(wide[:, 4:64].unflatten(1, (3, 20)), (5, 3, 20)) == 100
    assert rows(wide[:1, :60], (1, 60)) == 60
    assert rows(wide[:, :1].unsqueeze(-1), (5, 1, 1)) == 100
    assert rows(wide[:, :20].unsqueeze(1), (5, 1, 20)) == 100
    for bad, shape in ((wide.t()[:60], (60, 5)), (wide[:, ::2], (5, 50)), (wide[:1].expand(5, 100), (5, 100)),
                       (wide[:, :60].unflatten(1, (3, 20))[:, :, :10], (5, 3, 10)), (wide[:, ::2].unsqueeze(1), (5, 1, 50)),
                       (wide, (5, 99)), (wide.double(), (5, 100))):
        with pytest.raises(ValueError):
            rows(bad, shape)
