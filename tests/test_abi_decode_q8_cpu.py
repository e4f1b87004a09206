"""What eg_mla_decode_q8's binding, and the status word of the packed-token calls, are held to before a pointer is
passed on: shapes, types, devices, contiguity.  Tensors on the CPU stand for the device's; the library call is a
stand-in that records its arguments."""
import pytest
import torch

from paper_2509_16686_gb300 import _lib

BF16 = torch.bfloat16
B, H, DN, DR, DV, DC, VOCAB, PAGES, WIDTH = 3, 16, 32, 64, 24, 256, 50, 4, 2


class Elsewhere(torch.Tensor):
    """A tensor that says it is on another device than the CPU's -1."""

    def get_device(self):
        return 1


def elsewhere(t):
    return t.clone().as_subclass(Elsewhere)


class Library:
    """Takes any call and records it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(_lib, "load", lambda: fake)
    monkeypatch.setattr(_lib, "_stream_on", lambda dev, stream: 7)
    return fake


def arguments(gate_mode="mul_ln", dtype="bf16", ids=True):
    t = BF16 if dtype == "bf16" else torch.float32
    dims = _lib.make_dims(H, DN, DR, DV, DC, VOCAB, dtype=dtype, gate=gate_mode != "none",
                          gate_op="mul_ln" if gate_mode == "none" else gate_mode)
    gated = gate_mode != "none"
    return dict(dims=dims, q=torch.zeros(B, H, DN + DR, dtype=t), c8_pool=torch.zeros(PAGES, 64, DC, dtype=torch.uint8),
                scale_pool=torch.zeros(PAGES, 64), krope_pool=torch.zeros(PAGES, 64, DR, dtype=t),
                id_pool=torch.zeros(PAGES, 64, dtype=torch.int32) if ids else None,
                block_table=torch.zeros(B, WIDTH, dtype=torch.int32), seq_lens=torch.zeros(B, dtype=torch.int32), max_seq_len=100,
                gate_table=torch.zeros(VOCAB, DC, dtype=t) if gated else None, ln_gamma=torch.zeros(DC) if gated else None,
                ln_beta=torch.zeros(DC) if gated else None, w_uk=torch.zeros(H, DN, DC, dtype=t),
                w_uv=torch.zeros(H, DV, DC, dtype=t), out=torch.zeros(B, H, DV, dtype=t),
                workspace=torch.zeros(4096, dtype=torch.uint8), dev_status=torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("gate", ["mul_ln", "mul", "add_ln", "none"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_good_arguments_are_passed_on(lib, gate, dtype):
    a = arguments(gate, dtype)
    _lib.eg_mla_decode_q8(**a)
    (name, args), = lib.calls
    assert name == "eg_mla_decode_q8" and len(args) == len(_lib_argtypes())
    order = ("q", "c8_pool", "scale_pool", "krope_pool", "id_pool", "block_table")
    assert [args[1 + i] for i in range(6)] == [a[n].data_ptr() for n in order]
    assert args[7:12] == (WIDTH, a["seq_lens"].data_ptr(), 100, B, PAGES)
    ln = gate in ("mul_ln", "add_ln")
    assert args[12:15] == (a["gate_table"].data_ptr() if gate != "none" else None, a["ln_gamma"].data_ptr() if ln else None,
                           a["ln_beta"].data_ptr() if ln else None)
    assert args[15:18] == tuple(a[n].data_ptr() for n in ("w_uk", "w_uv", "out"))
    assert args[18:] == (0, a["workspace"].data_ptr(), 4096, a["dev_status"].data_ptr(), 7)


def _lib_argtypes():
    import ctypes
    lib = ctypes.CDLL(_lib._build.build())
    _lib._declare(lib)
    return lib.eg_mla_decode_q8.argtypes


def bad_forms(t, name):
    """(tensor, what the error says) for everything that a tensor can be wrong in here."""
    yield torch.zeros((*t.shape[:-1], t.shape[-1] + 1), dtype=t.dtype), "shape"
    if name != "gate_table":
        yield torch.zeros((t.shape[0] + 1, *t.shape[1:]), dtype=t.dtype), "shape"
    yield torch.zeros((t.shape[0] - 1, *t.shape[1:]), dtype=t.dtype), "shape"
    yield t.unsqueeze(0), "shape"
    yield t.to(torch.float16), "expected, got"
    yield t.double(), "expected, got"
    yield elsewhere(t), "device"
    if t.dim() > 1:
        yield torch.zeros(t.shape[::-1], dtype=t.dtype).permute(*reversed(range(t.dim()))), "contiguous"
    else:
        yield torch.zeros(2 * t.shape[0], dtype=t.dtype)[::2], "contiguous"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", ["q", "gate_table", "ln_gamma", "ln_beta", "w_uk", "w_uv", "out"])
def test_every_tensor_is_checked(lib, name, dtype):
    a = arguments("mul_ln", dtype)
    for bad, says in bad_forms(a[name], name):
        with pytest.raises(ValueError, match=f"{name}: .*{says}"):
            _lib.eg_mla_decode_q8(**dict(a, **{name: bad}))
    other = torch.float32 if dtype == "bf16" else BF16   # the other model type
    if not name.startswith("ln_"):
        with pytest.raises(ValueError, match=name):
            _lib.eg_mla_decode_q8(**dict(a, **{name: a[name].to(other)}))
    assert lib.calls == []


def test_workspace_and_status_words(lib):
    a = arguments()
    for bad in (torch.zeros(8192, dtype=torch.uint8)[::2], elsewhere(a["workspace"])):
        with pytest.raises(ValueError, match="workspace"):
            _lib.eg_mla_decode_q8(**dict(a, workspace=bad))
    d, rope = a["dims"], _lib.make_rope()
    q, k, pos = torch.zeros(B, H, DN + DR, dtype=BF16), torch.zeros(B, DR, dtype=BF16), torch.zeros(B, dtype=torch.int32)
    c, cache = torch.zeros(B, DC, dtype=BF16), (a["c8_pool"], a["scale_pool"], a["krope_pool"], a["id_pool"])
    table = a["block_table"]
    calls = (lambda s: _lib.eg_mla_decode_q8(**dict(a, dev_status=s)),
             lambda s: _lib.eg_mla_rope(d, rope, q, q, k, k, pos, dev_status=s),
             lambda s: _lib.eg_mla_append_latent_q8(d, *cache, c, k, pos, table, pos, dev_status=s),
             lambda s: _lib.eg_mla_read_latent_q8(d, *cache, table, c, k, pos, pos, dev_status=s))
    for call in calls:
        for bad in (torch.zeros(1), torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32),
                    elsewhere(a["dev_status"])):
            with pytest.raises(ValueError, match="dev_status"):
                call(bad)
        assert lib.calls == []
        for good in (None, torch.zeros(1, dtype=torch.int32), torch.zeros((), dtype=torch.int32), torch.zeros(9, dtype=torch.int32)):
            call(good)
        assert len(lib.calls) == 4
        lib.calls.clear()


def test_a_padded_gate_table_is_taken(lib):
    _lib.eg_mla_decode_q8(**dict(arguments(), gate_table=torch.zeros(VOCAB + 14, DC, dtype=BF16)))
    assert len(lib.calls) == 1


def test_what_a_form_does_not_use_is_not_looked_at(lib):
    odd = torch.zeros(3, dtype=torch.float64)
    _lib.eg_mla_decode_q8(**dict(arguments("none"), gate_table=odd, ln_gamma=odd, ln_beta=odd))
    _lib.eg_mla_decode_q8(**dict(arguments("mul"), ln_gamma=odd, ln_beta=odd))
    _lib.eg_mla_decode_q8(**dict(arguments("mul_ln"), ln_gamma=None, ln_beta=None))
    assert [args[12:15] for _, args in lib.calls][0] == (None, None, None)
