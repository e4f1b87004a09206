"""Rotary positions and the latent cache held in 8 bits: plain forms and the library's calls.

A case is a dict of plain values; ``kind`` names the operator:

  rope     eg_mla_rope: the rotary embedding of packed tokens' queries and keys
  append   eg_mla_append_latent_q8: new tokens into the paged cache, the latent
           in e4m3 with a power-of-two scale per token
  read     eg_mla_read_latent_q8: cached tokens back as packed rows
  decode   eg_mla_decode_q8: one decode step over that cache

Lengths are part of the case (drawn from ``lens_seed``), everything else is
drawn on the GPU from the seed of the state.  Value distributions are those of
the library's synthetic workloads (latents 0.5 N(0, 1), gate table N(1, 0.1),
weights N(0, d_c^-1/2)).
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 64
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", batch=1, lo=1, hi=1, lens_seed=0, d_rope=64)
    if kind == "rope":
        c.update(heads=16, d_nope=128, step=False, far=0, layout="interleaved", scaling="none", theta=10000.0,
                 factor=1.0, original=4096, inverse=False)
    else:
        c.update(d_c=256)
    if kind in ("append", "read"):
        c.update(step=False, past=0, ids=True)
    if kind == "decode":
        c.update(heads=16, d_nope=128, gate="mul_ln", vocab=32000, ids="uniform", affine=True)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step: a token of each of 64 sequences somewhere in its text
        _case("rope", name="rope_step", batch=64, step=True, far=32768),
        # a full batch of prompts from the projections' rows to what the prefill takes
        _case("rope", name="rope_prompts", batch=8, lo=4096, hi=4096),
        # the gradient on the way back through a long-context model's positions, far into long texts
        _case("rope", name="rope_back", batch=13, lo=100, hi=4096, lens_seed=1, far=1 << 20, layout="half",
              scaling="yarn", theta=500000.0, factor=32.0, original=32768, inverse=True),
        # the tokens of a decode step of 64 sequences
        _case("append", name="append_step", batch=64, step=True, past=8192, lens_seed=2),
        # a full batch of prompts
        _case("append", name="append_prompts", batch=8, lo=4096, hi=4096),
        # one sequence's last turn back, an odd number of tokens from the middle of a page
        _case("read", name="read_turn", lo=1501, hi=1501, past=2999, d_c=192),
        # long prefixes read back to be processed on
        _case("read", name="read_prefixes", batch=16, lo=500, hi=16384, lens_seed=3),
        # a handful of short chats: latency
        _case("decode", name="decode_small", batch=4, lo=60, hi=700, lens_seed=4),
        # long context: 8 sequences of 32K tokens
        _case("decode", name="decode_32k", batch=8, lo=32768, hi=32768, affine=False),
        # a mixed batch, the narrower latent, Zipf ids
        _case("decode", name="decode_ragged", batch=128, lo=128, hi=16384, lens_seed=5, d_c=192, vocab=50000,
              ids="zipf"),
        # the plain MLA model on the same kind of batch
        _case("decode", name="decode_mla", batch=128, lo=128, hi=16384, lens_seed=5, gate="none", d_c=512),
        # single precision, the setting of a numerical check
        _case("decode", name="decode_fp32", dtype="fp32", batch=8, lo=100, hi=3000, lens_seed=6),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "read", "decode", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    common = dict(dtype=dtype, lens_seed=rng.randrange(1 << 20))
    width = 2 if dtype == "bf16" else 4
    if kind == "rope":
        heads, d_nope = _log_int(rng, 1, 64), rng.choice([0, 32, 64, 128, 128])
        d_rope = rng.choice([64, 64, 64, 16, 32, 128, 10])
        most = max(1, min(32768, 200000000 // ((heads * (d_nope + d_rope) + d_rope + 64) * width)))
        step = rng.random() < 0.3
        batch = _log_int(rng, 1, min(512, most))
        hi = 1 if step else _log_int(rng, 1, max(1, most // batch))
        return _case("rope", **common, heads=heads, d_nope=d_nope, d_rope=d_rope, batch=batch, step=step,
                     lo=rng.choice([hi, max(1, hi // 30)]), hi=hi, far=rng.choice([0, 4096, 1 << 17, 1 << 20]),
                     layout=rng.choice(["interleaved", "half"]), scaling=rng.choice(["none", "linear", "ntk", "yarn"]),
                     theta=rng.choice([10000.0, 500000.0, 1000000.0]), factor=rng.choice([1.0, 2.0, 8.0, 32.0]),
                     original=rng.choice([2048, 4096, 32768]), inverse=rng.random() < 0.4)
    if kind != "decode":
        step = rng.random() < 0.3
        batch = _log_int(rng, 1, 512)
        hi = 1 if step else _log_int(rng, 1, max(1, (100000 if kind == "read" else 32768) // batch))
        return _case(kind, **common, batch=batch, step=step, lo=rng.choice([hi, max(1, hi // 30)]), hi=hi,
                     past=rng.choice([0, 0, 100, 8192]), d_c=rng.choice([64, 128, 192, 256, 256, 512]),
                     d_rope=rng.choice([32, 64, 64]), ids=rng.random() < 0.8)
    common.update(ids=rng.choice(["uniform", "zipf"]), affine=rng.random() < 0.5, vocab=_log_int(rng, 1000, 50000))
    gate = rng.choice(["mul_ln", "mul_ln", "mul_ln", "mul", "add_ln", "none"])
    batch = _log_int(rng, 1, 128)
    hi = _log_int(rng, 1, max(1, min(65536, 300000 // batch)))
    if dtype == "fp32":
        batch = min(batch, 8)
        hi = min(hi, 4096)
        return _case("decode", **common, batch=batch, lo=max(1, hi // 30), hi=hi, heads=rng.choice([4, 12, 16]),
                     d_nope=rng.choice([32, 64, 128]), d_rope=rng.choice([16, 64]), d_c=rng.choice([64, 128, 256]),
                     gate=rng.choice(["mul_ln", "none"]))
    d_c = rng.choice([192, 256, 256, 512])
    return _case("decode", **common, batch=batch, lo=rng.choice([hi, max(1, hi // 30)]), hi=hi, d_c=d_c,
                 d_nope=rng.choice([64, 128, 128]), gate="none" if d_c == 512 else gate)


# ------------------------------------------------------------------ lengths
def _lengths(case):
    r = random.Random(case["lens_seed"])
    return [_log_int(r, case["lo"], case["hi"]) for _ in range(case["batch"])]


def _firsts(case, most):
    """Position of each sequence's first token, up to `most`."""
    r = random.Random(case["lens_seed"] + 1)
    return [_log_int(r, 1, most) if most else 0 for _ in range(case["batch"])]


def _pages(n):
    return (n + PAGE - 1) // PAGE


# ------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _drawer(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(shape, std=1.0, mean=0.0, dtype=torch.float32):
        # drawn in chunks, so that a large tensor needs no second one in fp32
        n = math.prod(shape)
        out = torch.empty(n, dtype=dtype, device=DEV)
        for i in range(0, n, 1 << 26):
            m = min(1 << 26, n - i)
            out[i:i + m] = torch.randn(m, generator=g, device=DEV).mul_(std).add_(mean)
        return out.view(shape)

    return g, normal


def _offsets(lens):
    return _ints([0] + torch.tensor(lens).cumsum(0).tolist())


def _rope_inputs(case, seed):
    _, normal = _drawer(seed)
    lens, H, dn, dr = _lengths(case), case["heads"], case["d_nope"], case["d_rope"]
    total, dq = sum(lens), case["d_nope"] + case["d_rope"]
    # the projections' rows: the queries of all heads, a latent, the shared key
    rows = normal((total, H * dq + 64 + dr), dtype=TYPES[case["dtype"]])
    return dict(lens=lens, total=total, q=rows[:, :H * dq].unflatten(1, (H, dq)), k=rows[:, H * dq + 64:],
                cu=None if case["step"] else _offsets(lens), positions=_ints(_firsts(case, case["far"])))


def _cache_inputs(case, seed):
    """New or cached tokens of every sequence, over the shuffled pages of one pool."""
    g, normal = _drawer(seed)
    lens, dt, dc, dr = _lengths(case), TYPES[case["dtype"]], case["d_c"], case["d_rope"]
    firsts = _firsts(case, case["past"])
    pages = [_pages(f + n) for f, n in zip(firsts, lens)]
    total, width = sum(pages), max(pages)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    held = torch.arange(width, device=DEV) < _ints(pages)[:, None]
    table = torch.zeros((case["batch"], width), dtype=torch.int32, device=DEV)
    table[held] = order
    d = dict(lens=lens, total=sum(lens), num_pages=total, table=table, positions=_ints(firsts),
             cu=None if case["step"] else _offsets(lens))

    def rows(n):
        return dict(c=normal((n, dc), 0.5, dtype=dt), kr=normal((n, dr), dtype=dt),
                    ids=torch.randint(0, 32000, (n,), generator=g, device=DEV, dtype=torch.int32) if case["ids"] else None)

    if case["kind"] == "append":
        d.update(rows(d["total"]))
        d.update(c8_pool=torch.zeros((total, PAGE, dc), dtype=torch.float8_e4m3fn, device=DEV),
                 scale_pool=torch.ones((total, PAGE), device=DEV),
                 kr_pool=torch.zeros((total, PAGE, dr), dtype=dt, device=DEV),
                 id_pool=torch.zeros((total, PAGE), dtype=torch.int32, device=DEV) if case["ids"] else None)
    else:
        p = rows(total * PAGE)
        c8, scale = _quantise(p["c"].float())
        d.update(c8_pool=c8.view(total, PAGE, dc), scale_pool=scale.view(total, PAGE), kr_pool=p["kr"].view(total, PAGE, dr),
                 id_pool=p["ids"].view(total, PAGE) if case["ids"] else None)
    return d


def _decode_inputs(case, seed):
    g, normal = _drawer(seed)
    dt, scale = TYPES[case["dtype"]], 0.5 if case["dtype"] == "bf16" else 1.0
    H, dn, dr, dc, V = (case[k] for k in ("heads", "d_nope", "d_rope", "d_c", "vocab"))
    lens = _lengths(case)
    B, pages = len(lens), [_pages(n) for n in lens]
    total, width = sum(pages), max(pages)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    held = torch.arange(width, device=DEV) < _ints(pages)[:, None]
    table = torch.zeros((B, width), dtype=torch.int32, device=DEV)
    table[held] = order
    n = total * PAGE
    c8 = torch.empty((total, PAGE, dc), dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty((total, PAGE), device=DEV)
    for i in range(0, total, 4096):   # what earlier steps have written
        c8[i:i + 4096], scales[i:i + 4096] = _quantise(normal((min(4096, total - i), PAGE, dc), scale, dtype=dt).float())
    if case["ids"] == "zipf":   # ranks with probability ~ r^-1.1
        cdf = torch.arange(1, V + 1, device=DEV, dtype=torch.float64).pow_(-1.1).cumsum(0)
        u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * cdf[-1]
        ids = torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)
    else:
        ids = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    d = dict(lens=lens, longest=max(lens), num_pages=total, table=table, seq_lens=_ints(lens), c8_pool=c8,
             scale_pool=scales, kr_pool=normal((total, PAGE, dr), dtype=dt), id_pool=ids.view(total, PAGE),
             gate_table=normal((V, dc), 0.1, 1.0, dt), w_uk=normal((H, dn, dc), dc ** -0.5, dtype=dt),
             w_uv=normal((H, dn, dc), dc ** -0.5, dtype=dt), q=normal((B, H, dn + dr), dtype=dt))
    if case["affine"]:
        d.update(gamma=normal((dc,), 0.1, 1.0), beta=normal((dc,), 0.1))
    else:
        d.update(gamma=torch.ones(dc, device=DEV), beta=torch.zeros(dc, device=DEV))
    return d


def _inputs(case, seed):
    return {"rope": _rope_inputs, "append": _cache_inputs, "read": _cache_inputs,
            "decode": _decode_inputs}[case["kind"]](case, seed)


def prepare(case, seed):
    s = dict(_inputs(case, seed), kind=case["kind"], case=case)
    dt = TYPES[case["dtype"]]
    if case["kind"] == "rope":
        s.update(q_out=torch.zeros(s["q"].shape, dtype=dt, device=DEV), k_out=torch.zeros(s["k"].shape, dtype=dt, device=DEV))
    elif case["kind"] == "read":
        s.update(c=torch.zeros((s["total"], case["d_c"]), dtype=dt, device=DEV),
                 kr=torch.zeros((s["total"], case["d_rope"]), dtype=dt, device=DEV),
                 ids=torch.zeros(s["total"], dtype=torch.int32, device=DEV) if case["ids"] else None)
    elif case["kind"] == "decode":
        s["out"] = torch.zeros((case["batch"], case["heads"], case["d_nope"]), dtype=dt, device=DEV)
    return s


# -------------------------------------------------------------- plain forms
def _quantise(x):
    """e4m3 codes and power-of-two scales of rows x (32 bits): the least scale under which 448 holds the row."""
    m, e = torch.frexp(x.abs().amax(-1))   # m in [0.5, 1): 448 is 0.875 2^9
    e = (e - 9 + (m > 0.875)).clamp(min=-100)
    scale, inverse = ((t + 127 << 23).view(torch.float32) for t in (e, -e))   # 2^e and 2^-e, exactly
    return (x * inverse[..., None]).to(torch.float8_e4m3fn), scale


def _sequences(s):
    """Sequence and position of every packed token."""
    k = torch.arange(s["total"], device=DEV)
    if s["cu"] is None:
        return k, s["positions"].long()
    b = torch.searchsorted(s["cu"][1:].contiguous(), k, right=True)
    return b, s["positions"].long()[b] + k - s["cu"].long()[b]


def _plain_rope(s):
    case = s["case"]
    d, theta, factor = case["d_rope"], case["theta"], case["factor"]
    i, magnitude = torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d, 1.0
    if case["scaling"] == "ntk":
        theta = theta * factor ** (d / (d - 2))
    freq = theta ** -i
    if case["scaling"] == "linear":
        freq = freq / factor
    if case["scaling"] == "yarn":
        whole = ((case["original"] * freq / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        freq = freq * (whole + (1 - whole) / factor)
        magnitude = 0.1 * math.log(factor) + 1.0
    angle = _sequences(s)[1].double()[:, None] * freq   # 32 bits lose the angles of far positions
    cos, sin = (magnitude * angle.cos()).float(), (magnitude * angle.sin()).float()
    if case["inverse"]:
        sin = -sin

    def turned(x, c, n):
        x = x.float()
        if case["layout"] == "half":
            a, b = x[..., :d // 2], x[..., d // 2:]
            return torch.cat([a * c - b * n, a * n + b * c], -1)
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2)

    dn = case["d_nope"]
    s["q_out"][..., :dn] = s["q"][..., :dn]
    s["q_out"][..., dn:] = turned(s["q"][..., dn:], cos[:, None], sin[:, None])
    s["k_out"].copy_(turned(s["k"], cos, sin))


def _rows(s):
    """Row of the pool of every packed token."""
    b, pos = _sequences(s)
    return s["table"][b, pos // PAGE].long() * PAGE + pos % PAGE


def _plain_append(s):
    rows = _rows(s)
    c8, scale = _quantise(s["c"].float())
    s["c8_pool"].view(torch.uint8).view(-1, s["case"]["d_c"])[rows] = c8.view(torch.uint8)
    s["scale_pool"].view(-1)[rows] = scale
    s["kr_pool"].view(-1, s["case"]["d_rope"])[rows] = s["kr"]
    if s["ids"] is not None:
        s["id_pool"].view(-1)[rows] = s["ids"]


def _plain_read(s):
    rows = _rows(s)
    c8 = s["c8_pool"].view(torch.uint8).view(-1, s["case"]["d_c"])[rows].view(torch.float8_e4m3fn)
    s["c"].copy_(c8.float() * s["scale_pool"].view(-1)[rows][:, None])
    s["kr"].copy_(s["kr_pool"].view(-1, s["case"]["d_rope"])[rows])
    if s["ids"] is not None:
        s["ids"].copy_(s["id_pool"].view(-1)[rows])


def _plain_decode(s):
    case, t = s["case"], s["table"].long()
    dn, dc, gate = case["d_nope"], case["d_c"], case["gate"]
    B, H = case["batch"], case["heads"]
    z = (s["c8_pool"].view(torch.uint8)[t].view(torch.float8_e4m3fn).float() * s["scale_pool"][t][..., None]).view(B, -1, dc)
    if gate != "none":
        g = s["gate_table"][s["id_pool"][t].long()].view(B, -1, dc).float()
        z = z + g if gate == "add_ln" else z * g
    if gate.endswith("ln"):
        z = z - z.mean(-1, keepdim=True)
        z = z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt()
        z = z * s["gamma"] + s["beta"]
    q, kr = s["q"].float(), s["kr_pool"][t].float().view(B, -1, case["d_rope"])
    p = torch.bmm(torch.einsum("bhd,hdc->bhc", q[..., :dn], s["w_uk"].float()), z.transpose(1, 2))
    p = (p + torch.bmm(q[..., dn:], kr.transpose(1, 2))) * (dn + case["d_rope"]) ** -0.5
    p.masked_fill_((torch.arange(z.shape[1], device=DEV) >= s["seq_lens"][:, None])[:, None], -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp_()
    o = torch.bmm(p, z) / p.sum(-1, keepdim=True)
    s["out"].copy_(torch.einsum("bhc,hdc->bhd", o, s["w_uv"].float()))


# ------------------------------------------------------------ the library's
def _call(s):
    """The library's call on a state; its dims and workspace are made once, as a serving loop does."""
    from paper_2509_16686_gb300 import _lib

    case, kind = s["case"], s["kind"]
    if "dims" not in s:
        gate = case.get("gate", "mul_ln")
        s["dims"] = _lib.make_dims(case.get("heads", 16), case.get("d_nope", 128), case["d_rope"], case.get("d_nope", 128),
                                   case.get("d_c", 256), case.get("vocab", 32000), dtype=case["dtype"],
                                   gate=gate != "none", gate_op="mul_ln" if gate == "none" else gate)
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if kind == "rope":
            s["rope"] = _lib.make_rope(case["layout"], case["scaling"], theta=case["theta"], factor=case["factor"],
                                       original_len=case["original"], inverse=case["inverse"])
        if kind == "decode":
            need = _lib.eg_mla_decode_workspace_size(s["dims"], case["batch"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    if kind == "rope":
        _lib.eg_mla_rope(s["dims"], s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], s["positions"], s["cu"],
                         dev_status=s["status"])
        return
    cache = (s["c8_pool"], s["scale_pool"], s["kr_pool"], s["id_pool"])
    if kind == "append":
        _lib.eg_mla_append_latent_q8(s["dims"], *cache, s["c"], s["kr"], s["ids"], s["table"], s["positions"], s["cu"],
                                     dev_status=s["status"])
    elif kind == "read":
        _lib.eg_mla_read_latent_q8(s["dims"], *cache, s["table"], s["c"], s["kr"], s["ids"], s["positions"], s["cu"],
                                   dev_status=s["status"])
    else:
        _lib.eg_mla_decode_q8(s["dims"], s["q"], *cache, s["table"], s["seq_lens"], s["longest"], s["gate_table"],
                              s["gamma"], s["beta"], s["w_uk"], s["w_uv"], s["out"], s["workspace"],
                              dev_status=s["status"])


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}
_OUTPUTS = {"rope": ("q_out", "k_out"), "append": ("c8_pool", "scale_pool", "kr_pool", "id_pool"),
            "read": ("c", "kr", "ids"), "decode": ("out",)}


def run(s):
    (_call if own else _PLAIN[s["kind"]])(s)
    return {k: s[k] for k in _OUTPUTS[s["kind"]]}


# --------------------------------------------------------------------- work
def _distinct(case, n):
    """The expected number of distinct ids among n tokens."""
    V = case["vocab"]
    if case["ids"] == "zipf":
        total = sum(r ** -1.1 for r in range(1, V + 1))
        return sum(1 - math.exp(-n * r ** -1.1 / total) for r in range(1, V + 1))
    return V * (1 - math.exp(-n / V))


def work(case):
    lens, e, dr = _lengths(case), 2 if case["dtype"] == "bf16" else 4, case["d_rope"]
    T, B = sum(lens), case["batch"]
    if case["kind"] == "rope":
        H, dq = case["heads"], case["d_nope"] + dr
        return {"bytes": 2 * T * (H * dq + dr) * e + 4 * B * (1 if case["step"] else 2), "flops": 3 * T * (H + 1) * dr}
    dc = case["d_c"]
    held = dc + 4 + dr * e   # of a token in the cache, without its id
    if case["kind"] != "decode":
        pages = sum(_pages(f + n) - f // PAGE for f, n in zip(_firsts(case, case["past"]), lens))
        return {"bytes": T * (held + (dc + dr) * e + (8 if case["ids"] else 0)) + 4 * (pages + B * (1 if case["step"] else 2)),
                "flops": 2 * T * dc}
    H, dn, gated = case["heads"], case["d_nope"], case["gate"] != "none"
    cache = T * (held + (4 if gated else 0)) + (int(_distinct(case, T)) * dc * e if gated else 0)
    return {"bytes": cache + 4 * (sum(_pages(n) for n in lens) + B) + 2 * H * dn * dc * e + B * H * (2 * dn + dr) * e,
            "flops": 2 * H * (2 * dc + dr) * T + 4 * B * H * dn * dc}


# -------------------------------------------------------------------- exact
def _packed64(d):
    """(sequence, position) of every packed token, from the lengths."""
    first = d["positions"].tolist()
    b = torch.repeat_interleave(torch.arange(len(d["lens"])), torch.tensor(d["lens"]))
    pos = torch.cat([torch.arange(f, f + n) for f, n in zip(first, d["lens"])])
    return b.to(DEV), pos.to(DEV)


def _exact_rope(case, d):
    dr, pos, m = case["d_rope"], _packed64(d)[1].double(), 1.0
    base = case["theta"] * (case["factor"] ** (dr / (dr - 2)) if case["scaling"] == "ntk" else 1.0)
    rates = []
    for i in range(dr // 2):
        f = math.exp(-2 * i / dr * math.log(base))
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "yarn":
            turns = case["original"] * f / (2 * math.pi)
            kept = min(1.0, max(0.0, (turns - 1) / 31))
            f = (1 - kept) * f / case["factor"] + kept * f
        rates.append(f)
    if case["scaling"] == "yarn":
        m = 1 + math.log(case["factor"]) / 10
    phi = pos[:, None] * torch.tensor(rates, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(phi, m), -phi if case["inverse"] else phi)
    out = {}
    for name, x in (("q_out", d["q"][..., case["d_nope"]:]), ("k_out", d["k"][:, None])):
        x = x.double()
        x = x.unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else x.unflatten(-1, (-1, 2))
        y = torch.view_as_real(torch.view_as_complex(x.contiguous()) * turn[:, None])
        out[name] = (y.transpose(-1, -2) if case["layout"] == "half" else y).flatten(-2)
    return {"q_out": torch.cat([d["q"][..., :case["d_nope"]].double(), out["q_out"]], -1), "k_out": out["k_out"][:, 0]}


def _exact_append(case, d):
    """Codes as the nearest points of e4m3's grid, found in 64 bits."""
    b, pos = _packed64(d)
    row = d["table"][b, pos // PAGE].long() * PAGE + pos % PAGE
    c = d["c"].double()

    def power(e):
        return (e.long() + 1023 << 52).view(torch.float64)

    m, e = torch.frexp(c.abs().amax(-1) / 448)
    scale = power((e - (m == 0.5).int()).clamp(min=-100))
    y = c / scale[:, None]
    step = power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)   # three bits behind the first
    out = {"c8_pool": torch.zeros(d["c8_pool"].shape, dtype=torch.float64, device=DEV),
           "scale_pool": torch.ones(d["scale_pool"].shape, dtype=torch.float64, device=DEV),
           "kr_pool": torch.zeros(d["kr_pool"].shape, dtype=torch.float64, device=DEV), "id_pool": None}
    out["c8_pool"].view(-1, case["d_c"])[row] = (y / step).round() * step
    out["scale_pool"].view(-1)[row] = scale
    out["kr_pool"].view(-1, case["d_rope"])[row] = d["kr"].double()
    return out


def _values64(d, rows):
    c8 = d["c8_pool"].view(torch.uint8).view(-1, d["c8_pool"].shape[-1])[rows].view(torch.float8_e4m3fn)
    return c8.double() * d["scale_pool"].view(-1)[rows].double()[:, None]


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(case, d)
    if case["kind"] == "append":
        return _exact_append(case, d)
    if case["kind"] == "read":
        b, pos = _packed64(d)
        row = d["table"][b, pos // PAGE].long() * PAGE + pos % PAGE
        return {"c": _values64(d, row), "kr": d["kr_pool"].view(-1, case["d_rope"])[row].double(), "ids": None}
    H, dn, dr, dc, gate = (case[k] for k in ("heads", "d_nope", "d_rope", "d_c", "gate"))
    q, w_uk, w_uv = d["q"].double(), d["w_uk"].double(), d["w_uv"].double()
    u = torch.zeros((case["batch"], H, dn), dtype=torch.float64, device=DEV)
    for b, n in enumerate(d["lens"]):
        rows = (d["table"][b, :_pages(n)].long()[:, None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(-1)[:n]
        z = _values64(d, rows)
        if gate != "none":
            g = d["gate_table"][d["id_pool"].view(-1)[rows].long()].double()
            z = z + g if gate == "add_ln" else z * g
            if gate != "mul":
                mu = z.sum(-1, keepdim=True) / dc
                var = ((z - mu) ** 2).sum(-1, keepdim=True) / dc
                z = (z - mu) / torch.sqrt(var + 1e-5) * d["gamma"].double() + d["beta"].double()
        qa = torch.einsum("hd,hdc->hc", q[b, :, :dn], w_uk)
        kr = d["kr_pool"].view(-1, dr)[rows].double()
        p = ((qa @ z.T + q[b, :, dn:] @ kr.T) / math.sqrt(dn + dr)).softmax(-1)
        u[b] = torch.einsum("hc,hdc->hd", p @ z, w_uv)
    return {"out": u}
