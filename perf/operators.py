"""What a serving loop needs around the latent decode: plain forms and the library's calls.

A case is a dict of plain values; ``kind`` names the operator:

  plan     eg_mla_page_plan: pages, block table and slot map of a step's new
           tokens, from the lengths of its requests
  shared   eg_mla_decode_shared: one decode step of sequences that share a
           prefix, the prefix computed once for all of them
  summary  eg_mla_page_summary: the mean key of every page that became full
  sparse   eg_mla_decode_sparse: one decode step over the pages of each
           sequence whose mean keys score best

Lengths are part of the case (drawn from ``lens_seed``), everything else is
drawn on the GPU from the seed of the state.  Value distributions are those of
the library's synthetic workloads (latents 0.5 N(0, 1), gate table N(1, 0.1),
weights N(0, d_c^-1/2)); in the sparse cases the RoPE keys of a page share a
direction with the query to a degree of the page's own (exponentially
distributed), as the pages of a long text that matter to a query are few.
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 64


def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", gate="mul_ln", batch=1, lo=1, hi=1, lens_seed=0, heads=16, d_nope=128, d_rope=64,
             d_c=256, vocab=32000, ids="uniform", affine=True)
    if kind == "plan":
        c = dict(kind=kind, batch=1, lo=1, hi=1, lens_seed=0, prompts=0.0, longest=1, leaving=0.0, scarce=False)
    elif kind == "shared":
        c["prefix"] = 0
    elif kind == "summary":
        c.update(new=0, full=0.0)
    else:
        c.update(budget=0, first=1, last=2)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step's pages: 64 sequences, a token each
        _case("plan", name="plan_decode", batch=64, lo=60, hi=8192, lens_seed=1),
        # a busy server's step: 1024 sequences, one in sixteen a new prompt, as many leaving
        _case("plan", name="plan_mixed", batch=1024, lo=1, hi=8192, lens_seed=2, prompts=0.06, longest=8192,
              leaving=0.06),
        # a few chats under one system prompt: latency
        _case("shared", name="shared_small", batch=8, prefix=2048, lo=1, hi=300, lens_seed=3),
        # a document of 32K tokens asked about by 64 sequences
        _case("shared", name="shared_32k", batch=64, prefix=32768, lo=128, hi=1024, lens_seed=4, affine=False),
        # an odd prefix, ragged sequences, Zipf ids, the narrower latent
        _case("shared", name="shared_ragged", batch=37, prefix=10007, lo=1, hi=3000, lens_seed=5, d_c=192,
              vocab=50000, ids="zipf"),
        # sampling from one prompt, the model without a gate
        _case("shared", name="shared_plain", batch=128, prefix=8191, lo=1, hi=256, lens_seed=6, gate="none"),
        # the pages that a decode step of 64 sequences completed (a quarter of them one)
        _case("summary", name="summary_step", batch=64, lo=128, hi=8192, lens_seed=7, new=1, full=0.25),
        # all pages of eight long prompts
        _case("summary", name="summary_prompts", batch=8, lo=32768, hi=32768, lens_seed=8, new=32768, affine=False),
        # a few sequences, 32 pages of each
        _case("sparse", name="sparse_8k", batch=4, lo=2000, hi=8192, lens_seed=9, budget=32),
        # 32 sequences of 32K tokens, an eighth of the pages
        _case("sparse", name="sparse_32k", batch=32, lo=32768, hi=32768, lens_seed=10, budget=64, affine=False),
        # the plain MLA model, ragged, short sequences whole
        _case("sparse", name="sparse_mla", batch=64, lo=1000, hi=16384, lens_seed=11, gate="none", d_c=512, budget=48),
        # single precision, the setting of a numerical check
        _case("sparse", name="sparse_fp32", dtype="fp32", batch=4, lo=1500, hi=4000, lens_seed=12, budget=16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["plan", "shared", "shared", "summary", "sparse", "sparse"])
    common = dict(lens_seed=rng.randrange(1 << 20))
    if kind == "plan":
        batch, hi = _log_int(rng, 1, 4096), _log_int(rng, 64, 8192)
        return _case("plan", **common, batch=batch, lo=max(1, hi // 128), hi=hi, prompts=rng.choice([0.0, 0.05, 0.3]),
                     longest=_log_int(rng, 16, min(8192, 500000 // batch + 16)), leaving=rng.choice([0.0, 0.1]),
                     scarce=rng.random() < 0.3)
    common.update(ids=rng.choice(["uniform", "zipf"]), affine=rng.random() < 0.5, vocab=_log_int(rng, 1000, 50000))
    gate = rng.choice(["mul_ln", "mul_ln", "mul_ln", "mul", "add_ln", "none"])
    if kind == "shared":
        batch = _log_int(rng, 1, 128)
        hi = _log_int(rng, 1, 1 + 100000 // batch)
        return _case("shared", **common, batch=batch, prefix=_log_int(rng, 1, min(65536, 2000000 // batch)),
                     lo=rng.choice([hi, max(1, hi // 100)]), hi=hi, d_c=rng.choice([192, 256]), gate=gate,
                     d_nope=rng.choice([64, 128, 128]))
    if kind == "summary":
        batch = _log_int(rng, 1, 128)
        hi = _log_int(rng, 16, max(16, min(32768, 250000 // batch)))
        return _case("summary", **common, batch=batch, lo=rng.choice([hi, max(1, hi // 30)]), hi=hi,
                     new=_log_int(rng, 1, hi), full=rng.choice([0.0, 0.25, 1.0]), d_c=rng.choice([192, 256]), gate=gate)
    batch = _log_int(rng, 1, 64)
    hi = _log_int(rng, 100, min(32768, 1000000 // batch))
    shape = rng.choice(["gated", "gated", "mla", "fp32"])
    budget = _log_int(rng, 4, 128)
    if shape == "fp32":
        batch = min(batch, 8)
        hi = min(hi, 4096)
        return _case("sparse", **common, dtype="fp32", batch=batch, lo=max(1, hi // 3), hi=hi,
                     heads=rng.choice([4, 12, 16]), d_nope=rng.choice([32, 64, 128]), d_rope=rng.choice([16, 64]),
                     d_c=rng.choice([64, 128, 256]), gate=rng.choice(["mul_ln", "none"]), budget=min(budget, 32))
    return _case("sparse", **common, batch=batch, lo=rng.choice([hi, max(1, hi // 30)]), hi=hi, budget=budget,
                 first=rng.choice([0, 1, 2]), last=rng.choice([1, 2]), d_c=512 if shape == "mla" else rng.choice([192, 256]),
                 gate="none" if shape == "mla" else gate)


# ------------------------------------------------------------------ lengths
def _lengths(case):
    r = random.Random(case["lens_seed"])
    return [_log_int(r, case["lo"], case["hi"]) for _ in range(case["batch"])]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _requests(case):
    """Lengths and new tokens of a plan: -1 leaves, a prompt starts from nothing, the others grow by a token."""
    r = random.Random(case["lens_seed"] + 1)
    lens, new = _lengths(case), []
    for b in range(len(lens)):
        x = r.random()
        if x < case["prompts"]:
            lens[b] = 0
            new.append(_log_int(r, 1, case["longest"]))
        else:
            new.append(-1 if x < case["prompts"] + case["leaving"] else 1)
    return lens, new


def _full_lengths(case):
    """Lengths of a summary case: a share `full` of the sequences ends at a page's end."""
    r = random.Random(case["lens_seed"] + 1)
    return [_pages(n) * PAGE if r.random() < case["full"] else n for n in _lengths(case)]


# ------------------------------------------------------------------- inputs
def _plan_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    lens, new = _requests(case)
    have = [_pages(n) for n in lens]
    need = [_pages(n + max(t, 0)) - h for n, t, h in zip(lens, new, have)]
    width = max(1, max(h + n for h, n in zip(have, need)))
    free = sum(need) // 2 if case["scarce"] else sum(need) + 64
    num_pages = sum(have) + free
    order = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    have_t = torch.tensor(have, device=DEV)
    held = torch.arange(width, device=DEV) < have_t[:, None]
    table = torch.zeros((len(lens), width), dtype=torch.int32, device=DEV)
    table[held] = order[:sum(have)]
    stack = torch.zeros(num_pages, dtype=torch.int32, device=DEV)
    stack[:free] = order[sum(have):]
    return dict(block_table=table, free_pages=stack, num_pages=num_pages,
                seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                new_tokens=torch.tensor(new, dtype=torch.int32, device=DEV),
                free_count=torch.tensor([free], dtype=torch.int32, device=DEV),
                capacity=max(1, sum(max(t, 0) for t in new)))


def _inputs(case, seed):
    """Everything an attention or summary call reads, on the GPU, from the seed."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    scale = 0.5 if case["dtype"] == "bf16" else 1.0
    H, dn, dr, dc, V = (case[k] for k in ("heads", "d_nope", "d_rope", "d_c", "vocab"))

    def normal(shape, std=1.0, mean=0.0, dtype=dt):
        # drawn in chunks, so that a large tensor needs no second one in fp32
        n = math.prod(shape)
        out = torch.empty(n, dtype=dtype, device=DEV)
        for i in range(0, n, 1 << 26):
            m = min(1 << 26, n - i)
            out[i:i + m] = torch.randn(m, generator=g, device=DEV).mul_(std).add_(mean)
        return out.view(shape)

    def token_ids(n):
        if case["ids"] == "zipf":   # ranks with probability ~ r^-1.1
            cdf = torch.arange(1, V + 1, device=DEV, dtype=torch.float64).pow_(-1.1).cumsum(0)
            u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * cdf[-1]
            return torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)
        return torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)

    lens = _full_lengths(case) if case["kind"] == "summary" else _lengths(case)
    B = len(lens)
    pages = [_pages(n) for n in lens]
    prefix = _pages(case.get("prefix", 0))
    total, width = sum(pages) + prefix, max(pages)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    held = torch.arange(width, device=DEV) < torch.tensor(pages, device=DEV)[:, None]
    table = torch.zeros((B, width), dtype=torch.int32, device=DEV)
    table[held] = order[prefix:]
    d = dict(lens=lens, longest=max(lens), num_pages=total, block_table=table,
             seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             c_pool=normal((total, PAGE, dc), scale), kr_pool=normal((total, PAGE, dr)),
             id_pool=token_ids(total * PAGE).view(total, PAGE), gate_table=normal((V, dc), 0.1, 1.0))
    if case["affine"]:
        d.update(gamma=normal((dc,), 0.1, 1.0, torch.float32), beta=normal((dc,), 0.1, 0.0, torch.float32))
    else:
        d.update(gamma=torch.ones(dc, device=DEV), beta=torch.zeros(dc, device=DEV))
    if case["kind"] == "summary":
        d["new_tokens"] = d["seq_lens"].clamp(max=case["new"])
        return d
    d.update(w_uk=normal((H, dn, dc), dc ** -0.5), w_uv=normal((H, dn, dc), dc ** -0.5), q=normal((B, H, dn + dr)))
    if case["kind"] == "shared":
        d.update(prefix_table=order[:prefix].contiguous(),
                 prefix_len=torch.tensor([case["prefix"]], dtype=torch.int32, device=DEV))
        return d
    # the pages' degrees of relevance, along a direction of each sequence
    e = torch.nn.functional.normalize(torch.randn((B, dr), generator=g, device=DEV), dim=-1)
    rel = torch.empty((B, width), device=DEV).exponential_(1.0, generator=g)
    d["q"][..., dn:] += (1.5 * math.sqrt(dn + dr) * e)[:, None].to(dt)
    d["kr_pool"][table[held].long()] += (rel[..., None] * e[:, None])[held][:, None].to(dt)
    return d


def prepare(case, seed):
    if case["kind"] == "plan":
        s = dict(_plan_inputs(case, seed), kind="plan", case=case)
        B = case["batch"]
        s.update(seq_lens_out=torch.zeros(B, dtype=torch.int32, device=DEV),
                 free_count_out=torch.zeros(1, dtype=torch.int32, device=DEV),
                 positions=torch.zeros(B, dtype=torch.int32, device=DEV),
                 cu_seqlens=torch.zeros(B + 1, dtype=torch.int32, device=DEV),
                 slots=torch.zeros(s["capacity"], dtype=torch.int32, device=DEV))
        return s
    s = dict(_inputs(case, seed), kind=case["kind"], case=case)
    H, dn, dc, dr = (case[k] for k in ("heads", "d_nope", "d_c", "d_rope"))
    if case["kind"] == "summary":
        s["summary"] = torch.zeros((s["num_pages"], dc + dr), device=DEV)
        return s
    s["out"] = torch.zeros((case["batch"], H, dn), dtype=s["q"].dtype, device=DEV)
    if case["kind"] == "sparse":   # what earlier steps have left: the mean keys of the full pages
        s["summary"] = torch.zeros((s["num_pages"], dc + dr), device=DEV)
        _plain_summary(dict(s, new_tokens=s["seq_lens"]))
    return s


# -------------------------------------------------------------- plain forms
def _plain_plan(s):
    table, stack = s["block_table"], s["free_pages"]
    B, width = table.shape
    length, n, free = s["seq_lens"].long(), s["new_tokens"].long(), s["free_count"].long()
    col = torch.arange(width, device=DEV)
    have, ask, leaves = (length + PAGE - 1) // PAGE, n.clamp(min=0), n < 0
    fits = length + ask <= width * PAGE
    need = torch.where(fits, (length + ask + PAGE - 1) // PAGE - have, 0)
    # released pages onto the stack, in the order of the batch
    back = torch.where(leaves, have, 0)
    at = free + (back.cumsum(0) - back)[:, None] + col
    gone = col < back[:, None]
    stack[at[gone]] = table[gone]
    # new pages from its top, first come first served
    avail = free + back.sum()
    before = need.cumsum(0) - need
    granted = fits & ~leaves & ((need == 0) | (before + need <= avail))
    take = torch.where(granted, need, 0)
    fresh = (col >= have[:, None]) & (col < (have + take)[:, None])
    at = avail - 1 - (before - have)[:, None] - col
    table[fresh] = stack[at[fresh]]
    t = torch.where(granted, ask, 0)
    s["seq_lens_out"].copy_(torch.where(leaves, 0, length + t))
    s["free_count_out"].copy_(avail - take.sum())
    s["positions"].copy_(torch.where(t > 0, length, -1))
    s["cu_seqlens"][1:] = t.cumsum(0)
    s["cu_seqlens"][0] = 0
    k = torch.arange(s["slots"].shape[0], device=DEV)
    b = torch.searchsorted(s["cu_seqlens"][1:].contiguous(), k, right=True).clamp(max=B - 1)
    pos = (length[b] + k - s["cu_seqlens"][b]).clamp(0, width * PAGE - 1)
    slot = table[b, pos // PAGE].long() * PAGE + pos % PAGE
    s["slots"].copy_(torch.where(k < s["cu_seqlens"][B], slot, -1))


def _plain_gate(s, c, ids):
    """The latents c (32 bits) under the gate, normalised where the mode says so."""
    gate = s["case"]["gate"]
    if gate == "none":
        return c
    g = s["gate_table"][ids.long()].float()
    if gate == "mul":
        return c * g
    z = c + g if gate == "add_ln" else c * g
    z = z - z.mean(-1, keepdim=True)
    z = z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    return z * s["gamma"] + s["beta"]


def _plain_keys(s, pages):
    """Keys [c~ ; k^R] of whole pages (any shape of page ids), in 32 bits."""
    p = pages.long()
    return torch.cat([_plain_gate(s, s["c_pool"][p].float(), s["id_pool"][p]), s["kr_pool"][p].float()], -1)


def _plain_summary(s):
    table, length = s["block_table"], s["seq_lens"].long()
    col = torch.arange(table.shape[1], device=DEV)
    first = (length - s["new_tokens"].long()) // PAGE
    pages = table[(col >= first[:, None]) & (col < (length // PAGE)[:, None])].long()
    s["summary"][pages] = _plain_keys(s, pages).mean(1)


def _plain_queries(s):
    """[q^ ; q^R] of every head, in 32 bits: W_UK absorbed."""
    dn = s["case"]["d_nope"]
    q = s["q"].float()
    return torch.cat([torch.einsum("bhd,hdc->bhc", q[..., :dn], s["w_uk"].float()), q[..., dn:]], -1)


def _plain_values(s, o):
    s["out"].copy_(torch.einsum("bhc,hdc->bhd", o, s["w_uv"].float()))


def _plain_shared(s):
    case = s["case"]
    dc, scale = case["d_c"], (case["d_nope"] + case["d_rope"]) ** -0.5
    q = _plain_queries(s) * scale
    B, H, D = q.shape
    kp = _plain_keys(s, s["prefix_table"]).reshape(-1, D)[:case["prefix"]]
    ko = _plain_keys(s, s["block_table"]).reshape(B, -1, D)
    sp = (q.reshape(B * H, D) @ kp.T).view(B, H, -1)
    so = torch.bmm(q, ko.transpose(1, 2))
    so.masked_fill_((torch.arange(ko.shape[1], device=DEV) >= s["seq_lens"][:, None])[:, None], -math.inf)
    top = torch.maximum(sp.amax(-1), so.amax(-1))[..., None]
    sp, so = (sp - top).exp_(), (so - top).exp_()
    o = (sp.view(B * H, -1) @ kp[:, :dc]).view(B, H, dc) + torch.bmm(so, ko[..., :dc])
    _plain_values(s, o / (sp.sum(-1) + so.sum(-1))[..., None])


def _plain_sparse(s):
    case = s["case"]
    dc, scale = case["d_c"], (case["d_nope"] + case["d_rope"]) ** -0.5
    q = _plain_queries(s) * scale
    B, H, D = q.shape
    table, count = s["block_table"], ((s["seq_lens"].long() + PAGE - 1) // PAGE)[:, None]
    col = torch.arange(table.shape[1], device=DEV)
    score = torch.bmm(q, s["summary"][table.long()].transpose(1, 2)).amax(1)
    score.masked_fill_((col < case["first"]) | (col >= count - case["last"]), math.inf)
    score.masked_fill_(col >= count, -math.inf)
    # the best pages, the lowest of equal ones first
    pages = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :case["budget"]]
    k = _plain_keys(s, table.gather(1, pages)).reshape(B, -1, D)
    pos = (pages[..., None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(B, 1, -1)
    p = torch.bmm(q, k.transpose(1, 2)).masked_fill_(pos >= s["seq_lens"][:, None, None], -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp_()
    _plain_values(s, torch.bmm(p, k[..., :dc]) / p.sum(-1, keepdim=True))


# ------------------------------------------------------------ the library's
def _call(s):
    """The library's call on a state; its dims and workspace are made once, as a serving loop does."""
    from paper_2509_16686_gb300 import _lib

    case, kind = s["case"], s["kind"]
    if kind == "plan":
        if "status" not in s:
            s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        _lib.eg_mla_page_plan(s["new_tokens"], s["seq_lens"], s["seq_lens_out"], s["block_table"], s["free_pages"],
                              s["free_count"], s["free_count_out"], s["cu_seqlens"], s["positions"], s["slots"],
                              dev_status=s["status"])
        return
    if "dims" not in s:
        gated = case["gate"] != "none"
        s["dims"] = _lib.make_dims(case["heads"], case["d_nope"], case["d_rope"], case["d_nope"], case["d_c"],
                                   case["vocab"], dtype=case["dtype"], gate=gated,
                                   gate_op=case["gate"] if gated else "mul_ln")
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        need = 0
        if kind == "shared":
            need = _lib.eg_mla_decode_shared_workspace_size(s["dims"], case["batch"], case["prefix"])
        elif kind == "sparse":
            need = _lib.eg_mla_decode_sparse_workspace_size(s["dims"], case["batch"], s["block_table"].shape[1],
                                                            case["budget"])
        s["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device=DEV)
    cache = (s["c_pool"], s["kr_pool"], s["id_pool"])
    gate = (s["gate_table"], s["gamma"], s["beta"])
    if kind == "summary":
        _lib.eg_mla_page_summary(s["dims"], *cache, s["block_table"], s["seq_lens"], s["longest"], *gate, s["summary"],
                                 new_tokens=s["new_tokens"], max_new_tokens=min(case["new"], s["longest"]),
                                 dev_status=s["status"])
    elif kind == "shared":
        _lib.eg_mla_decode_shared(s["dims"], s["q"], *cache, s["prefix_table"], s["prefix_len"], case["prefix"],
                                  s["block_table"], s["seq_lens"], s["longest"], *gate, s["w_uk"], s["w_uv"],
                                  s["out"], s["workspace"], dev_status=s["status"])
    else:
        _lib.eg_mla_decode_sparse(s["dims"], s["q"], *cache, s["block_table"], s["seq_lens"], s["longest"],
                                  s["summary"], case["budget"], case["first"], case["last"], *gate, s["w_uk"],
                                  s["w_uv"], s["out"], s["workspace"], dev_status=s["status"])


_PLAIN = {"plan": _plain_plan, "shared": _plain_shared, "summary": _plain_summary, "sparse": _plain_sparse}
_OUTPUTS = {"plan": ("seq_lens_out", "block_table", "free_pages", "free_count_out", "cu_seqlens", "positions", "slots"),
            "shared": ("out",), "summary": ("summary",), "sparse": ("out",)}


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
    if case["kind"] == "plan":
        lens, new = _requests(case)
        tokens = sum(max(t, 0) for t in new)
        # per sequence two values in and three out, a page granted or released from one list to the
        # other, the page that a new token starts in, a slot per token
        moved = sum(_pages(n + t) - _pages(n) if t > 0 else _pages(n) if t < 0 else 0 for n, t in zip(lens, new))
        started = sum(1 for n, t in zip(lens, new) if t > 0 and n % PAGE)
        return {"bytes": 4 * (5 * len(lens) + 2 * moved + started + tokens + 3), "flops": 0}
    H, dn, dr, dc = (case[k] for k in ("heads", "d_nope", "d_rope", "d_c"))
    e = 2 if case["dtype"] == "bf16" else 4
    gated = case["gate"] != "none"

    def cache(n):
        return n * ((dc + dr) * e + (4 if gated else 0)) + (int(_distinct(case, n)) * dc * e if gated else 0)

    if case["kind"] == "summary":
        pages = sum(n // PAGE - (n - min(n, case["new"])) // PAGE for n in _full_lengths(case))
        return {"bytes": cache(pages * PAGE) + pages * (4 + (dc + dr) * 4) + 8 * case["batch"],
                "flops": pages * PAGE * (8 * dc + dr)}
    lens = _lengths(case)
    B = len(lens)
    fixed = 2 * H * dn * dc * e + B * H * (2 * dn + dr) * e
    ends = 4 * B * H * dc * dn
    if case["kind"] == "shared":
        T = case["prefix"]
        return {"bytes": cache(T + sum(lens)) + 4 * (_pages(T) + sum(_pages(n) for n in lens)) + fixed,
                "flops": 2 * H * (2 * dc + dr) * (B * T + sum(lens)) + ends}
    # pages that can be left out are ranked by their mean keys
    ranked = sum(_pages(n) - case["first"] - case["last"] for n in lens if _pages(n) > case["budget"])
    tokens = sum(min(n, case["budget"] * PAGE) for n in lens)
    return {"bytes": cache(tokens) + ranked * (4 + (dc + dr) * 4) + fixed,
            "flops": 2 * H * (2 * dc + dr) * tokens + 2 * H * (dc + dr) * ranked + ends}


# -------------------------------------------------------------------- exact
def _latent64(case, d, rows):
    """c~ of rows of the cache, in 64 bits."""
    c, dc = d["c_pool"].view(-1, case["d_c"])[rows].double(), case["d_c"]
    if case["gate"] == "none":
        return c
    g = d["gate_table"][d["id_pool"].view(-1)[rows].long()].double()
    x = c + g if case["gate"] == "add_ln" else c * g
    if case["gate"] == "mul":
        return x
    mu = x.sum(-1, keepdim=True) / dc
    var = ((x - mu) ** 2).sum(-1, keepdim=True) / dc
    return (x - mu) / torch.sqrt(var + 1e-5) * d["gamma"].double() + d["beta"].double()


def _rows64(pages, n):
    return (pages.long()[:, None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(-1)[:n]


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":   # whole numbers
        return None
    d = _inputs(case, seed)
    H, dn, dr, dc = (case[k] for k in ("heads", "d_nope", "d_rope", "d_c"))
    kr_pool = d["kr_pool"].view(-1, dr)
    if kind == "summary":
        out = torch.zeros((d["num_pages"], dc + dr), dtype=torch.float64, device=DEV)
        for b, n in enumerate(d["lens"]):
            for p in d["block_table"][b, (n - min(n, case["new"])) // PAGE:n // PAGE].split(1024):
                rows = _rows64(p, None)
                keys = torch.cat([_latent64(case, d, rows), kr_pool[rows].double()], -1)
                out[p.long()] = keys.view(len(p), PAGE, dc + dr).sum(1) / PAGE
        return {"summary": out}
    scale = 1 / math.sqrt(dn + dr)
    q, w_uk, w_uv = d["q"].double(), d["w_uk"].double(), d["w_uv"].double()
    u = torch.zeros((case["batch"], H, dn), dtype=torch.float64, device=DEV)
    if kind == "shared":
        # each head's own keys and values of every token, without absorption
        rows = _rows64(d["prefix_table"], case["prefix"])
        zp, rp = _latent64(case, d, rows), kr_pool[rows].double()
        mine = [_rows64(d["block_table"][b, :_pages(n)], n) for b, n in enumerate(d["lens"])]
        own_z = [_latent64(case, d, r) for r in mine]
        own_r = [kr_pool[r].double() for r in mine]
        for h in range(H):
            kp, vp = torch.cat([zp @ w_uk[h].T, rp], -1), zp @ w_uv[h].T
            sp = q[:, h] @ kp.T * scale
            for b in range(case["batch"]):
                k = torch.cat([own_z[b] @ w_uk[h].T, own_r[b]], -1)
                p = torch.cat([sp[b], k @ q[b, h] * scale]).softmax(0)
                u[b, h] = p[:case["prefix"]] @ vp + p[case["prefix"]:] @ own_z[b] @ w_uv[h].T
        return {"out": u}
    for b, n in enumerate(d["lens"]):
        table = d["block_table"][b, :_pages(n)]
        qa = torch.einsum("hd,hdc->hc", q[b, :, :dn], w_uk)
        keep = torch.arange(len(table), device=DEV)
        if len(table) > case["budget"]:
            best = torch.full((len(table),), math.inf, dtype=torch.float64, device=DEV)
            middle = table[case["first"]:len(table) - case["last"]]
            rows = _rows64(middle, None)
            keys = torch.cat([_latent64(case, d, rows), kr_pool[rows].double()], -1).view(len(middle), PAGE, dc + dr).mean(1)
            best[case["first"]:len(table) - case["last"]] = \
                ((qa @ keys[:, :dc].T + q[b, :, dn:] @ keys[:, dc:].T) * scale).max(0)[0]
            keep = best.sort(descending=True, stable=True)[1][:case["budget"]].sort()[0]
        rows = (table[keep].long()[:, None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(-1)
        pos = (keep[:, None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(-1)
        rows = rows[pos < n]
        z = _latent64(case, d, rows)
        p = ((qa @ z.T + q[b, :, dn:] @ kr_pool[rows].double().T) * scale).softmax(-1)
        u[b] = torch.einsum("hc,hdc->hd", p @ z, w_uv)
    return {"out": u}
