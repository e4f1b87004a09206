"""A small serving loop on a cache that holds the latent in 8 bits, on synthetic inputs.

Prompts are planned, rotated, prefilled and written into the cache in 8 bits; each step
then plans a token for every sequence, rotates its query and key, writes it and decodes
over the cache.  Beside it a bf16 cache takes the same tokens unrounded, and at the end the
8-bit cache's values are read back into another: the decode over them has the same result
within its bounds.

    python examples/serve_q8.py [--prompts 300 70 64 1] [--steps 5]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_16686_gb300 import _lib  # noqa: E402

PAGE, HEADS, D_NOPE, D_ROPE, D_C, VOCAB = 64, 16, 128, 64, 256, 1000
BF16 = torch.bfloat16


def pages_of(n):
    return (n + PAGE - 1) // PAGE


def zeros(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def scratch(n):
    return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")


def main(prompts=(300, 70, 64, 1), steps=5, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mean).to(BF16)

    B = len(prompts)
    width = max(pages_of(n + steps) for n in prompts)
    pages = sum(pages_of(n + steps) for n in prompts)
    # positions four times as far as trained: YaRN's temperature over the whole score, of which rope turns a part
    temperature = (0.1 * math.log(4.0) + 1.0) ** 2
    dims = _lib.make_dims(HEADS, D_NOPE, D_ROPE, D_NOPE, D_C, VOCAB, softmax_scale=temperature * (D_NOPE + D_ROPE) ** -0.5)
    rope = _lib.make_rope(scaling="yarn", factor=4.0, original_len=4096, magnitude=1.0)
    gate = (normal(VOCAB, D_C, std=0.1, mean=1.0), torch.ones(D_C, device="cuda"), torch.zeros(D_C, device="cuda"))
    weights = [normal(HEADS, D_NOPE, D_C, std=D_C ** -0.5) for _ in range(2)]
    c8 = zeros(pages, PAGE, D_C, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale, kr_pool, id_pool = zeros(pages, PAGE, dtype=torch.float32), zeros(pages, PAGE, D_ROPE, dtype=BF16), zeros(pages, PAGE)
    cache = (c8, scale, kr_pool, id_pool)
    unrounded = zeros(pages, PAGE, D_C, dtype=BF16)   # (it shares the keys and ids)
    lens, table, status = zeros(B), zeros(B, width), zeros(1)
    free, count = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0), torch.full((1,), pages, dtype=torch.int32, device="cuda")
    cu, positions = zeros(B + 1), zeros(B)

    def plan(new):
        _lib.eg_mla_page_plan(torch.tensor(new, dtype=torch.int32, device="cuda"), lens, lens, table, free, count, count,
                              cu, positions, dev_status=status)

    def tokens(n):
        """Synthetic latents and ids, and rotated queries and keys, of n packed tokens of the planned step."""
        rows = normal(n, HEADS * (D_NOPE + D_ROPE) + D_ROPE)   # the projections' output
        q, k = rows[:, :-D_ROPE].unflatten(1, (HEADS, D_NOPE + D_ROPE)), rows[:, -D_ROPE:]
        q_out, k_out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty((n, D_ROPE), dtype=BF16, device="cuda")
        _lib.eg_mla_rope(dims, rope, q, q_out, k, k_out, positions, cu, dev_status=status)
        ids = torch.randint(0, VOCAB, (n,), generator=gen, device="cuda", dtype=torch.int32)
        return normal(n, D_C, std=0.5), k_out, ids, q_out

    total = sum(prompts)
    plan(prompts)
    c, kr, ids, q = tokens(total)
    u = torch.empty((total, HEADS, D_NOPE), dtype=BF16, device="cuda")
    ws = scratch(_lib.eg_mla_prefill_workspace_size(dims, B, total))
    _lib.eg_mla_prefill(dims, q, c, kr, ids, cu, max(prompts), *gate, *weights, u, ws, unrounded, kr_pool, id_pool, table,
                        dev_status=status)
    _lib.eg_mla_append_latent_q8(dims, *cache, c, kr, ids, table, positions, cu, dev_status=status)

    out = torch.empty((B, HEADS, D_NOPE), dtype=BF16, device="cuda")
    ws = scratch(_lib.eg_mla_decode_workspace_size(dims, B))
    for step in range(steps):
        plan([1] * B)
        c, kr, ids, q = tokens(B)
        _lib.eg_mla_append_latent_q8(dims, *cache, c, kr, ids, table, positions, dev_status=status)
        _lib.eg_mla_append_latent(dims, unrounded, kr_pool, id_pool, c, kr, ids, table, positions, status)
        longest = max(prompts) + step + 1
        _lib.eg_mla_decode_q8(dims, q, *cache, table, lens, longest, *gate, *weights, out, ws, dev_status=status)

    # the same tokens' values, packed and in a bf16 cache of their own
    n = sum(prompts) + steps * B
    values, kr, ids = torch.empty((n, D_C), dtype=BF16, device="cuda"), torch.empty((n, D_ROPE), dtype=BF16, device="cuda"), zeros(n)
    cu[1:] = lens.cumsum(0)
    _lib.eg_mla_read_latent_q8(dims, *cache, table, values, kr, ids, cu_seqlens=cu, dev_status=status)
    rounded_pool = torch.zeros_like(unrounded)
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), lens.long())
    pos = torch.arange(n, device="cuda") - cu[b].long()
    rounded_pool.view(-1, D_C)[table[b, pos // PAGE].long() * PAGE + pos % PAGE] = values

    def dense(pool):
        o = torch.empty_like(out)
        _lib.eg_mla_decode(dims, q, pool, kr_pool, id_pool, table, lens, longest, *gate, *weights, o, ws, dev_status=status)
        return o

    def apart(want):
        return float((out.double() - want.double()).norm() / want.double().norm())

    values_apart, rounded = apart(dense(rounded_pool)), apart(dense(unrounded))
    plan([-1] * B)
    all_free = int(count.item()) == pages
    print(f"{B} prompts of {min(prompts)} to {max(prompts)} tokens, {steps} steps: rel-L2 {values_apart:.1e} from the "
          f"decode over the same values in bf16, {rounded:.1e} from that over the unrounded ones; status {int(status.item())}")
    return values_apart, rounded, all_free, int(status.item())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompts", type=int, nargs="+", default=[300, 70, 64, 1])
    ap.add_argument("--steps", type=int, default=5)
    main(**vars(ap.parse_args()))
