"""A small serving loop on the paged latent cache, on synthetic inputs.

One document is prefilled.  Several sequences ask about it: each step plans the
pages of their new tokens, appends the tokens and decodes over the document (once
for all of them) and each sequence's own tokens.  Then one sequence goes on alone
over its whole text, decoding over the pages that matter most to its query, and
leaves.  Each form is compared with the dense decode over the same tokens.

    python examples/serve.py [--document 1000] [--sequences 12] [--steps 70] [--budget 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_16686_gb300 import _lib  # noqa: E402

PAGE, HEADS, D_NOPE, D_ROPE, D_C, VOCAB = 64, 16, 128, 64, 256, 1000


def pages_of(n):
    return (n + PAGE - 1) // PAGE


class Layer:
    """One attention layer's weights and cache, and the page bookkeeping of its sequences."""

    def __init__(self, sequences, num_pages, max_pages, seed=0):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dims = _lib.make_dims(HEADS, D_NOPE, D_ROPE, D_NOPE, D_C, VOCAB)
        self.gate = (self.normal(VOCAB, D_C, std=0.1, mean=1.0), torch.ones(D_C, device="cuda"),
                     torch.zeros(D_C, device="cuda"))
        self.w_uk, self.w_uv = (self.normal(HEADS, D_NOPE, D_C, std=D_C ** -0.5) for _ in range(2))
        self.c_pool = torch.zeros((num_pages, PAGE, D_C), dtype=torch.bfloat16, device="cuda")
        self.kr_pool = torch.zeros((num_pages, PAGE, D_ROPE), dtype=torch.bfloat16, device="cuda")
        self.id_pool = self.ints(num_pages, PAGE)
        self.summary = torch.zeros((num_pages, D_C + D_ROPE), device="cuda")
        self.lens, self.table = self.ints(sequences), self.ints(sequences, max_pages)
        self.free = torch.arange(num_pages, dtype=torch.int32, device="cuda")
        self.free_count = torch.full((1,), num_pages, dtype=torch.int32, device="cuda")
        self.cu, self.positions, self.status = self.ints(sequences + 1), self.ints(sequences), self.ints(1)
        self.slots = self.ints(max(max_pages * PAGE, sequences))
        self.most = [0] * sequences   # the host's bound of every length

    @staticmethod
    def ints(*shape):
        return torch.zeros(shape, dtype=torch.int32, device="cuda")

    def normal(self, *shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=self.gen, device="cuda").mul_(std).add_(mean).bfloat16()

    def tokens(self, n):
        """Synthetic latents, RoPE keys and ids of n tokens, and queries of n sequences."""
        ids = torch.randint(0, VOCAB, (n,), generator=self.gen, device="cuda", dtype=torch.int32)
        return self.normal(n, D_C, std=0.5), self.normal(n, D_ROPE), ids, self.normal(n, HEADS, D_NOPE + D_ROPE)

    def cache(self):
        return self.c_pool, self.kr_pool, self.id_pool

    def plan(self, new):
        """Pages for new[b] tokens of every sequence (negative: it leaves), in place."""
        self.new = torch.tensor(new, dtype=torch.int32, device="cuda")
        self.most = [m + n if n >= 0 else 0 for m, n in zip(self.most, new)]
        _lib.eg_mla_page_plan(self.new, self.lens, self.lens, self.table, self.free, self.free_count, self.free_count,
                              self.cu, self.positions, self.slots, dev_status=self.status)

    def prefill(self, b, n):
        """A prompt of n tokens as sequence b's, whose pages are planned."""
        c, kr, ids, q = self.tokens(n)
        out = torch.empty((n, HEADS, D_NOPE), dtype=torch.bfloat16, device="cuda")
        cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        ws = self.bytes(_lib.eg_mla_prefill_workspace_size(self.dims, 1, n))
        _lib.eg_mla_prefill(self.dims, q, c, kr, ids, cu, n, *self.gate, self.w_uk, self.w_uv, out, ws, *self.cache(),
                            self.table[b:b + 1], dev_status=self.status)

    def append(self):
        """A token for every sequence that the plan gave one."""
        c, kr, ids, q = self.tokens(len(self.lens))
        _lib.eg_mla_append_latent(self.dims, *self.cache(), c, kr, ids, self.table, self.positions, self.status)
        return q

    def summarise(self):
        """Mean keys of the pages that the planned tokens completed."""
        longest = max(self.most)
        _lib.eg_mla_page_summary(self.dims, *self.cache(), self.table, self.lens, longest, *self.gate, self.summary,
                                 new_tokens=self.new, max_new_tokens=longest, dev_status=self.status)

    @staticmethod
    def bytes(n):
        return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")

    def dense(self, q, table, lens, longest):
        out = torch.empty((len(lens), HEADS, D_NOPE), dtype=torch.bfloat16, device="cuda")
        ws = self.bytes(_lib.eg_mla_decode_workspace_size(self.dims, len(lens)))
        _lib.eg_mla_decode(self.dims, q, *self.cache(), table, lens, longest, *self.gate, self.w_uk, self.w_uv, out, ws,
                           0, self.status)
        return out


def apart(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm())


def main(document=1000, sequences=12, steps=70, budget=8):
    document -= document % PAGE   # (whole pages, so that the dense decode can be given the same tokens)
    rows = 1 + sequences          # sequence 0 holds the document
    max_pages = pages_of(document + steps)
    layer = Layer(rows, max_pages + sequences * pages_of(steps), max_pages)

    layer.plan([document] + [0] * sequences)
    layer.prefill(0, document)
    layer.summarise()

    # the questions: a token each per step, over the document and their own tokens
    prefix = layer.table[0, :pages_of(document)].contiguous()
    prefix_len = torch.full((1,), document, dtype=torch.int32, device="cuda")
    out = torch.empty((sequences, HEADS, D_NOPE), dtype=torch.bfloat16, device="cuda")
    ws = layer.bytes(_lib.eg_mla_decode_shared_workspace_size(layer.dims, sequences, document))
    for _ in range(steps):
        layer.plan([0] + [1] * sequences)
        q = layer.append()[1:].contiguous()
        _lib.eg_mla_decode_shared(layer.dims, q, *layer.cache(), prefix, prefix_len, document,
                                  layer.table[1:].contiguous(), layer.lens[1:].contiguous(), max(layer.most[1:]),
                                  *layer.gate, layer.w_uk, layer.w_uv, out, ws, dev_status=layer.status)
    joint = torch.cat([prefix.expand(sequences, -1), layer.table[1:, :pages_of(steps)]], 1).contiguous()
    shared = apart(out, layer.dense(q, joint, layer.lens[1:] + document, document + steps))

    # the document's own sequence goes on, over its best pages
    one = torch.empty((1, HEADS, D_NOPE), dtype=torch.bfloat16, device="cuda")
    chosen = layer.ints(1, budget)
    ws = layer.bytes(_lib.eg_mla_decode_sparse_workspace_size(layer.dims, 1, max_pages, budget))
    for _ in range(steps):
        layer.plan([1] + [0] * sequences)
        q = layer.append()[:1].contiguous()
        layer.summarise()
        _lib.eg_mla_decode_sparse(layer.dims, q, *layer.cache(), layer.table[:1], layer.lens[:1], layer.most[0],
                                  layer.summary, budget, 1, 1, *layer.gate, layer.w_uk, layer.w_uv, one, ws,
                                  selected=chosen, dev_status=layer.status)
    kept = chosen[0][chosen[0] >= 0].long()
    length = document + steps - (pages_of(document + steps) - len(kept)) * PAGE
    few = layer.table[:1, kept].contiguous()
    sparse = apart(one, layer.dense(q, few, torch.full((1,), length, dtype=torch.int32, device="cuda"), length))

    layer.plan([-1] * rows)
    free, status = int(layer.free_count.item()), int(layer.status.item())
    print(f"{sequences} sequences over a document of {document} tokens, {steps} steps: rel-L2 {shared:.1e} from the "
          f"dense decode over the same tokens")
    print(f"1 sequence of {document + steps} tokens, pages {kept.tolist()}: rel-L2 {sparse:.1e}")
    print(f"all left: {free} of {layer.c_pool.shape[0]} pages free, status {status}")
    return shared, sparse, free == layer.c_pool.shape[0], status


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("document", 1000), ("sequences", 12), ("steps", 70), ("budget", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    main(**vars(ap.parse_args()))
