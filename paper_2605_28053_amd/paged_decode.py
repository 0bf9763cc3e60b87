"""Decode steps of a small In-Place TTT model: paged attention, then the fast-weight MLP.

    python -m paper_2605_28053_amd.paged_decode [--owners 8] [--layers 2] [--steps 200]

Every layer of a step projects the owners' tokens to queries, keys and values,
turns queries and keys to their positions (``--rotary``), stores the keys and values
in the owners' pages, attends -- over all rows, or
over the selected pages once a context is longer than ``keep`` pages -- and
passes the result through the MLP whose down-projection is the owners'
fast-weight READ.  Requests come and go: an owner that has generated its tokens
returns its pages and starts over as the next request.  Weights are random, so
the tokens mean nothing; the projections around the two stateful operators are
plain torch products.
"""

import argparse
import time

import torch

from . import _rwttt as R
from .paged import PagedCache, Rotary


class Model:
    """Random weights of a decoder with fast-weight down-projections."""

    def __init__(self, n_layers=2, d_model=1024, n_heads=8, n_kv_heads=2, head_dim=128, d_ff=2816, vocab=1000,
                 dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def w(rows, cols, std=None):
            std = rows ** -0.5 if std is None else std
            return torch.randn((rows, cols), generator=g, device=device).mul_(std).to(dtype)

        self.n_heads, self.n_kv_heads, self.head_dim, self.d_ff, self.d_model = n_heads, n_kv_heads, head_dim, d_ff, d_model
        self.dtype, self.n_layers, self.vocab = dtype, n_layers, vocab
        self.embed = w(vocab, d_model, 1.0)
        self.head = w(d_model, vocab)
        qkv = (n_heads + 2 * n_kv_heads) * head_dim
        self.layers = [{"qkv": w(d_model, qkv), "out": w(n_heads * head_dim, d_model), "up": w(d_model, 2 * d_ff),
                        "w0": w(d_ff, d_model)} for _ in range(n_layers)]


def norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.pow(2).mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    """A model with the state of n_owners requests: fast weights and pages."""

    def __init__(self, model, n_owners, max_rows, page_rows=64, keep=0, cache_dtype=None, window=0, device="cuda",
                 rotary=None):
        m = self.model = model
        self.rotary = rotary
        self.n_owners, self.keep, self.window = n_owners, keep, window
        io = "f32" if m.dtype == torch.float32 else "bf16"
        max_pages = -(-max_rows // page_rows)
        self.cache = PagedCache(n_owners, m.n_layers, m.n_heads, m.n_kv_heads, m.head_dim, n_owners * max_pages, max_pages,
                                page_rows, io, cache_dtype or io, bound_step=0.05 if keep else None, k_scale=0.02,
                                v_scale=0.02, device=device)
        self.state = [[[torch.zeros((m.d_ff, m.d_model), dtype=torch.float32, device=device) for _ in range(2)]
                       for _ in range(m.n_layers)] for _ in range(n_owners)]
        slots = [s.data_ptr() for owner in self.state for layer in owner for s in layer]
        cfg = R.make_config(n_owners, m.n_layers, m.d_ff, m.d_model, R.RWTTT_F32 if io == "f32" else R.RWTTT_BF16,
                            R.RWTTT_F32, min(R.RWTTT_MAX_GROUP, n_owners), [w["w0"].data_ptr() for w in m.layers], slots)
        self.workspace = torch.empty(R.rwttt_workspace_bytes(cfg), dtype=torch.uint8, device=device)
        cfg.workspace, cfg.workspace_bytes = self.workspace.data_ptr(), self.workspace.numel()
        self.ctx = R.rwttt_create(cfg)
        # one READ takes RWTTT_MAX_GROUP owners at most
        self.groups = [R.make_group(R.RWTTT_READ, i, min(R.RWTTT_MAX_GROUP, n_owners - i))
                       for i in range(0, n_owners, R.RWTTT_MAX_GROUP)]
        self.owners = R.u32_array(range(n_owners))
        self.status = torch.zeros(1, dtype=torch.int32, device=device)   # the worst of all steps (errors are negative)

    def close(self):
        R.rwttt_destroy(self.ctx)
        self.cache.close()

    def extend(self, want):
        """Open a step of the cache.  One that does not fit leaves the lengths as they are; ``status`` keeps it."""
        self.cache.extend(want)
        torch.minimum(self.status, self.cache.result[:1], out=self.status)

    def step(self, tokens, want):
        """Logits [n_owners, vocab] of one token per owner; ``want`` are the owners' rows after it."""
        m, n, stream = self.model, self.n_owners, torch.cuda.current_stream().cuda_stream
        self.extend(want)
        x = m.embed[tokens]
        for l, w in enumerate(m.layers):
            qkv = (norm(x) @ w["qkv"]).view(n, m.n_heads + 2 * m.n_kv_heads, m.head_dim)
            q, k, v = qkv.split([m.n_heads, m.n_kv_heads, m.n_kv_heads], dim=1)
            if self.rotary is not None:      # every owner has one new token, in owner order
                self.cache.rotate(self.rotary, q, k)
            self.cache.append(l, k, v)
            pages = self.cache.select(l, q, self.keep) if self.keep else None
            a = self.cache.attend(l, q, pages=pages, window=self.window)
            x = x + a.view(n, -1) @ w["out"]
            gate, up = (norm(x) @ w["up"]).split(m.d_ff, dim=1)
            u = (torch.nn.functional.silu(gate.float()) * up.float()).to(m.dtype)
            y = torch.empty_like(x)
            for group in self.groups:
                st = R.rwttt_read(self.ctx, group, self.owners, l, u.data_ptr(), y.data_ptr(), stream)
                if st != R.RWTTT_OK:
                    raise R.RwtttError(st, "rwttt_read")
            x = x + y
        self.cache.commit()
        return norm(x) @ m.head


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--owners", type=int, default=8)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--keep", type=int, default=0, help="pages a query attends to (0: all)")
    ap.add_argument("--cache", choices=["bf16", "fp8", "fp4"], default="bf16")
    ap.add_argument("--rotary", action="store_true", help="rotary positions in queries and keys")
    a = ap.parse_args(argv)
    model = Model(n_layers=a.layers)
    dec = Decoder(model, a.owners, max_rows=a.steps + 64, keep=a.keep, cache_dtype=a.cache,
                  rotary=Rotary(model.head_dim) if a.rotary else None)
    tokens = torch.arange(a.owners, device="cuda") % model.vocab
    # request r ends after its own number of tokens: then its owner starts over, which
    # first returns the pages of the old one
    lives = torch.tensor([a.steps // 2 + 7 * r % (a.steps // 2 + 1) for r in range(a.owners)], dtype=torch.int32,
                         device="cuda").clamp_(min=1)
    ended, begin = 0, None
    for t in range(a.steps):
        if t == a.steps // 10:
            torch.cuda.synchronize()
            begin = time.perf_counter()
        over = dec.cache.lengths >= lives
        if bool(over.any()):
            ended += int(over.sum())
            dec.extend(torch.where(over, 0, dec.cache.lengths))
            dec.cache.commit()
        tokens = dec.step(tokens, dec.cache.lengths + 1).argmax(dim=1)
    torch.cuda.synchronize()
    steps = a.steps - a.steps // 10
    took = (time.perf_counter() - begin) / steps
    code = int(dec.status)
    print(f"{a.owners} owners, {a.layers} layers: {took * 1e6:.0f} us a step, {ended} requests ended, "
          f"rows {dec.cache.lengths.tolist()}, free pages {int(dec.cache.pos[1])}, status {code}")
    dec.close()
    return code


if __name__ == "__main__":
    raise SystemExit(main())
