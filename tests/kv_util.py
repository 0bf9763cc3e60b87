"""Paged caches for the tests, and the operators' definitions in 64 bits on the CPU."""

import math

import numpy as np
import torch

from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd import _rwttt_kv as KV

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
CODE = {"f32": R.RWTTT_F32, "bf16": R.RWTTT_BF16, "fp8": KV.RWTTT_FP8}


def pages_of(n, page):
    return -(-n // page)


def dev(t):
    return t.cuda().contiguous()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


def ok(status):
    assert status == R.RWTTT_OK, R.rwttt_strerror(status)


class Cache:
    """A handle with its buffers on the GPU and a float64 copy of the values on the CPU.

    The table's unused entries name pages of other owners and the rows behind an
    owner's length hold NaN: neither may reach a result."""

    no_workspace = False

    def __init__(self, lens, H, G, D, page, io, cache, seed=0, max_pages=None, extra_pages=2, std=1.0, n_layers=1,
                 poison=True):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H, self.G, self.D, self.page, self.io, self.cache = lens, H, G, D, page, io, cache
        self.R = len(lens)
        used = [pages_of(n, page) for n in lens]
        self.MP = max_pages or max(1, max(used)) + 1
        self.N = sum(used) + extra_pages
        order = torch.randperm(self.N, generator=g).tolist()
        self.table_h = torch.randint(0, self.N, (self.R, self.MP), generator=g, dtype=torch.int32)
        at = 0
        for r, n in enumerate(used):
            self.table_h[r, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = dev(self.table_h)
        shape = (self.N, H, page, D)
        fp8 = cache == "fp8"
        mul = 30.0 if fp8 else std
        self.k, self.v = ((torch.randn(shape, generator=g) * mul).to(DT[cache]) for _ in range(2))
        if poison:
            for c in (self.k, self.v):
                raw = c.view(torch.uint8) if fp8 else c
                bad = 0x7f if fp8 else float("nan")
                held = set()
                for r, n in enumerate(lens):
                    for j in range(used[r]):
                        p = int(self.table_h[r, j])
                        held.add(p)
                        raw[p, :, max(0, min(page, n - j * page)):] = bad
                for p in range(self.N):
                    if p not in held:
                        raw[p] = bad
        self.k_scale_h = (0.02 + 0.02 * torch.rand(H, generator=g)) if fp8 else torch.ones(H)
        self.v_scale_h = (0.02 + 0.02 * torch.rand(H, generator=g)) if fp8 else torch.ones(H)
        self.step_h = 0.03 + 0.02 * torch.rand(H, generator=g)
        self.kd, self.vd = dev(self.k), dev(self.v)
        self.bounds_h = torch.zeros((self.N, H, 2, D), dtype=torch.int8)
        self.bounds = dev(self.bounds_h)
        self.ring = torch.full((self.N,), -1, dtype=torch.int32, device="cuda")
        self.free = order[at:]
        self.ring[:len(self.free)] = i32(self.free) if self.free else i32([])
        self.k_scale, self.v_scale, self.step = dev(self.k_scale_h), dev(self.v_scale_h), dev(self.step_h)
        self.lengths = i32(lens)
        self.q_h = torch.randn((self.R, H * G, D), generator=g).to(DT[io])
        self.kv = self.handle()

    def handle(self):
        fp8 = self.cache == "fp8"
        cfg = KV.make_kv_config(
            self.R, 1, self.N, self.page, self.MP, self.H * self.G, self.H, self.D, CODE[self.io], CODE[self.cache],
            table=self.table.data_ptr(), ring=self.ring.data_ptr(), k=[self.kd.data_ptr()], v=[self.vd.data_ptr()],
            bounds=[self.bounds.data_ptr()], k_scale=self.k_scale.data_ptr() if fp8 else 0,
            v_scale=self.v_scale.data_ptr() if fp8 else 0, bound_step=self.step.data_ptr())
        if not self.no_workspace:
            self.ws = torch.zeros(KV.rwttt_kv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            cfg.workspace, cfg.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
        return KV.rwttt_kv_create(cfg)

    def close(self):
        KV.rwttt_kv_destroy(self.kv)

    # ---- calls --------------------------------------------------------------
    def attend(self, q=None, rows=None, window=0, pages=None, scale=None, out=None, lengths=None):
        """(out, lse) of the call; rows that it should not touch hold 7."""
        q = dev(self.q_h) if q is None else q
        heads = self.H * self.G
        out = torch.full((self.R, heads, self.D), 7.0, dtype=DT[self.io], device="cuda") if out is None else out
        lse = torch.full((self.R, heads), 7.0, dtype=torch.float32, device="cuda")
        lengths = self.lengths if lengths is None else lengths
        ok(KV.rwttt_kv_attend(
            self.kv, 0, q.data_ptr(), q.stride(0), lengths.data_ptr(), 0 if rows is None else rows.data_ptr(),
            self.R if rows is None else rows.numel(), self.D ** -0.5 if scale is None else scale, window,
            0 if pages is None else pages.data_ptr(), 0 if pages is None else pages.shape[-1],
            out.data_ptr(), out.stride(0), lse.data_ptr(), stream()))
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    # ---- definitions --------------------------------------------------------
    def rows_of(self, r, h, which, at):
        """Values of positions `at` of owner r in float64."""
        c = self.k if which == "k" else self.v
        s = (self.k_scale_h if which == "k" else self.v_scale_h)[h]
        at = torch.as_tensor(at, dtype=torch.int64)
        page, row = self.table_h[r].long()[at // self.page], at % self.page
        c = c.view(torch.uint8)[page, h, row].view(DT["fp8"]).float() if self.cache == "fp8" else c[page, h, row]
        return c.double() * (float(s) if self.cache == "fp8" else 1.0)

    def attend_ref(self, r, window=0, listed=None, scale=None):
        """(out [H*G, D], lse [H*G], tolerance of out's fp32 arithmetic, of lse) of one owner.

        The tolerance bounds the fp32 work: a score's product sum over D channels is
        off by (D + 4) 2^-24 sum |q k| scale at most, a probability by twice that
        relative to itself, and the sums over the rows by their number times 2^-23."""
        n, scale = self.lens[r], self.D ** -0.5 if scale is None else scale
        out = torch.zeros((self.H * self.G, self.D), dtype=torch.float64)
        lse = torch.full((self.H * self.G,), -math.inf, dtype=torch.float64)
        tol, ltol = torch.zeros(self.H * self.G), torch.zeros(self.H * self.G)
        for h in range(self.H):
            if listed is not None:
                at = [p * self.page + i for p in listed[h] if 0 <= p < pages_of(n, self.page)
                      for i in range(min(self.page, n - p * self.page))]
            else:
                at = range(max(0, n - window) if window else 0, n)
            if len(at) == 0:
                continue
            at = torch.tensor(list(at))
            k, v = self.rows_of(r, h, "k", at), self.rows_of(r, h, "v", at)
            hs = slice(h * self.G, (h + 1) * self.G)
            q = self.q_h[r, hs].double()
            s = (q @ k.t()) * scale
            out[hs] = torch.softmax(s, dim=1) @ v
            lse[hs] = torch.logsumexp(s, dim=1)
            delta = (self.D + 4) * 2.0 ** -24 * abs(scale) * float((q.abs() @ k.abs().t()).max())
            tol[hs] = (2 * delta + len(at) * 2.0 ** -23 + 2.0 ** -16) * float(v.abs().max())
            ltol[hs] = 2 * delta + len(at) * 2.0 ** -23 + 2.0 ** -20 * (1 + float(lse[hs].abs().max()))
        return out, lse, tol, ltol

    def check(self, got, r, **kw):
        out, lse = got
        ref, rl, tol, ltol = self.attend_ref(r, **kw)
        half = 2.0 ** -8 if self.io == "bf16" else 2.0 ** -24          # one rounding to 8 or 24 bits
        err = (out[r].double() - ref).abs()
        assert torch.isfinite(out[r].double()).all()
        assert bool((err <= half * 1.01 * ref.abs() + tol[:, None]).all()), (r, self.lens[r], float(err.max()))
        fin = torch.isfinite(rl)
        assert torch.equal(fin, torch.isfinite(lse[r])) and bool((lse[r][~fin] == -math.inf).all())
        assert bool(((lse[r].double() - rl).abs()[fin] <= ltol[fin]).all()), (lse[r], rl)


# ---------------------------------------------------------------------------
# extend, append, select by the book
# ---------------------------------------------------------------------------

def extend_ref(have, want, front, count, table, ring, page, cap):
    """Pure-Python extend: dict of its outputs; table and ring are copied."""
    R, MP, N = len(have), len(table[0]), len(ring)
    table, ring = [list(t) for t in table], list(ring)
    grow = [max(0, pages_of(w, page) - pages_of(h, page)) for h, w in zip(have, want)]
    back = [max(0, pages_of(h, page) - pages_of(w, page)) for h, w in zip(have, want)]
    add = [max(0, w - h) for h, w in zip(have, want)]
    code = 0
    if any(x < 0 or x > MP * page for x in have + want) or not 0 <= front < N or not 0 <= count <= N:
        code = R_INVALID
    elif sum(grow) > count or sum(add) > cap:
        code = R_CAPACITY
    elif count - sum(grow) + sum(back) > N:
        code = R_INVALID
    if code:
        return {"table": table, "ring": ring, "pos": [front, count], "lengths": have, "start": [0] * (R + 1),
                "slots": [-1] * cap, "owners": [-1] * cap, "positions": [-1] * cap, "result": [code, 0, 0, 0]}
    old = [list(t) for t in table]
    f = front
    for r in range(R):
        for i in range(grow[r]):
            table[r][pages_of(have[r], page) + i] = ring[f]
            f = (f + 1) % N
    b = (front + count) % N
    for r in range(R):
        for i in range(back[r]):
            ring[b] = old[r][pages_of(want[r], page) + i]
            b = (b + 1) % N
    slots, owners, positions, start = [], [], [], [0]
    for r in range(R):
        for j in range(have[r], have[r] + add[r]):
            slots.append(table[r][j // page] * page + j % page)
            owners.append(r)
            positions.append(j)
        start.append(len(slots))
    pad = [-1] * (cap - len(slots))
    return {"table": table, "ring": ring, "pos": [f, count - sum(grow) + sum(back)], "lengths": want, "start": start,
            "slots": slots + pad, "owners": owners + pad, "positions": positions + pad,
            "result": [0, sum(add), sum(grow), sum(back)]}


R_INVALID, R_CAPACITY = -1, -7


def stored(x, scale, cache):
    """[n, H, D] new rows as the cache holds them (CPU)."""
    if cache == "fp8":
        return (x.float() * (1.0 / scale)[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return x.float().to(DT[cache])


def bounds_ref(bounds, k, slots, scale, step, cache, page):
    """Page bounds (int8 numpy, copied) after the rows k [n, H, D] went to their slots."""
    out = bounds.numpy().astype(np.int64).copy()
    x = k.float() * scale[:, None] if cache == "fp8" else k.float()
    x = (x * (1.0 / step)[:, None]).numpy().astype(np.float64)
    fresh = {s // page for s in slots if s >= 0 and s % page == 0}
    for p in fresh:
        out[p, :, 0], out[p, :, 1] = 127, -127
    for t, s in enumerate(slots):
        if s < 0:
            continue
        p = s // page
        lo, hi = np.clip(np.floor(x[t]), -127, 127), np.clip(np.ceil(x[t]), -127, 127)
        fine = ~np.isnan(x[t])
        out[p, :, 0] = np.where(fine, np.minimum(out[p, :, 0], np.where(fine, lo, 0)), out[p, :, 0])
        out[p, :, 1] = np.where(fine, np.maximum(out[p, :, 1], np.where(fine, hi, 0)), out[p, :, 1])
    return out.astype(np.int8)


def select_ref(q, bounds, pages, first, last, keep):
    """Pages of one owner and kv head: q [G, D] float32 numpy, bounds [np, 2, D] of its pages."""
    n = len(pages)
    if n <= keep:
        return list(range(n)) + [-1] * (keep - n)
    a = np.float32(np.abs(q).max())
    to = np.float32(1.0) / a * np.float32(127.0) if a > 0 else np.float32(0.0)
    q8 = np.rint(q * to).astype(np.int64)
    b = bounds[pages].astype(np.int64)
    score = np.maximum(q8[None] * b[:, None, 0], q8[None] * b[:, None, 1]).sum(axis=(1, 2))
    forced = [j for j in range(n) if j < first or j >= n - last]
    rest = sorted((j for j in range(n) if j not in set(forced)), key=lambda j: (-score[j], j))
    return sorted(forced + rest[:keep - len(forced)])
