"""Caches of 4 bits for the tests: codes and powers by the book, and handles over them."""

import math

import torch

from paper_2605_28053_amd import _rwttt_kv as KV
from tests.kv_util import DT, Cache, dev, i32, ok, pages_of, stream

KV_FP4 = KV.RWTTT_FP4
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
BLOCK = 32


def encode_ref(x):
    """Codes (integers) [..., D] and powers E [..., D / 32] of rows x, in 64 bits."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    finite = torch.isfinite(b).all(dim=-1)
    clean = torch.where(finite[..., None], b, 0.0)
    m, e = torch.frexp(clean.abs().amax(dim=-1))                  # m in [1/2, 1): the mantissa is 2 m, the exponent e - 1
    E = e - 1 + (m >= 0.875).int() - 2 + 127
    E = torch.where(m == 0, 2, E).clamp(2, 252)
    y = clean.abs() / torch.exp2((E - 127).double())[..., None]
    dist = (y[..., None] - torch.tensor(GRID, dtype=torch.float64)).abs()
    even, odd = dist[..., 0::2].min(dim=-1), dist[..., 1::2].min(dim=-1)
    code = torch.where(odd.values < even.values, 2 * odd.indices + 1, 2 * even.indices)
    code = code + 8 * torch.signbit(clean).long()
    return code.flatten(-2), torch.where(finite, E, 255)


def decode_ref(code, E):
    """Values in float64 of codes [..., D] and powers [..., D / 32]."""
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
    unit = torch.where(E == 255, math.nan, torch.exp2((E - 127).double()))
    return (grid[code].unflatten(-1, (-1, BLOCK)) * unit[..., None]).flatten(-2)


def stored4(x):
    return decode_ref(*encode_ref(x))


def pack(code, E):
    """Bytes [N, H, P * D * 17 / 32] of codes [N, H, P, D] and powers [N, H, P, D / 32]."""
    low, high = code[..., 0::2], code[..., 1::2]
    return torch.cat([(low | high << 4).flatten(2), E.transpose(-1, -2).flatten(2)], dim=2).to(torch.uint8)


def unpack(raw, P, D):
    """The codes [N, H, P, D] and powers [N, H, P, D / 32] of a cache's bytes."""
    N, H, _ = raw.shape
    byte = raw[..., :P * D // 2].reshape(N, H, P, D // 2).long()
    return (torch.stack([byte & 15, byte >> 4], dim=-1).flatten(-2),
            raw[..., P * D // 2:].reshape(N, H, D // BLOCK, P).transpose(-1, -2).long())


class Cache4(Cache):
    """A handle over a cache of 4 bits.  Unused table entries name other owners' pages, and what
    lies behind an owner's rows is NaN (E = 255)."""

    def __init__(self, lens, H, G, D, page, io, seed=0, max_pages=None, extra_pages=2, poison=True, spread=3, bounds=True):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H, self.G, self.D, self.page, self.io, self.cache = lens, H, G, D, page, io, "fp4"
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
        self.code, self.E = {}, {}
        for x in "kv":
            self.code[x] = torch.randint(0, 16, (self.N, H, page, D), generator=g)
            # powers that differ from row to row and block to block
            self.E[x] = 126 + torch.randint(-spread, 1, (self.N, H, page, D // BLOCK), generator=g)
            if poison:
                keep = torch.zeros((self.N, page), dtype=torch.bool)
                for r, n in enumerate(lens):
                    for j in range(used[r]):
                        keep[int(self.table_h[r, j]), :max(0, min(page, n - j * page))] = True
                self.E[x][~keep[:, None, :, None].expand_as(self.E[x])] = 255
        self.step_h = 0.1 + 0.05 * torch.rand(H, generator=g)
        self.step = dev(self.step_h)
        self.bounds_h = torch.zeros((self.N, H, 2, D), dtype=torch.int8)
        self.bounds = dev(self.bounds_h) if bounds else None
        self.lengths = i32(lens)
        self.q_h = torch.randn((self.R, H * G, D), generator=g).to(DT[io])
        self.upload()

    def upload(self):
        self.kd, self.vd = (dev(pack(self.code[x], self.E[x])) for x in "kv")
        self.kv = self.handle()

    def handle(self):
        cfg = KV.make_kv_config(
            self.R, 1, self.N, self.page, self.MP, self.H * self.G, self.H, self.D, 0 if self.io == "f32" else 1, KV_FP4,
            table=self.table.data_ptr(), k=[self.kd.data_ptr()], v=[self.vd.data_ptr()],
            bounds=[self.bounds.data_ptr()] if self.bounds is not None else None, bound_step=self.step.data_ptr())
        self.ws = torch.zeros(KV.rwttt_kv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        cfg.workspace, cfg.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
        return KV.rwttt_kv_create(cfg)

    def rows_of(self, r, h, which, at):
        at = torch.as_tensor(at, dtype=torch.int64)
        page, row = self.table_h[r].long()[at // self.page], at % self.page
        return decode_ref(self.code[which][page, h, row], self.E[which][page, h, row])


def gather(kv, owners, positions, lengths, heads, D, io, strides=(0, 0), sides="kv", fill=7.0):
    """(k, v) of the call on the CPU; rows that it should not touch hold `fill`."""
    n, out = len(owners), {}
    o, p = i32(owners), i32(positions)
    for x, extra in zip("kv", strides):
        buf = torch.full((n, heads * D + extra), fill, dtype=DT[io], device="cuda")
        out[x] = buf
    args = [out[x].data_ptr() if x in sides else 0 for x in "kv"]
    ok(KV.rwttt_kv_gather(kv, 0, o.data_ptr(), p.data_ptr(), lengths.data_ptr(), n, args[0], out["k"].stride(0), args[1],
                          out["v"].stride(0), stream()))
    torch.cuda.synchronize()
    for x in "kv":                       # nothing is written between the rows
        assert bool((out[x][:, heads * D:] == fill).all())
    return tuple(out[x][:, :heads * D].reshape(n, heads, D).cpu() for x in "kv")
