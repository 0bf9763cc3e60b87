"""Paths of the 4-bit cache's kernels that ordinary sizes do not reach."""

import math
import random

import pytest
import torch

from paper_2605_28053_amd import _rwttt_kv as KV
from tests.kv4_util import KV_FP4, Cache4, gather, stored4
from tests.kv_util import DT, bounds_ref, dev, i32, ok, stream
from tests.test_gpu_kv4 import after, append, same_bytes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,D", [(5, 64), (4, 128), (4, 256)])
@pytest.mark.parametrize("kind", ["scattered", "runs", "ends"])
def test_many_pages_in_a_block(io, H, D, kind):
    """More rows than the one-token-a-wave kernel takes.  Scattered: every token alone in its page.
    Runs: of 1 to 40 tokens, some padded ones between.  Ends: only tokens 64 k - 1 and 64 k share a page."""
    rng, g, n, P = random.Random(D), torch.Generator().manual_seed(D), 1100, 16 if kind != "runs" else 32
    c = Cache4([1], H=H, G=1, D=D, page=P, io=io, seed=1, extra_pages=n, poison=False)
    c.bounds_h = torch.randint(-9, 9, c.bounds_h.shape, generator=g).sort(dim=2).values.to(torch.int8)
    c.bounds.copy_(c.bounds_h)
    pages, slots = rng.sample(range(c.N), n), []
    if kind == "scattered":
        slots = [p * P + rng.randrange(P) for p in pages]
        slots[100], slots[700] = -1, c.N * P + 3
    elif kind == "runs":
        while len(slots) < n:
            p, first = pages.pop(), rng.choice([0, 0, rng.randrange(P)])
            slots += [p * P + i for i in range(first, min(P, first + rng.randint(1, 40)))]
            slots += [-1] * rng.choice([0, 0, 0, 2])
        slots = slots[:n]
    else:
        for t in range(n):
            slots.append(slots[-1] + 1 if t and t % 64 == 0 else pages[t] * P + rng.randrange(P - 1))
    k, v = (torch.randn((n, H, D), generator=g).to(DT[io]) for _ in range(2))
    k[3, 1, 40], k[200, 0, 1], k[64, 2, 3] = math.nan, math.inf, -math.inf
    k[640:704, 0, :32] = math.nan                          # pages that hold NaN alone in a block
    raw = append(c, k, v, slots, strided=True)
    same_bytes(raw[0], *after(c, "k", k, slots), P, D)
    same_bytes(raw[1], *after(c, "v", v, slots), P, D)
    live = [s if 0 <= s < c.N * P else -1 for s in slots]
    want = bounds_ref(c.bounds_h, stored4(k).float(), live, torch.ones(H), c.step_h, "f32", P)
    assert torch.equal(c.bounds.cpu(), torch.from_numpy(want))
    c.close()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("P", [16, 64, 256])
def test_pages_that_span_blocks(io, D, P):
    """3000 tokens in order from row 100 on, without bounds and with them."""
    n, H, g = 3000, 2, torch.Generator().manual_seed(P)
    k, v = (torch.randn((n, H, D), generator=g).to(DT[io]) for _ in range(2))
    for bounds in (True, False):
        c = Cache4([n + 100], H=H, G=1, D=D, page=P, io=io, seed=2, bounds=bounds)
        slots = [int(c.table_h[0, t // P]) * P + t % P for t in range(100, n + 100)]
        raw = append(c, k, v, slots)
        same_bytes(raw[0], *after(c, "k", k, slots), P, D)
        same_bytes(raw[1], *after(c, "v", v, slots), P, D)
        if bounds:
            want = bounds_ref(c.bounds_h, stored4(k).float(), slots, torch.ones(H), c.step_h, "f32", P)
            assert torch.equal(c.bounds.cpu(), torch.from_numpy(want))
        c.close()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.25, 1e-30, 3.0])
def test_any_scale(io, scale):
    """None at all makes all rows alike, a negative one turns the order round."""
    c = Cache4([1, 70, 0, 300], H=2, G=3, D=128, page=16, io=io, seed=3)
    got = c.attend(scale=scale)
    for r in range(c.R):
        c.check(got, r, scale=scale)
    got = c.attend(scale=scale, window=33)
    for r in range(c.R):
        c.check(got, r, scale=scale, window=33)
    c.close()


@pytest.mark.parametrize("G", [1, 4, 5, 6, 8, 9, 16, 21])
def test_probabilities_keep_the_bits_that_cancel(G):
    """Three rows an owner: the largest score with values of 0, and two of nearly equal scores with
    values of 1 and -1, whose difference is what remains.

    The scores are exact: one product of 1 by a code, and one of a power of two.  A probability
    of fp32 arithmetic is off by 2^-22 of itself at most (its exponent is one fused product, 2^-24
    of at most 2; the exponential as much), so out by 2 * 2^-22 and its own rounding; one of 16
    bits would be off by up to 2^-17."""
    c = Cache4([3] * 60, H=1, G=G, D=64, page=16, io="bf16", seed=1, poison=False)
    delta = -15
    for r in range(c.R):
        page = int(c.table_h[r, 0])
        for x in "kv":
            c.code[x][page] = 0
            c.E[x][page] = 127
        c.code["k"][page, 0, 1:3, 0], c.E["k"][page, 0, 1:3, 0] = 9 + r % 7, 126 - r % 3       # of -1/2 .. -6, times 1/2 to 1/8
        c.code["k"][page, 0, 2, 40], c.E["k"][page, 0, 2, 1] = 2, 127 + delta
        c.code["v"][page, 0, 1], c.code["v"][page, 0, 2] = 2, 10
    c.close()
    c.upload()
    c.q_h.zero_()
    c.q_h[:, :, 0] = (torch.arange(G) % 4 + 1).to(torch.bfloat16) / 4
    c.q_h[:, :, 40] = 1.0
    out, _ = c.attend(scale=1.0)
    worst = 0.0
    for r in range(c.R):
        ref = c.attend_ref(r, scale=1.0)[0]
        worst = max(worst, float(((out[r].double() - ref).abs() - 2.0 ** -8 * ref.abs()).max()))
    assert worst <= 2.0 ** -21, worst
    c.close()


def test_pages_beyond_four_gigabytes():
    """Rows stored, read back and attended to at both ends of pools of 5.6 GB."""
    H, D, P, N = 8, 256, 256, 20000
    k, v = (torch.zeros((N, H, P * D * 17 // 32), dtype=torch.uint8, device="cuda") for _ in range(2))
    lens = [700, 130]
    table = torch.zeros((2, 4), dtype=torch.int32)
    table[0, :3], table[1, :1] = torch.tensor([N - 1, 0, N - 2], dtype=torch.int32), N - 3
    td, lengths = dev(table), i32(lens)
    cfg = KV.make_kv_config(2, 1, N, P, 4, 16, H, D, 1, KV_FP4, table=td.data_ptr(), k=[k.data_ptr()], v=[v.data_ptr()])
    ws = torch.zeros(KV.rwttt_kv_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.workspace, cfg.workspace_bytes = ws.data_ptr(), ws.numel()
    kv = KV.rwttt_kv_create(cfg)
    g = torch.Generator().manual_seed(4)
    owners = [0] * 700 + [1] * 130
    positions = list(range(700)) + list(range(130))
    slots = i32([int(table[r, p // P]) * P + p % P for r, p in zip(owners, positions)])
    nk, nv = (torch.randn((830, H, D), generator=g).bfloat16() for _ in range(2))
    kd, vd = dev(nk), dev(nv)
    for a, b in ((0, 830), (690, 700), (0, 1)):              # in blocks, and one token a wave
        ok(KV.rwttt_kv_append(kv, 0, kd[a:].data_ptr(), H * D, vd[a:].data_ptr(), H * D, slots[a:b].clone().data_ptr(), b - a, stream()))
    gk, gv = gather(kv, owners, positions, lengths, H, D, "bf16")
    ek, ev = stored4(nk), stored4(nv)
    assert torch.equal(gk.double(), ek) and torch.equal(gv.double(), ev)
    q = torch.randn((2, 16, D), generator=g).bfloat16()
    qd, out = dev(q), torch.zeros((2, 16, D), dtype=torch.bfloat16, device="cuda")
    ok(KV.rwttt_kv_attend(kv, 0, qd.data_ptr(), 16 * D, lengths.data_ptr(), 0, 2, D ** -0.5, 0, 0, 0, out.data_ptr(), 16 * D, 0,
                          stream()))
    for r, at in ((0, slice(0, 700)), (1, slice(700, 830))):
        for i in range(16):
            y = torch.softmax(ek[at, i // 2] @ q[r, i].double() * D ** -0.5, dim=0) @ ev[at, i // 2]
            assert bool(((out[r, i].double().cpu() - y).abs() <= 1.01 * 2.0 ** -8 * y.abs() + 1e-4).all())
    # nothing else was written
    torch.cuda.synchronize()
    for x in (k, v):
        assert int((x[1:N - 3] != 0).sum()) == 0
    KV.rwttt_kv_destroy(kv)


def test_strides_and_offsets_beyond_four_gigabytes():
    """Tokens two to five gigabytes apart, turned in place, stored and read back."""
    H, D, n, step = 2, 128, 3, 1 << 30                       # elements: 2 GB in bf16
    big = torch.zeros(2 * step + 4096, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(5)
    x = torch.randn((n, 2 * H, D), generator=g).bfloat16()
    view = big.as_strided((n, 2 * H, D), (step, D, 1))
    view.copy_(x)
    k, v = view[:, :H], view[:, H:]
    c = Cache4([n], H=H, G=1, D=D, page=16, io="bf16", seed=6)
    at = i32([int(c.table_h[0, 0]) * 16 + i for i in range(n)])
    ok(KV.rwttt_kv_append(c.kv, 0, k.data_ptr(), step, v.data_ptr(), step, at.data_ptr(), n, stream()))
    torch.cuda.synchronize()
    same_bytes(c.kd.cpu(), *after(c, "k", x[:, :H], at.tolist()), 16, D)
    view.zero_()
    zero, positions = i32([0] * n), i32(list(range(n)))
    ok(KV.rwttt_kv_gather(c.kv, 0, zero.data_ptr(), positions.data_ptr(), c.lengths.data_ptr(), n, k.data_ptr(), step,
                          v.data_ptr(), step, stream()))
    torch.cuda.synchronize()
    assert torch.equal(view.cpu().double(), stored4(x))
    view.copy_(x)
    units = KV.rwttt_kv_turns(D, 1e4)
    table = torch.tensor(units, dtype=torch.uint64).cuda()
    rot = KV.make_rotary(D, KV.RWTTT_ROTARY_HALF, table.data_ptr())
    small = dev(x[:, :H])
    for t, s in ((k, step), (small, H * D)):
        ok(KV.rwttt_kv_rotate(c.kv, rot, positions.data_ptr(), n, 0, 0, 0, 0, t.data_ptr(), s, t.data_ptr(), s, stream()))
    torch.cuda.synchronize()
    assert torch.equal(k, small) and not torch.equal(small.cpu()[1:], x[1:, :H]) and int((big[4096:step] != 0).sum()) == 0
    c.close()


def test_rows_of_pages_swapped_for_junk():
    """Table entries and listed pages out of range read some page of the pool, and lengths beyond the
    table are those it holds; nothing faults and other owners are as ever."""
    c = Cache4([300, 40], H=1, G=2, D=128, page=32, io="bf16", seed=7, poison=False)
    c.table[0, 3], c.table[0, 5] = 1 << 30, -5
    c.check(c.attend(), 1)
    got = c.attend(lengths=i32([1 << 30, 40]))
    c.check(got, 1)
    pages = i32([[[0, 1 << 20, -9, 3]], [[0, 1, -1, -1]]])
    got = c.attend(pages=pages)
    c.check(got, 1, listed=[[0, 1]])
    k, _ = gather(c.kv, [0, 1], [100, 7], i32([1 << 30, 40]), 1, 128, "bf16")
    assert torch.equal(k[1].double(), c.rows_of(1, 0, "k", [7]))
    c.close()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,n", [(64, 5000), (128, 5000), (256, 3000)])
def test_infinite_scores_anywhere_in_a_split_row(io, D, n):
    """Products beyond fp32: one -inf score weighs nothing, -inf alone gives 0 and -inf, +inf and a
    NaN block give NaN, each in the first rows, in the middle and in the last ones."""
    places = [0, 1, n // 2, n - 2, n - 1]
    cases = [(at, x) for at in places for x in ("-inf", "inf", "nan")] + [(None, "-inf")]
    c = Cache4([n] * len(cases), H=1, G=1, D=D, page=16, io=io, seed=1, poison=False, bounds=False)
    c.code["k"].fill_(1)
    c.E["k"].fill_(125)
    c.code["k"][..., 5] = 0
    for r, (at, x) in enumerate(cases):
        pages = c.table_h[r, :-(-n // 16)].long()
        page, row = (pages, slice(None)) if at is None else (pages[at // 16], at % 16)
        c.E["k"][page, 0, row, 0] = 255 if x == "nan" else 127 + 100
        c.code["k"][page, 0, row, 5] = 15 if x == "-inf" else 7
        c.code["k"][page, 0, row, :5] = 0
        c.code["k"][page, 0, row, 6:32] = 0
    c.close()
    c.upload()
    q = torch.ones((c.R, 1, D))
    q[..., 5] = 2.0 ** 126                                   # one bf16 term
    out, lse = c.attend(q=dev(q.to(DT[io])))
    for r, (at, x) in enumerate(cases):
        if at is None:
            assert bool((out[r] == 0).all()) and float(lse[r, 0]) == -math.inf
        elif x == "-inf":
            v = c.rows_of(r, 0, "v", [j for j in range(n) if j != at]).mean(dim=0)
            half = 2.0 ** -8 if io == "bf16" else 2.0 ** -24
            assert bool(((out[r, 0].double() - v).abs() <= 1.01 * half * v.abs() + 1e-4).all())
        else:
            assert bool(torch.isnan(out[r]).all()) and bool(torch.isnan(lse[r]).all()), (at, x)
    c.close()
