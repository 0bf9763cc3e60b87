"""The paged key-value cache on the GPU against its definitions in 64 bits."""

import random

import numpy as np
import pytest
import torch

from tests.kv_util import (CODE, DT, Cache, bounds_ref, dev, extend_ref, i32, ok, pages_of, select_ref, stored, stream)
from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd import _rwttt_kv as KV

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "bf16"), ("f32", "fp8")]
# no row, one, the edges of a tile's halves, of a tile, of a page, and a few of each
EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 130, 0, 257]


# ---------------------------------------------------------------------------
# attend
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64])
def test_attend_at_the_edges_of_tiles_and_pages(io, cache, D, page):
    c = Cache(EDGES, H=2, G=3, D=D, page=page, io=io, cache=cache, seed=D + page)
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 2), (1, 5), (2, 8), (1, 16), (2, 17), (1, 40), (1, 128)])
@pytest.mark.parametrize("io,cache", [("bf16", "bf16"), ("f32", "f32")])
def test_attend_head_layouts(H, G, io, cache):
    c = Cache([70, 0, 33, 129], H=H, G=G, D=64, page=32, io=io, cache=cache, seed=G)
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)


@pytest.mark.parametrize("io,cache", TYPES)
def test_attend_long_rows_are_split_and_joined(io, cache):
    """Lengths from one row to 60000: the parts begin and end inside rows, and one
    row is spread over most of them."""
    c = Cache([60000, 1, 0, 700, 5000, 31], H=2, G=4, D=128, page=128, io=io, cache=cache, seed=5)
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)


@pytest.mark.parametrize("io,cache", [("bf16", "fp8"), ("f32", "f32")])
def test_attend_many_short_rows_beside_long_ones(io, cache):
    """More rows than blocks; the blocks' parts begin and end at any point of a row."""
    rng = random.Random(3)
    lens = [rng.choice([0, 1, 5, 16, 40, 90, 150]) for _ in range(700)]
    lens[13], lens[400], lens[699] = 9000, 3000, 1
    c = Cache(lens, H=2, G=2, D=64, page=16, io=io, cache=cache, seed=6)
    got = c.attend()
    for r in list(range(0, 700, 9)) + [13, 400, 699]:
        c.check(got, r)
    again = c.attend()
    assert torch.equal(got[0].float(), again[0].float()) and torch.equal(got[1], again[1])


def test_attend_the_most_owners_and_the_widest_rows():
    """4096 owners, sixteen queries of 256 channels a head: the most LDS a call asks for."""
    rng = random.Random(8)
    lens = [rng.choice([0, 1, 3, 16]) for _ in range(4096)]
    lens[2000] = 700
    c = Cache(lens, H=1, G=16, D=256, page=16, io="bf16", cache="bf16", seed=1, poison=False)
    got = c.attend()
    for r in list(range(0, 4096, 101)) + [2000, 4095]:
        c.check(got, r)
    rows = i32([4095 - r for r in range(4096)])
    again = c.attend(rows=rows)
    for r in (0, 1, 2000, 4095):
        c.check(again, r)


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("window", [1, 16, 31, 100, 1000])
def test_attend_window(page, window):
    c = Cache([0, 1, 30, 100, 101, 999, 1001, 3001], H=2, G=2, D=64, page=page, io="bf16", cache="bf16", seed=window)
    got = c.attend(window=window)
    for r in range(c.R):
        c.check(got, r, window=window)


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("page", [16, 64])
def test_attend_over_listed_pages(io, cache, page):
    """Different pages for each kv head; -1 behind the list, -1 and unheld pages inside it."""
    lens = [0, 1, 40, 500, 1030, 2000]
    c = Cache(lens, H=2, G=4, D=128, page=page, io=io, cache=cache, seed=3)
    rng, keep = random.Random(4), 9
    lists = []
    for r, n in enumerate(lens):
        per = []
        for h in range(c.H):
            held = pages_of(n, page)
            chosen = sorted(rng.sample(range(held), min(held, keep)))
            if r == 3:
                chosen[2] = -1
            if r == 4:
                chosen[-1] = held + 5
            if r == 5 and h == 1:
                chosen = [-1] * keep                     # a head that attends to nothing
            per.append(chosen + [-1] * (keep - len(chosen)))
        lists.append(per)
    got = c.attend(pages=i32(lists))
    for r in range(c.R):
        c.check(got, r, listed=lists[r])


def test_attend_touches_the_listed_owners_only():
    c = Cache([40, 100, 0, 33, 257, 12], H=2, G=2, D=64, page=32, io="bf16", cache="bf16", seed=8)
    rows = [4, 2, -1, 0, 77]                             # out of range ids are passed over
    out, lse = c.attend(rows=i32(rows))
    for r in range(c.R):
        if r in rows:
            c.check((out, lse), r)
        else:
            assert bool((out[r] == 7).all()) and bool((lse[r] == 7).all())
    full = c.attend()
    assert torch.equal(full[0][0], out[0]) or torch.allclose(full[0][0].float(), out[0].float(), rtol=2 ** -7)


def test_attend_strides():
    """q is part of a wider projection, out of a wider buffer."""
    c = Cache([70, 3, 200], H=2, G=2, D=64, page=16, io="bf16", cache="bf16", seed=9)
    wide_q = torch.randn((c.R, 3, 4, 64), device="cuda").to(torch.bfloat16)
    wide_q[:, 1] = dev(c.q_h)
    wide_o = torch.full((c.R, 5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    _, lse = c.attend(q=wide_q[:, 1], out=wide_o[:, 2])
    host = wide_o.cpu()
    for r in range(c.R):
        c.check((host[:, 2], lse), r)
    assert bool((host[:, [0, 1, 3, 4]] == 7).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attend_scales(scale):
    c = Cache([70, 1, 500], H=1, G=4, D=64, page=16, io="f32", cache="f32", seed=10)
    got = c.attend(scale=scale)
    for r in range(c.R):
        c.check(got, r, scale=scale)


def test_attend_infinite_and_missing_scores():
    """-inf scores weigh nothing; a row of them alone gives 0 and -inf; +inf and NaN give NaN."""
    c = Cache([40, 40, 40, 40], H=1, G=1, D=64, page=64, io="f32", cache="f32", seed=11, poison=False)
    q = torch.ones((4, 1, 64))
    k = c.k.clone()
    for r in range(4):
        k[int(c.table_h[r, 0])] = 0.1
    page = [int(c.table_h[r, 0]) for r in range(4)]
    k[page[0], 0, 3, 5] = -torch.inf
    k[page[1], 0, :, 5] = -torch.inf
    k[page[2], 0, 3, 5] = torch.inf
    k[page[3], 0, 3, 5] = torch.nan
    c.kd.copy_(k)
    out, lse = c.attend(q=dev(q))
    v = c.v[page[0], 0, :40].double()
    keep = [j for j in range(40) if j != 3]
    assert torch.allclose(out[0, 0].double(), v[keep].mean(dim=0), atol=1e-5)
    assert bool((out[1] == 0).all()) and float(lse[1, 0]) == -np.inf
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3]).all())


def test_attend_lowest_values_and_large_scores():
    """Keys at the type's lowest value and scores of +-1000: no overflow on the way."""
    c = Cache([100, 64], H=1, G=2, D=64, page=32, io="f32", cache="f32", seed=12, std=30.0)
    c.q_h = c.q_h * 30
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)


def test_attend_offsets_beyond_32_bits():
    """Pages of a cache whose bytes and elements pass 2^32."""
    H, D, page, N = 8, 128, 64, 70000
    lens = [130, 64]
    c = Cache(lens, H=H, G=4, D=D, page=page, io="bf16", cache="bf16", seed=13)
    big_k = torch.empty((N, H, page, D), dtype=torch.bfloat16, device="cuda")
    big_v = torch.empty((N, H, page, D), dtype=torch.bfloat16, device="cuda")
    far = [N - 1, 35000, N - 7, 69000]
    table = torch.zeros((2, c.MP), dtype=torch.int32)
    at = 0
    for r, n in enumerate(lens):
        for j in range(pages_of(n, page)):
            big_k[far[at]] = c.k[int(c.table_h[r, j])].cuda()
            big_v[far[at]] = c.v[int(c.table_h[r, j])].cuda()
            table[r, j] = far[at]
            at += 1
    c.N = N
    c.kd, c.vd, c.table = big_k, big_v, dev(table)
    c.close()
    c.kv = c.handle()
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)


def test_attend_equal_calls_give_equal_bits_on_any_stream():
    c = Cache([9000, 3, 0, 777], H=2, G=4, D=128, page=64, io="bf16", cache="bf16", seed=14)
    first = c.attend()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            again = c.attend()
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16))
        assert torch.equal(first[1], again[1])


@pytest.mark.parametrize("lens,H", [([60000], 1), ([9000, 3, 0, 777, 20000, 4500], 2), ([4200] * 8, 8)])
def test_attend_calls_in_turn_see_their_own_partial_results(lens, H):
    """Three queries in turn on one handle, nothing waited for in between: what one call
    leaves in the workspace is never taken for another's."""
    c = Cache(lens, H=H, G=4, D=128, page=64, io="bf16", cache="bf16", seed=15, poison=False)
    g = torch.Generator().manual_seed(2)
    qs = [dev((torch.randn(c.q_h.shape, generator=g) * (1 + i)).to(torch.bfloat16)) for i in range(3)]
    first = [c.attend(q=q) for q in qs]
    outs = [torch.zeros((c.R, c.H * c.G, c.D), dtype=torch.bfloat16, device="cuda") for _ in range(30)]
    for i, out in enumerate(outs):
        q = qs[i % 3]
        ok(KV.rwttt_kv_attend(c.kv, 0, q.data_ptr(), q.stride(0), c.lengths.data_ptr(), 0, c.R, c.D ** -0.5, 0, 0, 0,
                              out.data_ptr(), out.stride(0), 0, stream()))
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out.cpu().view(torch.int16), first[i % 3][0].view(torch.int16)), i


# ---------------------------------------------------------------------------
# extend
# ---------------------------------------------------------------------------

def run_extend(have, want, front, count, table, ring, page, cap):
    n, N, MP = len(have), len(ring), len(table[0])
    t, f = i32(table), i32(ring)
    cfg = KV.make_kv_config(n, 1, N, page, MP, 1, 1, 64, R.RWTTT_BF16, R.RWTTT_BF16, table=t.data_ptr(),
                            ring=f.data_ptr())
    kv = KV.rwttt_kv_create(cfg)
    h, w, pos = i32(have), i32(want), i32([front, count])
    o = {"pos": i32([9, 9]), "lengths": i32([9] * n), "start": i32([9] * (n + 1)), "result": i32([9] * 4),
         "slots": i32([9] * max(1, cap)), "owners": i32([9] * max(1, cap)), "positions": i32([9] * max(1, cap))}
    for _ in range(2):       # the inputs stay as they are: a call may be repeated
        ok(KV.rwttt_kv_extend(kv, h.data_ptr(), w.data_ptr(), pos.data_ptr(), o["pos"].data_ptr(),
                              o["lengths"].data_ptr(), o["start"].data_ptr(), o["slots"].data_ptr(),
                              o["owners"].data_ptr(), o["positions"].data_ptr(), cap, o["result"].data_ptr(),
                              stream()))
    torch.cuda.synchronize()
    KV.rwttt_kv_destroy(kv)
    got = {k: x.cpu().tolist()[:cap] if k in ("slots", "owners", "positions") else x.cpu().tolist()
           for k, x in o.items()}
    return dict(got, table=t.cpu().tolist(), ring=f.cpu().tolist())


def extend_case(rng, n, page, MP, top, front=None):
    have = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, MP * page)]) for _ in range(n)]
    want = [min(MP * page, max(0, rng.choice([h, h + 1, 0, h + rng.randint(0, top), h - rng.randint(0, top)])))
            for h in have]
    used = [pages_of(h, page) for h in have]
    N = sum(used) + sum(max(0, pages_of(w, page) - u) for w, u in zip(want, used)) + rng.randint(1, 4)
    deal = rng.sample(range(N), N)
    table, at = [], 0
    for u in used:
        table.append(deal[at:at + u] + [-5] * (MP - u))
        at += u
    front = rng.randrange(N) if front is None else front
    ring = [-1] * N
    for i, p in enumerate(deal[at:]):
        ring[(front + i) % N] = p
    return have, want, front, N - at, table, ring


@pytest.mark.parametrize("n,page,MP,top", [(1, 16, 4, 20), (2, 16, 3, 40), (8, 64, 20, 200), (63, 32, 9, 64),
                                           (257, 16, 6, 30), (1000, 128, 5, 300), (4096, 16, 3, 20)])
def test_extend_matches_the_book(n, page, MP, top):
    for seed in range(4):
        rng = random.Random(100 * n + seed)
        have, want, front, count, table, ring = extend_case(rng, n, page, MP, top)
        cap = sum(max(0, w - h) for h, w in zip(have, want)) + rng.choice([0, 1, 77])
        ref = extend_ref(have, want, front, count, table, ring, page, cap)
        got = run_extend(have, want, front, count, table, ring, page, cap)
        assert ref["result"][0] == 0
        for k in ref:
            assert got[k] == ref[k], (k, seed)


def test_extend_fills_lists_longer_than_a_block():
    n, page, MP = 3, 16, 2000
    have, want = [0, 5, 20000], [30000, 31000, 7]
    used = [pages_of(h, page) for h in have]
    N = 6000
    deal = random.Random(1).sample(range(N), N)
    table, at = [], 0
    for u in used:
        table.append(deal[at:at + u] + [0] * (MP - u))
        at += u
    ring = deal[at:] + [-1] * at
    ref = extend_ref(have, want, 0, N - at, table, ring, page, 70000)
    got = run_extend(have, want, 0, N - at, table, ring, page, 70000)
    for k in ref:
        assert got[k] == ref[k], k


def test_extend_returns_and_takes_many_pages_without_a_map():
    """All owners end at once in a large cache: no new rows, 40000 pages; then they grow
    again past the ring's end, the maps alone too small."""
    page, MP, N = 16, 900, 41000
    rng = random.Random(2)
    have = [16 * 800 - rng.randint(0, 15) for _ in range(50)]
    deal = rng.sample(range(N), N)
    table = [deal[800 * r:800 * (r + 1)] + [-5] * 100 for r in range(50)]
    front = N - 300
    ring = [-1] * N
    for i, p in enumerate(deal[40000:]):
        ring[(front + i) % N] = p
    for want in ([0] * 50, [rng.choice([0, 5, 16 * 400]) for _ in range(50)]):
        ref = extend_ref(have, want, front, 1000, table, ring, page, 0)
        got = run_extend(have, want, front, 1000, table, ring, page, 0)
        assert ref["result"][0] == 0 and ref["result"][3] > 20000
        for k in ref:
            assert got[k] == ref[k], k
    refused = run_extend([0] * 50, [3] * 50, got["pos"][0], got["pos"][1], got["table"], got["ring"], page, 149)
    assert refused["result"] == [-7, 0, 0, 0] and refused["ring"] == got["ring"]


def test_extend_that_does_not_fit_changes_nothing():
    page, MP = 16, 4
    table = [[0, 1, -5, -5], [2, -5, -5, -5]]
    ring = [3, 4, 5, -1, -1, -1]
    fits = ([20, 10], [40, 30], 0, 3, table, ring, page, 40)
    assert extend_ref(*fits)["result"] == [0, 40, 2, 0]
    for bad in [([20, 10], [64, 64], 0, 3, table, ring, page, 200),           # pages
                ([20, 10], [40, 30], 0, 3, table, ring, page, 39),            # cap
                ([20, 10], [65, 10], 0, 3, table, ring, page, 200),           # longer than an owner may be
                ([20, -1], [40, 10], 0, 3, table, ring, page, 200),
                ([20, 10], [40, -2], 0, 3, table, ring, page, 200),
                ([20, 10], [40, 30], 6, 3, table, ring, page, 200),           # ring position
                ([20, 10], [40, 30], -1, 3, table, ring, page, 200),
                ([20, 10], [40, 30], 0, 7, table, ring, page, 200),
                ([20, 10], [0, 0], 0, 6, table, ring, page, 200)]:            # more pages than there are
        ref = extend_ref(*bad)
        assert ref["result"][0] < 0
        got = run_extend(*bad)
        for k in ref:
            assert got[k] == ref[k], (k, bad)


def test_extend_without_maps():
    got = run_extend([16], [3], 1, 1, [[0, -5]], [-1, 1, -1], 16, 0)
    assert got["result"] == [0, 0, 0, 0] and got["lengths"] == [3]


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

def append_case(c, new, seed, pad=0, dup=None):
    """Slots of `new[r]` tokens behind each owner's length, and their rows."""
    slots = []
    for r, n in enumerate(new):
        for j in range(c.lens[r], c.lens[r] + n):
            slots.append(int(c.table_h[r, j // c.page]) * c.page + j % c.page)
    slots += [-1] * pad
    g = torch.Generator().manual_seed(seed)
    kv = (torch.randn((len(slots), 2, c.H, c.D), generator=g) * 1.5).to(DT[c.io])
    return slots, kv


def cache_with_room(lens, new, **kw):
    """A cache whose owners already hold the pages of their new tokens."""
    c = Cache([a + b for a, b in zip(lens, new)], poison=False, **kw)
    c.lens = lens
    return c


def check_append(c, slots, kv, got_k, got_v, got_b, old_b):
    k, v = stored(kv[:, 0], c.k_scale_h, c.cache), stored(kv[:, 1], c.v_scale_h, c.cache)
    bits = {"f32": torch.int32, "bf16": torch.int16, "fp8": torch.uint8}[c.cache]
    ref_k, ref_v = c.k.clone().view(bits), c.v.clone().view(bits)
    for t, s in enumerate(slots):
        if 0 <= s < c.N * c.page:
            ref_k[s // c.page, :, s % c.page] = k[t].view(bits)
            ref_v[s // c.page, :, s % c.page] = v[t].view(bits)
    for got, ref in ((got_k, ref_k), (got_v, ref_v)):
        nan = torch.isnan(ref.view(DT[c.cache]).float())          # a NaN's other bits are free
        assert torch.equal(nan, torch.isnan(got.float()))
        assert torch.equal(got.view(bits)[~nan], ref[~nan])
    live = [s if 0 <= s < c.N * c.page else -1 for s in slots]
    ref = bounds_ref(old_b, k, live, c.k_scale_h, c.step_h, c.cache, c.page)
    assert np.array_equal(got_b.numpy(), ref)


def run_append(c, slots, kv):
    old = torch.randint(-90, 91, c.bounds_h.shape, dtype=torch.int8, generator=torch.Generator().manual_seed(6))
    c.bounds.copy_(old)
    d, s = dev(kv), i32(slots)
    k, v = d[:, 0], d[:, 1]
    for _ in range(2):       # storing the same rows again changes nothing
        ok(KV.rwttt_kv_append(c.kv, 0, k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), s.data_ptr(),
                              len(slots), stream()))
    torch.cuda.synchronize()
    check_append(c, slots, kv, c.kd.cpu(), c.vd.cpu(), c.bounds.cpu(), old)


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_append_stores_rows_and_bounds(io, cache, D):
    lens, new = [0, 1, 15, 16, 100, 31, 0], [1, 1, 1, 1, 1, 70, 33]
    c = cache_with_room(lens, new, H=3, G=1, D=D, page=16 if D == 64 else 64, io=io, cache=cache, seed=D)
    slots, kv = append_case(c, new, 2, pad=3)
    run_append(c, slots, kv)


@pytest.mark.parametrize("page", [16, 128, 256])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_append_of_a_prefill(page, cache):
    """More tokens than the short path takes, pages that begin and end inside a wave's run."""
    lens, new = [0, 3, 250, 1000, 17], [700, 513, 255, 1, 90]
    c = cache_with_room(lens, new, H=2, G=1, D=64, page=page, io="bf16", cache=cache, seed=page)
    slots, kv = append_case(c, new, 3, pad=1)
    run_append(c, slots, kv)


def test_append_special_values_and_foreign_slots():
    """Overflow, infinities, NaN and signed zeros; slots outside the cache are skipped."""
    for cache in ("bf16", "fp8"):
        lens, new = [0, 10], [40, 5]
        c = cache_with_room(lens, new, H=2, G=1, D=64, page=16, io="bf16", cache=cache, seed=4)
        slots, kv = append_case(c, new, 5, pad=2)
        slots[15] = c.N * c.page                         # a page's last row and a page's first
        slots[32] = -9
        for i, x in enumerate([float("inf"), float("-inf"), float("nan"), 1e30, -1e30, -0.0, 1e-30]):
            kv[1 + 3 * i, 0, i % 2, 11 + i] = x
        run_append(c, slots, kv)


# ---------------------------------------------------------------------------
# select
# ---------------------------------------------------------------------------

def run_select(c, keep, first, last, rows=None, q=None, spread=90):
    g = torch.Generator().manual_seed(keep)
    lo = torch.randint(-spread, spread, (c.N, c.H, 1, c.D), generator=g)
    hi = lo + torch.randint(0, spread, (c.N, c.H, 1, c.D), generator=g)
    b = torch.cat([lo, hi], dim=2).clamp(-127, 127).to(torch.int8)
    c.bounds.copy_(b)
    q = c.q_h if q is None else q
    dq = dev(q)
    out = torch.full((c.R, c.H, keep), 99, dtype=torch.int32, device="cuda")
    ok(KV.rwttt_kv_select(c.kv, 0, dq.data_ptr(), dq.stride(0), c.lengths.data_ptr(),
                          0 if rows is None else rows.data_ptr(), c.R if rows is None else rows.numel(), first, last,
                          keep, out.data_ptr(), stream()))
    torch.cuda.synchronize()
    out = out.cpu()
    for r in range(c.R):
        for h in range(c.H):
            if rows is not None and r not in rows.tolist():
                assert bool((out[r, h] == 99).all())
                continue
            pages = c.table_h[r, :pages_of(c.lens[r], c.page)].long().numpy()
            ref = select_ref(q[r, h * c.G:(h + 1) * c.G].float().numpy(), b[:, h].numpy(), pages, first, last, keep)
            assert out[r, h].tolist() == ref, (r, h)
    return out


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G", [(64, 2, 1), (128, 1, 5), (256, 2, 16)])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 1, 0), (7, 1, 2), (64, 0, 4), (33, 3, 30)])
def test_select_matches_the_book(io, D, H, G, keep, first, last):
    lens = [0, 1, 16, 17, 7 * 16, 7 * 16 + 1, 64 * 16, 65 * 16, 333 * 16 - 3]
    c = Cache(lens, H=H, G=G, D=D, page=16, io=io, cache="bf16" if io == "bf16" else "f32", seed=keep + D,
              poison=False)
    run_select(c, keep, first, last)


def test_select_ties_go_to_the_lowest_page():
    """Bounds of few values: nearly all scores tie."""
    c = Cache([500 * 16], H=2, G=4, D=64, page=16, io="bf16", cache="bf16", seed=2, poison=False)
    run_select(c, 50, 1, 1, spread=1)
    run_select(c, 51, 0, 0, q=torch.zeros_like(c.q_h))          # no score at all


def test_select_many_heads_in_a_group_and_long_tables():
    c = Cache([9000 * 16, 100], H=1, G=128, D=64, page=16, io="bf16", cache="bf16", seed=7, poison=False)
    run_select(c, 257, 1, 2)
    c = Cache([40, 20000 * 16 + 3], H=1, G=4, D=64, page=16, io="bf16", cache="fp8", seed=8, poison=False,
              max_pages=32768)
    run_select(c, 1000, 1, 2)


@pytest.mark.parametrize("lens", [[601], [1999, 512, 513, 1], [2048, 2047], [4099, 77, 260]])
def test_select_shared_by_several_blocks(lens):
    """Few rows and wide tables: parts of odd sizes, parts without pages; twice, since
    each call has to leave the counters as it found them."""
    c = Cache([16 * n - 5 for n in lens], H=2, G=4, D=64, page=16, io="bf16", cache="fp8", seed=len(lens), poison=False,
              max_pages=max(4200, max(lens)))
    for keep in (3, 64, 250, 599):
        run_select(c, keep, 1, 2)


def test_select_without_a_workspace_or_with_owners_listed_twice():
    c = Cache([16 * 900 - 5, 16 * 300], H=1, G=4, D=64, page=16, io="bf16", cache="fp8", seed=3, poison=False,
              max_pages=2000)
    first = run_select(c, 64, 1, 2)
    assert torch.equal(first, run_select(c, 64, 1, 2, rows=i32([0, 1, 1, 0, 0])))
    c.no_workspace = True
    c.close()
    c.kv = c.handle()
    assert torch.equal(first, run_select(c, 64, 1, 2))


def test_select_touches_the_listed_owners_only():
    c = Cache([300, 20, 700, 600], H=2, G=2, D=64, page=16, io="bf16", cache="bf16", seed=9, poison=False)
    run_select(c, 5, 1, 1, rows=i32([3, 0]))


# ---------------------------------------------------------------------------
# the step together
# ---------------------------------------------------------------------------

def test_selected_bounds_hold_the_pages_keys():
    """What append keeps bounds every stored key, so a score bounds the logits."""
    lens, new = [0, 0], [100, 37]
    c = cache_with_room(lens, new, H=2, G=2, D=64, page=16, io="bf16", cache="bf16", seed=1)
    slots, kv = append_case(c, new, 1)
    d, s = dev(kv), i32(slots)
    ok(KV.rwttt_kv_append(c.kv, 0, d[:, 0].data_ptr(), d.stride(0), d[:, 1].data_ptr(), d.stride(0), s.data_ptr(),
                          len(slots), stream()))
    torch.cuda.synchronize()
    step = c.step_h.double()[None, :, None]
    b = c.bounds.cpu().double() * step[..., None]
    k = kv[:, 0].double().clamp(-127 * step, 127 * step)          # the bounds' range
    for t, slot in enumerate(slots):
        assert bool((k[t] >= b[slot // 16, :, 0] - 1e-6).all()) and bool((k[t] <= b[slot // 16, :, 1] + 1e-6).all())


def test_a_captured_step_replays():
    """extend, append, select and attend in one graph, replayed with new inputs in place."""
    page, H, G, D, R_, keep = 16, 2, 4, 64, 3, 4
    c = Cache([30, 100, 200], H=H, G=G, D=D, page=page, io="bf16", cache="bf16", seed=20, extra_pages=40,
              poison=False, max_pages=40)
    c.bounds.copy_(torch.randint(-90, 0, c.bounds_h.shape, dtype=torch.int8))
    have, want, pos = i32(c.lens), i32([31, 101, 201]), i32([0, 40])
    new_pos, lengths, start, result = i32([0, 0]), i32([0] * 3), i32([0] * 4), i32([0] * 4)
    slots, owners, positions = (i32([0] * 4) for _ in range(3))
    kv = torch.zeros((4, 2, H, D), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((3, H * G, D), dtype=torch.bfloat16, device="cuda")
    pages = i32([[[0] * keep] * H] * 3)
    out = torch.zeros_like(q)

    def step():
        s = stream()
        ok(KV.rwttt_kv_extend(c.kv, have.data_ptr(), want.data_ptr(), pos.data_ptr(), new_pos.data_ptr(),
                              lengths.data_ptr(), start.data_ptr(), slots.data_ptr(), owners.data_ptr(),
                              positions.data_ptr(), 4, result.data_ptr(), s))
        ok(KV.rwttt_kv_append(c.kv, 0, kv[:, 0].data_ptr(), kv.stride(0), kv[:, 1].data_ptr(), kv.stride(0),
                              slots.data_ptr(), 4, s))
        ok(KV.rwttt_kv_select(c.kv, 0, q.data_ptr(), q.stride(0), lengths.data_ptr(), 0, 3, 1, 2, keep,
                              pages.data_ptr(), s))
        ok(KV.rwttt_kv_attend(c.kv, 0, q.data_ptr(), q.stride(0), lengths.data_ptr(), 0, 3, D ** -0.5, 0,
                              pages.data_ptr(), keep, out.data_ptr(), out.stride(0), 0, s))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in range(5):
        kv.copy_(torch.randn(kv.shape))
        q.copy_(torch.randn(q.shape))
        graph.replay()
        torch.cuda.synchronize()
        got, chosen = out.clone(), pages.clone()
        state = [x.clone() for x in (c.kd, c.vd, c.bounds, c.table, c.ring)]
        step()                                           # the same step again, eagerly
        torch.cuda.synchronize()
        assert result.tolist()[0] == 0
        assert torch.equal(got.view(torch.int16), out.view(torch.int16)) and torch.equal(chosen, pages)
        for x, y in zip(state, (c.kd, c.vd, c.bounds, c.table, c.ring)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        have.copy_(lengths)                              # adopt the step
        pos.copy_(new_pos)
        want.copy_(have + i32([1, 1, 1 if t % 2 else -17]))
