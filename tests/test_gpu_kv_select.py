"""Page selection where scores are neighbours: exactly `keep` pages, and nothing written behind them."""

import numpy as np
import pytest
import torch

from tests.kv_util import Cache, dev, ok, pages_of, select_ref, stream
from paper_2605_28053_amd import _rwttt_kv as KV

pytestmark = pytest.mark.gpu
GUARD = 256


def select(c, q, keep, first, last):
    """The selection of all owners [R, H, keep]; the words around it stay as they are."""
    dq = dev(q)
    n = c.R * c.H * keep
    flat = torch.full((GUARD + n + GUARD,), 77, dtype=torch.int32, device="cuda")
    out = flat[GUARD:GUARD + n]
    ok(KV.rwttt_kv_select(c.kv, 0, dq.data_ptr(), dq.stride(0), c.lengths.data_ptr(), 0, c.R, first, last, keep,
                          out.data_ptr(), stream()))
    torch.cuda.synchronize()
    host = flat.cpu()
    assert bool((host[:GUARD] == 77).all()) and bool((host[GUARD + n:] == 77).all())
    return host[GUARD:GUARD + n].view(c.R, c.H, keep)


def check(c, q, b, keep, first, last):
    got = select(c, q, keep, first, last)
    for r in range(c.R):
        pages = c.table_h[r, :pages_of(c.lens[r], c.page)].long().numpy()
        for h in range(c.H):
            ref = select_ref(q[r, h * c.G:(h + 1) * c.G].float().numpy(), b[:, h].numpy(), pages, first, last, keep)
            assert got[r, h].tolist() == ref, (r, h, keep, first, last)


@pytest.mark.parametrize("max_pages", [21, 2048])           # one block a row, and several
@pytest.mark.parametrize("values", [2, 3])
def test_every_number_of_pages_of_neighbouring_scores(max_pages, values):
    """Scores of 0, 1 and 2: one channel sets the queries' unit, another one the score."""
    n = 20
    c = Cache([16 * n] * 6, H=2, G=1, D=64, page=16, io="f32", cache="f32", seed=1, poison=False, max_pages=max_pages)
    g = torch.Generator().manual_seed(values)
    b = torch.zeros((c.N, c.H, 2, c.D), dtype=torch.int8)
    b[:, :, :, 1] = torch.randint(0, values, (c.N, c.H, 1), generator=g, dtype=torch.int8)
    c.bounds.copy_(b)
    q = torch.zeros((c.R, c.H, c.D))
    q[:, :, 0], q[:, :, 1] = 127.0, 1.0
    for keep in range(1, n):
        for first, last in [(0, 0), (1, 0), (1, 2)]:
            if first + last <= keep:
                check(c, q, b, keep, first, last)
    c.close()


def test_neighbouring_scores_of_rows_that_several_blocks_share():
    """1500 pages, the cut at every place among scores that are neighbours."""
    n = 1500
    c = Cache([16 * n, 16 * n - 9], H=1, G=1, D=64, page=16, io="f32", cache="f32", seed=2, poison=False, max_pages=2048)
    g = torch.Generator().manual_seed(5)
    b = torch.zeros((c.N, c.H, 2, c.D), dtype=torch.int8)
    b[:, :, :, 1] = torch.randint(0, 3, (c.N, c.H, 1), generator=g, dtype=torch.int8)
    c.bounds.copy_(b)
    q = torch.zeros((c.R, c.H, c.D))
    q[:, :, 0], q[:, :, 1] = 127.0, 1.0
    for r in range(c.R):
        pages = c.table_h[r, :n].long()
        twos, ones = (int((b[pages, 0, 0, 1] >= x).sum()) for x in (2, 1))
        for keep in (twos - 1, twos, twos + 1, ones - 1, ones, ones + 1):
            check(c, q, b, keep, 0, 0)
    c.close()


@pytest.mark.parametrize("io,cache", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n,keep", [(65, 64), (17, 16), (40, 30)])
def test_coarse_bounds(io, cache, n, keep):
    """Bounds of a few units, as a large step leaves them, under ordinary queries."""
    c = Cache([16 * n - 3] * 60, H=2, G=1, D=64, page=16, io=io, cache=cache, seed=n, poison=False)
    g = torch.Generator().manual_seed(keep)
    k = torch.randn((c.N, c.H, 16, c.D), generator=g)
    for step in (0.5, 1.0, 3.0):
        lo, hi = torch.floor(k.amin(dim=2) / step), torch.ceil(k.amax(dim=2) / step)
        b = torch.stack([lo, hi], dim=2).to(torch.int8)
        c.bounds.copy_(b)
        check(c, c.q_h, b, keep, 1, 2)
        one = torch.zeros_like(c.q_h)                       # few channels that count
        one[:, :, :2] = c.q_h[:, :, :2]
        check(c, one, b, keep, 1, 2)
    assert np.unique(b.numpy()).size < 12
    c.close()


@pytest.mark.parametrize("io,cache", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("size", [0.0, 1e-39, 3e-39, 1e-37, 3.5e-37])
def test_queries_too_small_for_a_unit_tie(io, cache, size):
    """All scores are 0 then, whatever the channels hold: the lowest pages, and the forced ones."""
    n, keep = 40, 9
    c = Cache([16 * n - 3] * 3, H=2, G=2, D=64, page=16, io=io, cache=cache, seed=3, poison=False)
    b = torch.randint(-90, 91, c.bounds_h.shape, dtype=torch.int8, generator=torch.Generator().manual_seed(1))
    c.bounds.copy_(b.sort(dim=2).values)
    q = torch.zeros_like(c.q_h)
    q[:, :, ::3] = size
    q[:, :, 1::3] = -size / 2
    got = select(c, q, keep, 1, 2)
    assert (got == torch.tensor(list(range(keep - 2)) + [n - 2, n - 1], dtype=torch.int32)).all()
    c.close()


@pytest.mark.parametrize("max_pages", [10960, 11500, 12288, 12289])
@pytest.mark.parametrize("D", [64, 256])
def test_tables_around_64_kb_of_lds(max_pages, D):
    """Where a block's scores and its other LDS pass what a launch has without asking."""
    c = Cache([16 * 1300, 16 * 40 - 3], H=1, G=2, D=D, page=16, io="bf16", cache="fp8", seed=D, poison=False,
              max_pages=max_pages)
    g = torch.Generator().manual_seed(1)
    b = torch.randint(-90, 91, c.bounds_h.shape, dtype=torch.int8, generator=g).sort(dim=2).values
    c.bounds.copy_(b)
    check(c, c.q_h, b, 30, 1, 2)
    c.close()
