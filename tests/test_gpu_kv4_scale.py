"""A scale of zero over a cache of 4 bits."""

import math

import pytest
import torch

from tests.kv4_util import Cache4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G", [3, 7, 12])
def test_products_of_any_size_weigh_alike(io, D, G):
    """q . k of up to 2^125, of both signs and far apart: at a scale of zero every row counts as much, in all
    of a context, in a window and behind a mask."""
    c = Cache4([1, 70, 0, 300], H=2, G=G, D=D, page=16, io=io, seed=D, spread=40)
    c.E["k"] = torch.where(c.E["k"] == 255, 255, c.E["k"] + 110)      # up to 6 * 2^109 a key
    c.close()
    c.upload()
    c.q_h = (c.q_h.float() * 2.0 ** 4).to(c.q_h.dtype)
    for kw in (dict(), dict(window=33)):
        got = c.attend(scale=0.0, **kw)
        for r in range(c.R):
            c.check(got, r, scale=0.0, **kw)
            n = min(c.lens[r], kw.get("window", c.lens[r]))
            # the logarithm of the number of rows, to 2 ulp of its base 2 and of the product
            want = math.log(n) if n else -math.inf
            assert all(x == want or abs(x - want) <= 2.0 ** -22 * want for x in got[1][r].double().tolist()), r
    c.close()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_what_is_not_finite_stays_so(io):
    """0 times an infinite or NaN query, or a NaN key: the head's out and lse are NaN, the others' are not."""
    c = Cache4([50, 50, 50], H=2, G=2, D=64, page=16, io=io, seed=1)
    c.q_h[0, 0, 3], c.q_h[1, 2, 40] = math.inf, math.nan
    c.E["k"][int(c.table_h[2, 1]), 1, 4, 0] = 255
    c.close()
    c.upload()
    out, lse = c.attend(scale=0.0)
    bad = torch.zeros((3, 4), dtype=torch.bool)
    bad[0, 0] = bad[1, 2] = bad[2, 2] = bad[2, 3] = True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(out).all(dim=2), bad)
    assert torch.isfinite(out[~bad]).all()
    c.close()
