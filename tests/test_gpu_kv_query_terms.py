"""Queries in fp32 over caches of fewer bits: their terms have one sign, so that a score of -inf
stays one."""

import math

import pytest
import torch

from tests.kv4_util import Cache4
from tests.kv_util import Cache, dev

pytestmark = pytest.mark.gpu

N, CHANNEL, AT = 70, 5, 33
# of 1, 2 and 3 terms of 8 bits, nearest ones of both signs; the largest, which bf16 rounds to infinity
LARGE = [2.0 ** 126, 2.0 ** 126 * (1 + 3 * 2.0 ** -9), 2.0 ** 126 * (1 + 3 * 2.0 ** -9 - 2.0 ** -18),
         2.0 ** 127 * (1 + 2.0 ** -8 + 2.0 ** -23), float(torch.finfo(torch.float32).max)]


def build(cache, D, owners, low):
    """Keys of one small positive number, 0 in CHANNEL but for the rows of `low` (owner -> rows): there
    the lowest a key may be, or 2^102 of it."""
    if cache == "fp4":
        c = Cache4([N] * owners, H=1, G=1, D=D, page=16, io="f32", seed=D, bounds=False)
        c.code["k"][..., :] = 1
        c.code["k"][..., :32] = 0
        c.E["k"][c.E["k"] != 255] = 125
        for r, rows in low.items():
            for j in rows:
                page = int(c.table_h[r, j // 16])
                c.code["k"][page, 0, j % 16, CHANNEL], c.E["k"][page, 0, j % 16, 0] = 15, 227
        c.close()
        c.upload()
        return c
    c = Cache([N] * owners, H=1, G=1, D=D, page=16, io="f32", cache=cache, seed=D)
    k = c.k.float()
    k = torch.where(torch.isnan(k), k, 0.125)
    k[..., :32] = torch.where(torch.isnan(k[..., :32]), k[..., :32], 0.0)
    for r, rows in low.items():
        for j in rows:
            k[int(c.table_h[r, j // 16]), 0, j % 16, CHANNEL] = -448.0 if cache == "fp8" else -6 * 2.0 ** 100
    c.kd.copy_(k.to(c.k.dtype))
    return c


@pytest.mark.parametrize("cache", ["fp4", "fp8", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_score_of_minus_infinity_weighs_nothing(cache, D, sign):
    """One row whose product is beyond fp32 among rows of equal scores, and rows that all are."""
    owners = 2 * len(LARGE)
    low = {r: [AT] if r < len(LARGE) else range(N) for r in range(owners)}
    c = build(cache, D, owners, low)
    q = torch.ones((owners, 1, D))
    q[:, 0, CHANNEL] = sign * torch.tensor(LARGE * 2, dtype=torch.float64).float()
    out, lse = c.attend(q=dev(q), scale=sign * D ** -0.5)
    rest = [j for j in range(N) if j != AT]
    for r in range(owners):
        if r < len(LARGE):
            v = c.rows_of(r, 0, "v", rest)
            # weights of 1/69 each, rounded, and a sum of 69 products in fp32
            assert bool(((out[r, 0].double() - v.mean(dim=0)).abs() <= 200 * 2.0 ** -24 * v.abs().amax()).all()), r
            # the other channels' score, the same in all rows
            assert math.isfinite(float(lse[r, 0])), r
        elif cache != "fp8":                 # an 8-bit key times its scale is not as large
            assert bool((out[r] == 0).all()) and float(lse[r, 0]) == -math.inf, r
    c.close()


@pytest.mark.parametrize("cache", ["fp4", "fp8", "bf16"])
@pytest.mark.parametrize("D", [64, 256])
def test_queries_that_are_not_finite(cache, D):
    """Infinite: against keys of the other sign all scores are -inf, of the same sign +inf.  NaN, also where only its
    last bit is set: NaN."""
    c = build(cache, D, 4, {r: range(N) for r in range(4)})
    q = torch.ones((4, 1, D))
    q[0, 0, CHANNEL], q[1, 0, CHANNEL], q[2, 0, CHANNEL] = math.inf, -math.inf, math.nan
    q.view(torch.int32)[3, 0, CHANNEL] = 0x7f800001
    out, lse = c.attend(q=dev(q))
    assert bool((out[0] == 0).all()) and float(lse[0, 0]) == -math.inf
    for r in (1, 2, 3):
        assert bool(torch.isnan(out[r]).all()) and math.isnan(float(lse[r, 0])), r
    c.close()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("x", [1.0, -1.0, 1 + 2.0 ** -9, 0.3, -2.0 ** -60, 2.0 ** 100])
def test_infinite_keys(D, x):
    """Stored in bf16, against queries of one, two and three terms: -inf in a row weighs nothing, in all rows
    it gives 0 and -inf, +inf and a NaN give NaN, and behind the rows they have no influence."""
    kinds = [("low", [AT]), ("low", [0]), ("low", [N - 1]), ("low", range(N)), ("high", [AT]), ("nan", [AT])]
    c = build("bf16", D, len(kinds), {})
    k = c.kd.cpu()
    # -inf where the product with x is
    value = {"low": -math.inf if x > 0 else math.inf, "high": math.inf if x > 0 else -math.inf, "nan": math.nan}
    k[torch.isnan(k)] = math.inf
    for r, (kind, rows) in enumerate(kinds):
        for j in rows:
            k[int(c.table_h[r, j // 16]), 0, j % 16, CHANNEL] = value[kind]
    c.kd.copy_(k)
    q = torch.ones((len(kinds), 1, D))
    q[:, 0, CHANNEL] = x
    out, lse = c.attend(q=dev(q))
    for r, (kind, rows) in enumerate(kinds):
        if kind != "low":
            assert bool(torch.isnan(out[r]).all()) and math.isnan(float(lse[r, 0])), r
        elif len(rows) == N:
            assert bool((out[r] == 0).all()) and float(lse[r, 0]) == -math.inf, r
        else:
            v = c.rows_of(r, 0, "v", [j for j in range(N) if j not in rows])
            assert bool(((out[r, 0].double() - v.mean(dim=0)).abs() <= 200 * 2.0 ** -24 * v.abs().amax()).all()), r
    c.close()
