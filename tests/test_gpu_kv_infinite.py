"""Scores that are infinite or NaN in rows that several blocks hold and join."""

import pytest
import torch

from tests.kv_util import Cache, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,n", [(64, 5000), (256, 3000)])
def test_infinite_scores_anywhere_in_a_split_row(D, n):
    """One -inf score weighs nothing, -inf alone gives 0 and -inf, +inf and NaN give NaN, each in
    the first rows, in the middle and in the last ones."""
    places = [0, 1, n // 2, n - 2, n - 1]
    kinds = [float("-inf"), float("inf"), float("nan")]
    cases = [(at, x) for at in places for x in kinds] + [(None, float("-inf"))]
    c = Cache([n] * len(cases), H=1, G=1, D=D, page=16, io="f32", cache="f32", seed=1, poison=False)
    k = torch.full(c.k.shape, 0.125)
    for r, (at, x) in enumerate(cases):
        pages = c.table_h[r, :-(-n // 16)].long()
        if at is None:
            k[pages, 0, :, 5] = x
        else:
            k[pages[at // 16], 0, at % 16, 5] = x
    c.kd.copy_(k)
    out, lse = c.attend(q=dev(torch.ones((c.R, 1, D))))
    for r, (at, x) in enumerate(cases):
        if at is None:
            assert bool((out[r] == 0).all()) and float(lse[r, 0]) == float("-inf")
        elif x == float("-inf"):
            v = c.rows_of(r, 0, "v", [j for j in range(n) if j != at])
            assert torch.allclose(out[r, 0].double(), v.mean(dim=0), atol=1e-5)
        else:
            assert bool(torch.isnan(out[r]).all()) and bool(torch.isnan(lse[r]).all()), (at, x)
    c.close()
