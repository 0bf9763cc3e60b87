"""Caches of one 16-row page an owner: the smallest there are."""

import pytest

from tests.kv_util import Cache

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "bf16"), ("f32", "fp8")]


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("owners", [1, 2, 8, 64, 500])
def test_attend_writes_every_row(io, cache, owners):
    """Lengths 0 to 16 (one owner: 10); the outputs hold 7 before the call."""
    lens = [10] if owners == 1 else [(5 * r + 3) % 17 for r in range(owners)]
    c = Cache(lens, H=1, G=3, D=64, page=16, io=io, cache=cache, seed=owners, max_pages=1)
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)
    again = c.attend(window=3)
    for r in range(c.R):
        c.check(again, r, window=3)
    c.close()
