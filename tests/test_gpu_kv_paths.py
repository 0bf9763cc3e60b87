"""The paged cache's kernels at the sizes where they take their other paths: prefills of more
tokens than a wave holds, joins of more columns than a block has threads, loads with the hint."""

import pytest
import torch

from tests.kv_util import Cache
from tests.test_gpu_kv import TYPES, append_case, cache_with_room, run_append

pytestmark = pytest.mark.gpu


def prefill(io, cache, H, D, page, tokens, seed):
    """Five ragged owners that gain `tokens` rows: pages that begin and end inside a wave's
    run, that span several runs, and one single new row."""
    lens = [0, 3, 250, 1000, 17]
    new = [tokens // 2, 513, 255, 1]
    new.append(tokens - sum(new))
    assert min(new) > 0
    c = cache_with_room(lens, new, H=H, G=1, D=D, page=page, io=io, cache=cache, seed=seed)
    slots, kv = append_case(c, new, 3, pad=5)
    slots[page - 1] = c.N * page                         # a slot outside the cache, at a page's end
    run_append(c, slots, kv)
    c.close()


def rows_a_load(io, D):
    return 64 * (8 if io == "bf16" else 4) // D


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_append_of_a_prefill_of_one_load_a_wave(io, cache, D):
    """More than 4096 pairs of a token and a head: a wave takes as many tokens as it loads at once."""
    H, tokens = 3, 1800
    assert 4096 < H * tokens < 4 * 4096 * rows_a_load(io, D)
    prefill(io, cache, H, D, 64, tokens, D)


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 256])
def test_append_of_a_prefill_of_four_loads_a_wave(io, cache, D, page):
    tokens = 2100
    H = -(-4 * 4096 * rows_a_load(io, D) // tokens)
    assert H * tokens >= 4 * 4096 * rows_a_load(io, D)
    prefill(io, cache, H, D, page, tokens, page)


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D,G", [(64, 16), (128, 16), (256, 16), (256, 5), (128, 17)])
def test_rows_of_many_columns_are_split_and_joined(io, cache, D, G):
    """Sixteen queries of 128 or 256 channels have more columns than a block threads; the long
    row is held by more blocks than are joined at once, the others by a few."""
    c = Cache([20000, 0, 1, 2100, 700], H=1, G=G, D=D, page=64, io=io, cache=cache, seed=D + G)
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)
    again = c.attend()
    assert torch.equal(got[0].float(), again[0].float()) and torch.equal(got[1], again[1])
    c.close()


@pytest.mark.parametrize("io,cache", TYPES)
@pytest.mark.parametrize("D", [64, 256])
def test_attend_in_a_large_pool(io, cache, D):
    """A pool of more than 64 MB, which the owners could hold: its rows are loaded with the hint."""
    H, page, size = 2, 64, {"f32": 4, "bf16": 2, "fp8": 1}[cache]
    extra = (65 << 20) // (2 * H * page * D * size)
    c = Cache([0, 1, 40, 3000, 257, 700], H=H, G=3, D=D, page=page, io=io, cache=cache, seed=D, extra_pages=extra,
              poison=False, max_pages=extra)
    assert 2 * c.N * H * page * D * size > 64 << 20
    got = c.attend()
    for r in range(c.R):
        c.check(got, r)
    windowed = c.attend(window=100)
    for r in range(c.R):
        c.check(windowed, r, window=100)
    c.close()
