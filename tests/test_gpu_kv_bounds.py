"""How far a page's key bounds hold its keys."""

import pytest
import torch

from tests.kv_util import dev, i32, ok, stream
from tests.test_gpu_kv import append_case, cache_with_room
from paper_2605_28053_amd import _rwttt_kv as KV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io,cache", [("f32", "f32"), ("f32", "bf16"), ("bf16", "fp8")])
def test_bounds_hold_keys_within_127_steps(io, cache):
    """Keys at multiples of the step, one and two units in the last place beside them, ordinary
    ones, and some beyond 127 steps.  A product with 1 / step has two roundings, 2^-24 each:
    a key sticks out by less than 2^-22 of itself, and beyond the range the bound is 127."""
    lens, new = [0, 5, 30], [100, 37, 300]
    c = cache_with_room(lens, new, H=2, G=1, D=64, page=16, io=io, cache=cache, seed=2)
    slots, kv = append_case(c, new, 1)
    g = torch.Generator().manual_seed(4)
    step = c.step_h[None, :, None]
    k = kv[:, 0].float()
    units = torch.randint(-130, 131, k.shape, generator=g).float() * step
    near = units * (1 + torch.randint(-2, 3, k.shape, generator=g) * 2.0 ** -23)
    k = torch.where(torch.rand(k.shape, generator=g) < 0.5, near, 3 * k)
    few = torch.rand((1, 1, c.D), generator=g) < 0.7                  # most channels stay in range
    kv[:, 0] = torch.where(few, k.clamp(-100 * step, 100 * step), k).to(kv.dtype)
    d, s = dev(kv), i32(slots)
    c.bounds.fill_(0)
    ok(KV.rwttt_kv_append(c.kv, 0, d[:, 0].data_ptr(), d.stride(0), d[:, 1].data_ptr(), d.stride(0), s.data_ptr(),
                          len(slots), stream()))
    torch.cuda.synchronize()
    b, held = c.bounds.cpu().double(), c.kd.cpu().float().double()
    if cache == "fp8":
        held = held * c.k_scale_h.double()[None, :, None, None]
    step = c.step_h.double()[:, None]
    inside = beyond = 0
    for slot in slots:
        x, (lo, hi) = held[slot // 16, :, slot % 16], b[slot // 16].unbind(1)
        fits = x.abs() <= 127 * step * (1 - 2.0 ** -22)
        slack = x.abs() * 2.0 ** -22
        assert bool(((lo * step <= x + slack) & (x - slack <= hi * step))[fits].all())
        assert bool((torch.where(x > 0, hi, -lo) == 127)[~fits].all())
        inside, beyond = inside + int(fits.sum()), beyond + int((~fits).sum())
    assert inside > 10 * beyond > 0
    c.close()
