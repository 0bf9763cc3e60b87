"""What the paged attention holds between its rounded inputs and its rounded output is fp32."""

import pytest
import torch

from tests.kv_util import Cache, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_probabilities_keep_the_bits_that_cancel(cache):
    """Three rows an owner: the largest score with values of 0, and two of nearly equal
    scores with values of 1 and -1, whose difference is what remains.

    The scores are exact (one product of 8 by 2 bits, one of the step delta).  A
    probability of fp32 arithmetic is off by 2^-22 of itself at most (its exponent, below
    1, is one product and one difference: 2^-23; the exponential as much), so out by
    2 * 2^-22 and its own rounding; probabilities of 16 bits would be off by up to 2^-17."""
    c = Cache([3] * 64, H=1, G=4, D=64, page=16, io="bf16", cache=cache, seed=1, poison=False)
    g = torch.Generator().manual_seed(2)
    step = 2.0 ** -6 if cache == "fp8" else 1.0                    # of a stored key
    delta = 2.0 ** -15 / step                                      # 2^-9 is the least e4m3 number
    c.k_scale_h.fill_(step)
    c.v_scale_h.fill_(1.0)
    k, v = torch.zeros(c.k.shape), torch.zeros(c.v.shape)
    for r in range(c.R):
        page = int(c.table_h[r, 0])
        a = (-0.65 * torch.rand((), generator=g) / step).to(c.k.dtype).float()
        k[page, 0, 1:3, 0] = a
        k[page, 0, 2, 1] = delta
        v[page, 0, 1], v[page, 0, 2] = 1.0, -1.0
    c.k, c.v = k.to(c.k.dtype), v.to(c.v.dtype)
    c.kd, c.vd, c.k_scale, c.v_scale = dev(c.k), dev(c.v), dev(c.k_scale_h), dev(c.v_scale_h)
    c.close()
    c.kv = c.handle()
    c.q_h.zero_()
    c.q_h[:, :, 0] = torch.tensor([1.0, 0.75, 0.5, 0.25]).to(torch.bfloat16)
    c.q_h[:, :, 1] = 1.0
    out, _ = c.attend(scale=1.0)
    worst = 0.0
    for r in range(c.R):
        ref = c.attend_ref(r, scale=1.0)[0]
        err = (out[r].double() - ref).abs() - 2.0 ** -8 * ref.abs()
        worst = max(worst, float(err.max()))
    assert worst <= 2.0 ** -21, worst
    c.close()
