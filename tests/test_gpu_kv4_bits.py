"""All 24 bits of a probability over a cache of 4 bits, in every layout of its terms."""

import pytest
import torch

from tests.kv4_util import Cache4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 5, 6, 9, 21])
@pytest.mark.parametrize("top,one,other", [(0, 1, 2), (299, 1, 70), (10, 150, 290)])
def test_probabilities_keep_the_bits_that_cancel(io, D, G, top, one, other):
    """Of 300 rows three weigh: the largest score with values of 0, and two of nearly equal scores with
    values of 1 and -1, whose difference is what remains; in one tile, in tiles of several waves, before and
    after the largest.

    The scores are exact: a product of at most 1 and a code, and one of a power of two, 3 at most in
    all; the other rows' are below -300, their weights 0.  In units of 2^-24 a probability is off by 3
    (the exponent, one fused product of up to 4.4) + 2 (the exponential) + 1.5 (the scale in base 2),
    where its tile or wave had another maximum twice by 3 (the maxima's difference) + 2 + 1, by 3
    for the sums it is added to and 2 for the division: 24 of itself.  It is 1/2 at most, so the
    difference of two is off by 24.  One of 16 bits would be off by up to 60."""
    c = Cache4([300] * 20, H=1, G=G, D=D, page=16, io=io, seed=1, poison=False, bounds=False)
    far = D - 20                           # in another block than the first channels
    c.code["k"].zero_()
    c.code["v"].zero_()
    c.E["k"].fill_(127)
    c.E["v"].fill_(127)
    c.code["k"][..., 3], c.E["k"][..., 0] = 15, 133            # -6 * 2^6 in every row but these
    for r in range(c.R):
        def row(x, at, r=r):
            page = int(c.table_h[r, at // 16])
            return c.code[x][page, 0, at % 16], c.E[x][page, 0, at % 16]
        for at in (top, one, other):
            row("k", at)[0][3] = 0
        for at in (one, other):
            code, E = row("k", at)
            code[0], E[0] = 9 + r % 7, 126 - r % 3             # of -1/2 .. -6, times 1/2 to 1/8
        code, E = row("k", other)
        code[far], E[far // 32] = 2, 127 - 15
        row("v", one)[0][:], row("v", other)[0][:] = 2, 10     # 1 and -1
    c.close()
    c.upload()
    c.q_h.zero_()
    c.q_h[:, :, 0] = (torch.arange(G) % 4 + 1).to(c.q_h.dtype) / 4
    c.q_h[:, :, 3] = 1.0
    c.q_h[:, :, far] = 1.0
    out, _ = c.attend(scale=1.0)
    half = 2.0 ** -8 if io == "bf16" else 2.0 ** -24
    for r in range(c.R):
        ref = c.attend_ref(r, scale=1.0)[0]
        worst = float(((out[r].double() - ref).abs() - half * ref.abs()).max())
        assert worst <= 24 * 2.0 ** -24, (r, worst * 2.0 ** 24)
    c.close()
