"""Rotary positions on the GPU against the definition in 64 bits."""

import math

import pytest
import torch

from paper_2605_28053_amd import _rwttt_kv as KV
from tests.kv_util import DT, dev, i32, ok, stream

pytestmark = pytest.mark.gpu


class Rotor:
    """A handle of a head layout and a rotary's table on the GPU."""

    def __init__(self, H, K, D, turning, layout="half", io="bf16", base=1e4, gain=1.0, inverse=False, scaling=0, factor=1.0):
        self.H, self.K, self.D, self.turning, self.layout, self.io = H, K, D, turning, layout, io
        self.gain, self.inverse = gain, inverse
        self.kv = KV.rwttt_kv_create(KV.make_kv_config(1, 1, 1, 16, 1, H, K, D, 0 if io == "f32" else 1, 1))
        self.units = KV.rwttt_kv_turns(turning, base, scaling, factor)
        self.table = torch.tensor(self.units, dtype=torch.uint64).cuda()
        self.rot = KV.make_rotary(turning, KV.RWTTT_ROTARY_HALF if layout == "half" else KV.RWTTT_ROTARY_INTERLEAVED,
                                  self.table.data_ptr(), gain, inverse)

    def close(self):
        KV.rwttt_kv_destroy(self.kv)

    def __call__(self, positions, q=None, q_out=None, k=None, k_out=None):
        def at(t):
            return (0, 0) if t is None else (t.data_ptr(), t.stride(0))

        ok(KV.rwttt_kv_rotate(self.kv, self.rot, positions.data_ptr(), positions.numel(), *at(q), *at(q_out), *at(k), *at(k_out),
                              stream()))

    def ref(self, x, positions):
        """(values in float64, bound of the fp32 work) of the rows x [n, heads, D] (CPU).

        The angle is exact to 2^-40 turns and is rounded to 24 bits (below a half turn: off
        by pi 2^-24); sine and cosine, each off by 2 ulp at most, and gain, products and
        sum each round once: 8 * 2^-24 of |a| + |b| in all."""
        frac = torch.tensor([[(int(p) * u % 2 ** 64) / 2.0 ** 64 for u in self.units] for p in positions], dtype=torch.float64)
        angle = 2 * math.pi * frac * (-1 if self.inverse else 1)
        cos, sin = (self.gain * f(angle)[:, None] for f in (torch.cos, torch.sin))
        d, out = self.turning, x.double().clone()
        tol = torch.zeros_like(out)
        one, two = (slice(0, d // 2), slice(d // 2, d)) if self.layout == "half" else (slice(0, d, 2), slice(1, d, 2))
        a, b = x.double()[..., one], x.double()[..., two]
        out[..., one], out[..., two] = a * cos - b * sin, b * cos + a * sin
        tol[..., one] = tol[..., two] = 8 * 2.0 ** -24 * abs(self.gain) * (a.abs() + b.abs())
        return out, tol

    def check(self, got, x, positions):
        out, tol = self.ref(x, positions)
        half = 2.0 ** -8 if self.io == "bf16" else 2.0 ** -24
        err = (got.double() - out).abs()
        assert bool((err <= half * 1.01 * out.abs() + tol).all()), float((err - tol).max())
        assert torch.equal(got[..., self.turning:], x[..., self.turning:])       # the other channels bit for bit


POSITIONS = [0, 1, 2, 63, 1000, 4223, 131071, 8388607, 2 ** 31 - 1, 77]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,turning", [(64, 64), (128, 128), (256, 256), (128, 64), (64, 16), (256, 8), (64, 2), (128, 50),
                                       (64, 34), (256, 250), (128, 20), (64, 62), (128, 126), (256, 14)])
def test_rotation_matches_the_definition(io, layout, D, turning):
    """Whole heads, parts of them, halves that are no whole pieces; near and the farthest positions;
    queries and keys as strided parts of one projection, into outputs with strides of their own."""
    g = torch.Generator().manual_seed(D + turning)
    f = Rotor(6, 3, D, turning, layout, io, base=5e5, gain=1.25)
    x = torch.randn((len(POSITIONS), 12, D), generator=g).to(DT[io])
    xd = dev(x)
    q, k = xd[:, :6], xd[:, 6:9]
    qo = torch.full((len(POSITIONS), 7, D), 7.0, dtype=DT[io], device="cuda")
    ko = torch.full((len(POSITIONS), 3, D), 7.0, dtype=DT[io], device="cuda")
    f(i32(POSITIONS), q, qo, k, ko)
    torch.cuda.synchronize()
    f.check(qo[:, :6].cpu(), x[:, :6], POSITIONS)
    f.check(ko.cpu(), x[:, 6:9], POSITIONS)
    assert bool((qo[:, 6] == 7.0).all()) and torch.equal(xd.cpu(), x)
    # in place, the same bits; the values beside them stay
    f(i32(POSITIONS), q, q, k, k)
    torch.cuda.synchronize()
    assert torch.equal(q, qo[:, :6]) and torch.equal(k, ko) and torch.equal(xd[:, 9:].cpu(), x[:, 9:])
    f.close()


@pytest.mark.parametrize("H,K,n", [(1, 1, 1), (40, 8, 3), (8, 8, 700), (64, 1, 5), (128, 1, 2), (3, 3, 5000)])
def test_head_layouts_and_lengths(H, K, n):
    g = torch.Generator().manual_seed(n)
    f = Rotor(H, K, 64, 64, "half", "bf16")
    pos = torch.randint(0, 1 << 20, (n,), generator=g)
    q, k = torch.randn((n, H, 64), generator=g).bfloat16(), torch.randn((n, K, 64), generator=g).bfloat16()
    qd, kd = dev(q), dev(k)
    f(i32(pos.tolist()), qd, qd, kd, kd)
    torch.cuda.synchronize()
    f.check(qd.cpu(), q, pos)
    f.check(kd.cpu(), k, pos)
    # one side alone gives the same bits
    q2, k2 = dev(q), dev(k)
    f(i32(pos.tolist()), q=q2, q_out=q2)
    f(i32(pos.tolist()), k=k2, k_out=k2)
    torch.cuda.synchronize()
    assert torch.equal(q2, qd) and torch.equal(k2, kd)
    f.close()


@pytest.mark.parametrize("layout,turning", [("half", 64), ("interleaved", 64), ("half", 50)])
def test_padded_tokens_are_left_as_they_were(layout, turning):
    f = Rotor(2, 1, 64, turning, layout, "f32")
    pos = [5, -1, 9, -2 ** 31, -7]
    q = torch.randn((5, 2, 64))
    qd, qo = dev(q), torch.full((5, 2, 64), 7.0, device="cuda")
    f(i32(pos), q=qd, q_out=qo)
    f(i32(pos), q=qd, q_out=qd)
    torch.cuda.synchronize()
    live = torch.tensor([p >= 0 for p in pos])
    f.check(qo.cpu()[live], q[live], [5, 9])
    assert bool((qo.cpu()[~live] == 7.0).all()) and torch.equal(qd.cpu()[~live], q[~live])
    assert torch.equal(qd.cpu()[live], qo.cpu()[live])
    f.close()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_inverse_is_the_gradient(layout):
    """Of sum(c * rotate(x)): against the formula, and against differences, which are exact but for
    rounding since the map is linear."""
    D, turning, gain = 64, 48, 1.25
    f, b = (Rotor(2, 1, D, turning, layout, "f32", gain=gain, inverse=inv) for inv in (False, True))
    g = torch.Generator().manual_seed(3)
    pos = [0, 3, 70000, 8000000]
    x, c = torch.randn((4, 2, D), generator=g), torch.randn((4, 2, D), generator=g)
    grad = dev(c)
    b(i32(pos), q=grad, q_out=grad)
    torch.cuda.synchronize()
    grad = grad.cpu()
    b.check(grad, c, pos)

    def loss(y):
        yd = dev(y)
        f(i32(pos), q=yd, q_out=yd)
        torch.cuda.synchronize()
        return (c.double() * yd.double().cpu()).sum(dim=(1, 2))

    for i in (0, 1, 24, 25, 47, 48, 63):
        e = torch.zeros_like(x)
        e[:, 1, i] = 4.0
        diff = (loss(x + e) - loss(x - e)) / 8.0
        # 128 outputs of up to |x| + 4 < 10, each off by 2^-24 of itself and 8 2^-24 (|a| + |b|) gain, twice, over 8
        bound = 2 * 128 * 3 * (2.0 ** -24 + 16 * 2.0 ** -24) * 10 * gain / 8
        assert bool(((diff - grad[:, 1, i].double()).abs() <= bound).all())
    # there and back is gain^2 times the turned channels
    y = dev(x)
    f(i32(pos), q=y, q_out=y)
    b(i32(pos), q=y, q_out=y)
    torch.cuda.synchronize()
    want = x.clone().double()
    want[..., :turning] *= gain * gain
    assert float((y.cpu().double() - want).abs().max()) <= 2 * 9 * 2.0 ** -24 * gain * gain * 2 * float(x.abs().max())
    f.close()
    b.close()


def test_rotation_depends_on_the_distance_alone():
    """What positions are for: q . k of turned heads, at 8000000 as at 0."""
    f = Rotor(1, 1, 128, 128, "half", "f32", base=1e6)
    g = torch.Generator().manual_seed(4)
    x, y = torch.randn(128, generator=g), torch.randn(128, generator=g)
    first = torch.tensor([0, 100, 131072, 8000000])
    q, k = dev(x.expand(4, 1, 128)), dev(y.expand(4, 1, 128))
    f(i32((first + 17).tolist()), q=q, q_out=q)
    f(i32(first.tolist()), k=k, k_out=k)
    torch.cuda.synchronize()
    dot = (q.double() * k.double()).sum(dim=(1, 2)).cpu()
    size = float((x.abs().view(2, 64).sum(0) * y.abs().view(2, 64).sum(0)).sum())
    assert float((dot - dot[0]).abs().max()) <= 4 * 9 * 2.0 ** -24 * size
    f.close()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_infinities_and_nan_stay_in_their_pairs(io):
    """A pair with an infinite channel becomes what the two products and their sum are; its
    neighbours do not change."""
    f = Rotor(2, 1, 64, 64, "half", io)
    g = torch.Generator().manual_seed(6)
    x = torch.randn((3, 2, 64), generator=g).to(DT[io])
    clean = dev(x)
    x[0, 0, 3], x[0, 1, 40], x[1, 0, 7], x[2, 1, 1], x[2, 1, 33] = math.inf, -math.inf, math.nan, math.inf, -math.inf
    pos = [3, 100, 4321]
    xd = dev(x)
    for t in (clean, xd):
        f(i32(pos), q=t, q_out=t)
    torch.cuda.synchronize()
    want, _ = f.ref(x, pos)
    bad = ~torch.isfinite(want)
    assert int(bad.sum()) == 8
    assert torch.equal(xd.cpu().double()[bad].nan_to_num(0.5), want[bad].nan_to_num(0.5))
    assert torch.equal(xd.cpu()[~bad], clean.cpu()[~bad])
    f.close()


def test_another_stream_and_a_graph():
    f = Rotor(8, 2, 128, 128)
    pos = i32([5, 9, -1])
    q, out = torch.randn((3, 8, 128), device="cuda").bfloat16(), torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    f(pos, q=q, q_out=out)
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f(pos, q=q, q_out=out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(pos, q=q, q_out=out)
    for i in range(3):
        out.zero_()
        pos.add_(i)                      # replays read the positions anew
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        f(pos, q=q, q_out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    f.close()
