"""A cache of 4 bits and rotary positions as they are used: the operators of a step together, rolled
back, captured, and in the decode example."""

import math

import pytest
import torch

from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd import paged_decode
from paper_2605_28053_amd.paged import PagedCache, Rotary
from paper_2605_28053_amd.paged_decode import Decoder, Model
from tests.kv4_util import stored4
from tests.test_gpu_paged_decode import Dense

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def turned(x, positions, base=10000.0):
    """Rows [n, heads, D] turned by halves, in float64 on the CPU."""
    x, d = x.double().cpu(), x.shape[-1]
    angle = positions.double().cpu()[:, None] * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


class Shadow:
    """The rows that a cache of 4 bits holds, in float64, from the keys and values it was given."""

    def __init__(self, cache):
        self.c, self.rows = cache, [[[] for _ in range(cache.n_layers)] for _ in range(cache.n_owners)]

    def append(self, layer, k, v):
        k, v = stored4(k.cpu()), stored4(v.cpu())
        for t, (r, p) in enumerate(zip(self.c.owners.tolist(), self.c.positions.tolist())):
            if r >= 0:
                del self.rows[r][layer][p:]                  # rows of a step that was rolled back
                self.rows[r][layer].append((k[t], v[t]))

    def attend(self, layer, q, r):
        K = torch.stack([a for a, _ in self.rows[r][layer]])
        V = torch.stack([b for _, b in self.rows[r][layer]])
        group, out = self.c.n_heads // self.c.n_kv_heads, []
        for i in range(self.c.n_heads):
            p = torch.softmax(K[:, i // group] @ q[i].double().cpu() * self.c.head_dim ** -0.5, dim=0)
            out.append(p @ V[:, i // group])
        return torch.stack(out)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_the_operators_of_a_step_together(io):
    """Steps that grow, roll back, end and grow again: rotate, append, attend and gather agree with
    the rows by the book.  Attention: one rounding to io and fp32 work of a few rows (1e-5)."""
    H, G, D, P = 2, 3, 64, 16
    dt = torch.float32 if io == "f32" else torch.bfloat16
    c = PagedCache(3, 1, H * G, H, D, n_pages=30, max_pages=8, page_rows=P, io_dtype=io, cache_dtype="fp4", max_new=90,
                   bound_step=0.1)
    rot, shadow, g = Rotary(D), Shadow(c), torch.Generator(device="cuda").manual_seed(1)
    lens = [0, 0, 0]
    for step, want in enumerate([[30, 1, 17], [31, 16, 18], [40, 17, 60], [41, 18, 0], [42, 40, 1]]):
        for fails in ([True, False] if step in (1, 2) else [False]):
            odd = [x + 9 for x in lens] if fails else want
            c.extend(i32(odd))
            n = sum(max(0, a - b) for a, b in zip(odd, lens))
            qkv = torch.randn((n, H * G + 2 * H, D), generator=g, device="cuda").to(dt)
            q, k, v = qkv.split([H * G, H, H], dim=1)
            before, at = k.clone(), c.positions[:n].clone()
            c.rotate(rot, q, k)
            ref = turned(before, at)
            half = 2.0 ** -24 if io == "f32" else 2.0 ** -8
            assert bool(((k.double().cpu() - ref).abs() <= 1.01 * half * ref.abs() + 1e-5).all())
            c.append(0, k, v)
            if fails:
                c.rollback()
                continue
            shadow.append(0, k, v)
            for r in range(3):
                del shadow.rows[r][0][want[r]:]
            query = torch.randn((3, H * G, D), generator=g, device="cuda").to(dt)
            out = c.attend(0, query).double().cpu()
            assert c.result.tolist()[0] == 0
            c.commit()
            lens = want
            for r in range(3):
                if want[r] == 0:
                    assert bool((out[r] == 0).all())
                    continue
                y = shadow.attend(0, query[r], r)
                assert bool(((out[r] - y).abs() <= 1.01 * half * y.abs() + 1e-5 * 6).all()), (step, r)
        # all rows read back, in reverse
        pairs = [(r, p) for r in range(3) for p in range(lens[r])][::-1] + [(1, lens[1]), (-1, 0)]
        gk, gv = c.gather(0, i32([r for r, _ in pairs]), i32([p for _, p in pairs]))
        for t, (r, p) in enumerate(pairs[:-2]):
            ek, ev = shadow.rows[r][0][p]
            assert torch.equal(gk[t].double().cpu(), ek) and torch.equal(gv[t].double().cpu(), ev)
        assert bool((gk[-2:] == 0).all()) and bool((gv[-2:] == 0).all())
    c.close()


def test_a_graph_of_two_steps():
    """Captured and replayed three times beside the same steps made eagerly: the same bits."""
    def make():
        return PagedCache(3, 1, 4, 2, 128, n_pages=30, max_pages=8, page_rows=32, cache_dtype="fp4", bound_step=0.1)

    rot, g = Rotary(128, scaling="linear", factor=2.0), torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn((3, 8, 128), generator=g, device="cuda").bfloat16()
    want = i32([0, 0, 0])

    def steps(c, out):
        for _ in range(2):
            want.copy_(c.lengths + 1)
            c.extend(want)
            q, k, v = qkv.clone().split([4, 2, 2], dim=1)
            c.rotate(rot, q, k)
            c.append(0, k, v)
            pages = c.select(0, q, 3)
            out.copy_(c.attend(0, q, pages=pages))
            c.commit()

    a, b = make(), make()
    out_a, out_b = (torch.zeros((3, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for c, out in ((a, out_a), (b, out_b)):
        steps(c, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(a, out_a)
    for i in range(3):
        qkv.neg_()
        graph.replay()
        torch.cuda.synchronize()
        steps(b, out_b)
        torch.cuda.synchronize()
        assert torch.equal(out_a, out_b) and a.lengths.tolist() == b.lengths.tolist() == [4 + 2 * i] * 3
    a.close()
    b.close()


class DenseTurned(Dense):
    """The dense model with rotary positions: a row's position is its place in the owner's list."""

    def step(self, tokens, active):
        rows, m = self.rows, self.m
        real = torch.Tensor.split

        def split(x, sizes, *a, **kw):
            got = real(x, sizes, *a, **kw)
            if isinstance(sizes, list) and sizes == [m.n_heads, m.n_kv_heads, m.n_kv_heads]:
                at = torch.tensor([len(rows[self.owner][self.layer])])
                q, k, v = got
                q, k = (turned(t[None], at)[0] for t in (q, k))
                self.layer += 1
                if self.layer == m.n_layers:
                    self.owner, self.layer = self.owner + 1, 0
                return q, k, v
            return got

        self.owner = self.layer = 0
        torch.Tensor.split = split
        try:
            return super().step(tokens, active)
        finally:
            torch.Tensor.split = real


def test_decoder_with_rotary_positions_matches_a_dense_model():
    """25 steps in fp32 against 64 bits, to the same 1e-4 as without positions."""
    m = Model(n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, vocab=50, dtype=torch.float32)
    dec, ref = Decoder(m, 3, max_rows=64, page_rows=16, rotary=Rotary(64)), DenseTurned(m, 3)
    plain = Decoder(m, 3, max_rows=64, page_rows=16)
    g = torch.Generator().manual_seed(1)
    for t in range(25):
        tokens = torch.randint(0, 50, (3,), generator=g)
        got = dec.step(tokens.cuda(), dec.cache.lengths + 1).double().cpu()
        other = plain.step(tokens.cuda(), plain.cache.lengths + 1).double().cpu()
        for r, y in enumerate(ref.step(tokens.tolist(), {0, 1, 2})):
            assert float((got[r] - y).norm() / y.norm()) < 1e-4, (t, r)
    assert float((got - other).norm() / got.norm()) > 1e-2      # positions do something
    dec.close()
    plain.close()


def test_decoder_over_4_bits_attends_to_what_it_stored(monkeypatch):
    """Every attention of 40 steps against the rows by the book, with an owner that starts over."""
    m = Model(n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, vocab=50)
    dec = Decoder(m, 3, max_rows=64, page_rows=16, cache_dtype="fp4", rotary=Rotary(64))
    shadow, append, attend, checked = Shadow(dec.cache), PagedCache.append, PagedCache.attend, []

    def append_too(self, layer, k, v):
        append(self, layer, k, v)
        shadow.append(layer, k, v)

    def attend_and_check(self, layer, q, **kw):
        out = attend(self, layer, q, **kw)
        for r in range(3):
            y = shadow.attend(layer, q[r], r)
            # one rounding to bf16, and fp32 work far below it
            assert bool(((out[r].double().cpu() - y).abs() <= 1.01 * 2.0 ** -8 * y.abs() + 1e-4).all()), (layer, r)
        checked.append(layer)
        return out

    monkeypatch.setattr(PagedCache, "append", append_too)
    monkeypatch.setattr(PagedCache, "attend", attend_and_check)
    for t in range(40):
        if t == 20:
            dec.cache.extend(i32([20, 0, 20]))
            dec.cache.commit()
        logits = dec.step(torch.tensor([t, t + 1, 7], device="cuda"), dec.cache.lengths + 1)
    assert len(checked) == 80 and bool(torch.isfinite(logits).all()) and dec.cache.lengths.tolist() == [40, 20, 40]
    assert int(dec.status) == R.RWTTT_OK
    dec.close()


@pytest.mark.parametrize("args", [["--owners", "3", "--steps", "60", "--cache", "fp4"],
                                  ["--owners", "4", "--steps", "150", "--keep", "4", "--cache", "fp4", "--rotary"]])
def test_the_example_runs(args, capsys):
    assert paged_decode.main(args) == R.RWTTT_OK
    assert "requests ended" in capsys.readouterr().out


def test_gradients_of_a_rotation():
    """Rotary.inverse is the transposed map: <R x, c> = <x, R' c>, over 384 products each off by a few 2^-24."""
    c = PagedCache(1, 1, 2, 1, 64, n_pages=2, max_pages=2, page_rows=16, io_dtype="f32", cache_dtype="fp4")
    rot, at = Rotary(48, layout="interleaved", gain=1.25), i32([0, 5, 100000])
    g = torch.Generator(device="cuda").manual_seed(3)
    x, y = (torch.randn((3, 2, 64), generator=g, device="cuda") for _ in range(2))
    rx, ry = torch.empty_like(x), torch.empty_like(y)
    c.rotate(rot, q=x, positions=at, q_out=rx)
    c.rotate(rot.inverse(), q=y, positions=at, q_out=ry)
    left, right = float((rx.double() * y.double()).sum()), float((x.double() * ry.double()).sum())
    assert math.isclose(left, right, abs_tol=16 * 2.0 ** -24 * 1.25 * 2 * float((x.abs().double() * y.abs().max().double()).sum()))
    c.close()
