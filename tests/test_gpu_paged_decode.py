"""PagedCache and the decode example: the operators together, against a dense computation in 64 bits."""

import math

import pytest
import torch

from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd.paged import PagedCache
from paper_2605_28053_amd.paged_decode import Decoder, Model, main
from tests.kv_util import select_ref

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def norm64(x):
    return x * torch.rsqrt(x.pow(2).mean(dim=-1, keepdim=True) + 1e-6)


class Dense:
    """The same model in float64 on the CPU, every owner's rows in a list."""

    def __init__(self, model, n_owners, window=0):
        self.m, self.window = model, window
        self.rows = [[[] for _ in range(model.n_layers)] for _ in range(n_owners)]
        self.w = [{k: v.double().cpu() for k, v in w.items()} for w in model.layers]
        self.embed, self.head = model.embed.double().cpu(), model.head.double().cpu()

    def forget(self, r):
        self.rows[r] = [[] for _ in range(self.m.n_layers)]

    def step(self, tokens, active):
        m, out = self.m, []
        for r, tok in enumerate(tokens):
            if r not in active:
                out.append(None)
                continue
            x = self.embed[tok]
            for l, w in enumerate(self.w):
                qkv = (norm64(x) @ w["qkv"]).view(-1, m.head_dim)
                q, k, v = qkv.split([m.n_heads, m.n_kv_heads, m.n_kv_heads])
                self.rows[r][l].append((k, v))
                rows = self.rows[r][l][-self.window:] if self.window else self.rows[r][l]
                K, V = torch.stack([a for a, _ in rows]), torch.stack([b for _, b in rows])   # [t, H, D]
                group = m.n_heads // m.n_kv_heads
                a = []
                for i in range(m.n_heads):
                    p = torch.softmax(K[:, i // group] @ q[i] * m.head_dim ** -0.5, dim=0)
                    a.append(p @ V[:, i // group])
                x = x + torch.cat(a) @ w["out"]
                gate, up = (norm64(x) @ w["up"]).split(m.d_ff)
                x = x + (gate * torch.sigmoid(gate) * up) @ w["w0"]
            out.append(norm64(x) @ self.head)
        return out


@pytest.mark.parametrize("window", [0, 9])
def test_decoder_matches_a_dense_model(window):
    """40 steps in fp32; an owner ends in between, returns its pages and starts over.
    Every product is fp32 with sums of at most 512 terms and the residual stream
    passes through 2 layers: errors of a few 1e-6 of the logits' size, held to 1e-4."""
    m = Model(n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, vocab=50, dtype=torch.float32)
    dec, ref = Decoder(m, 3, max_rows=64, page_rows=16, window=window), Dense(m, 3, window)
    g = torch.Generator().manual_seed(1)
    for t in range(40):
        tokens = torch.randint(0, 50, (3,), generator=g)
        if t == 20:
            dec.cache.extend(i32([20, 0, 20]))
            dec.cache.commit()
            ref.forget(1)
        got = dec.step(tokens.cuda(), dec.cache.lengths + 1).double().cpu()
        for r, y in enumerate(ref.step(tokens.tolist(), {0, 1, 2})):
            assert float((got[r] - y).norm() / y.norm()) < 1e-4, (t, r)
    assert dec.cache.lengths.tolist() == [40, 20, 40] and int(dec.cache.pos[1]) == 3 * 4 - 3 - 2 - 3
    dec.close()


def test_a_rolled_back_step_leaves_no_trace():
    """A step with other tokens, rolled back, then the same steps as a run without it."""
    m = Model(n_layers=1, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, vocab=50)
    runs = []
    for fail in (False, True):
        dec, out = Decoder(m, 2, max_rows=64, page_rows=16), []
        for t in range(35):
            if fail and t in (0, 15, 16, 33):
                dec.cache.extend(dec.cache.lengths + i32([5, 20]))
                k = torch.full((dec.cache.max_new, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
                dec.cache.append(0, k, k)
                dec.cache.rollback()
            out.append(dec.step(torch.tensor([t, t + 1], device="cuda"), dec.cache.lengths + 1).clone())
        runs.append((torch.stack(out), dec.cache.lengths.tolist(), dec.cache.pos.tolist()))
        dec.close()
    assert torch.equal(runs[0][0].view(torch.int16), runs[1][0].view(torch.int16))
    assert runs[0][1:] == runs[1][1:]


def test_selected_pages_of_a_filled_cache():
    """Prefill through the slot map, then select and attend: the pages are those of the
    bounds of what was stored, and attention is over them alone."""
    R_, H, G, D, P, keep = 3, 2, 4, 64, 16, 5
    c = PagedCache(R_, 1, H * G, H, D, n_pages=80, max_pages=30, page_rows=P, max_new=700, bound_step=0.03)
    g = torch.Generator().manual_seed(3)
    lens = [300, 17, 150]
    c.extend(i32(lens))
    n = sum(lens)
    k, v = (torch.randn((n, H, D), generator=g).to(torch.bfloat16) for _ in range(2))
    c.append(0, k.cuda(), v.cuda())
    c.commit()
    q = torch.randn((R_, H * G, D), generator=g).to(torch.bfloat16)
    pages = c.select(0, q.cuda(), keep)
    lse = torch.zeros((R_, H * G), device="cuda")
    out = c.attend(0, q.cuda(), pages=pages, lse=lse).double().cpu()
    assert c.result.tolist() == [0, n, 19 + 2 + 10, 0]
    at = 0
    for r, rows in enumerate(lens):
        K, V = k[at:at + rows].double(), v[at:at + rows].double()
        at += rows
        table = c.table[r, :-(-rows // P)].long().cpu().numpy()
        for h in range(H):
            ref = select_ref(q[r, h * G:(h + 1) * G].float().numpy(), c.bounds[0][:, h].cpu().numpy(), table, 1, 2, keep)
            assert pages[r, h].tolist() == ref
            seen = [i for p in ref if p >= 0 for i in range(p * P, min(rows, (p + 1) * P))]
            for i in range(h * G, (h + 1) * G):
                s = K[seen, h] @ q[r, i].double() * D ** -0.5
                y = torch.softmax(s, dim=0) @ V[seen, h]
                # one rounding to bf16, and fp32 arithmetic far below it
                assert bool(((out[r, i] - y).abs() <= 2.0 ** -8 * y.abs() + 1e-4).all())
                assert math.isclose(float(lse[r, i]), float(torch.logsumexp(s, dim=0)), rel_tol=1e-5, abs_tol=1e-5)
    c.close()


@pytest.mark.parametrize("args", [["--owners", "3", "--steps", "60"],
                                  ["--owners", "4", "--steps", "150", "--keep", "4", "--cache", "fp8"]])
def test_the_example_runs(args, capsys):
    assert main(args) == R.RWTTT_OK
    assert "requests ended" in capsys.readouterr().out


def test_refusals():
    c = PagedCache(2, 1, 4, 2, 64, n_pages=8, max_pages=4, page_rows=16)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: c.attend(0, q.float()), lambda: c.attend(0, q[:1]), lambda: c.attend(0, q.transpose(0, 1)),
                 lambda: c.extend(torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: c.extend(i32([1, 2, 3])),
                 lambda: c.attend(0, q, lse=torch.zeros((2, 4), dtype=torch.float64, device="cuda")),
                 lambda: c.attend(0, q, pages=i32([[[0]]]))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: c.select(0, q, 2), lambda: c.attend(1, q), lambda: c.attend(0, q, window=3, pages=i32([[[0]] * 2] * 2))):
        with pytest.raises(R.RwtttError):
            call()
    for call in (c.commit, c.rollback, lambda: c.append(0, q[:, :2], q[:, :2])):
        with pytest.raises(RuntimeError):
            call()
    c.close()
