"""Steps of a PagedCache as a whole: rolled back after they took effect, and captured in a graph."""

import pytest
import torch

from paper_2605_28053_amd.paged import PagedCache

pytestmark = pytest.mark.gpu

R_, H, G, D, P = 3, 2, 2, 64, 16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows(gen, n, heads):
    return torch.randn((n, heads, D), generator=gen, device="cuda").to(torch.bfloat16)


def make(cache_dtype="bf16", max_new=80):
    return PagedCache(R_, 1, H * G, H, D, n_pages=40, max_pages=12, page_rows=P, cache_dtype=cache_dtype, max_new=max_new,
                      bound_step=0.05, k_scale=0.02, v_scale=0.02)


def held(c, bits):
    """The rows and bounds that belong to the owners, by position: pages may differ."""
    out = []
    for r, n in enumerate(c.lengths.tolist()):
        for j in range(-(-n // P)):
            page = int(c.table[r, j])
            out += [x[0][page, :, :min(P, n - j * P)].contiguous().view(bits).cpu() for x in (c.k, c.v)]
    return out


@pytest.mark.parametrize("cache_dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("kind", ["grow", "shrink", "both"])
def test_a_step_that_took_effect_is_rolled_back(cache_dtype, kind):
    """Rows stored, bounds widened, pages taken and returned, then rolled back and the owners
    grown again: rows, free pages and attention are those of a cache without that step.
    The steps before and after cross pages' ends; rolled back, bounds may be wider, never
    narrower."""
    bits = torch.uint8 if cache_dtype == "fp8" else torch.int16
    caches = [make(cache_dtype), make(cache_dtype)]
    got = []
    for c, fails in zip(caches, (False, True)):
        g = torch.Generator(device="cuda").manual_seed(7)
        other = torch.Generator(device="cuda").manual_seed(8)
        lens, out = [0, 0, 0], []
        for want in ([30, 16, 5], [31, 17, 6], [33, 40, 16], [0, 41, 17], [20, 42, 60]):
            if fails:
                odd = {"grow": [x + 20 for x in lens], "shrink": [x // 3 for x in lens],
                       "both": [0, lens[1] + 25, lens[2] // 2]}[kind]
                new = sum(max(0, a - b) for a, b in zip(odd, lens))
                c.extend(i32(odd))
                result = c.result.tolist()
                assert result[:2] == [0, new] and bool((c.slots[:new] >= 0).all())
                pages = [-(-x // P) for x in lens], [-(-x // P) for x in odd]
                assert result[2:] == [sum(max(0, b - a) for a, b in zip(*pages)), sum(max(0, a - b) for a, b in zip(*pages))]
                if new:
                    c.append(0, 9 * rows(other, new, H), 9 * rows(other, new, H))
                c.attend(0, rows(other, R_, H * G))
                c.rollback()
            c.extend(i32(want))
            n = sum(max(0, a - b) for a, b in zip(want, lens))
            assert c.result.tolist()[:2] == [0, n]
            c.append(0, rows(g, n, H), rows(g, n, H))
            q = rows(g, R_, H * G)
            out.append(c.attend(0, q).clone())
            c.commit()
            lens = want
            assert c.lengths.tolist() == lens and int(c.pos[1]) == 40 - sum(-(-x // P) for x in lens)
        got.append((torch.stack(out), held(c, bits)))
    (a, rows_a), (b, rows_b) = got
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert len(rows_a) == len(rows_b) and all(torch.equal(x, y) for x, y in zip(rows_a, rows_b))
    for r, n in enumerate(caches[0].lengths.tolist()):
        for j in range(-(-n // P)):
            x, y = (c.bounds[0][int(c.table[r, j])].cpu() for c in caches)
            assert bool((y[:, 0] <= x[:, 0]).all()) and bool((y[:, 1] >= x[:, 1]).all())
    # no page belongs to two owners, or to an owner and the ring
    for c in caches:
        used = [int(c.table[r, j]) for r, n in enumerate(c.lengths.tolist()) for j in range(-(-n // P))]
        front, count = c.pos.tolist()
        free = [int(c.ring[(front + i) % 40]) for i in range(count)]
        assert sorted(used + free) == list(range(40))
        c.close()


def test_two_captured_steps_replay():
    """commit swaps two sets of buffers, so a graph holds an even number of steps: replayed,
    it goes on from where the last replay ended."""
    def two_steps(c, x):
        out = []
        for i in range(2):
            c.extend(c.lengths + 1)
            kv = x[i, :, :2 * H].view(R_, 2, H, D)
            c.append(0, kv[:, 0], kv[:, 1])
            q = x[i, :, 2 * H:]
            out.append(c.attend(0, q, pages=c.select(0, q, 4)))
            c.commit()
        return out

    x = torch.zeros((2, R_, 2 * H + H * G, D), dtype=torch.bfloat16, device="cuda")
    eager, graphed = make(max_new=R_), make(max_new=R_)
    for c in (eager, graphed):
        two_steps(c, x)                  # the first call of a kernel is not captured
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = two_steps(graphed, x)
    g = torch.Generator(device="cuda").manual_seed(3)
    for t in range(50):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        want = two_steps(eager, x)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), t
        assert graphed.lengths.tolist() == eager.lengths.tolist() == [2 * t + 4] * R_
        assert torch.equal(graphed.table, eager.table) and torch.equal(graphed.pos, eager.pos)
    assert graphed.result.tolist()[0] == 0
    eager.close()
    graphed.close()
