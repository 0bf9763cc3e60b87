"""PagedCache's rotate and gather, and its caches of 4 bits, on the CPU: the library's calls are
recorded, not made."""

import pytest
import torch

pytest.importorskip("paper_2605_28053_amd._rwttt",
                    reason="librwttt.so not built (python -m paper_2605_28053_amd.build)")
from paper_2605_28053_amd import _rwttt as R  # noqa: E402
from paper_2605_28053_amd import _rwttt_kv as KV  # noqa: E402
from paper_2605_28053_amd import paged  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(paged.KV, "rwttt_kv_create", lambda cfg: made.append(("create", cfg)) or 1)
    monkeypatch.setattr(paged.KV, "rwttt_kv_destroy", lambda kv: 0)
    for name in ("extend", "append", "rotate", "gather"):
        monkeypatch.setattr(paged.KV, "rwttt_kv_" + name, lambda *a, n=name: made.append((n, a)) or 0)
    monkeypatch.setattr(paged, "_stream", lambda: 0)
    yield made
    while caches:                        # their handles are made up
        caches.pop().kv = None


caches = []


def cache(heads=4, kv_heads=2, owners=2, **kw):
    caches.append(paged.PagedCache(owners, 1, heads, kv_heads, 64, n_pages=8, max_pages=4, page_rows=16, device="cpu", **kw))
    return caches[-1]


def rotary(turning=64, **kw):
    return paged.Rotary(turning, device="cpu", **kw)


def rows(*shape, dtype=torch.bfloat16, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device)


I32 = torch.int32


def test_pages_of_4_bits_are_bytes(calls):
    c = cache(cache_dtype="fp4")
    assert c.k[0].dtype == torch.uint8 and tuple(c.k[0].shape) == (8, 2, 16 * 32 + 2 * 16)
    cfg = calls[0][1]
    assert cfg.cache_dtype == KV.RWTTT_FP4 and cfg.k_scale is None and cfg.v_scale is None


def test_rotate_turns_in_place_at_the_steps_positions(calls):
    c, r = cache(), rotary()
    qkv = rows(2, 8, 64)
    q, k = qkv[:, :4], qkv[:, 4:6]
    c.extend(torch.ones(2, dtype=I32))
    assert c.rotate(r, q, k) == (q, k)
    name, a = calls[-1]
    assert name == "rotate" and a[1] is r.struct and a[2:4] == (c.positions.data_ptr(), 2)
    assert a[4:12] == (q.data_ptr(), 512, q.data_ptr(), 512, k.data_ptr(), 512, k.data_ptr(), 512)
    out, at = rows(2, 4, 64), torch.zeros(2, dtype=I32)
    assert c.rotate(r, q=q, positions=at, q_out=out) == (out, None)
    assert calls[-1][1][2:12] == (at.data_ptr(), 2, q.data_ptr(), 512, out.data_ptr(), 256, 0, 0, 0, 0)


def test_rotate_refuses(calls):
    c, r = cache(), rotary()
    q, k, at = rows(2, 4, 64), rows(2, 2, 64), torch.zeros(2, dtype=I32)
    with pytest.raises(RuntimeError):
        c.rotate(r, q, k)                                    # no open step
    bad = [lambda: c.rotate(r), lambda: c.rotate(r, q, k, at[:1]), lambda: c.rotate(r, q, k[:1], at),
           lambda: c.rotate(r, q.float(), k, at), lambda: c.rotate(r, q, k, at.long()), lambda: c.rotate(r, k, q, at),
           lambda: c.rotate(r, q=q, positions=at, k_out=k), lambda: c.rotate(r, k=k, positions=at, q_out=q),
           lambda: c.rotate(r, q, k, at, q_out=rows(3, 4, 64)), lambda: c.rotate(r, q, k, at, k_out=rows(2, 2, 64).float()),
           lambda: c.rotate(r, q.transpose(0, 1), k, at), lambda: c.rotate(r, rows(2, 4, 64, device="meta"), k, at),
           lambda: c.rotate(r, q, k, torch.zeros(2, dtype=I32, device="meta"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    elsewhere = rotary()
    elsewhere.turns = torch.zeros(32, dtype=torch.uint64, device="meta")
    with pytest.raises(ValueError):
        c.rotate(elsewhere, q, k, at)
    c.extend(torch.ones(2, dtype=I32))
    with pytest.raises(ValueError):
        c.rotate(r, rows(3, 4, 64))                          # more than the step's maps hold
    assert [n for n, _ in calls] == ["create", "extend"]


def test_rotary_and_its_inverse(calls):
    r = rotary(32, base=500.0, layout="interleaved", scaling="linear", factor=2.0, gain=1.5)
    assert r.turns.tolist() == KV.rwttt_kv_turns(32, 500.0, KV.RWTTT_ROTARY_LINEAR, 2.0)
    s, i = r.struct, r.inverse()
    assert (s.turning, s.layout, s.gain, s.inverse, s.turns) == (32, KV.RWTTT_ROTARY_INTERLEAVED, 1.5, 0, r.turns.data_ptr())
    assert i.struct.inverse == 1 and i.struct.turns == s.turns and i.inverse().struct.inverse == 0
    for kw in (dict(layout="other"), dict(scaling="other"), dict(turning=-2), dict(turning=1 << 32)):
        with pytest.raises(ValueError):
            rotary(**kw)
    for kw in (dict(turning=0), dict(turning=7), dict(base=1.0), dict(scaling="linear", factor=0.0)):
        with pytest.raises(R.RwtttError):
            rotary(**kw)


def test_gather_marshals_and_refuses(calls):
    c = cache()
    owners, positions = torch.zeros(3, dtype=I32), torch.ones(3, dtype=I32)
    k, v = c.gather(0, owners, positions)
    assert tuple(k.shape) == tuple(v.shape) == (3, 2, 64) and bool((k == 0).all())
    assert calls[-1][1][1:10] == (0, owners.data_ptr(), positions.data_ptr(), c.lengths.data_ptr(), 3, k.data_ptr(), 128,
                                  v.data_ptr(), 128)
    c.extend(torch.ones(2, dtype=I32))                       # an open step's rows are held
    both = rows(3, 4, 64)
    assert c.gather(0, owners, positions, k=both[:, :2], v=both[:, 2:])[1].data_ptr() == both[:, 2:].data_ptr()
    assert calls[-1][1][4] == c.new_lengths.data_ptr() and calls[-1][1][7] == 256
    made = len(calls)
    for call in (lambda: c.gather(0, owners, positions[:2]), lambda: c.gather(0, owners.long(), positions),
                 lambda: c.gather(0, owners, positions, k=rows(2, 2, 64)), lambda: c.gather(0, owners, positions, v=k.float()),
                 lambda: c.gather(-1, owners, positions), lambda: c.gather(0, torch.zeros(3, dtype=I32, device="meta"), positions),
                 lambda: c.gather(0, owners, positions, k=rows(3, 2, 64, device="meta"))):
        with pytest.raises(ValueError):
            call()
    assert len(calls) == made
    k, v = c.gather(0, owners[:0], positions[:0])
    assert tuple(k.shape) == (0, 2, 64) and calls[-1][1][5] == 0


def test_outputs_that_require_a_gradient_are_refused(calls):
    """Autograd does not see what the calls write: its gradients would be those of the values before."""
    c, r, at = cache(), rotary(), torch.zeros(2, dtype=I32)
    q, k = rows(2, 4, 64).requires_grad_(), rows(2, 2, 64)
    bad = [lambda: c.rotate(r, q, k, at), lambda: c.rotate(r, q=rows(2, 4, 64), positions=at, q_out=q),
           lambda: c.rotate(r, q=q * 2, positions=at), lambda: c.rotate(r, k=k.clone().requires_grad_(), positions=at),
           lambda: c.gather(0, at, at, k=k.clone().requires_grad_()), lambda: c.gather(0, at, at, v=k.clone().requires_grad_())]
    made = len(calls)
    for call in bad:
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert len(calls) == made
    with torch.no_grad():
        for call in bad:
            call()
    out = rows(2, 4, 64)
    assert c.rotate(r, q=q, positions=at, q_out=out) == (out, None) and not out.requires_grad
    assert c.rotate(r, q=q.detach(), positions=at)[0] is not None
