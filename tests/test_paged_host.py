"""PagedCache's checks and argument marshalling, on the CPU: the library's calls are recorded,
not made."""

import pytest
import torch

pytest.importorskip("paper_2605_28053_amd._rwttt",
                    reason="librwttt.so not built (python -m paper_2605_28053_amd.build)")
from paper_2605_28053_amd import paged  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(paged.KV, "rwttt_kv_create", lambda cfg: 1)
    monkeypatch.setattr(paged.KV, "rwttt_kv_destroy", lambda kv: 0)
    for name in ("extend", "append", "select", "attend"):
        monkeypatch.setattr(paged.KV, "rwttt_kv_" + name, lambda *a, n=name: made.append((n, a)) or 0)
    monkeypatch.setattr(paged, "_stream", lambda: 0)
    yield made
    while caches:                        # their handles are made up
        caches.pop().kv = None


caches = []


def cache(heads=4, kv_heads=2, owners=2, **kw):
    caches.append(paged.PagedCache(owners, 1, heads, kv_heads, 64, n_pages=8, max_pages=4, page_rows=16,
                                   bound_step=0.05, device="cpu", **kw))
    return caches[-1]


def elsewhere(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_tensors_of_another_device_are_refused(calls):
    """Their addresses would go to the kernels."""
    c = cache()
    i32, q, kv = torch.int32, torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    rows = torch.zeros(1, dtype=i32)
    refused = [lambda: c.extend(elsewhere(2, dtype=i32)),
               lambda: c.attend(0, elsewhere(2, 4, 64)),
               lambda: c.attend(0, q, out=elsewhere(2, 4, 64)),
               lambda: c.attend(0, q, lse=elsewhere(2, 4, dtype=torch.float32)),
               lambda: c.attend(0, q, rows=elsewhere(1, dtype=i32)),
               lambda: c.attend(0, q, pages=elsewhere(2, 2, 3, dtype=i32)),
               lambda: c.select(0, elsewhere(2, 4, 64), 3),
               lambda: c.select(0, q, 3, rows=elsewhere(1, dtype=i32)),
               lambda: c.select(0, q, 3, out=elsewhere(2, 2, 3, dtype=i32))]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    c.extend(torch.ones(2, dtype=i32))
    for k, v in ((elsewhere(2, 2, 64), kv), (kv, elsewhere(2, 2, 64))):
        with pytest.raises(ValueError):
            c.append(0, k, v)
    assert [name for name, _ in calls] == ["extend"]
    c.append(0, kv, kv)
    pages = c.select(0, q, 3, rows=rows)
    c.attend(0, q, pages=pages, rows=rows, lse=torch.zeros((2, 4)))
    assert [name for name, _ in calls] == ["extend", "append", "select", "attend"]


def test_an_empty_list_of_owners_computes_none(calls):
    c = cache()
    q, none = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros(0, dtype=torch.int32)
    out, pages = torch.full_like(q, 7.0), torch.full((2, 2, 3), 7, dtype=torch.int32)
    assert c.attend(0, q, rows=none, out=out) is out and c.select(0, q, 3, rows=none, out=pages) is pages
    for name, args in calls:             # a list of no owners, and not a missing one, which means all of them
        assert args[5] != 0 and args[6] == 0, name


def test_strides_of_dimensions_of_one_do_not_matter(calls):
    """torch gives a dimension of one any stride: one owner, one new row, one head."""
    q = torch.zeros((4, 1, 64), dtype=torch.bfloat16).transpose(0, 1)                # [1, 4, 64], stride 64 between rows
    c = cache(owners=1)
    c.extend(torch.ones(1, dtype=torch.int32))
    kv = torch.zeros((2, 1, 64), dtype=torch.bfloat16).transpose(0, 1)
    c.append(0, kv, kv)
    c.attend(0, q, out=torch.zeros((4, 1, 64), dtype=torch.bfloat16).transpose(0, 1))
    c.select(0, q, 3)
    (_, append), (_, attend), (_, select) = calls[1:]
    assert append[3] == append[5] == 2 * 64 and attend[3] == attend[12] == select[3] == 4 * 64
    one = cache(heads=1, kv_heads=1)
    one.attend(0, torch.zeros(400, dtype=torch.bfloat16).as_strided((2, 1, 64), (192, 7, 1)))
    assert calls[-1][1][3] == 192


def test_negative_numbers_are_refused(calls):
    """ctypes would wrap them: a window of -1 meant all rows."""
    c, q = cache(), torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: c.attend(0, q, window=-1), lambda: c.attend(-1, q), lambda: c.select(0, q, 3, first=-1),
                 lambda: c.select(0, q, 3, last=-1), lambda: c.select(-1, q, 3), lambda: c.select(0, q, -1)):
        with pytest.raises((ValueError, RuntimeError)):
            call()
    assert calls == []


def test_outputs_are_filled_only_where_owners_are_left_out(calls, monkeypatch):
    """With all owners the kernels write every row: a fill is a launch too many."""
    c, q, one = cache(), torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.ones(1, dtype=torch.int32)
    out, pages = c.attend(0, q, rows=one), c.select(0, q, 3, rows=one)
    assert bool((out == 0).all()) and bool((pages == -1).all())
    for name in ("zeros", "full"):
        monkeypatch.setattr(paged.torch, name, lambda *a, **kw: pytest.fail("filled"))
    assert c.attend(0, q).shape == q.shape and c.select(0, q, 3).shape == (2, 2, 3)
