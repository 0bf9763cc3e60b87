"""Host-side checks of the paged cache's C ABI that need no GPU: exports and refusals.

Every refusal happens before a launch; the fake device addresses below are
never dereferenced.
"""

import os
import re
import subprocess

import pytest

R = pytest.importorskip("paper_2605_28053_amd._rwttt",
                        reason="librwttt.so not built (python -m paper_2605_28053_amd.build)")
from paper_2605_28053_amd import _rwttt_kv as KV  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x10000 * (i + 1) for i in range(40)]       # distinct 16- and 256-byte aligned addresses
GOOD = dict(n_owners=4, n_layers=2, n_pages=100, page_rows=64, max_pages=16, n_heads=8, n_kv_heads=2, head_dim=128,
            io_dtype=R.RWTTT_BF16, cache_dtype=R.RWTTT_BF16)
BUFFERS = dict(table=A[0], ring=A[1], k=A[2:4], v=A[4:6], bounds=A[6:8], bound_step=A[8], workspace=A[9],
               workspace_bytes=1 << 30)


def config(**kw):
    return KV.make_kv_config(**{**GOOD, **BUFFERS, **kw})


def create(**kw):
    return KV.rwttt_kv_create(config(**kw))


def refuses(status, **kw):
    with pytest.raises(R.RwtttError) as e:
        create(**kw)
    assert e.value.status == status


def test_library_exports_every_declared_symbol_and_binds_it():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rwttt_kv.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rwttt_kv_[a-z_]+)\s*\(", text)))
    assert len(names) == 8
    out = subprocess.run(["nm", "-D", "--defined-only", R.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT (rwttt_\w+)", out))
    for n in names:
        assert n in exported and hasattr(R.lib(), n) and callable(getattr(KV, n)), n


def test_header_is_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "rwttt_kv.h"\nint main(void) { rwttt_kv_config c; c.reserved = 0; return (int)c.reserved; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(tmp_path / "h")], check=True)


def test_create_accepts_partial_buffers():
    for kw in ({}, dict(k=None, v=None), dict(bounds=None, bound_step=0), dict(table=0, ring=0),
               dict(workspace=0, workspace_bytes=0), dict(cache_dtype=KV.RWTTT_FP8, k_scale=A[20], v_scale=A[21])):
        assert KV.rwttt_kv_destroy(create(**kw)) == R.RWTTT_OK


@pytest.mark.parametrize("kw", [
    dict(n_owners=0), dict(n_owners=4097), dict(n_layers=0, k=[], v=[], bounds=[]), dict(page_rows=8), dict(page_rows=48),
    dict(page_rows=512), dict(n_pages=0), dict(n_pages=1 << 26), dict(max_pages=0), dict(max_pages=(1 << 17) + 1),
    dict(n_heads=0), dict(n_heads=9), dict(n_kv_heads=0), dict(n_heads=258, n_kv_heads=2), dict(head_dim=96),
    dict(head_dim=0), dict(io_dtype=2), dict(io_dtype=-1), dict(cache_dtype=3), dict(cache_dtype=R.RWTTT_F32),
    dict(table=A[0] + 4), dict(ring=A[1] + 8), dict(k=None), dict(v=None), dict(k=[A[2], 0]), dict(k=[A[2], A[3] + 2]),
    dict(bounds=[0, A[7]]), dict(bound_step=0), dict(bound_step=A[8] + 4), dict(k_scale=A[20]), dict(v_scale=A[20]),
    dict(workspace=A[9] + 16)])
def test_create_refuses(kw):
    refuses(R.RWTTT_E_INVALID, **kw)


def test_create_refuses_reserved_and_small_workspace():
    cfg = config()
    cfg.reserved = 1
    with pytest.raises(R.RwtttError):
        KV.rwttt_kv_create(cfg)
    need = KV.rwttt_kv_workspace_bytes(config())
    refuses(R.RWTTT_E_CAPACITY, workspace_bytes=need - 1)
    assert KV.rwttt_kv_destroy(create(workspace_bytes=need)) == R.RWTTT_OK
    assert KV.rwttt_kv_destroy(None) == R.RWTTT_E_INVALID
    with pytest.raises(ValueError):
        config(k=A[2:3])


def test_workspace_follows_the_head_layout_and_the_table():
    a = KV.rwttt_kv_workspace_bytes(config())
    assert a == KV.rwttt_kv_workspace_bytes(config(n_pages=10 ** 6))
    assert a < KV.rwttt_kv_workspace_bytes(config(head_dim=256))
    # at most 256 rows of scores, whatever the number of owners
    b = KV.rwttt_kv_workspace_bytes(config(n_owners=4096, max_pages=4000))
    assert b == KV.rwttt_kv_workspace_bytes(config(n_owners=128, max_pages=4000)) <= a + 256 * 4000 * 4 + 256


EXTEND = dict(have=A[10], want=A[11], pos=A[12], new_pos=A[13], lengths=A[14], start=A[15], slots=A[16], owners=A[17],
              positions=A[18], cap=5, result=A[19])


@pytest.mark.parametrize("kw", [
    *({n: 0} for n in EXTEND if n != "cap"), *({n: EXTEND[n] + 4} for n in EXTEND if n != "cap"),
    dict(lengths=A[10]), dict(lengths=A[11]), dict(new_pos=A[12]), dict(start=A[14]), dict(slots=A[17]),
    dict(result=A[13]), dict(cap=1 << 31)])
def test_extend_refuses(kw):
    kv = create()
    assert KV.rwttt_kv_extend(kv, **{**EXTEND, **kw}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


@pytest.mark.parametrize("missing", ["table", "ring"])
def test_extend_needs_table_and_ring(missing):
    kv = create(**{missing: 0})
    assert KV.rwttt_kv_extend(kv, **EXTEND) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_extend(None, **EXTEND) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


APPEND = dict(layer=1, k=A[10], k_stride=256, v=A[11], v_stride=256, slots=A[12], n=3)


@pytest.mark.parametrize("kw", [
    dict(layer=2), dict(k=0), dict(k=A[10] + 2), dict(v=0), dict(v=A[11] + 8), dict(slots=0), dict(slots=A[12] + 4),
    dict(k_stride=255), dict(v_stride=260), dict(v_stride=128), dict(k_stride=0), dict(n=(1 << 24) + 1)])
def test_append_refuses(kw):
    kv = create()
    assert KV.rwttt_kv_append(kv, **{**APPEND, **kw}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_append(kv, **{**APPEND, "n": 0, "k": 0}) == R.RWTTT_OK
    KV.rwttt_kv_destroy(kv)


SELECT = dict(layer=0, q=A[10], q_stride=1024, lengths=A[11], rows=0, n=4, first=1, last=2, keep=8, pages=A[12])


@pytest.mark.parametrize("kw", [
    dict(layer=2), dict(q=0), dict(q=A[10] + 4), dict(q_stride=1020), dict(q_stride=1025), dict(lengths=0),
    dict(lengths=A[11] + 4), dict(rows=A[13] + 4), dict(n=3), dict(n=5), dict(rows=A[13], n=4097), dict(keep=0),
    dict(first=7), dict(last=8), dict(first=(1 << 32) - 1, last=2), dict(pages=0), dict(pages=A[12] + 4),
    dict(keep=1 << 20)])
def test_select_refuses(kw):
    kv = create()
    assert KV.rwttt_kv_select(kv, **{**SELECT, **kw}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_select(kv, **{**SELECT, "rows": A[13], "n": 0}) == R.RWTTT_OK
    KV.rwttt_kv_destroy(kv)


def test_select_needs_bounds_and_a_table_it_can_hold():
    kv = create(bounds=None, bound_step=0)
    assert KV.rwttt_kv_select(kv, **SELECT) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)
    kv = create(page_rows=16, max_pages=KV.RWTTT_KV_MAX_SELECT + 1)
    assert KV.rwttt_kv_select(kv, **SELECT) == R.RWTTT_E_CAPACITY
    KV.rwttt_kv_destroy(kv)


ATTEND = dict(layer=0, q=A[10], q_stride=1024, lengths=A[11], rows=0, n=4, scale=0.1, window=0, pages=0, keep=0,
              out=A[12], out_stride=1024, lse=A[14])


@pytest.mark.parametrize("kw", [
    dict(layer=2), dict(q=0), dict(q=A[10] + 4), dict(q_stride=1020), dict(lengths=0), dict(rows=A[13] + 4), dict(n=3),
    dict(rows=A[13], n=4097), dict(out=0), dict(out=A[12] + 2), dict(out_stride=1023), dict(out_stride=512),
    dict(lse=A[14] + 4), dict(pages=A[15]), dict(keep=4), dict(pages=A[15] + 4, keep=4),
    dict(pages=A[15], keep=4, window=3), dict(pages=A[15], keep=4, window=1 << 31), dict(pages=A[15], keep=1 << 20)])
def test_attend_refuses(kw):
    kv = create()
    assert KV.rwttt_kv_attend(kv, **{**ATTEND, **kw}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_attend(kv, **{**ATTEND, "rows": A[13], "n": 0}) == R.RWTTT_OK
    KV.rwttt_kv_destroy(kv)


def test_attend_needs_cache_table_and_workspace():
    for kw in (dict(k=None, v=None), dict(table=0), dict(workspace=0)):
        kv = create(**kw)
        assert KV.rwttt_kv_attend(kv, **ATTEND) == R.RWTTT_E_INVALID
        KV.rwttt_kv_destroy(kv)
    assert KV.rwttt_kv_attend(None, **ATTEND) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_last_hip_error(None) == 0
