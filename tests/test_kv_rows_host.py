"""Host-side checks of the cache's operators on rows that need no GPU: exports, refusals, the
frequencies' table.  The fake device addresses are never dereferenced."""

import ctypes
import math
import os
import re
import subprocess
from fractions import Fraction

import pytest

R = pytest.importorskip("paper_2605_28053_amd._rwttt",
                        reason="librwttt.so not built (python -m paper_2605_28053_amd.build)")
from paper_2605_28053_amd import _rwttt_kv as KV  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x1000000 * (i + 1) for i in range(20)]
GOOD = dict(n_owners=4, n_layers=2, n_pages=100, page_rows=64, max_pages=16, n_heads=8, n_kv_heads=2, head_dim=128,
            io_dtype=R.RWTTT_BF16, cache_dtype=KV.RWTTT_FP4)
BUFFERS = dict(table=A[0], k=A[2:4], v=A[4:6])


def create(**kw):
    return KV.rwttt_kv_create(KV.make_kv_config(**{**GOOD, **BUFFERS, **kw}))


def test_library_exports_every_declared_symbol_and_binds_it():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rwttt_kv_rows.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rwttt_kv_[a-z_]+)\s*\(", text)))
    assert names == ["rwttt_kv_gather", "rwttt_kv_rotate", "rwttt_kv_turns"]
    out = subprocess.run(["nm", "-D", "--defined-only", R.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT (rwttt_\w+)", out))
    for n in names:
        assert n in exported and hasattr(R.lib(), n) and callable(getattr(KV, n)), n


def test_header_is_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "rwttt_kv_rows.h"\nint main(void) { rwttt_kv_rotary r; r.inverse = 0; return (int)r.inverse; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(tmp_path / "h")], check=True)


def test_a_cache_of_4_bits_takes_either_io_type_and_no_scales():
    for kw in (dict(), dict(io_dtype=R.RWTTT_F32), dict(head_dim=64), dict(bounds=A[6:8], bound_step=A[8])):
        assert KV.rwttt_kv_destroy(create(**kw)) == R.RWTTT_OK
    for kw in (dict(k_scale=A[9]), dict(v_scale=A[9]), dict(cache_dtype=3), dict(cache_dtype=5)):
        with pytest.raises(R.RwtttError) as e:
            create(**kw)
        assert e.value.status == R.RWTTT_E_INVALID


GATHER = dict(layer=1, owners=A[10], positions=A[11], lengths=A[12], n=3, k=A[13], k_stride=256, v=A[14], v_stride=256)


@pytest.mark.parametrize("kw", [
    dict(layer=2), dict(owners=0), dict(owners=A[10] + 4), dict(positions=0), dict(positions=A[11] + 8), dict(lengths=0),
    dict(lengths=A[12] + 4), dict(k=A[13] + 8), dict(v=A[14] + 2), dict(k=0, v=0), dict(k_stride=255), dict(v_stride=260),
    dict(v_stride=128), dict(k_stride=0), dict(n=(1 << 24) + 1), dict(v=A[13]), dict(v=A[13] + 256),
    dict(v=A[13] + 512, k_stride=512), dict(v=A[13] + 512, k_stride=384, v_stride=384)])
def test_gather_refuses(kw):
    kv = create()
    assert KV.rwttt_kv_gather(kv, **{**GATHER, **kw}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_gather(kv, **{**GATHER, "n": 0, "k": 0}) == R.RWTTT_OK
    KV.rwttt_kv_destroy(kv)


def test_gather_needs_cache_and_table():
    for kw in (dict(k=None, v=None), dict(table=0)):
        kv = create(**kw)
        assert KV.rwttt_kv_gather(kv, **GATHER) == R.RWTTT_E_INVALID
        KV.rwttt_kv_destroy(kv)
    assert KV.rwttt_kv_gather(None, **GATHER) == R.RWTTT_E_INVALID


Q, K = 8 * 128, 2 * 128
ROTATE = dict(positions=A[10], n=3, q=A[11], q_stride=Q, q_out=A[12], q_out_stride=Q, k=A[13], k_stride=K, k_out=A[14],
              k_out_stride=K)
STRIDE = Q + 2 * K
PARTS = dict(q=A[11], q_stride=STRIDE, k=A[11] + 2 * Q, k_stride=STRIDE)


@pytest.mark.parametrize("kw", [
    dict(positions=0), dict(positions=A[10] + 4), dict(n=(1 << 24) + 1), dict(q=0), dict(q_out=0), dict(k=0), dict(k_out=0),
    dict(q=0, q_out=0, k=0, k_out=0), dict(q=A[11] + 2), dict(q_out=A[12] + 8), dict(k=A[13] + 4), dict(k_out=A[14] + 8),
    dict(q_stride=Q - 8), dict(q_out_stride=Q + 4), dict(k_stride=0), dict(k_out_stride=K - 8), dict(k_stride=1 << 41),
    # outputs over other rows, in part or with another stride
    dict(q_out=A[11] + 16), dict(q_out=A[11], q_out_stride=Q + 8), dict(q_out=A[11] + 2 * Q), dict(k_out=A[11]),
    dict(k_out=A[12]), dict(q_out=A[13]), dict(k_out=A[12] + 2 * Q),
    # within the rows of one projection: the keys' place is theirs, not the queries'
    dict(**PARTS, q_out=A[11] + 2 * Q, q_out_stride=STRIDE), dict(**PARTS, k_out=A[11], k_out_stride=STRIDE),
    dict(**PARTS, k_out=A[11] + 2 * Q + 2 * K - 16, k_out_stride=STRIDE),
    dict(**PARTS, k_out=A[11] + 2 * STRIDE - 16, k_out_stride=STRIDE)])
def test_rotate_refuses(kw):
    kv = create()
    rot = KV.make_rotary(128, KV.RWTTT_ROTARY_HALF, A[15])
    assert KV.rwttt_kv_rotate(kv, rot, **{**ROTATE, **kw}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_rotate(kv, rot, **{**ROTATE, "n": 0, "q": 0}) == R.RWTTT_OK
    KV.rwttt_kv_destroy(kv)


@pytest.mark.parametrize("args", [
    (0, 0, A[15]), (3, 0, A[15]), (130, 0, A[15]), (128, 2, A[15]), (128, -1, A[15]), (128, 0, 0), (128, 0, A[15] + 8),
    (128, 0, A[15], math.nan), (128, 0, A[15], math.inf), (128, 0, A[15], 1.0, 2), (128, 1, A[15], 1.0, -1)])
def test_rotate_refuses_a_bad_rotary(args):
    kv = create()
    assert KV.rwttt_kv_rotate(kv, KV.make_rotary(*args), **ROTATE) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_rotate(None, KV.make_rotary(128, 0, A[15]), **ROTATE) == R.RWTTT_E_INVALID
    assert R.lib().rwttt_kv_rotate(kv, None, A[10], 3, A[11], Q, A[12], Q, A[13], K, A[14], K, None) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


# outputs of three rows of 512 bytes, at A[13] and A[14], 512 apart unless said; queries' rows are of 2048
AT_K, AT_V, WIDE = A[13], A[14], dict(k_stride=1024, v_stride=1024)


@pytest.mark.parametrize("kw", [
    # the first and the last byte of either output, from below and from within
    dict(owners=AT_K), dict(owners=AT_K - 16, n=5), dict(owners=AT_K + 1536 - 16), dict(owners=AT_V + 512),
    dict(positions=AT_K), dict(positions=AT_V + 1536 - 16), dict(positions=AT_V - 16, n=5), dict(lengths=AT_V), dict(lengths=AT_K + 16),
    # between rows that are apart, where an array reaches the next one
    dict(**WIDE, owners=AT_K + 2048 - 16, n=5), dict(**WIDE, positions=AT_V + 2048 - 16, n=5)])
def test_gather_refuses_outputs_over_what_it_reads(kw):
    kv = create()
    assert KV.rwttt_kv_gather(kv, **{**GATHER, **kw}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


CACHE = 100 * 2 * 64 * 128 * 17 // 32           # bytes of a layer's keys or values
TABLE = 4 * 16 * 4


@pytest.mark.parametrize("kw", [
    dict(k=A[3]), dict(v=A[5]), dict(k=A[5]), dict(v=A[3]), dict(k=A[3] + CACHE - 16), dict(v=A[5] - 1536 + 16),
    dict(k=A[0]), dict(v=A[0] + TABLE - 16), dict(k=A[0] - 1536 + 16), dict(v=0, k=A[5] + 4096), dict(k=0, v=A[3] + 4096)])
def test_gather_refuses_outputs_over_the_pages_or_the_table(kw):
    kv = create()
    assert KV.rwttt_kv_gather(kv, **{**GATHER, **kw}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


@pytest.mark.parametrize("scale", ["k_scale", "v_scale"])
@pytest.mark.parametrize("side", ["k", "v"])
def test_gather_refuses_outputs_over_the_scales(scale, side):
    kv = create(cache_dtype=KV.RWTTT_FP8, k_scale=A[16], v_scale=A[17])
    at = A[16] if scale == "k_scale" else A[17]
    assert KV.rwttt_kv_gather(kv, **{**GATHER, side: at}) == R.RWTTT_E_INVALID
    assert KV.rwttt_kv_gather(kv, **{**GATHER, side: at - 1536 + 16}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


AT_Q, ROWS3 = A[12], 3 * 2 * Q                  # q_out: three rows of 2048 bytes


@pytest.mark.parametrize("kw", [
    dict(positions=AT_Q), dict(positions=AT_Q + ROWS3 - 16), dict(positions=AT_Q - 16, n=5), dict(positions=A[14]),
    dict(positions=A[14] + 3 * 2 * K - 16), dict(positions=A[11], q_out=A[11]), dict(positions=A[13] + 512, k_out=A[13]),
    dict(q=0, q_out=0, positions=A[14] + 512), dict(k=0, k_out=0, positions=AT_Q + 2048),
    # the queries of one projection turned in place: the place of keys and values is free, the next row is not
    dict(**PARTS, q_out=A[11], q_out_stride=STRIDE, n=300, positions=A[11] + 2 * Q)])
def test_rotate_refuses_outputs_over_the_positions(kw):
    kv = create()
    assert KV.rwttt_kv_rotate(kv, KV.make_rotary(128, 0, A[15]), **{**ROTATE, **kw}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


@pytest.mark.parametrize("turns", [AT_Q, AT_Q + ROWS3 - 16, AT_Q - 512 + 16, A[14], A[14] + 3 * 2 * K - 16, A[14] - 512 + 16])
def test_rotate_refuses_outputs_over_the_table(turns):
    """Of 64 pairs: 512 bytes."""
    kv = create()
    assert KV.rwttt_kv_rotate(kv, KV.make_rotary(128, 1, turns), **ROTATE) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)


# ---------------------------------------------------------------------------
# frequencies
# ---------------------------------------------------------------------------

PI = Fraction(3141592653589793238462643383279502884197169399375, 10 ** 48)


def power(x, e):
    """x^e for x > 0 to 2^-80 of itself: exp(e log x) in fractions."""
    def ln(v):
        k = 0
        while v > 2:
            v, k = v / 2, k + 1
        while v < 1:
            v, k = v * 2, k - 1
        z = (v - 1) / (v + 1)
        series = lambda z: 2 * sum(round_(z ** (2 * i + 1)) / (2 * i + 1) for i in range(60))  # noqa: E731
        return series(z) + k * series(Fraction(1, 3))

    def round_(v, bits=160):
        return Fraction(round(v * 2 ** bits), 2 ** bits)

    t = round_(e * ln(Fraction(x)))
    halvings = 0
    while abs(t) > Fraction(1, 4):
        t, halvings = t / 2, halvings + 1
    term, total = Fraction(1), Fraction(1)
    for i in range(1, 40):
        term = round_(term * t / i)
        total += term
    for _ in range(halvings):
        total = round_(total * total, 200)
    return total


@pytest.mark.parametrize("turning,base", [(2, 10000.0), (6, 10000.0), (64, 500000.0), (50, 1e6), (128, 1e7)])
@pytest.mark.parametrize("scaling", [KV.RWTTT_ROTARY_PLAIN, KV.RWTTT_ROTARY_LINEAR, KV.RWTTT_ROTARY_BASE, KV.RWTTT_ROTARY_PARTS])
def test_frequencies(turning, base, scaling):
    """Against fractions: the long double steps, a dozen of 2^-64, may be off by 16 * 2^-64 of the
    frequency (below 1/6 turn: 3 units; the base's logarithm scales the power's error, 24 at most), and the rounding by one."""
    if scaling == KV.RWTTT_ROTARY_BASE and turning == 2:
        with pytest.raises(R.RwtttError):
            KV.rwttt_kv_turns(turning, base, scaling, 8.0)
        return
    low, high, context, factor = 1.0, 32.0, 8192.0, 8.0
    got = KV.rwttt_kv_turns(turning, base, scaling, factor, low, high, context)
    assert len(got) == turning // 2
    for i, u in enumerate(got):
        e = Fraction(-2 * i, turning)
        w = power(base, e)
        if scaling == KV.RWTTT_ROTARY_BASE:
            w *= power(factor, e * Fraction(turning, turning - 2))
        t = w / (2 * PI)
        if scaling == KV.RWTTT_ROTARY_LINEAR:
            t /= Fraction(factor)
        if scaling == KV.RWTTT_ROTARY_PARTS:
            r = min(Fraction(1), max(Fraction(0), (Fraction(context) * t - Fraction(low)) / Fraction(high - low)))
            t *= r + (1 - r) / Fraction(factor)
        assert abs(u - t * 2 ** 64) <= 1 + 24 * float(t), (i, u)


def test_frequencies_by_hand():
    one = KV.rwttt_kv_turns(2, 10000.0)
    assert abs(one[0] - 2 ** 64 / (2 * math.pi)) <= 2 ** 12          # a turn in 2 pi positions
    plain, base = KV.rwttt_kv_turns(64, 1e4), KV.rwttt_kv_turns(64, 1e4, KV.RWTTT_ROTARY_BASE, 4.0)
    assert plain[0] == base[0] and abs(plain[-1] / base[-1] - 4.0) < 1e-9
    parts = KV.rwttt_kv_turns(64, 1e4, KV.RWTTT_ROTARY_PARTS, 4.0, 1.0, 32.0, 4096.0)
    assert parts[0] == plain[0] and abs(plain[-1] / parts[-1] - 4.0) < 1e-9


@pytest.mark.parametrize("args", [
    (0, 1e4), (3, 1e4), (64, 1.0), (64, math.nan), (64, math.inf), (64, -5.0), (64, 1e4, 4), (64, 1e4, -1),
    (64, 1e4, 1, 0.0), (64, 1e4, 1, -2.0), (64, 1e4, 1, math.nan), (64, 1e4, 2, math.inf), (2, 1e4, 2, 4.0),
    (64, 1e4, 3, 4.0, 1.0, 1.0, 100.0), (64, 1e4, 3, 4.0, 2.0, 1.0, 100.0), (64, 1e4, 3, 4.0, 1.0, 32.0, 0.0),
    (258, 1e4),
    (64, 1e4, 3, 4.0, math.nan, 32.0, 100.0), (64, 1e4, 3, 4.0, 1.0, math.inf, 100.0), (64, 1e4, 3, 4.0, 1.0, 32.0, math.nan)])
def test_frequencies_refuse(args):
    with pytest.raises(R.RwtttError) as e:
        KV.rwttt_kv_turns(*args)
    assert e.value.status == R.RWTTT_E_INVALID
    out = ctypes.POINTER(ctypes.c_uint64)()
    assert R.lib().rwttt_kv_turns(64, 1e4, 0, 1.0, 0.0, 1.0, 1.0, out) == R.RWTTT_E_INVALID
