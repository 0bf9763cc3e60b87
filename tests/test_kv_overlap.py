"""extend's arrays must not overlap, in part neither.  No GPU: every refusal comes before a launch."""

import pytest

pytest.importorskip("paper_2605_28053_amd._rwttt",
                    reason="librwttt.so not built (python -m paper_2605_28053_amd.build)")
from paper_2605_28053_amd import _rwttt as R  # noqa: E402
from paper_2605_28053_amd import _rwttt_kv as KV  # noqa: E402
from tests.test_kv_host import A, EXTEND, create  # noqa: E402


@pytest.mark.parametrize("kw", [
    dict(lengths=A[10] + 16), dict(lengths=A[11] - 16), dict(start=A[12] - 16), dict(new_pos=A[14] + 16),
    dict(owners=A[16] + 16), dict(positions=A[17] - 16), dict(result=A[15] + 16),
    dict(lengths=A[0] + 240), dict(slots=A[0] + 16), dict(result=A[1]), dict(owners=A[1] + 384), dict(start=A[1] - 16),
    dict(have=A[0]), dict(want=A[1] + 32), dict(pos=A[0] + 64)])
def test_extend_refuses_arrays_that_overlap(kw):
    """Eight owners of 16 pages, 100 pages, maps of 8: an output over an input, another output,
    the table or the ring; an input over the table or the ring."""
    kv = create(n_owners=8)
    assert KV.rwttt_kv_extend(kv, **{**EXTEND, "cap": 8, **kw}) == R.RWTTT_E_INVALID
    KV.rwttt_kv_destroy(kv)
