"""Arrays that lie between the rows of an output do not overlap it, and are read as they are elsewhere."""

import pytest
import torch

from paper_2605_28053_amd import _rwttt_kv as KV
from tests.kv4_util import Cache4
from tests.kv_util import ok, stream

pytestmark = pytest.mark.gpu


def rows_with_gaps(n, width, gap, fill):
    """Rows [n, width] of bf16 with `gap` bytes behind each, and the bytes of a gap."""
    buf = torch.full((n, width + gap // 2), fill, dtype=torch.bfloat16, device="cuda")

    def between(i, values, dtype=torch.int32):
        at = buf[i, width:].view(dtype)[:len(values)]
        at.copy_(torch.tensor(values, dtype=dtype))
        return at
    return buf, buf[:, :width], between


def test_gather_between_rows():
    c = Cache4([40, 90], H=2, G=1, D=64, page=16, io="bf16", seed=1)
    owners, positions = [1, 0, 1, -1, 0], [89, 0, 17, 3, 39]
    k_buf, k, in_k = rows_with_gaps(5, 128, 64, 7.0)
    v_buf, v, in_v = rows_with_gaps(5, 128, 64, 7.0)
    o, p, lengths = in_k(0, owners), in_v(3, positions), in_k(3, [40, 90])
    before = [b[:, 128:].clone() for b in (k_buf, v_buf)]
    ok(KV.rwttt_kv_gather(c.kv, 0, o.data_ptr(), p.data_ptr(), lengths.data_ptr(), 5, k.data_ptr(), k.stride(0), v.data_ptr(),
                          v.stride(0), stream()))
    torch.cuda.synchronize()
    for x, rows in (("k", k), ("v", v)):
        for i in range(5):
            want = c.rows_of(owners[i], 0, x, [positions[i]]) if owners[i] >= 0 else None
            got = rows[i, :64].double().cpu()
            assert bool((got == 7.0).all()) if want is None else torch.equal(got[None], want), (x, i)
    assert all(torch.equal(b[:, 128:].view(torch.int16), a.view(torch.int16)) for a, b in zip(before, (k_buf, v_buf)))
    c.close()
