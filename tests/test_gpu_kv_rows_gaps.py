"""Arrays that lie between the rows of an output do not overlap it, and are read as they are elsewhere."""

import pytest
import torch

from paper_2605_28053_amd import _rwttt_kv as KV
from tests.kv4_util import Cache4
from tests.kv_util import dev, i32, ok, stream
from tests.test_gpu_rotary import Rotor

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


@pytest.mark.parametrize("in_place", [True, False])
def test_rotate_between_rows(in_place):
    f = Rotor(2, 1, 64, 64, "half", "bf16")
    pos, x = [5, -1, 100000, 0], torch.randn((4, 128), generator=torch.Generator().manual_seed(1)).bfloat16()
    buf, q, between = rows_with_gaps(4, 128, 320, 7.0)
    q.copy_(x)
    src = q if in_place else dev(x)
    at, table = between(0, pos), between(2, f.units[:32], torch.uint64)
    before = buf[:, 128:].clone()
    rot = KV.make_rotary(64, KV.RWTTT_ROTARY_HALF, table.data_ptr())
    ok(KV.rwttt_kv_rotate(f.kv, rot, at.data_ptr(), 4, src.data_ptr(), src.stride(0), q.data_ptr(), q.stride(0), 0, 0, 0, 0,
                          stream()))
    want = dev(x).view(4, 2, 64)
    f(i32(pos), q=want, q_out=want)
    torch.cuda.synchronize()
    assert torch.equal(q, want.view(4, 128)) and torch.equal(buf[:, 128:].view(torch.int16), before.view(torch.int16))
    f.close()
