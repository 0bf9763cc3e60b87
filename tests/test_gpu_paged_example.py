"""The decode example: what does not fit, many owners, fast weights that are not zero."""

import pytest
import torch

from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd import paged_decode
from paper_2605_28053_amd.paged import PagedCache
from paper_2605_28053_amd.paged_decode import Decoder, Model
from tests.test_gpu_paged_decode import Dense

pytestmark = pytest.mark.gpu


def test_a_step_that_did_not_fit_is_reported_at_the_end(monkeypatch, capsys):
    extend, calls = PagedCache.extend, []

    def fifth_too_long(self, want):
        calls.append(1)
        return extend(self, want + (10 ** 6 if len(calls) == 5 else 0))

    monkeypatch.setattr(PagedCache, "extend", fifth_too_long)
    assert paged_decode.main(["--owners", "3", "--steps", "40", "--layers", "1"]) == R.RWTTT_E_INVALID
    assert f"status {R.RWTTT_E_INVALID}" in capsys.readouterr().out
    assert len(calls) > 30


@pytest.mark.parametrize("owners", [2, 66])
def test_owners_read_their_own_fast_weights(owners):
    """More owners than a READ group holds, states that are not zero: against the model in
    64 bits with each owner's W0 + D."""
    m = Model(n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, vocab=50, dtype=torch.float32)
    dec = Decoder(m, owners, max_rows=16, page_rows=16)
    g = torch.Generator().manual_seed(2)
    checked = sorted({0, 1, owners - 2, owners - 1})
    refs = {}
    for r in checked:
        refs[r] = Dense(m, 1)
        for l in range(2):
            d = 0.02 * torch.randn((512, 256), generator=g)
            dec.state[r][l][0].copy_(d)
            refs[r].w[l]["w0"] = refs[r].w[l]["w0"] + d.double()
    for t in range(4):
        tokens = torch.randint(0, 50, (owners,), generator=g)
        got = dec.step(tokens.cuda(), dec.cache.lengths + 1).double().cpu()
        for r in checked:
            (y,) = refs[r].step([int(tokens[r])], {0})
            assert float((got[r] - y).norm() / y.norm()) < 1e-4, (t, r)
    assert int(dec.status) == R.RWTTT_OK
    dec.close()
