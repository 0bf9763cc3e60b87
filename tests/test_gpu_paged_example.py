"""The decode example where something does not fit."""

import pytest
import torch

from paper_2605_28053_amd import _rwttt as R
from paper_2605_28053_amd import paged_decode
from paper_2605_28053_amd.paged import PagedCache

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
