"""The comparison that attention's tests on pools in 4 bits rest on: what it must not let pass."""
import math

import pytest
import torch

from held_calls import compare


def case():
    g = torch.Generator().manual_seed(1)
    out, lse = torch.randn((3, 2, 8), generator=g).double(), torch.randn((3, 2), generator=g).double()
    out[2, 1], lse[2, 1] = 0.0, -math.inf
    return out, lse, torch.full_like(out, 0.01), torch.full_like(lse, 1e-5)


def test_results_within_their_bounds_pass():
    out, lse, off, lse_off = case()
    compare((out + 0.005).half(), (lse + 1e-7).float(), (out, lse, off, lse_off))
    compare((out + 0.005).half(), None, (out, lse, off, lse_off))


@pytest.mark.parametrize("wrong", [math.nan, math.inf, -math.inf, 100.0])
def test_results_that_are_wrong_do_not(wrong):
    want = case()
    for at in ((0, 0, 0), (2, 1, 7), slice(None)):
        got = want[0].half()
        got[at] = wrong
        with pytest.raises(AssertionError):
            compare(got, want[1].float(), want)
        with pytest.raises(AssertionError):
            compare(got, None, want)
    for at in ((0, 0), (2, 1), slice(None)):
        norm = want[1].float()
        norm[at] = wrong
        if wrong == -math.inf and at == (2, 1):
            continue
        with pytest.raises(AssertionError):
            compare(want[0].half(), norm, want)
