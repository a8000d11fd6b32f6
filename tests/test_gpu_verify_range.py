"""Verification of drafts where logits over tau are large, one way or the other: the
definition is p = softmax(z / tau) whatever their size.

Tolerances are those of test_gpu_draft.py: whole numbers equal wherever no decision is within
10^-3 of its border, ln p to 2^-16 + 2^-21 |ln p|.  (The exponent (z - max) log2(e) / tau has
three roundings, 3 * 2^-24 of it, and each of them counts the same in ln p.)
"""
import numpy as np
import pytest

import test_gpu_draft as td
import test_gpu_paged as tp
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [2, 40])
@pytest.mark.parametrize("over", [1, 10, 42, 80])
def test_a_logit_just_past_what_sums_take_at_once(sbd, B, over):  # noqa: F811
    """2^23 tau and a little: whatever else is there, it takes all."""
    rng = np.random.default_rng(over)
    for tau in (1.0, 2.0 ** -20):
        for drawn in (True, False):
            V = 5003
            target = rng.normal(size=(B, 3, V)) * 0.5 * tau
            draft = rng.normal(size=(B, 3, V)) * 0.5 * tau
            at = rng.integers(0, V, B)
            target[np.arange(B), 0, at] = np.float32((2.0 ** 23 + over) * tau)
            parent = np.repeat([[-1, 0, 1]], B, 0).astype(np.int32)
            token = np.stack([np.zeros(B), at, rng.integers(0, V, B)], 1).astype(np.int32)
            case = (target, draft if drawn else None, parent, token, np.full((B, 3), 0.5), rng.gumbel(size=(B, V)))
            _, tokens, logprob, count = td._verify(sbd, case, tau, "float32", 0.4)
            assert (count >= 2).all() and (tokens[:, 0] == at).all() and (np.abs(logprob[:, 0]) <= 2.0 ** -16).all()
    assert sbd.sbd_device_error() == 0
