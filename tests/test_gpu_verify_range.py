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


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("x", [-np.inf, np.nan, 3e38])
def test_rows_that_the_walk_does_not_come_to_change_nothing(sbd, dtype, x):  # noqa: F811
    """Bit for bit, also where two rows are worked on at once: a first child's row is masked
    altogether, or full of what the fast sums do not take."""
    import torch
    rng = np.random.default_rng(4)
    for V in (777, 128256) + 30 * (20011,):
        target, draft = 2 * rng.normal(size=(2, 1, 4, V))
        p, q = (np.exp(z[0, 0]) / np.exp(z[0, 0]).sum() for z in (target, draft))
        token = np.array([[0, int(np.argmax(q - p)), 1, 2]], np.int32)             # refused
        args = [tp._i32([[-1, 0, 1, 1]]), tp._i32(token), td._f32(np.full((1, 4), 0.9999)), td._f32(rng.gumbel(size=(1, V))), 1.0]
        outs = []
        for bad in (False, True):
            z, d = (torch.from_numpy(y.astype(np.float32)).to(getattr(torch, dtype)).cuda() for y in (target, draft))
            if bad:
                z[:, 1:], d[:, 1:] = x, x
            outs.append(sbd.sbd_verify_tree(z, d, *args))
        assert outs[0][3].tolist() == [1]
        for a, b in zip(*outs):
            assert torch.equal(a, b), V
    assert sbd.sbd_device_error() == 0
