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


TAUS = [2.0 ** -20, 1e-6, 1e-5, 1e-3]


def _rounded(x, dtype):
    import torch
    return torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).double().numpy()


def _near_greedy(rng, B, n, V, drawn, tau, lo, hi, dtype):
    """Logits between lo and hi, in most rows the best ones some tau apart, and drafts like
    them or not; drafted tokens drawn from those, or given: the best ones or any of them."""
    target = rng.uniform(lo, hi, (B, n, V))
    best = rng.integers(0, V, (B, n, 4))
    for b in range(B):
        for i in range(n):
            if rng.random() < 0.7:
                target[b, i, best[b, i]] = target[b, i].max() + tau * rng.uniform(0, 3, 4)
    like = rng.random((B, n, 1)) < 0.5
    draft = np.where(like, target + 0.3 * tau * rng.normal(size=target.shape), rng.uniform(lo, hi, target.shape))
    target, draft = _rounded(target, dtype), _rounded(draft, dtype)
    parent = td._trees(rng, B, n)
    token = np.zeros((B, n), np.int32)
    for b in range(B):
        for i in range(1, n):
            p = parent[b, i]
            if p >= 0:
                token[b, i] = np.argmax((draft if drawn else target)[b, p] / tau + rng.gumbel(size=V))
                if not drawn and rng.random() < 0.3:
                    token[b, i] = rng.choice(best[b, p])
    return target, draft if drawn else None, parent, token, rng.random((B, n)), rng.gumbel(size=(B, V))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("B,n,V", [(3, 5, 1001), (60, 6, 300), (1, 4, 50257), (200, 3, 4099)])
def test_small_temperatures(sbd, dtype, drawn, tau, B, n, V):  # noqa: F811
    tau = float(np.float32(tau))
    rng = np.random.default_rng(B + V)
    for lo, hi in ((10, 100), (-100, -10), (-5, 5)):
        case = _near_greedy(rng, B, n, V, drawn, tau, lo, hi, dtype)
        td._verify(sbd, case, tau, dtype, 0.7 if B > 9 else 0.0)
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tau", TAUS + [0.5, 2.0 ** 20])
def test_three_logits(sbd, dtype, tau):  # noqa: F811
    """(20, 12, 9): nothing but the first where tau is small."""
    import torch
    z = torch.full((1, 2, 100), -40.0, device="cuda").to(getattr(torch, dtype))
    z[0, :, [3, 50, 99]] = torch.tensor([20.0, 12.0, 9.0], device="cuda").to(z.dtype)
    g = torch.zeros(1, 100, device="cuda")
    for x, accepted in ((3, True), (50, tau > 1)):
        u = torch.full((1, 2), 1e-4 if tau > 1 else 0.9999 if tau < 0.5 else 1e-3, device="cuda")
        _, tokens, logprob, count = sbd.sbd_verify_tree(z, None, tp._i32([[-1, 0]]), tp._i32([[0, x]]), u, g, tau)
        assert count.tolist() == [2 if accepted else 1] and tokens[0, 0].item() == (x if accepted else 3)
        assert tau >= 0.5 or abs(logprob[0, 0].item()) <= 2.0 ** -16
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("tau", TAUS + [1.0, 0.0])
def test_masked_logits_never_come_out(sbd, dtype, drawn, tau):  # noqa: F811
    """Rows of a few logits among masked ones, which lie at -inf, at NaN or at a type's lowest
    value, and whose ordinary ones are all far below zero (log-probabilities), far above it,
    or so far that only the type's range bounds them."""
    import torch
    tau = float(np.float32(tau))
    rng = np.random.default_rng(11)
    low = float(torch.finfo(getattr(torch, dtype)).min)
    rows = [(m, c) for m in (-np.inf, np.nan, low) for c in (-30.0, -3e3, 30.0, 1e9, -1e9, 1e30, -1e30)]
    B, n = len(rows), 3
    for V in (64, 1003, 20000):
        keep = rng.permutation(V)[:4]
        out = np.flatnonzero(~np.isin(np.arange(V), keep))
        target, draft = np.empty((2, B, n, V))
        for b, (m, c) in enumerate(rows):
            target[b], draft[b] = m, m
            for z in (target, draft):
                z[b][:, keep] = c * (1 + 0.25 * rng.random((n, 4)))
        target, draft = _rounded(target, dtype), _rounded(draft, dtype)
        parent = np.repeat([[-1, 0, 0]], B, 0).astype(np.int32)
        token = np.zeros((B, n), np.int32)
        token[:, 1] = keep[draft[:, 0][:, keep].argmax(1)] if drawn else out[0]
        token[:, 2] = keep[draft[:, 0][:, keep].argmax(1)] if drawn else rng.choice(keep, B)
        case = (target, draft if drawn else None, parent, token, np.maximum(rng.random((B, n)), 1e-6), rng.gumbel(size=(B, V)))
        _, tokens, logprob, _ = td._verify(sbd, case, tau, dtype, 0.5)
        assert set(tokens.ravel().tolist()) <= {-1, *keep.tolist()}
        assert np.isfinite(logprob).all()
    assert sbd.sbd_device_error() == 0
