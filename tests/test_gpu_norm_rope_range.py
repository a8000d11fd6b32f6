"""Norms and rotation at the ends of their ranges."""
import math

import numpy as np
import pytest

from oracle import draft_oracle as do
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
def test_angles_of_far_positions(sbd, interleaved, sign):  # noqa: F811
    """Of the pair (1, 0) the cosine and the sine come out.  Angles are within 2^-26 of a turn
    and 2^-52 of the whole turns (the header's bound), cosine and sine within two units of 1."""
    import torch
    inv = sign * np.array([1e-12, 3.3e-11, 7.7e-10, 2e-8, 1e-6, 5e-5, 0.0123, 0.9], np.float32)
    far = np.array([2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 10 ** 6 + 3, 4099, 1, -1, 0], np.int32)
    x = torch.zeros(len(far), 1, 64, device="cuda")
    one, two = (slice(0, 16, 2), slice(1, 16, 2)) if interleaved else (slice(0, 8), slice(8, 16))
    x[..., one] = 1
    q, _, _ = sbd.sbd_qk_norm_rope(x, x, None, torch.from_numpy(far).cuda(), torch.from_numpy(inv).cuda(), interleaved=interleaved)
    q = q.double().cpu().numpy()
    for t, pos in enumerate(far):
        for j, f in enumerate(inv):
            a = 2 * math.pi * do.turn(pos, f)
            turns = abs(float(pos) * float(f)) / (2 * math.pi)
            tol = 2 * math.pi * (2.0 ** -26 + 2.0 ** -52 * turns) + 2 * 2.0 ** -24
            got = q[t, 0, one][j], q[t, 0, two][j]
            assert abs(got[0] - math.cos(a)) <= tol and abs(got[1] - math.sin(a)) <= tol, (pos, f)
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("size,eps", [(1e18, 1e-6), (1e25, 1e-6), (3e37, 0.0), (3e37, 3e38), (1e-18, 0.0), (1e-25, 0.0), (1e-37, 0.0),
                                      (1e-20, 1e-38), (1e-25, 1e-6)])
@pytest.mark.parametrize("T,interleaved", [(5, True), (6, False), (5000, False)])
def test_norms_of_rows_large_and_small(sbd, dtype, size, eps, T, interleaved):  # noqa: F811
    """Squares past fp32's range, or below it.  Tolerance as in test_gpu_draft.py: half a step of the
    output, 40 * 2^-24 of the pair, and what a step of the smallest inputs makes."""
    import torch
    dt = getattr(torch, dtype)
    D, Hq, H = 128, 3, 2
    gen = torch.Generator().manual_seed(T)
    x = (size * torch.randn(T, Hq + H, D, generator=gen).clamp(-4, 4)).to(dt)
    x[1] *= 0 if eps else 1                          # a row of zeros
    x[2, 0, 7:] = 0                                  # a few elements make the row
    x[3, :, ::2] *= 1e-3
    w = (1 + 0.3 * torch.randn(2, D, generator=gen)).to(dt)
    inv = (1e4 ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    pos = torch.arange(T, dtype=torch.int32)
    out = sbd.sbd_qk_norm_rope(x[:, :Hq].cuda(), x[:, Hq:].cuda(), None, pos.cuda(), inv.cuda(), *w.cuda(), eps=eps, interleaved=interleaved)
    eps = float(np.float32(eps))
    some = np.unique(np.concatenate([np.arange(5), np.arange(T - 3, T)]))
    half = torch.finfo(dt).eps / 2
    for got, rows, weight in zip(out, (x[:, :Hq], x[:, Hq:]), w):
        rows = rows[torch.from_numpy(some)].double().numpy()
        args = (weight.double().numpy(), eps, interleaved)
        ref, y = do.norm_rope(rows, pos.numpy()[some], inv.numpy(), *args), do.norm_rope(rows, None, None, *args)
        pair = np.abs(y)
        if interleaved:
            pair[..., 0:64:2] = pair[..., 1:64:2] = pair[..., 0:64:2] + pair[..., 1:64:2]
        else:
            pair[..., :32] = pair[..., 32:64] = pair[..., :32] + pair[..., 32:64]
        got = got[torch.from_numpy(some).cuda()].double().cpu().numpy()
        worst = (np.abs(got - ref) / (half * np.abs(ref) + 40 * 2.0 ** -24 * pair + 1e-35)).max()
        assert worst <= 1.0, worst
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_norms_of_powers_of_two_apart(sbd, dtype):  # noqa: F811
    """Without eps a row and a power of two times it have the same norm (rounded sums: a step)."""
    import torch
    dt = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(4, 2, 64, generator=gen).to(dt).cuda()
    w = torch.ones(64, dtype=dt, device="cuda")
    ref, _, _ = sbd.sbd_qk_norm_rope(x, x, None, None, None, w, w, eps=0.0)
    for e in (-100, -80, -60, -40, 40, 60, 80, 100, 120):
        q, _, _ = sbd.sbd_qk_norm_rope(x * 2.0 ** e, x, None, None, None, w, w, eps=0.0)
        step = torch.finfo(dt).eps
        assert ((q - ref).float().abs() <= step * ref.float().abs()).all(), e
    # an infinity is its own row's matter, and what it leaves is the formula's: 0, and NaN where it is
    x[1, 0, 5] = float("inf")
    q, _, _ = sbd.sbd_qk_norm_rope(x, x, None, None, None, w, w)
    assert torch.isnan(q[1, 0, 5]) and (torch.cat([q[1, 0, :5], q[1, 0, 6:]]) == 0).all() and torch.isfinite(q[0]).all()
    assert sbd.sbd_device_error() == 0
