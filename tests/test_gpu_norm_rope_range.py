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
