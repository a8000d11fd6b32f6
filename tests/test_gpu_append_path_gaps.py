"""The append of a path some of whose entries are not stored: the others are, as if the runs
between them were appended by one call after the other (equal: scales and codes)."""
import numpy as np
import pytest

import test_gpu_draft as td
import test_gpu_paged as tp
from oracle import paged_oracle as po
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


def _case(rng, lens, new, n, page, H, D):
    """Requests of `lens` tokens that gain `new`: path, starts, slots and a cache of random codes."""
    B = len(lens)
    path = np.full((B, n), -1, np.int32)
    for b in range(B):
        path[b, :new[b]] = np.sort(rng.permutation(n)[:new[b]])
    pages = int(sum(-(-(x + y) // page) for x, y in zip(lens, new))) + 2
    table, _ = tp._table(rng, np.asarray(lens) + new, page, pages, int(max(-(-(x + y) // page) for x, y in zip(lens, new))) + 1)
    start = np.concatenate([[0], np.cumsum(new)])
    slots = np.concatenate([table[b, p // page] * page + p % page for b in range(B) for p in [np.arange(lens[b], lens[b] + new[b])]])
    codes = [po.e4m3_encode(rng.normal(size=(pages, H, page, D)) * 30) for _ in range(2)]
    scale = [2.0 ** rng.integers(-12, -6, (pages, H)).astype(np.float32) for _ in range(2)]
    return path, start, slots, codes, scale


@pytest.mark.parametrize("dtype,D", [("bfloat16", 128), ("bfloat16", 64), ("float32", 64), ("float32", 128)])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("growing", [True, False])
def test_an_entry_out_of_range_in_each_place(sbd, dtype, D, page, growing):  # noqa: F811
    rng = np.random.default_rng(page + D)
    n, H = 9, 2
    lens, new = [5, 0, 11], [8, 9, 7]
    path, start, slots, codes, scale = _case(rng, lens, new, n, page, H, D)
    x = rng.normal(size=(3, n, H, D)) * np.exp2(np.arange(n) * (1.5 if growing else -1.5))[None, :, None, None]
    for j in range(7):
        for value in (n, -1, 2 ** 31 - 1, -2 ** 31):
            p = path.copy()
            p[:, j] = value
            td._append(sbd, x, p, start, slots, codes, scale, page, dtype)
            assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE
    p = path.copy()
    p[:, 1::2] = -1                                  # every other one: as many segments as can be
    td._append(sbd, x, p, start, slots, codes, scale, page, dtype)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("page", [16, 64])
def test_a_slot_that_is_not_stored_in_each_place(sbd, dtype, page):  # noqa: F811
    rng = np.random.default_rng(page)
    n, H, D = 12, 3, 64
    path, start, slots, codes, scale = _case(rng, [3, 14], [12, 10], n, page, H, D)
    x = rng.normal(size=(2, n, H, D)) * np.exp2(rng.permutation(n))[None, :, None, None]
    for j in range(10):
        for value, code in ((-1, 0), (codes[0].shape[0] * page, sbd.SBD_DEVERR_PAGE)):
            s = slots.copy()
            s[start[:2] + j] = value
            td._append(sbd, x, path, start, s, codes, scale, page, dtype)
            assert sbd.sbd_device_error() == code


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_the_longest_path_with_gaps(sbd, dtype):  # noqa: F811
    """64 nodes in a page, and over four of them, every third one out of range; again and again alike."""
    rng = np.random.default_rng(64)
    n, H, D = 64, 2, 128
    for page, length in ((128, 60), (16, 7)):
        path, start, slots, codes, scale = _case(rng, [length, 0, 1], [64, 64, 40], n, page, H, D)
        x = rng.normal(size=(3, n, H, D)) * np.exp2(rng.integers(-8, 9, n))[None, :, None, None]
        p = path.copy()
        p[:, 1::3] = 64
        for _ in range(5):
            td._append(sbd, x, p, start, slots, codes, scale, page, dtype)
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE


def test_slots_in_another_order(sbd):  # noqa: F811
    """Slots that go down, jump back into a page or come twice: one after the other, too."""
    rng = np.random.default_rng(5)
    n, H, D, page = 8, 2, 64, 16
    codes = [po.e4m3_encode(rng.normal(size=(4, H, page, D)) * 30) for _ in range(2)]
    scale = [2.0 ** rng.integers(-12, -6, (4, H)).astype(np.float32) for _ in range(2)]
    path = np.arange(n, dtype=np.int32)[None]
    for slots in ([9, 8, 7, 6, 5, 4, 3, 2], [3, 4, 20, 21, 5, 6, 22, 23], [3, 3, 3, 4, 4, 5, 5, 6], [18, 16, 17, 18, 16, 5, 0, 1]):
        x = rng.normal(size=(1, n, H, D)) * np.exp2(np.arange(n))[None, :, None, None]
        td._append(sbd, x, path, np.array([0, n]), np.array(slots), codes, scale, page, "float32")
    assert sbd.sbd_device_error() == 0
