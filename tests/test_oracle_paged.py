"""The 64-bit forms of the paged cache operators against hand-made cases and
against independent statements of the same thing (CPU only)."""
import math

import numpy as np
import pytest

import oracle
from oracle import paged_oracle as po


def test_e4m3_values_and_rounding():
    assert po.E4M3[0x7e] == 448.0 and po.E4M3[0x01] == 2.0 ** -9 and po.E4M3[0x08] == 2.0 ** -6
    assert math.isnan(po.E4M3[0x7f]) and math.isnan(po.E4M3[0xff])
    finite = [c for c in range(256) if c & 127 != 127]
    assert (po.e4m3_encode(po.E4M3[finite]) == finite).all()
    # ties go to the even code, beyond the range to the largest value
    assert po.E4M3[po.e4m3_encode([17.0, 19.0, 1e9, -np.inf, 2.0 ** -10, 3 * 2.0 ** -10])].tolist() == \
        [16.0, 20.0, 448.0, -448.0, 0.0, 2.0 ** -8]


def test_e4m3_agrees_with_torch():
    import torch
    x = np.random.default_rng(0).normal(size=20000) * 2.0 ** np.random.default_rng(1).integers(-12, 9, 20000)
    x = np.clip(x, -448, 448).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (po.e4m3_encode(x) == ref).all()


@pytest.mark.parametrize("amax,scale", [(448.0, 1.0), (448.5, 2.0), (0.0, 2.0 ** -126), (1.75, 2.0 ** -8),
                                        (1.0, 2.0 ** -8), (1.76, 2.0 ** -7), (3e38, 2.0 ** 120)])
def test_scale_is_the_smallest_power_of_two(amax, scale):
    assert po.scale_for(amax) == scale


def test_tables_by_hand():
    # pages of 4; request 0 grows 3 -> 6, request 1 ends (2 pages back), request 2 is new
    table = np.array([[7, -1, -1], [3, 5, -1], [-1, -1, -1]], np.int32)
    free = np.array([0, 1, 9, 9, 9], np.int32)
    t, length, start, slots, n, f = po.block_tables([3, 7, 0], [6, 0, 5], table, free, 2, 4, 10)
    # released: 3 then 5, the first one topmost; granted 3 to request 0, then 5, 1 to request 2
    assert t.tolist() == [[7, 3, -1], [-1, -1, -1], [5, 1, -1]]
    assert length.tolist() == [6, 0, 5] and start.tolist() == [0, 3, 3, 8]
    assert slots.tolist() == [31, 12, 13, 20, 21, 22, 23, 4, -1, -1]
    assert n == 1 and f.tolist() == [0, 1, 5, 3, 9]


def test_tables_refuse_what_does_not_fit():
    table = np.full((3, 4), -1, np.int32)
    free = np.arange(3, dtype=np.int32)
    t, length, start, slots, n, _ = po.block_tables([0, 0, 0], [8, 8, 4], table, free, 3, 4, 100)
    assert length.tolist() == [8, 0, 0] and n == 1 and (t[1:] == -1).all()
    assert start.tolist() == [0, 8, 16, 20] and (slots[8:20] == -1).all()
    # the slot map bounds them too
    _, length, _, slots, n, _ = po.block_tables([0, 0, 0], [4, 4, 4], table, free, 3, 4, 7)
    assert length.tolist() == [4, 0, 0] and slots.tolist() == [8, 9, 10, 11, -1, -1, -1] and n == 2


def test_shrinking_what_was_granted_restores_the_pages():
    rng = np.random.default_rng(0)
    for _ in range(50):
        B, P, cols = int(rng.integers(1, 7)), 16, 6
        lens = rng.integers(0, 40, B)
        perm = rng.permutation(64).astype(np.int32)
        table = np.full((B, cols), -1, np.int32)
        at = 0
        for b in range(B):
            m = -(-int(lens[b]) // P)
            table[b, :m] = perm[at:at + m]
            at += m
        free = np.full(64, -7, np.int32)
        free[:64 - at] = perm[at:]
        grown = lens + rng.integers(0, 50, B)
        t, length, _, _, n, f = po.block_tables(lens, grown, table, free, 64 - at, P, 1000)
        assert (length == grown).all()
        t2, length2, _, _, n2, f2 = po.block_tables(length, lens, t, f, n, P, 0)
        assert (t2 == table).all() and n2 == 64 - at and (f2[:n2] == free[:n2]).all()


def test_append_rescales_the_page():
    codes = np.zeros((2, 1, 16, 4), np.uint8)
    scale = np.full((2, 1), np.nan, np.float32)
    x = np.full((3, 1, 4), 1.75)
    codes, scale = po.cache_append(x, [16, 17, -1], codes, scale, 16)
    assert scale[1, 0] == 2.0 ** -8 and (po.E4M3[codes[1, 0, :2]] == 448).all()
    assert np.isnan(scale[0, 0]) and (codes[1, 0, 2:] == 0).all()
    codes, scale = po.cache_append(np.full((1, 1, 4), 7.0), [18], codes, scale, 16)
    assert scale[1, 0] == 2.0 ** -6
    assert (po.E4M3[codes[1, 0, :3]] * scale[1, 0] == [[1.75] * 4, [1.75] * 4, [7.0] * 4]).all()


def test_attention_agrees_with_the_dense_oracle():
    rng = np.random.default_rng(3)
    B, k, Hq, H, D, P, cols = 2, 3, 4, 2, 64, 16, 3
    codes = [po.e4m3_encode(rng.normal(size=(8, H, P, D)) * 100) for _ in range(2)]
    scale = [2.0 ** rng.integers(-9, -6, (8, H)).astype(np.float64) for _ in range(2)]
    table = np.array([[3, 1, 6], [0, -1, -1]], np.int32)
    lens = np.array([37, 0], np.int32)
    q, kb, vb = (rng.normal(size=(B, k, h, D)) for h in (Hq, H, H))
    dense = [np.zeros((B, cols * P, H, D)) for _ in range(2)]
    for w in range(2):
        for b in range(B):
            x = po.paged_keys(codes[w], scale[w], table[b], int(lens[b]), P)
            dense[w][b, :lens[b]] = x.transpose(1, 0, 2)
    ref = oracle.block_attention(q, dense[0], dense[1], lens, kb, vb)
    out, spread, _ = po.block_attention(q, codes[0], codes[1], scale[0], scale[1], table, lens, kb, vb)
    assert np.abs(out - ref).max() < 1e-12 * np.abs(ref).max() * 1e3
    assert (spread >= np.abs(out) - 1e-12).all()
