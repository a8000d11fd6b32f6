"""The paged 8-bit cache on the GPU against its 64-bit forms.

Tables and append are exact: whole numbers, and codes and scales whose
arithmetic (division by a power of two, one rounding) is exact in fp32.
Attention is held to a bound per element, from what its steps round:
  bf16  probabilities enter the second product with 8 significant bits (2^-8
        of sum p |v|, both sides together), the output is rounded once
        (2^-9 |o|), q and the block's keys and values are carried to 2^-17 of
        their row's largest element, which moves a score by 2^-17 wobble;
  fp32  sums of n terms in fp32: (n + D) 2^-24 of sum p |v| and D 2^-24 wobble.
"""
import numpy as np
import pytest

from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbd():
    import paper_2509_04185_gb300 as m
    return m


def _i32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def _f8(codes):
    import torch
    return torch.from_numpy(np.ascontiguousarray(codes)).cuda().view(torch.float8_e4m3fn)


def _bytes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def _table(rng, lens, page, n_pages, cols, spare=0):
    perm = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), cols), -1, np.int32)
    at = 0
    for b, x in enumerate(lens):
        m = -(-int(x) // page)
        table[b, :m] = perm[at:at + m]
        at += m
    return table, perm[at:]


# ------------------------------------------------------------------ tables

def _tables(sbd, lens, target, table, free, n_free, page, max_new):
    ref = po.block_tables(lens, target, table, free, n_free, page, max_new)
    f = _i32(free)
    got = sbd.sbd_block_tables(_i32(lens), _i32(target), _i32(table), f, _i32([n_free]), page, max_new)
    for name, g, r in zip(("table", "length", "start", "slots"), got, ref):
        assert (g.cpu().numpy() == r).all(), name
    assert got[4].item() == ref[4]
    assert (f.cpu().numpy()[:ref[4]] == ref[5][:ref[4]]).all()
    return got, f


@pytest.mark.parametrize("batch,page,hi,pool", [(1, 16, 1, 1.5), (1, 64, 100000, 1.5), (3, 16, 50, 0.5), (33, 32, 300, 1.5),
                                                (257, 128, 2000, 0.9), (300, 16, 700, 0.6), (4096, 64, 200, 1.2)])
@pytest.mark.parametrize("seed", range(3))
def test_tables(sbd, batch, page, hi, pool, seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, hi + 1, batch)
    target = np.where(rng.random(batch) < 0.3, rng.integers(0, lens + 1),
                      lens + rng.integers(0, hi + 2, batch) * (rng.random(batch) < 0.8))
    cols = -(-(2 * hi + 2) // page) + int(rng.integers(0, 3))
    held = int((-(-lens // page)).sum())
    n_pages = max(held, int(pool * (-(-target // page)).sum()), 1)
    table, spare = _table(rng, lens, page, n_pages, cols)
    free = np.full(n_pages, -5, np.int32)
    free[:len(spare)] = spare
    total = int(np.maximum(target - lens, 0).sum())
    _tables(sbd, lens, target, table, free, len(spare), page, total + int(rng.integers(0, 9)) if seed else total * 3 // 4)
    assert sbd.sbd_device_error() == 0


def test_tables_grow_then_shrink_is_nothing(sbd):
    rng = np.random.default_rng(5)
    lens, page, cols = rng.integers(0, 900, 40), 32, 64
    table, spare = _table(rng, lens, page, 4000, cols)
    free = np.concatenate([spare, np.full(4000 - len(spare), -1, np.int32)])
    (t, length, _, _, n), f = _tables(sbd, lens, lens + 700, table, free, len(spare), page, 28000)
    t2, length2, _, slots, n2 = sbd.sbd_block_tables(length, _i32(lens), t, f, n, page, 0)
    assert (t2.cpu().numpy() == table).all() and (length2.cpu().numpy() == lens).all() and slots.numel() == 0
    assert n2.item() == len(spare) and (f.cpu().numpy()[:len(spare)] == spare).all()


def test_tables_without_lengths_in_range_stay(sbd):
    table = np.array([[0, 1], [2, -1], [-1, -1]], np.int32)
    free = np.array([3, 4, 5, 0, 0, 0], np.int32)
    _tables(sbd, np.array([20, -3, 40]), np.array([99, 16, 16]), table, free, 3, 16, 50)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_CACHE_LEN
    got = sbd.sbd_block_tables(_i32([0]), _i32([16]), _i32([[-1]]), _i32([0]), _i32([7]), 16, 16)
    assert got[4].item() == 0 and sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE


# ------------------------------------------------------------------ append

def _append(sbd, x, slots, codes, scale, page, dtype, layout):
    """Appends x as keys and -2 x as values; layout: how the tokens lie in memory."""
    import torch
    T, H, D = x[0].shape
    t = [torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(dtype).cuda() for a in x]
    if layout == "fused":                                   # slices of one projection
        w = torch.randn(T, 2 * H + 3, D, device="cuda").to(dtype)
        w[:, 3:3 + H], w[:, 3 + H:] = t[0], t[1]
        t = [w[:, 3:3 + H], w[:, 3 + H:]]
    elif layout == "blocks":                                # leading rows of blocks of 8 (T % 5 == 0)
        w = torch.randn(2, T // 5, 8, H, D, device="cuda").to(dtype)
        for i in range(2):
            w[i, :, :5] = t[i].view(T // 5, 5, H, D)
        t = [w[0][:, :5], w[1][:, :5]]
    caches, scales = [_f8(c) for c in codes], [torch.from_numpy(s.copy()).cuda() for s in scale]
    sbd.sbd_cache_append_q8(t[0], t[1], _i32(slots), *caches, *scales)
    for i in range(2):
        flat = t[i].float().cpu().numpy().reshape(T, H, D)
        rc, rs = po.cache_append(flat, slots, codes[i], scale[i], page)
        assert np.array_equal(scales[i].cpu().numpy(), rs, equal_nan=True)
        got = _bytes(caches[i])
        nan = (rc & 127) == 127
        assert ((got & 127) == 127)[nan].all() and (got == rc)[~nan].all()
    return caches, scales


def _slots(rng, lens, new, page, n_pages):
    after = np.asarray(lens) + np.asarray(new)
    table, _ = _table(rng, after, page, n_pages, max(int((-(-after // page)).max()), 1))
    return np.concatenate([[int(table[b, i // page]) * page + i % page for i in range(lens[b], after[b])]
                           for b in range(len(lens))]).astype(np.int64)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("page,D,H,layout", [(16, 128, 8, "plain"), (32, 64, 1, "fused"), (64, 128, 3, "blocks"),
                                             (128, 64, 2, "plain"), (128, 128, 2, "fused")])
@pytest.mark.parametrize("batch,lo,hi", [(1, 1, 1), (4, 5, 5), (5, 200, 300), (70, 1, 1), (45, 0, 30)])
def test_append(sbd, dtype, page, D, H, layout, batch, lo, hi):
    import torch
    rng = np.random.default_rng(batch * page + D)
    if layout == "blocks":
        lo = hi = 5
    lens, new = rng.integers(0, 200, batch), rng.integers(lo, hi + 1, batch)
    slots = _slots(rng, lens, new, page, int((-(-(lens + new) // page)).sum()) + 2)
    if not len(slots):
        pytest.skip("no token")
    n_pages = int(slots.max()) // page + 1
    size = 2.0 ** rng.integers(-6, 6, (len(slots), 1, 1))
    x = rng.normal(size=(len(slots), H, D)) * size
    codes = [rng.integers(0, 256, (n_pages, H, page, D)).astype(np.uint8) for _ in range(2)]
    scale = [(2.0 ** rng.integers(-14, 0, (n_pages, H))).astype(np.float32) for _ in range(2)]
    _append(sbd, (x, -2 * x), slots, codes, scale, page, getattr(torch, dtype), layout)
    assert sbd.sbd_device_error() == 0


def test_append_special_values(sbd):
    import torch
    rng = np.random.default_rng(1)
    x = rng.normal(size=(40, 2, 64)).astype(np.float32)
    x[0, 0, :5] = [np.inf, -np.inf, np.nan, -0.0, 1e-30]
    x[1] = 0                                                    # a page of zeros alone
    x[2, 0], x[2, 1] = np.nan, np.inf                           # nothing finite
    x[3] = 3e38
    x[4] = 1e-39
    x[5:, 1] = 448.0 * 2.0 ** -3
    x[20, 1, 3] = np.nextafter(np.float32(448.0 * 2.0 ** -3), np.float32(1e9))
    slots = np.concatenate([[0, 16, 32, 48, 64], np.arange(5, 40) + 75]).astype(np.int64)
    slots[37:] = -1                                             # not stored
    codes = [np.zeros((8, 2, 16, 64), np.uint8) for _ in range(2)]
    scale = [np.full((8, 2), np.nan, np.float32) for _ in range(2)]
    _append(sbd, (x, x), slots, codes, scale, 16, torch.float32, "plain")
    assert sbd.sbd_device_error() == 0


def test_append_skips_slots_past_the_cache(sbd):
    import torch
    x = torch.ones(3, 1, 64, device="cuda")
    c, s = [torch.zeros(2, 1, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)], \
        [torch.zeros(2, 1, device="cuda") for _ in range(2)]
    sbd.sbd_cache_append_q8(x, x, _i32([31, 32, 2 ** 31 - 1]), *c, *s)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
    assert c[0].float()[:1].abs().sum().item() == 0


def test_append_in_pieces_is_append_at_once(sbd):
    """A page filled token by token holds what it would have held had its
    final scale been known, wherever codes stay in the normal range."""
    import torch
    rng = np.random.default_rng(7)
    x = torch.from_numpy((rng.uniform(1, 2, (100, 2, 64)) * 2.0 ** (np.arange(100) // 25)[:, None, None]).astype(np.float32)).cuda()
    mk = lambda: ([torch.zeros(3, 2, 128, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)],  # noqa: E731
                  [torch.zeros(3, 2, device="cuda") for _ in range(2)])
    c1, s1 = mk()
    c2, s2 = mk()
    slots = _i32(np.arange(100) + 128)
    sbd.sbd_cache_append_q8(x, x, slots, *c1, *s1)
    for t in range(0, 100, 5):
        sbd.sbd_cache_append_q8(x[t:t + 5], x[t:t + 5], slots[t:t + 5].clone(), *c2, *s2)
    assert torch.equal(s1[0], s2[0]) and torch.equal(c1[0].view(torch.uint8), c2[0].view(torch.uint8))


# ------------------------------------------------------------------ attention

def _attention_case(rng, B, k, Hq, H, D, page, lens, extra_cols=1, spread=2.0, sink=0.0):
    cols = max(1, int(max(-(-np.asarray(lens) // page)))) + extra_cols
    n_pages = int((-(-np.asarray(lens) // page)).sum()) + 2
    table, spare = _table(rng, lens, page, n_pages, cols)
    channel = np.exp(0.5 * rng.normal(size=(H, 1, D)))
    codes, scale = [], []
    for w in range(2):
        x = rng.normal(size=(n_pages, H, page, D)) * (channel if w == 0 else np.exp(rng.normal(size=(n_pages, H, 1, 1))))
        s = np.array([[po.scale_for(np.abs(x[p, h]).max()) for h in range(H)] for p in range(n_pages)])
        codes.append(po.e4m3_encode(x / s[..., None, None]))
        scale.append(s.astype(np.float32))
    q = spread * rng.normal(size=(B, k, Hq, D)) / np.repeat(channel[:, 0], Hq // H, 0)
    if sink:                                    # the first token draws nearly everything, and says little
        c = rng.choice([-1.0, 1.0], (H, D))
        q += 1.5 * spread * np.repeat(c / channel[:, 0], Hq // H, 0)
        for b in range(B):
            if lens[b]:
                first = table[b, 0]
                codes[0][first, :, 0] = po.e4m3_encode(sink * c * channel[:, 0] / scale[0][first][:, None])
                codes[1][first, :, 0] = 0
    # what no request holds is poisoned
    for b in range(B):
        if lens[b] % page:
            for w in range(2):
                codes[w][table[b, lens[b] // page], :, lens[b] % page:] = 0x7F
    for p in spare:
        for w in range(2):
            codes[w][p] = 0xFF
            scale[w][p] = np.nan
    kb, vb = rng.normal(size=(B, k, H, D)) * channel[:, 0], rng.normal(size=(B, k, H, D))
    return q, codes, scale, table, np.asarray(lens, np.int32), kb, vb


def _attend(sbd, case, dtype="bfloat16", n_causal=0, scale=0.0, num_splits=0, check=True):
    import torch
    q, codes, scales, table, lens, kb, vb = case
    dt = getattr(torch, dtype)
    dev = [torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda() for x in (q, kb, vb)]
    f = [x.float().cpu().numpy().astype(np.float64) for x in dev]
    out = sbd.sbd_block_attention_q8(dev[0], _f8(codes[0]), _f8(codes[1]), torch.from_numpy(scales[0]).cuda(),
                                     torch.from_numpy(scales[1]).cuda(), _i32(table), _i32(lens), dev[1], dev[2],
                                     n_causal=n_causal, scale=scale, num_splits=num_splits)
    got = out.float().cpu().numpy().astype(np.float64)
    if not check:
        return got
    ref, spread, wobble = po.block_attention(f[0], codes[0], codes[1], scales[0], scales[1], table, lens, f[1], f[2],
                                             n_causal=n_causal, scale=scale or None)
    n, D = int(lens.max()) + q.shape[1], q.shape[3]
    if dtype == "bfloat16":
        tol = spread * (2.0 ** -8 + 2.0 ** -16 * wobble[..., None]) + 2.0 ** -9 * np.abs(ref) + 1e-30
    else:
        tol = spread * ((n + D) * 2.0 ** -24 + 2 * D * 2.0 ** -24 * wobble[..., None]) + 2.0 ** -24 * np.abs(ref) + 1e-30
    assert np.isfinite(got).all()
    worst = float((np.abs(got - ref) / tol).max())
    assert worst <= 1.0, worst
    assert sbd.sbd_device_error() == 0
    return got


SHAPES = [  # k, Hq, Hkv, D, page
    (1, 4, 1, 128, 64), (1, 8, 8, 64, 16), (3, 6, 2, 128, 16), (4, 4, 2, 64, 32), (8, 8, 2, 128, 128), (16, 8, 2, 128, 64),
    (16, 4, 2, 64, 128), (32, 4, 1, 128, 32), (32, 6, 2, 64, 64), (5, 10, 2, 128, 64), (32, 8, 1, 128, 16)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("k,Hq,H,D,page", SHAPES)
@pytest.mark.parametrize("lens", [[0], [1, 0, 17], [64, 63, 65, 128], [700, 0, 129, 2049]])
def test_attention(sbd, dtype, k, Hq, H, D, page, lens):
    rng = np.random.default_rng(k * 1000 + D + page + len(lens))
    _attend(sbd, _attention_case(rng, len(lens), k, Hq, H, D, page, lens), dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("k,n_causal", [(1, 1), (8, 4), (7, 7), (32, 16)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_causal_rows(sbd, dtype, k, n_causal, D):
    rng = np.random.default_rng(k + D)
    _attend(sbd, _attention_case(rng, 3, k, 4, 1, D, 32, [0, 100, 513]), dtype, n_causal=n_causal)


def test_attention_causal_rows_do_not_see_later_values(sbd):
    """Values a causal row must not see may be infinite."""
    rng = np.random.default_rng(2)
    for dtype in ("bfloat16", "float32"):
        case = _attention_case(rng, 1, 4, 4, 1, 128, 32, [40])
        case[6][:, 3] = np.inf
        got = _attend(sbd, case, dtype, n_causal=3, check=False)
        assert np.isfinite(got[:, :3]).all() and not np.isfinite(got[:, 3]).any()


@pytest.mark.parametrize("num_splits", [1, 2, 5, 16])
@pytest.mark.parametrize("dtype,D,k", [("bfloat16", 128, 16), ("bfloat16", 64, 4), ("float32", 128, 4), ("bfloat16", 128, 32)])
def test_attention_splits(sbd, num_splits, dtype, D, k):
    rng = np.random.default_rng(num_splits)
    _attend(sbd, _attention_case(rng, 2, k, 8, 2, D, 64, [1500, 31]), dtype, num_splits=num_splits)


@pytest.mark.parametrize("B,k,Hq,H,D,page,hi", [
    (200, 1, 2, 1, 128, 16, 700), (97, 3, 4, 2, 64, 32, 300), (45, 8, 16, 4, 128, 64, 900), (513, 2, 1, 1, 64, 16, 90),
    (170, 1, 1, 1, 128, 128, 0), (30, 16, 16, 8, 64, 128, 400), (21, 32, 8, 2, 128, 64, 3000), (160, 5, 1, 1, 128, 64, 260)])
def test_attention_of_more_jobs_than_sms(sbd, B, k, Hq, H, D, page, hi):
    """Sequences of all lengths, empty ones among them, whose tiles the CTAs share out."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, hi + 1, B) * (rng.random(B) < 0.9)
    _attend(sbd, _attention_case(rng, B, k, Hq, H, D, page, lens), n_causal=k // 2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k,Hq,H,n_causal", [(9, 8, 2, 0), (16, 8, 1, 8), (16, 12, 2, 16), (32, 4, 1, 16), (25, 16, 2, 3), (32, 12, 1, 1)])
def test_attention_of_many_rows(sbd, k, Hq, H, n_causal, D):
    """33 to 384 packed rows of a KV head: rows on the lanes, 128 a CTA."""
    rng = np.random.default_rng(k + Hq + D)
    for page, lens, splits in ((16, [0, 5, 1000], 0), (128, [129, 2300], 1), (64, [640, 31, 0], 3)):
        _attend(sbd, _attention_case(rng, len(lens), k, Hq, H, D, page, lens), n_causal=n_causal, num_splits=splits)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_many_rows_extremes(sbd, D):
    rng = np.random.default_rng(D)
    for spread, scale in ((30.0, 0.0), (0.01, 0.0), (2.0, 1e-6)):
        _attend(sbd, _attention_case(rng, 2, 32, 4, 1, D, 64, [900, 333], spread=spread), scale=scale)
    got = _attend(sbd, _attention_case(rng, 1, 32, 4, 1, D, 64, [6000], spread=1.0, sink=0.85))
    assert np.abs(got).max() > 0
    # block values that a causal row does not see, rows of NaN, and a NaN in the cache
    case = _attention_case(rng, 2, 32, 4, 1, D, 32, [40, 300])
    case[6][0, 20] = np.inf
    case[0][1, 3] = np.nan
    got = _attend(sbd, case, n_causal=32, check=False)
    assert np.isfinite(got[0, :20]).all() and not np.isfinite(got[0, 20:]).any()
    assert np.isnan(got[1, 3]).all() and np.isfinite(np.delete(got[1], 3, 0)).all()
    case = _attention_case(rng, 2, 32, 4, 1, D, 32, [40, 300])
    case[1][1][case[3][0, 0], :, 7] = 0x7F
    got = _attend(sbd, case, check=False)
    assert np.isnan(got[0]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("k,D", [(4, 64), (8, 128), (16, 128), (32, 64)])
def test_attention_of_partial_tiles_after_nan_everywhere(sbd, k, D):
    """A call before this one has left NaN all over shared memory: nothing of a
    tile's places without a page may reach the result."""
    import torch
    rng = np.random.default_rng(k)
    nan = [np.full((160, 8, 4, 128), np.nan), [np.full((322, 2, 16, 128), 0x7F, np.uint8)] * 2, [np.full((322, 2), np.nan, np.float32)] * 2,
           np.arange(320, dtype=np.int32).reshape(160, 2), np.full(160, 32, np.int32), *[np.full((160, 8, 2, 128), np.nan)] * 2]
    case = _attention_case(rng, 160, k, 4, 2, D, 16, rng.integers(1, 120, 160))
    _attend(sbd, case)
    for _ in range(3):
        _attend(sbd, nan, "float32", check=False)
        torch.cuda.synchronize()
        _attend(sbd, case)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_peaked_flat_and_scaled(sbd, dtype):
    rng = np.random.default_rng(9)
    for spread, scale in ((30.0, 0.0), (0.01, 0.0), (1.0, 0.3), (2.0, 1e-6)):
        _attend(sbd, _attention_case(rng, 2, 8, 8, 2, 128, 64, [900, 333], spread=spread), dtype, scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_many_weak_keys_beside_a_strong_one(sbd, D):
    """One key takes almost all the weight and its value is zero: what is left is
    the sum of thousands of small probabilities."""
    rng = np.random.default_rng(4)
    case = _attention_case(rng, 1, 4, 4, 1, D, 64, [6000], spread=1.0, sink=0.85)
    got = _attend(sbd, case)
    assert np.abs(got).max() > 0


def test_attention_refuses_pages_out_of_range(sbd):
    rng = np.random.default_rng(6)
    for dtype in ("bfloat16", "float32"):
        case = _attention_case(rng, 1, 2, 2, 1, 128, 64, [128])
        case[3][0, 1] = 10 ** 6
        got = _attend(sbd, case, dtype, check=False)
        assert np.isfinite(got).all() and sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
        case[3][0, 1] = -1
        _attend(sbd, case, dtype, check=False)
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE


def test_attention_clamps_lengths(sbd):
    rng = np.random.default_rng(8)
    case = list(_attention_case(rng, 2, 2, 2, 1, 64, 16, [64, 5], extra_cols=0))
    full = _attend(sbd, case, "float32")
    case[4] = np.array([1000, -4], np.int32)
    got = _attend(sbd, case, "float32", check=False)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_CACHE_LEN
    assert np.allclose(got[0], full[0], rtol=1e-5, atol=1e-6)


def test_attention_of_a_large_cache(sbd):
    """Offsets past 32 bits: the pages of one request lie at the end of a cache of
    more than 4 GB."""
    import torch
    D, H, P = 128, 8, 128
    n_pages = (1 << 32) // (D * H * P) + 40
    rng = np.random.default_rng(3)
    case = _attention_case(rng, 1, 4, 4, 1, D, P, [700])
    q, codes, scales, table, lens, kb, vb = case
    kc, vc = (torch.zeros(n_pages, H, P, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(n_pages, H, device="cuda") for _ in range(2))
    base = n_pages - codes[0].shape[0]
    for dst, src in ((kc, codes[0]), (vc, codes[1])):
        dst[base:, H - 1] = torch.from_numpy(src[:, 0]).cuda()
    for dst, src in ((ks, scales[0]), (vs, scales[1])):
        dst[base:, H - 1] = torch.from_numpy(src[:, 0]).cuda()
    f8 = torch.float8_e4m3fn
    for dt in (torch.bfloat16, torch.float32):
        dev = [torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda() for x in (q, kb, vb)]
        wide = [torch.zeros(1, 4, H * x.shape[2], D, dtype=dt, device="cuda") for x in dev]
        for w, x in zip(wide, dev):
            w[:, :, -x.shape[2]:] = x
        tab = np.where(table >= 0, table + base, -1)
        out = sbd.sbd_block_attention_q8(wide[0], kc.view(f8), vc.view(f8), ks, vs, _i32(tab), _i32(lens), wide[1], wide[2])
        small = sbd.sbd_block_attention_q8(dev[0], _f8(codes[0]), _f8(codes[1]), torch.from_numpy(scales[0]).cuda(),
                                           torch.from_numpy(scales[1]).cuda(), _i32(table), _i32(lens), dev[1], dev[2])
        tol = 2e-2 if dt == torch.bfloat16 else 1e-5
        assert (out[:, :, -4:].float() - small.float()).abs().max().item() <= tol * small.abs().max().item()
    # the append reaches there, too
    x = torch.randn(3, H, D, device="cuda")
    slots = _i32((n_pages - 1) * P + np.arange(3))
    sbd.sbd_cache_append_q8(x, x, slots, kc.view(f8), vc.view(f8), ks, vs)
    got = kc.view(f8)[-1, :, :3].float() * ks[-1][:, None, None]
    assert (got.transpose(0, 1) - x).abs().max().item() <= 2.0 ** -4 * x.abs().max().item()
    assert sbd.sbd_device_error() == 0


def test_on_another_stream(sbd):
    import torch
    rng = np.random.default_rng(12)
    case = _attention_case(rng, 2, 4, 4, 2, 128, 64, [300, 40])
    ref = _attend(sbd, case)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = _attend(sbd, case, check=False)
    st.synchronize()
    assert (got == ref).all()


@pytest.mark.parametrize("B,k,D", [(1, 32, 64), (1, 16, 128), (40, 8, 64), (40, 2, 128), (160, 2, 64)])
def test_attention_refusals_in_every_kernel(sbd, B, k, D):
    """Pages out of range count as zeros, lengths out of range are clamped, in
    splits, in more CTAs than a wave, with rows and with keys on the lanes."""
    rng = np.random.default_rng(B + k)
    case = list(_attention_case(rng, B, k, 16, 4, D, 32, [300] * B, extra_cols=0))
    full = _attend(sbd, tuple(case), check=True)
    bad = [x.copy() if isinstance(x, np.ndarray) else x for x in case]
    bad[3][0, 2] = 10 ** 6
    bad[3][B - 1, 5] = -7
    got = _attend(sbd, tuple(bad), check=False)
    assert np.isfinite(got).all() and sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
    assert (got[1:B - 1] == full[1:B - 1]).all()
    ref = [x.copy() if isinstance(x, np.ndarray) else x for x in case]
    ref[1] = [c.copy() for c in case[1]]
    for w in range(2):                               # those pages as zeros
        ref[1][w][case[3][0, 2]] = 0
        ref[1][w][case[3][B - 1, 5]] = 0
    assert np.abs(got - _attend(sbd, tuple(ref))).max() <= 2e-2
    long = list(case)
    long[4] = np.array([10 ** 6] + [300] * (B - 2) + [-3] * (B > 1), np.int32)
    got = _attend(sbd, tuple(long), check=False)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_CACHE_LEN
    assert (got[1:B - 1] == full[1:B - 1]).all()


def test_a_turn_in_a_cuda_graph(sbd):
    """Tables, append and attention of a step, captured and replayed."""
    import torch
    rng = np.random.default_rng(21)
    B, H, D, P, n_pages = 5, 2, 128, 64, 40
    lens, grow = np.array([0, 63, 64, 200, 5], np.int32), np.array([1, 16, 7, 16, 0], np.int32)
    table, spare = _table(rng, lens, P, n_pages, 8)
    free = np.zeros(n_pages, np.int32)
    free[:len(spare)] = spare
    state = dict(len=_i32(lens), target=_i32(lens + grow), table=_i32(table), free=_i32(free), n_free=_i32([len(spare)]))
    codes = [torch.zeros(n_pages, H, P, D, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.ones(n_pages, H, device="cuda") for _ in range(2)]
    new = torch.randn(int(grow.sum()), 2 * H, D, device="cuda").bfloat16()
    outs = sbd.block_tables_outputs(state["len"], state["table"], int(grow.sum()))
    blocks = [[torch.randn(B, k, h, D, device="cuda").bfloat16() for h in (4 * H, H, H)] for k in (1, 8, 32)]
    results = [torch.empty_like(q) for q, _, _ in blocks]

    def turn():
        sbd.sbd_block_tables(*state.values(), P, outputs=outs)
        sbd.sbd_cache_append_q8(new[:, :H], new[:, H:], outs[3], *codes, *scales)
        for (q, kb, vb), out in zip(blocks, results):
            sbd.sbd_block_attention_q8(q, *codes, *scales, outs[0], outs[1], kb, vb, out)

    turn()
    torch.cuda.synchronize()
    want = [x.clone() for x in results] + [c.view(torch.uint8).clone() for c in codes]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for x in results + [c.view(torch.uint8) for c in codes]:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(results + [c.view(torch.uint8) for c in codes], want):
        assert torch.equal(got, ref)
    assert sbd.sbd_device_error() == 0
