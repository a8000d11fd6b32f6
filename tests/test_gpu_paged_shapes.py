"""Configurations of the paged 8-bit cache's kernels beyond the small ones: prompts
(long chunks of tokens, two planes a CTA), long segments behind short ones, two CTAs
an SM with splits, fp32 attention in several waves, values and scales that are not
ordinary; and the same call again and again, which answers the same bits."""
import numpy as np
import pytest

import test_gpu_paged as tp
from oracle import paged_oracle as po
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ append

def _segments(slots, page):
    """(first token, tokens) of every segment."""
    cut = np.flatnonzero((np.diff(slots) != 1) | (slots[1:] % page == 0)) + 1
    begin, end = np.concatenate([[0], cut]), np.concatenate([cut, [len(slots)]])
    return [(a, b - a) for a, b in zip(begin, end)]


def _reference(x, slots, codes, scale, page):
    """po.cache_append for many tokens (all stored, scales powers of two): codes of all at once."""
    codes, scale = codes.copy(), scale.astype(np.float64)
    x = x.astype(np.float64)
    per_token = np.empty(x.shape[:2])
    for t, n in _segments(slots, page):
        pg, off = slots[t] // page, slots[t] % page
        amax = np.abs(x[t:t + n]).max((0, 2))
        new = 2.0 ** np.maximum(np.ceil(np.log2(np.maximum(amax, 1e-300) / 448.0)), -126.0)
        assert (amax <= 448.0 * new).all() and (amax > 224.0 * new).all()
        if off:
            new = np.maximum(new, scale[pg])
            codes[pg, :, :off] = po.e4m3_encode(po.E4M3[codes[pg, :, :off]] * (scale[pg] / new)[:, None, None])
        scale[pg] = new
        per_token[t:t + n] = new
    codes[slots // page, :, slots % page] = po.e4m3_encode(x / per_token[:, :, None])
    return codes, scale.astype(np.float32)


@pytest.mark.parametrize("dtype,H,D,page,lens,new", [
    ("bfloat16", 8, 128, 64, [3, 0, 130], [900, 1700, 1]),          # long chunks
    ("bfloat16", 8, 64, 16, [5, 64], [2500, 333]),
    ("bfloat16", 8, 64, 128, [5, 64, 1], [1500, 1000, 700]),
    ("bfloat16", 3, 128, 16, [1, 17], [7000, 300]),
    ("float32", 8, 128, 128, [100, 0], [2000, 900]),
    ("float32", 8, 64, 32, [31], [2777]),
    ("bfloat16", 8, 128, 128, [37, 0], [12000, 8500]),              # and two planes a CTA
    ("float32", 8, 64, 64, [1], [20011]),
    ("bfloat16", 7, 64, 32, [11, 3], [16000, 7007])])
def test_append_of_prompts(sbd, dtype, H, D, page, lens, new):  # noqa: F811
    import torch
    rng = np.random.default_rng(H * D + page)
    dt = getattr(torch, dtype)
    slots = tp._slots(rng, np.asarray(lens), np.asarray(new), page, int(sum(-(-(a + b) // page) for a, b in zip(lens, new))) + 2)
    n_pages, T = int(slots.max()) // page + 1, len(slots)
    gen = torch.Generator(device="cuda").manual_seed(T)
    fused = torch.randn(T, 2 * H + 1, D, generator=gen, device="cuda")
    fused *= torch.exp2(torch.randint(-6, 7, (T, 1, 1), generator=gen, device="cuda").float())
    fused = fused.to(dt)
    new_kv = [fused[:, 1:1 + H], fused[:, 1 + H:]]
    codes = [rng.integers(0, 256, (n_pages, H, page, D)).astype(np.uint8) for _ in range(2)]
    codes = [np.where((c & 127) == 127, c - 1, c) for c in codes]   # (no NaN)
    scale = [(2.0 ** rng.integers(-14, 0, (n_pages, H))).astype(np.float32) for _ in range(2)]
    caches, scales = [tp._f8(c) for c in codes], [torch.from_numpy(s.copy()).cuda() for s in scale]
    sbd.sbd_cache_append_q8(*new_kv, tp._i32(slots), *caches, *scales)
    for w in range(2):
        rc, rs = _reference(new_kv[w].float().cpu().numpy(), slots, codes[w], scale[w], page)
        assert np.array_equal(scales[w].cpu().numpy(), rs)
        got = tp._bytes(caches[w])
        assert (po.E4M3[got] == po.E4M3[rc]).all()
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("D,layout", [(64, "plain"), (128, "fused"), (128, "blocks")])
def test_append_of_a_long_segment_behind_short_ones(sbd, dtype, D, layout):  # noqa: F811
    """Eight single tokens and then a page of 128: a warp has more of it than it keeps in
    registers, with and without an infinity that makes it read the segment again."""
    import torch
    rng = np.random.default_rng(D)
    page, H = 128, 2
    for special in (False, True):
        n = 120 if layout == "blocks" else 127
        off = 128 - n
        slots = np.concatenate([np.arange(8) * page + 5, 9 * page + off + np.arange(n), 10 * page + np.arange(2)]).astype(np.int64)
        T = len(slots)
        x = rng.normal(size=(T, H, D)) * 2.0 ** rng.integers(-6, 6, (T, 1, 1))
        if special:
            x[60, 0, 3], x[61, 1, 7], x[62, 1, 8], x[70], x[T - 1] = np.inf, -np.inf, np.nan, 0.0, -0.0
        codes = [rng.integers(0, 127, (12, H, page, D)).astype(np.uint8) for _ in range(2)]
        scale = [(2.0 ** rng.integers(-16, -9, (12, H))).astype(np.float32) for _ in range(2)]
        tp._append(sbd, (x, -2 * x), slots, codes, scale, page, getattr(torch, dtype), layout)
    assert sbd.sbd_device_error() == 0


def test_append_special_values_bf16(sbd):  # noqa: F811
    import torch
    rng = np.random.default_rng(1)
    x = rng.normal(size=(200, 2, 128)).astype(np.float32)
    x[0, 0, :5] = [np.inf, -np.inf, np.nan, -0.0, 1e-30]
    x[1] = 0
    x[2, 0], x[2, 1] = np.nan, np.inf
    x[3] = 3e38
    x[4] = 1e-39                                                # below bf16's and fp32's normal range
    x[5:60, 1] = 448.0 * 2.0 ** -3
    x[20, 1, 3] = 450.0 * 2.0 ** -3                             # the next larger bf16 value
    x[60:, 0] *= 1e-38                                          # scales at their smallest
    x[60:, 1] *= 2e37
    x[100, 1, :3] = [-np.inf, np.nan, np.inf]
    slots = np.concatenate([[0, 64, 128, 192, 256], np.arange(5, 60) + 315, np.arange(60, 200) + 448 - 60]).astype(np.int64)
    slots[57:60] = -1
    codes = [np.zeros((10, 2, 64, 128), np.uint8) for _ in range(2)]
    scale = [np.full((10, 2), np.nan, np.float32) for _ in range(2)]
    v = np.float32(0.5) * x                                     # (-2 x may not be finite)
    x, v = (torch.from_numpy(y).bfloat16() for y in (x, v))
    for layout in ("plain", "fused"):
        tp._append(sbd, (x.float().numpy(), v.float().numpy()), slots, codes, scale, 64, torch.bfloat16, layout)
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_append_to_pages_with_a_scale_of_the_callers_own(sbd, dtype):  # noqa: F811
    """Held scales that are no powers of two: kept where they suffice (codes of x / s),
    replaced where they do not (codes of c s_old / s).  Both quotients are rounded to
    fp32 before they become codes, so a quotient within 2^-23 of itself of the middle
    between two codes may go to either."""
    import torch
    rng = np.random.default_rng(3)
    page, H, D, n = 32, 4, 128, 40
    slots = np.concatenate([p * page + 8 + np.arange(rng.integers(1, 25)) for p in range(n)]).astype(np.int64)
    x = torch.from_numpy((rng.normal(size=(len(slots), H, D)) * 2.0 ** rng.integers(-3, 4, (len(slots), H, 1))).astype(np.float32)).to(getattr(torch, dtype))
    codes = np.where(rng.random((n, H, page, D)) < 0.5, 0, 128).astype(np.uint8) + rng.integers(0, 127, (n, H, page, D)).astype(np.uint8)
    scale = np.exp(rng.uniform(-8, 0, (n, H))).astype(np.float32)
    caches, scales = [tp._f8(codes) for _ in range(2)], [torch.from_numpy(scale.copy()).cuda() for _ in range(2)]
    sbd.sbd_cache_append_q8(x.cuda(), x.cuda(), tp._i32(slots), *caches, *scales)
    rc, rs = po.cache_append(x.float().numpy(), slots, codes, scale, page)
    kept = rs == scale
    assert kept.any() and (~kept).any()
    values = np.unique(po.E4M3[np.isfinite(po.E4M3)])
    for c, s in zip(caches, scales):
        assert np.array_equal(s.cpu().numpy(), rs)
        got = po.E4M3[tp._bytes(c)]
        exact = po.E4M3[codes] * np.where(kept, 1.0, scale.astype(np.float64) / rs)[..., None, None]
        exact[slots // page, :, slots % page] = x.double().numpy() / rs.astype(np.float64)[slots // page][:, :, None]
        exact = np.clip(exact, -448, 448)
        i = np.clip(np.searchsorted(values, exact), 1, len(values) - 1)
        middle = (values[i - 1] + values[i]) / 2
        either = np.abs(exact - middle) <= 2.0 ** -23 * np.abs(exact)
        assert ((got == po.E4M3[rc]) | (either & ((got == values[i - 1]) | (got == values[i])))).all()
    assert sbd.sbd_device_error() == 0


def test_append_stores_what_stands_beside_slots_past_the_cache(sbd):  # noqa: F811
    import torch
    for dt in (torch.float32, torch.bfloat16):
        x = torch.tensor([3.0, 5.0, 7.0, 1.5], device="cuda")[:, None, None].expand(4, 2, 64).contiguous().to(dt)
        c, s = [torch.zeros(2, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)], \
            [torch.zeros(2, 2, device="cuda") for _ in range(2)]
        sbd.sbd_cache_append_q8(x, -x, tp._i32([31, 32, 2 ** 31 - 1, 0]), *c, *s)
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
        for w, sign in ((0, 1.0), (1, -1.0)):
            assert s[w].tolist() == [[2.0 ** -8] * 2, [2.0 ** -7] * 2]       # 1.5 = 384 2^-8, 3 = 384 2^-7
            v = c[w].float() * s[w][:, :, None, None]
            assert (v[1, :, 15] == 3 * sign).all() and (v[0, :, 0] == 1.5 * sign).all()
            assert (v[1, :, :15] == 0).all() and (v[0, :, 1:] == 0).all()


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("k,Hq,H,B,lens", [
    (1, 32, 8, 4, [5700, 3, 0, 2049]),                          # one wave, long caches
    (4, 16, 8, 2, [10400, 130]), (2, 8, 8, 3, [7600, 6999, 128])])
def test_attention_in_splits_on_shared_sms(sbd, k, Hq, H, B, lens):  # noqa: F811
    """64 dimensions, up to 16 rows: clusters whose CTAs share an SM with others."""
    rng = np.random.default_rng(B)
    tp._attend(sbd, tp._attention_case(rng, B, k, Hq, H, 64, 64, lens), n_causal=k // 2)


@pytest.mark.parametrize("num_splits", [2, 3, 8, 16])
@pytest.mark.parametrize("k,G,D", [(2, 2, 64), (4, 4, 64), (8, 4, 64), (8, 4, 128), (2, 2, 128)])
def test_attention_in_asked_splits_of_more_ctas_than_sms(sbd, num_splits, k, G, D):  # noqa: F811
    rng = np.random.default_rng(num_splits + k)
    lens = rng.integers(0, 700, 45) * (rng.random(45) < 0.9)
    tp._attend(sbd, tp._attention_case(rng, 45, k, 2 * G, 2, D, 32, lens), num_splits=num_splits, n_causal=1)


@pytest.mark.parametrize("B,k,Hq,H,D,page,hi", [
    (200, 1, 2, 1, 128, 16, 300), (97, 3, 4, 4, 64, 32, 300), (120, 8, 8, 4, 64, 64, 200), (45, 32, 8, 8, 128, 64, 150)])
def test_attention_fp32_in_several_waves(sbd, B, k, Hq, H, D, page, hi):  # noqa: F811
    rng = np.random.default_rng(B)
    lens = rng.integers(0, hi + 1, B) * (rng.random(B) < 0.9)
    tp._attend(sbd, tp._attention_case(rng, B, k, Hq, H, D, page, lens), "float32", n_causal=k // 2)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("k,D", [(1, 128), (4, 64), (8, 128), (16, 64), (32, 128)])
def test_attention_with_scales_of_the_callers_own(sbd, dtype, k, D):  # noqa: F811
    """Page scales that are no powers of two.  With bf16 activations a value scale enters
    as fp16, relative to the largest among the same keys, and multiplies what is rounded
    to fp16: 2^-11 each, 2^-10 of sum p |v| on top of what powers of two cost."""
    import torch
    rng = np.random.default_rng(D + k)
    lens = [700, 0, 129, 2049]
    q, codes, scales, table, lens, kb, vb = tp._attention_case(rng, 4, k, 8, 2, D, 64, lens)
    scales = [(s * rng.uniform(0.3, 1.7, s.shape)).astype(np.float32) for s in scales]
    case = (q, codes, scales, table, lens, kb, vb)
    if dtype == "float32":
        tp._attend(sbd, case, dtype)
        return
    got = tp._attend(sbd, case, dtype, check=False)
    f = [torch.from_numpy(x.astype(np.float32)).bfloat16().double().numpy() for x in (q, kb, vb)]
    ref, spread, wobble = po.block_attention(f[0], *codes, *scales, table, lens, f[1], f[2])
    tol = spread * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -16 * wobble[..., None]) + 2.0 ** -9 * np.abs(ref) + 1e-30
    assert np.isfinite(got).all() and (np.abs(got - ref) <= tol).all()
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype,B,k,Hq,H,D,page,hi,splits", [
    ("bfloat16", 32, 8, 32, 8, 64, 16, 2047, 0), ("bfloat16", 4, 1, 32, 8, 128, 128, 16000, 0),
    ("bfloat16", 1, 16, 32, 8, 128, 64, 4096, 0), ("bfloat16", 16, 32, 32, 8, 128, 64, 2000, 0),
    ("bfloat16", 1, 1, 32, 8, 64, 64, 9000, 0), ("bfloat16", 45, 4, 8, 2, 64, 32, 700, 8),
    ("bfloat16", 70, 8, 32, 8, 128, 32, 500, 0), ("bfloat16", 3, 32, 12, 2, 64, 32, 900, 7),
    ("float32", 1, 4, 8, 2, 128, 32, 3000, 0), ("float32", 60, 8, 8, 4, 64, 32, 300, 0)])
def test_the_same_call_answers_the_same_bits(sbd, dtype, B, k, Hq, H, D, page, hi, splits):  # noqa: F811
    """200 times, calls of another shape and other inputs between them: no result depends
    on what ran before or on the order in which warps and CTAs get along."""
    import torch
    rng = np.random.default_rng(hi)
    calls = []
    for b, n in ((B, hi), (max(1, B // 2), hi // 3 + 1)):
        lens = np.linspace(0, n, b).astype(np.int64) if b > 1 else [n]
        cols = -(-n // page) + 1
        pages = int(sum(-(-int(x) // page) for x in lens)) + 2
        table, _ = tp._table(rng, lens, page, pages, cols)
        gen = torch.Generator(device="cuda").manual_seed(n)
        mk = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        dt = getattr(torch, dtype)
        codes = [(mk(pages, H, page, D) * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.exp2(torch.randint(-9, -5, (pages, H), generator=gen, device="cuda").float()) for _ in range(2)]
        calls.append((mk(b, k, Hq, D).to(dt), *codes, *scales, tp._i32(table), tp._i32(lens), mk(b, k, H, D).to(dt), mk(b, k, H, D).to(dt)))
    run = lambda c: sbd.sbd_block_attention_q8(*c, n_causal=k // 2, num_splits=splits)  # noqa: E731
    first = [run(c) for c in calls]
    assert all(torch.isfinite(x).all() for x in first)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        for c, x in zip(calls, first):
            differ += (run(c) != x).sum()
    assert differ.item() == 0 and sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("k,Hq,D,num_splits", [(1, 2, 128, 0), (4, 8, 64, 0), (8, 8, 128, 3), (8, 8, 64, 1), (16, 12, 128, 0), (32, 8, 64, 2)])
def test_attention_keeps_nan_where_it_belongs(sbd, dtype, k, Hq, D, num_splits):  # noqa: F811
    """NaN and infinities in a row of q, a cached key, a cached value, a block key and a
    block value: whoever does not see them answers the same bits as without them."""
    rng = np.random.default_rng(k)
    case = tp._attention_case(rng, 3, k, Hq, 2, D, 32, [300, 40, 129])
    copy = lambda: [x.copy() if isinstance(x, np.ndarray) else [y.copy() for y in x] for x in case]  # noqa: E731
    run = lambda c: tp._attend(sbd, tuple(c), dtype, n_causal=k - 1, num_splits=num_splits, check=False)  # noqa: E731
    want = run(case)
    assert np.isfinite(want).all()
    g = Hq // 2

    def others(got, b, i, heads):                   # all but rows i (a slice) of these heads of request b
        seen = np.ones(got.shape[:3], bool)
        seen[b, i, heads] = False
        return (got[seen] == want[seen]).all()

    for bad in (np.nan, np.inf):
        c = copy()
        c[0][1, k // 2, g, 5] = bad                 # q: one row
        got = run(c)
        assert np.isnan(got[1, k // 2, g]).all() and others(got, 1, k // 2, g)
    every, second = slice(None), slice(g, None)     # the second KV head's
    c = copy()
    c[1][0][case[3][0, 3], 1, 17, 3] = 0x7F         # a cached key: every row of its request and head
    got = run(c)
    assert np.isnan(got[0, :, second]).all() and others(got, 0, every, second)
    c = copy()
    c[1][1][case[3][0, 9], 1, 11, 3] = 0xFF         # a cached value (the last token): one dimension
    got = run(c)
    assert np.isnan(got[0, :, second, 3]).all() and others(got, 0, every, second)
    rest = np.arange(D) != 3
    assert (got[0, :, second][..., rest] == want[0, :, second][..., rest]).all()
    for bad in (np.nan, np.inf):
        last = slice(k - 1, None)
        c = copy()
        c[5][2, k - 1, 1, 4] = bad                  # the last block key: only the last row sees it
        got = run(c)
        assert others(got, 2, last, second) and (bad == np.inf or np.isnan(got[2, k - 1, second]).all())
        c = copy()
        c[6][2, k - 1, 1, 4] = bad                  # its value
        got = run(c)
        assert others(got, 2, last, second) and not np.isfinite(got[2, k - 1, second, 4]).any()
    # slots past the length
    c = copy()
    c[1][0][case[3][2, 4], :, 1:] = 0x7F
    c[1][1][case[3][2, 4], :, 1:] = 0xFF
    assert (run(c) == want).all() and sbd.sbd_device_error() == 0
