"""Drafted decoding on the GPU against its 64-bit forms.

Norms and rotation, per element: the output's rounding (half a step, eps / 2 of it), and
40 * 2^-24 of the pair's |y1| + |y2| for what is done in fp32: the sum of D squares (a lane's
16 in turn, then a tree: 20 roundings, halved by the root), the root (2 units), the factors
(3), cosine and sine (4 units of 1, and 4 more of an angle that is exact to 2^-31 of a turn
before it is a float: pi 2^-24 for half a turn) and the products (3).
Attention: the bounds of test_gpu_paged.py.
Verification: whole numbers, equal wherever no decision is within 10^-3 of its border (what
is compared are fp32 sums and exponentials, exact to 2^-17; a remainder p - q loses what p and
q have in common); ln p to 2^-16 + 2^-21 |ln p| (a sum of exponentials, each to 2^-18 with
exponents up to 64, in a tree; the difference of two numbers of the size of ln p).
Append: equal, scales and codes.
"""
import numpy as np
import pytest

import test_gpu_paged as tp
from oracle import draft_oracle as do
from oracle import paged_oracle as po
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu

BORDER = 1e-3


def _f32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()


# ------------------------------------------------------------------ norms and rotation

def _rope(sbd, T, Hq, H, D, R, dtype, norm, interleaved, positions, layout="fused", theta=1e4, scale=1.0, values=True):  # noqa: F811
    import torch
    dt = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(T + Hq * D + R)
    w = (scale * torch.randn(T, Hq + 2 * H, D, generator=gen)).to(dt)
    weights = [(1 + 0.3 * torch.randn(D, generator=gen)).to(dt) if norm else None for _ in range(2)]
    inv = (theta ** (-torch.arange(R // 2, dtype=torch.float64) / (R // 2))).float() if R else None
    pos = torch.from_numpy(np.asarray(positions, np.int32)) if R else None
    x = w.cuda()
    if layout == "blocks":                       # the last 3 rows of blocks of 5
        wide = torch.randn(T // 3, 5, Hq + 2 * H, D).to(dt).cuda()
        wide[:, 2:] = x.view(T // 3, 3, Hq + 2 * H, D)
        x = wide[:, 2:]
    parts = [x[..., :Hq, :], x[..., Hq:Hq + H, :], x[..., Hq + H:, :]]
    if layout == "plain":
        parts = [p.contiguous() for p in parts]
    cuda = [None if t is None else t.cuda() for t in (pos, inv, *weights)]
    out = sbd.sbd_qk_norm_rope(parts[0], parts[1], parts[2] if values else None, *cuda, eps=1e-5, interleaved=interleaved)
    half = torch.finfo(dt).eps / 2
    for i, (got, rows) in enumerate(zip(out, (w[:, :Hq], w[:, Hq:Hq + H]))):
        assert got.is_contiguous() and got.shape == parts[i].shape
        args = None if weights[i] is None else weights[i].double().numpy()
        ref = do.norm_rope(rows.double().numpy(), None if pos is None else pos.numpy(), None if inv is None else inv.numpy(),
                           args, 1e-5, interleaved)
        y = do.norm_rope(rows.double().numpy(), None, None, args, 1e-5, interleaved)
        size = np.abs(y)
        r = R // 2
        if interleaved:
            size[..., 0:R:2] = size[..., 1:R:2] = size[..., 0:R:2] + size[..., 1:R:2]
        else:
            size[..., :r] = size[..., r:R] = size[..., :r] + size[..., r:R]
        got = got.double().cpu().numpy().reshape(ref.shape)
        worst = (np.abs(got - ref) / (half * np.abs(ref) + 40 * 2.0 ** -24 * size + 1e-35)).max() if T else 0.0
        assert worst <= 1.0, (i, worst)
    assert out[2] is None if not values else torch.equal(out[2], parts[2])
    assert sbd.sbd_device_error() == 0
    return out


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,Hq,H,D,R,norm,interleaved,layout", [
    (1, 32, 8, 128, 128, True, False, "fused"), (1, 1, 1, 64, 64, True, True, "plain"), (16, 32, 8, 128, 128, False, False, "fused"),
    (9, 6, 2, 64, 32, True, True, "blocks"), (33, 5, 5, 128, 16, True, False, "plain"), (3, 8, 2, 64, 0, True, False, "fused"),
    (12, 40, 8, 128, 64, True, False, "blocks"), (301, 3, 1, 128, 96, False, True, "fused"), (700, 8, 4, 64, 48, True, False, "fused"),
    (0, 4, 2, 128, 128, True, False, "plain"), (5, 7, 1, 64, 64, False, False, "plain")])
def test_norm_rope(sbd, dtype, T, Hq, H, D, R, norm, interleaved, layout):  # noqa: F811
    rng = np.random.default_rng(T)
    _rope(sbd, T, Hq, H, D, R, dtype, norm, interleaved, rng.integers(0, 5000, T), layout, values=T != 33)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,Hq,H,D,R,norm,interleaved,layout", [
    (9000, 3, 2, 64, 64, True, False, "fused"), (9001, 2, 1, 128, 32, True, True, "plain"), (9999, 1, 1, 64, 48, False, False, "blocks"),
    (8100, 9, 5, 128, 128, True, False, "fused"), (7500, 19, 1, 64, 0, True, False, "fused"), (24001, 1, 1, 128, 128, False, True, "plain")])
def test_norm_rope_of_prompts(sbd, dtype, T, Hq, H, D, R, norm, interleaved, layout):  # noqa: F811
    """Tokens enough for the kernel that streams them through shared memory: the same bits as
    of a few tokens at a time."""
    import torch
    dt = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, Hq + 2 * H, D, generator=gen, device="cuda").to(dt)
    if layout == "blocks":                       # the last 3 rows of blocks of 5
        wide = torch.randn(T // 3, 5, Hq + 2 * H, D, generator=gen, device="cuda").to(dt)
        wide[:, 2:] = x.view(T // 3, 3, Hq + 2 * H, D)
        x = wide[:, 2:]
    parts = [x[..., :Hq, :], x[..., Hq:Hq + H, :], x[..., Hq + H:, :]]
    if layout == "plain":
        parts = [p.contiguous() for p in parts]
    w = (1 + 0.3 * torch.randn(2, D, generator=gen, device="cuda")).to(dt) if norm else (None, None)
    inv = torch.rand(R // 2, generator=gen, device="cuda") if R else None
    pos = torch.randint(0, 100000, (T,), generator=gen, device="cuda", dtype=torch.int32)
    for values in (True, False):
        outs = [torch.full((T + 2, h, D), 7, dtype=dt, device="cuda") for h in (Hq, H, H)]
        got = [o[1:-1] for o in outs]
        shaped = [o.view(p.shape) for o, p in zip(got, parts)]
        sbd.sbd_qk_norm_rope(*parts[:2], parts[2] if values else None, pos, inv, *w, *shaped[:2], shaped[2] if values else None,
                             eps=1e-5, interleaved=interleaved)
        flat = [p.reshape(T, -1, D) for p in parts]
        for i in range(0, T, 1000):
            few = sbd.sbd_qk_norm_rope(*(f[i:i + 1000].contiguous() for f in flat), pos[i:i + 1000].clone(), inv, *w, eps=1e-5,
                                       interleaved=interleaved)
            for j in range(3 if values else 2):
                assert torch.equal(got[j][i:i + 1000], few[j]), (i, j)
        for o in outs:
            assert (o[0] == 7).all() and (o[-1] == 7).all()
        assert values or (outs[2] == 7).all()
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_far_positions(sbd, interleaved):  # noqa: F811
    far = [0, 1, -1, 2 ** 20, 10 ** 7 + 1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 999999937]
    for theta in (1e4, 5e5):
        _rope(sbd, len(far), 4, 2, 128, 128, "float32", False, interleaved, far, theta=theta)
    # frequencies that are not below 1: whole turns a position fall away
    import torch
    x = torch.randn(4, 1, 64, device="cuda")
    inv = torch.tensor([1e6, -3.5, 100.25, 6.2831855, 0.0, -1e-12, 7.0, 1e-30], device="cuda")
    pos = torch.tensor([3, -7, 12345, 0], dtype=torch.int32, device="cuda")
    q, _, _ = sbd.sbd_qk_norm_rope(x, x, None, pos, inv, interleaved=interleaved)
    ref = do.norm_rope(x.double().cpu().numpy(), pos.tolist(), inv.double().tolist(), None, 0, interleaved)
    assert np.abs(q.double().cpu().numpy() - ref).max() <= 1e-5


def test_norm_rope_extremes(sbd):  # noqa: F811
    """Rows of zeros, tiny and large rows, a NaN that stays in its row."""
    import torch
    for dt in ("bfloat16", "float32"):
        _rope(sbd, 7, 4, 2, 128, 128, dt, True, False, range(7), scale=1e-18)
        _rope(sbd, 7, 4, 2, 128, 128, dt, True, False, range(7), scale=1e15)
        x = torch.randn(4, 6, 64).to(getattr(torch, dt)).cuda()
        x[1, 2] = 0
        x[2, 3, 5] = float("nan")
        w = torch.ones(64, dtype=x.dtype, device="cuda")
        inv = torch.ones(32, device="cuda")
        pos = torch.arange(4, dtype=torch.int32, device="cuda")
        q, k, v = sbd.sbd_qk_norm_rope(x[:, :4], x[:, 4:5], x[:, 5:], pos, inv, w, w, eps=1e-6)
        assert (q[1, 2] == 0).all() and torch.isnan(q[2, 3]).all()
        q[2, 3] = 0
        assert torch.isfinite(q).all() and torch.isfinite(k).all() and torch.equal(v, x[:, 5:])


def test_norm_rope_leaves_its_surroundings(sbd):  # noqa: F811
    import torch
    x = torch.randn(5, 7, 64, device="cuda")
    outs = [torch.full((9, h, 64), 7.0, device="cuda") for h in (4, 1, 2)]
    pos, inv = torch.arange(5, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    sbd.sbd_qk_norm_rope(x[:, :4], x[:, 4:5], None, pos, inv, None, None, outs[0][2:7], outs[1][2:7], eps=0.0)
    for o in outs[:2]:
        assert (o[:2] == 7).all() and (o[7:] == 7).all() and (o[2:7] != 7).any()
    assert (outs[2] == 7).all()


def test_norm_rope_of_many_tokens(sbd):  # noqa: F811
    """Offsets past 2^31 elements."""
    import torch
    T, Hq, H, D = 360000, 32, 8, 128
    x = torch.zeros(T, Hq + 2 * H, D, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(3, Hq + 2 * H, D).bfloat16().cuda()
    x[-3:] = tail
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    inv = (1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    big = sbd.sbd_qk_norm_rope(x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], pos, inv, w, w)
    small = sbd.sbd_qk_norm_rope(tail[:, :Hq], tail[:, Hq:Hq + H], tail[:, Hq + H:], pos[-3:].clone(), inv, w, w)
    for a, b in zip(big, small):
        assert torch.equal(a[-3:], b)
        assert not a[:-3].any()


# ------------------------------------------------------------------ tree attention

def _trees(rng, B, n, kind="random"):
    parent = np.full((B, n), -1, np.int32)
    for b in range(B):
        for i in range(1, n):
            parent[b, i] = {"random": rng.integers(max(-1, i - 9), i), "chain": i - 1, "binary": (i - 1) // 2,
                            "star": 0, "none": -1, "deep": max(0, i - int(rng.integers(1, 3)))}[kind]
    return parent


def _attend(sbd, case, parent, dtype="bfloat16", scale=0.0, num_splits=0, check=True):  # noqa: F811
    import torch
    q, codes, scales, table, lens, kb, vb = case
    dt = getattr(torch, dtype)
    dev = [torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda() for x in (q, kb, vb)]
    out = sbd.sbd_tree_attention_q8(dev[0], tp._f8(codes[0]), tp._f8(codes[1]), _f32(scales[0]), _f32(scales[1]),
                                    tp._i32(table), tp._i32(lens), dev[1], dev[2], tp._i32(parent), scale=scale,
                                    num_splits=num_splits)
    got = out.double().cpu().numpy()
    if not check:
        return got
    ref, spread, wobble = do.tree_attention(dev[0].double().cpu().numpy(), *codes, *scales, table, lens,
                                            dev[1].double().cpu().numpy(), dev[2].double().cpu().numpy(), parent, scale or None)
    n, D = int(np.max(lens)) + q.shape[1], q.shape[3]
    if dtype == "bfloat16":
        tol = spread * (2.0 ** -8 + 2.0 ** -16 * wobble[..., None]) + 2.0 ** -9 * np.abs(ref) + 1e-30
    else:
        tol = spread * ((n + D) * 2.0 ** -24 + 2 * D * 2.0 ** -24 * wobble[..., None]) + 2.0 ** -24 * np.abs(ref) + 1e-30
    assert np.isfinite(got).all()
    worst = float((np.abs(got - ref) / tol).max())
    assert worst <= 1.0, worst
    assert sbd.sbd_device_error() == 0
    return got


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,Hq,H,D,page", [
    (1, 4, 1, 128, 64), (2, 8, 8, 64, 16), (5, 6, 2, 128, 16), (7, 8, 2, 64, 16), (8, 8, 2, 128, 128), (16, 8, 2, 128, 64),
    (31, 4, 2, 64, 128), (32, 4, 1, 128, 32), (33, 2, 2, 64, 64), (33, 3, 1, 128, 32), (48, 8, 2, 128, 64), (64, 2, 1, 64, 16),
    (64, 8, 1, 128, 64), (63, 1, 1, 128, 128)])
@pytest.mark.parametrize("lens", [[0], [1, 0, 17], [700, 0, 129, 2049]])
def test_tree_attention(sbd, dtype, n, Hq, H, D, page, lens):  # noqa: F811
    rng = np.random.default_rng(n * 100 + D + page + len(lens))
    case = tp._attention_case(rng, len(lens), n, Hq, H, D, page, lens)
    _attend(sbd, case, _trees(rng, len(lens), n), dtype)


@pytest.mark.parametrize("kind", ["chain", "binary", "star", "none", "deep"])
@pytest.mark.parametrize("n,D,dtype", [(64, 128, "bfloat16"), (64, 64, "bfloat16"), (32, 64, "bfloat16"), (17, 128, "float32"),
                                       (64, 64, "float32"), (7, 128, "bfloat16")])
def test_tree_attention_shapes_of_trees(sbd, kind, n, D, dtype):  # noqa: F811
    rng = np.random.default_rng(n + D)
    _attend(sbd, tp._attention_case(rng, 2, n, 4, 2, D, 32, [100, 0]), _trees(rng, 2, n, kind), dtype)


@pytest.mark.parametrize("num_splits", [1, 3, 16])
@pytest.mark.parametrize("n,D,dtype", [(64, 128, "bfloat16"), (40, 64, "bfloat16"), (9, 128, "bfloat16"), (4, 64, "bfloat16"),
                                       (12, 128, "float32")])
def test_tree_attention_splits(sbd, num_splits, n, D, dtype):  # noqa: F811
    rng = np.random.default_rng(num_splits)
    _attend(sbd, tp._attention_case(rng, 2, n, 8, 2, D, 64, [1500, 31]), _trees(rng, 2, n), dtype, num_splits=num_splits)


@pytest.mark.parametrize("B,n,Hq,H,D,page,hi", [(200, 1, 2, 1, 128, 16, 700), (97, 3, 4, 2, 64, 32, 300), (45, 8, 16, 4, 128, 64, 900),
                                                (30, 64, 8, 4, 64, 128, 400), (12, 64, 16, 4, 128, 64, 2000)])
def test_tree_attention_of_more_jobs_than_sms(sbd, B, n, Hq, H, D, page, hi):  # noqa: F811
    rng = np.random.default_rng(B)
    lens = rng.integers(0, hi + 1, B) * (rng.random(B) < 0.9)
    _attend(sbd, tp._attention_case(rng, B, n, Hq, H, D, page, lens), _trees(rng, B, n))


@pytest.mark.parametrize("dtype,n,D", [("bfloat16", 1, 64), ("bfloat16", 6, 128), ("bfloat16", 32, 128), ("float32", 32, 64)])
def test_a_chain_is_the_causal_block(sbd, dtype, n, D):  # noqa: F811
    """Bit for bit: the same kernels, the same sums."""
    rng = np.random.default_rng(n)
    case = tp._attention_case(rng, 3, n, 8, 2, D, 32, [300, 0, 77])
    a = _attend(sbd, case, _trees(rng, 3, n, "chain"), dtype, check=False)
    assert (a == tp._attend(sbd, case, dtype, n_causal=n, check=False)).all()


@pytest.mark.parametrize("dtype,n,D", [("bfloat16", 4, 64), ("bfloat16", 16, 128), ("bfloat16", 64, 64), ("bfloat16", 50, 128),
                                       ("float32", 6, 128), ("float32", 64, 64)])
def test_what_a_node_does_not_see_stays_out(sbd, dtype, n, D):  # noqa: F811
    """Keys and values that are infinite or NaN reach only the nodes below them."""
    rng = np.random.default_rng(n)
    case = tp._attention_case(rng, 2, n, 8, 2, D, 32, [40, 0])
    parent = _trees(rng, 2, n, "random")
    sick = n // 2
    below = np.array([[sick in do.ancestors(parent[b], i) for i in range(n)] for b in range(2)])
    full = _attend(sbd, case, parent, dtype)
    for w, x in ((6, np.inf), (6, np.nan), (5, np.nan)):
        bad = [c.copy() if isinstance(c, np.ndarray) else c for c in case]
        bad[w][:, sick] = x
        got = _attend(sbd, bad, parent, dtype, check=False)
        assert (got[~below] == full[~below]).all() and not np.isfinite(got[below]).any()
    # and a query that is NaN is its own row's matter
    bad = [c.copy() if isinstance(c, np.ndarray) else c for c in case]
    bad[0][:, sick] = np.nan
    got = _attend(sbd, bad, parent, dtype, check=False)
    assert np.isnan(got[:, sick]).all() and (np.delete(got, sick, 1) == np.delete(full, sick, 1)).all()
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype,n", [("bfloat16", 5), ("bfloat16", 64), ("float32", 40)])
def test_parents_out_of_range_are_told(sbd, dtype, n):  # noqa: F811
    rng = np.random.default_rng(n)
    case = tp._attention_case(rng, 2, n, 8, 2, 64, 32, [40, 3])
    parent = _trees(rng, 2, n, "chain")
    parent[0, 2], parent[1, n - 1] = -100, -1       # roots
    good = _attend(sbd, case, parent, dtype)
    for x, y in ((2, n - 1), (n, 10 ** 9), (3, 2 ** 31 - 1)):
        parent[0, 2], parent[1, n - 1] = x, y
        assert (_attend(sbd, case, parent, dtype, check=False) == good).all()
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE


# ------------------------------------------------------------------ verification

def _verify_case(rng, B, n, V, drawn, tau, kind="random", alike=0.5):
    target = 2.0 * rng.normal(size=(B, n, V))
    target[:, :, rng.integers(V, size=max(1, V // 50))] += 3
    draft = target + alike * rng.normal(size=(B, n, V))
    parent = _trees(rng, B, n, kind)
    token = np.zeros((B, n), np.int32)
    for b in range(B):
        for i in range(1, n):
            p = parent[b, i]
            if p >= 0:
                z = (draft[b, p] if rng.random() < 0.7 else target[b, p]) / (tau or 1.0)
                token[b, i] = np.argmax(z + (rng.gumbel(size=V) if tau else 0.3 * rng.normal(size=V)))
    return target, draft if drawn else None, parent, token, rng.random((B, n)), rng.gumbel(size=(B, V))


def _verify(sbd, case, tau, dtype="bfloat16", compare=0.8):  # noqa: F811
    import torch
    target, draft, parent, token, uniform, gumbel = case
    dt = getattr(torch, dtype)
    logits = [None if x is None else torch.from_numpy(np.asarray(x, np.float32)).to(dt).cuda() for x in (target, draft)]
    u, g = (None, None) if tau == 0 else (_f32(uniform), _f32(gumbel))
    out = sbd.sbd_verify_tree(*logits, tp._i32(parent), tp._i32(token), u, g, tau)
    path, tokens, logprob, count = (x.cpu().numpy() for x in out)
    B, n = parent.shape
    seen = 0
    for b in range(B):
        ref = do.verify(logits[0][b].double().cpu().numpy(), None if draft is None else logits[1][b].double().cpu().numpy(),
                        parent[b], token[b], None if u is None else u[b].double().cpu().numpy(),
                        None if g is None else g[b].double().cpu().numpy(), tau)
        m = int(count[b])
        assert 1 <= m <= n and (path[b, m:] == -1).all() and (tokens[b, m:] == -1).all() and (logprob[b, m:] == 0).all()
        if ref[3] < BORDER:
            continue
        seen += 1
        assert path[b, :m].tolist() == ref[0] and tokens[b, :m].tolist() == ref[1], b
        want = np.asarray(ref[2])
        assert (np.isinf(want) == np.isinf(logprob[b, :m])).all()
        ok = np.isfinite(want)
        assert (np.abs(logprob[b, :m] - want)[ok] <= 2.0 ** -16 + 2.0 ** -21 * np.abs(want[ok])).all()
    assert seen >= compare * B
    return path, tokens, logprob, count


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("mode", ["drawn", "given", "greedy"])
@pytest.mark.parametrize("B,n,V,tau", [(1, 1, 1000, 1.0), (1, 8, 128256, 1.0), (3, 1, 1, 1.0), (5, 4, 2, 1.0), (7, 6, 7, 0.8), (40, 12, 333, 1.0),
                                       (9, 7, 50257, 0.5), (170, 5, 1001, 1.3), (2, 64, 4099, 1.0), (33, 16, 2048, 2.0), (1, 2, 1 << 24, 1.0), (10, 3, 131072, 1.0)])
def test_verify(sbd, dtype, mode, B, n, V, tau):  # noqa: F811
    rng = np.random.default_rng(B * n + V)
    tau = 0.0 if mode == "greedy" else tau
    kind = "chain" if n == 8 else "random"
    _verify(sbd, _verify_case(rng, B, n, V, mode == "drawn", tau, kind), tau, dtype)
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("mode", ["drawn", "given"])
@pytest.mark.parametrize("kind", ["star", "binary", "chain"])
def test_verify_shapes_of_trees(sbd, mode, kind):  # noqa: F811
    """Many rejected children of one node, and drafts that are nothing like the target."""
    rng = np.random.default_rng(1)
    for alike in (0.1, 3.0):
        case = _verify_case(rng, 30, 10, 600, mode == "drawn", 1.0, kind, alike)
        _, _, _, count = _verify(sbd, case, 1.0, "float32")
        assert count.max() > 1
    # siblings with the same token
    case[3][:, 2::2] = case[3][:, 1:2]
    _verify(sbd, case, 1.0, "float32")
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_verify_special_logits(sbd, dtype):  # noqa: F811
    rng = np.random.default_rng(5)
    for mode, tau in (("drawn", 1.0), ("given", 0.7), ("greedy", 0.0)):
        case = _verify_case(rng, 12, 5, 777, mode == "drawn", tau, "chain")
        z = case[0]
        z[0, :, 100:] = -np.inf                    # a constrained vocabulary
        z[1, 0, 5] = np.nan                        # counts as -inf
        z[2, 0, 700] = np.inf                      # takes all
        z[3, 0, [3, 9]] = np.inf                   # share it
        z[4, 0] = -np.inf                          # nothing to say
        z[5, 0] = np.nan
        z[6, 0] = -3.0e38
        z[7, 0, :] = 0.0
        z[8, 0, 0] = 3.0e38
        z[9] *= 200
        if case[1] is not None:
            case[1][0, :, 50:] = -np.inf
            case[1][10, 0] = -np.inf
            case[1][11, 0, 4] = np.inf
        with np.errstate(invalid="ignore"):
            path, tokens, logprob, count = _verify(sbd, case, tau, dtype, 0.6)
        for b in (4, 5):                           # all alike
            assert tau or tokens[b, 0] == 0
            assert abs(logprob[b, 0] + np.log(777)) < 2.0 ** -15
    assert sbd.sbd_device_error() == 0


@pytest.mark.parametrize("V", [5, 64, 1003, 40000])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_verify_among_nothing_but_nan_and_infinities(sbd, dtype, V):  # noqa: F811
    """Rows of which only a few logits are ordinary, or none: what is masked does not come out."""
    rng = np.random.default_rng(V)
    for mode, tau in (("drawn", 1.0), ("given", 2.0), ("greedy", 0.0)):
        case = _verify_case(rng, 8, 4, V, mode == "drawn", tau, "chain")
        z = case[0]
        keep = rng.permutation(V)[:3]
        masked = np.ones(V, bool)
        masked[keep] = False
        for b, x in enumerate((np.nan, -np.inf, -3.38e38, np.nan)):
            z[b][:, masked] = x
            if case[1] is not None and b < 3:
                case[1][b][:, masked] = x
        z[4] = -np.inf
        z[5, 0] = np.nan
        z[6, :, ::2] = np.nan
        for b in range(4):
            case[3][b, 1:] = keep[0]
        _, tokens, _, _ = _verify(sbd, case, tau, dtype, 0.5)
        for b in range(4):
            assert set(tokens[b]) <= {-1, *keep.tolist()}, (mode, b)
    assert sbd.sbd_device_error() == 0


def test_verify_ties_go_to_the_lowest_index(sbd):  # noqa: F811
    import torch
    for V in (4, 1000, 128256):
        z = torch.zeros(2, 2, V, device="cuda").bfloat16()
        z[1, 0, [V - 1, V // 2, V // 2 + 1]] = 5.0
        parent, token = tp._i32([[-1, 0]] * 2), tp._i32([[0, 1], [0, V // 2]])
        path, tokens, _, count = sbd.sbd_verify_tree(z, None, parent, token, None, None, 0.0)
        assert tokens.tolist() == [[0, -1], [V // 2, 0]] and count.tolist() == [1, 2]
        g, u = torch.zeros(2, V, device="cuda"), torch.ones(2, 2, device="cuda")
        _, tokens, _, count = sbd.sbd_verify_tree(z, z, parent, token, u, g, 1.0)
        assert tokens.tolist() == [[0, -1], [V // 2, -1]] and count.tolist() == [1, 1]   # refused, and nothing left


def test_verify_refusals(sbd):  # noqa: F811
    """Parents and tokens out of range are told, passed over, and change nothing else."""
    rng = np.random.default_rng(7)
    case = list(_verify_case(rng, 6, 6, 500, True, 1.0, "chain"))
    case[4][:] = 0.0                               # all accepted
    _, _, _, count = _verify(sbd, case, 1.0, "float32", 0.0)
    assert (count == 6).all()
    for x in (-1, 500, 2 ** 31 - 1):
        case[3] = case[3].copy()
        case[3][:, 3] = x
        assert (_verify(sbd, case, 1.0, "float32", 0.0)[3] == 3).all()
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE
    case[3][:, 3] = 0
    for x in (3, 4, 10 ** 6):
        case[2] = case[2].copy()
        case[2][:, 3] = x
        assert (_verify(sbd, case, 1.0, "float32", 0.0)[3] == 3).all()
        assert sbd.sbd_device_error() == sbd.SBD_DEVERR_TREE
    case[2][:, 3] = -5                             # padding, with any token
    case[3][:, 3] = -9
    assert (_verify(sbd, case, 1.0, "float32", 0.0)[3] == 3).all()
    assert sbd.sbd_device_error() == 0


def test_verify_of_many_logits(sbd):  # noqa: F811
    """Offsets past 2^31 elements."""
    import torch
    B, n, V = 280, 64, 128251
    rng = np.random.default_rng(0)
    z = torch.zeros(B, n, V, dtype=torch.bfloat16, device="cuda")
    small = _verify_case(rng, 1, n, V, True, 1.0, "chain")
    small[4][:] *= 0.5
    z[-1] = torch.from_numpy(small[0][0].astype(np.float32)).bfloat16().cuda()
    parent, token = np.repeat(small[2], B, 0), np.repeat(small[3], B, 0)
    u, g = _f32(np.repeat(small[4], B, 0)), torch.zeros(B, V, device="cuda")
    big = sbd.sbd_verify_tree(z, None, tp._i32(parent), tp._i32(token), u, g, 1.0)
    one = sbd.sbd_verify_tree(z[-1:].contiguous(), None, tp._i32(parent[:1]), tp._i32(token[:1]), u[:1].contiguous(), g[:1].contiguous(), 1.0)
    # (a request alone is more CTAs: sums in another order, the same decisions)
    for a, b in zip(big, one):
        assert torch.allclose(a[-1:].float(), b.float(), rtol=0, atol=2.0 ** -15)
    assert (big[3][:-1] == 1).all() and (big[1][:-1, 0] == 0).all()


# ------------------------------------------------------------------ append of a path

def _path_case(rng, B, n, page, hi):
    lens = rng.integers(0, hi + 1, B)
    new = rng.integers(0, n + 1, B)
    path = np.full((B, n), -1, np.int32)
    for b in range(B):
        path[b, :new[b]] = np.sort(rng.permutation(n)[:new[b]])
    pages = int(sum(-(-(a + c) // page) for a, c in zip(lens, new))) + 2
    table, _ = tp._table(rng, lens + new, page, pages, int((-(-(lens + new) // page)).max()) + 1)
    start = np.concatenate([[0], np.cumsum(new)])
    slots = np.full(int(start[-1]) + 3, -1, np.int32)
    for b in range(B):
        pos = np.arange(lens[b], lens[b] + new[b])
        slots[start[b]:start[b + 1]] = table[b, pos // page] * page + pos % page
    return path, start, slots, pages


def _append(sbd, x, path, start, slots, codes, scale, page, dtype, fused=True):  # noqa: F811
    import torch
    B, n, H, D = x.shape
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(getattr(torch, dtype)).cuda()
    new = [t, -2 * t]
    if fused:
        w = torch.randn(B, n + 2, 2 * H + 3, D, device="cuda").to(t.dtype)
        w[:, 1:n + 1, 3:3 + H], w[:, 1:n + 1, 3 + H:] = new[0], new[1]
        new = [w[:, 1:n + 1, 3:3 + H], w[:, 1:n + 1, 3 + H:]]
    caches, scales = [tp._f8(c) for c in codes], [_f32(s) for s in scale]
    sbd.sbd_cache_append_path_q8(*new, tp._i32(path), tp._i32(start), tp._i32(slots), *caches, *scales)
    for w in range(2):
        with np.errstate(invalid="ignore"):
            ref = do.append_path(new[w].double().cpu().numpy(), path, start, slots, codes[w], scale[w], page)
        assert (scales[w].cpu().numpy() == ref[1]).all(), w
        got = tp._bytes(caches[w])
        bad = got != ref[0]
        assert not (bad & ~((got & 127 == 127) & (ref[0] & 127 == 127))).any(), w   # (NaN has two codes)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("B,n,H,D,page,hi", [(1, 1, 1, 64, 16, 0), (1, 16, 8, 128, 64, 100), (5, 7, 2, 64, 16, 50), (40, 33, 4, 64, 16, 300),
                                             (16, 64, 3, 128, 32, 200), (9, 64, 2, 128, 128, 500), (300, 3, 1, 128, 64, 90)])
def test_append_path(sbd, dtype, B, n, H, D, page, hi):  # noqa: F811
    rng = np.random.default_rng(B * n + D)
    path, start, slots, pages = _path_case(rng, B, n, page, hi)
    codes = [po.e4m3_encode(rng.normal(size=(pages, H, page, D)) * 30) for _ in range(2)]
    scale = [2.0 ** rng.integers(-12, 0, (pages, H)).astype(np.float32) for _ in range(2)]
    x = rng.normal(size=(B, n, H, D)) * np.exp(rng.normal(size=(B, n, 1, 1)))
    _append(sbd, x, path, start, slots, codes, scale, page, dtype, fused=B != 5)
    assert sbd.sbd_device_error() == 0


def test_append_path_special_values_and_refusals(sbd):  # noqa: F811
    rng = np.random.default_rng(3)
    path, start, slots, pages = _path_case(rng, 6, 9, 16, 40)
    codes, scale = [np.full((pages, 2, 16, 64), 0x30, np.uint8)] * 2, [np.full((pages, 2), 0.25, np.float32)] * 2
    x = rng.normal(size=(6, 9, 2, 64))
    x[0, :, 0, 3], x[1, 2, :, 5], x[2] = np.inf, np.nan, 0.0
    x[3] *= 1e-30
    x[4] = 3e38
    _append(sbd, x, path, start, slots, codes, scale, 16, "float32")
    assert sbd.sbd_device_error() == 0
    x = rng.normal(size=(6, 9, 2, 64))
    b = int(np.argmax(np.diff(start)))               # a request that gains the most
    for where, value, code in ((path, 9, sbd.SBD_DEVERR_TREE), (path, -1, sbd.SBD_DEVERR_TREE), (path, -2 ** 31, sbd.SBD_DEVERR_TREE),
                               (slots, pages * 16, sbd.SBD_DEVERR_PAGE), (slots, 2 ** 31 - 1, sbd.SBD_DEVERR_PAGE), (slots, -7, 0)):
        p, s = path.copy(), slots.copy()
        (p[b:b + 1, :1] if where is path else s[start[b]:start[b] + 1])[...] = value
        _append(sbd, x, p, start, s, codes, scale, 16, "bfloat16")
        assert sbd.sbd_device_error() == code
    # starts out of range, or that go down: nothing lies in the map, nothing is stored
    for shift in (-10 ** 6, 10 ** 6, 2 ** 31 - 200):
        _append(sbd, x, path, start + shift, slots, codes, scale, 16, "bfloat16")
    _append(sbd, x, path, start[::-1].copy(), slots, codes, scale, 16, "bfloat16")
    assert sbd.sbd_device_error() == 0


def test_append_path_is_append(sbd):  # noqa: F811
    """A chain that is accepted as a whole: what sbd_cache_append_q8 writes."""
    import torch
    rng = np.random.default_rng(9)
    B, n, page = 4, 8, 16
    path, start, slots, pages = _path_case(rng, B, n, page, 60)
    x = torch.randn(B, n, 4, 128, device="cuda").bfloat16()
    kept = np.concatenate([b * n + path[b, :start[b + 1] - start[b]] for b in range(B)])
    outs = []
    for by_path in (True, False):
        cache = [torch.zeros(pages, 2, page, 128, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
        scale = [torch.zeros(pages, 2, device="cuda") for _ in range(2)]
        if by_path:
            sbd.sbd_cache_append_path_q8(x[:, :, :2], x[:, :, 2:], tp._i32(path), tp._i32(start), tp._i32(slots), *cache, *scale)
        else:
            y = x.view(B * n, 4, 128)[torch.from_numpy(kept).cuda()]
            sbd.sbd_cache_append_q8(y[:, :2], y[:, 2:], tp._i32(slots), *cache, *scale)
        outs.append([c.view(torch.uint8) for c in cache] + scale)
    for a, b in zip(*outs):
        assert torch.equal(a, b)
