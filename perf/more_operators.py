"""The operators of a turn of drafted decoding over the paged 8-bit cache, as cases to time.

A turn checks a tree of drafted tokens against the model: node 0 is the last token that was kept, ``parent[b, i]``
the node that node i follows (a node with parent -1 that is not node 0 is padding).  ``qk_norm_rope`` splits the
nodes' fused projection into normed and rotated queries, keys and values; ``tree_attention_q8`` lets every node see
the cache, itself and its ancestors; ``verify_tree`` walks down from node 0, accepting drafted tokens by the target's
probabilities and given random numbers; ``cache_append_path_q8`` brings the accepted nodes' keys and values into the
cache.

A case is one pass through one of them.  The plain forms are elementary torch operations in 32 bits (angles, sums
over the vocabulary and comparisons of probabilities in 64); the framework's calls are the ones bound to fixed
tensors (``prepare_*``), as a decode loop uses them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------ cases

def _rope(name=None, dtype="bf16", batch=1, nodes=16, q_heads=32, kv_heads=8, head_dim=128, rotary=128, norm=True,
          interleaved=False, pos_lo=4096, pos_hi=4096, theta=1e6):
    return dict(kind="rope", name=name, dtype=dtype, batch=batch, nodes=nodes, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, rotary=rotary, norm=norm, interleaved=interleaved, pos_lo=pos_lo, pos_hi=pos_hi,
                theta=theta)


def _tree(name=None, dtype="bf16", batch=1, page=64, nodes=16, width=2, pad=0.0, q_heads=32, kv_heads=8, head_dim=128,
          len_lo=4096, len_hi=4096):
    return dict(kind="tree", name=name, dtype=dtype, batch=batch, page=page, nodes=nodes, width=width, pad=pad,
                q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, len_lo=len_lo, len_hi=len_hi)


def _verify(name=None, dtype="bf16", batch=1, nodes=8, width=1, pad=0.0, vocab=128256, draft=True, tau=1.0, acc_lo=3,
            acc_hi=3):
    return dict(kind="verify", name=name, dtype=dtype, batch=batch, nodes=nodes, width=width, pad=pad, vocab=vocab,
                draft=draft, tau=tau, acc_lo=acc_lo, acc_hi=acc_hi)


def _path(name=None, dtype="bf16", batch=16, page=64, nodes=16, width=2, q_heads=32, kv_heads=8, head_dim=128,
          len_lo=512, len_hi=2048, acc_lo=0, acc_hi=3):
    return dict(kind="path", name=name, dtype=dtype, batch=batch, page=page, nodes=nodes, width=width, q_heads=q_heads,
                kv_heads=kv_heads, head_dim=head_dim, len_lo=len_lo, len_hi=len_hi, acc_lo=acc_lo, acc_hi=acc_hi)


def listed():
    return [
        # One user's tree of sixteen nodes, query and key norms with their weights.
        _rope("rope_b1_n16"),
        # Plain next-token decoding of a large batch, contexts of up to a million tokens, no norms, half of the
        # dimensions rotated, fp32 activations, narrow heads, neighbours as pairs.
        _rope("rope_f32_b250_n1", dtype="f32", batch=250, nodes=1, q_heads=6, kv_heads=2, head_dim=64, rotary=32,
              norm=False, interleaved=True, pos_lo=0, pos_hi=1000000, theta=1e4),
        # Prompts: every token of 32768.
        _rope("rope_prefill_32768", nodes=32768, pos_lo=0, pos_hi=0),
        # One user's binary tree over 4096 cached tokens.
        _tree("tree_b1_n16"),
        # A serving batch of uneven lengths, small pages, narrow heads, a few nodes, some of them padding.
        _tree("tree_ragged_b32_n7_d64", batch=32, page=16, nodes=7, pad=0.3, head_dim=64, len_lo=0, len_hi=2047),
        # fp32 activations, one chain of drafted tokens.
        _tree("tree_f32_b2_n5", dtype="f32", batch=2, page=32, nodes=5, width=1, q_heads=8, kv_heads=2, len_lo=100,
              len_hi=701),
        # The widest trees over a full batch.
        _tree("tree_b16_n64", batch=16, nodes=64, width=4, len_lo=8192, len_hi=8192),
        # One user's chain of seven drafted tokens, three of which are accepted.
        _verify("verify_b1_n8"),
        # A serving batch of trees whose requests accept from none to all levels, some nodes padding.
        _verify("verify_b64_n15", batch=64, nodes=15, width=2, pad=0.2, acc_lo=0, acc_hi=3),
        # Greedy decoding, drafts without probabilities, an odd vocabulary.
        _verify("verify_greedy_b9_odd", dtype="f32", batch=9, nodes=6, vocab=50257, draft=False, tau=0.0, acc_lo=0,
                acc_hi=5),
        # The accepted nodes of sixteen users enter the cache.
        _path("path_b16_n16"),
        # A large batch of long chains, small pages, fp32, narrow heads.
        _path("path_f32_b200_n33_d64", dtype="f32", batch=200, page=16, nodes=33, width=1, kv_heads=4, head_dim=64,
              len_lo=0, len_hi=333, acc_lo=0, acc_hi=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rope", "tree", "tree", "verify", "verify", "path"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 3, 4, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128])
    nodes, width = _log_int(rng, 1, 64), rng.choice([1, 2, 2, 3, 4])
    if kind == "rope":
        rows = (group + 2) * kv_heads * head_dim * SIZE[dtype]
        tokens = _log_int(rng, 1, min(32768, 32768 * 48 * 256 // rows))
        batch = _log_int(rng, 1, min(256, tokens))
        return _rope(dtype=dtype, batch=batch, nodes=max(1, tokens // batch), q_heads=group * kv_heads,
                     kv_heads=kv_heads, head_dim=head_dim, rotary=rng.choice([head_dim, head_dim, head_dim // 2, 16]),
                     norm=rng.choice([True, True, False]), interleaved=rng.choice([True, False, False]), pos_lo=0,
                     pos_hi=_log_int(rng, 1, 1000000), theta=rng.choice([1e4, 5e5, 1e6]))
    if kind == "tree":
        hi = _log_int(rng, 16, 4001 if dtype == "f32" else 16000)
        batch = _log_int(rng, 1, max(1, min(64, (16384 if dtype == "f32" else 131072) // hi)))
        if dtype == "f32":
            nodes = min(nodes, 24)
        return _tree(dtype=dtype, batch=batch, page=page, nodes=nodes, width=width, pad=rng.choice([0.0, 0.3]),
                     q_heads=min(group, 4) * kv_heads, kv_heads=kv_heads, head_dim=head_dim,
                     len_lo=rng.choice([0, hi // 4, hi]), len_hi=hi)
    if kind == "verify":
        vocab = _log_int(rng, 1000, 152000)
        batch = _log_int(rng, 1, max(1, min(256, 120000000 * 2 // (SIZE[dtype] * vocab * nodes))))
        return _verify(dtype=dtype, batch=batch, nodes=nodes, width=width, pad=rng.choice([0.0, 0.3]), vocab=vocab,
                       draft=rng.choice([True, True, False]), tau=rng.choice([1.0, 1.0, 0.7, 0.0]), acc_lo=0,
                       acc_hi=rng.randint(0, 8))
    hi = _log_int(rng, 16, 4000)
    batch = _log_int(rng, 1, max(1, min(256, 100000 // hi)))
    return _path(dtype=dtype, batch=batch, page=page, nodes=nodes, width=width, q_heads=group * kv_heads,
                 kv_heads=kv_heads, head_dim=head_dim, len_lo=rng.randint(0, hi), len_hi=hi, acc_lo=0,
                 acc_hi=rng.randint(0, 16))


def _spread(lo, hi, n):
    """n whole numbers evenly spread over [lo, hi]: the same total whatever their order."""
    return [lo + (hi - lo) * (2 * i + 1) // (2 * n) if n > 1 else hi for i in range(n)]


def _pages(length, page):
    return -(-length // page)


def _parents(nodes, width):
    """A tree whose nodes have `width` children each, in index order (1: a chain)."""
    return [-1] + [(i - 1) // width for i in range(1, nodes)]


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _trees(case):
    """(nodes in use, drafted tokens to accept) of every request, before the seed puts them in an order."""
    n, m = case["batch"], case["nodes"]
    used = [max(1, m - int(case.get("pad", 0.0) * m)) if b % 2 else m for b in range(n)]
    deep = _depths(_parents(m, case["width"]))
    return used, [min(a, deep[u - 1]) for a, u in zip(_spread(case["acc_lo"], case["acc_hi"], n), used)]


def work(case):
    n, m, e = case["batch"], case["nodes"], SIZE[case["dtype"]]
    if case["kind"] == "rope":
        t, h, q, d = n * m, case["kv_heads"], case["q_heads"], case["head_dim"]
        return {"bytes": 2 * t * (q + 2 * h) * d * e + 4 * t + 2 * case["rotary"] + 2 * d * e * case["norm"],
                "flops": t * (q + h) * (4 * d * case["norm"] + 3 * case["rotary"])}
    if case["kind"] == "verify":
        used, acc = _trees(case)
        deep = _depths(_parents(m, case["width"]))
        rows = sum(a + 1 for a in acc)
        if case["tau"] > 0 and case["draft"]:
            # the draft's row counts where a node has children to decide on
            rows += sum(min(a + 1, deep[u - 1]) for a, u in zip(acc, used))
        noise = n * case["vocab"] * 4 if case["tau"] > 0 else 0
        return {"bytes": rows * case["vocab"] * e + noise + 4 * n * m * 6 + 4 * n, "flops": 8 * rows * case["vocab"]}
    h, d, q = case["kv_heads"], case["head_dim"], case["q_heads"]
    lens = _spread(case["len_lo"], case["len_hi"], n)
    if case["kind"] == "path":
        t = sum(a + 1 for a in _trees(case)[1])
        return {"bytes": 2 * t * h * d * (e + 1) + 8 * t + 4 * n, "flops": 6 * t * h * d}
    pages = sum(_pages(x, case["page"]) for x in lens)
    return {"bytes": 2 * sum(lens) * h * d + pages * (8 * h + 4) + n * m * ((2 * q + 2 * h) * d * e + 4),
            "flops": 4 * q * m * d * sum(lens)}


# ------------------------------------------------------------------ inputs

def _rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)


def _dev(values, dtype=torch.int32):
    return torch.as_tensor(np.asarray(values), dtype=dtype, device="cuda")


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _table(r, lens, page, n_pages, most):
    """A block table whose requests hold pages of a shuffled pool."""
    perm = r.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), most), -1, dtype=np.int32)
    at = 0
    for b, x in enumerate(lens):
        m = _pages(x, page)
        table[b, :m] = perm[at:at + m]
        at += m
    return table


def _scale_of(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return (torch.where(amax > 0, e + 127, 1) << 23).view(torch.float32)


def _codes(x):
    return x.clamp(-448.0, 448.0).to(E4M3)


def _cache(g, s, n_pages, h, p, d):
    """A filled cache: keys with a few strong channels, values whose size differs from page to page."""
    channel = torch.exp(0.5 * _randn(g, h, 1, d))
    for w in ("k", "v"):
        x = _randn(g, n_pages, h, p, d)
        x *= channel if w == "k" else torch.exp(0.4 * _randn(g, n_pages, h, 1, 1))
        scale = _scale_of(x.abs().amax((2, 3)))
        s[w + "_cache"], s[w + "_scale"] = _codes(x / scale[:, :, None, None]), scale
    return channel


def _order(r, values):
    return [values[i] for i in r.permutation(len(values))]


def _tree_inputs(case, r):
    """Trees in an order of the seed: parents [B, n], and a path of accepted nodes each."""
    m = case["nodes"]
    parents = _parents(m, case["width"])
    deep = np.asarray(_depths(parents))
    pairs = _order(r, list(zip(*_trees(case))))
    table, paths = np.full((case["batch"], m), -1, dtype=np.int32), []
    for b, (used, acc) in enumerate(pairs):
        table[b, :used] = parents[:used]
        node, path = int(r.choice(np.flatnonzero(deep[:used] == acc))), []
        while node >= 0:
            path.append(node)
            node = parents[node]
        paths.append(path[::-1])
    return table, paths


def _rope_inputs(case, seed):
    g, r = _rng(seed)
    n, m, q, h, d = case["batch"], case["nodes"], case["q_heads"], case["kv_heads"], case["head_dim"]
    dt = DTYPES[case["dtype"]]
    x = _randn(g, n, m, q + 2 * h, d).to(dt)
    x[:, :, :q + h] *= torch.exp(0.5 * _randn(g, q + h, d)).to(dt)
    first = _dev(_order(r, _spread(case["pos_lo"], case["pos_hi"], n)))
    pos = first[:, None] + torch.arange(m, device="cuda", dtype=torch.int32)
    half = case["rotary"] // 2
    inv = case["theta"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    s = dict(case=case, q=x[:, :, :q], k=x[:, :, q:q + h], v=x[:, :, q + h:], positions=pos, inv_freq=inv.float(),
             q_weight=None, k_weight=None)
    if case["norm"]:
        s.update(q_weight=(1 + 0.2 * _randn(g, d)).to(dt), k_weight=(1 + 0.2 * _randn(g, d)).to(dt))
    return s


def _attn_inputs(case, seed):
    g, r = _rng(seed)
    n, p, m, h, d, q = (case[x] for x in ("batch", "page", "nodes", "kv_heads", "head_dim", "q_heads"))
    dt = DTYPES[case["dtype"]]
    lens = _order(r, _spread(case["len_lo"], case["len_hi"], n))
    n_pages = sum(_pages(x, p) for x in lens) + 3
    table = _table(r, lens, p, n_pages, max(1, _pages(case["len_hi"], p)) + 1)
    s = dict(case=case, page=p)
    channel = _cache(g, s, n_pages, h, p, d)
    # What lies past a request's last token in its last page is left over from other requests: poisoned here.
    tail = [(int(table[b, x // p]), x % p) for b, x in enumerate(lens) if x % p]
    if tail:
        pages, offs = _dev([a for a, _ in tail], torch.int64), _dev([o for _, o in tail])
        stale = (torch.arange(p, device="cuda")[None] >= offs[:, None])[:, None, :, None]
        for w in ("k_cache", "v_cache"):
            u = s[w].view(torch.uint8)
            u[pages] = torch.where(stale, torch.full_like(u[:1], 0x7F), u[pages])
    u = _randn(g, h, 1, d)
    x = _randn(g, n, m, h, q // h, d) + 0.7 * u
    s["q"] = (1.5 * x / channel).reshape(n, m, q, d).to(dt)
    first = _dev([int(table[b, 0]) for b, x in enumerate(lens) if x], torch.int64)
    if len(first):  # the first token draws a good share of the attention
        s["k_cache"].view(torch.uint8)[first, :, 0] = _codes(
            (1.2 * u * channel)[None, :, 0] / s["k_scale"][first][:, :, None]).view(torch.uint8)
    s["k_blk"] = (_randn(g, n, m, h, d) * channel[:, 0]).to(dt)
    s["v_blk"] = _randn(g, n, m, h, d).to(dt)
    parents = np.full((n, m), -1, dtype=np.int32)
    for b in range(n):
        used = max(1, m - int(case["pad"] * m)) if b % 2 else m
        parents[b, :used] = _parents(used, case["width"])
    s.update(block_table=_dev(table), cache_len=_dev(lens), parent=_dev(parents))
    return s


def _softmax64(z, tau):
    z = z.double()
    e = torch.exp((z - z.amax(-1, keepdim=True)) / tau)
    return e / e.sum(-1, keepdim=True)


def _verify_inputs(case, seed):
    """Logits of a target and of a draft that is like it; the drafted tokens and the numbers that decide on them are
    drawn as such a draft's tokens are, given which of them are to be accepted."""
    g, r = _rng(seed)
    n, m, v, tau = case["batch"], case["nodes"], case["vocab"], case["tau"]
    dt = DTYPES[case["dtype"]]
    parent, paths = _tree_inputs(case, r)
    target = torch.empty(n, m, v, device="cuda", dtype=dt)
    draft = torch.empty(n, m, v, device="cuda", dtype=dt)
    for i in range(m):  # (a node at a time: 32 bits of all of them are a lot)
        z = 2.5 * _randn(g, n, v)
        z.scatter_(1, torch.randint(v, (n, 8), generator=g, device="cuda"), 9 + 2 * _randn(g, n, 8))
        target[:, i] = z.to(dt)
        draft[:, i] = (z + 0.5 * _randn(g, n, v)).to(dt)
    token = torch.zeros(n, m, dtype=torch.int64, device="cuda")
    u = _rand(g, n, m).double()
    rows, par = torch.arange(n, device="cuda"), _dev(parent, torch.int64)
    plan = torch.zeros(n, m, dtype=torch.bool, device="cuda")
    for b, path in enumerate(paths):
        plan[b, path] = True
    cur = torch.zeros(n, dtype=torch.int64, device="cuda")
    p = None if tau == 0 else _softmax64(target[:, 0], tau)
    for c in range(1, m):
        at = par[:, c].clamp(min=0)
        zq = draft[rows, at]
        here, take = par[:, c] == cur, plan[:, c]
        if tau == 0:
            best = target[rows, at].float().argmax(-1)
            token[:, c] = torch.where(take, best, (best + c) % v)
        else:
            q = _softmax64(zq, tau)
            x = torch.argmax(zq.float() / tau - torch.log(-torch.log(_rand(g, n, v).clamp(1e-9, 1 - 1e-7))), -1)
            if case["draft"]:
                w = torch.where(take[:, None], torch.minimum(p, q), (q - p).clamp(min=0))
                x = torch.where(here, torch.multinomial(w.float() + 1e-30, 1, generator=g)[:, 0], x)
                ratio = (p[rows, x] / q[rows, x]).clamp(max=1)
            else:
                ratio = p[rows, x].clamp(max=1)
            token[:, c] = x
            u[:, c] = torch.where(here, torch.where(take, u[:, c] * ratio, ratio + u[:, c] * (1 - ratio)), u[:, c])
            left = (p - q).clamp(min=0) if case["draft"] else p.scatter(1, x[:, None], 0.0)
            p = torch.where((here & ~take)[:, None], left / left.sum(-1, keepdim=True).clamp(min=1e-300), p)
            p = torch.where((here & take)[:, None], _softmax64(target[:, c], tau), p)
        cur = torch.where(here & take, c, cur)
    s = dict(case=case, target=target, draft=draft if case["draft"] and tau > 0 else None, parent=_dev(parent),
             token=token.int(), uniform=None, gumbel=None)
    if tau > 0:
        s["uniform"] = u.float()
        s["gumbel"] = -torch.log(-torch.log(_rand(g, n, v).clamp(1e-9, 1 - 1e-7)))
    return s


def _path_inputs(case, seed):
    g, r = _rng(seed)
    n, p, m, h, d, q = (case[x] for x in ("batch", "page", "nodes", "kv_heads", "head_dim", "q_heads"))
    _, paths = _tree_inputs(case, r)
    lens = _order(r, _spread(case["len_lo"], case["len_hi"], n))
    new = [len(x) for x in paths]
    after = [x + y for x, y in zip(lens, new)]
    n_pages = sum(_pages(x, p) for x in lens) + n * _pages(m, p) + 3
    table = _table(r, after, p, n_pages, _pages(case["len_hi"] + m, p))
    slots = np.full(n * m, -1, dtype=np.int32)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    path = np.full((n, m), -1, dtype=np.int32)
    for b in range(n):
        pos = np.arange(lens[b], after[b])
        slots[start[b]:start[b + 1]] = table[b, pos // p] * p + pos % p
        path[b, :new[b]] = paths[b]
    s = dict(case=case, page=p)
    _cache(g, s, n_pages, h, p, d)
    x = _randn(g, n, m, q + 2 * h, d) * torch.exp(0.6 * _randn(g, n, m, 1, 1))
    x = x.to(DTYPES[case["dtype"]])  # the keys and values are slices of the fused projection
    s.update(k_new=x[:, :, q:q + h], v_new=x[:, :, q + h:], path=_dev(path), new_start=_dev(start), slot_map=_dev(slots))
    return s


_INPUTS = dict(rope=_rope_inputs, tree=_attn_inputs, verify=_verify_inputs, path=_path_inputs)


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    if not own:
        return s
    import paper_2509_04185_gb300 as sbd
    if case["kind"] == "rope":
        s["out"] = [torch.empty(s[w].shape, dtype=s[w].dtype, device="cuda") for w in "qkv"]
        s["call"] = sbd.prepare_qk_norm_rope(
            s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], *s["out"],
            eps=1e-6, interleaved=case["interleaved"])
    elif case["kind"] == "tree":
        s["out"] = torch.empty_like(s["q"])
        s["call"] = sbd.prepare_tree_attention_q8(
            s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"], s["cache_len"],
            s["k_blk"], s["v_blk"], s["parent"], s["out"])
    elif case["kind"] == "verify":
        s["out"] = [torch.empty_like(s["token"]), torch.empty_like(s["token"]),
                    torch.empty(s["token"].shape, device="cuda"), torch.empty_like(s["token"][:, 0])]
        s["call"] = sbd.prepare_verify_tree(s["target"], s["draft"], s["parent"], s["token"], s["uniform"], s["gumbel"],
                                            case["tau"], *s["out"])
    else:
        s["call"] = sbd.prepare_cache_append_path_q8(s["k_new"], s["v_new"], s["path"], s["new_start"], s["slot_map"],
                                                     s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"rope": _plain_rope, "tree": _plain_tree, "verify": _plain_verify, "path": _plain_path}[kind](state)
    state["call"]()
    if kind == "rope":
        return dict(zip("qkv", state["out"]))
    if kind == "tree":
        return state["out"]
    if kind == "verify":
        return dict(zip(("path", "tokens", "logprob", "count"), state["out"]))
    return {w: state[w] for w in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _plain_rope(s):
    c = s["case"]
    half = c["rotary"] // 2
    angle = s["positions"].double()[..., None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    out = dict(v=s["v"].contiguous())
    for w in "qk":
        x = s[w].float()
        if c["norm"]:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * s[w + "_weight"].float()
        a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if c["interleaved"] else (x[..., :half], x[..., half:2 * half])
        first, second = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([first, second], -1).flatten(-2) if c["interleaved"] else torch.cat([first, second], -1)
        out[w] = torch.cat([turned, x[..., 2 * half:]], -1).to(s[w].dtype)
    return {w: out[w] for w in "qkv"}


def _seen_nodes(parent):
    """[B, n, n]: whether row i sees node j."""
    n = parent.shape[1]
    i = torch.arange(n, device=parent.device)
    seen = (i[:, None] == i[None]).expand(parent.shape[0], n, n)
    up = (parent.long()[:, :, None] == i).float()          # one step up
    reach, step = seen.float(), 1
    while step < n:                                        # paths of up to 2 step - 1 steps
        reach = ((reach + torch.matmul(up, reach)) > 0).float()
        up = (torch.matmul(up, up) > 0).float()
        step *= 2
    return reach > 0


def _plain_tree(s):
    q, table, length = s["q"], s["block_table"], s["cache_len"]
    n, m, hq, d = q.shape
    h = s["k_cache"].shape[1]
    most, p = table.shape[1], s["page"]
    at = table.clamp(min=0).long()
    seen = torch.arange(most * p, device="cuda")[None] < length[:, None]                 # [n, keys]
    keys = {}
    for w in ("k", "v"):
        x = s[w + "_cache"].view(torch.uint8)[at].view(E4M3).float() * s[w + "_scale"][at][..., None, None]
        x = x.permute(0, 2, 1, 3, 4).reshape(n, h, most * p, d)
        x = torch.where(seen[:, None, :, None], x, 0.0)
        keys[w] = torch.cat([x, s[w + "_blk"].float().permute(0, 2, 1, 3)], 2)
    mask = torch.cat([seen[:, None].expand(n, m, most * p), _seen_nodes(s["parent"])], 2)
    out = torch.empty_like(q).view(n, m, h, hq // h, d)
    for g in range(hq // h):
        x = q.view(n, m, h, hq // h, d)[:, :, :, g].float().transpose(1, 2)              # [n, h, m, d]
        score = torch.matmul(x, keys["k"].transpose(2, 3)) / math.sqrt(d)
        score = torch.where(mask[:, None], score, -math.inf)
        e = torch.exp(score - score.amax(-1, keepdim=True))
        out[:, :, :, g] = (torch.matmul(e, keys["v"]) / e.sum(-1, keepdim=True)).transpose(1, 2).to(q.dtype)
    return out.view(n, m, hq, d)


def _lowest_of_largest(x):
    """The lowest index of a row's largest value."""
    v = x.shape[-1]
    i = torch.arange(v, device=x.device)
    return torch.where(x == x.amax(-1, keepdim=True), i, v).amin(-1)


def _probabilities(z, tau):
    z = z.float()
    e = torch.exp((z - z.amax(-1, keepdim=True)) / tau).double()
    return e / e.sum(-1, keepdim=True)


def _plain_verify(s):
    target, draft, tau = s["target"], s["draft"], s["case"]["tau"]
    n, m, _ = target.shape
    parent, token = s["parent"].long(), s["token"].long()
    rows = torch.arange(n, device="cuda")
    cur = torch.zeros_like(rows)
    count = torch.ones_like(rows)
    path = torch.full((n, m), -1, dtype=torch.int64, device="cuda")
    tokens = path.clone()
    logprob = torch.zeros((n, m), device="cuda")
    path[:, 0] = 0
    law = _probabilities(target[:, 0], tau or 1.0)         # the target's at the present node, and what is left of it
    p = target[:, 0].float() if tau == 0 else law
    for c in range(1, m):
        here, x = parent[:, c] == cur, token[:, c]
        if tau == 0:
            take = here & (_lowest_of_largest(p) == x)
            p = torch.where(take[:, None], target[:, c].float(), p)
        else:
            q = None if draft is None else _probabilities(draft[rows, cur], tau)
            at_x = p[rows, x]
            u = s["uniform"][:, c].double()
            take = here & (u * (1.0 if q is None else q[rows, x]) < at_x)
            left = p.scatter(1, x[:, None], 0.0) if q is None else (p - q).clamp(min=0)
            total = left.sum(-1, keepdim=True)
            p = torch.where((here & ~take)[:, None] & (total > 0), left / total, p)
            p = torch.where(take[:, None], _probabilities(target[:, c], tau), p)
        said = torch.log(law[rows, x]).float()
        law = torch.where(take[:, None], _probabilities(target[:, c], tau or 1.0), law)
        at = torch.where(take, count, m - 1)
        path[rows, at] = torch.where(take, c, path[rows, at])
        tokens[rows, at - 1] = torch.where(take, x, tokens[rows, at - 1])
        logprob[rows, at - 1] = torch.where(take, said, logprob[rows, at - 1])
        cur, count = torch.where(take, c, cur), count + take
    score = p if tau == 0 else torch.log(p) + s["gumbel"].double()
    last = _lowest_of_largest(score)
    tokens[rows, count - 1] = last
    logprob[rows, count - 1] = torch.log(law[rows, last]).float()
    return dict(path=path.int(), tokens=tokens.int(), logprob=logprob, count=count.int())


def _plain_path(s):
    p, slots, path, start = s["page"], s["slot_map"].long(), s["path"].long(), s["new_start"].long()
    n, m = path.shape
    pages = s["k_cache"].shape[0]
    j = torch.arange(m, device="cuda")
    mine = j[None] < (start[1:] - start[:-1])[:, None]
    slot = slots[(start[:-1, None] + j).clamp(max=len(slots) - 1)]
    keep = mine & (slot >= 0)
    page, off = torch.where(keep, slot // p, pages).reshape(-1), (slot % p).reshape(-1)   # (a page that is dropped again)
    first = torch.full((pages + 1,), p, device="cuda").scatter_reduce(0, page, off, "amin")[:pages]
    touched, fresh = (first < p)[:, None], (first == 0)[:, None]
    held = (torch.arange(p, device="cuda")[None] < first[:, None])[:, None, :, None] & touched[:, :, None, None]
    out = {}
    for w in ("k", "v"):
        cache, scale = s[w + "_cache"], s[w + "_scale"]
        x = s[w + "_new"][torch.arange(n, device="cuda")[:, None], path.clamp(min=0)].float().flatten(0, 1)
        size = x.abs().amax(2)
        amax = torch.zeros(pages + 1, scale.shape[1], device="cuda").scatter_reduce(
            0, page[:, None].expand_as(size), size, "amax")[:pages]
        new = _scale_of(amax)
        new = torch.where(touched, torch.where(fresh, new, torch.maximum(new, scale)), scale)
        moved = _codes(cache.float() * torch.where(held, (scale / new)[:, :, None, None], 1.0))
        u = torch.cat([moved.view(torch.uint8), torch.zeros_like(moved[:1]).view(torch.uint8)])
        u[page, :, off] = _codes(x / torch.cat([new, new[:1]])[page][:, :, None]).view(torch.uint8)
        cache.view(torch.uint8).copy_(u[:pages])
        scale.copy_(new)
        out[w + "_cache"], out[w + "_scale"] = cache, scale
    return {x: out[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale")}


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    return {"rope": _exact_rope, "tree": _exact_tree, "verify": _exact_verify, "path": _exact_path}[case["kind"]](s)


def _exact_rope(s):
    c = s["case"]
    half, d = c["rotary"] // 2, c["head_dim"]
    # Pair j is a complex number that is multiplied by exp(i pos f_j).
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[..., None] * s["inv_freq"].double())
    one = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
    two = one + (1 if c["interleaved"] else half)
    out = {}
    for w in "qk":
        x = s[w].double()
        if c["norm"]:
            x *= torch.rsqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + 1e-6)
            x *= s[w + "_weight"].double()
        else:
            x = x.clone()
        z = torch.complex(x[..., one], x[..., two]) * turn[:, :, None]
        x[..., one], x[..., two] = z.real, z.imag
        out[w] = x
    out["v"] = s["v"].double()
    return out


def _exact_tree(s):
    q, p = s["q"].double(), s["page"]
    n, m, hq, d = q.shape
    h = s["k_cache"].shape[1]
    lens, parent, out = s["cache_len"].tolist(), s["parent"].tolist(), torch.empty_like(q)
    for b in range(n):
        kv = []
        for w in ("k", "v"):
            at = s["block_table"][b, :_pages(lens[b], p)].long()
            x = s[w + "_cache"].view(torch.uint8)[at].view(E4M3).double() * s[w + "_scale"][at].double()[..., None, None]
            x = x.transpose(0, 1).reshape(h, -1, d)[:, :lens[b]]
            kv.append(torch.cat([x, s[w + "_blk"][b].double().transpose(0, 1)], 1))
        hidden = torch.ones(m, lens[b] + m, dtype=torch.bool)
        hidden[:, :lens[b]] = False
        for i in range(m):
            j = i
            while j >= 0:
                hidden[i, lens[b] + j] = False
                j = parent[b][j]
        hidden = hidden.cuda()
        x = q[b].view(m, h, hq // h, d)
        for g in range(hq // h):
            z = (x[:, :, g].transpose(0, 1) @ kv[0].transpose(1, 2)) * d ** -0.5
            out[b].view(m, h, hq // h, d)[:, :, g] = (
                torch.softmax(z.masked_fill(hidden[None], -math.inf), -1) @ kv[1]).transpose(0, 1)
    return out


def _exact_verify(s):
    case = s["case"]
    n, m = s["parent"].shape
    tau = case["tau"]
    parent, token = s["parent"].tolist(), s["token"].tolist()
    path, tokens = [[-1] * m for _ in range(n)], [[-1] * m for _ in range(n)]
    logprob, count = torch.zeros(n, m, dtype=torch.float64), []
    for b in range(n):
        node, walk, said = 0, [0], []
        while True:
            z = s["target"][b, node].double()
            children = [c for c in range(1, m) if parent[b][c] == node]
            if tau == 0:
                best = int((z == z.max()).nonzero()[0])
                hit = [c for c in children if token[b][c] == best][:1]
                if not hit:
                    said.append(best)
                    break
                said.append(best)
                node = hit[0]
                walk.append(node)
                continue
            law = torch.exp(torch.log_softmax(z / tau, -1))
            q = None
            if s["draft"] is not None and children:
                q = torch.exp(torch.log_softmax(s["draft"][b, node].double() / tau, -1))
            found = None
            for c in children:
                x = token[b][c]
                if float(s["uniform"][b, c]) * (1.0 if q is None else float(q[x])) < float(law[x]):
                    found = c
                    break
                rest = law.clone()
                if q is None:
                    rest[x] = 0.0
                else:
                    rest = torch.relu(rest - q)
                if float(rest.sum()) > 0:
                    law = rest / rest.sum()
            if found is None:
                score = torch.log(law) + s["gumbel"][b].double()
                said.append(int((score == score.max()).nonzero()[0]))
                break
            said.append(token[b][found])
            node = found
            walk.append(node)
        count.append(len(walk))
        path[b][:len(walk)], tokens[b][:len(said)] = walk, said
        for j, (i, x) in enumerate(zip(walk, said)):
            z = s["target"][b, i].double() / (tau or 1.0)
            logprob[b, j] = float(z[x] - torch.logsumexp(z, 0))
    return dict(path=_dev(path), tokens=_dev(tokens), logprob=logprob.cuda(), count=_dev(count))


def _round_e4m3(x):
    """x (64 bits) rounded to the nearest e4m3 value, ties to even, saturating."""
    _, e = torch.frexp(x)
    step = (((e.long() - 1).clamp(min=-6) - 3 + 1023) << 52).view(torch.float64)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_path(s):
    p, slots, start, path = s["page"], s["slot_map"].tolist(), s["new_start"].tolist(), s["path"].tolist()
    runs = []  # (request, page, first place, nodes)
    for b in range(len(path)):
        for j, t in enumerate(range(start[b], start[b + 1])):
            if runs and runs[-1][0] == b and slots[t] % p and runs[-1][1] == slots[t] // p:
                runs[-1][3].append(path[b][j])
            else:
                runs.append((b, slots[t] // p, slots[t] % p, [path[b][j]]))
    out = {}
    for w in ("k", "v"):
        cache, scale = s[w + "_cache"].double(), s[w + "_scale"].double().cpu().numpy()
        x = s[w + "_new"].double().cpu().numpy()
        new = scale.copy()
        for b, page, off, nodes in runs:
            seg = x[b, nodes]                                                            # [nodes, h, d]
            e = np.maximum(np.ceil(np.log2(np.maximum(np.abs(seg).max((0, 2)), 1e-300) / 448.0)), -126)
            size = np.abs(seg).max((0, 2))
            e = np.where(size > 448.0 * 2.0 ** e, e + 1, np.where(size <= 448.0 * 2.0 ** (e - 1), e - 1, e))
            fresh = 2.0 ** np.maximum(e, -126)
            new[page] = np.maximum(scale[page], fresh) if off else fresh
            if off and (new[page] != scale[page]).any():
                f = torch.from_numpy(scale[page] / new[page]).cuda()[:, None, None]
                cache[page, :, :off] = _round_e4m3(cache[page, :, :off] * f)
            y = torch.from_numpy(seg / new[page][None, :, None]).cuda().transpose(0, 1)
            cache[page, :, off:off + len(nodes)] = _round_e4m3(y)
        out[w + "_cache"], out[w + "_scale"] = cache, torch.from_numpy(new).cuda()
    return {x: out[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale")}
