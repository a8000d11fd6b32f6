"""The calls of drafted decoding together: the example's turns against the 64-bit forms, a
turn captured in a CUDA graph and replayed, on another stream, again and again, and from
two threads at once."""
import importlib.util
import os
import threading

import numpy as np
import pytest

import test_gpu_draft as td
import test_gpu_paged as tp
from oracle import draft_oracle as do
from oracle import paged_oracle as po
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("drafted_decode", os.path.join(ROOT, "examples", "drafted_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("k,page,head_dim,tau", [(7, 16, 64, 1.0), (3, 64, 128, 0.0), (31, 32, 64, 0.7)])
def test_drafted_decode(example, sbd, k, page, head_dim, tau):  # noqa: F811
    import torch
    rng = np.random.default_rng(k)
    lens = [2, 131, 64, 17, 78]
    dec = example.DraftedDecoder(5, n_pages=64, max_pages=20, page=page, k=k, head_dim=head_dim, tau=tau)
    dec.admit([torch.from_numpy(rng.integers(0, dec.vocab, n).astype(np.int32)) for n in lens])
    assert dec.length.tolist() == [n - 1 for n in lens]
    for _ in range(3):
        before = [[c.view(torch.uint8).cpu().numpy() for c in dec.cache], [s.cpu().numpy() for s in dec.scale],
                  dec.length.cpu().numpy(), dec.table.cpu().numpy(), dec.free.cpu().numpy().copy(), int(dec.n_free)]
        tokens, count = dec.turn()
        s = {x: v.double().cpu().numpy() for x, v in dec.seen.items()}
        new, parent = count.cpu().numpy(), dec.chain.cpu().numpy()
        for b in range(5):
            path, said, logprob, margin = do.verify(s["target"][b], s["draft"][b], parent[b], s["rows"][b].astype(int), s["uniform"][b],
                                                    s["gumbel"][b], tau)
            if margin > td.BORDER:
                assert s["path"][b, :new[b]].tolist() == path and tokens[b, :new[b]].tolist() == said
                assert np.abs(s["logprob"][b, :new[b]] - logprob).max() <= 2.0 ** -16 + 2.0 ** -21 * np.abs(logprob).max()
        table, length, start, slots, n_free, _ = po.block_tables(before[2], before[2] + new, before[3], before[4], before[5], page, 5 * (k + 1))
        assert (dec.table.cpu().numpy() == table).all() and (dec.length.cpu().numpy() == length).all() and int(dec.n_free) == n_free
        for w, x in enumerate(("keys", "values")):
            codes, scale = do.append_path(s[x], s["path"].astype(int), start, slots, before[0][w], before[1][w], page)
            assert (dec.cache[w].view(torch.uint8).cpu().numpy() == codes).all()
            assert (dec.scale[w].cpu().numpy() == scale).all()
        assert (dec.last.cpu().numpy() == [tokens[b, new[b] - 1].item() for b in range(5)]).all()
    assert sbd.sbd_device_error() == 0


def test_a_drafted_token_that_holds_always(example, sbd):  # noqa: F811
    """A draft that is the target itself: everything is accepted."""
    import torch
    rng = np.random.default_rng(3)
    B, n, V = 6, 9, 3000
    z = torch.from_numpy(rng.normal(size=(B, n, V)).astype(np.float32)).bfloat16().cuda()
    token = torch.from_numpy(rng.integers(0, V, (B, n)).astype(np.int32)).cuda()
    parent = torch.arange(-1, n - 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    u = torch.rand(B, n, device="cuda") * (1 - 2.0 ** -20)
    path, tokens, _, count = sbd.sbd_verify_tree(z, z.clone(), parent, token, u, torch.randn(B, V, device="cuda"), 1.0)
    assert (count == n).all() and (path == torch.arange(n, device="cuda")).all() and (tokens[:, :-1] == token[:, 1:]).all()


class _Turn:
    """The calls of a turn on fixed tensors, outputs of one the inputs of the next."""

    def __init__(self, sbd, seed, B=5, n=9, H=2, D=128, P=32, V=4099):  # noqa: F811
        import torch
        rng = np.random.default_rng(seed)
        self.sbd, self.n = sbd, n
        lens = rng.integers(0, 200, B)
        table, spare = tp._table(rng, lens, P, 60, 12)
        free = np.zeros(60, np.int32)
        free[:len(spare)] = spare
        self.lens, self.table, self.free0, self.n_free = tp._i32(lens), tp._i32(table), tp._i32(free), tp._i32([len(spare)])
        self.free = self.free0.clone()
        self.cache0 = [tp._f8(po.e4m3_encode(rng.normal(size=(60, H, P, D)) * 30)) for _ in range(2)]
        self.scale0 = [td._f32(2.0 ** rng.integers(-8, 0, (60, H))) for _ in range(2)]
        self.cache, self.scale = [c.clone() for c in self.cache0], [s.clone() for s in self.scale0]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv = torch.randn(B, n, 6 * H, D, generator=g, device="cuda").bfloat16()
        self.pos = (self.lens[:, None] + torch.arange(n, device="cuda", dtype=torch.int32)).contiguous()
        self.inv = torch.logspace(0, -4, D // 2, device="cuda")
        self.w = (1 + 0.1 * torch.randn(2, D, generator=g, device="cuda")).bfloat16()
        self.parent = tp._i32(td._trees(rng, B, n))
        self.logits = [torch.randn(B, n, V, generator=g, device="cuda").bfloat16() for _ in range(2)]
        self.logits[1] = (self.logits[0] + 0.3 * torch.randn(B, n, V, generator=g, device="cuda")).bfloat16()
        self.token = torch.randint(0, V, (B, n), generator=g, device="cuda", dtype=torch.int32)
        self.u, self.g = torch.rand(B, n, generator=g, device="cuda"), torch.randn(B, V, generator=g, device="cuda")
        self.H = H
        self.P = P

    def reset(self):
        for a, b in zip([self.free] + self.cache + self.scale, [self.free0] + self.cache0 + self.scale0):
            a.copy_(b)

    def __call__(self, stream=None):
        sbd, H = self.sbd, self.H  # noqa: F811
        q, k, v = sbd.sbd_qk_norm_rope(self.qkv[:, :, :4 * H], self.qkv[:, :, 4 * H:5 * H], self.qkv[:, :, 5 * H:], self.pos, self.inv,
                                       *self.w, stream=stream)
        out = sbd.sbd_tree_attention_q8(q, *self.cache, *self.scale, self.table, self.lens, k, v, self.parent, stream=stream)
        path, tokens, logprob, count = sbd.sbd_verify_tree(*self.logits, self.parent, self.token, self.u, self.g, 1.0, stream=stream)
        table, length, start, slots, n_free = sbd.sbd_block_tables(
            self.lens, self.lens + count, self.table, self.free, self.n_free, self.P, 5 * self.n, stream=stream)
        sbd.sbd_cache_append_path_q8(k, v, path, start, slots, *self.cache, *self.scale, stream=stream)
        return [q, k, v, out, path, tokens, logprob, count, table, length, start, slots, n_free]

    def state(self, outs):
        import torch
        return [x.clone() for x in outs] + [c.view(torch.uint8).clone() for c in self.cache] + [s.clone() for s in self.scale]


def _same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_turn_in_a_cuda_graph_and_again(sbd):  # noqa: F811
    import torch
    turn = _Turn(sbd, 1)
    want = turn.state(turn())
    for _ in range(20):
        turn.reset()
        assert _same(turn.state(turn()), want)
    turn.reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = turn()
    for _ in range(5):
        turn.reset()
        for x in outs:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(turn.state(outs), want)
    assert sbd.sbd_device_error() == 0


def test_a_turn_on_another_stream(sbd):  # noqa: F811
    import torch
    turn = _Turn(sbd, 2)
    want = turn.state(turn())
    turn.reset()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        outs = turn()
    st.synchronize()
    assert _same(turn.state(outs), want)


def test_turns_at_once(sbd):  # noqa: F811
    """Two requests' turns captured in two graphs that are replayed on two streams, and from two threads."""
    import torch
    turns = [_Turn(sbd, 3), _Turn(sbd, 4)]
    want = [t.state(t()) for t in turns]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in turns]
    for t in turns:
        t.reset()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(t())
    for _ in range(10):
        for t in turns:
            t.reset()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for t, o, w in zip(turns, outs, want):
            assert _same(t.state(o), w)
    got = [None, None]

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(10):
                turns[i].reset()
                got[i] = turns[i].state(turns[i]())
            streams[i].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert _same(got[0], want[0]) and _same(got[1], want[1])
    assert sbd.sbd_device_error() == 0


def test_outputs_go_where_they_are_asked_to(sbd):  # noqa: F811
    """Outputs given by the caller, and bound calls, write the same."""
    import torch
    turn = _Turn(sbd, 5)
    q, k, v, out, path, tokens, logprob, count = turn()[:8]
    turn.reset()
    o = [torch.full_like(x, 7) for x in (q, k, v, out, path, tokens, logprob, count)]
    H = turn.H
    calls = [sbd.prepare_qk_norm_rope(turn.qkv[:, :, :4 * H], turn.qkv[:, :, 4 * H:5 * H], turn.qkv[:, :, 5 * H:], turn.pos, turn.inv,
                                      *turn.w, *o[:3]),
             sbd.prepare_tree_attention_q8(o[0], *turn.cache, *turn.scale, turn.table, turn.lens, o[1], o[2], turn.parent, o[3]),
             sbd.prepare_verify_tree(*turn.logits, turn.parent, turn.token, turn.u, turn.g, 1.0, *o[4:])]
    for c in calls:
        c()
    assert _same(o, (q, k, v, out, path, tokens, logprob, count))


def test_the_binding_refuses_what_does_not_fit(sbd):  # noqa: F811
    import torch
    t = _Turn(sbd, 6)
    H, D = t.H, 128
    q, k, v = t.qkv[:, :, :4 * H], t.qkv[:, :, 4 * H:5 * H], t.qkv[:, :, 5 * H:]
    for args, error in (((q, k[:, :-1], v, t.pos, t.inv), ValueError), ((q, k, v[:, :, :1], t.pos, t.inv), ValueError),
                        ((q, k, v, t.pos[:, 1:].contiguous(), t.inv), ValueError), ((q, k, v, None, t.inv), ValueError),
                        ((q, k, v, t.pos.long(), t.inv), TypeError), ((q, k, v, t.pos, t.inv.double()), TypeError),
                        ((q, k.float(), v, t.pos, t.inv), TypeError), ((q.transpose(2, 3), k, v, t.pos, t.inv), ValueError),
                        ((q, k, v, t.pos, t.inv, t.w[0, :64]), ValueError), ((q.half(), k.half(), v.half(), t.pos, t.inv), TypeError),
                        ((q, k, v, t.pos, t.inv[:60].contiguous()), sbd.SbdError)):
        with pytest.raises(error):
            sbd.sbd_qk_norm_rope(*args)
    qc, kc, vc = q.contiguous(), k.contiguous(), v.contiguous()
    for parent, error in ((t.parent[:, 1:].contiguous(), ValueError), (t.parent.long(), TypeError), (t.parent.cpu(), ValueError)):
        with pytest.raises(error):
            sbd.sbd_tree_attention_q8(qc, *t.cache, *t.scale, t.table, t.lens, kc, vc, parent)
    a = [*t.logits, t.parent, t.token, t.u, t.g]
    for i, x, error in ((0, t.logits[0][0], ValueError), (1, t.logits[1].float(), TypeError), (1, t.logits[1][:, 1:].contiguous(), ValueError),
                        (2, t.parent[:, 1:].contiguous(), ValueError), (3, t.token.long(), TypeError), (4, t.u.double(), TypeError),
                        (4, None, sbd.SbdError), (5, t.g[:, 1:].contiguous(), ValueError), (5, None, sbd.SbdError), (5, t.g[:, ::2], ValueError)):
        b = list(a)
        b[i] = x
        with pytest.raises(error):
            sbd.sbd_verify_tree(*b, 1.0)
    path, start, slots = t.parent, tp._i32(range(6)), tp._i32(range(9))
    for k_new, p, s, error in ((kc[0], path, start, ValueError), (kc, path[:, 1:].contiguous(), start, ValueError), (kc, path, start[1:].clone(), ValueError),
                               (kc[:, :, :1], path, start, ValueError), (kc, path.long(), start, TypeError)):
        with pytest.raises(error):
            sbd.sbd_cache_append_path_q8(k_new, vc, p, s, slots, *t.cache, *t.scale)
    assert sbd.sbd_device_error() == 0


def test_a_cache_of_more_than_4_gb(sbd):  # noqa: F811
    """Offsets past 32 bits: the pages lie at the end of the cache."""
    import torch
    D, H, P, n = 128, 8, 128, 40
    n_pages = (1 << 32) // (D * H * P) + 40
    rng = np.random.default_rng(3)
    q, codes, scales, table, lens, kb, vb = tp._attention_case(rng, 1, n, 4, 1, D, P, [700])
    parent = tp._i32(td._trees(rng, 1, n))
    cache = [torch.zeros(n_pages, H, P, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(n_pages, H, device="cuda") for _ in range(2)]
    base = n_pages - codes[0].shape[0]
    for w in range(2):
        cache[w][base:, H - 1] = torch.from_numpy(codes[w][:, 0]).cuda()
        scale[w][base:, H - 1] = torch.from_numpy(scales[w][:, 0]).cuda()
    f8 = [c.view(torch.float8_e4m3fn) for c in cache]
    for dt in (torch.bfloat16, torch.float32):
        dev = [torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda() for x in (q, kb, vb)]
        wide = [torch.zeros(1, n, H * x.shape[2], D, dtype=dt, device="cuda") for x in dev]
        for w, x in zip(wide, dev):
            w[:, :, -x.shape[2]:] = x
        out = sbd.sbd_tree_attention_q8(wide[0], *f8, *scale, tp._i32(np.where(table >= 0, table + base, -1)), tp._i32(lens), *wide[1:], parent)
        small = sbd.sbd_tree_attention_q8(dev[0], *(tp._f8(c) for c in codes), *(td._f32(s) for s in scales), tp._i32(table), tp._i32(lens),
                                          *dev[1:], parent)
        tol = 2e-2 if dt == torch.bfloat16 else 1e-5
        assert (out[:, :, -4:].float() - small.float()).abs().max().item() <= tol * small.abs().max().item()
    x = torch.randn(1, 4, H, D, device="cuda")
    path, start = tp._i32([[0, 2, 3, -1]]), tp._i32([0, 3])
    sbd.sbd_cache_append_path_q8(x, x, path, start, tp._i32((n_pages - 1) * P + np.arange(4)), *f8, *scale)
    got = f8[0][-1, :, :3].float() * scale[0][-1][:, None, None]
    assert (got.transpose(0, 1) - x[0, [0, 2, 3]]).abs().max().item() <= 2.0 ** -4 * x.abs().max().item()
    assert sbd.sbd_device_error() == 0


def test_many_requests(sbd):  # noqa: F811
    """More requests than a wave, each with a tree of its own."""
    import torch
    rng = np.random.default_rng(8)
    B, n, V = 5000, 4, 9
    case = td._verify_case(rng, B, n, V, True, 1.0)
    td._verify(sbd, case, 1.0, "float32", 0.9)
    path, start, slots, pages = td._path_case(rng, B, n, 16, 3)
    codes, scale = [np.full((pages, 1, 16, 64), 0x31, np.uint8)] * 2, [np.full((pages, 1), 2.0 ** -9, np.float32)] * 2
    td._append(sbd, rng.normal(size=(B, n, 1, 64)), path, start, slots, codes, scale, 16, "bfloat16")
    x = torch.randn(B, n, 3, 64, device="cuda").bfloat16()
    pos, inv = torch.zeros(B, n, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    q, k, v = sbd.sbd_qk_norm_rope(x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], pos, inv)
    assert torch.equal(q, x[:, :, :1]) and torch.equal(k, x[:, :, 1:2]) and torch.equal(v, x[:, :, 2:])
    assert sbd.sbd_device_error() == 0


def test_the_first_calls_of_a_process_are_captured():
    """No call has to be made before a capture."""
    import subprocess
    import sys
    code = """
import sys
sys.path[:0] = [%r, %r]
import torch
import paper_2509_04185_gb300 as sbd
import test_gpu_draft_turn as t
turn = t._Turn(sbd, 1)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    outs = turn()
graph.replay()
torch.cuda.synchronize()
got = turn.state(outs)
turn.reset()
assert t._same(got, turn.state(turn())) and sbd.sbd_device_error() == 0
print("captured")
""" % (ROOT, os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
