"""The calls of drafted decoding reject bad arguments on the host, before anything is
launched (CPU only), and the binding checks its tensors."""
import ctypes

import pytest

A = 1 << 20                              # a pointer that is never followed


@pytest.fixture(scope="module")
def sbd():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2509_04185_gb300
    return paper_2509_04185_gb300


def _pointers(f, sbd, desc, names, rest=(), optional=()):
    """Every pointer refused where it is NULL (unless optional) or misaligned, by its name."""
    for i, name in enumerate(names):
        for bad in (None, A + 4):
            if bad is None and name in optional:
                continue
            ptrs = [A + 4096 * j for j in range(len(names))]
            ptrs[i] = bad
            assert f(ctypes.byref(desc), *ptrs, *rest) == sbd.SBD_ERR_INVALID_ARG, name
            assert name.encode() in sbd.lib.sbd_last_error()


# ------------------------------------------------------------------ norms and rotation

def _rope(sbd, **over):
    d = dict(tokens=16, group=16, n_q_heads=32, n_kv_heads=8, head_dim=128, rotary_dim=128, interleaved=0,
             dtype=sbd.SBD_DTYPE_BF16, eps=1e-6, q_group_stride=0, q_token_stride=6144, k_group_stride=0,
             k_token_stride=6144, v_group_stride=0, v_token_stride=6144)
    d.update(over)
    return sbd.NormRopeDesc(**d)


ROPE = ("q", "k", "v", "positions", "inv_freq", "q_weight", "k_weight", "q_out", "k_out", "v_out")


@pytest.mark.parametrize("over,status", [
    (dict(tokens=-1), 1), (dict(group=0), 1), (dict(n_q_heads=0), 1), (dict(n_kv_heads=0), 1), (dict(head_dim=0), 1),
    (dict(head_dim=96), 2), (dict(rotary_dim=-16), 1), (dict(rotary_dim=144), 1), (dict(rotary_dim=24), 2),
    (dict(dtype=4), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(q_token_stride=6148), 2), (dict(k_group_stride=-8), 2), (dict(v_token_stride=4), 2),
    (dict(dtype=0, v_group_stride=2), 2), (dict(n_q_heads=70000), 2),
])
def test_norm_rope_rejects_bad_descriptors(sbd, over, status):
    st = sbd.lib.sbd_qk_norm_rope(ctypes.byref(_rope(sbd, **over)), *[A + 4096 * i for i in range(10)], None)
    assert st == status and sbd.lib.sbd_last_error() != b""


def test_norm_rope_rejects_bad_pointers(sbd):
    f = sbd.lib.sbd_qk_norm_rope
    assert f(None, *[A] * 10, None) == sbd.SBD_ERR_INVALID_ARG
    _pointers(f, sbd, _rope(sbd), ROPE, (None,), optional=("q_weight", "k_weight"))
    good = [A + 4096 * i for i in range(10)]
    for i, j in ((7, 0), (8, 1), (9, 2), (7, 8), (9, 8), (9, 7)):      # an output over an input or another output
        ptrs = list(good)
        ptrs[i] = good[j]
        assert f(ctypes.byref(_rope(sbd)), *ptrs, None) == sbd.SBD_ERR_INVALID_ARG
        assert b"other memory" in sbd.lib.sbd_last_error()
    assert f(ctypes.byref(_rope(sbd, tokens=0)), *[None] * 10, None) == sbd.SBD_OK


# ------------------------------------------------------------------ tree attention

def _attn(sbd, **over):
    d = dict(batch=1, block_k=16, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=64, max_pages=64,
             n_pages=100, dtype=sbd.SBD_DTYPE_BF16, n_causal=0, scale=0.0, num_splits=0)
    d.update(over)
    return sbd.AttnQ8Desc(**d)


@pytest.mark.parametrize("over,status", [
    (dict(batch=-1), 1), (dict(block_k=0), 1), (dict(block_k=65), 2), (dict(head_dim=96), 2), (dict(n_q_heads=30), 1),
    (dict(n_causal=1), 1), (dict(dtype=5), 1), (dict(page_size=48), 2), (dict(max_pages=0), 1), (dict(n_pages=0), 1),
    (dict(scale=-1.0), 1), (dict(num_splits=-1), 1), (dict(batch=1 << 17), 2), (dict(n_q_heads=2048, block_k=64), 2),
])
def test_tree_attention_rejects_bad_descriptors(sbd, over, status):
    d = _attn(sbd, **over)
    st = sbd.lib.sbd_tree_attention_q8(ctypes.byref(d), *[A] * 11, None, 0, None)
    assert st == status and sbd.lib.sbd_last_error() != b""
    assert sbd.lib.sbd_tree_attention_q8_workspace_size(ctypes.byref(d)) == 0


def test_tree_attention_rejects_bad_pointers(sbd):
    f = sbd.lib.sbd_tree_attention_q8
    assert f(None, *[A] * 11, None, 0, None) == sbd.SBD_ERR_INVALID_ARG
    _pointers(f, sbd, _attn(sbd, block_k=64), ("q", "k_cache", "v_cache", "k_scale", "v_scale", "block_table", "cache_len",
                                               "k_blk", "v_blk", "parent", "out"), (None, 0, None))
    assert f(ctypes.byref(_attn(sbd, batch=0)), *[None] * 11, None, 0, None) == sbd.SBD_OK
    # a block of 64 is a tree's only
    assert sbd.lib.sbd_block_attention_q8(ctypes.byref(_attn(sbd, block_k=33)), *[A] * 10, None, 0, None) == \
        sbd.SBD_ERR_UNSUPPORTED


# ------------------------------------------------------------------ verification

VERIFY = ("target_logits", "draft_logits", "parent", "token", "uniform", "gumbel")
OUT = ("path", "out_tokens", "logprob", "count")


def _call(sbd, desc, ins, tau, outs):
    return sbd.lib.sbd_verify_tree(ctypes.byref(desc) if desc else None, *ins, tau, *outs, None, 0, None)


@pytest.mark.parametrize("over,tau,status", [
    (dict(batch=-1), 1.0, 1), (dict(nodes=0), 1.0, 1), (dict(nodes=65), 1.0, 2), (dict(vocab=0), 1.0, 1), (dict(vocab=(1 << 24) + 1), 1.0, 2),
    (dict(dtype=2), 1.0, 1), (dict(batch=65536), 1.0, 2), ({}, -1.0, 1), ({}, float("nan"), 1), ({}, float("inf"), 1),
    ({}, 1e-7, 2), ({}, 2e6, 2),
])
def test_verify_rejects_bad_descriptors(sbd, over, tau, status):
    d = dict(batch=2, nodes=8, vocab=1000, dtype=sbd.SBD_DTYPE_BF16)
    d.update(over)
    p = [A + 4096 * i for i in range(10)]
    assert _call(sbd, sbd.VerifyDesc(**d), p[:6], tau, p[6:]) == status and sbd.lib.sbd_last_error() != b""
    assert sbd.lib.sbd_verify_tree_workspace_size(ctypes.byref(sbd.VerifyDesc(**d))) == 0


def test_verify_rejects_bad_pointers(sbd):
    d = sbd.VerifyDesc(2, 8, 1000, sbd.SBD_DTYPE_F32)
    good = [A + 4096 * i for i in range(10)]
    assert _call(sbd, None, good[:6], 1.0, good[6:]) == sbd.SBD_ERR_INVALID_ARG
    for i, name in enumerate(VERIFY + OUT):
        for bad in (None, A + 8):
            if bad is None and name == "draft_logits":
                continue
            p = list(good)
            p[i] = bad
            assert _call(sbd, d, p[:6], 1.0, p[6:]) == sbd.SBD_ERR_INVALID_ARG, name
            assert name.encode() in sbd.lib.sbd_last_error()
    for i, j in ((6, 2), (6, 3), (7, 2), (7, 3), (7, 6)):
        p = list(good)
        p[i] = good[j]
        assert _call(sbd, d, p[:6], 1.0, p[6:]) == sbd.SBD_ERR_INVALID_ARG
        assert b"other memory" in sbd.lib.sbd_last_error()
    assert _call(sbd, sbd.VerifyDesc(0, 8, 1000, 0), [None] * 6, 1.0, [None] * 4) == sbd.SBD_OK


# ------------------------------------------------------------------ append of a path

def _path(sbd, **over):
    d = dict(batch=4, nodes=16, n_kv_heads=8, head_dim=128, page_size=64, n_pages=10, max_new=64,
             dtype=sbd.SBD_DTYPE_BF16, k_batch_stride=16384, k_node_stride=1024, v_batch_stride=16384, v_node_stride=1024)
    d.update(over)
    return sbd.AppendPathDesc(**d)


@pytest.mark.parametrize("over,status", [
    (dict(batch=-1), 1), (dict(nodes=0), 1), (dict(nodes=65), 2), (dict(n_kv_heads=0), 1), (dict(head_dim=80), 2),
    (dict(dtype=3), 1), (dict(page_size=8), 2), (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 2), (dict(max_new=-1), 1),
    (dict(k_node_stride=1020), 2), (dict(v_batch_stride=4), 2), (dict(v_node_stride=-1024), 2), (dict(batch=65536), 2),
    (dict(dtype=0, k_batch_stride=1022), 2),
])
def test_append_path_rejects_bad_descriptors(sbd, over, status):
    d = _path(sbd, **over)
    assert sbd.lib.sbd_cache_append_path_q8(ctypes.byref(d), *[A] * 9, None) == status


def test_append_path_rejects_bad_pointers(sbd):
    f = sbd.lib.sbd_cache_append_path_q8
    assert f(None, *[A] * 9, None) == sbd.SBD_ERR_INVALID_ARG
    _pointers(f, sbd, _path(sbd), ("k_new", "v_new", "path", "new_start", "slot_map", "k_cache", "v_cache", "k_scale",
                                   "v_scale"), (None,))
    assert f(ctypes.byref(_path(sbd, batch=0)), *[None] * 9, None) == sbd.SBD_OK
    assert f(ctypes.byref(_path(sbd, max_new=0)), *[None] * 9, None) == sbd.SBD_OK


# ------------------------------------------------------------------ the binding

def test_binding_refuses_cpu_tensors(sbd):
    import torch
    i = torch.zeros(2, 3, dtype=torch.int32)
    x = torch.zeros(2, 3, 1, 64)
    c = torch.zeros(2, 1, 16, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 1)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_qk_norm_rope(x, x, x, i, s[0])
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_tree_attention_q8(x, c, c, s, s, i, i[:, 0], x, x, i)
    with pytest.raises(ValueError, match="parent"):
        sbd.sbd_tree_attention_q8(x, c, c, s, s, i, i[:, 0], x, x, None)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_verify_tree(x[:, :, 0], None, i, i, x[:, :, 0, 0], x[:, 0, 0], 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_cache_append_path_q8(x, x, i, i[0], i[0], c, c, s, s)


def test_binding_refuses_tensors_of_another_device(sbd, monkeypatch):
    import torch

    class Fake:
        device = torch.device("cuda:1")

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        sbd._need_here(x=None, y=Fake())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    sbd._need_here(x=None, y=Fake())
