"""The paged cache's calls reject bad arguments on the host, before anything is
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


def _attn(sbd, **over):
    d = dict(batch=1, block_k=16, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=64, max_pages=64,
             n_pages=100, dtype=sbd.SBD_DTYPE_BF16, n_causal=0, scale=0.0, num_splits=0)
    d.update(over)
    return sbd.AttnQ8Desc(**d)


@pytest.mark.parametrize("over,status", [
    (dict(batch=-1), 1), (dict(block_k=0), 1), (dict(block_k=33), 2), (dict(head_dim=96), 2), (dict(head_dim=0), 1),
    (dict(n_q_heads=30), 1), (dict(n_kv_heads=0), 1), (dict(dtype=5), 1), (dict(page_size=48), 2),
    (dict(page_size=0), 1), (dict(page_size=256), 2), (dict(max_pages=0), 1), (dict(n_pages=0), 1),
    (dict(n_pages=1 << 25), 2), (dict(max_pages=1 << 25), 2), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(n_causal=-1), 1), (dict(n_causal=17), 1), (dict(num_splits=-1), 1), (dict(batch=1 << 17), 2),
    (dict(n_q_heads=8192), 2),
])
def test_attention_rejects_bad_descriptors(sbd, over, status):
    d = _attn(sbd, **over)
    st = sbd.lib.sbd_block_attention_q8(ctypes.byref(d), *[A] * 10, None, 0, None)
    assert st == status and sbd.lib.sbd_last_error() != b""
    assert sbd.lib.sbd_block_attention_q8_workspace_size(ctypes.byref(d)) == 0


def test_attention_rejects_bad_pointers(sbd):
    d = _attn(sbd)
    f = sbd.lib.sbd_block_attention_q8
    assert f(None, *[A] * 10, None, 0, None) == sbd.SBD_ERR_INVALID_ARG
    names = ("q", "k_cache", "v_cache", "k_scale", "v_scale", "block_table", "cache_len", "k_blk", "v_blk", "out")
    for i, name in enumerate(names):
        for bad in (None, A + 4):
            ptrs = [A] * 10
            ptrs[i] = bad
            assert f(ctypes.byref(d), *ptrs, None, 0, None) == sbd.SBD_ERR_INVALID_ARG
            assert name.encode() in sbd.lib.sbd_last_error()
    assert f(ctypes.byref(_attn(sbd, batch=0)), *[None] * 10, None, 0, None) == sbd.SBD_OK


def _append(sbd, **over):
    d = dict(tokens=16, group=16, n_kv_heads=8, head_dim=128, page_size=64, n_pages=10, dtype=sbd.SBD_DTYPE_BF16,
             k_group_stride=0, k_token_stride=1024, v_group_stride=0, v_token_stride=1024)
    d.update(over)
    return sbd.AppendQ8Desc(**d)


@pytest.mark.parametrize("over,status", [
    (dict(tokens=-1), 1), (dict(group=0), 1), (dict(n_kv_heads=0), 1), (dict(head_dim=80), 2), (dict(dtype=3), 1),
    (dict(page_size=8), 2), (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 2), (dict(k_token_stride=1020), 2),
    (dict(v_group_stride=4), 2), (dict(v_token_stride=-1024), 2), (dict(dtype=0, k_token_stride=1022), 2),
])
def test_append_rejects_bad_descriptors(sbd, over, status):
    d = _append(sbd, **over)
    assert sbd.lib.sbd_cache_append_q8(ctypes.byref(d), *[A] * 7, None) == status


def test_append_rejects_bad_pointers(sbd):
    f = sbd.lib.sbd_cache_append_q8
    assert f(None, *[A] * 7, None) == sbd.SBD_ERR_INVALID_ARG
    for i, name in enumerate(("k_new", "v_new", "slot_map", "k_cache", "v_cache", "k_scale", "v_scale")):
        for bad in (None, A + 8):
            ptrs = [A] * 7
            ptrs[i] = bad
            assert f(ctypes.byref(_append(sbd)), *ptrs, None) == sbd.SBD_ERR_INVALID_ARG
            assert name.encode() in sbd.lib.sbd_last_error()
    assert f(ctypes.byref(_append(sbd, tokens=0)), *[None] * 7, None) == sbd.SBD_OK


@pytest.mark.parametrize("over,status", [
    (dict(batch=0), 1), (dict(batch=5000), 2), (dict(page_size=20), 2), (dict(max_pages=0), 1), (dict(n_pages=0), 1),
    (dict(max_new=-1), 1), (dict(batch=4096, max_pages=1 << 20), 2), (dict(max_pages=1 << 26), 2),
])
def test_tables_reject_bad_descriptors(sbd, over, status):
    d = dict(batch=4, page_size=64, max_pages=10, n_pages=100, max_new=8)
    d.update(over)
    ptrs = [A + 4096 * i for i in range(10)]
    assert sbd.lib.sbd_block_tables(ctypes.byref(sbd.TablesDesc(**d)), *ptrs, None) == status


def test_tables_reject_bad_pointers(sbd):
    f = sbd.lib.sbd_block_tables
    d = sbd.TablesDesc(4, 64, 10, 100, 8)
    good = [A + 4096 * i for i in range(10)]
    assert f(None, *good, None) == sbd.SBD_ERR_INVALID_ARG
    for i, name in enumerate(("cache_len", "target_len", "block_table", "free_pages", "n_free", "block_table_out",
                              "len_out", "new_start", "slot_map", "n_free_out")):
        for bad in (None, good[i] + 4):
            ptrs = list(good)
            ptrs[i] = bad
            assert f(ctypes.byref(d), *ptrs, None) == sbd.SBD_ERR_INVALID_ARG
            assert name.encode() in sbd.lib.sbd_last_error()
    for i, j in ((5, 2), (6, 0), (6, 1), (9, 4)):      # an output over an input
        ptrs = list(good)
        ptrs[i] = good[j]
        assert f(ctypes.byref(d), *ptrs, None) == sbd.SBD_ERR_INVALID_ARG


def test_binding_refuses_cpu_tensors(sbd):
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_block_tables(i, i, torch.zeros(2, 3, dtype=torch.int32), i, i[:1], 16, 4)
    c = torch.zeros(2, 1, 16, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 1)
    x = torch.zeros(1, 1, 64)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_cache_append_q8(x, x, i, c, c, s, s)
    with pytest.raises(ValueError, match="CUDA"):
        sbd.sbd_block_attention_q8(x[None], c, c, s, s, i[None], i[:1], x[None], x[None])
