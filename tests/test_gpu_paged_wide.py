"""The paged cache's calls at the far end of what they accept: 32-bit places that the
next step would leave."""
import numpy as np
import pytest

from test_gpu_paged import _i32, sbd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,k,P,clamped", [("float32", 15, 16, False), ("bfloat16", 15, 16, True), ("float32", 1, 128, True)])
def test_attention_over_the_longest_table(sbd, dtype, k, P, clamped):  # noqa: F811
    """A request of as many keys as a block table has places for, 2^31 - 1 with the
    block's (or one whose length is clamped to that).  All of its pages are one and the
    same but the last, whose keys outweigh the others by e^128: the result is the mean
    of the last page's values."""
    import torch
    D, cols = 64, (1 << 31) // P - 1
    table = torch.zeros(1, cols, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    kc = torch.zeros(2, 1, P, D, device="cuda")
    kc[1] = 1.0
    vc = torch.full((2, 1, P, D), 7.0, device="cuda")
    want = torch.arange(D, device="cuda") % 8 + 0.5
    vc[1, 0] = torch.arange(D, device="cuda") % 8 + (torch.arange(P, device="cuda") % 2)[:, None]
    one = torch.ones(2, 1, device="cuda")
    dt = getattr(torch, dtype)
    q = torch.full((1, k, 1, D), 16.0, device="cuda", dtype=dt)
    block = torch.zeros(1, k, 1, D, device="cuda", dtype=dt)
    f8 = torch.float8_e4m3fn
    length = (1 << 31) - 1 if clamped else cols * P
    out = sbd.sbd_block_attention_q8(q, kc.to(f8), vc.to(f8), one, one, table, _i32([length]), block, block - 3)
    assert sbd.sbd_device_error() == (sbd.SBD_DEVERR_CACHE_LEN if clamped else 0)
    # the weights of the last page are equal, their sum and the products exact in either type
    assert (out.float() - want).abs().max().item() <= 1e-5


def test_append_of_as_many_tokens_as_there_are_places(sbd):  # noqa: F811
    """2^31 - 1 tokens (one row of memory, a stride of 0) of which the last three are stored."""
    import torch
    T = (1 << 31) - 1
    slots = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    slots[-3:] = torch.arange(16, 19, dtype=torch.int32, device="cuda")
    row = torch.arange(64, device="cuda").bfloat16().view(1, 1, 64)
    codes = [torch.zeros(2, 1, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(2, 1, device="cuda") for _ in range(2)]
    sbd.sbd_cache_append_q8(row.expand(T, 1, 64), (-row).expand(T, 1, 64), slots, *codes, *scales)
    assert sbd.sbd_device_error() == 0
    want = (row.float() * 4).to(torch.float8_e4m3fn).float().view(64) / 4       # 63 <= 448 / 4, > 448 / 8
    for c, s, sign in zip(codes, scales, (1, -1)):
        assert s.tolist() == [[0.0], [0.25]]
        v = c.float() * 0.25
        assert (v[1, 0, :3] == sign * want).all() and (v[1, 0, 3:] == 0).all() and (v[0] == 0).all()


def test_tables_that_give_back_nearly_all_places(sbd):  # noqa: F811
    """4096 requests of 524287 pages each end at once: 2^31 - 4096 pages, more than the
    stack has room for, which is told; what fits is on it in order."""
    import torch
    B, cols, n_pages = 4096, (1 << 19) - 1, 1024
    table = torch.zeros(B, cols, dtype=torch.int32, device="cuda")
    table[-1, -n_pages:] = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), 16 * cols, dtype=torch.int32, device="cuda")
    free = torch.full((n_pages,), -5, dtype=torch.int32, device="cuda")
    out = sbd.sbd_block_tables(lens, torch.zeros_like(lens), table, free, _i32([0]), 16, 0)
    assert sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
    assert out[0].max().item() == -1 and out[0].min().item() == -1 and (out[1] == 0).all()
    assert out[4].item() == n_pages
    assert (free == torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device="cuda")).all()
