"""Paged attention whose splits are mostly empty, directly followed by a kernel that
takes tensor memory before it waits (sbd_linear), in turn and in a graph."""
import numpy as np
import pytest

import test_gpu_paged as tp
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k,D,Hq,lens", [(1, 128, 8, [0, 1, 5]), (8, 64, 8, [0, 300, 0]), (16, 128, 8, [3, 0, 0]),
                                         (32, 64, 8, [200, 0, 1]), (4, 64, 8, [0] * 60)])
def test_attention_and_linear_in_turn(sbd, k, D, Hq, lens):  # noqa: F811
    import torch
    rng = np.random.default_rng(k)
    q, codes, scales, table, lens, kb, vb = tp._attention_case(rng, len(lens), k, Hq, 2, D, 32, lens, extra_cols=200)
    dev = [torch.from_numpy(x.astype(np.float32)).bfloat16().cuda() for x in (q, kb, vb)]
    cache = [tp._f8(c) for c in codes] + [torch.from_numpy(s).cuda() for s in scales]
    table, lens = tp._i32(table), tp._i32(lens)
    w = torch.randn(512, Hq * D, device="cuda").bfloat16()
    rows = min(len(q) * k, 512)

    def turn():
        out = sbd.sbd_block_attention_q8(dev[0], *cache, table, lens, dev[1], dev[2], num_splits=16)
        return out, sbd.sbd_linear(out.view(-1, Hq * D)[:rows], w)

    out, y = turn()
    torch.cuda.synchronize()
    want = out.view(-1, Hq * D)[:rows].double() @ w.double().T
    assert (y.double() - want).norm() <= 2.0 ** -8 * want.norm()
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(100):
        o, z = turn()
        differ += (o != out).sum() + (z != y).sum()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(20):
            o, z = turn()
    for _ in range(5):
        graph.replay()
        differ += (o != out).sum() + (z != y).sum()
    assert differ.item() == 0 and sbd.sbd_device_error() == 0
