"""The example of a serving loop over the paged 8-bit cache: blocks tables, append,
attention, head and select of uneven requests that end and are replaced."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_decode", os.path.join(ROOT, "examples", "paged_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _cached(dec, b):
    """Keys and values of request b in the cache, [len, Hkv, D]."""
    import torch
    n, table = int(dec.length[b]), dec.table.cpu().numpy()[b]
    out = []
    for w in range(2):
        codes, scale = dec.cache[w].view(torch.uint8).cpu().numpy(), dec.scale[w].cpu().numpy()
        out.append(po.paged_keys(codes, scale, table, n, dec.page))
    return out


@pytest.mark.parametrize("k,page,head_dim", [(8, 16, 64), (16, 64, 128)])
def test_paged_decode(example, k, page, head_dim):
    import torch
    rng = np.random.default_rng(k)
    lens = [5, 130, 0, 64, 77]
    dec = example.PagedDecoder(5, n_pages=64, max_pages=24, page=page, k=k, head_dim=head_dim)
    text = {b: torch.from_numpy(rng.integers(0, dec.vocab, n).astype(np.int32)) for b, n in enumerate(lens) if n}
    assert dec.admit(text).tolist() == [True, True, False, True, True]
    text = {b: [t] for b, t in text.items()}
    pages = lambda: int((dec.table >= 0).sum())  # noqa: E731
    for block in range(4):
        if block == 2:                               # one ends, one comes
            dec.finish([1])
            del text[1]
            new = torch.from_numpy(rng.integers(0, dec.vocab, 40).astype(np.int32))
            dec.last[2] = new[-k:].cuda()            # its last tokens are the block before its first
            assert bool(dec.admit({2: new[:-k]})[2])
            text[2] = [new]
        tokens = dec.decode_block()
        assert int(tokens.min()) >= 0 and int(tokens.max()) < dec.vocab
        for b in text:
            text[b].append(tokens[b].cpu())
        assert int(dec.n_free) + pages() == 64
        held = dec.free[:int(dec.n_free)].tolist() + dec.table[dec.table >= 0].tolist()
        assert sorted(held) == list(range(64))
    q, kv, d = dec.heads
    for b, parts in text.items():
        seq = torch.cat(parts).cuda()
        assert int(dec.length[b]) == len(seq) - k    # the last block is not in the cache yet
        _, qkv = dec._project(seq[:-k], torch.arange(len(seq) - k, device="cuda"))
        want = [qkv[:, q:q + kv].float().cpu().numpy(), qkv[:, q + kv:].float().cpu().numpy()]
        for got, ref in zip(_cached(dec, b), want):
            # One rounding to 4 bits (scales grow by powers of two, which leaves codes as they are) and one
            # to 8 that the projection's order of sums may turn; below the codes' range half a step of
            # 2^-9 s, s < 2^-7.8 of the largest, for each of at most five times a page is written to.
            top = np.abs(ref).max(axis=(0, 2))[:, None, None]
            ref = ref.transpose(1, 0, 2)
            assert (np.abs(got - ref) <= (2.0 ** -4 + 2.0 ** -7) * np.abs(ref) + 2.0 ** -15 * top).all()
    assert example.sbd.sbd_device_error() == 0


def test_paged_decode_refuses_a_prompt_without_pages(example):
    import torch
    dec = example.PagedDecoder(2, n_pages=4, max_pages=8, page=16)
    taken = dec.admit({0: torch.zeros(48, dtype=torch.int32), 1: torch.zeros(32, dtype=torch.int32)})
    assert taken.tolist() == [True, False] and dec.length.tolist() == [48, 0] and int(dec.n_free) == 1
    assert dec.decode_block().min() >= 0
