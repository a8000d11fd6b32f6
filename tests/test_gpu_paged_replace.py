"""The serving example where a request takes another one's place, and where a
running one finds no page: through admit(), decode_block() and finish() alone."""
import numpy as np
import pytest

from test_gpu_paged_example import _cached, example  # noqa: F401

pytestmark = pytest.mark.gpu


def _check_cache(dec, b, text, k):
    """What the cache holds of request b is what its text without the last block projects to
    (the bound of the example's own test)."""
    import torch
    seq = torch.cat(text).cuda()
    assert int(dec.length[b]) == len(seq) - k
    q, kv, _ = dec.heads
    _, qkv = dec._project(seq[:-k], torch.arange(len(seq) - k, device="cuda"))
    for got, ref in zip(_cached(dec, b), (qkv[:, q:q + kv], qkv[:, q + kv:])):
        ref = ref.float().cpu().numpy()
        top = np.abs(ref).max(axis=(0, 2))[:, None, None]
        ref = ref.transpose(1, 0, 2)
        assert (np.abs(got - ref) <= (2.0 ** -4 + 2.0 ** -7) * np.abs(ref) + 2.0 ** -15 * top).all()


def _check_pages(dec, n_pages):
    held = dec.free[:int(dec.n_free)].tolist() + dec.table[dec.table >= 0].tolist()
    assert sorted(held) == list(range(n_pages))


@pytest.mark.parametrize("k,page,new_len", [(8, 16, 40), (8, 32, 3), (16, 64, 100)])
def test_a_request_takes_the_place_of_an_ended_one(example, k, page, new_len):  # noqa: F811
    import torch
    rng = np.random.default_rng(k + page)
    mk = lambda n: torch.from_numpy(rng.integers(0, 2000, n).astype(np.int32))  # noqa: E731
    dec = example.PagedDecoder(4, n_pages=64, max_pages=24, page=page, k=k)
    text = {0: [mk(70)], 1: [mk(130)], 3: [mk(9)]}
    assert dec.admit({b: t[0] for b, t in text.items()}).tolist() == [True, True, False, True]
    for block in range(5):
        if block == 2:                               # in the place of one that ends
            dec.finish([1])
            text[1] = [mk(new_len)]
            assert bool(dec.admit({1: text[1][0]})[1])
        if block == 3:                               # in a place that was never taken
            text[2] = [mk(new_len + 1)]
            assert bool(dec.admit({2: text[2][0]})[2])
        tokens = dec.decode_block()
        for b in text:
            text[b].append(tokens[b].cpu())
        _check_pages(dec, 64)
    for b in text:
        _check_cache(dec, b, text[b], k)
    assert example.sbd.sbd_device_error() == 0


def test_a_running_request_that_finds_no_page_gives_its_pages_back(example):  # noqa: F811
    import torch
    k, page, n_pages = 8, 16, 5
    rng = np.random.default_rng(3)
    mk = lambda n: torch.from_numpy(rng.integers(0, 2000, n).astype(np.int32))  # noqa: E731
    dec = example.PagedDecoder(2, n_pages=n_pages, max_pages=8, page=page, k=k)
    text = {0: [mk(30)], 1: [mk(48)]}                # 2 and 3 pages: none is left
    assert dec.admit({b: t[0] for b, t in text.items()}).tolist() == [True, True]
    tokens = dec.decode_block()
    text[0].append(tokens[0].cpu())
    dec.decode_block()                               # both ask for a page and there is none
    assert dec.alive.tolist() == [False, False]
    assert dec.length.tolist() == [0, 0] and int(dec.n_free) == n_pages and (dec.table == -1).all()
    _check_pages(dec, n_pages)
    # their places and pages serve others
    text = {1: [mk(20)]}
    assert dec.admit({1: text[1][0]}).tolist() == [False, True]
    for _ in range(3):
        text[1].append(dec.decode_block()[1].cpu())
    _check_cache(dec, 1, text[1], k)
    assert example.sbd.sbd_device_error() == 0


def test_one_is_refused_and_the_others_go_on(example):  # noqa: F811
    import torch
    k, page, n_pages = 8, 16, 6
    rng = np.random.default_rng(4)
    mk = lambda n: torch.from_numpy(rng.integers(0, 2000, n).astype(np.int32))  # noqa: E731
    dec = example.PagedDecoder(3, n_pages=n_pages, max_pages=8, page=page, k=k)
    text = {0: [mk(16)], 1: [mk(32)], 2: [mk(17)]}   # 1, 2 and 2 pages, one is left
    assert dec.admit({b: t[0] for b, t in text.items()}).tolist() == [True, True, True]
    for _ in range(2):
        tokens = dec.decode_block()
        for b in text:
            text[b].append(tokens[b].cpu())
    # request 0 took the last page, request 1 found none, request 2 has room
    assert dec.alive.tolist() == [True, False, True] and dec.length.tolist() == [24, 0, 25]
    _check_pages(dec, n_pages)
    tokens = dec.decode_block()
    for b in (0, 2):
        text[b].append(tokens[b].cpu())
        _check_cache(dec, b, text[b], k)
    assert dec.alive.tolist() == [True, False, True]
    assert example.sbd.sbd_device_error() == 0


def test_a_running_request_is_not_taken_in_again(example):  # noqa: F811
    import torch
    dec = example.PagedDecoder(2, n_pages=8, max_pages=8, page=16)
    dec.admit({0: torch.zeros(20, dtype=torch.int32)})
    with pytest.raises(ValueError, match="running"):
        dec.admit({0: torch.zeros(40, dtype=torch.int32)})
    assert dec.length.tolist() == [20, 0]
