"""sbd_block_tables with page ids out of range: in the free stack, in a page that
a request keeps, in one that it gives back.  Such an id becomes -1 wherever the
call writes it, its tokens get slot -1, and SBD_DEVERR_PAGE is set; nothing else
changes.  Among the ids are some whose slot wraps into the cache in 32 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

BAD = [-1, 8, 10 ** 6, (1 << 28) + 3, 1 << 27, -(1 << 31), (1 << 31) - 1, -(1 << 28) + 3]


@pytest.fixture(scope="module")
def sbd():
    import paper_2509_04185_gb300 as m
    return m


def _i32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def _call(sbd, lens, target, table, free, n_free, max_new):
    """Pages of 16 tokens, 8 of them; the five outputs and the stack as lists."""
    f = _i32(free + [0] * (8 - len(free)))
    out = sbd.sbd_block_tables(_i32(lens), _i32(target), _i32(table), f, _i32([n_free]), 16, max_new)
    return [x.tolist() for x in out] + [f.tolist()], sbd.sbd_device_error()


@pytest.mark.parametrize("bad", BAD)
def test_in_the_free_stack(sbd, bad):
    (table, length, start, slots, n_free, _), err = _call(sbd, [0, 0], [16, 20], [[-1, -1]] * 2, [7, 2, bad, 5], 4, 36)
    assert table == [[5, -1], [-1, 2]] and length == [16, 20] and start == [0, 16, 36] and n_free == [1]
    assert slots == list(range(80, 96)) + [-1] * 16 + list(range(32, 36))
    assert err == sbd.SBD_DEVERR_PAGE


@pytest.mark.parametrize("bad", BAD)
def test_in_a_kept_page(sbd, bad):
    (table, length, _, slots, n_free, _), err = _call(sbd, [20, 3], [34, 5], [[1, bad, -1], [6, -1, -1]], [4, 3], 2, 16)
    assert table == [[1, -1, 3], [6, -1, -1]] and length == [34, 5] and n_free == [1]
    assert slots == [-1] * 12 + [48, 49, 99, 100]
    assert err == sbd.SBD_DEVERR_PAGE
    # a request that gains nothing
    (table, length, _, _, _, _), err = _call(sbd, [20, 3], [20, 3], [[1, bad], [6, -1]], [4, 3], 2, 0)
    assert table == [[1, -1], [6, -1]] and length == [20, 3] and err == sbd.SBD_DEVERR_PAGE


@pytest.mark.parametrize("bad", BAD)
def test_in_a_released_page(sbd, bad):
    # pages 3 and `bad` go back, the first one topmost
    (table, length, _, _, n_free, free), err = _call(sbd, [44], [10], [[1, 3, bad]], [7], 1, 0)
    assert table == [[1, -1, -1]] and length == [10] and n_free == [3]
    assert free[:3] == [7, -1, 3] and err == sbd.SBD_DEVERR_PAGE
    # and is granted in the same call
    (table, length, _, slots, n_free, _), err = _call(sbd, [32, 0, 0], [10, 5, 2], [[1, bad], [-1, -1], [-1, -1]], [7], 1, 7)
    assert table == [[1, -1], [-1, -1], [7, -1]] and length == [10, 5, 2] and n_free == [0]
    assert slots == [-1] * 5 + [112, 113] and err == sbd.SBD_DEVERR_PAGE


def test_ids_that_are_not_used_do_not_matter(sbd):
    """Past a request's pages and above the top of the stack anything may stand."""
    (table, length, _, slots, n_free, _), err = _call(sbd, [20, 16], [25, 17], [[1, 2, 99], [6, -7, 1 << 30]], [4, 3, 500, -9], 2, 6)
    assert table == [[1, 2, -1], [6, 3, -1]] and length == [25, 17] and n_free == [1]
    assert slots == [36, 37, 38, 39, 40, 48] and err == 0


def test_in_large_tables(sbd):
    """One bad id among many: of 300 requests and of a request of 3,000 pages."""
    rng = np.random.default_rng(0)
    for B, cols, page in ((300, 10, 32), (1, 3100, 16)):
        n_pages = 2 * B * cols
        perm = rng.permutation(n_pages).astype(np.int32)
        held = cols - 3
        table = np.full((B, cols), -1, np.int32)
        table[:, :held] = perm[:B * held].reshape(B, held)
        free = np.zeros(n_pages, np.int32)
        free[:n_pages - B * held] = perm[B * held:]
        lens, target = np.full(B, held * page - 1), np.full(B, held * page + page)
        for where in ("kept", "granted"):
            t, f = table.copy(), free.copy()
            if where == "kept":
                t[B // 2, held - 1] = n_pages
            else:
                f[n_pages - B * held - 1 - B // 2] = -3          # of request B // 2
            out = sbd.sbd_block_tables(_i32(lens), _i32(target), _i32(t), _i32(f), _i32([n_pages - B * held]), page, B * (page + 1))
            assert sbd.sbd_device_error() == sbd.SBD_DEVERR_PAGE
            got, slots = out[0].cpu().numpy(), out[3].cpu().numpy().reshape(B, page + 1)
            want = t.copy()
            want[:, held] = f[n_pages - B * held - 1 - np.arange(B)]
            want[B // 2, held - 1 if where == "kept" else held] = -1
            assert (got == want).all()
            ref = np.concatenate([(want[:, held - 1] * page + page - 1)[:, None], want[:, held, None] * page + np.arange(page)], 1)
            if where == "kept":
                ref[B // 2, 0] = -1
            else:
                ref[B // 2, 1:] = -1
            assert (slots == ref).all()
