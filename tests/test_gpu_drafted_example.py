"""The drafted serving loop at its smallest: prompts of one token, and more than the cache holds."""
import pytest

from test_gpu_draft_turn import example  # noqa: F401
from test_gpu_paged import sbd  # noqa: F401

pytestmark = pytest.mark.gpu


def test_prompts_of_one_token(example, sbd):  # noqa: F811
    """Nothing enters the cache before the first turn."""
    import torch
    for lens in ([1, 1, 1], [1, 5, 1]):
        dec = example.DraftedDecoder(3, n_pages=6, max_pages=2, page=64, k=3)
        dec.admit([torch.arange(n, dtype=torch.int32) for n in lens])
        assert dec.length.tolist() == [n - 1 for n in lens] and dec.last.tolist() == [n - 1 for n in lens]
        for _ in range(2):
            before = dec.length.clone()
            tokens, count = dec.turn()
            assert (count >= 1).all() and torch.equal(dec.length, before + count)
            assert ((tokens >= 0) & (tokens < dec.vocab)).sum(1).tolist() == count.tolist()
    assert sbd.sbd_device_error() == 0


def test_prompts_that_find_no_pages(example, sbd):  # noqa: F811
    import torch
    dec = example.DraftedDecoder(2, n_pages=2, max_pages=4, page=16, k=3)
    with pytest.raises(RuntimeError, match="full"):
        dec.admit([torch.zeros(n, dtype=torch.int32) for n in (20, 30)])
    assert sbd.sbd_device_error() in (0, sbd.SBD_DEVERR_PAGE)
