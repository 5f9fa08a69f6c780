"""A tensor that a call needs and does not get is refused as every other argument is: an HttmError, on the host."""
import pytest
import torch

import paper_2511_21317_amd as httm


class Cache:
    """What the calls read of a PagedCache, which itself takes tensors on the GPU only."""
    H_kv, n_seqs, page_size = 2, 1, 16


def test_new_tokens_need_keys_and_values():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    off, lens = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for q, k, v in ((x, None, x), (None, None, x), (None, None, None)):
        with pytest.raises(httm.HttmError):
            httm.cache_append(httm.NormRope(), q, k, v, None, Cache, off, lens, q)


def test_attention_needs_queries():
    off, lens = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(httm.HttmError):
        httm.attention_cached(None, None, None, Cache, off, lens, None, workspace=torch.zeros(256, dtype=torch.uint8))


def test_a_cache_needs_its_pages_and_its_table():
    pages, table = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 3, dtype=torch.int32)
    for missing in range(3):
        with pytest.raises(httm.HttmError):
            httm.PagedCache(*(None if i == missing else t for i, t in enumerate((pages, pages, table))))


@pytest.mark.gpu
def test_other_tensors_that_are_missing():
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, pages = torch.zeros(4, 2, 64, **bf), torch.zeros(3, 2, 16, 64, **bf)
    table, off, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([[0, 1, 2]], [0, 4], [4]))
    cache = httm.PagedCache(pages, pages.clone(), table)
    nr, out = httm.NormRope(norm="none", axes=0), torch.zeros(4, 128, **bf)
    ws = torch.empty(httm.attention_cached_workspace(4, 1, 2, 2, 0), dtype=torch.uint8, device="cuda")
    for o, n, y in ((None, lens, out), (off, None, out), (off, lens, None)):
        with pytest.raises(httm.HttmError):
            httm.attention_cached(x, None, None, cache, o, n, y, workspace=ws)
    for o, n in ((None, lens), (off, None)):
        with pytest.raises(httm.HttmError):
            httm.cache_append(nr, None, x, x, None, cache, o, n, None)
    with pytest.raises(httm.HttmError):
        httm.PagedCache(pages, None, table)
