"""Numbers that do not fit the C side's types are refused, not taken modulo 2^32 or 2^64."""
import pytest
import torch

import paper_2511_21317_amd as httm


@pytest.mark.parametrize("at", range(5))
@pytest.mark.parametrize("more", [1 << 31, 1 << 32, 1 << 64, -1 << 32, -1 << 64])
def test_workspace(at, more):
    sizes = [5, 2, 1, 1, 7]
    sizes[at] += more
    with pytest.raises(httm.HttmError):
        httm.attention_cached_workspace(*sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("first", [-1, 1 << 31, 1 << 32, 1 << 64, (1 << 64) + 3])
def test_first_position(first):
    x, pages = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 2, 64), (3, 2, 16, 64)))
    table, off, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([[0, 1, 2]], [0, 4], [4]))
    cache = httm.PagedCache(pages, pages.clone(), table)
    with pytest.raises(httm.HttmError):
        httm.cache_append(httm.NormRope(norm="none", axes=1), None, x, x, None, cache, off, lens, None, first_pos=first)
    httm.cache_append(httm.NormRope(norm="none", axes=1), None, x, x, None, cache, off, lens, None, first_pos=(1 << 31) - 1)
