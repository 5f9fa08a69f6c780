"""How far the logarithms of attention's sums and the weights that follow from them may be off: the bounds that include/httm.h states."""
import pytest
import torch

import paper_2511_21317_amd as httm
from mx4_util import PackedBatch
from test_gpu_attention_cached import Batch, D

pytestmark = pytest.mark.gpu

SUMS = 2.0 ** -8                  # of a logarithm in tiles of 256 rows: a weight rounded to bf16, half a step


@pytest.mark.parametrize("store", [Batch, PackedBatch])
def test_rows_that_see_one_key(store):
    """Beginnings of prompts in tiles of 256 rows: nothing averages out, the sum is the one weight as it was rounded.  Its logarithm is off by
    that, at most ln(1 + 2^-8) below or above; the key's score by sums of 64 products in fp32, shift and logarithm by a few steps of fp32."""
    B, n, H = 12, 700, 16
    b = store([n] * B, [n] * B, 0, H, H, 64, seed=2)
    lse, out = torch.empty(b.n, H, device="cuda"), torch.empty(b.n, H * D, dtype=torch.bfloat16, device="cuda")
    httm.attention_cached(b.q, None, None, b.cache, b.offsets, b.seq_lens, out, causal=True, workspace=b.ws, lse=lse)
    first = torch.tensor(b.off[:-1], device="cuda")
    q, k = b.q[first].double(), torch.stack([x[:, 0] for x in b.k]).double()          # [B, H, 64]
    score, size = (q * k).sum(-1) * 0.125, (q.abs() * k.abs()).sum(-1) * 0.125
    fp32 = 2.0 ** -17 * size + 2.0 ** -20 * score.abs()
    off = (lse[first].double() - score).abs()
    assert (off <= SUMS + fp32).all(), float((off / (SUMS + fp32)).max())
    # what such a row leaves with its key, alone: the same batch without the other tokens
    alone = store([1] * B, [1] * B, 0, H, H, 64, seed=2)
    alone.q.copy_(b.q[first])
    at, was = alone.cache.page_table[:, 0].long(), b.cache.page_table[:, 0].long()
    for name in ("k_pages",) if store is Batch else ("k_codes", "scales"):
        getattr(alone.cache, name)[at, :, 0] = getattr(b.cache, name)[was, :, 0]
    one = torch.zeros(B, H, alone.cache.page_table.shape[1] * 64, device="cuda")
    httm.cache_weigh(alone.q, lse[first].contiguous(), alone.cache, alone.offsets, alone.seq_lens, one, causal=True)
    assert ((one[:, :, 0].double() - 1).abs() <= torch.expm1(SUMS + 2 * fp32)).all()
