"""How far the logarithms of attention's sums, the weights that follow from them and rows in 4 bits may be off: the bounds that include/httm.h states."""
import math

import pytest
import torch

import paper_2511_21317_amd as httm
from mx4_util import PackedBatch
from test_gpu_attention_cached import Batch, D

pytestmark = pytest.mark.gpu

SUMS = 2.0 ** -8                  # of a logarithm in tiles of 256 rows: a weight rounded to bf16, half a step
LARGEST = 1 / 5                   # of a value above its block's unit: 5 units become 4


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


def test_values_in_4_bits():
    """Blocks whose largest value goes over a whole octave in 2^-12 steps, and ends on every border."""
    m = torch.cat([1 + torch.arange(4096, device="cuda") / 4096, torch.tensor([1.25, 1.75, 1.125, 1.5], device="cuda")])
    n = m.numel()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = m[:, None] * (2 * torch.rand((n, D), generator=g, device="cuda") - 1)
    x[:, 7], x[:, 40] = m, -m
    x = (x * 2.0 ** torch.randint(-20, 20, (n, 1), generator=g, device="cuda"))[:, None].contiguous()
    codes = [torch.zeros(-(-n // 256), 1, 256, 32, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.arange(-(-n // 256), dtype=torch.int32, device="cuda")[None].contiguous()
    cache = httm.PackedCache(*codes, torch.zeros(-(-n // 256), 1, 256, 4, dtype=torch.uint8, device="cuda"), table)
    off, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, n], [n]))
    httm.cache_append(httm.NormRope(norm="none", axes=0), None, x, x, None, cache, off, lens, None)
    k, v = (torch.empty(n, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    httm.cache_read(cache, off, lens, k, v)
    unit = 2.0 ** (cache.scales.flatten(0, 2)[:n, 0::2].double() - 127).repeat_interleave(32, -1)
    x, k = x[:, 0].double(), k[:, 0].double()
    off = (k - x).abs()
    assert (off <= LARGEST * x.abs())[x.abs() >= unit].all() and (off <= 0.25 * unit)[x.abs() <= 2 * unit].all()
    assert math.isclose(float((off / x.abs())[:, [7, 40]].max()), LARGEST)         # 5 units, a tie: the even code is that of 4
