"""Attention to a cache in 4 bits, and the logarithms of sums over either kind: every key counts once, exactly.  All weights are equal (q = 0), the
values mark 8192 keys at a time, 128 in a channel, and a logarithm is that of the number of keys that the row sees."""
import pytest
import torch

import paper_2511_21317_amd as httm
from mx4_util import PackedBatch, pack
from test_gpu_attention_cached import SHAPES, Batch, D, spread
from test_gpu_attention_cached_coverage import WINDOW, marks, own_rows, seen_of_window

pytestmark = pytest.mark.gpu

# long own rows behind a prefix that has a launch of its own, by the room in the page table
APART = {"apart, streams": ([1] * 30, spread(0, 9000, 30), 3607, 8, 4, 64), "apart, drafts": ([3, 1, 5, 2, 4] * 4, spread(5, 20000, 20), 6201, 8, 4, 64),
         "apart, pieces": ([2, 0, 30] * 8, spread(0, 12000, 24), 9001, 8, 4, 64)}
ALL = {**SHAPES, **APART}


def seen(b, causal):
    """How many keys every token sees: the first of prefix and own rows."""
    m = torch.zeros(b.n, dtype=torch.int64, device="cuda")
    for i, (n, length) in enumerate(zip(b.new, b.lens)):
        own = (length - n + 1 + torch.arange(n, device="cuda")).clamp(0, length) if causal else torch.full((n,), length, device="cuda")
        m[b.off[i]:b.off[i + 1]] = b.P + own
    return m


def run(b, causal):
    out, lse = torch.full((b.n, b.H_q * D), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((b.n, b.H_q), 5.0, device="cuda")
    httm.attention_cached(b.q, b.kp if b.P else None, b.vp if b.P else None, b.cache, b.offsets, b.seq_lens, out, causal=causal, workspace=b.ws, lse=lse)
    return out.double().view(b.n, b.H_q, D), lse


def check_counts(lse, b, m):
    """ln m: of a sum that is a whole number, by a logarithm in base 2 and a product, 2^-23 of the value each and 2^-22 beside it; one key of 50 000 is 2e-5"""
    assert (lse[:b.off[0]] == 5).all() and (lse[b.off[-1]:] == 5).all()
    real = slice(b.off[0], b.off[-1])
    got, m = lse[real].double(), m[real, None].expand(-1, b.H_q)
    assert torch.equal(got == -float("inf"), m == 0)
    ref = torch.log(m.clamp(min=1).double())
    off = torch.where(m == 0, 0.0, (got - ref).abs())
    tol = 2.0 ** -22 * (ref + 1)
    assert m.numel() == 0 or float((1.0 / m.clamp(min=1)).min()) > 2 * float(tol.max())
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", ALL, ids=lambda s: s.replace(" ", "_").replace(",", ""))
def test_every_key_counts_once(shape, causal):
    b = PackedBatch(*ALL[shape], seed=1, pad_front=3, pad=4)
    if shape in APART:
        assert b.cache.page_table.numel() * b.cache.page_size * b.H_kv > 1000000
    b.q.zero_()
    page, row, key = own_rows(b)
    m = seen(b, causal)
    real = slice(b.off[0], b.off[-1])
    for start in range(0, max(1, b.P + max(b.lens)), WINDOW):
        b.vp[:] = marks(torch.arange(b.P, device="cuda"), start)
        codes, e = pack(marks(key, start))          # ones and zeros: exact
        b.cache.v_codes[page, :, row] = codes[:, None]
        b.cache.scales[page, :, row, 1], b.cache.scales[page, :, row, 3] = e[:, None, 0], e[:, None, 1]
        got, lse = run(b, causal)
        assert (got[:b.off[0]] == 5).all() and (got[b.off[-1]:] == 5).all()
        ref = (seen_of_window(m, start).double() / m.clamp(min=1)[:, None].double())[real, None]
        # weights are 1 and sums whole numbers; a reciprocal and a product in fp32, half a bf16 step of the result
        bad = (got[real] - ref).abs() > ref * (2.0 ** -8 + 2.0 ** -21)
        assert not bad.any(), f"keys from {start}: {int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}"
        check_counts(lse, b, m)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.replace(" ", "_").replace(",", ""))
def test_logarithms_over_a_cache_in_16_bits(shape, causal):
    b = Batch(*SHAPES[shape], seed=1, pad_front=3, pad=4)
    b.q.zero_()
    check_counts(run(b, causal)[1], b, seen(b, causal))
