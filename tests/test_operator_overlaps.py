"""Outputs of the calls around the layer that lie over their sources: refused on the host, before any launch, where a row would be written that
another wave still reads.  The addresses here are made up; what is accepted runs on the GPU, on tensors."""
import ctypes as C

import pytest
import torch

import paper_2511_21317_amd as httm
from test_operator_refusals import INVALID, norm_rope, paged, rows

A = 1 << 20
FAR = 1 << 30
ROW = 128


def call_cached(q, o, n, H_q):
    return httm.lib().httm_attention_cached(C.byref(q), FAR, FAR, 7, C.byref(paged(k_pages=FAR, v_pages=FAR)), FAR, FAR, n, H_q, 64, 0.125, 0, o,
                                            FAR, 1 << 40, None)


def call_norm_rope(q, k, v, out, N=5, H=3, dtype=0):
    return httm.lib().httm_qk_norm_rope(C.byref(norm_rope()), *map(C.byref, (q, k, v)), dtype, FAR, N, H, H, 64, *out, None)


def call_append(q, k, v, q_out, n=5, H=3, dtype=0):
    return httm.lib().httm_cache_append(C.byref(norm_rope()), *map(C.byref, (q, k, v)), dtype, FAR, 0, n, H, 64,
                                        C.byref(paged(H_kv=H, k_pages=FAR, v_pages=FAR)), FAR, FAR, q_out, None)


DENSE = rows(data=A, token_stride=3 * 64, head_stride=64)            # [5, 3, 64]
HEADWISE = rows(data=A, token_stride=64, head_stride=5 * 64)         # [3, 5, 64]
ELSEWHERE = rows(data=2 * FAR, token_stride=3 * 64, head_stride=64)
SIZE = 5 * 3 * ROW


@pytest.mark.parametrize("q,o", [
    (DENSE, A), (HEADWISE, A), (DENSE, A + ROW), (DENSE, A - SIZE + 16), (DENSE, A + SIZE - 16), (rows(data=A, token_stride=0, head_stride=0), A),
    # rows far apart: over the last token's last head, and over one in between
    (rows(data=A, token_stride=1 << 14, head_stride=1 << 10), A + 4 * (1 << 15) + 2 * (1 << 11) + ROW - 16),
    (rows(data=A, token_stride=1 << 10, head_stride=1 << 14), A + 1 * (1 << 15) + 3 * (1 << 11) - SIZE + 16)])
def test_attention(q, o):
    assert call_cached(q, o, 5, 3) == INVALID


@pytest.mark.parametrize("q,k,v,out,dtype", [
    (DENSE, ELSEWHERE, ELSEWHERE, (A, 3 * FAR, 4 * FAR), 0), (DENSE, ELSEWHERE, ELSEWHERE, (5 * FAR, A, 4 * FAR), 0),
    (ELSEWHERE, DENSE, ELSEWHERE, (5 * FAR, 3 * FAR, A + SIZE - 16), 0),
    (HEADWISE, ELSEWHERE, ELSEWHERE, (A + ROW, 3 * FAR, 4 * FAR), 0), (HEADWISE, ELSEWHERE, ELSEWHERE, (A, 3 * FAR, 4 * FAR), 1),
    (HEADWISE, ELSEWHERE, ELSEWHERE, (A, 3 * FAR, 4 * FAR), 2), (HEADWISE, HEADWISE, ELSEWHERE, (A, 3 * FAR, 4 * FAR), 0),
    (ELSEWHERE, ELSEWHERE, ELSEWHERE, (5 * FAR, 5 * FAR + SIZE - 16, 4 * FAR), 0)])
def test_norm_rope(q, k, v, out, dtype):
    assert call_norm_rope(q, k, v, out, dtype=dtype) == INVALID


@pytest.mark.parametrize("q,k,v,q_out,dtype", [
    (HEADWISE, ELSEWHERE, ELSEWHERE, A, 0), (ELSEWHERE, DENSE, ELSEWHERE, A, 0), (ELSEWHERE, ELSEWHERE, DENSE, A + 16, 0),
    (DENSE, ELSEWHERE, ELSEWHERE, A + 3 * ROW, 0), (DENSE, ELSEWHERE, ELSEWHERE, A, 1), (DENSE, DENSE, ELSEWHERE, A, 0)])
def test_append(q, k, v, q_out, dtype):
    assert call_append(q, k, v, q_out, dtype=dtype) == INVALID


def filled(shape, **kw):
    torch.manual_seed(sum(shape))
    return torch.randn(shape, device="cuda").to(torch.bfloat16, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("N,H", [(1, 3), (5, 1), (1003, 5), (4001, 11)])
def test_rows_may_become_what_is_made_of_them(N, H):
    nr = httm.NormRope(norm="layer", axes=1, base=100.0)
    pos = torch.arange(N, device="cuda", dtype=torch.int32)[:, None].contiguous()
    q, k, v = (filled((H, N, 64)) + i for i in range(3))
    want = [torch.empty_like(q) for _ in range(3)]
    httm.qk_norm_rope(nr, *(t.transpose(0, 1) for t in (q, k, v)), pos, *want)
    tokenwise = torch.empty(N, H, 64, dtype=torch.bfloat16, device="cuda").copy_(q.transpose(0, 1))
    httm.qk_norm_rope(nr, *(t.transpose(0, 1) for t in (q, k, v)), pos, q, k, v)
    assert all(torch.equal(a, b) for a, b in zip((q, k, v), want))
    cache = httm.PagedCache(*(torch.zeros(-(-N // 16), H, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                            torch.arange(-(-N // 16), dtype=torch.int32, device="cuda")[None].contiguous())
    off, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, N], [N]))
    httm.cache_append(nr, tokenwise, k.transpose(0, 1), v.transpose(0, 1), pos, cache, off, lens, tokenwise)
    assert torch.equal(tokenwise.transpose(0, 1), want[0])


@pytest.mark.gpu
def test_outputs_between_rows_are_taken():
    """An output in the room that strided rows leave: behind the tokens of each head, or behind the heads of the one token."""
    n, H = 6, 2
    wide = filled((H, 64, 64))                      # room for 64 tokens a head
    q, out = wide[:, :n].transpose(0, 1), wide[0, 8:8 + n * H].view(n, H * 64)
    off, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, n], [n]))
    cache = httm.PagedCache(filled((1, H, 16, 64)), filled((1, H, 16, 64)), torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    ws = torch.empty(httm.attention_cached_workspace(n, 1, H, H, 0), dtype=torch.uint8, device="cuda")
    want = httm.attention_cached(q.contiguous(), None, None, cache, off, lens, torch.empty(n, H * 64, dtype=torch.bfloat16, device="cuda"), workspace=ws)
    httm.attention_cached(q, None, None, cache, off, lens, out, workspace=ws)
    assert torch.equal(out, want)
    with pytest.raises(httm.HttmError):
        httm.attention_cached(q, None, None, cache, off, lens, wide[0, 3:3 + n * H].view(n, H * 64), workspace=ws)
    dense = q.contiguous()
    with pytest.raises(httm.HttmError):
        httm.attention_cached(dense, None, None, cache, off, lens, dense.view(n, H * 64), workspace=ws)
