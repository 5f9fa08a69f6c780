"""What the calls of the cache in 4 bits and of its budget refuse, on the host, before any launch: the addresses here are made up."""
import ctypes as C

import pytest
import torch

import paper_2511_21317_amd as httm
from test_operator_refusals import BAD_CACHES, INVALID, SMALL, UNSUPPORTED, norm_rope, paged, rows

# 10 pages of a head, 16 rows each: 5120 bytes of codes, 640 of scales, 20480 of bf16 rows
K, V, S, T = 1 << 20, 2 << 20, 3 << 20, 4 << 20
A, B, W, X = 5 << 20, 6 << 20, 7 << 20, 8 << 20


def packed(**kw):
    return paged(**{**dict(k_pages=K, v_pages=V, page_table=T), **kw})


def call_append(cache=None, scales=S, n=5, H_q=1, d_head=64, offsets=A, seq_lens=A, q_out=W, dtype=0, k=None):
    r = [rows(data=X), k or rows(data=X), rows(data=X)]
    return httm.lib().httm_cache_append_mx4(C.byref(norm_rope()), *map(C.byref, r), dtype, A, 0, n, H_q, d_head, C.byref(cache or packed()), scales,
                                            offsets, seq_lens, q_out, None)


def call_read(cache=None, scales=S, offsets=A, seq_lens=A, n=5, d_head=64, k_out=W, v_out=X):
    return httm.lib().httm_cache_read(C.byref(cache or packed()), scales, offsets, seq_lens, n, d_head, k_out, v_out, None)


def call_attention(cache=None, scales=S, q=None, n=5, H_q=1, lse=W, o=B, workspace=X, size=1 << 30, offsets=A, scale=0.125, P=0, d_head=64):
    return httm.lib().httm_attention_cached_lse(C.byref(q or rows(data=9 << 20)), None, None, P, C.byref(cache or packed()), scales, offsets, A, n,
                                                H_q, d_head, scale, 0, o, lse, workspace, size, None)


def call_weigh(cache=None, scales=S, q=None, lse=B, offsets=A, seq_lens=A, n=5, H_q=1, d_head=64, scale=0.125, decay=1.0, weights=W, columns=64):
    return httm.lib().httm_cache_weigh(C.byref(q or rows(data=9 << 20)), lse, C.byref(cache or packed()), scales, offsets, seq_lens, n, H_q, d_head,
                                       scale, 0, decay, weights, columns, None)


def call_evict(cache=None, scales=S, seq_lens=A, weights=W, columns=64, d_head=64, keep=32, first=1, last=2, new_lens=B, kept=X,
               workspace=9 << 20, size=1 << 30):
    return httm.lib().httm_cache_evict(C.byref(cache or packed()), scales, seq_lens, weights, columns, d_head, keep, first, last, new_lens, kept,
                                       workspace, size, None)


CALLS = [call_append, call_read, call_attention, call_weigh, call_evict]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
@pytest.mark.parametrize("call", CALLS)
def test_caches(call, kw, code):
    if call in (call_read, call_evict) and kw == dict(H_kv=2):
        return      # (nothing that has to be a multiple of it; the ranges are larger)
    assert call(cache=packed(**kw)) == code


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", [
    dict(scales=S + 4), dict(scales=K + 5120 - 16), dict(scales=V), dict(scales=K - 640 + 16), dict(cache=packed(v_pages=K + 5120 - 16)),
    dict(cache=packed(v_pages=K))])
def test_codes_and_scales_that_lie_over_each_other(call, kw):
    assert call(**kw) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(scales=None), INVALID), (dict(d_head=128), UNSUPPORTED), (dict(n=1 << 25), UNSUPPORTED), (dict(n=-1), INVALID), (dict(offsets=None), INVALID),
    (dict(seq_lens=A + 2), INVALID), (dict(q_out=None), INVALID), (dict(dtype=3), INVALID), (dict(k=rows(data=None)), INVALID), (dict(n=0), 0)])
def test_append(kw, code):
    assert call_append(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=32), UNSUPPORTED), (dict(n=1 << 25), UNSUPPORTED), (dict(n=-1), INVALID), (dict(offsets=None), INVALID), (dict(seq_lens=None), INVALID),
    (dict(offsets=A + 1), INVALID), (dict(k_out=None), INVALID), (dict(v_out=None), INVALID), (dict(k_out=W + 8), INVALID),
    (dict(v_out=W), INVALID), (dict(v_out=W + 5 * 128 - 16), INVALID), (dict(k_out=K + 16), INVALID), (dict(v_out=S - 16), INVALID),
    (dict(scales=None, v_out=V + 10000), INVALID), (dict(n=0, k_out=None, v_out=None), 0)])
def test_read(kw, code):
    assert call_read(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(lse=W + 2), INVALID), (dict(lse=B), INVALID), (dict(lse=B + 5 * 128 - 4), INVALID), (dict(lse=X + 256), INVALID), (dict(lse=9 << 20), INVALID),
    (dict(lse=K + 4), INVALID), (dict(lse=S), INVALID), (dict(q=rows(data=None)), INVALID), (dict(size=0), SMALL), (dict(scale=0.0), INVALID),
    (dict(n=1 << 20), UNSUPPORTED), (dict(d_head=128), UNSUPPORTED), (dict(P=3), INVALID), (dict(offsets=None), INVALID), (dict(n=0), 0)])
def test_attention(kw, code):
    assert call_attention(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=128), UNSUPPORTED), (dict(n=1 << 20), UNSUPPORTED), (dict(n=-1), INVALID), (dict(columns=63), INVALID), (dict(columns=1 << 31), INVALID),
    (dict(weights=None), INVALID), (dict(weights=W + 2), INVALID), (dict(lse=None), INVALID), (dict(lse=B + 1), INVALID), (dict(q=rows(data=None)), INVALID),
    (dict(q=rows(data=9 << 20, token_stride=4)), INVALID), (dict(offsets=None), INVALID), (dict(seq_lens=A + 3), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=-1.0), INVALID), (dict(decay=-0.5), INVALID), (dict(decay=float("inf")), INVALID), (dict(decay=float("nan")), INVALID),
    (dict(lse=W + 64 * 8 - 4), INVALID), (dict(q=rows(data=W)), INVALID), (dict(weights=K), INVALID), (dict(weights=S - 4), INVALID),
    (dict(scales=None, weights=K + 20000), INVALID)])
def test_weigh(kw, code):
    assert call_weigh(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=128), UNSUPPORTED), (dict(keep=0), INVALID), (dict(keep=-1), INVALID), (dict(first=-1), INVALID), (dict(last=-1), INVALID),
    (dict(keep=2), INVALID), (dict(first=33, last=0), INVALID), (dict(first=(1 << 63) - 1), INVALID), (dict(keep=(1 << 30) + 1, size=1 << 40), UNSUPPORTED),
    (dict(columns=63), INVALID), (dict(columns=1 << 31), INVALID), (dict(seq_lens=None), INVALID), (dict(new_lens=None), INVALID), (dict(weights=None), INVALID),
    (dict(workspace=None), INVALID), (dict(workspace=(9 << 20) + 16), INVALID), (dict(size=0), SMALL), (dict(kept=X + 2), INVALID),
    (dict(new_lens=A), INVALID), (dict(new_lens=A + 4), INVALID), (dict(kept=W), INVALID), (dict(weights=A - 4), INVALID), (dict(kept=9 << 20), INVALID),
    (dict(new_lens=T), INVALID), (dict(kept=T + 16), INVALID), (dict(weights=K), INVALID), (dict(kept=S), INVALID), (dict(new_lens=V + 5116), INVALID)])
def test_evict(kw, code):
    assert call_evict(**kw) == code


def test_workspace_is_what_the_call_asks_for():
    need = httm.cache_evict_workspace(2, 1, 32)
    assert need > 0 and call_evict(size=need - 1) == SMALL
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (4097, 1, 1), (1, 65, 1), (1, 1, (1 << 30) + 1), (1 << 32, 1, 1), (1, 1, 1 << 64), (-1, 1, 1)):
        with pytest.raises(httm.HttmError):
            httm.cache_evict_workspace(*bad)


class Cache:
    """What the calls read of a cache, which itself takes tensors on the GPU only."""
    H_kv, n_seqs, page_size, scales_at = 2, 1, 16, None


def test_the_binding_wants_tensors_and_wants_them_on_the_gpu():
    u8, i32 = torch.uint8, torch.int32
    codes, scales, table = torch.zeros(3, 2, 16, 32, dtype=u8), torch.zeros(3, 2, 16, 4, dtype=u8), torch.zeros(1, 3, dtype=i32)
    for bad in ((None, codes, scales, table), (codes, codes, scales, None), (codes, codes, scales, table), (scales, codes, scales, table)):
        with pytest.raises(httm.HttmError):
            httm.PackedCache(*bad)
    x, off, lens, w = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(1, 2, 48)
    for call in (lambda: httm.cache_read(Cache, off, lens, x, x), lambda: httm.cache_read(Cache, off, lens, None, x),
                 lambda: httm.cache_weigh(x, w, Cache, off, lens, w), lambda: httm.cache_weigh(None, w, Cache, off, lens, w),
                 lambda: httm.cache_evict(Cache, lens, w, 4, lens, workspace=codes), lambda: httm.cache_evict(Cache, None, w, 4, lens),
                 lambda: httm.cache_evict(Cache, lens, w, 1 << 31, lens), lambda: httm.cache_evict(Cache, lens, w, 4, lens, first=-1)):
        with pytest.raises(httm.HttmError):
            call()
