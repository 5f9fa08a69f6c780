"""What the calls around the layer refuse, on the host: every refusal comes before any launch, so no GPU is needed and the
addresses here are made up."""
import ctypes as C

import pytest
import torch

import paper_2511_21317_amd as httm
from paper_2511_21317_amd import binding as bd

INVALID, UNSUPPORTED, SMALL = -1, -2, -3
ADDR = 1 << 20      # aligned, never read


def norm_rope(**kw):
    d = dict(norm=2, axes=2, rot_dim=64, pairing=0, base=100.0, eps=1e-6, k_scale=1.0, q_weight=None, q_bias=None, k_weight=None,
             k_bias=None)
    d.update(kw)
    return bd.NormRopeStruct(*d.values())


def rows(**kw):
    d = dict(data=ADDR, token_stride=192, head_stride=64)
    d.update(kw)
    return bd.RowsStruct(*d.values())


def paged(**kw):
    d = dict(k_pages=ADDR, v_pages=ADDR, page_table=ADDR, n_pages=10, n_seqs=2, table_stride=4, page_size=16, H_kv=1)
    d.update(kw)
    return bd.PagedStruct(*d.values())


def call_norm_rope(nr=None, q=None, k=None, v=None, dtype=0, pos=ADDR, N=5, H_q=1, H_kv=1, d_head=64, out=(ADDR, ADDR, ADDR)):
    r = [x if x is not None else rows() for x in (q, k, v)]
    return httm.lib().httm_qk_norm_rope(C.byref(nr or norm_rope()), *map(C.byref, r), dtype, pos, N, H_q, H_kv, d_head, *out, None)


def call_append(nr=None, q=None, k=None, v=None, dtype=0, pos=ADDR, first_pos=0, n=5, H_q=1, d_head=64, cache=None, offsets=ADDR,
                seq_lens=ADDR, q_out=ADDR):
    r = [x if x is not None else rows() for x in (q, k, v)]
    return httm.lib().httm_cache_append(C.byref(nr or norm_rope()), *map(C.byref, r), dtype, pos, first_pos, n, H_q, d_head,
                                        C.byref(cache or paged()), offsets, seq_lens, q_out, None)


def call_cached(q=None, kp=ADDR, vp=ADDR, P=7, cache=None, offsets=ADDR, seq_lens=ADDR, n=5, H_q=1, d_head=64, scale=0.125, o=ADDR,
                workspace=ADDR, size=1 << 40):
    return httm.lib().httm_attention_cached(C.byref(q or rows()), kp, vp, P, C.byref(cache or paged()), offsets, seq_lens, n, H_q,
                                            d_head, scale, 0, o, workspace, size, None)


@pytest.mark.parametrize("kw", [
    dict(nr=norm_rope(norm=3)), dict(nr=norm_rope(axes=4)), dict(nr=norm_rope(axes=-1)), dict(nr=norm_rope(rot_dim=0)),
    dict(nr=norm_rope(rot_dim=48)), dict(nr=norm_rope(rot_dim=128)), dict(nr=norm_rope(pairing=2)), dict(nr=norm_rope(base=0.5)),
    dict(nr=norm_rope(base=float("nan"))), dict(nr=norm_rope(eps=-1.0)), dict(nr=norm_rope(eps=float("inf"))),
    dict(nr=norm_rope(k_scale=float("nan"))), dict(nr=norm_rope(q_weight=ADDR + 4)), dict(dtype=3), dict(dtype=-1),
    dict(q=rows(data=ADDR + 8)), dict(q=rows(token_stride=4)), dict(k=rows(head_stride=-8)), dict(v=rows(token_stride=1 << 31)), dict(N=-1),
    dict(H_q=0)])
def test_rows_that_both_calls_refuse(kw):
    assert call_norm_rope(**kw) == INVALID
    kw = {{"N": "n"}.get(a, a): b for a, b in kw.items()}
    assert call_append(**kw) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=128), UNSUPPORTED), (dict(H_q=65), UNSUPPORTED), (dict(H_kv=65), UNSUPPORTED), (dict(N=1 << 25), UNSUPPORTED),
    (dict(pos=None), INVALID), (dict(pos=ADDR + 2), INVALID), (dict(out=(None, ADDR, ADDR)), INVALID),
    (dict(q=rows(data=None)), INVALID), (dict(out=(ADDR, ADDR + 8, ADDR)), INVALID),
    (dict(q=rows(data=None), k=rows(data=None), v=rows(data=None), out=(None, None, None)), INVALID), (dict(N=0), 0),
    (dict(N=0, pos=None, q=rows(data=None)), 0)])
def test_norm_rope(kw, code):
    assert call_norm_rope(**kw) == code


BAD_CACHES = [(dict(k_pages=None), INVALID), (dict(v_pages=ADDR + 8), INVALID), (dict(page_table=ADDR + 2), INVALID), (dict(n_pages=0), INVALID),
              (dict(n_pages=1 << 31), UNSUPPORTED), (dict(n_seqs=0), INVALID), (dict(n_seqs=4097), UNSUPPORTED), (dict(table_stride=0), INVALID),
              (dict(page_size=24), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED),
              (dict(page_size=0), INVALID), (dict(H_kv=0), INVALID), (dict(H_kv=2), INVALID),
              (dict(table_stride=1 << 27), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches(kw, code):
    assert call_append(cache=paged(**kw)) == code
    assert call_cached(cache=paged(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=32), UNSUPPORTED), (dict(n=1 << 25), UNSUPPORTED), (dict(k=rows(data=None)), INVALID), (dict(v=rows(data=None)), INVALID),
    (dict(q=rows(data=None)), INVALID), (dict(q_out=None), INVALID), (dict(q_out=ADDR + 8), INVALID), (dict(pos=None), INVALID),
    (dict(offsets=None), INVALID), (dict(seq_lens=ADDR + 1), INVALID), (dict(first_pos=-1), INVALID), (dict(first_pos=1 << 31), INVALID),
    (dict(H_q=65, cache=paged(H_kv=65)), UNSUPPORTED), (dict(n=0), 0)])
def test_append(kw, code):
    assert call_append(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(d_head=128), UNSUPPORTED), (dict(n=1 << 21), UNSUPPORTED), (dict(n=-1), INVALID), (dict(P=-1), INVALID), (dict(P=1 << 24), UNSUPPORTED),
    (dict(kp=None), INVALID), (dict(vp=ADDR + 8), INVALID), (dict(q=rows(data=None)), INVALID), (dict(q=rows(head_stride=12)), INVALID),
    (dict(o=None), INVALID), (dict(workspace=None), INVALID), (dict(workspace=ADDR + 16), INVALID), (dict(size=0), SMALL),
    (dict(scale=0.0), INVALID), (dict(scale=-0.125), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID),
    (dict(offsets=None), INVALID), (dict(seq_lens=ADDR + 2), INVALID), (dict(n=0, workspace=None, o=None), 0)])
def test_cached(kw, code):
    assert call_cached(**kw) == code


def test_workspace_is_what_the_call_asks_for():
    need = httm.attention_cached_workspace(5, 2, 1, 1, 7)
    assert need > 0 and call_cached(size=need - 1) == SMALL
    for bad in ((-1, 1, 1, 1, 0), (1, 0, 1, 1, 0), (1, 1, 3, 2, 0), (1, 1, 1, 1, -1), (1, 5000, 1, 1, 0), (1, 1, 65, 1, 0), (1 << 21, 1, 1, 1, 0)):
        with pytest.raises(httm.HttmError):
            httm.attention_cached_workspace(*bad)


def test_the_binding_wants_tensors_on_the_gpu():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(httm.HttmError):
        httm.PagedCache(torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16),
                        torch.zeros(1, 3, dtype=torch.int32))
    with pytest.raises(httm.HttmError):
        httm.qk_norm_rope(httm.NormRope(), x, x, x, torch.zeros(4, 2, dtype=torch.int32), x, x, x)
    with pytest.raises(httm.HttmError):
        httm.NormRope(q_weight=torch.ones(64))
