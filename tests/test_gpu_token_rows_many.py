"""qk_norm_rope and cache_append with as many rows as it takes for every number of heads that a wave walks over: 1, 2, 4, 8, 12 and 16, and
for rows that go past the caches."""
import pytest
import torch

import paper_2511_21317_amd as httm
from test_gpu_token_rows import D, DTYPES, affine, check, formula, make_cache, positions

pytestmark = pytest.mark.gpu

FORMS = {   # norm, axes, rot_dim, pairing, base
    "layer": ("layer", 2, 64, "halves", 100.0), "rms": ("rms", 1, 48, "neighbours", 10000.0), "none": ("none", 3, 48, "halves", 10000.0),
}


def data(N, H_q, H_kv, dtype):
    torch.manual_seed(N + H_q)
    x = (torch.randn(N, H_q + 2 * H_kv, D, device="cuda") * 1.7 + 0.8).to(DTYPES[dtype])
    return x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]


def make(form, **kw):
    norm, axes, rot_dim, pairing, base = FORMS[form]
    weights = affine(norm, 5)
    return httm.NormRope(norm=norm, eps=1e-5, axes=axes, rot_dim=rot_dim, pairing=pairing, base=base, **weights, **kw), weights


def expected(t, name, form, weights, pos, scale=1.0):
    norm, axes, rot_dim, pairing, base = FORMS[form]
    return formula(t, norm, weights.get(name + "_weight"), weights.get(name + "_bias"), 1e-5, axes, rot_dim, pairing, base, pos, scale)


@pytest.mark.parametrize("N,H_q,H_kv,dtype,form", [
    (1003, 5, 3, "bf16", "rms"),
    (2003, 5, 3, "bf16", "layer"), (2003, 5, 3, "fp16", "rms"), (2003, 5, 3, "fp32", "none"),      # two heads, which divide neither
    (4001, 5, 3, "bf16", "layer"), (4001, 5, 3, "fp16", "none"), (4001, 5, 3, "fp32", "rms"),      # four
    (4001, 6, 1, "bf16", "none"), (5501, 9, 7, "bf16", "rms"),
    (11003, 16, 16, "bf16", "layer"), (12501, 21, 11, "fp16", "rms"), (11003, 16, 16, "fp32", "layer"),     # eight
    (17003, 16, 16, "bf16", "none"), (20203, 19, 10, "bf16", "layer"),                             # twelve
    (22003, 16, 16, "bf16", "layer"), (30003, 17, 9, "bf16", "rms"), (30003, 17, 9, "fp16", "layer"),        # sixteen, past the caches
    (30003, 17, 9, "fp32", "rms")])
def test_norm_rope(N, H_q, H_kv, dtype, form):
    q, k, v = data(N, H_q, H_kv, dtype)
    nr, weights = make(form, k_scale=0.25)
    pos = positions(N, FORMS[form][1], 4000, 9)
    out = [torch.full((H + 2, N, D), float("nan"), dtype=torch.bfloat16, device="cuda") for H in (H_q, H_kv, H_kv)]
    httm.qk_norm_rope(nr, q, k, v, pos, *(o[1:-1] for o in out))
    for name, t, got, scale in (("q", q, out[0], 1.0), ("k", k, out[1], 0.25)):
        ref, tol = expected(t, name, form, weights, pos, scale)
        check(got[1:-1].transpose(0, 1), ref, tol, name)
    assert torch.equal(out[2][1:-1].transpose(0, 1), v.to(torch.bfloat16))
    for o in out:       # what lies in front of and behind an output
        assert torch.isnan(o[0]).all() and torch.isnan(o[-1]).all()


@pytest.mark.parametrize("new,H_q,H_kv,dtype,form,page", [
    ([700, 1, 0, 1290, 12], 6, 3, "bf16", "rms", 16), ([2003], 6, 3, "fp32", "layer", 64),         # two heads
    ([1500, 3, 2498], 5, 5, "bf16", "layer", 32), ([4001], 10, 5, "fp16", "none", 256), ([41] * 98, 6, 3, "fp32", "rms", 16),    # four
    ([3001, 2, 8000], 16, 16, "bf16", "layer", 64), ([12000, 501], 22, 11, "fp16", "rms", 128),   # eight
    ([17003], 16, 16, "bf16", "rms", 64),                                                          # twelve
    ([9000, 13003], 16, 16, "bf16", "layer", 64), ([30003], 18, 9, "fp32", "rms", 16)])            # sixteen
def test_append(new, H_q, H_kv, dtype, form, page):
    front, back = 3, 10
    n = front + sum(new) + back
    lens = [a + (37 * i + 11) % 90 for i, a in enumerate(new)]
    q, k, v = data(n, H_q, H_kv, dtype)
    nr, weights = make(form)
    pos = positions(n, FORMS[form][1], 4000, 9)
    cache = make_cache(lens, page, H_kv, 1)
    want_k, want_v = cache.k_pages.double(), cache.v_pages.clone()
    off = [front]
    for a in new:
        off.append(off[-1] + a)
    offsets, seq_lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (off, lens))
    q_out = torch.full((n, H_q, D), 7.0, dtype=torch.bfloat16, device="cuda")
    httm.cache_append(nr, q, k, v, pos, cache, offsets, seq_lens, q_out)
    real = slice(front, n - back)
    ref, tol = expected(q[real], "q", form, weights, pos[real])
    check(q_out[real], ref, tol, "q")
    assert (q_out[:front] == 7).all() and (q_out[n - back:] == 7).all()
    row = torch.cat([torch.arange(m - a, m) for a, m in zip(new, lens)]).cuda()
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
    at = cache.page_table[seq, row // page].long(), row % page
    ref, tol_k = expected(k[real], "k", form, weights, pos[real])
    tol = torch.zeros_like(want_k)          # 0 where nothing is to be written
    want_k[at[0], :, at[1]], tol[at[0], :, at[1]] = ref, tol_k
    want_v[at[0], :, at[1]] = v[real].to(torch.bfloat16)
    check(cache.k_pages, want_k, tol, "k pages")
    assert torch.equal(cache.v_pages, want_v)
