"""Streams with rotation whose cache is cut again and again: rows keep the positions that they came with, and new tokens are given theirs."""
import math

import pytest
import torch

import paper_2511_21317_amd as httm
from test_gpu_attention_cached import D
from test_gpu_token_rows import formula

pytestmark = pytest.mark.gpu

BASE = 10000.0
THETA = dict(norm="rms", axes=1, rot_dim=64, pairing="halves", base=BASE, eps=1e-6)


def empty_cache(store, n_pages, H, page, table):
    if store == "mx4":
        u8 = dict(dtype=torch.uint8, device="cuda")
        return httm.PackedCache(torch.zeros(n_pages, H, page, 32, **u8), torch.zeros(n_pages, H, page, 32, **u8), torch.zeros(n_pages, H, page, 4, **u8), table)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    return httm.PagedCache(torch.zeros(n_pages, H, page, D, **bf), torch.zeros(n_pages, H, page, D, **bf), table)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def held_within(store, got, ref, tol):
    """Whether rows of the cache are those of the formula: to bf16, or to a fifth above a block's unit and a quarter of the unit below two (its largest is
    3.5 to 7 units)."""
    if store == "mx4":
        top = (ref.abs() + tol).unflatten(-1, (2, 32)).amax(-1, keepdim=True).expand(-1, -1, -1, 32).flatten(-2)
        tol = 1.2 * tol + torch.maximum(ref.abs() / 5, top / 14)
    return bool(((got.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("store", ["bf16", "mx4"])
def test_positions_count_on_behind_evictions(store):
    H, G, B, page, keep, first, last = 2, 2, 2, 16, 48, 4, 12
    torch.manual_seed(31)
    table = torch.randperm(B * 8 + 2, device="cuda")[:B * 8].view(B, 8).to(torch.int32).contiguous()
    cache = empty_cache(store, B * 8 + 2, H, page, table)
    weights = torch.zeros(B, H, 8 * page, device="cuda")
    nr = httm.NormRope(**THETA)
    lens, seen = [0] * B, [0] * B           # rows that a sequence has, and tokens that came so far: the next one's position
    k_sim = [[torch.empty(0, D, device="cuda").double() for _ in range(H)] for _ in range(B)]
    v_sim = [[torch.empty(0, D, device="cuda").double() for _ in range(H)] for _ in range(B)]
    cut = 0
    for step in range(8):
        new = [[30, 1], [17, 40], [1, 1], [64, 5]][step % 4]
        off, n = [0, new[0], sum(new)], sum(new)
        lens = [a + b for a, b in zip(lens, new)]
        offsets, seq_lens = i32(off), i32(lens)
        pos = torch.cat([torch.arange(seen[b], seen[b] + new[b], device="cuda") for b in range(B)])[:, None].to(torch.int32).contiguous()
        q, k, v = (torch.randn(n, h, D, device="cuda").bfloat16() for h in (H * G, H, H))
        q_out = torch.empty(n, H * G, D, dtype=torch.bfloat16, device="cuda")
        httm.cache_append(nr, q, k, v, pos, cache, offsets, seq_lens, q_out)
        rows = [torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        httm.cache_read(cache, offsets, seq_lens, *rows)
        args = ("rms", None, None, 1e-6, 1, 64, "halves", BASE)
        ref, tol = formula(q, *args, pos)
        assert ((q_out.double() - ref).abs() <= tol).all()
        ref, tol = formula(k, *args, pos)
        assert held_within(store, rows[0], ref, tol)
        if cut:     # the check sees a wrong position: that of a token's row
            late = torch.cat([torch.arange(lens[b] - new[b], lens[b], device="cuda") for b in range(B)])[:, None]
            assert not held_within(store, rows[0], *formula(k, *args, late))
        out, lse = torch.empty(n, H * G * D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H * G, device="cuda")
        ws = torch.empty(max(httm.attention_cached_workspace(n, B, H * G, H, 0), httm.cache_evict_workspace(B, H, keep)), dtype=torch.uint8, device="cuda")
        httm.attention_cached(q_out, None, None, cache, offsets, seq_lens, out, causal=True, workspace=ws, lse=lse)
        httm.cache_weigh(q_out, lse, cache, offsets, seq_lens, weights, causal=True)
        for b in range(B):
            for h in range(H):
                sl = slice(off[b], off[b + 1])
                k_sim[b][h], v_sim[b][h] = (torch.cat([x[b][h], y[sl, h].double()]) for x, y in zip((k_sim, v_sim), rows))
                s = q_out[sl, h * G:(h + 1) * G].double() @ k_sim[b][h].T * 0.125
                hidden = torch.arange(lens[b], device="cuda")[None] > lens[b] - new[b] + torch.arange(new[b], device="cuda")[:, None]
                p = torch.softmax(s.masked_fill(hidden[:, None], -math.inf), -1)
                ref = p @ v_sim[b][h]
                got = out.view(n, H * G, D)[sl, h * G:(h + 1) * G].double()
                # weights and the result rounded to bf16; scores to 2^-14
                assert ((got - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * (p @ v_sim[b][h].abs())).all(), (step, b, h)
        kept, new_lens = torch.empty(B, H, keep, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        httm.cache_evict(cache, seq_lens, weights, keep, new_lens, first=first, last=last, kept=kept, workspace=ws)
        for b in range(B):
            cut += lens[b] > keep
            for h in range(H):
                place = kept[b, h, :min(lens[b], keep)].long()
                assert place.unique().numel() == place.numel()
                k_sim[b][h], v_sim[b][h] = k_sim[b][h][place], v_sim[b][h][place]
        lens, seen = new_lens.tolist(), [a + b for a, b in zip(seen, new)]
    assert cut > 4 and all(s > n for s, n in zip(seen, lens))


@pytest.mark.parametrize("store", ["bf16", "mx4"])
def test_without_positions_a_token_has_that_of_its_row(store):
    """What `pos` left out means does not know of evictions: first_pos and the row in the sequence as long as it is now."""
    H, page = 2, 16
    torch.manual_seed(32)
    table = i32([[3, 1, 0, 2], [5, 4, 7, 6]])
    nr = httm.NormRope(**THETA)
    k, v = (torch.randn(70, H, D, device="cuda").bfloat16() for _ in range(2))
    lens, new_lens, weights = i32([40, 30]), i32([0, 0]), torch.rand(2, H, 64, device="cuda")
    caches = [empty_cache(store, 8, H, page, table) for _ in range(2)]
    ws = torch.empty(httm.cache_evict_workspace(2, H, 24), dtype=torch.uint8, device="cuda")
    for c in caches:
        httm.cache_append(nr, None, k, v, None, c, i32([0, 40, 70]), lens, None)
        httm.cache_evict(c, lens, weights.clone(), 24, new_lens, first=2, last=8, workspace=ws)
    offsets, lens = i32([0, 5, 9]), new_lens + i32([5, 4])
    pos = torch.cat([torch.arange(24, 29), torch.arange(24, 28)])[:, None].to(torch.int32).cuda() + 100
    httm.cache_append(nr, None, k[:9], v[:9], None, caches[0], offsets, lens, None, first_pos=100)
    httm.cache_append(nr, None, k[:9], v[:9], pos, caches[1], offsets, lens, None)
    for a, b in zip(*([c.k_codes, c.v_codes, c.scales] if store == "mx4" else [c.k_pages, c.v_pages] for c in caches)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
