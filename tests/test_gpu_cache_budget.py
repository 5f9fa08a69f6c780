"""Accumulated attention weights and eviction against their definitions, over caches of both kinds."""
import math

import pytest
import torch

import paper_2511_21317_amd as httm
from mx4_util import PackedBatch, pack, unpack
from test_gpu_attention_cached import SHAPES, Batch, D, spread

pytestmark = pytest.mark.gpu

STORES = {"bf16": Batch, "mx4": PackedBatch}


# ---- weights ---------------------------------------------------------------------------------------------------

class Weighed:
    """A batch, the weights its keys have, and its rows' lse: those of attention to prefix and own keys."""

    def __init__(self, store, *shape, seed=0, more=0, lse=None, **kw):
        self.b = b = STORES[store](*shape, seed=seed, **kw)
        capacity = b.cache.page_table.shape[1] * b.cache.page_size + more
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        self.before = torch.exp(2 * torch.randn((len(b.lens), b.H_kv, capacity), generator=g, device="cuda") - 3)
        self.lse = torch.full((b.n, b.H_q), float("nan"), device="cuda")
        self.causal = None

    def attend(self, causal):
        """lse in 64 bits, rounded"""
        b, G = self.b, self.b.H_q // self.b.H_kv
        for i, (n, L) in enumerate(zip(b.new, b.lens)):
            for h in range(b.H_kv if n else 0):
                s = self.scores(i, h, causal)
                p = b.q[b.off[i]:b.off[i + 1], h * G:(h + 1) * G].double() @ b.kp[h].double().T * 0.125
                s = torch.cat([s, p], -1)
                self.lse[b.off[i]:b.off[i + 1], h * G:(h + 1) * G] = (torch.logsumexp(s, -1) if s.shape[-1] else torch.full(s.shape[:2], -math.inf)).float()

    def scores(self, i, h, causal, scale=0.125):
        b, G = self.b, self.b.H_q // self.b.H_kv
        n, L = b.new[i], b.lens[i]
        s = b.q[b.off[i]:b.off[i + 1], h * G:(h + 1) * G].double() @ b.k[i][h].double().T * scale
        if causal:
            r, j = torch.arange(n, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
            s.masked_fill_((j > L - n + r)[:, None], -math.inf)
        return s

    def run(self, causal, decay=1.0, scale=0.125, q=None):
        w = self.before.clone()
        b = self.b
        return httm.cache_weigh(b.q if q is None else q, self.lse, b.cache, b.offsets, b.seq_lens, w, scale=scale, causal=causal, decay=decay)

    def reference(self, causal, decay=1.0, scale=0.125, drop=None):
        """Weights in 64 bits and what fp32 may be off by."""
        b, G = self.b, self.b.H_q // self.b.H_kv
        ref, tol = self.before.double().clone(), torch.zeros_like(self.before).double()
        for i, (n, L) in enumerate(zip(b.new, b.lens)):
            old = torch.arange(L, device="cuda") < L - n
            for h in range(b.H_kv):
                total, t = torch.zeros(L, device="cuda").double(), torch.zeros(L, device="cuda").double()
                if n and L:
                    s = self.scores(i, h, causal, scale)
                    lse = self.lse[b.off[i]:b.off[i + 1], h * G:(h + 1) * G].double()[..., None]
                    x = torch.where(lse == -math.inf, -math.inf, s - torch.where(lse == -math.inf, 0.0, lse))
                    p = torch.exp(x)
                    size = b.q[b.off[i]:b.off[i + 1], h * G:(h + 1) * G].double().abs() @ b.k[i][h].double().abs().T * scale
                    x = torch.where(p > 0, x.abs(), 0.0)
                    # a score: a sum of 64 products, kept in fp32; the exponent in base 2: two roundings of its size; exp2: 2^-22
                    t = (p * (2.0 ** -18 * size + 2.0 ** -22 * x + 2.0 ** -21)).sum((0, 1))
                    total = p.sum((0, 1))
                if drop is not None:
                    total, t = torch.where(drop[i], 0.0, total), torch.where(drop[i], 0.0, t)
                # one addition after the other for a row in sixteen, then sixteen
                t = t + total * 2.0 ** -24 * (n * G / 16 + 24)
                w = self.before[i, h, :L].double()
                ref[i, h, :L] = torch.where(old, decay * w, 0.0) + total
                tol[i, h, :L] = t + 2.0 ** -23 * ref[i, h, :L].abs()
        return ref, tol

    def check(self, causal, decay=1.0, scale=0.125, **kw):
        got = self.run(causal, decay, scale)
        ref, tol = self.reference(causal, float(torch.tensor(decay, dtype=torch.float32)), scale, **kw)
        err = (got.double() - ref).abs()
        bad = ~(err <= tol)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}, worst {(err / tol.clamp_min(1e-30)).max():.2f} times"
        return got


WEIGHED = ["one token, one row", "prefix alone", "nothing at all", "one token", "long cache", "streams", "empty sequences", "drafts", "many streams",
           "grouped", "pieces of prompts", "a frame", "a prompt", "more tokens than rows", "more streams than lanes", "one long among short",
           "rows of 64 heads", "a prompt of grouped heads", "a prompt behind another", "prompts of odd groups"]


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", WEIGHED, ids=lambda s: s.replace(" ", "_").replace(",", ""))
def test_weights(shape, causal, store):
    w = Weighed(store, *SHAPES[shape], seed=len(shape), pad_front=2, pad=3, more=5)
    w.attend(causal)
    w.check(causal, decay=0.75 if causal else 1.0)


@pytest.mark.parametrize("store", STORES)
def test_a_row_gives_all_that_it_has(store):
    """Without a prefix the weights that a token gives its keys sum up to one for each of its heads: attention's own lse."""
    for shape in ("streams without prefix", "a prompt", "grouped"):
        args = list(SHAPES[shape])
        args[2] = 0
        w = Weighed(store, *args, seed=5)
        b = w.b
        out = torch.empty(b.n, b.H_q * D, dtype=torch.bfloat16, device="cuda")
        httm.attention_cached(b.q, None, None, b.cache, b.offsets, b.seq_lens, out, causal=True, workspace=b.ws, lse=w.lse)
        w.before.zero_()
        got = w.check(True).double().sum(-1)
        rows = torch.tensor([n if L else 0 for n, L in zip(b.new, b.lens)], device="cuda").double()[:, None] * (b.H_q // b.H_kv)
        # (lse of tiles of 256 rows: half a step of bf16)
        assert ((got - rows).abs() <= rows * 2.0 ** -7).all()


@pytest.mark.parametrize("store", STORES)
def test_decays_scales_and_strides(store):
    for shape in ("drafts", "a prompt"):
        w = Weighed(store, *SHAPES[shape], seed=7)
        w.attend(True)
        for decay in (0.0, 0.3, 2.0):
            w.check(True, decay=decay)
        w.check(True, scale=0.05)
        b, want = w.b, w.run(True)
        wide = torch.full((b.n, 2 * b.H_q, 2 * D), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, ::2, :D] = b.q
        assert torch.equal(w.run(True, q=wide[:, ::2, :D]), want)
        assert torch.equal(w.run(True, q=b.q.transpose(0, 1).contiguous().transpose(0, 1)), want)
        for bad in (dict(decay=-1.0), dict(scale=0.0), dict(q=b.q.float())):
            with pytest.raises(httm.HttmError):
                w.run(True, **bad)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("new,lens", [([3, 1, 30], [100, 50, 200]), ([90, 80, 130], [100, 100, 200])])
def test_pages_that_are_none_get_nothing(store, new, lens):
    w = Weighed(store, new, lens, 0, 4, 2, 16, seed=3)
    w.attend(True)
    drop = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in lens]
    for i, j, bad in ((0, 2, -1), (1, 0, 2**31 - 1), (2, 12, int(values(w.b.cache).shape[0]))):
        w.b.cache.page_table[i, j] = bad
        drop[i][16 * j:16 * j + 16] = True
    w.check(True, decay=0.5, drop=drop)


def values(cache):
    return cache.k_codes if isinstance(cache, httm.PackedCache) else cache.k_pages


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("new,lens", [([5, 3], [40, 35]), ([100, 200], [120, 333])])
def test_rows_without_keys_and_keys_that_are_not_finite(store, new, lens):
    """A row whose lse is minus infinity adds nothing; a key that is NaN has a weight that is NaN, and no other key has."""
    w = Weighed(store, new, lens, 0, 4, 2, 16, seed=4)
    w.attend(True)
    w.lse[0], w.lse[new[0] + 1, 2] = -math.inf, -math.inf
    w.check(True)
    L, b = lens[1], w.b
    page, row = int(b.cache.page_table[1, (L - 2) // 16]), (L - 2) % 16
    if store == "mx4":
        b.cache.scales[page, 1, row, 0] = 255
    else:
        b.cache.k_pages[page, 1, row, 9] = float("nan")
    got = w.run(True)
    ref, tol = w.reference(True)
    ref[1, 1, L - 2] = float("nan")
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    fine = ~torch.isnan(ref)
    assert ((got.double() - ref).abs() <= tol)[fine].all()


@pytest.mark.parametrize("store", STORES)
def test_weights_are_the_same_every_time_and_shared_pages_are_read(store):
    for shape in ("many streams", "a prompt behind another"):
        w = Weighed(store, *SHAPES[shape], seed=6)
        w.attend(False)
        want = w.run(False)
        for _ in range(3):
            assert torch.equal(w.run(False), want)
    w = Weighed(store, [1, 1], [64, 64], 0, 2, 2, 32, seed=6)
    w.b.cache.page_table[1, 0] = w.b.cache.page_table[0, 0]
    w.b.k[1][:, :32] = w.b.k[0][:, :32]
    w.attend(False)
    w.check(False)


@pytest.mark.parametrize("store", STORES)
def test_weights_of_lengths_out_of_range(store):
    """More rows than the table has count as its rows, fewer than none as none; columns behind them stay."""
    w = Weighed(store, [2, 1, 1], [48, 48, 48], 0, 2, 2, 16, seed=10, more=7)
    b, c = w.b, w.b.cache
    table = c.page_table[:, :3].contiguous()
    b.cache = httm.PackedCache(c.k_codes, c.v_codes, c.scales, table) if store == "mx4" else httm.PagedCache(c.k_pages, c.v_pages, table)
    w.attend(True)
    b.seq_lens.copy_(torch.tensor([2**31 - 1, 48, -7]))
    b.lens[2], b.k[2], b.v[2] = 0, b.k[2][:, :0], b.v[2][:, :0]
    w.check(True, decay=0.5)
    with pytest.raises(httm.HttmError):
        httm.cache_weigh(b.q, w.lse, b.cache, b.offsets, b.seq_lens, w.before[:, :, :47].contiguous())
    for bad in ((None, w.lse, w.before), (b.q, None, w.before), (b.q, w.lse, None), (b.q, w.lse[:-1], w.before), (b.q, w.lse, w.before.double())):
        with pytest.raises(httm.HttmError):
            httm.cache_weigh(bad[0], bad[1], b.cache, b.offsets, b.seq_lens, bad[2])


@pytest.mark.parametrize("store", STORES)
def test_steps_without_tokens_let_the_weights_decay(store):
    w = Weighed(store, [0, 0, 0], [100, 0, 33], 0, 4, 2, 16, seed=8)
    got = w.check(True, decay=0.5)
    assert torch.equal(got[0, :, :100], 0.5 * w.before[0, :, :100])
    w.before[0, 0, 3], w.before[0, 0, 4] = math.inf, math.nan
    got = w.run(True, decay=0.0)
    assert not got[0, :, :100].any() and torch.equal(got[0, :, 100:], w.before[0, :, 100:])


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 100, 3], [20, 9, 30]])
def test_graph_of_weights_follows_the_lengths(store, new):
    w = Weighed(store, new, [300, 200, 150], 0, 4, 2, 16, seed=9)
    w.attend(True)
    b, weights = w.b, w.before.clone()
    call = lambda t: httm.cache_weigh(b.q, w.lse, b.cache, b.offsets, b.seq_lens, t, causal=True, decay=0.5)  # noqa: E731
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(weights)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            call(weights)
    for lens in ([300, 200, 150], [120, 130, 31], [299, 100, 150], [91, 101, 31]):
        b.seq_lens.copy_(torch.tensor(lens))
        weights.copy_(w.before)
        graph.replay()
        want = call(w.before.clone())
        torch.cuda.synchronize()
        assert torch.equal(weights, want), lens


# ---- eviction --------------------------------------------------------------------------------------------------

def expected(w, L, keep, first, last):
    """Where the rows of a head that stay come from: by place and by weight, a loop over the row."""
    if L <= keep:
        return list(range(L))
    def order(p):
        x = float(w[p])
        return (1, 0.0, p) if math.isnan(x) else (0, -x, p)
    middle = sorted(range(first, L - last), key=order)[:keep - first - last]
    gap, stays = keep - last, set(middle)
    behind = sorted(p for p in middle if p >= gap)
    place = list(range(gap)) + list(range(L - last, L))
    free = [p for p in range(first, gap) if p not in stays]
    assert len(free) == len(behind)
    for d, p in zip(free, behind):
        place[d] = p
    return place


class Evicted:
    """Sequences with weights in a cache of either kind."""

    def __init__(self, store, lens, H, page, seed=0, more=0, weights=None):
        self.b = b = STORES[store]([0] * len(lens), lens, 0, H, H, page, seed=seed)
        self.store = store
        capacity = b.cache.page_table.shape[1] * page + more
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 2)
        w = torch.randn((len(lens), H, capacity), generator=g, device="cuda")
        if weights == "few values":
            w = torch.round(2 * w)
        elif weights == "alike":
            w = torch.full_like(w, 0.25)
        elif weights == "wide":
            w = torch.exp(20 * w)
        elif weights == "strange":
            pick = torch.rand(w.shape, generator=g, device="cuda")
            for i, x in enumerate((math.inf, -math.inf, math.nan, -math.nan, 0.0, -0.0, 1e-45, -1e-45)):
                w = torch.where((pick >= i / 16) & (pick < (i + 1) / 16), x, w)
        self.weights = w.contiguous()

    def tensors(self):
        c = self.b.cache
        return [c.k_codes, c.v_codes, c.scales] if self.store == "mx4" else [c.k_pages, c.v_pages]

    def check(self, keep, first=0, last=0, kept=True, untouched=()):
        b, page, lens = self.b, self.b.cache.page_size, self.b.lens
        H, n = b.H_kv, len(lens)
        old, want_w = [t.clone() for t in self.tensors()], self.weights.clone()
        want = [t.clone() for t in old]
        places = torch.full((n, H, keep), -1, dtype=torch.int32)
        table, w = b.cache.page_table.cpu(), self.weights.cpu()
        for i, L in enumerate(lens):
            if i in untouched:
                continue
            for h in range(H):
                src = torch.tensor(expected(w[i, h], L, keep, first, last), dtype=torch.long)
                places[i, h, :len(src)] = src.int()
                dst = torch.arange(len(src))
                ps, pd = table[i, src // page].long().cuda(), table[i, dst // page].long().cuda()
                rs, rd = (src % page).cuda(), (dst % page).cuda()
                for t, o in zip(want, old):
                    t[pd, h, rd] = o[ps, h, rs]
                want_w[i, h, dst.cuda()] = self.weights[i, h, src.cuda()]
        new_lens = torch.full((n,), -9, dtype=torch.int32, device="cuda")
        ws = torch.full((httm.cache_evict_workspace(n, H, keep),), 0xFF, dtype=torch.uint8, device="cuda")
        got = torch.full((n, H, keep), -7, dtype=torch.int32, device="cuda") if kept else None
        httm.cache_evict(b.cache, b.seq_lens, self.weights, keep, new_lens, first=first, last=last, kept=got, workspace=ws)
        assert new_lens.tolist() == [L if i in untouched else min(L, keep) for i, L in enumerate(lens)]
        if kept:
            assert torch.equal(got.cpu(), places), (got.cpu() != places).nonzero()[:4].tolist()
        for name, a, x in zip(("keys", "values", "scales"), self.tensors(), want):
            assert torch.equal(a.view(torch.uint8), x.view(torch.uint8)), name
        assert torch.equal(self.weights.view(torch.int32), want_w.view(torch.int32))
        return new_lens


EVICTED = {   # lengths, key heads, page, keep, first, last
    "one of two": ([2], 1, 16, 1, 0, 0), "one too many": ([65], 2, 16, 64, 0, 0), "nothing to do": ([10, 64, 0], 2, 16, 64, 4, 8),
    "streams": ([70, 64, 65, 300, 0, 1, 129], 3, 16, 64, 4, 16), "first alone": ([100, 40], 2, 32, 40, 40, 0), "last alone": ([100, 41, 500], 2, 32, 40, 0, 40),
    "first and last": ([100, 57, 90], 2, 16, 56, 24, 32), "all but one": ([130, 90], 2, 16, 64, 30, 33), "last by one": ([1000], 2, 64, 999, 0, 500),
    "one row a page over": ([257, 258], 1, 256, 256, 3, 3), "half": ([2001, 999, 1500], 5, 64, 750, 10, 100), "a little": ([4160] * 3, 2, 64, 4096, 4, 256),
    "frames": ([5496, 2748], 4, 128, 1400, 1374, 20), "long": ([30011, 3], 2, 256, 9000, 100, 1374), "many": (spread(0, 90, 150), 2, 16, 33, 2, 5),
}


@pytest.mark.parametrize("weights", [None, "few values", "alike", "strange", "wide"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("case", EVICTED, ids=lambda s: s.replace(" ", "_"))
def test_eviction(case, store, weights):
    lens, H, page, keep, first, last = EVICTED[case]
    Evicted(store, lens, H, page, seed=len(case), weights=weights, more=3).check(keep, first, last)


def test_without_places_and_again():
    """kept is not needed; a second call cuts what the first has left."""
    for store in STORES:
        e = Evicted(store, [500, 70, 300], 2, 16, seed=1, weights="few values")
        new = e.check(200, 4, 20, kept=False)
        e.b.lens, e.b.seq_lens = new.tolist(), new
        new = e.check(64, 4, 20)
        e.b.lens, e.b.seq_lens = new.tolist(), new
        e.check(64, 0, 0)


def test_a_sequence_without_one_of_its_pages_is_left_as_it_is():
    for store in STORES:
        e = Evicted(store, [100, 100, 100, 100], 2, 16, seed=2)
        e.b.cache.page_table[0, 3] = -1
        e.b.cache.page_table[1, 6] = 2**31 - 1
        e.b.cache.page_table[2, 7] = -5           # behind its rows
        e.check(40, 2, 10, untouched=(0, 1))


def test_lengths_out_of_range_are_bounded():
    e = Evicted("bf16", [112, 100], 1, 16, seed=3)      # 112: all the rows of the table but its last column, which has no page
    c = e.b.cache
    e.b.cache = httm.PagedCache(c.k_pages, c.v_pages, c.page_table[:, :7].contiguous())
    e.b.seq_lens.copy_(torch.tensor([2**31 - 1, -3]))
    e.b.lens = [112, 0]
    e.check(50, 1, 1)


def test_beginnings_that_sequences_share_stay():
    """Pages within `first` may belong to several sequences: they are not written."""
    e = Evicted("mx4", [96, 96], 2, 32, seed=4)
    e.b.cache.page_table[1, 0] = e.b.cache.page_table[0, 0]
    e.check(64, 32, 8)


def test_eviction_beyond_32_bit_offsets():
    page, H = 256, 16
    n_pages = (9 << 30) // (page * H * 128)
    e = Evicted("bf16", [700, 300], H, page, seed=5)
    c = e.b.cache
    k, v = (torch.zeros(n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    used = c.k_pages.shape[0]
    k[-used:], v[-used:] = c.k_pages, c.v_pages
    table = torch.where(c.page_table >= 0, c.page_table + (n_pages - used), -1).to(torch.int32).contiguous()
    small = e.b.cache
    e.b.cache = httm.PagedCache(k, v, table)
    new = torch.empty(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(httm.cache_evict_workspace(2, H, 256), dtype=torch.uint8, device="cuda")
    w = e.weights.clone()
    httm.cache_evict(e.b.cache, e.b.seq_lens, w, 256, new, first=3, last=30, workspace=ws)
    httm.cache_evict(small, e.b.seq_lens, e.weights, 256, new, first=3, last=30, workspace=ws)
    assert torch.equal(k[-used:].view(torch.int16), small.k_pages.view(torch.int16)) and torch.equal(v[-used:].view(torch.int16), small.v_pages.view(torch.int16))
    assert torch.equal(w, e.weights) and not k[:-used].any()


def test_evictions_on_two_streams_and_with_any_workspace():
    """Two caches at once, a workspace each, whatever is in it."""
    pairs = [Evicted("mx4", [900, 300, 70], 4, 16, seed=11), Evicted("bf16", [5000, 2000], 2, 64, seed=12)]
    results = []
    for fill in (0, 0xFF):
        streams = [torch.cuda.Stream() for _ in pairs]
        kept = []
        copies = [[t.clone() for t in (*e.tensors(), e.weights)] for e in pairs]
        torch.cuda.synchronize()
        for e, s in zip(pairs, streams):
            n, H = len(e.b.lens), e.b.H_kv
            with torch.cuda.stream(s):
                new, k = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, H, 250, dtype=torch.int32, device="cuda")
                ws = torch.full((httm.cache_evict_workspace(n, H, 250),), fill, dtype=torch.uint8, device="cuda")
                httm.cache_evict(e.b.cache, e.b.seq_lens, e.weights, 250, new, first=3, last=40, kept=k, workspace=ws)
                kept += [k, new, ws]
        torch.cuda.synchronize()
        results.append([t.clone() for e in pairs for t in (*e.tensors(), e.weights)] + [t for t in kept if t.dtype is torch.int32])
        for e, old in zip(pairs, copies):
            for t, o in zip((*e.tensors(), e.weights), old):
                t.copy_(o)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*results))
    for e in pairs:
        e.check(250, 3, 40)


def test_graph_follows_the_lengths():
    e = Evicted("mx4", [200, 150, 90], 2, 16, seed=6)
    start, w0 = [t.clone() for t in e.tensors()], e.weights.clone()
    new, kept = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, 2, 64, dtype=torch.int32, device="cuda")
    ws = torch.empty(httm.cache_evict_workspace(3, 2, 64), dtype=torch.uint8, device="cuda")

    def step():
        httm.cache_evict(e.b.cache, e.b.seq_lens, e.weights, 64, new, first=2, last=9, kept=kept, workspace=ws)

    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step()
    for lens in ([200, 150, 90], [70, 64, 3], [199, 0, 65], [1, 150, 90]):
        for t, x in zip([*e.tensors(), e.weights], [*start, w0]):
            t.copy_(x)
        e.b.seq_lens.copy_(torch.tensor(lens))
        graph.replay()
        got = [t.clone() for t in [*e.tensors(), e.weights, new, kept]]
        for t, x in zip([*e.tensors(), e.weights], [*start, w0]):
            t.copy_(x)
        e.b.lens = lens
        e.check(64, 2, 9)
        step_new = [*e.tensors(), e.weights]
        torch.cuda.synchronize()
        assert all(torch.equal(a, x) for a, x in zip(got, step_new)) and got[-2].tolist() == [min(64, L) for L in lens]


# ---- together --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("store", STORES)
def test_a_stream_within_its_budget(store):
    """As they are used: frames come, attend, leave their weight with the keys that they looked at, and the cache is cut back; against a plain
    simulation that holds every head's rows in a list."""
    H, G, B, page, keep, first, last = 2, 2, 3, 16, 60, 4, 12
    torch.manual_seed(21)
    pages_of = 8
    table = torch.randperm(B * pages_of + 2, device="cuda")[:B * pages_of].view(B, pages_of).to(torch.int32).contiguous()
    n_pages = B * pages_of + 2
    if store == "mx4":
        u8 = dict(dtype=torch.uint8, device="cuda")
        cache = httm.PackedCache(torch.zeros(n_pages, H, page, 32, **u8), torch.zeros(n_pages, H, page, 32, **u8), torch.zeros(n_pages, H, page, 4, **u8), table)
    else:
        bf = dict(dtype=torch.bfloat16, device="cuda")
        cache = httm.PagedCache(torch.zeros(n_pages, H, page, D, **bf), torch.zeros(n_pages, H, page, D, **bf), table)
    weights = torch.zeros(B, H, pages_of * page, device="cuda")
    nr = httm.NormRope(norm="none", axes=0)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    k_sim, v_sim, w_sim = ([[torch.empty(0, D).double().cuda() for _ in range(H)] for _ in range(B)] for _ in range(3))
    w_sim = [[torch.empty(0).double().cuda() for _ in range(H)] for _ in range(B)]
    cut = 0
    for step in range(9):
        new = [[30, 1, 7], [40, 1, 0], [1, 64, 9]][step % 3]
        off = [0, new[0], new[0] + new[1], sum(new)]
        offsets, n = torch.tensor(off, dtype=torch.int32, device="cuda"), sum(new)
        lens = lens + torch.tensor(new, dtype=torch.int32, device="cuda")
        q, k, v = torch.randn(n, H * G, D, device="cuda").bfloat16(), torch.randn(n, H, D, device="cuda").bfloat16(), torch.randn(n, H, D, device="cuda").bfloat16()
        out, lse = torch.empty(n, H * G * D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H * G, device="cuda")
        ws = torch.empty(max(httm.attention_cached_workspace(n, B, H * G, H, 0), httm.cache_evict_workspace(B, H, keep)), dtype=torch.uint8, device="cuda")
        httm.cache_append(nr, None, k, v, None, cache, offsets, lens, None)
        httm.attention_cached(q, None, None, cache, offsets, lens, out, causal=True, workspace=ws, lse=lse)
        httm.cache_weigh(q, lse, cache, offsets, lens, weights, causal=True, decay=0.9)
        held = [unpack(*pack(x)) if store == "mx4" else x.double() for x in (k, v)]
        for b in range(B):
            for h in range(H):
                sl = slice(off[b], off[b + 1])
                k_sim[b][h], v_sim[b][h] = (torch.cat([x, y[sl, h]]) for x, y in ((k_sim[b][h], held[0]), (v_sim[b][h], held[1])))
                L, m = k_sim[b][h].shape[0], new[b]
                s = q[sl, h * G:(h + 1) * G].double() @ k_sim[b][h].T * 0.125
                hidden = torch.arange(L, device="cuda")[None] > L - m + torch.arange(m, device="cuda")[:, None]
                s.masked_fill_(hidden[:, None], -math.inf)
                p = torch.softmax(s, -1)
                ref = p @ v_sim[b][h]
                got = out.view(n, H * G, D)[sl, h * G:(h + 1) * G].double()
                # weights and the result rounded to bf16; scores to 2^-14
                assert ((got - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * (p @ v_sim[b][h].abs())).all(), (step, b, h)
                w_sim[b][h] = torch.cat([0.9 * w_sim[b][h], torch.zeros(m, device="cuda").double()]) + p.sum((0, 1))
                assert ((weights[b, h, :L].double() - w_sim[b][h]).abs() <= 2.0 ** -8 * w_sim[b][h] + 1e-6).all()
        kept, new_lens = torch.empty(B, H, keep, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        measured = weights.clone()
        httm.cache_evict(cache, lens, weights, keep, new_lens, first=first, last=last, kept=kept, workspace=ws)
        for b in range(B):
            L = int(lens[b])
            cut += L > keep
            for h in range(H):
                place = expected(measured[b, h].cpu(), L, keep, first, last)
                assert kept[b, h, :len(place)].tolist() == place
                k_sim[b][h], v_sim[b][h], w_sim[b][h] = (x[b][h][torch.tensor(place, dtype=torch.long, device="cuda")] for x in (k_sim, v_sim, w_sim))
        lens = new_lens
    assert cut > 6
    rows = [torch.empty(int(lens.sum()), H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    offsets = torch.cat([torch.zeros(1, device="cuda"), lens.cumsum(0)]).to(torch.int32)
    httm.cache_read(cache, offsets, lens, *rows)
    for got, sim in zip(rows, (k_sim, v_sim)):
        for b in range(B):
            for h in range(H):
                assert torch.equal(got[int(offsets[b]):int(offsets[b + 1]), h].double(), sim[b][h])
