"""attention_cached against softmax attention in 64 bits."""
import math

import pytest
import torch

import paper_2511_21317_amd as httm

pytestmark = pytest.mark.gpu

D = 64


class Batch:
    """Sequences with `new` tokens and `lens` rows in a cache whose other rows hold NaN, and a shared prefix."""

    def __init__(self, new, lens, P, H_q, H_kv, page, seed=1, spare=3, pad_front=0, pad=0, v_scale=1.0, k_scale=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        need = [-(-n // page) for n in lens]
        order = torch.randperm(sum(need) + spare, generator=g, device="cuda").to(torch.int32)
        table = torch.full((len(lens), max(need + [0]) + 1), -1, dtype=torch.int32, device="cuda")
        k_pages, v_pages = (torch.full((order.numel(), H_kv, page, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        at = 0
        self.k, self.v = [], []
        for b, (n, m) in enumerate(zip(need, lens)):
            pages = order[at:at + n].long()
            table[b, :n] = order[at:at + n]
            at += n
            k, v = (rand(H_kv, m, D) * k_scale).bfloat16(), (rand(H_kv, m, D) * v_scale).bfloat16()
            self.k.append(k), self.v.append(v)
            for i in range(n):
                rows = min(page, m - i * page)
                k_pages[pages[i], :, :rows] = k[:, i * page:i * page + rows]
                v_pages[pages[i], :, :rows] = v[:, i * page:i * page + rows]
        self.cache = httm.PagedCache(k_pages, v_pages, table)
        off = [pad_front]
        for a in new:
            off.append(off[-1] + a)
        self.n = off[-1] + pad
        self.off, self.new, self.lens, self.P, self.H_q, self.H_kv = off, new, lens, P, H_q, H_kv
        self.offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = rand(self.n, H_q, D).bfloat16()
        self.kp, self.vp = (rand(H_kv, P, D) * k_scale).bfloat16(), (rand(H_kv, P, D) * v_scale).bfloat16()
        self.ws = torch.full((httm.attention_cached_workspace(self.n, len(lens), H_q, H_kv, P),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, causal=False, scale=0.125, q=None, out=None, ws=None):
        out = torch.full((self.n, self.H_q * D), 5.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        return httm.attention_cached(self.q if q is None else q, self.kp if self.P else None, self.vp if self.P else None, self.cache,
                                     self.offsets, self.seq_lens, out, scale=scale, causal=causal, workspace=self.ws if ws is None else ws)

    def reference(self, causal=False, scale=0.125, drop=None):
        """o in 64 bits and how far fp32 statistics, weights rounded to bf16 and one rounding of the result may be off."""
        ref = torch.full((self.n, self.H_q, D), 5.0, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(ref)
        G = self.H_q // self.H_kv
        for b, (n, L) in enumerate(zip(self.new, self.lens)):
            for h in range(self.H_kv if n else 0):
                k, v = (torch.cat([x[h], y[b][h]]).double() for x, y in ((self.kp, self.k), (self.vp, self.v)))
                q = self.q[self.off[b]:self.off[b + 1], h * G:(h + 1) * G].double().reshape(n * G, D)
                s = q @ k.T * scale
                size = (q.abs() @ k.abs().T * scale).amax(-1, keepdim=True) if k.shape[0] else torch.zeros(n * G, 1, device="cuda").double()
                seen = torch.ones(n, self.P + L, dtype=torch.bool, device="cuda")
                if causal:
                    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
                    seen[:, self.P:] = j <= L - n + i
                if drop is not None:
                    seen[:, self.P:] &= ~drop[b][None]
                seen = seen.repeat_interleave(G, 0)
                s = torch.where(seen, s, -math.inf)
                top = torch.where(seen.any(-1, keepdim=True), s.amax(-1, keepdim=True) if s.shape[1] else torch.zeros_like(size), 0.0)
                p = torch.exp(s - top)
                total = p.sum(-1, keepdim=True)
                p = p / torch.where(total == 0, 1.0, total)
                vv = torch.where(torch.isfinite(v), v, 0.0)     # (of keys that no row below sees, or their weight is 0)
                o, a = p @ vv, p @ vv.abs()
                # weights: half a bf16 step; scores: sums of 64 products, a relative error of the weights on both sides; sums over the
                # keys, one after the other in units of 32; the result: half a bf16 step
                t = 2.0 ** -8 * (o.abs() + a) + a * (2.0 ** -17 * size + 2.0 ** -22 * ((self.P + L) / 32 + 64))
                at = slice(self.off[b], self.off[b + 1]), slice(h * G, (h + 1) * G)
                ref[at], tol[at] = o.view(n, G, D), t.view(n, G, D)
        return ref.view(self.n, -1), tol.view(self.n, -1) + 1e-30

    def check(self, causal=False, scale=0.125, **kw):
        got = self.run(causal, scale)
        ref, tol = self.reference(causal, scale, **kw)
        err = (got.double() - ref).abs()
        bad = ~(err <= tol)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}, worst {(err / tol).max():.2f} times"
        return got


def spread(lo, hi, n, start=0.3):
    return [lo + int((hi - lo + 1) * ((start + 0.6180339887498949 * i) % 1.0)) for i in range(n)]


SHAPES = {   # new tokens, rows, prefix, heads, key heads, page
    "one token, one row": ([1], [1], 0, 1, 1, 16),
    "prefix alone": ([1], [0], 1, 2, 1, 16),
    "nothing at all": ([2, 1], [0, 0], 0, 2, 2, 16),
    "one token": ([1], [300], 517, 16, 16, 64),
    "long cache": ([1], [9001], 0, 4, 2, 128),
    "long prefix": ([1], [0], 20011, 3, 3, 16),
    "streams": ([1] * 7, [1, 31, 32, 33, 16, 500, 129], 1003, 4, 4, 16),
    "streams without prefix": ([1] * 5, [64, 65, 1, 0, 700], 0, 8, 2, 32),
    "empty sequences": ([0, 1, 0, 0, 3, 0], [5, 9, 0, 70, 3, 1], 40, 2, 2, 16),
    "drafts": ([3, 1, 5, 2, 4], [3, 100, 77, 2, 1029], 333, 12, 4, 16),
    "many streams": ([1] * 70, spread(0, 400, 70), 100, 2, 1, 64),
    "grouped": ([2] * 3, [50, 60, 70], 95, 64, 2, 16),
    "pieces of prompts": ([1, 130, 64, 65, 17], [1, 200, 64, 1000, 900], 77, 6, 3, 16),
    "a frame": ([261], [783], 1000, 4, 4, 64),
    "frames": ([261, 261, 200], [261, 522, 999], 2001, 2, 2, 256),
    "a prompt": ([700], [700], 0, 3, 1, 128),
    "more tokens than rows": ([40, 5], [13, 2], 0, 2, 1, 16),
    "pieces for many streams": ([20] * 60, spread(20, 90, 60), 301, 2, 2, 16),
    "more streams than lanes": (spread(0, 3, 150), spread(0, 70, 150, 0.7), 45, 2, 1, 16),
    "one long among short": ([1] * 20, [3] * 11 + [40000] + [5] * 8, 33, 2, 2, 64),
    "rows of 64 heads": ([1, 1, 2], [100, 1, 333], 65, 64, 1, 16),
    "a prompt of grouped heads": ([1500], [1500], 0, 5, 1, 16),
    "a prompt behind another": ([300, 700], [2300, 701], 129, 64, 1, 32),
    "prompts of odd groups": ([257, 511, 1], [300, 511, 70], 31, 12, 4, 16),
    # prefixes that are taken with the rows of all sequences together
    "together, a few rows": ([1] * 14, spread(0, 200, 14), 8001, 4, 4, 16),
    "together, streams": ([1] * 30, spread(0, 300, 30), 3607, 4, 4, 32),
    "together, drafts": ([3, 1, 5, 2, 4] * 4, spread(5, 400, 20), 6201, 12, 4, 16),
    "together, pieces": ([28, 27, 0, 30] * 6, spread(30, 200, 24), 15013, 4, 4, 64),
    "together, many rows": ([20] * 60, spread(20, 90, 60), 2603, 4, 4, 16),
    "together, more than lanes": ([1, 0, 2] * 60, spread(0, 70, 180, 0.7), 700, 8, 4, 16),
    "together, more rows": ([12] * 90, spread(0, 60, 90), 3501, 4, 4, 16),
    "together, a row each": ([1] * 1100, spread(0, 40, 1100), 1003, 1, 1, 16),
    # enough rows and keys for tiles of 256 rows
    "wide, a frame": ([261], [783], 29001, 4, 4, 64),
    "wide, frames": ([261, 261, 200], [261, 522, 999], 24001, 2, 2, 256),
    "wide, a prompt": ([3300], [3300], 0, 3, 1, 128),
    "wide, grouped heads": ([2500], [2500], 0, 5, 1, 16),
    "wide, odd groups": ([257, 511, 1], [300, 511, 70], 4031, 12, 4, 16),
    "wide, pieces of prompts": ([0, 400, 130, 64, 300] * 4, spread(0, 900, 20), 2500, 4, 4, 32),
    "wide, more tokens than rows": ([4000, 300], [1300, 20], 2001, 4, 4, 16),
    "a whole scene": ([1374, 1374], [1374, 2748], 5516, 2, 2, 64),
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.replace(" ", "_"))
def test_shapes(shape, causal):
    Batch(*SHAPES[shape], seed=len(shape), pad_front=3, pad=4).check(causal)


@pytest.mark.parametrize("shape", ["streams", "drafts", "frames", "together, drafts", "together, many rows", "wide, frames"])
def test_peaked_scores(shape):
    """Scores of some 100 nats between the keys: the shift has to follow, and most weights vanish."""
    Batch(*SHAPES[shape], seed=3, k_scale=30.0).check(True)


def test_rising_and_falling_scores():
    """Every unit of keys far above, or far below, all before it."""
    for sign in (1, -1):
        b = Batch([1, 1, 70], [900, 33, 400], 800, 2, 2, 16)
        b.q[:] = 1.0
        for x in [b.kp] + b.k:
            x[:] = (sign * 0.002 * torch.arange(x.shape[1], device="cuda")[None, :, None] * 10).bfloat16()
        for i, k in enumerate(b.k):
            for j in range(-(-k.shape[1] // 16)):
                part = k[:, 16 * j:16 * j + 16]
                b.cache.k_pages[int(b.cache.page_table[i, j]), :, :part.shape[1]] = part
        b.check()


def test_scale():
    Batch(*SHAPES["drafts"], seed=4).check(True, scale=0.7)
    Batch(*SHAPES["frames"], seed=4).check(False, scale=0.01)
    Batch(*SHAPES["wide, frames"], seed=4).check(False, scale=0.01)


def test_values_that_are_not_finite_stay_where_they_are_seen():
    """A later token's V of inf or NaN, or its K of NaN, reaches no earlier token."""
    for new, lens, P in (([5, 3], [40, 35], 50), ([200], [200], 100), ([1, 70], [9, 333], 64), ([5, 3] * 7, [40, 35] * 7, 17000),
                         ([1, 100], [9, 333], 64), ([200], [200], 40000)):
        b = Batch(new, lens, P, 4, 2, 16)
        for i, L in enumerate(lens):
            if new[i] < 2:
                continue
            page, row = int(b.cache.page_table[i, (L - 1) // 16]), (L - 1) % 16
            b.cache.v_pages[page, 0, row, 3] = float("inf")
            b.cache.v_pages[page, 0, row, 5] = float("nan")
            b.cache.k_pages[page, 1, row, 7] = float("nan")
        got = b.run(True).view(-1, 4, D)
        ref, tol = b.reference(True)
        ref, tol = ref.view(-1, 4, D), tol.view(-1, 4, D)
        last = torch.zeros(b.n, dtype=torch.bool, device="cuda")
        for i in range(len(new)):
            last[b.off[i + 1] - 1] = new[i] > 1
        err = (got.double() - ref).abs()
        assert (err[~last] <= tol[~last]).all()
        assert torch.isinf(got[last][:, :2, 3]).all() and torch.isnan(got[last][:, :2, 5]).all() and torch.isnan(got[last][:, 2:]).all()
        fine = [c for c in range(D) if c not in (3, 5)]
        assert (err[last][:, :2, fine] <= tol[last][:, :2, fine]).all()


def test_pages_that_are_none_are_left_out():
    b = Batch([2, 1, 90], [100, 50, 200], 33, 2, 2, 16)
    drop = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in b.lens]
    for i, j, bad in ((0, 2, -1), (0, 6, 2**31 - 1), (1, 0, -5), (2, 3, int(b.cache.k_pages.shape[0])), (2, 12, -1)):
        b.cache.page_table[i, j] = bad
        drop[i][16 * j:16 * j + 16] = True
    b.check(False, drop=drop)
    b.check(True, drop=drop)
    b = Batch([2, 1, 4] * 6, [100, 50, 200] * 6, 16000, 2, 2, 16)      # the prefix apart
    drop = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in b.lens]
    for i, j, bad in ((0, 2, -1), (4, 0, 2**31 - 1), (17, 12, -1)):
        b.cache.page_table[i, j] = bad
        drop[i][16 * j:16 * j + 16] = True
    b.check(True, drop=drop)
    b = Batch([2, 1, 690], [100, 50, 800], 24033, 2, 2, 16)            # tiles of 256 rows
    drop = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in b.lens]
    for i, j, bad in ((0, 2, -1), (2, 0, 2**31 - 1), (2, 12, -1), (2, 49, 1 << 20)):
        b.cache.page_table[i, j] = bad
        drop[i][16 * j:16 * j + 16] = True
    b.check(False, drop=drop)
    b.check(True, drop=drop)


def test_pages_that_sequences_share():
    b = Batch([1, 1], [64, 64], 0, 2, 2, 32)
    b.cache.page_table[1, 0] = b.cache.page_table[0, 0]
    b.k[1][:, :32], b.v[1][:, :32] = b.k[0][:, :32], b.v[0][:, :32]
    b.check()


def test_lengths_out_of_range_are_bounded():
    """More rows than the table has count as its rows, fewer than none as none."""
    b = Batch([1, 1, 1], [48, 48, 48], 20, 2, 2, 16)
    b.cache = httm.PagedCache(b.cache.k_pages, b.cache.v_pages, b.cache.page_table[:, :3].contiguous())
    b.seq_lens.copy_(torch.tensor([2**31 - 1, 48, -7]))
    got = b.run()
    b.lens[2] = 0
    b.k[2], b.v[2] = b.k[2][:, :0], b.v[2][:, :0]
    ref, tol = b.reference()
    assert ((got.double() - ref).abs() <= tol).all()


def test_queries_of_any_strides():
    b = Batch(*SHAPES["drafts"], seed=8)
    want = b.run(True)
    headwise = b.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(b.run(True, q=headwise), want)
    wide = torch.full((b.n, 2 * b.H_q, 2 * D), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, ::2, :D] = b.q
    assert torch.equal(b.run(True, q=wide[:, ::2, :D]), want)
    with pytest.raises(httm.HttmError):
        b.run(True, q=b.q.float())
    with pytest.raises(httm.HttmError):
        b.run(True, ws=b.ws[:-256])
    with pytest.raises(httm.HttmError):
        b.run(True, out=torch.empty(b.n, b.H_q * D - 64, dtype=torch.bfloat16, device="cuda"))


def test_runs_are_identical_and_workspaces_do_not_matter():
    for name in ("streams", "frames", "many streams", "together, drafts", "together, many rows", "wide, frames"):
        b = Batch(*SHAPES[name])
        want = b.run(True)
        for fill in (0, 0xFF, 0x7F):
            assert torch.equal(b.run(True, ws=torch.full((b.ws.numel() + 512,), fill, dtype=torch.uint8, device="cuda")), want)


def test_cache_beyond_32_bit_offsets():
    """Pages that lie more than 4 GB into their buffer."""
    page, H = 256, 16
    n_pages = (9 << 30) // (page * H * 128)
    b = Batch([1, 40], [500, 300], 50, H, H, page)
    k, v = (torch.empty(n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    used = b.cache.k_pages.shape[0]
    k[-used:], v[-used:] = b.cache.k_pages, b.cache.v_pages
    table = torch.where(b.cache.page_table >= 0, b.cache.page_table + (n_pages - used), -1).to(torch.int32).contiguous()
    b.cache = httm.PagedCache(k, v, table)
    b.check()
    x = torch.randn(41, 3 * H, D, device="cuda").bfloat16()
    q_out = torch.empty(41, H, D, dtype=torch.bfloat16, device="cuda")
    httm.cache_append(httm.NormRope(norm="none", axes=0), x[:, :H], x[:, H:2 * H], x[:, 2 * H:], None, b.cache, b.offsets, b.seq_lens, q_out)
    assert torch.equal(v[int(table[0, 1]), :, 499 - 256], x[0, 2 * H:]) and torch.equal(k[int(table[1, 1]), :, 299 - 256], x[40, H:2 * H])


def test_as_many_sequences_as_there_may_be():
    n = 4096
    Batch([1] * n, [(7 * i) % 19 for i in range(n)], 21, 1, 1, 16).check()
    with pytest.raises(httm.HttmError):
        httm.attention_cached_workspace(n, n + 1, 1, 1, 0)


def test_two_streams_at_once():
    a, b = Batch(*SHAPES["streams"], seed=1), Batch(*SHAPES["a whole scene"], seed=2)
    want_a, want_b = a.run(), b.run()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        with torch.cuda.stream(sa):
            got.append((a.run(), want_a))
        with torch.cuda.stream(sb):
            got.append((b.run(), want_b))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in got)


@pytest.mark.parametrize("B,n,P", [(4, 1, 700), (1, 1, 3000), (2, 100, 300), (2, 200, 300), (2, 200, 19000), (14, 1, 16000), (20, 8, 15000)])
def test_graph_follows_the_lengths(B, n, P):
    """A captured call reads the lengths on the device: replays serve the sequences as they grow."""
    b = Batch([n] * B, [n + 200] * B, P, 4, 2, 16)
    out = torch.zeros(b.n, b.H_q * D, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        b.run(True, out=out)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            b.run(True, out=out)
    torch.cuda.synchronize()
    for step in range(4):
        b.seq_lens.copy_(torch.tensor([n + step * 37 + i for i in range(B)]))
        b.q.copy_(torch.randn_like(b.q))
        graph.replay()
        want = b.run(True, ws=b.ws.clone())
        torch.cuda.synchronize()
        assert torch.equal(out, want), step


def test_a_scene_and_its_viewers():
    """The operators as they are used together: frames of a scene through norm and rotation, merged by stage 2 into a
    prefix; then new tokens of three viewers are appended and attend to the merged scene and their own, twice, with the scale that the merged keys carry."""
    H, S, Hp, Wp, page = 4, 6, 10, 12, 16
    plan = httm.Plan(httm.make_geom(S, Hp, Wp, 4, 2, 0.6, 0.5, H=H, log2_keys=True))
    torch.manual_seed(11)
    affine = {n: 1 + 0.2 * torch.randn(D, device="cuda") for n in ("q_weight", "q_bias", "k_weight", "k_bias")}
    nr = httm.NormRope(norm="layer", axes=2, base=100.0, **affine)
    cached = httm.NormRope(norm="layer", axes=2, base=100.0, k_scale=httm.LOG2_KEY_SCALE, **affine)
    qkv = torch.randn(plan.N, 3 * H, D, device="cuda").bfloat16()
    pos = torch.randint(0, 12, (plan.N, 2), device="cuda", dtype=torch.int32)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    q, k, v = (torch.empty(H, plan.N, D, **bf) for _ in range(3))
    httm.qk_norm_rope(nr, qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], pos, q, k, v)
    q_m, k_m, v_m = torch.empty(H, plan.M_q, D, **bf), torch.empty(H, plan.M_k, D, **bf), torch.empty(H, plan.M_k, D, **bf)
    aq, ak = (torch.empty(H, plan.N, dtype=torch.int32, device="cuda") for _ in range(2))
    httm.reorder_match_merge(plan, q, k, v, q_m, k_m, v_m, aq, ak)

    B, lens = 3, [0, 0, 0]
    cache = httm.PagedCache(torch.zeros(40, H, page, D, **bf), torch.zeros(40, H, page, D, **bf),
                            torch.randperm(40, device="cuda")[:36].view(3, 12).to(torch.int32).contiguous())
    k_own, v_own = [[] for _ in range(B)], [[] for _ in range(B)]
    for new in ([125, 1, 30], [1, 7, 0]):
        n = sum(new)
        lens = [a + b for a, b in zip(lens, new)]
        off = [0, new[0], new[0] + new[1], n]
        offsets, seq_lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (off, lens))
        x = torch.randn(n, 3 * H, D, device="cuda").bfloat16()
        p = torch.randint(0, 12, (n, 2), device="cuda", dtype=torch.int32)
        q_new, out = torch.empty(n, H, D, **bf), torch.empty(n, H * D, **bf)
        httm.cache_append(cached, x[:, :H], x[:, H:2 * H], x[:, 2 * H:], p, cache, offsets, seq_lens, q_new)
        ws = torch.empty(httm.attention_cached_workspace(n, B, H, H, plan.M_k), dtype=torch.uint8, device="cuda")
        httm.attention_cached(q_new, k_m, v_m, cache, offsets, seq_lens, out, scale=math.log(2.0), workspace=ws)
        # the same rows by the other entry point; then attention in 64 bits from the rows that a user holds
        q2, k2, v2 = (torch.empty(H, n, D, **bf) for _ in range(3))
        httm.qk_norm_rope(cached, x[:, :H], x[:, H:2 * H], x[:, 2 * H:], p, q2, k2, v2)
        assert torch.equal(q2.transpose(0, 1), q_new)
        for b in range(B):
            s = slice(off[b], off[b + 1])
            k_own[b].append(k2[:, s]), v_own[b].append(v2[:, s])
            kk, vv = (torch.cat([t] + own, 1).double() for t, own in ((k_m, k_own[b]), (v_m, v_own[b])))
            score = q2[:, s].double() @ kk.transpose(1, 2) * math.log(2.0)
            size = (q2[:, s].double().abs() @ kk.abs().transpose(1, 2)).amax(-1, keepdim=True) if new[b] else 0.0
            prob = torch.softmax(score, -1)
            ref, a = prob @ vv, prob @ vv.abs()
            tol = 2.0 ** -8 * (ref.abs() + a) + a * (2.0 ** -17 * size + 2.0 ** -22 * (kk.shape[1] / 32 + 64))
            got = out[s].view(-1, H, D).transpose(0, 1).double()
            assert ((got - ref).abs() <= tol).all(), (b, ((got - ref).abs() / tol).max())
