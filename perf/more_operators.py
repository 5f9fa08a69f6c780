"""A paged cache that is held in 4 bits and kept within a budget, as measurable cases.

Four operators of the library are measured here, each next to its plain form:

  append   cache_append to a PackedCache, and cache_read: rows of keys and values are rounded to 4 bits with a power of two per
           32 channels, go into the pages, and come back as the values that the cache holds
  packed   attention_cached over a PackedCache: the tokens of a batch of sequences attend to a prefix that all share and to
           their own pages
  weigh    cache_weigh: what weight the tokens of a step gave to every key of their sequence, added to what it had before
  evict    cache_evict: the keys with the least weight leave the cache, and the others close the gaps

Sizes are those of the scenes of this repository's benchmark (frames of 37 x 37 patches and 5 special tokens, merged lengths
from 266 to 28700) and of batches of streams that are served one token, a few tokens or a frame at a time. Where `own` is
true, run() calls the library; else it computes the plain form with elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

D = 64
BLOCK = 32                      # channels that share a power of two
SCALE = 0.125
WORKSPACE_BYTES = 256 << 20     # what a serving program keeps for partial results

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases ---------------------------------------------------------------------------------------------

def listed():
    return [
        # a token for each of 32 streams: latency
        _append("append_tokens", B=32, n_lo=1, n_hi=1, len_lo=40, len_hi=4000, H_kv=8),
        # a new frame for each of 8 scenes
        _append("append_frames", B=8, n_lo=1374, n_hi=1374, len_lo=1374, len_hi=5496),
        # ragged pieces of prompts in 32 bits, 16-token pages, three heads, padding behind the last sequence
        _append("append_odd", B=13, n_lo=0, n_hi=1800, len_lo=1, len_hi=5000, H_kv=3, page=16, dtype="fp32", pad=37),
        # one token of one stream that has watched four frames: latency
        _packed("packed_one_token", B=1, n_lo=1, n_hi=1, len_lo=5496, len_hi=5496),
        # a token for each of 64 streams with long histories, grouped heads
        _packed("packed_64_streams", B=64, n_lo=1, n_hi=1, len_lo=100, len_hi=21984, H_q=32, H_kv=8),
        # a new frame for each of 4 viewers of a merged scene, behind up to 20 frames of their own: the largest
        _packed("packed_frames", B=4, n_lo=1374, n_hi=1374, len_lo=1374, len_hi=27480, P=5516),
        # ragged prompts behind a shared beginning, some without a token, a padded batch
        _packed("packed_prompts", B=6, n_lo=0, n_hi=2000, len_lo=1, len_hi=9000, P=1001, H_q=16, H_kv=4, page=16, causal=True, pad=9),
        # what the token of each of the 64 streams looked at
        _weigh("weigh_64_streams", B=64, n_lo=1, n_hi=1, len_lo=100, len_hi=21984, H_q=32, H_kv=8),
        # what two new frames looked at, from a cache in 16 bits
        _weigh("weigh_frames", B=2, n_lo=1374, n_hi=1374, len_lo=5496, len_hi=13740, store="bf16"),
        # a few drafted tokens or short pieces for each of 7 streams
        _weigh("weigh_drafts", B=7, n_lo=0, n_hi=300, len_lo=1, len_hi=5000, H_q=12, H_kv=4, page=16, causal=True, pad=5, decay=0.9),
        # streams at their budget: what came since the last time has to go, some are not there yet; 16 bits
        _evict("evict_streams", B=64, len_lo=3300, len_hi=4352, keep=4096, first=4, last=256, H_kv=8, store="bf16"),
        # scenes that grew to 20 frames are cut to eight, the first and the last one among them, and read for a dense layer
        _evict("evict_frames", B=2, len_lo=13740, len_hi=27480, keep=10992, first=1374, last=1374),
    ]


def _case(kind, name, kw):
    case = {"kind": kind, "H_kv": 16, "page": 64, "store": "mx4"}
    if kind != "evict":
        case.update(pad=0)
    if kind == "append":
        case.update(dtype="bf16")
    if kind in ("packed", "weigh"):
        case.update(H_q=16, causal=False)
    if kind == "packed":
        case.update(P=0)
    if kind == "weigh":
        case.update(decay=1.0)
    case.update(kw)
    return dict(case, name=name) if name else case


def _append(name, **kw):
    return _case("append", name, kw)


def _packed(name, **kw):
    return _case("packed", name, kw)


def _weigh(name, **kw):
    return _case("weigh", name, kw)


def _evict(name, **kw):
    return _case("evict", name, kw)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case: any of the four operators, over the ranges of the list."""
    most = work(listed()[5])["flops"]
    while True:
        kind = rng.choice(["append", "packed", "packed", "weigh", "evict"])
        H_kv = rng.choice([16, 16, 8, 4, 3, 1])
        kw = {"H_kv": H_kv, "page": rng.choice([16, 32, 64, 128, 256])}
        if kind == "evict":
            hi = _log(rng, 64, 27480)
            keep = max(16, int(hi * rng.uniform(0.3, 1.05)))
            first, last = rng.choice([0, 1, 4, keep // 8]), rng.choice([0, 1, 32, keep // 8, keep // 2])
            case = _evict(None, B=_log(rng, 1, 64), len_lo=rng.randint(0, hi), len_hi=hi, keep=keep, first=min(first, keep // 4),
                          last=min(last, keep // 2), store=rng.choice(["mx4", "bf16"]), **kw)
        else:
            n_hi = rng.choice([1, 1, _log(rng, 1, 16), _log(rng, 16, 2000)])
            kw.update(n_lo=n_hi if rng.random() < 0.3 else rng.choice([0, 1]), n_hi=n_hi, len_lo=1,
                      B=_log(rng, 1, 96) if n_hi <= 16 else rng.randint(1, 8), pad=rng.choice([0, 0, 3, 17]))
            if kind == "append":
                case = _append(None, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), len_hi=n_hi + _log(rng, 1, 4000), **kw)
            else:
                kw.update(H_q=H_kv * (1 if H_kv == 16 else rng.choice([1, 2, 3, 4])), causal=rng.random() < 0.5,
                          len_hi=n_hi + _log(rng, 1, 21984))
                if kind == "packed":
                    case = _packed(None, P=rng.choice([0, 0, _log(rng, 266, 28700)]), **kw)
                else:
                    case = _weigh(None, store=rng.choice(["mx4", "bf16"]), decay=rng.choice([1.0, 1.0, 0.9, 0.5]), **kw)
        if kind == "evict":
            rows = case["B"] * case["len_hi"]
        else:
            n, length = _lengths(case)
            if sum(n) == 0:
                continue
            rows = case["B"] * max(length)
        # (the plain forms pad every sequence to the longest)
        if work(case)["flops"] <= most and rows * H_kv <= 12_000_000:
            return case


# ---- lengths: spread over the range by the golden ratio, so that they follow from the case alone ---------------

def _spread(lo, hi, n, start):
    return [lo + int((hi - lo + 1) * ((start + 0.6180339887498949 * i) % 1.0)) for i in range(n)]


def _lengths(case):
    """New tokens and length with them, of every sequence."""
    total = _spread(case["len_lo"], case["len_hi"], case["B"], 0.31)
    if case["kind"] == "evict":
        return [0] * case["B"], total
    n = _spread(case["n_lo"], case["n_hi"], case["B"], 0.5)
    return n, [max(a, b) for a, b in zip(n, total)]


# ---- inputs ------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(random.Random(seed).getrandbits(62))
    return g


def _rows(shape, g):
    """Rows of keys or values, [..., H, rows, 64]: heads and channels with a width of their own, some channels much wider."""
    width = torch.exp(0.6 * torch.randn((shape[-3], 1, D), generator=g, device="cuda"))
    mean = 0.7 * torch.randn((shape[-3], 1, D), generator=g, device="cuda")
    return torch.randn(shape, generator=g, device="cuda") * width + mean


def _pages(case, n_pages, g):
    """Pages as an earlier step left them."""
    H, page, bf = case["H_kv"], case["page"], case["store"] == "bf16"
    if bf:
        k, v = (torch.empty((n_pages, H, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        k, v = (torch.empty((n_pages, H, page, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
        scales = torch.empty((n_pages, H, page, 4), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 18) // (H * page))
    for i in range(0, n_pages, step):
        n = min(step, n_pages - i)
        x, y = _rows((n, H, page, D), g), _rows((n, H, page, D), g)
        if bf:
            k[i:i + n], v[i:i + n] = x, y
        else:
            (k[i:i + n], ke), (v[i:i + n], ve) = _pack(x), _pack(y)
            scales[i:i + n] = torch.stack([ke, ve], dim=-1).flatten(-2)
    return {"k_pages": k, "v_pages": v} if bf else {"k_pages": k, "v_pages": v, "scales": scales}


def prepare(case, seed):
    g = _generator(seed)
    n, length = _lengths(case)
    H_kv, page = case["H_kv"], case["page"]
    i32 = {"dtype": torch.int32, "device": "cuda"}
    off = [0]
    for a in n:
        off.append(off[-1] + a)
    N = off[-1] + case.get("pad", 0)
    st = {"case": case, "N": N, "n_max": max(n), "len_max": max(length), "q_offsets": torch.tensor(off, **i32),
          "seq_lens": torch.tensor(length, **i32)}
    # pages are handed out in any order; a table's entries behind a sequence's last page are -1
    need = [-(-a // page) for a in length]
    order = torch.randperm(sum(need) + 8, generator=g, device="cuda").to(torch.int32)
    width = max(need) + 1
    table, at = [], 0
    for a in need:
        table.append(torch.nn.functional.pad(order[at:at + a], (0, width - a), value=-1))
        at += a
    st["page_table"] = torch.stack(table).contiguous()
    st.update(_pages(case, order.numel(), g))
    bf = {"dtype": torch.bfloat16, "device": "cuda"}
    if case["kind"] == "append":
        x = torch.empty((N, 2 * H_kv, D), dtype=_DTYPES[case["dtype"]], device="cuda")
        x.copy_(_rows((2 * H_kv, N, D), g).transpose(0, 1))
        st["k"], st["v"] = x[:, :H_kv], x[:, H_kv:]
        st["k_out"], st["v_out"] = torch.zeros((N, H_kv, D), **bf), torch.zeros((N, H_kv, D), **bf)
    if case["kind"] in ("packed", "weigh"):
        st["q"] = torch.randn((N, case["H_q"], D), generator=g, **bf)
    if case["kind"] == "packed":
        # merged keys of a scene: many are alike, each head has a direction of its own
        P = case["P"]
        st["k_prefix"] = st["v_prefix"] = None
        if P:
            st["k_prefix"] = torch.randn((H_kv, P, D), generator=g, **bf)
            st["k_prefix"] += torch.randn((H_kv, 1, D), generator=g, **bf)
            st["v_prefix"] = torch.randn((H_kv, P, D), generator=g, **bf)
        st["out"] = torch.zeros((N, case["H_q"] * D), **bf)
        st["workspace"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    if case["kind"] in ("weigh", "evict"):
        # what keys gathered so far: most of them little, a few very much, and some that nothing looked at yet
        shape = (case["B"], H_kv, width * page)
        st["weights"] = torch.exp(1.5 * torch.randn(shape, generator=g, device="cuda") - 4.0)
        st["weights"] *= torch.rand(shape, generator=g, device="cuda") > 0.05
    if case["kind"] == "weigh":
        # the sums of attention, of which a shared prefix has a part
        s, seen = _scores(st)
        lse = torch.logsumexp(torch.where(seen, s, -math.inf), dim=-1)
        st["lse"] = torch.zeros((N, case["H_q"]), device="cuda")
        rows = lse.view(H_kv, case["B"], st["n_max"], -1).permute(1, 2, 0, 3).reshape(case["B"], st["n_max"], case["H_q"])
        token, real = _tokens(st)
        st["lse"][token[real]] = rows[real] + torch.log1p(3.0 * torch.rand(rows[real].shape, generator=g, device="cuda"))
    if case["kind"] == "evict":
        left = [min(a, case["keep"]) for a in length]
        st["kept"] = torch.empty((case["B"], H_kv, case["keep"]), **i32)
        st["new_lens"] = torch.empty(case["B"], **i32)
        st["workspace"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        st["read_offsets"] = torch.tensor([sum(left[:i]) for i in range(case["B"] + 1)], **i32)
        st["k_out"], st["v_out"] = torch.zeros((sum(left), H_kv, D), **bf), torch.zeros((sum(left), H_kv, D), **bf)
    return st


# ---- one pass ------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(state, kind)
    return {"append": _plain_append, "packed": _plain_packed, "weigh": _plain_weigh, "evict": _plain_evict}[kind](state)


def _own(st, kind):
    import paper_2511_21317_amd as httm

    case = st["case"]
    if case["store"] == "mx4":
        cache = httm.PackedCache(st["k_pages"], st["v_pages"], st["scales"], st["page_table"])
    else:
        cache = httm.PagedCache(st["k_pages"], st["v_pages"], st["page_table"])
    off, lens = st["q_offsets"], st["seq_lens"]
    if kind == "append":    # the rows have their norm and rotation
        httm.cache_append(httm.NormRope(norm="none", axes=0), None, st["k"], st["v"], None, cache, off, lens, None)
        return httm.cache_read(cache, off, lens, st["k_out"], st["v_out"])
    if kind == "packed":
        return httm.attention_cached(st["q"], st["k_prefix"], st["v_prefix"], cache, off, lens, st["out"], scale=SCALE,
                                     causal=case["causal"], workspace=st["workspace"])
    if kind == "weigh":
        return httm.cache_weigh(st["q"], st["lse"], cache, off, lens, st["weights"], scale=SCALE, causal=case["causal"],
                                decay=case["decay"])
    httm.cache_evict(cache, lens, st["weights"], case["keep"], st["new_lens"], first=case["first"], last=case["last"],
                     kept=st["kept"], workspace=st["workspace"])
    if case["store"] == "bf16":
        return st["kept"], st["new_lens"], st["weights"], st["k_pages"], st["v_pages"]
    rows = httm.cache_read(cache, st["read_offsets"], st["new_lens"], st["k_out"], st["v_out"])
    return st["kept"], st["new_lens"], st["weights"], *rows


def _unit(exponent):
    """2^(exponent - 127) in 32 bits, exactly."""
    return (exponent.int() << 23).view(torch.float32)


def _pack(x):
    """Rows in 4 bits: codes, two channels a byte, the even one low, and an exponent per 32 channels.

    A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, a value the code's times 2^(exponent - 127). The exponent is the one
    of the largest value in its block, rounded to two bits of significand, less two: nothing is off by more than half a step."""
    x = x.float()
    blocks = x.reshape(*x.shape[:-1], D // BLOCK, BLOCK)
    top = blocks.abs().amax(dim=-1)
    exponent = torch.clamp(((top.view(torch.int32) + 0x200000) >> 23) - 2, 1, 252)
    a = blocks.abs() / _unit(exponent)[..., None]
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * torch.signbit(blocks)).reshape(*x.shape[:-1], D // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), exponent.to(torch.uint8)


def _unpack(codes, exponents):
    """Codes [..., 32] and exponents [..., 2] as 32-bit values [..., 64]."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    m, e = c & 1, (c >> 1) & 3
    value = torch.where(e > 0, (2.0 + m) * _unit(e + 125), 0.5 * m)
    value = torch.where(c > 7, -value, value).unflatten(-1, (D // BLOCK, BLOCK))
    return (value * _unit(exponents)[..., None]).flatten(-2)


def _tokens(st):
    """Token of row i of sequence b, [B, n_max], and whether there is one."""
    off = st["q_offsets"].long()
    i = torch.arange(st["n_max"], device="cuda")
    return torch.clamp(off[:-1, None] + i, max=st["N"] - 1), i[None] < (off[1:] - off[:-1])[:, None]


def _gather(st, at):
    """Rows of the cache at (page, head, row) in 32 bits: keys and values."""
    if st["case"]["store"] == "bf16":
        return st["k_pages"][at].float(), st["v_pages"][at].float()
    e = st["scales"][at]
    return _unpack(st["k_pages"][at], e[..., 0::2]), _unpack(st["v_pages"][at], e[..., 1::2])


def _own_keys(st):
    """Keys and values of every sequence, padded to the longest: [H, B, L, 64] each."""
    j = torch.arange(st["len_max"], device="cuda")
    page = torch.clamp(st["page_table"].long()[:, j // st["case"]["page"]], min=0)
    heads = torch.arange(st["case"]["H_kv"], device="cuda")[:, None, None]
    return _gather(st, (page[None], heads, (j % st["case"]["page"])[None, None]))


def _query_rows(st):
    """[H, B, n * G, 64] in 32 bits, rows of every sequence, padded to the most any has."""
    case = st["case"]
    B, H, G, n = case["B"], case["H_kv"], case["H_q"] // case["H_kv"], st["n_max"]
    token, _ = _tokens(st)
    return st["q"][token].float().view(B, n, H, G, D).permute(2, 0, 1, 3, 4).reshape(H, B, n * G, D)


def _seen(st):
    """Which keys which rows see, [B, n * G, L]."""
    case, n, L = st["case"], st["n_max"], st["len_max"]
    lens, new = st["seq_lens"].long(), (st["q_offsets"][1:] - st["q_offsets"][:-1]).long()
    i, j = torch.arange(n, device="cuda"), torch.arange(L, device="cuda")
    seen = ((j[None] < lens[:, None])[:, None] & (i[None] < new[:, None])[:, :, None])
    if case["causal"]:
        seen = seen & (j[None, None] <= (lens - new)[:, None, None] + i[None, :, None])
    return seen.repeat_interleave(case["H_q"] // case["H_kv"], dim=1)


def _scores(st):
    k, _ = _own_keys(st)
    return (_query_rows(st) * SCALE) @ k.transpose(2, 3), _seen(st)[None]


def _plain_append(st):
    case = st["case"]
    off, lens, page = st["q_offsets"].long(), st["seq_lens"].long(), case["page"]
    token = torch.arange(st["N"], device="cuda")
    b = torch.searchsorted(off, token, right=True) - 1
    real = token < off[-1]
    token, b = token[real], b[real]
    place = lens[b] - off[b + 1] + token
    at = (st["page_table"][b, place // page].long()[:, None], torch.arange(case["H_kv"], device="cuda")[None], (place % page)[:, None])
    (st["k_pages"][at], ke), (st["v_pages"][at], ve) = _pack(st["k"][token]), _pack(st["v"][token])
    st["scales"][at] = torch.stack([ke, ve], dim=-1).flatten(-2)
    k, v = _gather(st, at)
    st["k_out"][token], st["v_out"][token] = k.to(torch.bfloat16), v.to(torch.bfloat16)
    return st["k_out"], st["v_out"]


def _plain_packed(st):
    case = st["case"]
    B, H, G, n = case["B"], case["H_kv"], case["H_q"] // case["H_kv"], st["n_max"]
    q = _query_rows(st) * SCALE
    k, v = _own_keys(st)
    s = torch.where(_seen(st)[None], q @ k.transpose(2, 3), -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    if case["P"]:
        s_prefix = (q.reshape(H, B * n * G, D) @ st["k_prefix"].float().transpose(1, 2)).view(H, B, n * G, -1)
        top = torch.maximum(top, s_prefix.amax(dim=-1, keepdim=True))
    s = torch.exp(s - top)
    o, total = s @ v, s.sum(dim=-1, keepdim=True)
    if case["P"]:
        s_prefix = torch.exp(s_prefix - top)
        o = o + (s_prefix.view(H, B * n * G, -1) @ st["v_prefix"].float()).view(H, B, n * G, D)
        total = total + s_prefix.sum(dim=-1, keepdim=True)
    o = (o / total).view(H, B, n, G, D).permute(1, 2, 0, 3, 4).reshape(B, n, H * G * D).to(torch.bfloat16)
    token, real = _tokens(st)
    st["out"][token[real]] = o[real]
    return st["out"]


def _plain_weigh(st):
    case, L = st["case"], st["len_max"]
    B, H, n = case["B"], case["H_kv"], st["n_max"]
    s, seen = _scores(st)
    token, _ = _tokens(st)
    lse = st["lse"][token].view(B, n, H, -1).permute(2, 0, 1, 3).reshape(H, B, -1, 1)
    looked = torch.where(seen, torch.exp(s - lse), 0.0).sum(dim=2).transpose(0, 1)
    j, lens = torch.arange(L, device="cuda"), st["seq_lens"].long()
    new = (st["q_offsets"][1:] - st["q_offsets"][:-1]).long()
    w = st["weights"][:, :, :L]
    before = torch.where((j[None] < (lens - new)[:, None])[:, None], w * case["decay"], 0.0)
    st["weights"][:, :, :L] = torch.where((j[None] < lens[:, None])[:, None], before + looked, w)
    return st["weights"]


def _plain_evict(st):
    case, L = st["case"], st["len_max"]
    B, H, K, page = case["B"], case["H_kv"], case["keep"], case["page"]
    lens = st["seq_lens"].long()[:, None, None]
    j = torch.arange(L, device="cuda")[None, None]
    inside = (j >= case["first"]) & (j < lens - case["last"])
    w = torch.where(inside, st["weights"][:, :, :L], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, torch.arange(L, device="cuda").expand_as(order))
    stays = inside & (rank < K - case["first"] - case["last"])
    # positions up to `gap` that are left free are filled by what stays behind it, both in ascending order
    gap = K - case["last"]
    free, moves = inside & ~stays & (j < gap), stays & (j >= gap)
    rank = torch.where(moves, moves.long().cumsum(-1) - 1, L)
    source = torch.zeros((B, H, L + 1), dtype=torch.long, device="cuda").scatter_(-1, rank, j.expand(B, H, L))
    d = torch.arange(K, device="cuda")[None, None]
    pad = torch.nn.functional.pad
    free = pad(free, (0, K - L)) if K > L else free[..., :K]
    to = torch.where(free, torch.gather(source, -1, torch.where(free, free.long().cumsum(-1) - 1, L)), d)
    to = torch.where(d < gap, to, d + lens - K)
    kept = torch.where(lens > K, to, torch.where(d < lens, d, -1))
    b, h, d = (kept >= 0).nonzero(as_tuple=True)
    p = kept[b, h, d]
    at, old = ((st["page_table"][b, x // page].long(), h, x % page) for x in (d, p))
    st["k_pages"][at], st["v_pages"][at] = st["k_pages"][old], st["v_pages"][old]
    if case["store"] == "mx4":
        st["scales"][at] = st["scales"][old]
    st["weights"][b, h, d] = st["weights"][b, h, p]
    st["kept"].copy_(kept)
    st["new_lens"].copy_(torch.clamp(st["seq_lens"], max=K))
    if case["store"] == "bf16":
        return st["kept"], st["new_lens"], st["weights"], st["k_pages"], st["v_pages"]
    one = h == 0
    b, d = b[one], d[one]
    rows = st["read_offsets"].long()[b] + d
    at = (st["page_table"][b, d // page].long()[:, None], torch.arange(H, device="cuda")[None], (d % page)[:, None])
    k, v = _gather(st, at)
    st["k_out"][rows], st["v_out"][rows] = k.to(torch.bfloat16), v.to(torch.bfloat16)
    return st["kept"], st["new_lens"], st["weights"], st["k_out"], st["v_out"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "packed": _exact_packed, "weigh": _exact_weigh, "evict": _exact_evict}[case["kind"]](st, case)


def _nearest(x):
    """The values that 4 bits hold for rows of 64 channels."""
    y = x.double().reshape(-1, D // BLOCK, BLOCK)
    top = y.abs().amax(dim=-1, keepdim=True)
    m, e = torch.frexp(top)                      # top = m 2^e, m from 0.5 to 1: 4 or 6 times the unit, or 8 of half of it
    e = torch.where(m >= 0.875, e + 1, e) - 3
    unit = (torch.clamp(e, -126, 125).long() + 1023 << 52).view(torch.float64)      # 2^e
    level = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")
    best, value = torch.full_like(y, math.inf), torch.zeros_like(y)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):           # of two that are as near, the one whose last bit is 0
        off = (y.abs() - level[i] * unit).abs()
        value = torch.where(off < best, level[i] * unit, value)
        best = torch.minimum(best, off)
    return (torch.sign(y) * value).reshape(x.shape)


def _exact_append(st, case):
    out = []
    n = int(st["q_offsets"][-1])
    for x, y in ((st["k"], st["k_out"]), (st["v"], st["v_out"])):
        y = y.double()
        for i in range(0, n, 16384):
            y[i:min(n, i + 16384)] = _nearest(x[i:min(n, i + 16384)])
        out.append(y)
    return tuple(out)


def _exact_rows(st, case, b, total):
    """Keys and values of sequence b, [H, total, 64]."""
    pages = st["page_table"][b, :-(-total // case["page"])].long()
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), dtype=torch.float64, device="cuda")
    out = []
    for name, which in (("k_pages", 0), ("v_pages", 1)):
        x = st[name][pages].transpose(0, 1).flatten(1, 2)[:, :total]
        if case["store"] == "mx4":
            y = torch.empty((*x.shape[:2], D), dtype=torch.float64, device="cuda")
            y[..., 0::2], y[..., 1::2] = level[(x % 16).long()], level[(x // 16).long()]
            e = st["scales"][pages].transpose(0, 1).flatten(1, 2)[:, :total, which::2].long()
            x = y * (e + 896 << 52).view(torch.float64).repeat_interleave(BLOCK, dim=-1)
        out.append(x.double())
    return out


def _hidden(case, n, total):
    if not case["causal"]:
        return None
    return torch.ones((n, total), dtype=torch.bool, device="cuda").triu(total - n + 1)


def _exact_packed(st, case):
    out = st["out"].double()
    n_new, length = _lengths(case)
    G, first = case["H_q"] // case["H_kv"], 0
    for b, (n, total) in enumerate(zip(n_new, length)):
        if n == 0:
            continue
        k_own, v_own = _exact_rows(st, case, b, total)
        hidden = _hidden(case, n, total)
        for h in range(case["H_kv"]):
            k, v = k_own[h], v_own[h]
            if case["P"]:
                k, v = torch.cat([st["k_prefix"][h].double(), k]), torch.cat([st["v_prefix"][h].double(), v])
            for hq in range(h * G, (h + 1) * G):
                s = (st["q"][first:first + n, hq].double() @ k.T) / 8.0
                if hidden is not None:
                    s[:, case["P"]:].masked_fill_(hidden, -math.inf)
                out[first:first + n, hq * D:(hq + 1) * D] = torch.softmax(s, dim=-1) @ v
        first += n
    return out


def _exact_weigh(st, case):
    w = st["weights"].double()
    n_new, length = _lengths(case)
    G, first = case["H_q"] // case["H_kv"], 0
    for b, (n, total) in enumerate(zip(n_new, length)):
        k, _ = _exact_rows(st, case, b, total)
        hidden = _hidden(case, n, total)
        w[b, :, :total - n] *= case["decay"]
        w[b, :, total - n:total] = 0.0
        for hq in range(case["H_q"] if n else 0):
            s = (st["q"][first:first + n, hq].double() @ k[hq // G].T) / 8.0 - st["lse"][first:first + n, hq:hq + 1].double()
            p = torch.exp(s)
            if hidden is not None:
                p = p.masked_fill(hidden, 0.0)
            w[b, hq // G, :total] += p.sum(dim=0)
        first += n
    return w


def _exact_evict(st, case):
    """Whole numbers and moved rows: nothing is rounded, and a loop over every head of every sequence says what goes where."""
    _, length = _lengths(case)
    keep, first, last, page, H = case["keep"], case["first"], case["last"], case["page"], case["H_kv"]
    kept = torch.full((case["B"], H, keep), -1, dtype=torch.int32)
    weights, table = st["weights"].cpu(), st["page_table"].cpu().long()
    old = weights.clone()
    k_pages, v_pages = st["k_pages"], st["v_pages"]
    rows_k, rows_v = st["k_out"].double(), st["v_out"].double()
    if case["store"] == "bf16":
        k_pages, v_pages = k_pages.double(), v_pages.double()
    begin = 0
    for b, total in enumerate(length):
        left = min(total, keep)
        k_old, v_old = _exact_rows(st, case, b, total)
        for h in range(H):
            place = torch.arange(left)
            if total > keep:
                w = old[b, h, first:total - last]
                # by weight, and by place among equals
                best = torch.argsort(w, descending=True, stable=True)[:keep - first - last] + first
                at, behind = keep - last, best[best >= keep - last].sort().values
                gone = torch.ones(at, dtype=torch.bool)
                gone[:first] = False
                gone[best[best < at]] = False
                place[:at][gone] = behind
                place[at:] = torch.arange(total - last, total)
            kept[b, h, :left] = place.int()
            weights[b, h, :left] = old[b, h, place]
            there = place.cuda()
            if case["store"] == "bf16":
                d = torch.arange(left)
                p, r = table[b, d // page].cuda(), (d % page).cuda()
                k_pages[p, h, r], v_pages[p, h, r] = k_old[h, there], v_old[h, there]
            else:
                rows_k[begin:begin + left, h], rows_v[begin:begin + left, h] = k_old[h, there], v_old[h, there]
        begin += left
    new_lens = torch.clamp(st["seq_lens"], max=keep)
    out = (k_pages, v_pages) if case["store"] == "bf16" else (rows_k, rows_v)
    return kept.cuda(), new_lens, weights.cuda(), *out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    H_kv = case["H_kv"]
    row = 2 * (D // 2 + D // BLOCK) if case["store"] == "mx4" else 4 * D      # key and value
    n, length = _lengths(case)
    N = sum(n)
    if case["kind"] == "append":        # rows in, their codes out, codes in again, values out
        size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
        return {"bytes": N * H_kv * (2 * D * size + 2 * row + 4 * D), "flops": 6 * N * H_kv * 2 * D}
    if case["kind"] == "evict":
        # weights in, places out; of the keys between the first and the last ones those behind the gaps move, as often as the
        # others stay, and the last ones; for 4 bits what stays is read then
        moved, total = 0, 0
        for a in length:
            if a > case["keep"]:
                share = (case["keep"] - case["first"] - case["last"]) / max(1, a - case["first"] - case["last"])
                moved += int((a - case["keep"]) * share) + case["last"]
            total += min(a, case["keep"])
        read = total * (row + 4 * D) if case["store"] == "mx4" else 0
        return {"bytes": H_kv * (4 * sum(length) + 4 * case["B"] * case["keep"] + 2 * moved * (row + 4) + read),
                "flops": 4 * H_kv * sum(length)}
    pairs = sum(a * ((b - a) + (a + 1) / 2 if case["causal"] else b) for a, b in zip(n, length))
    if case["kind"] == "weigh":         # keys and queries in, weights in and out
        return {"bytes": N * case["H_q"] * (2 * D + 4) + H_kv * sum(length) * (row // 2 + 8), "flops": int(2 * D * case["H_q"] * pairs)}
    P = case["P"]
    return {"bytes": 4 * N * case["H_q"] * D + H_kv * (4 * P * D + sum(length) * row), "flops": int(4 * D * case["H_q"] * (pairs + N * P))}
