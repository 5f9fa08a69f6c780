"""The operators around the merged attention of a scene, as measurable cases.

Three operators of the library are measured here, each next to its plain form:

  norm_rope   qk_norm_rope: the rows of a QKV projection become the layer's q, k, v - norms of queries and keys for
              each head and the position rotation in one pass
  append      cache_append: new tokens' keys and values go into a paged cache, norm and rotation applied on the way,
              and their queries into a buffer
  cached      attention_cached: the tokens of a batch of sequences attend to a prefix that all of them share (the merged
              keys and values of a scene) and to the pages of their own sequence

Sizes are those of the scenes of this repository's benchmark (2 to 100 frames of 16 x 16 to 37 x 37 patches, merged
lengths from 266 to 28700), and of batches of streams that are served one token, a few tokens or a frame at a time.
Where `own` is true, run() calls the library; else it computes the plain form with elementary torch operations in 32
bits (angles in 64).
"""
import math
import random

import torch

own = False

D = 64
WORKSPACE_BYTES = 256 << 20     # what a serving program keeps for partial results

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------

def listed():
    return [
        # two small frames of the vision transformer, as they enter its global attention layer: a call of a few
        # microseconds, where latency counts
        _rows("norm_rope_2_frames", N=522, grid=16),
        # eight full frames
        _rows("norm_rope_8_frames", N=10992, grid=37),
        # a long clip, the largest pass
        _rows("norm_rope_100_frames", N=137400, grid=37),
        # a text-like model with grouped heads: norms without a mean, neighbouring channels rotate, a part of them only,
        # at far positions, from a projection in 32 bits; nothing divides anything
        _rows("norm_rope_odd", N=7001, H_q=12, H_kv=4, norm="rms", axes=1, pairing="neighbours", rot_dim=48, base=10000.0,
              dtype="fp32", far=1 << 30),
        # a token for each of 32 streams
        _append("append_tokens", B=32, n_lo=1, n_hi=1, len_lo=40, len_hi=4000, H_q=32, H_kv=8, page=64, norm="rms", axes=1,
                base=500000.0),
        # a new frame for each of 8 scenes
        _append("append_frames", B=8, n_lo=1374, n_hi=1374, len_lo=1374, len_hi=5496, page=64, grid=37),
        # ragged pieces of prompts, 16-token pages, fp16 projection, some padding behind the last sequence
        _append("append_odd", B=13, n_lo=1, n_hi=1800, len_lo=1, len_hi=5000, H_q=12, H_kv=4, page=16, norm="rms", axes=1,
                pairing="neighbours", base=10000.0, dtype="fp16", pad=37),
        # one token of one stream against a small merged scene: latency
        _cached("cached_one_token", B=1, n_lo=1, n_hi=1, len_lo=300, len_hi=300, P=5516),
        # a token for each of 64 streams that share the longest merged scene
        _cached("cached_64_streams", B=64, n_lo=1, n_hi=1, len_lo=100, len_hi=5496, P=28700),
        # a few drafted tokens for each of 48 streams, grouped heads, 16-token pages, a padded batch
        _cached("cached_grouped_drafts", B=48, n_lo=1, n_hi=5, len_lo=5, len_hi=4000, P=6376, H_q=32, H_kv=8, page=16, causal=True,
                pad=7),
        # a new frame for each of 4 viewers of the same scene: whole frames see each other and the scene; the largest
        _cached("cached_frames", B=4, n_lo=1374, n_hi=1374, len_lo=1374, len_hi=5496, P=28650),
        # ragged prompts behind a shared beginning
        _cached("cached_prompts", B=6, n_lo=1, n_hi=2000, len_lo=1, len_hi=4100, P=1001, H_q=16, H_kv=4, page=16, causal=True),
    ]


def _case(kind, name, kw):
    case = {"kind": kind, "H_q": 16, "H_kv": 16, "dtype": "bf16"}
    if kind != "cached":
        case.update(norm="layer", axes=2, rot_dim=D, pairing="halves", base=100.0, grid=37, far=0)
    if kind != "norm_rope":
        case.update(page=64, pad=0)
    if kind == "cached":
        case.update(causal=False)
    case.update(kw)
    return dict(case, name=name) if name else case


def _rows(name, **kw):
    return _case("norm_rope", name, kw)


def _append(name, **kw):
    return _case("append", name, kw)


def _cached(name, **kw):
    return _case("cached", name, kw)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotation(rng):
    if rng.random() < 0.5:      # the vision transformer's
        return {"norm": "layer", "axes": 2, "rot_dim": 64, "pairing": "halves", "base": 100.0,
                "grid": rng.randint(16, 37)}
    axes = rng.choice([1, 1, 1, 3])
    return {"norm": rng.choice(["rms", "rms", "none"]), "axes": axes, "rot_dim": 48 if axes == 3 else rng.choice([64, 64, 32, 48, 16]),
            "pairing": rng.choice(["halves", "neighbours"]), "base": rng.choice([10000.0, 500000.0]),
            "far": rng.choice([0, 1 << 20, 1 << 30])}


def _draw_heads(rng):
    H_kv = rng.choice([16, 16, 8, 4, 3, 1])
    return {"H_kv": H_kv, "H_q": H_kv * (1 if H_kv == 16 else rng.choice([1, 2, 3, 4]))}


def draw(rng: random.Random):
    """One more case: any of the three operators, over the ranges of the list."""
    while True:
        kind = rng.choice(["norm_rope", "append", "cached", "cached"])
        kw = _draw_heads(rng)
        if kind == "norm_rope":
            kw.update(_draw_rotation(rng), N=_log(rng, 200, 137400), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
            case = _rows(None, **kw)
        elif kind == "append":
            n_hi = rng.choice([1, _log(rng, 1, 16), _log(rng, 16, 2000)])
            kw.update(_draw_rotation(rng), B=_log(rng, 1, 64) if n_hi <= 16 else rng.randint(1, 12), n_lo=1, n_hi=n_hi, len_lo=1,
                      len_hi=n_hi + _log(rng, 1, 4000), page=rng.choice([16, 32, 64, 128, 256]), pad=rng.choice([0, 0, 5, 40]),
                      dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
            case = _append(None, **kw)
        else:
            n_hi = rng.choice([1, 1, _log(rng, 1, 16), _log(rng, 16, 2000)])
            kw.update(B=_log(rng, 1, 96) if n_hi <= 16 else rng.randint(1, 8), n_lo=1 if rng.random() < 0.7 else n_hi, n_hi=n_hi,
                      len_lo=1, len_hi=n_hi + _log(rng, 1, 6000), P=_log(rng, 266, 28700), page=rng.choice([16, 32, 64, 128, 256]),
                      pad=rng.choice([0, 0, 3, 17]), causal=rng.random() < 0.5)
            case = _cached(None, **kw)
        w, top = work(case), work(listed()[10])
        if w["flops"] <= top["flops"] and w["bytes"] <= 1.6e9:
            return case


# ---- lengths: spread over the range by the golden ratio, so that they follow from the case alone ---------------

def _spread(lo, hi, n, start):
    return [lo + int((hi - lo + 1) * ((start + 0.6180339887498949 * i) % 1.0)) for i in range(n)]


def _lengths(case):
    """New tokens and length with them, of every sequence."""
    n = _spread(case["n_lo"], case["n_hi"], case["B"], 0.5)
    total = _spread(case["len_lo"], case["len_hi"], case["B"], 0.31)
    return n, [max(a, b) for a, b in zip(n, total)]


# ---- inputs ------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(random.Random(seed).getrandbits(62))
    return g


def _projection(case, N, g):
    """Rows of a QKV projection, [N, H_q + 2 H_kv, 64]: every head and channel with a mean and a width of its own, as
    projections have."""
    H = case["H_q"] + 2 * case["H_kv"]
    mean = 0.7 * torch.randn((1, H, D), generator=g, device="cuda")
    width = torch.exp(0.4 * torch.randn((1, H, D), generator=g, device="cuda"))
    x = torch.empty((N, H, D), dtype=_DTYPES[case["dtype"]], device="cuda")
    for i in range(0, N, 16384):
        n = min(16384, N - i)
        x[i:i + n] = torch.randn((n, H, D), generator=g, device="cuda") * width + mean
    return x


def _weights(case, g):
    affine = {n: None for n in ("q_weight", "q_bias", "k_weight", "k_bias")}
    if case["norm"] != "none":
        for n in ("q_weight", "k_weight"):
            affine[n] = 1.0 + 0.3 * torch.randn(D, generator=g, device="cuda")
    if case["norm"] == "layer":
        for n in ("q_bias", "k_bias"):
            affine[n] = 0.2 * torch.randn(D, generator=g, device="cuda")
    return affine


def _positions(case, N, g):
    """[N, axes] int32: grid rows and columns for the patches of frames; else places in a text, far ones on request."""
    axes = case["axes"]
    i = torch.arange(N, device="cuda")
    if axes == 2:
        side = case["grid"]
        slot = i % (side * side + 5) - 5       # 5 special tokens at the front of a frame stand at the origin
        pos = torch.stack([torch.div(slot, side, rounding_mode="floor") + 1, slot % side + 1], dim=1)
        pos = torch.where((slot < 0)[:, None], torch.zeros_like(pos), pos)
    else:
        pos = torch.randint(0, max(N, case["far"]), (N, axes), generator=g, device="cuda")
    return pos.to(torch.int32).contiguous()


def prepare(case, seed):
    g = _generator(seed)
    st = {"case": case}
    if case["kind"] == "norm_rope":
        x = _projection(case, case["N"], g)
        st["N"] = case["N"]
    else:
        n, length = _lengths(case)
        st["N"] = sum(n) + case["pad"]
        off = [0]
        for a in n:
            off.append(off[-1] + a)
        st["n_max"], st["len_max"] = max(n), max(length)
        st["q_offsets"] = torch.tensor(off, dtype=torch.int32, device="cuda")
        st["seq_lens"] = torch.tensor(length, dtype=torch.int32, device="cuda")
        # pages are handed out in any order; a table's entries behind a sequence's last page are -1
        need = [-(-a // case["page"]) for a in length]
        order = torch.randperm(sum(need) + 8, generator=g, device="cuda").to(torch.int32)
        width = max(need) + 1
        table, at = [], 0
        for a in need:
            table.append(torch.nn.functional.pad(order[at:at + a], (0, width - a), value=-1))
            at += a
        st["page_table"] = torch.stack(table).contiguous()
        shape = (order.numel(), case["H_kv"], case["page"], D)
        st["k_pages"] = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * 1.5
        st["v_pages"] = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
        x = _projection(case, st["N"], g) if case["kind"] == "append" else None
    bf = {"dtype": torch.bfloat16, "device": "cuda"}
    H_q, H_kv, N = case["H_q"], case["H_kv"], st["N"]
    if case["kind"] == "cached":
        st["q"] = torch.randn((N, H_q, D), generator=g, **bf)
        # merged keys of a scene: many are alike, each head has a direction of its own
        st["k_prefix"] = torch.randn((H_kv, case["P"], D), generator=g, **bf)
        st["k_prefix"] += torch.randn((H_kv, 1, D), generator=g, **bf)
        st["v_prefix"] = torch.randn((H_kv, case["P"], D), generator=g, **bf)
        st["out"] = torch.zeros((N, H_q * D), **bf)
        st["workspace"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
        return st
    st["q"], st["k"], st["v"] = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    st["affine"] = _weights(case, g)
    st["pos"] = _positions(case, N, g)
    if case["kind"] == "norm_rope":
        st["q_out"] = torch.empty((H_q, N, D), **bf)
        st["k_out"], st["v_out"] = torch.empty((H_kv, N, D), **bf), torch.empty((H_kv, N, D), **bf)
    else:
        st["q_out"] = torch.zeros((N, H_q, D), **bf)
    return st


# ---- one pass ------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(state, kind)
    return {"norm_rope": _plain_norm_rope, "append": _plain_append, "cached": _plain_cached}[kind](state)


def _own(st, kind):
    import paper_2511_21317_amd as httm

    case = st["case"]
    if kind == "cached":
        cache = httm.PagedCache(st["k_pages"], st["v_pages"], st["page_table"])
        return httm.attention_cached(st["q"], st["k_prefix"], st["v_prefix"], cache, st["q_offsets"], st["seq_lens"], st["out"],
                                     scale=0.125, causal=case["causal"], workspace=st["workspace"])
    nr = httm.NormRope(norm=case["norm"], eps=1e-6, axes=case["axes"], rot_dim=case["rot_dim"], pairing=case["pairing"],
                       base=case["base"], **st["affine"])
    if kind == "norm_rope":
        return httm.qk_norm_rope(nr, st["q"], st["k"], st["v"], st["pos"], st["q_out"], st["k_out"], st["v_out"])
    cache = httm.PagedCache(st["k_pages"], st["v_pages"], st["page_table"])
    httm.cache_append(nr, st["q"], st["k"], st["v"], st["pos"], cache, st["q_offsets"], st["seq_lens"], st["q_out"])
    return st["q_out"], st["k_pages"], st["v_pages"]


def _norm(x, case, weight, bias):
    if case["norm"] == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    if case["norm"] != "none":
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
        if weight is not None:
            x = x * weight
        if bias is not None:
            x = x + bias
    return x


def _cos_sin(case, pos):
    """[N, 1, axes, pairs] each; angles in 64 bits."""
    w = case["rot_dim"] // case["axes"]
    freq = case["base"] ** (-torch.arange(0, w, 2, device="cuda", dtype=torch.float64) / w)
    angle = pos.double()[:, None, :, None] * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rotate(x, case, cos, sin):
    N, H, _ = x.shape
    axes, rot = case["axes"], case["rot_dim"]
    w = rot // axes
    shape = (N, H, axes, 2, w // 2) if case["pairing"] == "halves" else (N, H, axes, w // 2, 2)
    dim = 3 if case["pairing"] == "halves" else 4
    a, b = x[..., :rot].reshape(shape).unbind(dim)
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=dim)
    return torch.cat([y.reshape(N, H, rot), x[..., rot:]], dim=-1)


def _plain_rows(st):
    case, affine = st["case"], st["affine"]
    cos, sin = _cos_sin(case, st["pos"])
    q = _rotate(_norm(st["q"].float(), case, affine["q_weight"], affine["q_bias"]), case, cos, sin)
    k = _rotate(_norm(st["k"].float(), case, affine["k_weight"], affine["k_bias"]), case, cos, sin)
    return q.to(torch.bfloat16), k.to(torch.bfloat16), st["v"].to(torch.bfloat16)


def _plain_norm_rope(st):
    q, k, v = _plain_rows(st)
    return q.transpose(0, 1).contiguous(), k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()


def _plain_append(st):
    q, k, v = _plain_rows(st)
    off, lens, page = st["q_offsets"].long(), st["seq_lens"].long(), st["case"]["page"]
    token = torch.arange(st["N"], device="cuda")
    b = torch.searchsorted(off, token, right=True) - 1
    real = b < lens.numel()
    b = torch.where(real, b, torch.zeros_like(b))
    place = lens[b] - off[b + 1] + token
    place = torch.where(real, place, torch.zeros_like(place))
    to = st["page_table"][b, place // page].long()
    at = (place % page)[:, None]
    heads = torch.arange(st["case"]["H_kv"], device="cuda")[None]
    # padding behind the last sequence writes back what is there
    here, there = to[:, None], (real[:, None, None],)
    st["k_pages"][here, heads, at] = torch.where(*there, k, st["k_pages"][here, heads, at])
    st["v_pages"][here, heads, at] = torch.where(*there, v, st["v_pages"][here, heads, at])
    st["q_out"].copy_(torch.where(*there, q, st["q_out"]))
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_cached(st):
    case = st["case"]
    B, H, G, n, L = case["B"], case["H_kv"], case["H_q"] // case["H_kv"], st["n_max"], st["len_max"]
    off, lens = st["q_offsets"].long(), st["seq_lens"].long()
    new = off[1:] - off[:-1]
    # rows of every sequence, padded to the most any has: [B, n, H_q, 64] -> [H, B, n * G, 64]
    i = torch.arange(n, device="cuda")
    token = torch.clamp(off[:-1, None] + i, max=st["N"] - 1)
    q = st["q"][token].float().view(B, n, H, G, D).permute(2, 0, 1, 3, 4).reshape(H, B, n * G, D) * 0.125
    s_prefix = (q.reshape(H, B * n * G, D) @ st["k_prefix"].float().transpose(1, 2)).view(H, B, n * G, -1)
    # own keys and values, gathered: [H, B, L, 64]
    j = torch.arange(L, device="cuda")
    page = torch.clamp(st["page_table"].long()[:, j // case["page"]], min=0)
    k = st["k_pages"][page, :, j % case["page"]].permute(2, 0, 1, 3).float()
    v = st["v_pages"][page, :, j % case["page"]].permute(2, 0, 1, 3).float()
    s_own = q @ k.transpose(2, 3)
    seen = (j[None] < lens[:, None])[:, None]
    if case["causal"]:
        seen = seen & (j[None, None] <= (lens - new)[:, None, None] + i[None, :, None])
    seen = seen.expand(B, n, L).repeat_interleave(G, dim=1)
    s_own = torch.where(seen[None], s_own, -math.inf)
    top = torch.maximum(s_prefix.amax(dim=-1, keepdim=True), s_own.amax(dim=-1, keepdim=True))
    s_prefix, s_own = torch.exp(s_prefix - top), torch.exp(s_own - top)
    o = (s_prefix.view(H, B * n * G, -1) @ st["v_prefix"].float()).view(H, B, n * G, D) + s_own @ v
    o = o / (s_prefix.sum(dim=-1, keepdim=True) + s_own.sum(dim=-1, keepdim=True))
    o = o.view(H, B, n, G, D).permute(1, 2, 0, 3, 4).reshape(B, n, H * G * D).to(torch.bfloat16)
    real = i[None] < new[:, None]
    st["out"][token[real]] = o[real]
    return st["out"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "cached":
        return _exact_cached(st, case)
    rows = {}
    for n in ("q", "k"):
        rows[n] = _exact_rows(st[n], case, st["affine"][n + "_weight"], st["affine"][n + "_bias"], st["pos"])
    rows["v"] = st["v"].double()
    if case["kind"] == "norm_rope":
        return tuple(rows[n].permute(1, 0, 2) for n in ("q", "k", "v"))
    q_out, k_pages, v_pages = st["q_out"].double(), st["k_pages"].double(), st["v_pages"].double()
    n_new, length = _lengths(case)
    table, first = st["page_table"].tolist(), 0
    for b, (n, total) in enumerate(zip(n_new, length)):
        q_out[first:first + n] = rows["q"][first:first + n]
        done = 0
        while done < n:             # a run of tokens that share a page
            place = total - n + done
            row = place % case["page"]
            run_ = min(n - done, case["page"] - row)
            p, s = table[b][place // case["page"]], slice(first + done, first + done + run_)
            k_pages[p, :, row:row + run_] = rows["k"][s].permute(1, 0, 2)
            v_pages[p, :, row:row + run_] = rows["v"][s].permute(1, 0, 2)
            done += run_
        first += n
    return q_out, k_pages, v_pages


def _exact_rows(x, case, weight, bias, pos):
    y = x.double()
    if case["norm"] != "none":
        mu = y.sum(-1, keepdim=True) / D if case["norm"] == "layer" else 0.0
        var = ((y - mu) ** 2).sum(-1, keepdim=True) / D
        y = (y - mu) * (var + 1e-6) ** -0.5
        y = y * weight.double() if weight is not None else y
        y = y + bias.double() if bias is not None else y
    w = case["rot_dim"] // case["axes"]
    z = y.clone()
    for axis in range(case["axes"]):
        for i in range(w // 2):
            t = (pos[:, axis].double() * math.exp(-2.0 * i / w * math.log(case["base"])))[:, None]
            a, b = (i, i + w // 2) if case["pairing"] == "halves" else (2 * i, 2 * i + 1)
            a, b = axis * w + a, axis * w + b
            z[..., a] = y[..., a] * torch.cos(t) - y[..., b] * torch.sin(t)
            z[..., b] = y[..., a] * torch.sin(t) + y[..., b] * torch.cos(t)
    return z


def _exact_cached(st, case):
    out = st["out"].double()
    n_new, length = _lengths(case)
    G, table, first = case["H_q"] // case["H_kv"], st["page_table"].long(), 0
    for b, (n, total) in enumerate(zip(n_new, length)):
        pages = table[b, :-(-total // case["page"])]
        hidden = None
        if case["causal"]:
            hidden = torch.ones((n, total), dtype=torch.bool, device="cuda").triu(total - n + 1)
        for h in range(case["H_kv"]):
            k = torch.cat([st["k_prefix"][h], st["k_pages"][pages, h].reshape(-1, D)[:total]]).double()
            v = torch.cat([st["v_prefix"][h], st["v_pages"][pages, h].reshape(-1, D)[:total]]).double()
            for hq in range(h * G, (h + 1) * G):
                s = (st["q"][first:first + n, hq].double() @ k.T) / 8.0
                if hidden is not None:
                    s[:, case["P"]:].masked_fill_(hidden, -math.inf)
                out[first:first + n, hq * D:(hq + 1) * D] = torch.softmax(s, dim=-1) @ v
        first += n
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    H_q, H_kv = case["H_q"], case["H_kv"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["kind"] == "norm_rope":
        N = case["N"]
    else:
        n, length = _lengths(case)
        N = sum(n)
    if case["kind"] != "cached":     # rows in, rows out, positions; norm and rotation
        rows = N * (H_q + 2 * H_kv) * D
        return {"bytes": rows * (size + 2) + 4 * N * case["axes"], "flops": 10 * N * (H_q + H_kv) * D}
    pairs = sum(a * (case["P"] + (b - a) + (a + 1) / 2 if case["causal"] else case["P"] + b) for a, b in zip(n, length))
    keys = case["P"] + sum(length)
    return {"bytes": 4 * N * H_q * D + 4 * keys * H_kv * D, "flops": int(4 * D * H_q * pairs)}
