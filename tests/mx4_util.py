"""Rows in 4 bits in plain 64-bit torch, and batches over a cache that holds them (not collected by pytest)."""
import torch

import paper_2511_21317_amd as httm
from test_gpu_attention_cached import Batch, D

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def power(e):
    """2^(e - 127) in 64 bits, exactly."""
    return (e.long() + 896 << 52).view(torch.float64)


def exponents(top):
    """Exponent byte of blocks by their largest |x| (64-bit): that of it rounded to two significant bits, less 2."""
    m, e = torch.frexp(top)                              # top = m 2^e, 0.5 <= m < 1
    e = torch.where(m >= 0.875, e + 1, e) - 3
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp(-126, 125) + 127
    return torch.where(torch.isfinite(top), e, torch.full_like(e, 255))


def nearest(x, exponent):
    """Index of the level nearest to |x| in units of 2^(exponent - 127), of two as near the even one.  x [..., 32], exponent [...]."""
    unit = power(exponent)[..., None]
    best, index = torch.full_like(x, float("inf")), torch.zeros(x.shape, dtype=torch.long, device=x.device)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):
        off = (x.abs() - LEVELS[i] * unit).abs()
        index = torch.where(off < best, i, index)
        best = torch.minimum(best, off)
    return index


def pack(x):
    """codes [..., 32] uint8 and exponents [..., 2] uint8 of rows [..., 64]."""
    y = x.double().unflatten(-1, (2, 32))
    nan = ~torch.isfinite(y).all(-1)
    e = exponents(torch.where(nan, torch.full_like(y[..., 0], float("inf")), y.abs().amax(-1)))
    code = nearest(torch.where(torch.isfinite(y), y, 0.0), torch.where(e == 255, torch.full_like(e, 127), e))
    code = (code + 8 * torch.signbit(y).long()).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), e.to(torch.uint8)


def unpack(codes, e):
    """Values [..., 64] in 64 bits."""
    level = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    unit = torch.where(e == 255, float("nan"), power(e))
    return level[c] * unit.repeat_interleave(32, -1)


def scales_of(ke, ve):
    return torch.stack([ke, ve], -1).flatten(-2)


def packed_cache(k, v, table):
    """A PackedCache that holds pages of values (rounded)."""
    (kc, ke), (vc, ve) = pack(k), pack(v)
    return httm.PackedCache(kc, vc, scales_of(ke, ve).contiguous(), table)


def values_of(cache):
    """k, v of all pages in 64 bits."""
    return unpack(cache.k_codes, cache.scales[..., 0::2]), unpack(cache.v_codes, cache.scales[..., 1::2])


class PackedBatch(Batch):
    """Batch over a cache in 4 bits: rows that no sequence has are NaN."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.repack(self.cache.k_pages, self.cache.v_pages)

    def repack(self, k_pages, v_pages):
        table, page = self.cache.page_table, self.cache.page_size
        self.cache = packed_cache(k_pages, v_pages, table)
        k, v = values_of(self.cache)
        for b, m in enumerate(self.lens):
            pages = table[b, :-(-m // page)].long()
            for rows, x in ((self.k, k), (self.v, v)):
                rows[b] = x[pages].transpose(0, 1).flatten(1, 2)[:, :m].to(torch.bfloat16)
