"""Outputs over what every wave of a launch reads to find its work, or over the shared prefix: refused on the host.  The addresses here are made up."""
import ctypes as C

import pytest

import paper_2511_21317_amd as httm
from test_operator_refusals import INVALID, SMALL, norm_rope, rows
from test_packed_refusals import A, K, S, T, V, call_read, call_weigh, packed

# 2 sequences, a table of 2 x 4: offsets 12 bytes, lengths 8, the table 32
OFF, LENS, FREE = A, A + 4096, 40 << 20
BATCH = [OFF, OFF + 8, LENS, LENS + 4, T, T + 28]


@pytest.mark.parametrize("scales", [S, None])
@pytest.mark.parametrize("at", BATCH)
def test_weights(at, scales):
    """2 sequences of 1 head and 64 columns: 512 bytes"""
    for weights in (at, at - 508):
        assert call_weigh(scales=scales, offsets=OFF, seq_lens=LENS, weights=weights) == INVALID


@pytest.mark.parametrize("n", [0, 5])
def test_weights_of_steps_without_tokens(n):
    assert call_weigh(offsets=OFF, seq_lens=LENS, weights=T - 508, n=n) == INVALID


@pytest.mark.parametrize("scales", [S, None])
@pytest.mark.parametrize("at", BATCH)
def test_rows_that_are_read(at, scales):
    """5 tokens of 1 head: 640 bytes"""
    at -= at % 16
    for out in (at, at - 640 + 16):
        assert call_read(scales=scales, offsets=OFF, seq_lens=LENS, k_out=out) == INVALID
        assert call_read(scales=scales, offsets=OFF, seq_lens=LENS, v_out=out) == INVALID


def call_append(scales=S, q_out=FREE, q=None, k=None, v=None, offsets=OFF, lens=LENS, n=5, dtype=0, pos=20 << 20):
    """5 tokens of 1 head into 10 pages of 16 rows: 5120 bytes of codes, 640 of scales"""
    r = [x or rows(data=(30 + i) << 20, token_stride=64) for i, x in enumerate((q, k, v))]
    L, nr = httm.lib(), C.byref(norm_rope(axes=1))
    args = nr, *map(C.byref, r), dtype, pos, 0, n, 1, 64, C.byref(packed())
    if scales:
        return L.httm_cache_append_mx4(*args, scales, offsets, lens, q_out, None)
    return L.httm_cache_append(*args, offsets, lens, q_out, None)


@pytest.mark.parametrize("scales", [S, None])
@pytest.mark.parametrize("at", [*BATCH, 20 << 20, (20 << 20) + 16])
def test_queries_of_an_append(at, scales):
    """Over what finds the tokens' places and positions: rows would go to others' places"""
    at -= at % 16
    for out in (at, at - 640 + 16):
        assert call_append(scales, q_out=out) == INVALID


@pytest.mark.parametrize("at", [K, K + 5120 - 16, V, V + 5120 - 16, S, S + 640 - 16])
def test_an_append_in_4_bits_over_its_pages(at):
    for out in (at, at - 640 + 16):
        assert call_append(q_out=out) == INVALID
    for name in ("q", "k", "v"):
        for dtype, row in ((0, 128), (1, 128), (2, 256)):
            assert call_append(dtype=dtype, **{name: rows(data=at, token_stride=64)}) == INVALID
            assert call_append(dtype=dtype, **{name: rows(data=at - 4 * row - row + 16, token_stride=64)}) == INVALID


KP, VP = 60 << 20, 61 << 20


def attend(scales=S, o=FREE, lse=41 << 20, size=1 << 30, P=7, entry="lse"):
    q = rows(data=30 << 20)
    args = C.byref(q), KP, VP, P, C.byref(packed())
    rest = OFF, LENS, 5, 1, 64, 0.125, 0, o
    if entry == "lse":
        return httm.lib().httm_attention_cached_lse(*args, scales, *rest, lse, 70 << 20, size, None)
    return httm.lib().httm_attention_cached(*args, *rest, 70 << 20, size, None)


@pytest.mark.parametrize("scales", [S, None])
@pytest.mark.parametrize("at", [*BATCH, KP, KP + 7 * 128 - 4, VP, VP + 7 * 128 - 4])
def test_attention(at, scales):
    """5 tokens of 1 head: 20 bytes of sums, 640 of outputs; 7 rows of prefix"""
    for lse in (at, at - 16):
        assert attend(scales, lse=lse) == INVALID
    at -= at % 16
    for o in (at, at - 640 + 16):
        assert attend(scales, o=o) == INVALID
        assert attend(scales, o=o, lse=None) == INVALID
        assert attend(o=o, entry="plain") == INVALID
        assert attend(scales, o=o, size=0) == SMALL
