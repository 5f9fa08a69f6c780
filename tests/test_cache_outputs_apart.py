"""Outputs over what every wave of a launch reads to find its work, or over the shared prefix: refused on the host.  The addresses here are made up."""
import ctypes as C

import pytest

import paper_2511_21317_amd as httm
from test_operator_refusals import INVALID, SMALL, rows
from test_packed_refusals import A, S, T, call_read, call_weigh, packed

# 2 sequences, a table of 2 x 4: offsets 12 bytes, lengths 8, the table 32
OFF, LENS = A, A + 4096
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


KP, VP, FREE = 60 << 20, 61 << 20, 40 << 20


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
