"""What workspace attention to a cache asks for, on the host: the addresses are made up, and a call whose workspace is large enough is refused
behind that check, for an output over its queries."""
import ctypes as C

import pytest

import paper_2511_21317_amd as httm
from test_operator_refusals import INVALID, SMALL, paged, rows

K, V, S, T, A, Q, W = (i << 32 for i in range(1, 8))

# tokens, sequences, query and key heads, rows of the prefix; bytes with the prefix and the own keys in one launch, and in one each
SHAPES = [(64, 64, 32, 8, 3000, 14123008, 41156608), (32, 32, 16, 16, 28700, 13398016, 41242624), (10, 10, 2, 1, 28700, 10877952, 37962240),
          (20, 20, 4, 4, 6201, 11238400, 38474752), (5, 2, 1, 1, 0, 6488320, 6488320), (4 * 1374, 4, 16, 16, 5516, 70612992, 70612992)]


def call(shape, size, scales=None, columns=16, entry="lse"):
    n, B, H_q, H_kv, P = shape
    cache = paged(k_pages=K, v_pages=V, page_table=T, n_pages=4, n_seqs=B, table_stride=columns, page_size=64, H_kv=H_kv)
    q = rows(data=Q, token_stride=64 * H_q, head_stride=64)
    L = httm.lib()
    if entry == "lse":
        return L.httm_attention_cached_lse(C.byref(q), K, V, P, C.byref(cache), scales, A, A, n, H_q, 64, 0.125, 0, Q, None, W, size, None)
    return L.httm_attention_cached(C.byref(q), K, V, P, C.byref(cache), A, A, n, H_q, 64, 0.125, 0, Q, W, size, None)


@pytest.mark.parametrize("entry", ["plain", "lse"])
@pytest.mark.parametrize("columns", [16, 4096])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_in_16_bits_go_in_one_launch_with_the_prefix(shape, columns, entry):
    *shape, one, _ = shape
    assert call(shape, one, columns=columns, entry=entry) == INVALID
    assert call(shape, one - 1, columns=columns, entry=entry) == SMALL


@pytest.mark.parametrize("shape", SHAPES)
def test_rows_in_4_bits_need_what_their_launches_do(shape):
    """Room for more than a million rows of all key heads in the page table: launches of their own, else one."""
    *shape, one, apart = shape
    B, H_kv = shape[1], shape[3]
    few = 1000000 // (64 * B * H_kv)
    for columns, need in ((few, one), (few + 1, apart)):
        assert call(shape, need, scales=S, columns=columns) == INVALID
        assert call(shape, need - 1, scales=S, columns=columns) == SMALL


@pytest.mark.parametrize("shape", SHAPES)
def test_the_query_is_enough_for_either(shape):
    *shape, one, apart = shape
    assert httm.attention_cached_workspace(*shape) == max(one, apart)
