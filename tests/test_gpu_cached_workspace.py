"""Attention in the smallest workspace that a call takes: the results are right, and what lies behind the workspace stays."""
import pytest
import torch

import paper_2511_21317_amd as httm
from mx4_util import PackedBatch
from test_gpu_attention_cached import Batch, spread

pytestmark = pytest.mark.gpu


def run_in(b, size, causal):
    """attention with `size` bytes of workspace in front of a mark"""
    room = torch.full((size + 4096,), 0xC3, dtype=torch.uint8, device="cuda")
    got = b.run(causal, ws=room[:size])
    assert (room[size:] == 0xC3).all()
    with pytest.raises(httm.HttmError):
        b.run(causal, ws=room[:size - 1])
    return got


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("new,lens,P,H_q,H_kv,one,apart", [
    ([1] * 64, spread(1, 200, 64), 3000, 32, 8, 14123008, 41156608), ([1] * 10, spread(1, 900, 10), 28700, 2, 1, 10877952, 37962240),
    ([1, 3, 0, 4, 2] * 4, spread(5, 100, 20), 12000, 8, 4, None, None), ([100, 30], [100, 90], 500, 4, 2, None, None)])
def test_smallest_workspace(new, lens, P, H_q, H_kv, one, apart, causal):
    b = Batch(new, lens, P, H_q, H_kv, 16, seed=3)
    size = b.ws.numel() if one is None else one
    got = b.run(causal)
    if one is not None:
        assert b.ws.numel() == apart
        assert torch.equal(run_in(b, one, causal), got)
        b = PackedBatch(new, lens, P, H_q, H_kv, 16, seed=3)
        assert torch.equal(run_in(b, size, causal), b.run(causal))
    b.check(causal)


@pytest.mark.parametrize("causal", [False, True])
def test_smallest_workspace_with_the_prefix_in_a_launch_of_its_own(causal):
    b = PackedBatch([1] * 20, spread(5, 20000, 20), 6201, 4, 4, 64, seed=4)
    assert b.cache.page_table.numel() * 64 * 4 > 1000000
    assert torch.equal(run_in(b, b.ws.numel(), causal), b.check(causal))
