"""attention_cached: every key counts once, exactly.  All weights are equal (q = 0), and the values mark 8192 keys at a time, 128 in a channel: a
channel is its number of keys over all that the row sees, in which one key lost or doubled is 1/128, twice what a rounding may be."""
import pytest
import torch

from test_gpu_attention_cached import SHAPES, Batch, D

pytestmark = pytest.mark.gpu

RUN = 128       # keys in a channel
WINDOW = RUN * D


def own_rows(b):
    """(page, row in the page, index of the key) of all rows in the cache."""
    page_size, table = b.cache.page_size, b.cache.page_table.cpu()
    pages, rows, keys = [], [], []
    for i, m in enumerate(b.lens):
        j = torch.arange(m)
        pages.append(table[i, j // page_size].long()), rows.append(j % page_size), keys.append(b.P + j)
    return [torch.cat(t).cuda() for t in (pages, rows, keys)]


def marks(keys, start):
    """[keys, 64]: 1 in the channel of a key's run of the window from `start` on."""
    channel = torch.div(keys - start, RUN, rounding_mode="floor")
    return (channel[:, None] == torch.arange(D, device="cuda")).bfloat16()


def seen_of_window(m, start):
    """[rows, 64]: how many of the keys 0 .. m - 1 are in a channel's run."""
    lo = start + RUN * torch.arange(D, device="cuda")
    return (torch.minimum(m[:, None], lo + RUN) - lo).clamp(min=0)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.replace(" ", "_"))
def test_every_key_counts_once(shape, causal):
    b = Batch(*SHAPES[shape], seed=1, pad_front=3, pad=4)
    b.q.zero_()
    page, row, key = own_rows(b)
    # keys that a token sees, as a prefix of the prefix and its sequence's rows
    m = torch.zeros(b.n, dtype=torch.int64, device="cuda")
    for i, (n, length) in enumerate(zip(b.new, b.lens)):
        own = (length - n + 1 + torch.arange(n, device="cuda")).clamp(0, length) if causal else torch.full((n,), length, device="cuda")
        m[b.off[i]:b.off[i + 1]] = b.P + own
    real = slice(b.off[0], b.off[-1])
    for start in range(0, max(1, b.P + max(b.lens)), WINDOW):
        b.vp[:] = marks(torch.arange(b.P, device="cuda"), start)
        b.cache.v_pages[page, :, row] = marks(key, start)[:, None]
        got = b.run(causal).double().view(b.n, b.H_q, D)
        assert (got[:b.off[0]] == 5).all() and (got[b.off[-1]:] == 5).all()
        ref = (seen_of_window(m, start).double() / m.clamp(min=1)[:, None].double())[real, None]
        # weights are 1 and sums whole numbers; a reciprocal and a product in fp32, half a bf16 step of the result
        bad = (got[real] - ref).abs() > ref * (2.0 ** -8 + 2.0 ** -21)
        assert not bad.any(), f"keys from {start}: {int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}"
