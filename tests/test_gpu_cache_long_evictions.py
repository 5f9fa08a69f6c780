"""Evictions of more rows than the selection holds in the LDS: 32 768 between the first and the last ones; it takes the others from memory."""
import pytest

from test_gpu_cache_budget import Evicted

pytestmark = pytest.mark.gpu

# lengths, key heads, page, keep, first, last.  A wave of the selection has a sixteenth of the rows between the first and last ones, in runs of 64, and 32
# of its runs in the LDS.
LONG = {
    # 39 301 between: 39 runs a wave, of 2496 rows; of those alike the first 7 waves and 2300 rows of the eighth stay
    "border in memory": ([40011, 39000], 2, 64, 7 * 2496 + 2300 + 710, 10, 700),
    "border in the LDS": ([40011, 33000, 5], 1, 64, 7 * 2496 + 900 + 710, 10, 700),
    "one row too many": ([32768 + 1 + 4 + 256, 32768 + 4 + 256], 2, 256, 20000, 4, 256),
    "almost all stay": ([40000, 36000], 1, 128, 35999, 0, 1374),
    "very few stay": ([70001], 1, 256, 300, 4, 256),
    "first and last": ([50000], 1, 256, 2000, 1500, 500),
}


@pytest.mark.parametrize("weights,store", [(None, "mx4"), ("few values", "bf16"), ("alike", "mx4"), ("alike", "bf16"), ("strange", "bf16")])
@pytest.mark.parametrize("case", LONG, ids=lambda s: s.replace(" ", "_"))
def test_long_evictions(case, weights, store):
    lens, H, page, keep, first, last = LONG[case]
    assert max(lens) - first - last > 32768
    Evicted(store, lens, H, page, seed=len(case), weights=weights, more=3).check(keep, first, last)
