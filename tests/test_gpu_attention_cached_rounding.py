"""attention_cached in tiles of 256 rows: a weight is rounded to bf16 once, also where the shift moves before its product."""
import math

import pytest
import torch

from test_gpu_attention_cached import Batch, D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("other", [200.0, 11.0])
def test_a_shift_that_moves_rounds_no_weight_again(other):
    """Scores in base 2.  Key 0 has 0 and sets the shift, key 37 has 9 and the only value, key 67 has a fraction t of the row's own, and for one
    row in 64 `other` on top, so that the shift of all its wave's rows moves by about t while the weight of key 37 waits for its product."""
    n, P, H = 1024, 8192, 16       # (a workgroup has some 900 keys of a tile, or more)
    b = Batch([n], [n], P, H, H, 16)
    t = (torch.arange(n, device="cuda") % 128) / 128.0
    b.q[:] = 0.0
    b.q[:, :, 0], b.q[:, :, 1] = 1.0, t[:, None].bfloat16()
    b.q[::64, :, 2] = 1.0
    for k, v in ((b.kp, b.vp), (b.k[0], b.v[0]), (b.cache.k_pages, b.cache.v_pages)):
        k[:], v[:] = 0.0, 0.0
        k[..., 0] = -100.0
    b.kp[:, 0, 0], b.kp[:, 37, 0], b.vp[:, 37] = 0.0, 9.0, 1.0
    b.kp[:, 67, 0], b.kp[:, 67, 1], b.kp[:, 67, 2] = 0.0, 1.0, other
    got = b.run(scale=math.log(2.0)).double()
    ref, _ = b.reference(scale=math.log(2.0))
    # Half a bf16 step of the result: 2^-8 of the power of two below it.  Half a step of every weight, in the product and in the sum that
    # divides it: for the row's one value 1, sum p |v - o| = 2 o (1 - o).  Scores are exact, but for a factor scale * log2(e) that is 1 to
    # 2^-22: 2^-22 * 9 of a weight; exp2 and sums of a hundred terms 2^-18.
    off = 2.0 ** -8 * 2 * ref * (1 - ref) + 2.0 ** -17 * ref + 1e-30
    tol = 2.0 ** -9 * torch.exp2(torch.frexp(ref + off).exponent.double()) + off
    err = (got - ref).abs()
    assert (err <= tol).all(), f"{int((err > tol).any(-1).sum())} of {n} rows off, worst {(err / tol).max():.2f} times"
