"""attention_cached where one query is not finite: it has its own row, and no other one's."""
import pytest
import torch

from test_gpu_attention_cached import Batch, D

pytestmark = pytest.mark.gpu


def batch(tiles, rest):
    """Sequences whose last tile has `rest` rows (in tiles of 256 rows: whose last wave has them)."""
    if tiles == "few rows":
        return Batch([rest, 3], [rest + 40, 50], 700, 4, 4, 16, seed=rest)
    if tiles == "few rows, together":       # 64 rows of all sequences a tile
        return Batch([1] * (64 + rest), [20 + i % 50 for i in range(64 + rest)], 3001, 4, 4, 16, seed=rest)
    if tiles == "256 rows":
        return Batch([256 + rest, 256 + rest], [300 + rest, 800], 16001, 4, 4, 16, seed=rest)
    n = 1024 + rest                         # 12 rows a sequence, 256 of all a tile
    new = [12] * (n // 12) + ([n % 12] if n % 12 else [])
    return Batch(new, [20 + i % 50 for i in range(len(new))], 3501, 4, 4, 16, seed=rest)


TILES = ["few rows", "few rows, together", "256 rows", "256 rows, together"]


@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("rest", [2, 17, 40, 48])
@pytest.mark.parametrize("tiles", TILES, ids=lambda s: s.replace(", ", "_").replace(" ", "_"))
def test_a_query_that_is_not_finite_has_its_own_row_alone(tiles, rest, value, rising):
    b = batch(tiles, rest)
    if rising:      # the shift has to follow all along the prefix
        b.kp *= torch.linspace(0.01, 60.0, b.P, device="cuda")[None, :, None].bfloat16()
    ref, tol = (t.view(b.n, b.H_q, D) for t in b.reference(True))
    # the last row of all, one in the middle and the first one, in a head each
    spoilt = [(b.off[-1] - 1, 1), (b.off[1] - 1, 2), (b.off[-1] // 2, 3), (b.off[0], 0)]
    fine = torch.ones(b.n, b.H_q, dtype=torch.bool, device="cuda")
    for t, h in spoilt:
        b.q[t, h, 5] = float(value)
        fine[t, h] = False
    got = b.run(True).view(b.n, b.H_q, D)
    bad = ~((got.double() - ref).abs() <= tol)[fine]
    assert not bad.any(), f"{int(bad.any(-1).sum())} of {bad.shape[0]} other rows off, {int(torch.isnan(got[fine]).any(-1).sum())} of them NaN"
    if value == "nan":
        assert torch.isnan(got[~fine]).all()


@pytest.mark.parametrize("new,lens,P", [([70], [170], 300), ([300, 530], [300, 700], 16001)], ids=["few_rows", "256_rows"])
def test_a_key_that_is_not_finite_reaches_later_rows_alone(new, lens, P):
    """Every token's own key is far above all that it has seen, and one token's is NaN: the shifts of the rows in front of it follow."""
    H = 4
    b = Batch(new, lens, P, H, H, 16, seed=7)
    for i, (n, m) in enumerate(zip(new, lens)):
        b.k[i][:, m - n:] = 30 * b.q[b.off[i]:b.off[i + 1]].transpose(0, 1)
        j = torch.arange(m)
        b.cache.k_pages[b.cache.page_table[i, (j // 16).cuda()].long(), :, (j % 16).cuda()] = b.k[i].transpose(0, 1)
    ref, tol = (t.view(b.n, H, D) for t in b.reference(True))
    hit = torch.zeros(b.n, dtype=torch.bool, device="cuda")
    for i, (n, m) in enumerate(zip(new, lens)):
        at = n - 19         # (the rows in front of it that share a step of 32 keys and a lane with rows behind it)
        row = m - n + at
        b.cache.k_pages[int(b.cache.page_table[i, row // 16]), :, row % 16, 9] = float("nan")
        hit[b.off[i] + at:b.off[i + 1]] = True
    got = b.run(True).view(b.n, H, D)
    assert torch.isnan(got[hit]).all()
    bad = ~((got.double() - ref).abs() <= tol)[~hit]
    assert not bad.any(), f"{int(bad.any(-1).sum())} of {bad.shape[0]} rows in front off"
