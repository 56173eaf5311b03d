"""Every form of the two expert products, against the formula in 64 bits (helpers and tolerances: test_gpu_moe.py, whose limits on D
and F hold here).  What chooses a form is the tokens, the tokens an expert, and the tiles of 16 rows against the experts: four tiles
a workgroup, two or one, with one, two or four groups of 16 columns, in either product; up to four tokens routed by the first
product's workgroups, more by a kernel for up to 64 experts or for more; grids over experts or over (token, expert) pairs."""
import pytest
from test_gpu_moe import check, make

pytestmark = pytest.mark.gpu

FOUR_TOKENS = [(4, 64, 40, 8, 2), (4, 104, 72, 40, 8), (4, 200, 520, 70, 16), (4, 1000, 136, 64, 16), (4, 264, 120, 200, 16)]  # 16: 64 pairs
FIVE_TOKENS = [(5, 264, 120, 40, 8), (5, 264, 520, 70, 8), (5, 1000, 136, 130, 3), (5, 64, 40, 8, 2)]
FOUR_TILES = [(16, 200, 520, 8, 4), (13, 200, 528, 8, 5), (25, 200, 520, 20, 7), (128, 200, 520, 8, 2), (125, 200, 520, 9, 3),       # first product
              (15, 1000, 200, 9, 5), (16, 1000, 88, 8, 8), (29, 1000, 200, 16, 5), (128, 1000, 200, 8, 2), (117, 1000, 200, 9, 3)]  # second
FOUR_GROUPS = [(128, 120, 360, 8, 2), (128, 120, 120, 8, 2), (128, 704, 200, 8, 2), (40, 520, 264, 7, 4), (31, 376, 1000, 24, 6)]
FEWER_PAIRS = [(100, 200, 104, 256, 2), (128, 72, 40, 200, 1), (70, 104, 520, 150, 2), (9, 264, 200, 64, 4), (17, 104, 136, 40, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,F,E,k", FOUR_TOKENS + FIVE_TOKENS + FOUR_TILES + FOUR_GROUPS + FEWER_PAIRS)
def test_values(dtype, n, D, F, E, k):
    a = make(n, D, F, E, dtype, seed=n + D + E)
    check(a, k, True)
    a["residual"] = None
    check(a, k, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,F,E,k", [(4, 104, 72, 40, 8), (100, 200, 520, 20, 3), (121, 1000, 200, 16, 2), (128, 200, 520, 8, 2), (127, 1000, 200, 8, 2),
                                       (100, 200, 104, 256, 2), (128, 72, 40, 200, 1)])
def test_all_tokens_with_the_same_experts(dtype, n, D, F, E, k):
    """More columns than an expert's groups hold at a time, and a last group that is not full; rows of x differ in scale alone."""
    import torch
    a = make(n, D, F, E, dtype, seed=n + E)
    a["x"] = (a["x"][:1].float() * torch.linspace(0.5, 2, n, device="cuda")[:, None]).to(a["x"].dtype)
    check(a, k, True)
    check(a, k, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,E,k", [(4, 40, 8), (5, 64, 3), (66, 200, 2), (128, 8, 2)])
def test_a_token_that_is_not_finite_stays_alone(dtype, n, E, k):
    import torch
    a = make(n, 200, 520, E, dtype, seed=n)
    good = check(a, k)
    a["x"][n - 2, 77] = float("nan")
    got = check(a, k, rows=[t for t in range(n) if t != n - 2])
    for t in range(n):
        assert torch.isnan(got[t]).all() if t == n - 2 else torch.equal(got[t], good[t]), t
