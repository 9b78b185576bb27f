"""bitcos_paged_attn on the GPU where a row's scores are all the same huge finite number.

Every query and key has one value, so every score is one product: the same for all keys of a row, whatever rounding it
has.  Then the weights are equal and the result is the mean of the values.  Bounds: bfloat16 rounds the result (2^-8 of
it) and the weights times an int8 value's scale (2^-8 of the mean of |v|), sums over `keys` fp32 terms are off by
(keys + 32) 2^-24 of it; lse is the score, a product of up to five fp32 factors, and ln(keys): 2^-20 of its size."""

import math

import pytest

from test_gpu_paged_attn import TYPES, Case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
api = pytest.importorskip("paper_2609_16338_amd.api")
from paper_2609_16338_amd import _native as N  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    N.lib()


def _check(c, scale, low, high, seed, same=False):
    """Scores spread over the exponents from low to high, of both signs; `same`: one score for all rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, dim = c.cache.k, c.cache.head_dim
    k.zero_()
    if c.cache.k_scale is None:
        k[..., 0] = 3.0
        c.cache.v.nan_to_num_(0.0)
        key = 3.0
    else:
        k[..., 0] = 1
        c.cache.k_scale.fill_(2.9)
        c.cache.v_scale.nan_to_num_(0.0)
        key = float(c.cache.k_scale.flatten()[0])
    size = torch.exp(math.log(low) + math.log(high / low) * torch.rand(c.q.shape[:2], device="cuda", generator=g, dtype=torch.float64))
    sign = torch.randint(0, 2, c.q.shape[:2], device="cuda", generator=g) * 2 - 1
    if same:
        size[:], sign[:] = size[0, 0].clone(), sign[0, 0].clone()
    c.q.zero_()
    c.q[..., 0] = (size * sign / (abs(scale) * key)).to(torch.bfloat16)
    score = c.q[..., 0].double() * key * scale
    out, lse = c.run(scale=scale, causal=False)
    group = c.hq // c.cache.kv_heads
    for r, kv in enumerate(c.kv):
        ids = c.table[r, :-(-kv // c.page)].long()
        rows = slice(c.cu[r], c.cu[r + 1])
        for h in range(c.hq):
            v = c.cache.v[ids, h // group].double()
            if c.cache.v_scale is not None:
                v = v * c.cache.v_scale[ids, h // group].double()[..., None]
            v = v.reshape(-1, dim)[:kv]
            mean, size = v.mean(dim=0), v.abs().mean(dim=0)
            bound = 2.0 ** -8 * mean.abs() + (2.0 ** -8 + (kv + 32) * 2.0 ** -24) * size
            got = out[rows, h].double()
            assert bool(((got - mean).abs() <= bound).all()), (r, h)
            want = score[rows, h] + math.log(kv)
            assert bool(((lse[rows, h].double() - want).abs() <= 2.0 ** -20 * want.abs()).all()), (r, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 80])
@pytest.mark.parametrize("n", [1, 6, 40, 150])
@pytest.mark.parametrize("low,high", [(1e5, 1e10), (1e10, 1e37)])
@pytest.mark.parametrize("scale", [0.09, -1.0])
def test_equal_scores(scale, low, high, n, dim, dtype):
    _check(Case([(n, n), (n + 77, n), (400, n)], 8, 2, dim, 16, dtype, seed=n), scale, low, high, 31)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv,n", [(5000, 1), (5000, 6), (6000, 150), (9000, 40)])
@pytest.mark.parametrize("low,high", [(1e5, 1e10), (1e10, 1e37)])
def test_equal_scores_of_an_item_in_parts(low, high, kv, n, dim, dtype):
    _check(Case([(kv, n)], 4, 1, dim, 64, dtype, seed=n), 0.09, low, high, 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv,n", [(150, 150), (6000, 150)])
def test_one_score_for_all_rows(kv, n, dim, dtype):
    """No other row's infinities bring a row's vanished weights to light."""
    for seed in range(12):
        _check(Case([(kv, n)], 4, 1, dim, 64, dtype, seed=n), 0.09, 1e7, 1e37, 40 + seed, same=True)
