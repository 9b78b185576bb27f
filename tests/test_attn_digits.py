"""How many digits the weights of attention keep: a bound for each kernel by its own rounding of them.

The few-row kernels multiply values by weights of twice bfloat16's digits (an upper and a lower half: off by 2^-8 of
2^-8), the general kernel by fp32 ones, the many-row kernels by bfloat16 ones (2^-8).  For this to show, everything
else has to be small: queries have four values, so a score is a sum of four products, and keys are few.  The result is
rounded to bfloat16 (2^-8 of it).  With `weight` = sum p |v| / l and `size` = the largest sum |q k| of a row:
  |error| <= 2^-8 (1 + 2^-6) |out| + (1 + 2^-6) (w + 2 d + (keys + 48) 2^-24) weight,
  d = (4 + 16) 2^-24 size + 2^-21 (a score's error: its products' sum, two factors, the exponential's own),
with w the weights' rounding as above and (keys + 48) 2^-24 that of the sums over keys and parts."""

import types

import pytest

import kv_reference as ref

torch = pytest.importorskip("torch")

FEW, MANY, GENERAL = 2.0 ** -16, 2.0 ** -8, 2.0 ** -24


def _inside(got, want, keys, w):
    out, _, weight, size = want
    d = (4 + 16) * 2.0 ** -24 * size + 2.0 ** -21
    more = 1 + 2.0 ** -6
    bound = 2.0 ** -8 * more * out.abs() + more * (w + 2 * d[..., None] + (keys + 48) * 2.0 ** -24) * weight + 1e-30
    return bool(((got.double() - out).abs() <= bound).all())


def _four_values(q, seed):
    g = torch.Generator(device=q.device).manual_seed(seed)
    at = torch.rand(q.shape, device=q.device, generator=g).argsort(dim=-1)[..., :4]
    return torch.zeros_like(q).scatter(-1, at, torch.randn(at.shape, device=q.device, generator=g).to(q.dtype))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv", [20, 100, 1000])
def test_the_bound_tells_one_half_from_two(kv, dim):
    """On the CPU: the arithmetic of the kernels, with the weights' lower half, without it, and with the wrong sign."""
    g = torch.Generator().manual_seed(kv)
    k, v = (torch.randn((-(-kv // 16), 1, 16, dim), generator=g).to(torch.bfloat16) for _ in range(2))
    cache = types.SimpleNamespace(k=k, v=v, k_scale=None, v_scale=None, pages=k.shape[0], kv_heads=1, page_size=16, head_dim=dim)
    q = _four_values(torch.zeros((1, 8, dim), dtype=torch.bfloat16), kv)
    want = ref.attention(q, cache, torch.arange(k.shape[0])[None, :], [kv], [0, 1], 1.0)
    kk, vv = (x.reshape(-1, dim)[:kv].float() for x in (k, v))
    s = q[0].float() @ kk.t()
    p = torch.exp(s - s.amax(dim=1, keepdim=True))
    hi = p.to(torch.bfloat16).float()
    lo = (p - hi).to(torch.bfloat16).float()
    result = lambda weights: (weights @ vv / p.sum(dim=1, keepdim=True)).to(torch.bfloat16)[None]  # noqa: E731
    assert _inside(result(p), want, kv, GENERAL)
    assert _inside(result(hi + lo), want, kv, FEW)
    assert _inside(result(hi), want, kv, MANY)
    assert not _inside(result(hi), want, kv, FEW)
    assert not _inside(result(hi - lo), want, kv, FEW)
    assert not _inside(result(hi), want, kv, GENERAL)


def _gpu_check(lens, hq, hk, dim, dtype, w, **more):
    from test_gpu_paged_attn import Case
    from paper_2609_16338_amd import _native as N
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    N.lib()
    c = Case(lens, hq, hk, dim, 16, dtype, seed=hq + dim)
    c.q = _four_values(c.q, 1)
    out, _ = c.run(scale=1.0, **more)
    want = ref.attention(c.q, c.cache, c.table, c.kv, c.cu, 1.0)
    assert bool(torch.isfinite(want[0]).all())
    assert _inside(out, want, max(c.kv), w)


TYPES = [torch.bfloat16, torch.int8]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,hq,hk,n", [(128, 1, 1, 1), (128, 40, 8, 1), (128, 8, 2, 4), (128, 8, 2, 8), (128, 32, 1, 1), (64, 24, 4, 1), (64, 24, 4, 5),
                                         (64, 8, 1, 8), (64, 1, 1, 16)])
def test_few_rows(dim, hq, hk, n, dtype):
    """Whole items and, with 1000 keys, items in parts."""
    _gpu_check([(kv, min(kv, n)) for kv in (1, 17, 33, 100, 300)], hq, hk, dim, dtype, FEW)
    _gpu_check([(1000, n)], hq, hk, dim, dtype, FEW)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,n", [(128, 40), (64, 100)])
def test_many_rows(dim, n, dtype):
    _gpu_check([(n, n), (300, n), (200, 1)], 8, 2, dim, dtype, MANY)
    _gpu_check([(1000, n)], 8, 2, dim, dtype, MANY)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [80, 96, 256])
def test_other_heads(dim, dtype):
    _gpu_check([(n + kv, n) for n, kv in ((1, 0), (3, 100), (20, 300))], 6, 2, dim, dtype, GENERAL)
