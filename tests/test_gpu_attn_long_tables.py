"""bitcos_paged_attn on the GPU at the longest lengths that a table can state: a window at the end of 2^31 keys, whose
results are those of the same pages at the start (bounds: kv_reference.check_attention)."""

import pytest

import kv_reference as ref
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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 80])
@pytest.mark.parametrize("n", [1, 5, 150])
@pytest.mark.parametrize("width", [(1 << 27) - 1, (1 << 27) - 513, (1 << 27) - 2000])
def test_windows_at_the_end_of_two_billion_keys(width, n, dim, dtype):
    """Widths on both sides of what the matrix-core kernels number."""
    c = Case([(304, n)], 8, 2, dim, 16, dtype, seed=n)
    want = ref.attention(c.q, c.cache, c.table, c.kv, c.cu, None, True, 100)
    table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
    table[0, -19:] = c.table[0, :19]
    kv = 16 * width
    out, lse = c.run(table=table, kv=[kv], max_kv=kv, window=100)
    ref.check_attention(out, lse, want, dim, 304)


def test_the_last_key_of_all():
    """One page of 2^31 - 1 tokens whose rows are one and the same: lse counts the keys seen."""
    dim, tokens = 8, (1 << 31) - 1
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((1, 1, 1, dim), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    cache = api.KVCache(*(x.expand(1, 1, tokens, dim) for x in (k, v)))
    q = torch.randn((3, 2, dim), device="cuda", generator=g).to(torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(api.paged_attention_workspace(cache, 3, 1, 2, 3, tokens), dtype=torch.uint8, device="cuda")
    api.paged_attention(q, cache, i32(0).view(1, 1), i32(tokens), i32(0, 3), out, ws, max_q=3, max_kv=tokens, window=1000, lse=lse)
    torch.cuda.synchronize()
    assert bool(((out.double() - v.double().view(1, 1, dim)).abs() <= 2.0 ** -8 * v.double().abs().view(1, 1, dim)).all())
    want = (q.double() * k.double().view(1, 1, dim)).sum(-1) / dim ** 0.5 + torch.log(torch.tensor(1000.0, dtype=torch.float64, device="cuda"))
    assert bool(((lse.double() - want).abs() <= 2.0 ** -14).all())
