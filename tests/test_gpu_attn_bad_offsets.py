"""bitcos_paged_attn on the GPU with a cu_q that does not ascend: rows hold some request's result or what they held, and
nothing else is touched."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
api = pytest.importorskip("paper_2609_16338_amd.api")
from paper_2609_16338_amd import _native as N  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    N.lib()


@pytest.mark.parametrize("max_q", [1, 200])
def test_every_other_request_names_all_tokens(max_q):
    """More key tiles than can be counted (15000 requests of 30000 tokens and 2^24 tiles each): nothing is done."""
    n, page, width, dim, hq = 30000, 1 << 20, 512, 64, 16
    cache = api.KVCache(*(torch.ones((1, 1, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table = torch.zeros((n, width), dtype=torch.int32, device="cuda")
    cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    cu[1::2] = n
    kv = torch.full((n,), width * page, dtype=torch.int32, device="cuda")
    q = torch.ones((n, hq, dim), dtype=torch.bfloat16, device="cuda")
    space = torch.full((n + 2, hq, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, hq), 9.0, device="cuda")
    ws = torch.empty(api.paged_attention_workspace(cache, n, n, hq, max_q, width * page), dtype=torch.uint8, device="cuda")
    api.paged_attention(q, cache, table, kv, cu, space[1:-1], ws, max_q=max_q, max_kv=width * page, lse=lse)
    torch.cuda.synchronize()
    assert bool((space == 9.0).all()) and bool((lse == 9.0).all())


@pytest.mark.parametrize("max_q", [1, 200])
def test_requests_that_share_tokens(max_q):
    """Few of them: every row is one of the requests' results (their keys are the same, so the results are, too)."""
    n, page, dim, hq = 40, 16, 64, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = api.KVCache(*(torch.randn((4, 1, page, dim), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)))
    table = torch.tensor([[2, 0, 3]] * 5, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn((n, hq, dim), device="cuda", generator=g).to(torch.bfloat16)
    out = [torch.full((n + 2, hq, dim), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for space, cu, kv in ((out[0], i32(0, n, 0, n, 0, n), i32(*[44] * 5)), (out[1], i32(0, n, n, n, n, n), i32(44, *[0] * 4))):
        ws = torch.empty(api.paged_attention_workspace(cache, n, 5, hq, max_q, 44), dtype=torch.uint8, device="cuda")
        api.paged_attention(q, cache, table, kv, cu, space[1:-1], ws, max_q=max_q, max_kv=44)
    torch.cuda.synchronize()
    # The same keys in other parts: results and weights are rounded to bfloat16 on either side, 2^-8 of each.
    size = out[1].double().abs() + float(cache.v.double().abs().max())
    assert bool(((out[0].double() - out[1].double()).abs() <= 2.0 ** -7 * size).all())
    for space in out:
        assert bool((space[0] == 9.0).all()) and bool((space[-1] == 9.0).all())
