"""bitcos_kv_append on the GPU with more rows than one launch of the vector kernel holds (2^32 threads)."""

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


@pytest.mark.parametrize("more", [-8, 0, 1000])
def test_rows_past_a_launch(more):
    """A padded step of 2^27 tokens, one row of each broadcast, of which a few have slots."""
    tokens, dim = (1 << 27) + more, 128
    cache = api.KVCache(*(torch.zeros((4, 1, 16, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    k, v = (torch.full((1, 1, dim), x, device="cuda").expand(tokens, 1, dim) for x in (3.0, 5.0))
    slots = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    slots[0], slots[tokens // 2], slots[-1] = 7, 40, 63
    api.kv_append(cache, k, v, slots)
    torch.cuda.synchronize()
    stored = torch.zeros(64, dtype=torch.bool, device="cuda")
    stored[[7, 40, 63]] = True
    for data, x in ((cache.k, 3.0), (cache.v, 5.0)):
        assert torch.equal(data.reshape(64, dim), torch.where(stored[:, None], x, 0.0).to(torch.bfloat16).expand(64, dim))
