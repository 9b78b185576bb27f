"""The key/value cache's binding refuses numbers that do not fit the C ABI's 32 bits, which would arrive as others (no GPU).

The stand-ins for GPU tensors and the recorder in place of the library are those of test_kv_devices."""

import pytest

from test_kv_devices import On, _attend, _cache, _plan, calls  # noqa: F401

torch = pytest.importorskip("torch")
api = pytest.importorskip("paper_2609_16338_amd.api")

PAST = [2**31, 2**32, 2**32 + 5, 2**63]


@pytest.mark.parametrize("value", PAST)
@pytest.mark.parametrize("name", ["window", "max_q", "max_kv"])
def test_attention(name, value, calls, monkeypatch):  # noqa: F811
    real = api.paged_attention
    with monkeypatch.context() as m:
        m.setattr(api, "paged_attention", lambda **a: real(**(a | {name: value})))
        with pytest.raises(ValueError):
            _attend(monkeypatch, None, None)
    assert not calls
    m = {"window": 2**31 - 1} if name == "window" else {}
    _attend(monkeypatch, None, None, **m)
    assert len(calls) == 1


@pytest.mark.parametrize("value", PAST)
@pytest.mark.parametrize("name", ["tokens", "requests", "q_heads", "max_q", "max_kv"])
def test_workspace(name, value, calls):  # noqa: F811
    counts = dict(tokens=4, requests=2, q_heads=8, max_q=2, max_kv=100) | {name: value}
    with pytest.raises(ValueError):
        api.paged_attention_workspace(_cache(), **counts)
    assert not calls


@pytest.mark.parametrize("value", PAST)
def test_page_size(value, calls, monkeypatch):  # noqa: F811
    real = api.kv_plan
    monkeypatch.setattr(api, "kv_plan", lambda **a: real(**(a | {"page_size": value})))
    with pytest.raises(ValueError):
        _plan(monkeypatch, None, None)
    assert not calls


@pytest.mark.parametrize("pages,page", [(2**32 + 1, 16), (1, 2**32 + 16), (2**31, 1), (2**20, 2**20)])
def test_caches(pages, page):
    k = On(torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16).expand(pages, 1, page, 64))
    with pytest.raises(ValueError):
        api.KVCache(k, k)
