"""The key/value cache's binding refuses tensors that are not on the call's GPU, before any call of the library.

The tensors are stand-ins: host tensors that say which GPU they are on.  The library is replaced by a recorder, so
nothing reaches a GPU, and a call that is let through is seen."""

import types

import pytest

torch = pytest.importorskip("torch")
api = pytest.importorskip("paper_2609_16338_amd.api")
from paper_2609_16338_amd import _native as N  # noqa: E402


class On:
    """A host tensor that says it is on a GPU (None: on the host)."""

    def __init__(self, t, gpu=0):
        self._t, self._gpu = t, gpu
        self.is_cuda = gpu is not None
        self.device = torch.device("cpu") if gpu is None else torch.device("cuda", gpu)

    def get_device(self):
        return -1 if self._gpu is None else self._gpu

    def __getattr__(self, name):
        return getattr(self._t, name)


TOKENS, REQUESTS = 3, 2


@pytest.fixture
def calls(monkeypatch):
    made = []
    note = lambda name: lambda *a: made.append(name) or N.OK  # noqa: E731
    monkeypatch.setattr(N, "lib", lambda: types.SimpleNamespace(**{name: note(name) for name in N.KV_SIGNATURES}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    return made


def _cache(gpu=0):
    return api.KVCache(*(On(torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), gpu) for _ in range(2)))


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _plan(monkeypatch, odd, gpu, **more):
    real = torch.zeros
    where = lambda name: gpu if name == odd else 0  # noqa: E731
    args = {name: On(t, where(name)) for name, t in (("kv_len", _i32(REQUESTS)), ("new_len", _i32(REQUESTS)), ("table", _i32(REQUESTS, 4)),
                                                     ("ring", _i32(9)), ("ring_state", torch.zeros(2, dtype=torch.int64)))}
    monkeypatch.setattr(torch, "zeros", lambda n, dtype, device: On(real(n, dtype=dtype), torch.device(device).index))
    plan = api.StepPlan(REQUESTS, TOKENS, device="cuda:%d" % (where("plan") or 0))
    monkeypatch.setattr(torch, "zeros", real)
    api.kv_plan(**args, page_size=16, plan=plan, **more)


def _append(monkeypatch, odd, gpu, **more):
    t = {"k": torch.zeros(TOKENS, 2, 64), "v": torch.zeros(TOKENS, 2, 64), "q": torch.zeros(TOKENS, 4, 64),
         "q_out": torch.zeros((TOKENS, 4, 64), dtype=torch.bfloat16), "slots": _i32(TOKENS), "positions": _i32(TOKENS),
         "cos": torch.zeros(10, 32), "sin": torch.zeros(10, 32)}
    a = {name: On(x, gpu if name == odd else 0) for name, x in t.items()}
    rope = (a.pop("cos"), a.pop("sin"))
    api.kv_append(_cache(gpu if odd == "cache" else 0), **a, rope=rope, **more)


def _attend(monkeypatch, odd, gpu, **more):
    t = {"q": torch.zeros((TOKENS, 4, 64), dtype=torch.bfloat16), "out": torch.zeros((TOKENS, 4, 64), dtype=torch.bfloat16),
         "table": _i32(REQUESTS, 4), "kv_len": _i32(REQUESTS), "cu_q": _i32(REQUESTS + 1), "workspace": torch.zeros(64, dtype=torch.uint8),
         "lse": torch.zeros(TOKENS, 4)}
    a = {name: On(x, gpu if name == odd else 0) for name, x in t.items()}
    api.paged_attention(cache=_cache(gpu if odd == "cache" else 0), max_q=2, max_kv=10, **a, **more)


CALLS = [(_plan, ("kv_len", "new_len", "table", "ring", "ring_state", "plan")),
         (_append, ("cache", "k", "v", "q", "q_out", "slots", "positions", "cos", "sin")),
         (_attend, ("cache", "q", "out", "table", "kv_len", "cu_q", "workspace", "lse"))]


@pytest.mark.parametrize("call,odd", [(call, name) for call, names in CALLS for name in names])
def test_a_tensor_of_another_gpu_is_refused(call, odd, calls, monkeypatch):
    with pytest.raises(ValueError):
        call(monkeypatch, odd, 1)
    assert not calls


@pytest.mark.parametrize("call,odd", [(call, name) for call, names in CALLS for name in names if name not in ("plan", "cache")])
def test_a_host_tensor_is_refused(call, odd, calls, monkeypatch):
    with pytest.raises(ValueError):
        call(monkeypatch, odd, None)
    assert not calls


@pytest.mark.parametrize("call", [call for call, _ in CALLS])
def test_tensors_of_the_current_gpu_are_taken(call, calls, monkeypatch):
    call(monkeypatch, None, None)
    call(monkeypatch, None, None, stream=types.SimpleNamespace(cuda_stream=5, device_index=0))
    call(monkeypatch, None, None, stream=5)
    assert len(calls) == 3


@pytest.mark.parametrize("call", [call for call, _ in CALLS])
def test_another_current_gpu_or_stream_is_refused(call, calls, monkeypatch):
    with pytest.raises(ValueError):
        call(monkeypatch, None, None, stream=types.SimpleNamespace(cuda_stream=5, device_index=1))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError):
        call(monkeypatch, None, None)
    assert not calls


def test_a_plan_on_the_host_is_refused():
    for device in ("cpu", torch.device("cpu")):
        with pytest.raises(ValueError):
            api.StepPlan(3, 5, device=device)
