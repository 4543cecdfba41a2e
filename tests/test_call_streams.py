"""Which stream the memory belongs to that the entry points make for themselves: the one that works on it.  No GPU: tensors that say they are on one, a library that does nothing."""
import pytest

torch = pytest.importorskip("torch")

import paper_2508_20258_amd as swz  # noqa: E402
from paper_2508_20258_amd import attention_layer as layer, binding  # noqa: E402


REAL = binding.lib


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)

    def record_stream(self, stream):
        World.now.recorded.append(stream)

    def zero_(self):
        World.now.filled.append(World.now.inside)
        return super().zero_()


class Side:                       # a stream of another library: a handle alone
    cuda_stream = 0x77


class Library:
    def __getattr__(self, name):
        if name in ("swz_status_string", "swz_gemm_plan"):
            return getattr(REAL, name)
        return (lambda *args: 64) if name.endswith("_workspace") else (lambda *args: 0)


class World:
    def __init__(self, monkeypatch):
        World.now = self
        self.inside, self.made, self.filled, self.recorded = None, [], [], []
        empty, full = torch.empty, torch.full

        def switch(s):
            self.inside = None if s == "current" else s

        def made(*args, **kw):
            if str(kw.get("device")) != "meta":
                self.made.append(self.inside)
            return empty(*args, **kw).as_subclass(OnDevice)

        def filled(*args, **kw):
            self.made.append(self.inside)
            return full(*args, **{**kw, "device": "cpu"}).as_subclass(OnDevice)

        monkeypatch.setattr(torch, "empty", made)
        monkeypatch.setattr(torch, "empty_like", lambda x: made(x.shape, dtype=x.dtype))
        monkeypatch.setattr(torch, "full", filled)
        monkeypatch.setattr(torch.cuda, "set_stream", switch)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.inside or "current")
        for module in (binding, layer):
            monkeypatch.setattr(module, "lib", Library())
            monkeypatch.setattr(module, "_launch_stream", lambda s, *tensors: 0)
        monkeypatch.setattr(binding, "_same_current_device", lambda s, *tensors: None)
        monkeypatch.setattr(binding, "_stream_handle", lambda s: 0)


@pytest.fixture
def world(monkeypatch):
    return World(monkeypatch)


def heads(n, h=2, d=64):
    return torch.zeros((n, h, d), dtype=torch.bfloat16).as_subclass(OnDevice)


def ints(*values):
    return torch.tensor(values, dtype=torch.int32).as_subclass(OnDevice)


def norm_inputs(n):
    w, t = torch.ones(64, dtype=torch.bfloat16).as_subclass(OnDevice), torch.zeros((4, 32)).as_subclass(OnDevice)
    return heads(n), heads(n, 1), w, w, t, t, ints(*range(n))


def cache():
    return swz.Cache4(*(t.as_subclass(OnDevice) for t in swz.kv_cache4(2, 2, 64, device="cpu")))


def lse(n):
    return torch.zeros((2, n)).as_subclass(OnDevice)


def matrix(m, n):
    return torch.zeros((m, n), dtype=torch.bfloat16).as_subclass(OnDevice)


def row(n):
    return torch.zeros(n, dtype=torch.bfloat16).as_subclass(OnDevice)


CALLS = {   # a call on `stream`, how many results and workspaces it makes
    "qk_norm_rope": (lambda s: swz.qk_norm_rope(*norm_inputs(3), stream=s), 2, 0),
    "qk_norm_rope_backward": (lambda s: swz.qk_norm_rope_backward(heads(3), heads(3, 1), *norm_inputs(3), stream=s), 3, 1),
    "attention": (lambda s: swz.attention(heads(3), heads(3), heads(3), ints(0, 3), stream=s), 2, 1),
    "attention_backward": (lambda s: swz.attention_backward(heads(3), heads(3), heads(3), heads(3), heads(3), lse(3), ints(0, 3), stream=s), 3, 1),
    "cache4_read": (lambda s: swz.cache4_read(cache(), ints(0, 3), ints(0), ints(0)[None], 3, stream=s), 2, 0),
    "cache4_attention": (lambda s: swz.cache4_attention(heads(1), cache(), ints(1), ints(0)[None], stream=s), 1, 1),
    "gemm": (lambda s: swz.gemm(matrix(8, 16), matrix(16, 8), stream=s), 1, 0),
    "gemm_probe": (lambda s: swz.gemm_probe(matrix(8, 16), matrix(16, 8), stream=s, num_xcd=8), 2, 0),
    "transpose": (lambda s: swz.transpose(matrix(8, 16), stream=s), 1, 0),
    "softmax": (lambda s: swz.softmax(matrix(8, 16), stream=s), 1, 0),
    "layernorm": (lambda s: swz.layernorm(matrix(8, 16), row(16), row(16), stream=s), 1, 0),
    "pid_map_device": (lambda s: swz.pid_map_device(2, 2, 8, 1, 0, stream=s), 2, 0),
    "pid_map_persistent_device": (lambda s: swz.pid_map_persistent_device(2, 2, 8, 1, 0, 4, stream=s), 2, 0),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_made_here_belongs_to_the_stream(world, name):
    call, results, workspaces = CALLS[name]
    call(Side)
    assert world.made == [("external", 0x77)] * (results + workspaces)
    assert set(world.recorded) == {"current"} and len(world.recorded) >= results       # what the caller gets may be used on the current stream too
    assert world.inside is None


@pytest.mark.parametrize("name", CALLS)
def test_without_a_stream_nothing_is_switched(world, name):
    call, results, workspaces = CALLS[name]
    call(None)
    assert world.made == [None] * (results + workspaces) and world.recorded == []


def test_gradients_of_no_tokens_are_filled_on_the_stream(world):
    swz.qk_norm_rope_backward(heads(0), heads(0, 1), *norm_inputs(0), stream=Side)
    assert world.filled == [("external", 0x77)]


def test_a_refusal_leaves_the_current_stream(world):
    with pytest.raises(AssertionError):
        swz.attention(heads(3), heads(3, 1), heads(3), ints(0, 3), stream=Side)
    assert world.inside is None and world.recorded == []
