"""Which stream the memory belongs to that the entry points of a step with drafted tokens make for themselves: the one that works on it; and what the binding refuses.  No GPU: tensors that say they are on one, a library
that does nothing."""
import pytest

torch = pytest.importorskip("torch")

import paper_2508_20258_amd as swz  # noqa: E402
from paper_2508_20258_amd import drafts  # noqa: E402
from test_call_streams import Library, OnDevice, Side, World, heads, ints  # noqa: E402


@pytest.fixture
def world(monkeypatch):
    w = World(monkeypatch)
    monkeypatch.setattr(drafts, "lib", Library())
    monkeypatch.setattr(drafts, "_launch_stream", lambda s, *tensors: 0)
    return w


def cache():
    return swz.Cache16(*(t.as_subclass(OnDevice) for t in swz.kv_cache16(2, 2, 64, device="cpu")))


def floats(*shape):
    return torch.zeros(shape).as_subclass(OnDevice)


def append(s=None, **change):
    args = dict(cache=cache(), k=heads(3), v=heads(3), cu=ints(0, 3), before=ints(0), block_table=ints(0)[None], q=heads(3, 4), cos=floats(8, 16), sin=floats(8, 16))
    return swz.cache16_append(**{**args, **change}, stream=s)


def attend(s=None, **change):
    args = dict(q=heads(3, 4), cache=cache(), cu=ints(0, 3), lengths=ints(3), block_table=ints(0)[None])
    return swz.cache16_attention(**{**args, **change}, stream=s)


def verify(s=None, **change):
    args = dict(target_probs=floats(3, 10), tokens=ints(0, 1, 2), cu=ints(0, 3), uniforms=floats(3), draft_probs=floats(3, 10), parents=ints(0, 0, 0))
    return swz.verify_drafts(**{**args, **change}, stream=s)


def keep(s=None, **change):
    args = dict(cache=cache(), cu=ints(0, 3), before=ints(0), path=ints(0, 2, -1), accepted=ints(1), block_table=ints(0)[None])
    return swz.cache16_keep(**{**args, **change}, stream=s)


@pytest.mark.parametrize("call,results,workspaces", [(append, 1, 0), (attend, 1, 1), (verify, 3, 1)])
def test_memory_made_here_belongs_to_the_stream(world, call, results, workspaces):
    call(Side)
    assert world.made == [("external", 0x77)] * (results + workspaces)
    assert set(world.recorded) == {"current"} and len(world.recorded) >= results
    assert world.inside is None
    world.made.clear(), world.recorded.clear()
    call()
    assert world.made == [None] * (results + workspaces) and world.recorded == []


def test_nothing_is_made_for_what_is_there(world):
    out = heads(3, 4)
    assert append(q_out=out) is out and append(q=None) is None and append(q=None, cos=None, sin=None) is None and keep() is None
    assert world.made == []
    assert attend(out=out) is out and world.made == [None]                # the workspace


BAD = [(append, dict(k=heads(2))), (append, dict(v=heads(3, 1))), (append, dict(k=heads(3, 2, 128), v=heads(3, 2, 128))), (append, dict(q=heads(2, 4))), (append, dict(cos=None)), (append, dict(cos=None, sin=None)),
       (append, dict(sin=floats(8, 8))), (append, dict(positions=ints(0, 1))), (append, dict(q=None, cos=None, sin=None, positions=ints(0, 1, 2))), (append, dict(before=ints(0, 1))),
       (append, dict(cu=ints(0, 1, 3))), (append, dict(block_table=ints(0))), (append, dict(q=None, q_out=heads(3, 4))), (append, dict(cos=floats(0, 16), sin=floats(0, 16))), (append, dict(q=None, cos=floats(0, 16), sin=floats(0, 16))), (append, dict(cos=floats(8, 16).double(), sin=floats(8, 16).double())),
       (attend, dict(tree=ints(0, 0, 0))), (attend, dict(tree=torch.zeros(2, dtype=torch.int64).as_subclass(OnDevice))), (attend, dict(lengths=ints(3, 3))), (attend, dict(q=heads(3, 4, 128))),
       (attend, dict(out=heads(3, 2))), (verify, dict(tokens=ints(0, 1))), (verify, dict(uniforms=floats(2))), (verify, dict(draft_probs=floats(3, 9))), (verify, dict(cu=ints(0))),
       (verify, dict(draft_probs=floats(3, 10).to(torch.bfloat16))), (verify, dict(target_probs=floats(10, 3).T)), (verify, dict(target_probs=floats(1, 10).expand(3, 10))), (verify, dict(parents=ints(0, 0))),
       (keep, dict(path=ints(0, 1)[None])), (keep, dict(accepted=ints(1, 1))), (keep, dict(before=ints()))]


@pytest.mark.parametrize("call,change", BAD)
def test_refusals(world, call, change):
    with pytest.raises(AssertionError):
        call(**change)
    with pytest.raises(AssertionError):
        call(Side, **change)
    assert world.inside is None


def test_no_tokens(world):
    assert append(k=heads(0), v=heads(0), q=heads(0, 4), cu=ints(0, 0)).shape == (0, 4, 64)
    assert attend(q=heads(0, 4), cu=ints(0, 0)).shape == (0, 4, 64)
    keep(path=ints(), cu=ints(0, 0), accepted=ints(0))


@pytest.mark.parametrize("pages", [dict(page_tokens=8), dict(page_tokens=24), dict(head_dim=96)])
def test_caches_that_are_not_made(pages):
    with pytest.raises(AssertionError):
        swz.kv_cache16(**{**dict(pages=2, k_heads=1, head_dim=64, device="cpu"), **pages})
