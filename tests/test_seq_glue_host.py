"""What torch_glue.rotary and decay_attention hand to the library, on the CPU: tensors that say they are on GPU 0, and a library that records its calls."""
import ctypes

import pytest
import torch

from paper_2510_08318_amd import binding as L, torch_glue as G


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    """The calls' arguments, the description first (its bytes are copied: the caller may keep it)."""
    got = []

    def record(desc, *args, **kw):
        got.append((type(desc).from_buffer_copy(desc), *args))
        return 0
    for name in ("linattn_rotary", "linattn_decay_fwd", "linattn_decay_bwd"):
        monkeypatch.setattr(L, name, record)
    monkeypatch.setattr(G, "_one_device", lambda: True)
    monkeypatch.setattr(G, "_raw_stream", lambda index: None)
    return got


KINDS = {"tensor": lambda x: torch.tensor(x), "number": lambda x: x}


def _rotary(**kw):
    return G.rotary(tensor(1, 2, 12, 64), dims=kw.pop("dims", (32, 16, 16)), **{"grid": (1, 3, 4), **kw})


def test_first_positions_that_change_in_place(calls):
    """The frame counter of a clip that is generated piece by piece."""
    t = torch.tensor(7)
    for want in (7, 12, 17):
        _rotary(first=(t, 0, 0))
        assert list(calls[-1][0].first) == [want, 0, 0]
        t += 5


def test_grid_and_dims_that_change_in_place(calls):
    t, d = torch.tensor(3), torch.tensor(16)
    _rotary(grid=(1, t, 4), dims=(32, d, 16))
    t.fill_(5), d.fill_(8)
    _rotary(grid=(1, t, 4), dims=(32, d, 16))
    assert [list(c[0].grid) for c in calls] == [[1, 3, 4], [1, 5, 4]] and [list(c[0].dims) for c in calls] == [[32, 16, 16], [32, 8, 16]]


def test_a_tensor_of_positions_that_changes_in_place(calls):
    t = torch.tensor([7, 0, 0])
    _rotary(first=t)
    t[0] = 9
    _rotary(first=t)
    assert [list(c[0].first) for c in calls] == [[7, 0, 0], [9, 0, 0]]


def test_base_that_changes_in_place(calls):
    t = torch.tensor(500.0, dtype=torch.float64)
    _rotary(base=t)
    t.fill_(2000.0)
    _rotary(base=t)
    assert [c[0].base for c in calls] == [500.0, 2000.0]


@pytest.mark.parametrize("backward", [False, True])
def test_scale_that_changes_in_place(calls, backward):
    q, g, t = tensor(1, 2, 5, 64), tensor(2, dtype=torch.float32), torch.tensor(0.5, requires_grad=True)
    for want in (0.5, 0.25):
        with torch.no_grad():
            t.fill_(want)
        if backward:
            G.decay_attention_backward(q, q, q, g, q, scale=t)
        else:
            G.decay_attention(q, q, q, g, scale=t)
        assert calls[-1][0].scale == want


def test_the_same_numbers_of_other_types(calls):
    """Integers and floats of numpy, lists."""
    import numpy as np
    _rotary(first=[np.int64(2), 3.0, np.float32(4)], dims=[32, np.int32(16), 16], grid=torch.Size((1, 3, 4)), base=np.float32(100.0))
    _rotary(first=(2, 3, 4), base=100)
    assert bytes(calls[0][0]) == bytes(calls[1][0])


def test_no_caller_s_object_is_kept(calls):
    """Neither as a key nor as a value."""
    import gc
    import weakref
    t, s = torch.tensor(7), torch.tensor(0.5)
    _rotary(first=(t, 0, 0))
    q, g = tensor(1, 2, 5, 64), tensor(2, dtype=torch.float32)
    G.decay_attention(q, q, q, g, scale=s)
    refs = [weakref.ref(x) for x in (t, s)]
    calls.clear()
    del t, s
    gc.collect()
    assert [r() for r in refs] == [None, None]


@pytest.mark.parametrize("kw", [dict(first=(0.5, 0, 0)), dict(grid=(1, 2.5, 4)), dict(dims=(32, 16.5, 15)), dict(first=(0, 0)), dict(first=(1 << 31, 0, 0)), dict(dims=()),
                                dict(dims=(16,) * 4), dict(pairs="both"), dict(first=(float("nan"), 0, 0)), dict(first=(float("inf"), 0, 0))])
def test_numbers_that_are_refused(calls, kw):
    with pytest.raises(ValueError):
        _rotary(**kw)
    assert not calls


def _saved(x):
    """A graph that holds x as it is now."""
    w = torch.ones(x.shape, dtype=x.dtype, requires_grad=True)
    return (w * torch.Tensor.as_subclass(x, torch.Tensor)).sum()


def _refused(graph):
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        graph.backward()


def test_autograd_sees_what_rotary_overwrites(calls):
    q, k = tensor(1, 2, 12, 64), tensor(1, 2, 12, 64)
    a, b = _saved(q), _saved(k)
    G.rotary(q, k)
    a.backward(retain_graph=True)                       # (results of their own leave q and k alone)
    G.rotary(q, k, q_out=q, k_out=k)
    _refused(a), _refused(b)


def test_autograd_sees_the_states_and_results_that_decay_attention_overwrites(calls):
    q, g = tensor(1, 2, 5, 64), tensor(2, dtype=torch.float32)
    for kw in (dict(), dict(slots=tensor(1, dtype=torch.int32))):
        state = tensor(1, 2, 64, 64, dtype=torch.float32)
        kept = _saved(state)
        G.decay_attention(q, q, q, g, state=state, state_out=False, **kw)
        kept.backward(retain_graph=True)
        G.decay_attention(q, q, q, g, state=state, **(kw or dict(state_out=state)))      # (with slots, in place without a word)
        _refused(kept)
    out = tensor(1, 2, 5, 64)
    kept = _saved(out)
    G.decay_attention(q, q, q, g, out=out)
    _refused(kept)


def test_autograd_sees_the_gradients_that_are_overwritten(calls):
    q, g, state = tensor(1, 2, 5, 64), tensor(2, dtype=torch.float32), tensor(1, 2, 64, 64, dtype=torch.float32)
    outs = dict(dq=tensor(1, 2, 5, 64), dk=tensor(1, 2, 5, 64), dv=tensor(1, 2, 5, 64), dstate_in=tensor(1, 2, 64, 64, dtype=torch.float32))
    kept = [_saved(x) for x in outs.values()]
    G.decay_attention_backward(q, q, q, g, q, state=state, **outs)
    for x in kept:
        _refused(x)


def test_tensors_of_inference_mode_have_no_count(calls):
    with torch.inference_mode():
        q = tensor(1, 2, 12, 64)
        assert G.rotary(q, q_out=q)[0] is q
    assert G.rotary(q, q_out=q)[0] is q
