"""Host-only checks of linattn_rotary and linattn_decay_*: every bad argument is refused before any HIP call."""
import ctypes
import math
import os
import re
import subprocess

import pytest

from paper_2510_08318_amd import binding as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, BIG = 0x10000000, 1 << 28          # a fake device address, and a distance between two


def _rotary(**kw):
    three = lambda x: (ctypes.c_int * 3)(*x)
    base = dict(dtype=L.BF16, B=2, H=4, HK=3, n=100, d=64, layout=0, axes=3, dims=(32, 16, 16), pairs=0, inverse=0, base=0.0, grid=(1, 8, 8), first=(0, 0, 0),
                positions=None, position_items=0, lengths=None)
    base.update(kw)
    for name in ("dims", "grid", "first"):
        base[name] = three(base[name])
    return L.RotaryDesc(**base)


def _decay(**kw):
    base = dict(dtype=L.BF16, B=2, H=4, HK=2, n=100, d=64, layout=0, scale=0.0, log_decay=P + 40 * BIG, lengths=None, slots=None, states=0, workspace=None,
                workspace_bytes=0)
    w = L.DecayDesc(**{**base, **kw})
    if "workspace" not in kw:
        w.workspace, w.workspace_bytes = P + 41 * BIG, 1 << 30
    return w


SHAPES = [(dict(dtype=0), "E_DTYPE"), (dict(dtype=4), "E_DTYPE"), (dict(B=0), "E_SHAPE"), (dict(H=0), "E_SHAPE"), (dict(HK=0), "E_SHAPE"), (dict(n=0), "E_SHAPE"),
          (dict(n=-1), "E_SHAPE"), (dict(n=(1 << 30) + 1), "E_SHAPE"), (dict(d=32), "E_SHAPE"), (dict(d=96), "E_SHAPE"), (dict(layout=2), "E_SHAPE"),
          (dict(B=40000), "E_SHAPE"), (dict(lengths=P + 2), "E_ALIGN")]


@pytest.mark.parametrize("change,status", SHAPES + [
    (dict(axes=0), "E_SHAPE"), (dict(axes=4), "E_SHAPE"), (dict(dims=(32, 16, 18)), "E_SHAPE"), (dict(dims=(32, 15, 16)), "E_SHAPE"), (dict(dims=(32, 0, 16)), "E_SHAPE"),
    (dict(dims=(32, -2, 16)), "E_SHAPE"), (dict(dims=(2 ** 31 - 2, 2, 2)), "E_SHAPE"), (dict(grid=(1, 0, 8)), "E_SHAPE"), (dict(grid=(1, 8, -1)), "E_SHAPE"),
    (dict(pairs=2), "E_VALUE"), (dict(pairs=-1), "E_VALUE"), (dict(base=0.5), "E_VALUE"), (dict(base=-3.0), "E_VALUE"), (dict(base=math.nan), "E_VALUE"),
    (dict(base=math.inf), "E_VALUE"), (dict(positions=P + 30 * BIG), "E_SHAPE"), (dict(positions=P + 30 * BIG, position_items=3), "E_SHAPE"),
    (dict(positions=P + 30 * BIG + 2, position_items=2), "E_ALIGN")])
def test_bad_rotary_descriptors(change, status):
    assert L.linattn_rotary(_rotary(**change), P, P + BIG, P + 2 * BIG, P + 3 * BIG, check=False) == getattr(L, status)


def test_bad_rotary_tensors():
    w = _rotary()
    q, k, a, b = [P + i * BIG for i in range(4)]
    f = lambda *t, w=w: L.linattn_rotary(w, *t, check=False)
    assert f(q, k, a, b, w=None) == L.E_NULL
    assert f(None, k, a, b) == L.E_NULL and f(q, k, None, b) == L.E_NULL and f(q, k, a, None) == L.E_NULL and f(q, None, a, b) == L.E_NULL
    for i in range(4):
        t = [q, k, a, b]
        t[i] += 8
        assert f(*t) == L.E_ALIGN
    qb, kb = 2 * 4 * 100 * 64 * 2, 2 * 3 * 100 * 64 * 2
    assert f(q, k, q + 16, b) == L.E_ALIAS and f(q, k, q + qb - 16, b) == L.E_ALIAS and f(q, k, k, b) == L.E_ALIAS and f(q, k, a, q) == L.E_ALIAS
    assert f(q, k, a, a + qb - 16) == L.E_ALIAS and f(q, k, a, k + 16) == L.E_ALIAS
    assert f(q, k, a, b, w=_rotary(positions=a + 16, position_items=1)) == L.E_ALIAS
    assert f(q, k, a, b, w=_rotary(lengths=b + kb - 4)) == L.E_ALIAS
    with pytest.raises(L.LinattnError) as e:
        L.linattn_rotary(w, None, k, a, b)
    assert e.value.status == L.E_NULL


@pytest.mark.parametrize("change,status", SHAPES + [
    (dict(HK=3), "E_SHAPE"), (dict(HK=8), "E_SHAPE"), (dict(scale=-1.0), "E_VALUE"), (dict(scale=math.nan), "E_VALUE"), (dict(scale=math.inf), "E_VALUE"),
    (dict(scale=2.0 ** -101), "E_VALUE"), (dict(log_decay=None), "E_NULL"), (dict(log_decay=P + 2), "E_ALIGN"), (dict(slots=P + 42 * BIG), "E_SHAPE"),
    (dict(slots=P + 42 * BIG, states=-1), "E_SHAPE"), (dict(slots=P + 42 * BIG + 1, states=4), "E_ALIGN"), (dict(slots=P + 42 * BIG, states=1 << 30), "E_SHAPE")])
def test_bad_decay_descriptors(change, status):
    w = _decay(**change)
    t = [P + i * BIG for i in range(10)]
    assert L.linattn_decay_fwd(w, *t[:6], check=False) == getattr(L, status)
    assert L.linattn_decay_bwd(w, *t, check=False) == getattr(L, status)
    assert L.linattn_decay_workspace_bytes(w) == 0 and L.linattn_decay_workspace_bytes(w, True) == 0


def test_bad_decay_forward_tensors():
    names = ("q", "k", "v", "state_in", "out", "state_out")
    good = {name: P + i * BIG for i, name in enumerate(names)}
    f = lambda w=_decay(), **kw: L.linattn_decay_fwd(w, *{**good, **kw}.values(), check=False)
    assert f(w=None) == L.E_NULL
    for name in ("q", "k", "v", "out"):
        assert f(**{name: None}) == L.E_NULL, name
    for name in names:
        assert f(**{name: good[name] + 8}) == L.E_ALIGN, name
    qb, sb = 2 * 4 * 100 * 64 * 2, 2 * 4 * 64 * 64 * 4
    for name in ("q", "k", "v", "state_in", "state_out"):
        assert f(out=good[name]) == L.E_ALIAS, name
    assert f(out=good["q"] + qb - 16) == L.E_ALIAS and f(state_out=good["out"] + qb - 16) == L.E_ALIAS
    assert f(state_out=good["state_in"] + 16) == L.E_ALIAS and f(state_out=good["state_in"] + sb - 16) == L.E_ALIAS
    assert f(state_out=good["v"]) == L.E_ALIAS
    assert f(w=_decay(log_decay=good["out"] + 16)) == L.E_ALIAS and f(w=_decay(lengths=good["state_out"] + 16)) == L.E_ALIAS
    pool = dict(slots=P + 42 * BIG, states=7)
    assert f(w=_decay(**pool), out=good["state_out"] + 7 * (sb // 2) - 16) == L.E_ALIAS
    assert f(w=_decay(slots=good["out"], states=7)) == L.E_ALIAS


def test_bad_decay_backward_tensors():
    names = ("q", "k", "v", "state_in", "dout", "dstate_out", "dq", "dk", "dv", "dstate_in")
    good = {name: P + i * BIG for i, name in enumerate(names)}
    f = lambda w=_decay(), **kw: L.linattn_decay_bwd(w, *{**good, **kw}.values(), check=False)
    assert f(w=None) == L.E_NULL
    for name in ("q", "k", "v", "dout", "dq", "dk", "dv"):
        assert f(**{name: None}) == L.E_NULL, name
    for name in names:
        assert f(**{name: good[name] + 8}) == L.E_ALIGN, name
    for out in ("dq", "dk", "dv", "dstate_in"):
        for name in names:
            if name != out:
                assert f(**{out: good[name]}) == L.E_ALIAS, (out, name)


@pytest.mark.parametrize("kw", [dict(), dict(HK=4), dict(n=1), dict(n=4000), dict(dtype=L.F32, n=500), dict(dtype=L.BF16_F32MATH, n=500), dict(B=16, H=64)])
def test_decay_workspace(kw):
    w = _decay(workspace=None, **kw)
    t = [P + i * BIG for i in range(10)]
    for backward, call in ((False, lambda w: L.linattn_decay_fwd(w, *t[:6], check=False)), (True, lambda w: L.linattn_decay_bwd(w, *t, check=False))):
        size = L.linattn_decay_workspace_bytes(w, backward)
        assert size % 256 == 0 and size == L.linattn_decay_workspace_bytes(_decay(workspace=None, layout=1, **kw), backward)
        if size:
            assert call(w) == L.E_WORKSPACE
            assert call(_decay(workspace=P + 41 * BIG, workspace_bytes=size - 1, **kw)) == L.E_WORKSPACE
            assert call(_decay(workspace=t[0], workspace_bytes=size, **kw)) == L.E_ALIAS
        assert call(_decay(workspace=P + 41 * BIG + 64, workspace_bytes=size, **kw)) == L.E_ALIGN


def test_tensors_off_the_gpu_are_refused_by_the_glue():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    x, g = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16), torch.zeros(2)
    for call in (lambda: G.rotary(x), lambda: G.decay_attention(x, x, x, g), lambda: G.decay_attention_backward(x, x, x, g, x)):
        with pytest.raises(ValueError):
            call()


def test_structures_match_the_header(tmp_path):
    """Offsets of the ctypes structures against the C compiler's."""
    lines, src = [], ['#include "linattn.h"', "#include <stdio.h>", "int main(void) {"]
    for cls, name in ((L.RotaryDesc, "linattn_rotary_desc"), (L.DecayDesc, "linattn_decay_desc")):
        src.append(f'printf("%zu ", sizeof({name}));')
        lines.append(ctypes.sizeof(cls))
        for field, _ in cls._fields_:
            src.append(f'printf("%zu ", offsetof({name}, {field}));')
            lines.append(getattr(cls, field).offset)
    src.append("return 0; }")
    (tmp_path / "t.c").write_text("\n".join(src))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == lines
    header = open(os.path.join(ROOT, "include", "linattn.h")).read()
    for name in ("PAIRS_ADJACENT", "PAIRS_HALVES"):
        assert int(re.search(rf"#define\s+LINATTN_{name}\s+(\d+)", header).group(1)) == getattr(L, name)
