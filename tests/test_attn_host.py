"""Host-only checks of linattn_window_* and linattn_cache_*: every bad argument is refused before any HIP call."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2510_08318_amd import binding as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, BIG = 0x10000000, 1 << 28          # a fake device address, and a distance between two


def _window(**kw):
    sight = L.Sight(kw.pop("left", -1), kw.pop("right", -1), kw.pop("sinks", 0), kw.pop("scale", 0.0))
    base = dict(dtype=L.BF16, B=2, H=4, HK=2, n=100, d=64, layout=0, sight=sight, lengths=None, workspace=None, workspace_bytes=0)
    return L.WindowDesc(**{**base, **kw})


BAD_WINDOWS = [(dict(dtype=0), "E_DTYPE"), (dict(dtype=4), "E_DTYPE"), (dict(B=0), "E_SHAPE"), (dict(H=0), "E_SHAPE"), (dict(HK=0), "E_SHAPE"),
               (dict(HK=3), "E_SHAPE"), (dict(HK=8), "E_SHAPE"), (dict(n=0), "E_SHAPE"), (dict(n=-1), "E_SHAPE"), (dict(n=(1 << 30) + 1), "E_SHAPE"),
               (dict(d=32), "E_SHAPE"), (dict(d=96), "E_SHAPE"), (dict(layout=2), "E_SHAPE"), (dict(B=40000), "E_SHAPE"),
               (dict(sinks=-1), "E_VALUE"), (dict(scale=-1.0), "E_VALUE"), (dict(scale=float("nan")), "E_VALUE"), (dict(scale=float("inf")), "E_VALUE"),
               (dict(lengths=P + 2), "E_ALIGN")]


@pytest.mark.parametrize("change,status", BAD_WINDOWS)
def test_bad_window_descriptors(change, status):
    w = _window(**change)
    t = [P + i * BIG for i in range(10)]
    assert L.linattn_window_fwd(w, *t[:4], t[4], check=False) == getattr(L, status)
    assert L.linattn_window_bwd(w, *t[:9], check=False) == getattr(L, status)
    assert L.linattn_window_workspace_bytes(w) == 0


@pytest.mark.parametrize("scale,good", [(0.0, True), (-0.0, True), (2.0 ** -100, True), (2.0 ** 100, True), (2.0 ** -101, False), (1e-40, False), (2.0 ** 101, False), (3e38, False)])
def test_range_of_the_scale(scale, good):
    w, c = _window(scale=scale), _cache()
    t = [P + i * BIG for i in range(9)]
    assert (L.linattn_window_workspace_bytes(w) > 0) == good
    assert L.linattn_window_bwd(w, *t, check=False) == (L.E_WORKSPACE if good else L.E_VALUE)
    q = [P + (20 + i) * BIG for i in range(2)]
    assert L.linattn_cache_attn(c, L.Sight(-1, 0, 0, scale), None if good else q[0], q[1], None, 4, 1, None, 0, check=False) == (L.E_NULL if good else L.E_VALUE)


def test_bad_window_tensors():
    w = _window()
    q, k, v, o, lse = [P + i * BIG for i in range(5)]
    f = lambda *a, **kw: L.linattn_window_fwd(kw.get("w", w), *a, check=False)
    assert f(q, k, v, o, lse, w=None) == L.E_NULL
    for i in range(4):
        a = [q, k, v, o]
        a[i] = None
        assert f(*a, lse) == L.E_NULL
        a[i] = P + i * BIG + 8
        assert f(*a, lse) == L.E_ALIGN
    assert f(q, k, v, o, lse + 2) == L.E_ALIGN
    nbytes = 2 * 4 * 100 * 64 * 2
    for other in (q, k, v):
        assert f(q, k, v, other, lse) == L.E_ALIAS
    assert f(q, k, v, q + nbytes - 16, lse) == L.E_ALIAS
    assert f(q, k, v, o, o + nbytes - 4) == L.E_ALIAS
    assert f(q, k, v, o, k + 4) == L.E_ALIAS
    with pytest.raises(L.LinattnError) as e:
        L.linattn_window_fwd(w, None, k, v, o)
    assert e.value.status == L.E_NULL


def test_a_forward_workspace_is_optional_but_checked():
    size = L.linattn_window_workspace_bytes(_window())
    t = [P + i * BIG for i in range(5)]
    f = lambda w: L.linattn_window_fwd(w, *t, check=False)
    assert f(_window(workspace=P + 20 * BIG, workspace_bytes=size - 1)) == L.E_WORKSPACE
    assert f(_window(workspace=P + 20 * BIG + 64, workspace_bytes=size)) == L.E_ALIGN
    assert f(_window(workspace=P, workspace_bytes=size)) == L.E_ALIAS
    # short fp32 sequences: room for parts of the sums; long ones need none
    extra = lambda n: L.linattn_window_workspace_bytes(_window(dtype=L.F32, n=n)) - 2 * 2 * 4 * n * 4
    assert extra(128) > 128 * 4 and extra(128 * 64) == 0


def test_sizes_without_memory_behind_them_are_refused():
    assert L.linattn_window_workspace_bytes(_window(B=1, H=64, HK=64, n=1 << 30)) == 0
    assert L.linattn_window_workspace_bytes(_window(B=1, H=8, HK=2, n=1 << 29)) == 0            # n times the heads of a group


def test_tensors_off_the_gpu_are_refused_by_the_glue():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    x = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        G.window_attention(x, x, x)
    with pytest.raises(ValueError):
        G.window_attention_backward(x, x, x, x, x, x)
    with pytest.raises(ValueError):
        G.PagedCache.empty(4, 16, 2, 64, 1, 4, device="cpu")


def test_bad_window_backward_calls():
    size = L.linattn_window_workspace_bytes(_window())
    assert size > 0 and size % 256 == 0
    work = P + 20 * BIG
    w = _window(workspace=work, workspace_bytes=size)
    names = ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv")
    good = {name: P + i * BIG for i, name in enumerate(names)}
    f = lambda w=w, **kw: L.linattn_window_bwd(w, *{**good, **kw}.values(), check=False)
    for name in names:
        assert f(**{name: None}) == L.E_NULL, name
        assert f(**{name: good[name] + 2}) == L.E_ALIGN, name
    for out in ("dq", "dk", "dv"):
        for other in names:
            if other != out:
                assert f(**{out: good[other]}) == L.E_ALIAS, (out, other)
        assert f(**{out: work}) == L.E_ALIAS
    assert f(q=work + size - 16) == L.E_ALIAS
    assert f(w=_window()) == L.E_WORKSPACE
    assert f(w=_window(workspace=work, workspace_bytes=size - 1)) == L.E_WORKSPACE
    assert f(w=_window(workspace=work + 16, workspace_bytes=size)) == L.E_ALIGN


def _cache(**kw):
    base = dict(type=L.CACHE_E4M3, B=2, H=2, d=64, page=16, pages=40, width=10, layout=0, k=P, v=P + BIG, k_exp=P + 2 * BIG, v_exp=P + 3 * BIG,
                table=P + 4 * BIG, lengths=P + 5 * BIG, counts=None)
    return L.CacheDesc(**{**base, **kw})


BAD_CACHES = [(dict(type=0), "E_DTYPE"), (dict(type=3), "E_DTYPE"), (dict(B=0), "E_SHAPE"), (dict(H=0), "E_SHAPE"), (dict(d=48), "E_SHAPE"),
              (dict(page=0), "E_SHAPE"), (dict(pages=0), "E_SHAPE"), (dict(width=0), "E_SHAPE"), (dict(page=1 << 20, width=1 << 11), "E_SHAPE"),
              (dict(layout=-1), "E_SHAPE"), (dict(pages=(1 << 31) - 1, H=1024, page=1024), "E_SHAPE"),
              (dict(k=None), "E_NULL"), (dict(v=None), "E_NULL"), (dict(k_exp=None), "E_NULL"), (dict(v_exp=None), "E_NULL"), (dict(table=None), "E_NULL"),
              (dict(lengths=None), "E_NULL"), (dict(k=P + 8), "E_ALIGN"), (dict(v=P + BIG + 4), "E_ALIGN"), (dict(table=P + 4 * BIG + 1), "E_ALIGN"),
              (dict(lengths=P + 2), "E_ALIGN"), (dict(counts=P + 2), "E_ALIGN"), (dict(v=P), "E_ALIAS"), (dict(k_exp=P + 16), "E_ALIAS"),
              (dict(v_exp=P + 2 * BIG + 64), "E_ALIAS")]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches(change, status):
    c, want = _cache(**change), getattr(L, status)
    x, y = P + 8 * BIG, P + 9 * BIG
    assert L.linattn_cache_write(c, x, y, 3, check=False) == want
    assert L.linattn_cache_read(c, x, y, 3, check=False) == want
    assert L.linattn_cache_attn(c, L.Sight(-1, 0, 0, 0.0), x, y, None, 4, 3, P + 10 * BIG, 1 << 30, check=False) == want
    assert L.linattn_cache_workspace_bytes(c, 4, 3) == 0


def test_bad_cache_calls():
    c = _cache()
    x, y, work = P + 8 * BIG, P + 9 * BIG, P + 10 * BIG
    for call in (L.linattn_cache_write, L.linattn_cache_read):
        f = lambda *a: call(*a, check=False)
        assert f(None, x, y, 3) == L.E_NULL
        assert f(c, None, y, 3) == L.E_NULL
        assert f(c, x, None, 3) == L.E_NULL
        assert f(c, x, y, 0) == L.E_SHAPE
        assert f(c, x + 8, y, 3) == L.E_ALIGN
        assert f(c, x, y + 8, 3) == L.E_ALIGN
        for at in (P, P + BIG, P + 2 * BIG, P + 3 * BIG):
            assert f(c, at, y, 3) == L.E_ALIAS
            assert f(c, x, at, 3) == L.E_ALIAS
    assert L.linattn_cache_read(c, x, x, 3, check=False) == L.E_ALIAS
    sight = L.Sight(-1, 0, 0, 0.0)
    f = lambda *a, s=sight, c=c, H=4, n=3: L.linattn_cache_attn(c, s, *a, H, n, work, 1 << 30, check=False)
    assert f(x, y, None, c=None) == L.E_NULL
    assert f(x, y, None, s=None) == L.E_NULL
    assert f(None, y, None) == L.E_NULL
    assert f(x, None, None) == L.E_NULL
    assert f(x, y, None, H=3) == L.E_SHAPE
    assert f(x, y, None, H=0) == L.E_SHAPE
    assert f(x, y, None, n=0) == L.E_SHAPE
    assert f(x, y, None, s=L.Sight(-1, 0, -1, 0.0)) == L.E_VALUE
    assert f(x, y, None, s=L.Sight(-1, 0, 0, float("nan"))) == L.E_VALUE
    assert f(x + 2, y, None) == L.E_ALIGN
    assert f(x, y, y + 2) == L.E_ALIGN
    assert f(x, x, None) == L.E_ALIAS
    assert f(x, P + 16, None) == L.E_ALIAS
    assert f(x, y, y + 4) == L.E_ALIAS


def test_cache_workspace():
    """A single token of many keys is split, and the split's parts need room."""
    work = P + 10 * BIG
    c = _cache(width=100, pages=300)
    need = L.linattn_cache_workspace_bytes(c, 4, 1)
    assert need > 0 and need % 256 == 0
    f = lambda w, size: L.linattn_cache_attn(c, L.Sight(-1, 0, 0, 0.0), P + 8 * BIG, P + 9 * BIG, None, 4, 1, w, size, check=False)
    assert f(None, need) == L.E_WORKSPACE
    assert f(work, need - 1) == L.E_WORKSPACE
    assert f(work + 128, need) == L.E_ALIGN
    assert f(P + 8 * BIG, need) == L.E_ALIAS


def test_header_names_and_layouts_match_the_binding(tmp_path):
    header = open(os.path.join(ROOT, "include", "linattn.h")).read()
    consts = dict((m.group(1), int(m.group(2))) for m in re.finditer(r"#define\s+LINATTN_(\w+)\s+(-?\d+)", header))
    assert consts["E_VALUE"] == L.E_VALUE and consts["CACHE_BF16"] == L.CACHE_BF16 and consts["CACHE_E4M3"] == L.CACHE_E4M3
    assert L.linattn_strerror(L.E_VALUE) != "unknown status"
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    fields = {"linattn_sight": L.Sight, "linattn_window_desc": L.WindowDesc, "linattn_cache_desc": L.CacheDesc}
    body = "".join(f'printf("%zu\\n", sizeof({t}));' + "".join(f'printf("%zu\\n", offsetof({t}, {f}));' for f, _ in c._fields_) for t, c in fields.items())
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "linattn.h"\nint main(void) {{ {body} return 0; }}\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [x for c in fields.values() for x in [ctypes.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]]
    assert got == want


def test_page_division_is_exact(tmp_path):
    """page_of against the division, for page sizes of every kind and positions up to the limit."""
    src, exe = tmp_path / "div.cpp", tmp_path / "div"
    src.write_text("""#include <stdio.h>
#include "attn.h"
using namespace linattn::attn;
int main() {
  const int pages[] = {1, 2, 3, 5, 7, 16, 24, 100, 127, 128, 1000, 1560, 65535, 65536, 1000003, (1 << 30) - 1, 1 << 30};
  for (int page : pages) {
    Pool p{};
    p.page = page;
    set_divisor(&p);
    auto check = [&](long long j) { return j < 0 || j > 0x7fffffffll || page_of(p, (int)j) == (int)(j / page); };
    for (long long i = 0; i < 200000; ++i)
      if (!check(i) || !check((1ll << 30) - i) || !check(0x7fffffffll - i) || !check(i * page) || !check(i * page - 1) || !check(i * 10007)) return printf("%d\\n", page), 1;
  }
  return 0;
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    "-I", os.path.join(ROOT, "paper_2510_08318_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


def test_the_refusal_of_a_number_names_the_range_in_force():
    """Of scales next to its ends, those that are refused lie outside what the message names."""
    text = L.lib().linattn_strerror(L.E_VALUE).decode()
    lo, hi = [2.0 ** int(x) for x in re.search(r"scale 0 or 2\^(-?\d+) to 2\^(-?\d+)", text).groups()]
    assert "sinks >= 0" in text
    for scale in (0.0, lo, hi, lo * 0.999, hi * 1.001, -lo, 1e-40, 3e38):
        assert (L.linattn_window_workspace_bytes(_window(scale=scale)) > 0) == (scale == 0.0 or lo <= scale <= hi), scale


def test_the_glue_says_that_autograd_records_nothing():
    """Their results carry no gradient even where the inputs ask for one; a caller has to learn that from the documentation."""
    from paper_2510_08318_amd import torch_glue as G
    for f in (G.window_attention, G.window_attention_backward, G.PagedCache.write, G.PagedCache.attend):
        assert "autograd" in f.__doc__, f.__name__
