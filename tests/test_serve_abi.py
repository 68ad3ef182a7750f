"""Checks of e2s_serve.h that need no GPU: exports, the rotary plan's numbers, and that
every invalid call is refused on the host before any launch (the fake device addresses
below are never dereferenced)."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

import _serve_helpers as R
from paper_2608_23253_amd import _lib as L
from paper_2608_23253_amd import _serve as S

lib = L.lib()
A = 1 << 20


def test_exports_every_declared_entry_point():
    names = L.header_entry_points(S.HEADER)
    assert len(names) == 7
    for n in names:
        assert hasattr(lib, n), n
        assert n in S.SIGNATURES
    assert lib.e2s_serve_abi_version() == 1


def test_header_is_plain_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    src = tmp_path / "h.c"
    # the binding's structures have the header's sizes
    names = {"e2s_rotary_spec": S.RotarySpec, "e2s_rotary_plan": S.RotaryPlan,
             "e2s_rotary_shape": S.RotaryShape, "e2s_cache": S.CacheDesc,
             "e2s_cache_append_shape": S.AppendShape, "e2s_cache_attend_shape": S.AttendShape,
             "e2s_cache_evict_shape": S.EvictShape}
    src.write_text('#include "e2s_serve.h"\n' + "".join(
        f"_Static_assert(sizeof({n}) == {ctypes.sizeof(t)}, \"{n}\");\n"
        for n, t in names.items()))
    inc = os.path.dirname(S.HEADER)
    run = subprocess.run([gcc, "-std=c11", "-Wall", "-Wextra", "-Werror", "-fsyntax-only",
                          f"-I{inc}", str(src)], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


# ---------------------------------------------------------------------------
# rotary
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [
    dict(rot_dim=128, base=1e4), dict(rot_dim=64, base=1e6, scaling="linear", factor=4.0),
    dict(rot_dim=96, base=1e4, scaling="base", factor=8.0),
    dict(rot_dim=2, base=1e4, scaling="base", factor=8.0),
    dict(rot_dim=128, base=1e4, scaling="ramp", factor=32.0, original_len=4096.0),
    dict(rot_dim=128, base=5e5, scaling="ramp", factor=8.0, original_len=8192.0, low=1.0,
         high=4.0, amplitude=1.0),
])
def test_plan_frequencies(kw):
    plan = S.rotary_plan(128, **kw)
    args = {k: v for k, v in kw.items() if k not in ("rot_dim", "base", "amplitude")}
    f = R.frequencies(kw["rot_dim"], kw["base"], **args)
    got = np.array(plan.turns[:kw["rot_dim"] // 2]) * 2 * math.pi
    assert np.allclose(got, f, rtol=1e-14, atol=0)
    amp = kw.get("amplitude") or (0.1 * math.log(kw["factor"]) + 1
                                  if kw.get("scaling") == "ramp" else 1.0)
    assert plan.amplitude == np.float32(amp)
    assert plan.axes == 1 and not any(plan.axis)


def test_plan_of_a_ramp_is_linear_below_and_plain_above():
    plan = S.rotary_plan(128, base=1e4, scaling="ramp", factor=4.0, original_len=4096.0)
    plain = S.rotary_plan(128, base=1e4)
    assert plan.turns[0] == plain.turns[0]                     # 652 turns: as trained
    assert plan.turns[63] == plain.turns[63] / 4               # 0.08 turns: interpolated


def test_plan_sections():
    plan = S.rotary_plan(128, sections=(16, 24, 24))
    assert plan.axes == 3
    assert list(plan.axis[:64]) == [0] * 16 + [1] * 24 + [2] * 24
    assert S.rotary_plan(128, sections=(0, 0, 64)).axes == 3


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=0), L.ERR_BAD_SHAPE), (dict(rot_dim=3), L.ERR_BAD_SHAPE),
    (dict(rot_dim=130), L.ERR_BAD_SHAPE), (dict(rot_dim=0), L.ERR_BAD_SHAPE),
    (dict(head_dim=258, rot_dim=2), L.ERR_UNSUPPORTED), (dict(layout=2), L.ERR_BAD_PARAM),
    (dict(scaling=4), L.ERR_BAD_PARAM), (dict(base=1.0), L.ERR_BAD_PARAM),
    (dict(base=float("nan")), L.ERR_BAD_PARAM), (dict(base=float("inf")), L.ERR_BAD_PARAM),
    (dict(scaling="linear", factor=0.5), L.ERR_BAD_PARAM),
    (dict(scaling="ramp", factor=2.0), L.ERR_BAD_PARAM),                     # no length
    (dict(scaling="ramp", factor=2.0, original_len=10.0, low=2.0, high=2.0), L.ERR_BAD_PARAM),
    (dict(scaling="ramp", factor=2.0, original_len=10.0, low=-1.0), L.ERR_BAD_PARAM),
    (dict(amplitude=-1.0), L.ERR_BAD_PARAM), (dict(amplitude=1e39), L.ERR_BAD_PARAM),
    (dict(sections=(1, 2, 3)), L.ERR_BAD_SHAPE), (dict(sections=(-1, 33, 32)), L.ERR_BAD_SHAPE),
])
def test_plan_refusals(kw, status):
    kw = dict(dict(head_dim=128), **kw)
    with pytest.raises(L.E2SError) as e:
        S.rotary_plan(**kw)
    assert e.value.status == status


def rotate(plan="good", pos=A, q=A, k=A, qo=A, ko=A, **kw):
    plan = S.rotary_plan(64) if plan == "good" else plan
    f = dict(batch=2, num_tokens=5, q_heads=4, k_heads=2, dtype=L.DTYPE_BF16, inverse=0)
    st = dict(q_stride=(1280, 320, 64), k_stride=(640, 320, 64), q_out_stride=(1280, 320, 64),
              k_out_stride=(640, 320, 64), pos_stride=(0, 5, 1))
    st.update({n: v for n, v in kw.items() if n in st})
    f.update({n: v for n, v in kw.items() if n not in st})
    sh = S.RotaryShape(*f.values())
    for n, v in st.items():
        getattr(sh, n)[:] = v
    return lib.e2s_rotate_positions(ctypes.byref(sh), ctypes.byref(plan) if plan else None, pos, q,
                                    k, qo, ko, None)


def test_rotate_refusals():
    assert rotate(plan=None) == L.ERR_NULL_POINTER
    for kw in (dict(pos=None), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None)):
        assert rotate(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_tokens=-1), dict(q_heads=-1), dict(q_heads=0, k_heads=0),
               dict(q_stride=(-1, 320, 64)), dict(q_out_stride=(1280, 0, 64)),
               dict(k_out_stride=(640, 320, 0)), dict(pos_stride=(0, -5, 1)),
               dict(k_stride=(1 << 62, 320, 64))):
        assert rotate(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(dtype=3), dict(inverse=2)):
        assert rotate(**kw) == L.ERR_BAD_PARAM, kw
    assert rotate(batch=1 << 12, num_tokens=1 << 12) == L.ERR_UNSUPPORTED
    assert rotate(q_heads=70000) == L.ERR_UNSUPPORTED
    assert rotate(q=A + 1) == L.ERR_MISALIGNED
    assert rotate(pos=A + 2) == L.ERR_MISALIGNED
    assert rotate(dtype=L.DTYPE_F32, ko=A + 2) == L.ERR_MISALIGNED
    assert rotate(num_tokens=0, q=None, k=None, qo=None, ko=None, pos=None) == L.OK
    # an absent tensor needs no pointer (the call then stops at the missing positions)
    assert rotate(k_heads=0, k=None, ko=None, pos=None) == L.ERR_NULL_POINTER
    for kw in (dict(axes=2), dict(rot_dim=66), dict(head_dim=512), dict(layout=7)):
        plan = S.rotary_plan(64)
        for n, v in kw.items():
            setattr(plan, n, v)
        assert rotate(plan=plan) in (L.ERR_BAD_PARAM, L.ERR_BAD_SHAPE), kw
    plan = S.rotary_plan(64)
    plan.axis[31] = 1                                   # beyond its one axis
    assert rotate(plan=plan) == L.ERR_BAD_PARAM


# ---------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------

def desc(**kw):
    f = dict(num_pages=9, page_tokens=16, num_kv_heads=2, head_dim=64, k_page_stride=2048,
             v_page_stride=2048, k=A, v=A, k_scale=A, v_scale=A)
    f.update(kw)
    return S.CacheDesc(*f.values())


def append(cache=None, pages=A, start=A, count=None, idx=None, k=A, v=A, **kw):
    f = dict(batch=3, num_tokens=5, src_tokens=5, dtype=L.DTYPE_BF16, max_pages=4, reserved=0,
             pages_stride=4)
    st = dict(k_stride=(640, 320, 64), v_stride=(640, 320, 64))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = S.AppendShape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    cache = desc() if cache is None else cache
    return lib.e2s_cache_append(ctypes.byref(cache), ctypes.byref(sh), pages, start, count, idx, k,
                                v, None)


CACHES = [
    (dict(num_pages=0), L.ERR_BAD_SHAPE), (dict(page_tokens=0), L.ERR_BAD_SHAPE),
    (dict(page_tokens=48), L.ERR_UNSUPPORTED), (dict(page_tokens=256), L.ERR_UNSUPPORTED),
    (dict(head_dim=96), L.ERR_UNSUPPORTED), (dict(num_kv_heads=129), L.ERR_UNSUPPORTED),
    (dict(k_page_stride=2032), L.ERR_BAD_SHAPE), (dict(v_page_stride=2056), L.ERR_MISALIGNED),
    (dict(k_page_stride=1 << 62), L.ERR_BAD_SHAPE), (dict(k=None), L.ERR_NULL_POINTER),
    (dict(v_scale=None), L.ERR_NULL_POINTER), (dict(v=A + 8), L.ERR_MISALIGNED),
    (dict(k_scale=A + 2), L.ERR_MISALIGNED),
]


@pytest.mark.parametrize("kw,status", CACHES)
def test_cache_refusals(kw, status):
    assert append(cache=desc(**kw)) == status
    assert attend(cache=desc(**kw), ws_bytes=1 << 40) == status
    assert evict(cache=desc(**kw)) == status


def test_append_refusals():
    for kw in (dict(pages=None), dict(start=None), dict(k=None), dict(v=None)):
        assert append(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_tokens=-1), dict(src_tokens=0), dict(max_pages=0),
               dict(pages_stride=-1), dict(k_stride=(640, -64, 64)), dict(src_tokens=4),
               dict(v_stride=(1 << 62, 320, 64))):
        assert append(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(dtype=7), dict(reserved=1)):
        assert append(**kw) == L.ERR_BAD_PARAM, kw
    for kw in (dict(k=A + 8), dict(pages=A + 1), dict(count=A + 2), dict(idx=A + 3),
               dict(k_stride=(640, 320, 68)), dict(v_stride=(644, 320, 64))):
        assert append(**kw) == L.ERR_MISALIGNED, kw
    assert append(num_tokens=(1 << 20) + 1, src_tokens=1 << 21) == L.ERR_UNSUPPORTED
    assert append(batch=1 << 22) == L.ERR_UNSUPPORTED
    assert append(num_tokens=0, pages=None, start=None, k=None, v=None) == L.OK
    # fewer rows than tokens are fine where an index picks them (stops at the missing table)
    assert append(src_tokens=4, idx=A, pages=None) == L.ERR_NULL_POINTER


def attend_shape(**kw):
    f = dict(batch=3, num_heads=4, num_queries=2, dtype=L.DTYPE_BF16, max_tokens=100, max_pages=7,
             causal=1, weights=0, scale=0.0, reserved=0, pages_stride=7)
    st = dict(q_stride=(512, 128, 64), out_stride=(512, 128, 64), weights_in_stride=(200, 100),
              weights_out_stride=(200, 100))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = S.AttendShape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    return sh


def attend(cache=None, pages=A, lengths=A, count=None, q=A, out=A, win=None, wout=None, ws=A,
           ws_bytes=None, **kw):
    cache = desc() if cache is None else cache
    sh = attend_shape(**kw)
    if ws_bytes is None:
        n = ctypes.c_size_t(0)
        st = lib.e2s_cache_attend_workspace_size(ctypes.byref(cache), ctypes.byref(sh),
                                                 ctypes.byref(n))
        ws_bytes = n.value if st == L.OK else 1 << 40
    return lib.e2s_cache_attend(ctypes.byref(cache), ctypes.byref(sh), pages, lengths, count, q,
                                out, win, wout, ws, ws_bytes, None)


def test_attend_refusals():
    for kw in (dict(pages=None), dict(lengths=None), dict(q=None), dict(out=None)):
        assert attend(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_heads=3), dict(num_heads=0), dict(num_queries=0),
               dict(max_tokens=0), dict(max_pages=0), dict(pages_stride=-7),
               dict(q_stride=(-512, 128, 64)), dict(out_stride=(512, 0, 64)),
               dict(weights=1, wout=A, weights_out_stride=(0, 100)),
               dict(weights=1, wout=A, weights_in_stride=(-1, 100))):
        assert attend(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(dtype=3), dict(causal=2), dict(weights=2), dict(scale=-1.0),
               dict(scale=float("nan")), dict(reserved=5), dict(weights=1), dict(wout=A),
               dict(win=A)):
        assert attend(**kw) == L.ERR_BAD_PARAM, kw
    for kw in (dict(num_heads=130), dict(max_tokens=(1 << 20) + 1),
               dict(num_queries=(1 << 20) + 1), dict(batch=1 << 20, num_queries=1 << 10)):
        assert attend(**kw) == L.ERR_UNSUPPORTED, kw
    for kw in (dict(q=A + 8), dict(out=A + 4), dict(lengths=A + 1), dict(count=A + 2),
               dict(q_stride=(512, 128, 60)), dict(out_stride=(516, 128, 64)),
               dict(weights=1, wout=A + 2), dict(weights=1, wout=A, win=A + 1),
               dict(max_tokens=5000, ws=A + 16)):
        assert attend(**kw) == L.ERR_MISALIGNED, kw
    assert attend(max_tokens=5000, ws=None) == L.ERR_NULL_POINTER
    assert attend(max_tokens=5000, ws_bytes=16) == L.ERR_WORKSPACE_TOO_SMALL
    assert attend(weights=1, wout=A, ws_bytes=16) == L.ERR_WORKSPACE_TOO_SMALL


def test_attend_workspace():
    """Nothing for a call of one part; with weights, few rows' logits (and the rows' sums,
    where the weights are a launch of their own)."""
    def size(**kw):
        n = ctypes.c_size_t(0)
        c = desc()
        assert lib.e2s_cache_attend_workspace_size(ctypes.byref(c),
                                                   ctypes.byref(attend_shape(**kw)),
                                                   ctypes.byref(n)) == L.OK
        return n.value

    def up(x):
        return (x + 255) // 256 * 256
    assert size() == 0
    rows = 3 * 2 * 2 * 2                                 # B Hkv (H / Hkv) T
    assert size(weights=1) == up(rows * 128 * 4)
    assert size(weights=1, num_queries=20) == up(10 * rows * 4)
    assert size(max_tokens=100000) > 0
    c = desc()
    sh = attend_shape()
    assert lib.e2s_cache_attend_workspace_size(ctypes.byref(c), ctypes.byref(sh), None) == \
        L.ERR_NULL_POINTER


def evict(cache=None, pages=A, lengths=A, weights=A, new=2 * A, keep=A, kept=A, left=None, **kw):
    f = dict(batch=3, max_tokens=100, budget=40, sinks=4, recent=8, max_pages=7, new_max_pages=3,
             left_tokens=40, pages_stride=7, new_pages_stride=3)
    st = dict(weights_stride=(200, 100), left_stride=(80, 40))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = S.EvictShape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    cache = desc() if cache is None else cache
    return lib.e2s_cache_evict(ctypes.byref(cache), ctypes.byref(sh), pages, lengths, weights, new,
                               keep, kept, left, None)


def test_evict_refusals():
    for kw in (dict(pages=None), dict(lengths=None), dict(weights=None), dict(new=None),
               dict(keep=None), dict(kept=None)):
        assert evict(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(max_tokens=0), dict(budget=0), dict(max_pages=0),
               dict(new_max_pages=0), dict(new_max_pages=2), dict(left_tokens=39),
               dict(pages_stride=-1), dict(weights_stride=(-1, 100)), dict(left_stride=(0, 40))):
        assert evict(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(sinks=-1), dict(recent=-1), dict(sinks=33, recent=8), dict(new=A),
               dict(left=A)):
        assert evict(**kw) == L.ERR_BAD_PARAM, kw
    for kw in (dict(max_tokens=(1 << 20) + 1), dict(batch=1 << 21)):
        assert evict(**kw) == L.ERR_UNSUPPORTED, kw
    for kw in (dict(pages=A + 2), dict(weights=A + 1), dict(keep=A + 2), dict(left=2 * A + 1)):
        assert evict(**kw) == L.ERR_MISALIGNED, kw


def test_in_place_only_with_the_same_strides():
    """Refused before anything is enqueued: an output in its input's place, laid out
    otherwise, and the new lengths in the old ones' place."""
    assert rotate(qo=A, q_out_stride=(1280, 64, 256)) == L.ERR_BAD_PARAM
    assert rotate(ko=A, k_out_stride=(640, 64, 128)) == L.ERR_BAD_PARAM
    for strides in ((300, 100), (200, 101)):
        assert attend(weights=1, win=A, wout=A, weights_out_stride=strides) == L.ERR_BAD_PARAM
    assert attend(scale=3e38) == L.ERR_BAD_PARAM
    assert evict(lengths=3 * A, kept=3 * A) == L.ERR_BAD_PARAM


def test_validation_under_asan_and_ubsan(tmp_path):
    """serve_validate.cpp on random, often extreme, arguments."""
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2608_23253_amd", "csrc")
    exe = tmp_path / "serve_fuzz"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           f"-I{os.path.join(root, 'include')}", f"-I{csrc}",
           os.path.join(root, "tests", "native", "serve_fuzz.cpp"),
           os.path.join(csrc, "serve_validate.cpp"), os.path.join(csrc, "e2s_validate.cpp"),
           "-o", str(exe)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "0 failures" in run.stdout, run.stdout + run.stderr


# ---------------------------------------------------------------------------
# the binding
# ---------------------------------------------------------------------------

def test_binding_refuses_cpu_tensors_and_wrong_types():
    torch = pytest.importorskip("torch")
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    plan = S.rotary_plan(64)
    with pytest.raises(ValueError):
        S.rotate_positions(x, None, torch.zeros(3, dtype=torch.int32), plan)
    with pytest.raises(ValueError):
        S.rotate_positions(None, None, None, plan)
    with pytest.raises(ValueError):
        S.PagedCache.of(*[torch.zeros((2, 1, 16, 64), dtype=S._torch().float8_e4m3fn)] * 2,
                        *[torch.zeros((2, 1))] * 2)
    with pytest.raises(ValueError):
        S.PagedCache(2, 1, 64, 16, device="cpu")
    with pytest.raises(ValueError):
        S.cache_attend(x, None, None, None)
