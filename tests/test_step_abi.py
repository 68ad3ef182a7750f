"""Checks of e2s_step.h that need no GPU: exports, structure sizes, plans, and that every
invalid call is refused on the host before any launch (the fake device addresses below are
never dereferenced)."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

from paper_2608_23253_amd import _lib as L
from paper_2608_23253_amd import _serve as V
from paper_2608_23253_amd import _step as S

lib = L.lib()
A = 1 << 20


def test_exports_every_declared_entry_point():
    names = L.header_entry_points(S.HEADER)
    assert sorted(names) == sorted(S.SIGNATURES)
    for n in names:
        assert hasattr(lib, n), n
    assert lib.e2s_step_abi_version() == 1


def test_header_is_plain_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    src = tmp_path / "h.c"
    names = {"e2s_norm_rotate_shape": S.NormRotateShape, "e2s_cache4": S.Cache4Desc,
             "e2s_cache4_read_shape": S.Read4Shape, "e2s_cache4_attend_shape": S.Attend4Shape}
    src.write_text('#include "e2s_step.h"\n' + "".join(
        f"_Static_assert(sizeof({n}) == {ctypes.sizeof(t)}, \"{n}\");\n"
        for n, t in names.items()))
    run = subprocess.run([gcc, "-std=c11", "-Wall", "-Wextra", "-Werror", "-fsyntax-only",
                          f"-I{os.path.dirname(S.HEADER)}", str(src)], capture_output=True,
                         text=True)
    assert run.returncode == 0, run.stderr


def test_packed_records_have_the_structures_layout():
    for packed, t in ((S._NORM, S.NormRotateShape), (S._READ, S.Read4Shape),
                      (S._ATTEND, S.Attend4Shape), (S._APPEND, V.AppendShape)):
        assert packed.size == ctypes.sizeof(t)
    sh = S.Attend4Shape.from_buffer_copy(S._ATTEND.pack(*range(7), 0.5, *range(8, 15)))
    assert (sh.batch, sh.causal, sh.scale, sh.pages_stride, sh.out_stride[2]) == (0, 6, 0.5, 8, 14)
    sh = S.NormRotateShape.from_buffer_copy(S._NORM.pack(*range(6), 0.5, 7, *range(8, 29)))
    assert (sh.weight_dtype, sh.eps, sh.q_stride[0], sh.pos_stride[2]) == (5, 0.5, 8, 28)


# ---------------------------------------------------------------------------
# norm_rotate
# ---------------------------------------------------------------------------

def norm_shape(**kw):
    f = dict(batch=2, num_tokens=5, q_heads=4, k_heads=2, dtype=L.DTYPE_BF16,
             weight_dtype=L.DTYPE_BF16, eps=1e-6, reserved=0)
    st = dict(q_stride=(1280, 320, 64), k_stride=(640, 320, 64), q_grad_stride=(1280, 320, 64),
              k_grad_stride=(640, 320, 64), q_out_stride=(1280, 320, 64),
              k_out_stride=(640, 320, 64), pos_stride=(0, 5, 1))
    st.update({n: v for n, v in kw.items() if n in st})
    f.update({n: v for n, v in kw.items() if n not in st})
    sh = S.NormRotateShape(*f.values())
    for n, v in st.items():
        getattr(sh, n)[:] = v
    return sh


def norm(plan="good", pos=A, q=2 * A, k=3 * A, qw=4 * A, kw_=5 * A, qo=6 * A, ko=7 * A, **kw):
    plan = V.rotary_plan(64) if plan == "good" else plan
    return lib.e2s_norm_rotate(ctypes.byref(norm_shape(**kw)),
                               ctypes.byref(plan) if plan else None, pos, q, k, qw, kw_, qo, ko,
                               None)


def norm_back(pos=A, q=2 * A, k=3 * A, qw=4 * A, kw_=5 * A, gq=6 * A, gk=7 * A, qo=8 * A,
              ko=9 * A, dqw=10 * A, dkw=11 * A, work=12 * A, size=1 << 20, **kw):
    plan = V.rotary_plan(64)
    return lib.e2s_norm_rotate_backward(ctypes.byref(norm_shape(**kw)), ctypes.byref(plan), pos, q,
                                        k, qw, kw_, gq, gk, qo, ko, dqw, dkw, work, size, None)


SHAPE_ERRORS = [
    (dict(batch=0), L.ERR_BAD_SHAPE), (dict(num_tokens=-1), L.ERR_BAD_SHAPE),
    (dict(q_heads=-1), L.ERR_BAD_SHAPE), (dict(q_heads=0, k_heads=0), L.ERR_BAD_SHAPE),
    (dict(q_stride=(-1, 320, 64)), L.ERR_BAD_SHAPE),
    (dict(q_out_stride=(1280, 0, 64)), L.ERR_BAD_SHAPE),
    (dict(k_out_stride=(640, 320, 0)), L.ERR_BAD_SHAPE),
    (dict(pos_stride=(0, -5, 1)), L.ERR_BAD_SHAPE),
    (dict(k_stride=(1 << 62, 320, 64)), L.ERR_BAD_SHAPE), (dict(dtype=3), L.ERR_BAD_PARAM),
    (dict(weight_dtype=L.DTYPE_F16), L.ERR_BAD_PARAM), (dict(reserved=1), L.ERR_BAD_PARAM),
    (dict(eps=0.0), L.ERR_BAD_PARAM), (dict(eps=-1.0), L.ERR_BAD_PARAM),
    (dict(eps=float("nan")), L.ERR_BAD_PARAM), (dict(eps=float("inf")), L.ERR_BAD_PARAM),
    (dict(batch=1 << 12, num_tokens=1 << 12), L.ERR_UNSUPPORTED),
    (dict(q_heads=70000), L.ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", SHAPE_ERRORS)
def test_norm_rotate_refuses_shapes(kw, status):
    assert norm(**kw) == status
    assert norm_back(**kw) == status
    n = ctypes.c_size_t(7)
    plan = V.rotary_plan(64)
    assert lib.e2s_norm_rotate_backward_workspace_size(
        ctypes.byref(norm_shape(**kw)), ctypes.byref(plan), 1, ctypes.byref(n)) == status
    assert n.value == 7


def test_norm_rotate_refuses_pointers():
    assert norm(plan=None) == L.ERR_NULL_POINTER
    for kw in (dict(pos=None), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None)):
        assert norm(**kw) == L.ERR_NULL_POINTER, kw
    assert norm(q=2 * A + 1) == L.ERR_MISALIGNED
    assert norm(pos=A + 2) == L.ERR_MISALIGNED
    assert norm(qw=4 * A + 1) == L.ERR_MISALIGNED
    assert norm(weight_dtype=L.DTYPE_F32, kw_=5 * A + 2) == L.ERR_MISALIGNED
    assert norm(dtype=L.DTYPE_F32, weight_dtype=L.DTYPE_F32, ko=7 * A + 2) == L.ERR_MISALIGNED
    # each output is written while the other tensor is read or written
    assert norm(qo=7 * A) == L.ERR_BAD_PARAM
    assert norm(qo=3 * A) == L.ERR_BAD_PARAM and norm(ko=2 * A) == L.ERR_BAD_PARAM
    # in its input's place with other strides
    assert norm(qo=2 * A, q_out_stride=(1280, 64, 256)) == L.ERR_BAD_PARAM
    assert norm(num_tokens=0, q=None, k=None, qo=None, ko=None, pos=None) == L.OK
    # an absent tensor needs no pointer (the call then stops at the missing positions)
    assert norm(k_heads=0, k=None, ko=None, pos=None) == L.ERR_NULL_POINTER


def test_norm_rotate_backward_refuses():
    for kw in (dict(pos=None), dict(q=None), dict(k=None), dict(gq=None), dict(gk=None),
               dict(qo=None), dict(ko=None), dict(work=None)):
        assert norm_back(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(gq=6 * A + 1), dict(dqw=10 * A + 1), dict(work=12 * A + 128)):
        assert norm_back(**kw) == L.ERR_MISALIGNED, kw
    assert norm_back(size=10 * 2 * 64 * 4 - 1) == L.ERR_WORKSPACE_TOO_SMALL
    # no output is an input, or another output
    outs = dict(qo=8, ko=9, dqw=10, dkw=11)
    for n, other in itertools.product(outs, (2, 3, 4, 5, 6, 7, 8, 9, 10, 11)):
        if other != outs[n]:
            assert norm_back(**{n: other * A}) == L.ERR_BAD_PARAM, (n, other)
    assert norm_back(q_grad_stride=(1280, -1, 64)) == L.ERR_BAD_SHAPE


def test_norm_rotate_backward_workspace():
    plan, n = V.rotary_plan(64), ctypes.c_size_t(0)

    def size(want, **kw):
        assert lib.e2s_norm_rotate_backward_workspace_size(
            ctypes.byref(norm_shape(**kw)), ctypes.byref(plan), want, ctypes.byref(n)) == L.OK
        return n.value
    assert size(0) == 0 and size(1) == 10 * 2 * 64 * 4 and size(1, num_tokens=0) == 0
    assert size(1, batch=1, num_tokens=1 << 20) == 2048 * 2 * 64 * 4
    sh = norm_shape()
    assert lib.e2s_norm_rotate_backward_workspace_size(ctypes.byref(sh), ctypes.byref(plan), 2,
                                                       ctypes.byref(n)) == L.ERR_BAD_PARAM
    assert lib.e2s_norm_rotate_backward_workspace_size(ctypes.byref(sh), ctypes.byref(plan), 1,
                                                       None) == L.ERR_NULL_POINTER
    assert lib.e2s_norm_rotate(None, ctypes.byref(plan), A, A, A, A, A, A, A,
                               None) == L.ERR_NULL_POINTER


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------

def cache(**kw):
    f = dict(num_pages=9, page_tokens=32, num_kv_heads=2, head_dim=64, k_page_stride=2048,
             v_page_stride=2048, k=A, v=2 * A, k_scale=3 * A, v_scale=4 * A)
    f.update(kw)
    return S.Cache4Desc(*f.values())


CACHE_ERRORS = [
    (dict(num_pages=0), L.ERR_BAD_SHAPE), (dict(page_tokens=0), L.ERR_BAD_SHAPE),
    (dict(page_tokens=16), L.ERR_UNSUPPORTED), (dict(page_tokens=48), L.ERR_UNSUPPORTED),
    (dict(page_tokens=256), L.ERR_UNSUPPORTED), (dict(num_kv_heads=129), L.ERR_UNSUPPORTED),
    (dict(head_dim=96), L.ERR_UNSUPPORTED), (dict(head_dim=-1), L.ERR_BAD_SHAPE),
    (dict(k_page_stride=2047), L.ERR_BAD_SHAPE), (dict(v_page_stride=2056), L.ERR_MISALIGNED),
    (dict(v_page_stride=1 << 62), L.ERR_BAD_SHAPE), (dict(k=None), L.ERR_NULL_POINTER),
    (dict(v=None), L.ERR_NULL_POINTER), (dict(k_scale=None), L.ERR_NULL_POINTER),
    (dict(v_scale=None), L.ERR_NULL_POINTER), (dict(k=A + 8), L.ERR_MISALIGNED),
    (dict(v=A + 8), L.ERR_MISALIGNED), (dict(k_scale=A + 8), L.ERR_MISALIGNED),
    (dict(v_scale=A + 8), L.ERR_MISALIGNED),
]


def append(c=None, pages=A, start=A, count=None, idx=None, k=A, v=A, **kw):
    f = dict(batch=2, num_tokens=5, src_tokens=5, dtype=L.DTYPE_BF16, max_pages=4, reserved=0,
             pages_stride=4)
    st = dict(k_stride=(640, 320, 64), v_stride=(640, 320, 64))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = V.AppendShape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    return lib.e2s_cache4_append(ctypes.byref(c or cache()), ctypes.byref(sh), pages, start, count,
                                 idx, k, v, None)


def read(c=None, pages=A, start=A, count=None, k=A, v=2 * A, **kw):
    f = dict(batch=2, num_tokens=5, dtype=L.DTYPE_BF16, max_pages=4, pages_stride=4)
    st = dict(k_out_stride=(640, 320, 64), v_out_stride=(640, 320, 64))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = S.Read4Shape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    return lib.e2s_cache4_read(ctypes.byref(c or cache()), ctypes.byref(sh), pages, start, count, k,
                               v, None)


def attend_shape(**kw):
    f = dict(batch=2, num_heads=4, num_queries=3, dtype=L.DTYPE_BF16, max_tokens=100, max_pages=4,
             causal=1, scale=0.0, pages_stride=4)
    st = dict(q_stride=(768, 192, 64), out_stride=(768, 192, 64))
    st.update({n: x for n, x in kw.items() if n in st})
    f.update({n: x for n, x in kw.items() if n not in st})
    sh = S.Attend4Shape(*f.values())
    for n, x in st.items():
        getattr(sh, n)[:] = x
    return sh


def attend(c=None, pages=A, lengths=A, count=None, q=A, out=2 * A, work=3 * A, size=1 << 30, **kw):
    return lib.e2s_cache4_attend(ctypes.byref(c or cache()), ctypes.byref(attend_shape(**kw)),
                                 pages, lengths, count, q, out, work, size, None)


@pytest.mark.parametrize("kw,status", CACHE_ERRORS)
def test_every_call_refuses_a_bad_cache(kw, status):
    for call in (append, read, attend):
        assert call(c=cache(**kw)) == status
    n = ctypes.c_size_t(0)
    assert lib.e2s_cache4_attend_workspace_size(
        ctypes.byref(cache(**kw)), ctypes.byref(attend_shape()), ctypes.byref(n)) == status


def test_append_refusals():
    for kw in (dict(pages=None), dict(start=None), dict(k=None), dict(v=None)):
        assert append(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_tokens=-1), dict(src_tokens=0), dict(max_pages=0),
               dict(src_tokens=4), dict(k_stride=(640, -320, 64)), dict(pages_stride=-1)):
        assert append(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(dtype=3), dict(reserved=1)):
        assert append(**kw) == L.ERR_BAD_PARAM, kw
    for kw in (dict(k=A + 8), dict(v=A + 8), dict(start=A + 2), dict(count=A + 2), dict(idx=A + 2),
               dict(v_stride=(640, 324, 64))):
        assert append(**kw) == L.ERR_MISALIGNED, kw
    assert append(num_tokens=(1 << 20) + 1, src_tokens=1 << 21) == L.ERR_UNSUPPORTED
    assert append(batch=1 << 22) == L.ERR_UNSUPPORTED
    assert append(num_tokens=0, k=None, v=None, pages=None, start=None) == L.OK


def test_read_refusals():
    for kw in (dict(pages=None), dict(start=None), dict(k=None, v=None)):
        assert read(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_tokens=-1), dict(max_pages=0),
               dict(k_out_stride=(640, 320, 0)), dict(v_out_stride=(0, 320, 64))):
        assert read(**kw) == L.ERR_BAD_SHAPE, kw
    assert read(dtype=3) == L.ERR_BAD_PARAM and read(k=A, v=A) == L.ERR_BAD_PARAM
    for kw in (dict(k=A + 8), dict(v=A + 8), dict(pages=A + 2), dict(count=A + 1),
               dict(k_out_stride=(640, 324, 64))):
        assert read(**kw) == L.ERR_MISALIGNED, kw
    assert read(num_tokens=(1 << 20) + 1) == L.ERR_UNSUPPORTED
    assert read(num_tokens=0, k=None, v=None, pages=None, start=None) == L.OK


def test_attend_refusals():
    for kw in (dict(pages=None), dict(lengths=None), dict(q=None), dict(out=None)):
        assert attend(**kw) == L.ERR_NULL_POINTER, kw
    for kw in (dict(batch=0), dict(num_heads=0), dict(num_heads=3), dict(num_queries=0),
               dict(max_tokens=0), dict(max_pages=0), dict(q_stride=(-768, 192, 64)),
               dict(out_stride=(768, 0, 64))):
        assert attend(**kw) == L.ERR_BAD_SHAPE, kw
    for kw in (dict(dtype=3), dict(causal=2), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=3e38), dict(out=A)):
        assert attend(**kw) == L.ERR_BAD_PARAM, kw
    for kw in (dict(q=A + 8), dict(out=2 * A + 8), dict(lengths=A + 2), dict(count=A + 2),
               dict(q_stride=(768, 196, 64))):
        assert attend(**kw) == L.ERR_MISALIGNED, kw
    for kw in (dict(num_heads=130), dict(max_tokens=(1 << 20) + 1), dict(num_queries=1 << 21),
               dict(batch=1 << 24)):
        assert attend(**kw) == L.ERR_UNSUPPORTED, kw
    split = dict(max_tokens=1 << 20, max_pages=1 << 15)
    assert attend(work=None, **split) == L.ERR_NULL_POINTER
    assert attend(work=3 * A + 128, **split) == L.ERR_MISALIGNED
    assert attend(size=100, **split) == L.ERR_WORKSPACE_TOO_SMALL
    n = ctypes.c_size_t(0)
    assert lib.e2s_cache4_attend_workspace_size(ctypes.byref(cache()), None,
                                                ctypes.byref(n)) == L.ERR_NULL_POINTER
    assert lib.e2s_cache4_attend_workspace_size(
        ctypes.byref(cache()), ctypes.byref(attend_shape()), None) == L.ERR_NULL_POINTER


# ---------------------------------------------------------------------------
# on host code alone, with sanitizers: plans of random calls hold together
# ---------------------------------------------------------------------------

def test_plans_and_checks_under_sanitizers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2608_23253_amd", "csrc")
    exe = tmp_path / "step_fuzz"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           f"-I{os.path.join(root, 'include')}", f"-I{csrc}",
           os.path.join(root, "tests", "native", "step_fuzz.cpp"),
           *(os.path.join(csrc, n) for n in ("step_validate.cpp", "serve_validate.cpp",
                                             "e2s_validate.cpp")), "-o", str(exe)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and " 0 failures" in run.stdout, run.stdout[-2000:] + run.stderr
