"""Host-side checks of the attention calls that need no GPU: struct layouts, workspace arithmetic and
the arguments that are refused before anything is enqueued."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

import paper_2502_11494_amd as D
from paper_2502_11494_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 4096  # never dereferenced


def test_struct_layouts_match_the_header():
    lines = []
    for name, cls in (("dart_rotation", D.DartRotation), ("dart_cache", D.DartCache)):
        lines += [f'printf("%zu ", sizeof({name}));']
        lines += [f'printf("%zu ", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "dart.h"\nint main(){%s return 0;}\n' % "\n".join(lines)
    with tempfile.TemporaryDirectory() as td:
        c, exe = os.path.join(td, "t.c"), os.path.join(td, "t")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        out = list(map(int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()))
    want = []
    for cls in (D.DartRotation, D.DartCache):
        want += [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert out == want


def cache(**kw):
    c = D.DartCache()
    v = dict(B=2, Hq=8, Hkv=2, d=128, dtype=D.DART_BF16, T=5, max_q=4, max_kv=300, cu_q=FAKE, kv_len=FAKE, pages=FAKE,
             pages_ld=20, n_pages=50, page_size=16, page_ld=2 * 16 * 128, head_ld=16 * 128, row_ld=128)
    v.update(kw)
    for k, x in v.items():
        setattr(c, k, x)
    return c


def rotation(**kw):
    r = D.DartRotation()
    v = dict(Hq=8, Hkv=2, d=128, dtype=D.DART_BF16, rot=128, planes=1, inv_freq=FAKE, eps=1e-6, scale=1.0)
    v.update(kw)
    sections = v.pop("sections", None)
    for k, x in v.items():
        setattr(r, k, x)
    if sections:
        r.sections[:len(sections)] = sections
    return r


BAD_CACHE = [
    (dict(B=-1), D.DART_ERR_SHAPE), (dict(B=2 ** 20 + 1), D.DART_ERR_SHAPE), (dict(T=-1), D.DART_ERR_SHAPE),
    (dict(T=2 ** 24 + 1), D.DART_ERR_SHAPE), (dict(max_q=-1), D.DART_ERR_SHAPE), (dict(max_kv=-1), D.DART_ERR_SHAPE),
    (dict(max_kv=2 ** 27 + 1), D.DART_ERR_SHAPE), (dict(Hq=9), D.DART_ERR_SHAPE), (dict(Hq=0), D.DART_ERR_SHAPE),
    (dict(Hkv=0), D.DART_ERR_SHAPE), (dict(Hq=1026), D.DART_ERR_SHAPE), (dict(d=0), D.DART_ERR_SHAPE),
    (dict(d=124), D.DART_ERR_SHAPE), (dict(d=264, row_ld=264), D.DART_ERR_SHAPE), (dict(dtype=2), D.DART_ERR_DTYPE),
    (dict(page_size=0), D.DART_ERR_SHAPE), (dict(page_size=24), D.DART_ERR_SHAPE), (dict(page_size=2 ** 21), D.DART_ERR_SHAPE),
    (dict(n_pages=0), D.DART_ERR_SHAPE), (dict(pages_ld=0), D.DART_ERR_SHAPE), (dict(row_ld=120), D.DART_ERR_SHAPE),
    (dict(row_ld=132), D.DART_ERR_ALIGN), (dict(head_ld=4), D.DART_ERR_ALIGN), (dict(page_ld=4100), D.DART_ERR_ALIGN),
    (dict(head_ld=-8), D.DART_ERR_SHAPE), (dict(page_ld=2 ** 41), D.DART_ERR_SHAPE), (dict(cu_q=None), D.DART_ERR_SHAPE),
    (dict(kv_len=None), D.DART_ERR_NULL), (dict(pages=None), D.DART_ERR_NULL),
    (dict(groups=3), D.DART_ERR_SHAPE), (dict(groups=-1), D.DART_ERR_SHAPE),
    (dict(groups=1, prefix_ld=4, max_prefix=9, group_cu=FAKE, prefix_pages=FAKE), D.DART_ERR_NULL),
    (dict(groups=1, prefix_ld=0, max_prefix=9, group_cu=FAKE, prefix_pages=FAKE, prefix_len=FAKE), D.DART_ERR_SHAPE),
    (dict(groups=1, prefix_ld=4, max_prefix=-1, group_cu=FAKE, prefix_pages=FAKE, prefix_len=FAKE), D.DART_ERR_SHAPE),
]


def attend(c, q=FAKE, q_ld=1024, kp=FAKE, vp=FAKE, scale=0.1, out=FAKE, out_ld=1024, ws=FAKE, ws_bytes=1 << 40):
    return binding.lib().dart_attend(C.byref(c) if c is not None else None, q, q_ld, kp, vp, scale, 1, out, out_ld, None, ws,
                                     ws_bytes, None, None)


def append(r, c, q=FAKE, q_ld=1536, k=FAKE, v=FAKE, k_ld=1536, v_ld=1536, pos=FAKE, plane=5, qo=FAKE, ko=None, ko_ld=0, kp=FAKE,
           vp=FAKE):
    return binding.lib().dart_norm_rotate_append(C.byref(r) if r is not None else None, C.byref(c) if c is not None else None, q,
                                                 q_ld, k, k_ld, v, v_ld, pos, plane, qo, 1024, ko, ko_ld, None, kp, vp, None, None)


def rotate(r, T=5, q=FAKE, q_ld=1536, k=FAKE, pos=FAKE, plane=5, qo=FAKE, ko=FAKE):
    return binding.lib().dart_norm_rotate(C.byref(r) if r is not None else None, T, q, q_ld, k, 1536, pos, plane, qo, 1024, ko, 256,
                                          None, None)


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches_are_refused(kw, code):
    c = cache(**kw)
    assert D.dart_attend_workspace_bytes(c) == 0
    assert attend(c) == code
    assert append(rotation(), c) == code


def test_workspace_grows_with_the_problem_and_is_asked_for():
    small, big = D.dart_attend_workspace_bytes(cache()), D.dart_attend_workspace_bytes(
        cache(B=64, T=64, cu_q=None, max_kv=100000, pages_ld=10000))
    assert 0 < small <= big and small % 256 == 0 and big % 256 == 0
    need = D.dart_attend_workspace_bytes(cache())
    assert attend(cache(), ws=None) == D.DART_ERR_WORKSPACE
    assert attend(cache(), ws=FAKE + 16) == D.DART_ERR_WORKSPACE
    assert attend(cache(), ws_bytes=need - 1) == D.DART_ERR_WORKSPACE
    with pytest.raises(D.DartError):
        D.alloc_attend_workspace(cache(page_size=3))


def test_bad_arguments_of_attend_are_refused():
    assert attend(None) == D.DART_ERR_NULL
    for kw in (dict(q=None), dict(kp=None), dict(vp=None), dict(out=None)):
        assert attend(cache(), **kw) == D.DART_ERR_NULL
    for kw in (dict(q=FAKE + 2), dict(kp=FAKE + 8), dict(vp=FAKE + 8), dict(out=FAKE + 8), dict(q_ld=1028), dict(out_ld=1028)):
        assert attend(cache(), **kw) == D.DART_ERR_ALIGN
    for kw in (dict(q_ld=1016), dict(out_ld=1016), dict(q_ld=2 ** 25), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(cache(), **kw) == D.DART_ERR_SHAPE
    # nothing to do: nothing else is looked at
    assert attend(cache(T=0), q=None) == D.DART_OK
    assert attend(cache(B=0, T=0, kv_len=None, pages=None), q=None) == D.DART_OK


BAD_ROTATION = [
    (dict(Hq=7), D.DART_ERR_SHAPE), (dict(d=20), D.DART_ERR_SHAPE), (dict(dtype=5), D.DART_ERR_DTYPE), (dict(rot=130), D.DART_ERR_SHAPE),
    (dict(rot=12), D.DART_ERR_SHAPE), (dict(rot=-8), D.DART_ERR_SHAPE), (dict(planes=0), D.DART_ERR_SHAPE),
    (dict(planes=5), D.DART_ERR_SHAPE), (dict(planes=2, sections=[32, 31]), D.DART_ERR_SHAPE),
    (dict(planes=2, sections=[32, 33]), D.DART_ERR_SHAPE), (dict(planes=2, sections=[-1, 65]), D.DART_ERR_SHAPE),
    (dict(planes=2, sections=[2 ** 31 - 1, 65]), D.DART_ERR_SHAPE),
    (dict(eps=-1.0), D.DART_ERR_SHAPE), (dict(eps=float("nan")), D.DART_ERR_SHAPE), (dict(eps=float("inf")), D.DART_ERR_SHAPE),
    (dict(scale=float("inf")), D.DART_ERR_SHAPE), (dict(inv_freq=None), D.DART_ERR_NULL), (dict(q_weight=FAKE + 2), D.DART_ERR_ALIGN),
    (dict(k_weight=FAKE + 8), D.DART_ERR_ALIGN),
]


@pytest.mark.parametrize("kw,code", BAD_ROTATION)
def test_bad_rotations_are_refused(kw, code):
    assert rotate(rotation(**kw)) == code
    assert append(rotation(**kw), cache()) == code


def test_bad_arguments_of_the_rotation_are_refused():
    assert rotate(None) == D.DART_ERR_NULL and append(None, cache()) == D.DART_ERR_NULL
    assert append(rotation(), None) == D.DART_ERR_NULL
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(qo=None), dict(ko=None)):
        assert rotate(rotation(), **kw) == D.DART_ERR_NULL
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(qo=None), dict(kp=None), dict(vp=None)):
        assert append(rotation(), cache(), **kw) == D.DART_ERR_NULL
    assert rotate(rotation(), q=FAKE + 4) == D.DART_ERR_ALIGN and rotate(rotation(), q_ld=1530) == D.DART_ERR_ALIGN
    assert rotate(rotation(), q_ld=1000) == D.DART_ERR_SHAPE
    assert rotate(rotation(planes=2, sections=[32, 32]), plane=4) == D.DART_ERR_SHAPE  # planes would overlap
    assert rotate(rotation(), T=-1) == D.DART_ERR_SHAPE and rotate(rotation(), T=2 ** 24 + 1) == D.DART_ERR_SHAPE
    assert append(rotation(), cache(), v_ld=248) == D.DART_ERR_SHAPE
    assert append(rotation(), cache(), ko=FAKE, ko_ld=8) == D.DART_ERR_SHAPE
    assert append(rotation(dtype=D.DART_F32), cache()) == D.DART_ERR_DTYPE
    assert append(rotation(Hq=4), cache()) == D.DART_ERR_SHAPE
    assert append(rotation(d=64, rot=64), cache()) == D.DART_ERR_SHAPE
    assert rotate(rotation(), T=0, q=None) == D.DART_OK and append(rotation(), cache(T=0), q=None) == D.DART_OK


def test_the_binding_refuses_tensors_that_do_not_fit():
    t = torch.bfloat16
    pool, pages, kv = torch.zeros((4, 2, 16, 64), dtype=t), torch.zeros((3, 2), dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    D.make_cache(4, pool, pages, kv, 32)
    D.make_cache(4, torch.zeros((4, 16, 2, 64), dtype=t).transpose(1, 2), pages, kv, 32)
    for bad in (lambda: D.make_cache(4, pool.transpose(2, 3), pages, kv, 32), lambda: D.make_cache(4, pool, pages.long(), kv, 32),
                lambda: D.make_cache(4, pool, pages, kv[:2], 32), lambda: D.make_cache(4, pool.half(), pages, kv, 32),
                lambda: D.make_cache(4, pool, pages, kv, 32, cu_q=torch.zeros(4, dtype=torch.int32)),
                lambda: D.make_cache(4, pool, pages, kv, 32, cu_q=torch.zeros(3, dtype=torch.int32), T=3),
                lambda: D.make_rotation(4, 2, 64, D.DART_BF16, torch.ones(32, dtype=torch.float64)),
                lambda: D.make_rotation(4, 2, 64, D.DART_BF16, torch.ones(32), sections=[16, 15]),
                lambda: D.make_rotation(4, 2, 64, D.DART_BF16, torch.ones(32), q_weight=torch.ones(64))):
        with pytest.raises(ValueError):
            bad()
    c = D.make_cache(4, pool, pages, kv, 32)
    r = D.make_rotation(4, 2, 64, D.DART_BF16, torch.ones(32))
    q, k, ws = torch.zeros((3, 256), dtype=t), torch.zeros((3, 128), dtype=t), torch.zeros(256, dtype=torch.uint8)
    pos = torch.zeros(3, dtype=torch.int64)
    for bad in (lambda: D.dart_attend(c, q.float(), pool, pool, q, ws, scale=1.0), lambda: D.dart_attend(c, q[:2], pool, pool, q, ws, scale=1.0),
                lambda: D.dart_attend(c, q, pool[:3], pool, q, ws, scale=1.0), lambda: D.dart_attend(c, q, pool, pool.transpose(1, 2), q, ws, scale=1.0),
                lambda: D.dart_attend(c, q, pool, pool, q, ws, scale=1.0, lse=torch.zeros((3, 3))),
                lambda: D.dart_norm_rotate(r, q, k, pos[:2], q, k), lambda: D.dart_norm_rotate(r, q, k, pos.int(), q, k),
                lambda: D.dart_norm_rotate(r, q, q, pos, q, k), lambda: D.dart_norm_rotate(r, q, k[:2], pos, q, k),
                lambda: D.dart_norm_rotate(r, q, k, pos, q, k, l1_out=torch.zeros(2)),
                lambda: D.dart_norm_rotate_append(r, c, q, k, q, pos, q, pool, pool)):
        with pytest.raises(ValueError):
            bad()
