"""Host-side checks of the calls on 4-bit pages, gathered weights and eviction that need no GPU: struct layout, workspace
arithmetic, the arguments that are refused before anything is enqueued, and the host code under the host sanitizers."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import more_util as U
import paper_2502_11494_amd as D
from paper_2502_11494_amd import binding, build
from test_attend_host import BAD_CACHE, FAKE, ROOT, cache


def test_the_eviction_descriptor_matches_the_header(tmp_path):
    fields = [f for f, _ in D.DartEviction._fields_]
    src = ('#include <stdio.h>\n#include <stddef.h>\n#include "dart.h"\nint main(){printf("%zu ", sizeof(dart_eviction));'
           + "".join(f'printf("%zu ", offsetof(dart_eviction, {f}));' for f in fields) + "return 0;}\n")
    (tmp_path / "t.c").write_text(src)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), tmp_path / "t.c", "-o", tmp_path / "t"], check=True)
    out = list(map(int, subprocess.run([tmp_path / "t"], capture_output=True, text=True, check=True).stdout.split()))
    assert out == [C.sizeof(D.DartEviction)] + [getattr(D.DartEviction, f).offset for f in fields]


def test_the_host_code_is_clean_under_asan_and_ubsan():
    outdir = os.path.join(ROOT, "_build")
    build.build_host_sanitized(outdir)
    exe = os.path.join(outdir, "more_host_sanitize")
    subprocess.run(["/opt/rocm/llvm/bin/clang", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "more_host_sanitize.c"), "-L", outdir,
                    "-ldart_hip_san", "-Wl,-rpath," + outdir, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "sanitize ok" in r.stdout, (r.returncode, r.stdout[-300:], r.stderr[-3000:])


def eviction(**kw):
    e = D.DartEviction()
    for k, x in dict(dict(budget=20, ratio_num=0, ratio_den=1, first=2, recent=3), **kw).items():
        setattr(e, k, x)
    return e


def ref(x):
    return None if x is None else C.byref(x)


def attend(c, q=FAKE, q_ld=1024, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, scale=0.1, out=FAKE, out_ld=1024, ws=FAKE, ws_bytes=1 << 40):
    return binding.lib().dart_attend_4bit(ref(c), q, q_ld, kc, ks, vc, vs, scale, 1, out, out_ld, None, ws, ws_bytes, None, None)


def append(c, k=FAKE, k_ld=256, v=FAKE, v_ld=256, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE):
    return binding.lib().dart_append_4bit(ref(c), k, k_ld, v, v_ld, kc, ks, vc, vs, None, None)


def read(c, k=FAKE, k_ld=256, v=FAKE, v_ld=256, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE):
    return binding.lib().dart_read_4bit(ref(c), kc, ks, vc, vs, k, k_ld, v, v_ld, None, None)


def weights(c, q=FAKE, q_ld=1024, k=FAKE, ks=None, lse=FAKE, scale=0.1, carry=1.0, w=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return binding.lib().dart_attend_weights(ref(c), q, q_ld, k, ks, lse, scale, 1, carry, w, ws, ws_bytes, None, None)


def evict(c, e, k=FAKE, ks=None, v=FAKE, vs=None, w=FAKE, w_out=None, kept=None, kept_ld=0, left=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return binding.lib().dart_evict(ref(c), ref(e), k, ks, v, vs, w, w_out, kept, kept_ld, left, ws, ws_bytes, None, None)


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches_are_refused(kw, code):
    c = cache(**kw)
    assert weights(c) == code and evict(c, eviction()) == code
    assert D.binding.lib().dart_attend_weights_workspace_bytes(C.byref(c), 0) == 0
    # (what is wrong with the strides of rows may do for codes, and the other way round)
    if not any(k.endswith("_ld") for k in kw) or kw.get("row_ld") == 264:
        assert attend(c) == code and append(c) == code and read(c) == code and weights(c, ks=FAKE) == code
        assert evict(c, eviction(), ks=FAKE, vs=FAKE) == code and D.dart_attend_4bit_workspace_bytes(c) == 0


@pytest.mark.parametrize("kw,code", [(dict(row_ld=136), D.DART_ERR_ALIGN), (dict(head_ld=2056), D.DART_ERR_ALIGN),
                                     (dict(page_ld=16), D.DART_ERR_ALIGN), (dict(d=72, row_ld=80), D.DART_ERR_SHAPE),
                                     (dict(row_ld=96), D.DART_ERR_SHAPE), (dict(page_ld=2 ** 34), D.DART_ERR_SHAPE)])
def test_strides_of_codes_are_whole_blocks(kw, code):
    c = cache(**kw)
    assert attend(c) == code and append(c) == code and read(c) == code and weights(c, ks=FAKE) == code
    assert evict(c, eviction(), ks=FAKE, vs=FAKE) == code


def test_bad_arguments_are_refused():
    c = cache()
    assert attend(None) == append(None) == read(None) == weights(None) == evict(None, eviction()) == D.DART_ERR_NULL
    for kw in (dict(q=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(out=None)):
        assert attend(c, **kw) == D.DART_ERR_NULL
    for kw in (dict(k=None), dict(v=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None)):
        assert append(c, **kw) == D.DART_ERR_NULL
    for kw in (dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None)):
        assert read(c, **kw) == D.DART_ERR_NULL
    for kw in (dict(q=None), dict(k=None), dict(lse=None), dict(w=None)):
        assert weights(c, **kw) == D.DART_ERR_NULL
    for kw in (dict(k=None), dict(v=None), dict(w=None), dict(left=None), dict(ks=FAKE), dict(vs=FAKE)):
        assert evict(c, eviction(), **kw) == D.DART_ERR_NULL
    assert evict(c, None) == D.DART_ERR_NULL
    assert attend(c, kc=FAKE + 8) == append(c, vc=FAKE + 8) == read(c, kc=FAKE + 8) == D.DART_ERR_ALIGN
    assert weights(c, k=FAKE + 8) == evict(c, eviction(), v=FAKE + 8) == D.DART_ERR_ALIGN
    assert append(c, k=FAKE + 2) == read(c, v=FAKE + 2) == weights(c, q=FAKE + 2) == D.DART_ERR_ALIGN
    assert append(c, k_ld=248) == read(c, v_ld=248) == weights(c, q_ld=1016) == D.DART_ERR_SHAPE
    for bad in (float("nan"), float("inf")):
        assert attend(c, scale=bad) == weights(c, scale=bad) == weights(c, carry=bad) == D.DART_ERR_SHAPE
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=0)):
        assert attend(c, **kw) == weights(c, **kw) == evict(c, eviction(), **kw) == D.DART_ERR_WORKSPACE
    for kw in (dict(budget=-1), dict(first=-1), dict(recent=-1), dict(first=2 ** 27 + 1), dict(recent=2 ** 31 - 1)):
        assert evict(c, eviction(**kw)) == D.DART_ERR_SHAPE
    for kw in (dict(ratio_den=0), dict(ratio_num=-1), dict(ratio_num=2)):
        assert evict(c, eviction(budget=0, **kw)) == D.DART_ERR_BUDGET
    assert evict(c, eviction(), kept=FAKE, kept_ld=19) == D.DART_ERR_SHAPE
    # nothing to do: nothing else is looked at
    for call in (attend, append, read, weights):
        assert call(cache(T=0)) == D.DART_OK
    assert read(c, k=None, v=None, kc=None) == D.DART_OK
    assert evict(cache(B=0, T=0, kv_len=None, pages=None), eviction(), k=None) == D.DART_OK
    # scales may begin anywhere, and codes need no cache of their own
    assert attend(c, ks=FAKE + 1, ws=None) == D.DART_ERR_WORKSPACE


def test_sizes():
    c = cache()
    assert binding.lib().dart_evict_most(C.byref(c), C.byref(eviction()), 0) == 20
    for kw, most in ((dict(budget=2), 5), (dict(budget=1000), 300), (dict(budget=0, ratio_num=1, ratio_den=7), 42),
                     (dict(budget=0), 5), (dict(first=200, recent=200), 300), (dict(first=2 ** 27, recent=2 ** 27), 300)):
        assert binding.lib().dart_evict_most(C.byref(c), C.byref(eviction(**kw)), 0) == most
    assert binding.lib().dart_evict_most(C.byref(cache(page_size=3)), C.byref(eviction()), 0) == -1
    assert binding.lib().dart_attend_weights_workspace_bytes(C.byref(cache(B=2 ** 20, T=2 ** 20, cu_q=None, max_kv=2 ** 27)), 0) == 0
    assert weights(cache(B=2 ** 20, T=2 ** 20, cu_q=None, max_kv=2 ** 27)) == D.DART_ERR_SHAPE
    assert binding.lib().dart_evict_workspace_bytes(C.byref(cache(B=2 ** 20, T=2 ** 20, cu_q=None, max_kv=2 ** 27)),
                                                    C.byref(eviction(budget=2 ** 27)), 0) == 0


def test_the_format_holds_what_it_says():
    """The definition of the tests against worked examples."""
    x = torch.zeros(2, 40)
    x[0, :8] = torch.tensor([6.0, -6.9, 0.25, 0.75, -1.25, 2.5, 3.5, 5.0])
    x[1, 0], x[1, 33] = 7.0, float("inf")
    codes, scales = U.pack(x)
    assert codes.shape == (2, 32) and scales.shape == (2, 2)
    assert U.unpack((codes, scales), 40)[0, :8].tolist() == [6.0, -6.0, 0.0, 1.0, -1.0, 2.0, 4.0, 4.0]
    assert scales.tolist() == [[127, 0], [128, 255]] and codes[0, :2].tolist() == [0xf7, 0x20]
    y = U.unpack((codes, scales), 40)
    assert y[1, 0] == 8.0 and torch.isnan(y[1, 32:]).all()  # (7 = 3.5 units of 2, a tie: 4)


def test_the_binding_refuses_tensors_that_do_not_fit():
    t, u8 = torch.bfloat16, torch.uint8
    pool = D.alloc_pool_4bit(4, 2, 16, 80, device="cpu")
    assert [x.shape for x in pool] == [(4, 2, 16, 48), (4, 2, 16, 3)]
    pages, kv = torch.zeros((3, 2), dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    make = lambda p, **kw: D.make_cache_4bit(kw.pop("Hq", 4), kw.pop("d", 80), kw.pop("dtype", D.DART_BF16), p, pages, kv, 32, **kw)  # noqa: E731
    c = make(pool)
    assert (c.row_ld, c.head_ld, c.page_ld) == (96, 16 * 96, 2 * 16 * 96)
    turned = tuple(torch.zeros((4, 16, 2, n), dtype=u8).transpose(1, 2) for n in (48, 3))
    r = make(turned)
    assert (r.row_ld, r.head_ld, r.page_ld) == (2 * 96, 96, 2 * 16 * 96)
    for bad in (lambda: make(pool, d=64), lambda: make((pool[0], pool[0])), lambda: make((pool[0], turned[1])), lambda: make((pool[0][:3], pool[1])),
                lambda: make((pool[0].int(), pool[1])), lambda: make(pool, dtype=7), lambda: make((pool[0].transpose(2, 3), pool[1]))):
        with pytest.raises(ValueError):
            bad()
    q, k = torch.zeros((3, 320), dtype=t), torch.zeros((3, 160), dtype=t)
    ws, w, lse, left = torch.zeros(256, dtype=u8), torch.zeros((4, 2, 16)), torch.zeros((3, 4)), torch.zeros(3, dtype=torch.int32)
    rows = torch.zeros((4, 2, 16, 80), dtype=t)
    plain = D.make_cache(4, rows, pages, kv, 32)
    e = D.make_eviction(budget=8)
    assert D.dart_evict_most(c, e) == D.dart_evict_most(plain, e) == 8
    with pytest.raises(ValueError):
        D.make_eviction(first=4)  # (which would keep nothing else)
    with pytest.raises(D.DartError):
        D.dart_evict_most(c, D.make_eviction(budget=-1))
    with pytest.raises(D.DartError):
        D.alloc_evict_workspace(c, D.make_eviction(ratio=(2, 1)), device="cpu")
    for bad in (lambda: D.dart_append_4bit(c, k, k, pool, turned), lambda: D.dart_append_4bit(c, k, q, pool, pool),
                lambda: D.dart_append_4bit(plain, k, k, pool, pool), lambda: D.dart_append_4bit(c, k, k, pool[0], pool),
                lambda: D.dart_read_4bit(c, pool, pool, k.float(), k), lambda: D.dart_read_4bit(c, rows, rows, k, k),
                lambda: D.dart_attend_4bit(c, q[:2], pool, pool, q, ws, scale=1.0), lambda: D.dart_attend_4bit(plain, q, rows, rows, q, ws, scale=1.0),
                lambda: D.dart_attend_4bit(c, q, pool, (pool[0], pool[1][:2]), q, ws, scale=1.0),
                lambda: D.dart_attend(c, q, pool, pool, q, ws, scale=1.0), lambda: D.dart_attend(c, q, pool[0], pool[0], q, ws, scale=1.0),
                lambda: D.dart_attend_weights(c, q, pool, None, w, ws, scale=1.0), lambda: D.dart_attend_weights(c, q, pool, lse[:2], w, ws, scale=1.0),
                lambda: D.dart_attend_weights(c, q, rows, lse, w, ws, scale=1.0), lambda: D.dart_attend_weights(plain, q, pool, lse, w, ws, scale=1.0),
                lambda: D.dart_attend_weights(c, q, pool, lse, w[:, :, :8], ws, scale=1.0),
                lambda: D.dart_evict(c, e, pool, pool, w.double(), left, ws), lambda: D.dart_evict(c, e, pool, pool, w, left.long(), ws),
                lambda: D.dart_evict(c, e, pool, pool, w, left, ws, kept=torch.zeros((3, 8), dtype=torch.int32)),
                lambda: D.dart_evict(c, e, pool, pool, w, left[:2], ws)):
        with pytest.raises(ValueError):
            bad()
