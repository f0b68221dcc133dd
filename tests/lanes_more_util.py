"""The kernels on caches held in 4 bits, on gathered weights and on eviction, built for the CPU like those of lanes_util: every
buffer between guard pages, so that an access out of bounds ends the process."""
import ctypes as C
import hashlib
import os
import re
import shutil
import subprocess

import torch

import lanes_util as L
import paper_2502_11494_amd as D
from paper_2502_11494_amd import binding

MORE = os.path.join(L.ROOT, "tests", "lanes_more")
OUT = os.path.join(L.ROOT, "_build", "lanes_more")
LAUNCH = re.compile(r"(k_\w+(?:<[^;]*?>)?)<<<(.*?)>>>\((.*?)\);", re.S)
NAMES = ("dart_append_4bit", "dart_read_4bit", "dart_attend_4bit_workspace_bytes", "dart_attend_4bit", "dart_attend_weights_workspace_bytes",
         "dart_attend_weights", "dart_evict_most", "dart_evict_workspace_bytes", "dart_evict")


def sources():
    """name -> text of what is compiled."""
    csrc = os.path.join(L.ROOT, "paper_2502_11494_amd", "csrc")
    read = lambda name: open(os.path.join(csrc, name)).read()  # noqa: E731
    files = L.sources()
    for name in ("fourbit_api", "evict_api"):
        api = read(name + ".hip")
        count = api.count("<<<")
        api, done = LAUNCH.subn(r"lanes_launch(__PRETTY_FUNCTION__, \2, [=] { lanes_shape(\2); \1(\3); });", api)
        assert count == done and "<<<" not in api
        files[name + ".cpp"] = L.replaced(api, '"../../include/dart.h"', '"dart.h"', 1)
    for name in ("fourbit.hpp", "k_fourbit.hpp", "k_attend4.hpp", "k_weights.hpp", "k_evict.hpp"):
        text = read(name).replace("extern __shared__ __align__(16) unsigned char lds[];", "unsigned char* const lds = lanes_lds();")
        text = text.replace('asm volatile("" : "+v"(x));', "")  # (which only holds the compiler)
        files[name] = text.replace("(__attribute__((address_space(3))) ", "(")
    # (a wave's loads have come back: on the CPU they always have)
    files["common.hpp"] = L.replaced(files["common.hpp"], 'asm volatile("s_waitcnt vmcnt(0)" ::: "memory");', "", 1)
    return files


def build():
    files = sources()
    own = [os.path.join(L.LANES, "lanes.cpp"), os.path.join(L.LANES, "hip", "hip_runtime.h"), os.path.join(MORE, "more.h"),
           os.path.join(L.ROOT, "include", "dart.h")]
    h = hashlib.sha256("".join(files[k] for k in sorted(files)).encode() + b"".join(open(p, "rb").read() for p in own)).hexdigest()
    lib, stamp = os.path.join(OUT, "liblanes_more.so"), os.path.join(OUT, "stamp")
    if os.path.exists(lib) and os.path.exists(stamp) and open(stamp).read() == h:
        return lib
    shutil.rmtree(OUT, ignore_errors=True)
    os.makedirs(OUT)
    for name, text in files.items():
        with open(os.path.join(OUT, name), "w") as f:
            f.write(text)
    with open(os.path.join(OUT, "shape.cpp"), "w") as f:
        f.write("#include <hip/hip_runtime.h>\ndim3 lanes_grid, lanes_block;\n")
    flags = ["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O3", "-march=native", "-g", "-fPIC", "-Wno-pass-failed", "-Wno-psabi",
             "-ffp-contract=off", "-fsanitize=bounds", "-fsanitize-trap=bounds", "-I", L.LANES, "-I", OUT, "-I",
             os.path.join(L.ROOT, "include")]
    parts = [os.path.join(OUT, x) for x in ("attend_api.cpp", "fourbit_api.cpp", "evict_api.cpp", "shape.cpp")]
    parts.append(os.path.join(L.LANES, "lanes.cpp"))
    runs = [subprocess.Popen([*flags, *(["-include", os.path.join(MORE, "more.h")] if "_api" in p else []), "-c", p, "-o",
                              os.path.join(OUT, os.path.basename(p) + ".o")]) for p in parts]
    assert [r.wait() for r in runs] == [0] * len(runs)
    subprocess.run([*flags, "-shared", *(os.path.join(OUT, os.path.basename(p) + ".o") for p in parts), "-o", lib], check=True)
    with open(stamp, "w") as f:
        f.write(h)
    return lib


_ready = False


def lib():
    """The library, which also stands behind lanes_util's buffers from here on."""
    global _ready
    if not _ready:
        M, ref = C.CDLL(build()), binding.lib()
        M.lanes_alloc.restype, M.lanes_alloc.argtypes = C.c_void_p, [C.c_size_t, C.c_size_t, C.c_int]
        M.lanes_free.argtypes = [C.c_void_p]
        M.lanes_launched.restype = C.c_char_p
        for name in (*NAMES, "dart_attend", "dart_attend_workspace_bytes", "dart_norm_rotate", "dart_norm_rotate_append"):
            f, like = getattr(M, name), getattr(ref, name)
            f.argtypes, f.restype = like.argtypes, like.restype
        L._lib, _ready = M, True
    return L._lib


def descriptor(c, buf, **how):
    """lanes_util's, with the strides of pools held in 4 bits where the case has those."""
    d = L.descriptor(c, buf, **how)
    if c.four is not None:
        page, Hkv, wide = c.page, d.Hkv, -(-c.d // 32) * 32
        d.row_ld, d.head_ld, d.page_ld = ((wide, page * wide, Hkv * page * wide) if c.order == "heads" else
                                          (Hkv * wide, wide, page * Hkv * wide))
    return d


class Call:
    """A library call's buffers: made, looked at and freed together."""

    def __init__(self, c, at_end=True, back=False, **how):
        self.L, self.buf = lib(), L.Buffers(at_end)
        self.L.lanes_order(int(back))
        self.c, self.d = c, descriptor(c, self.buf, **how)
        self.status = self.buf.copy(torch.zeros(1, dtype=torch.int32))
        self.L.lanes_forget()

    def pool(self, x):
        """Addresses of a pool: rows and None, or codes and scales."""
        if isinstance(x, tuple):
            return tuple(self.bytes(L.stored(self.c, t)) for t in x)
        return self.buf.copy(L.stored(self.c, x)), None

    def bytes(self, t):
        """(scales may begin anywhere; codes are a whole number of 16 bytes)"""
        t = t.contiguous()
        p = self.buf.room(t.numel(), 16 if t.numel() % 16 == 0 else 1)
        C.memmove(p, t.data_ptr(), t.numel())
        return p

    def pool_back(self, at, like):
        if isinstance(like, tuple):
            return tuple(self.pool_back((p, None), x) for p, x in zip(at, like))
        t = self.buf.back(at[0], like.dtype, L.stored(self.c, like).shape)
        return t.transpose(1, 2) if self.c.order == "rows" else t

    def ws(self, n):
        assert n > 0
        return self.buf.room(n, 256), n

    def done(self, rc):
        assert rc == D.DART_OK, rc
        return int(self.buf.back(self.status, torch.int32, 1))


def append(c, k, v, **how):
    """Pools after the call, the status word."""
    x = Call(c, **how)
    kp, vp = x.pool(c.four[0]), x.pool(c.four[1])
    width = x.d.Hkv * c.d
    status = x.done(x.L.dart_append_4bit(C.byref(x.d), x.buf.copy(k), width, x.buf.copy(v), width, *kp, *vp, x.status, None))
    got = x.pool_back(kp, c.four[0]), x.pool_back(vp, c.four[1]), status
    x.buf.free()
    return got


def read(c, fill=7.0, **how):
    x = Call(c, **how)
    width = x.d.Hkv * c.d
    out = [x.buf.copy(torch.full((c.T, width), fill, dtype=c.dtype)) for _ in range(2)]
    status = x.done(x.L.dart_read_4bit(C.byref(x.d), *x.pool(c.four[0]), *x.pool(c.four[1]), out[0], width, out[1], width, x.status, None))
    got = *(x.buf.back(p, c.dtype, (c.T, width)) for p in out), status
    x.buf.free()
    return got


def attend(c, *, scale, causal=True, **how):
    x = Call(c, **how)
    width = c.Hq * c.d
    out, lse = x.buf.room(c.T * width * c.q.element_size()), x.buf.room(c.T * c.Hq * 4, 4)
    ws, n = x.ws(x.L.dart_attend_4bit_workspace_bytes(C.byref(x.d)))
    status = x.done(x.L.dart_attend_4bit(C.byref(x.d), x.buf.copy(c.q), width, *x.pool(c.four[0]), *x.pool(c.four[1]), scale, int(causal), out,
                                         width, lse, ws, n, x.status, None))
    got = x.buf.back(out, c.dtype, (c.T, c.Hq, c.d)), x.buf.back(lse, torch.float32, (c.T, c.Hq)), status, x.L.lanes_launched().decode()
    x.buf.free()
    return got


def weights(c, lse, old, *, scale, causal=True, carry=1.0, **how):
    x = Call(c, **how)
    four = c.four is not None
    ws, n = x.ws(x.L.dart_attend_weights_workspace_bytes(C.byref(x.d), int(four)))
    w = x.buf.copy(old)
    status = x.done(x.L.dart_attend_weights(C.byref(x.d), x.buf.copy(c.q), c.Hq * c.d, *x.pool(c.four[0] if four else c.k_pool),
                                            x.buf.copy(lse), scale, int(causal), carry, w, ws, n, x.status, None))
    got = x.buf.back(w, torch.float32, old.shape), status, x.L.lanes_launched().decode()
    x.buf.free()
    return got


def evict(c, weights, *, budget=0, ratio=(0, 1), first=0, recent=0, out="other", keep=True, **how):
    """Pools, weights, kept places, lengths, status.  out: "other", "same" or None; keep: whether the places are asked for."""
    x = Call(c, **how)
    four = c.four is not None
    e = D.DartEviction()
    e.budget, e.ratio_num, e.ratio_den, e.first, e.recent = budget, *ratio, first, recent
    most = x.L.dart_evict_most(C.byref(x.d), C.byref(e), int(four))
    assert most >= 0
    ws, n = x.ws(x.L.dart_evict_workspace_bytes(C.byref(x.d), C.byref(e), int(four)))
    pools = [x.pool(p) for p in (c.four if four else (c.k_pool, c.v_pool))]
    w = x.buf.copy(weights)
    w_out = w if out == "same" else None if out is None else x.buf.copy(torch.full_like(weights, -5.0))
    kept = x.buf.copy(torch.full((x.d.B, x.d.Hkv, most), -1, dtype=torch.int32)) if keep else None
    left = x.buf.copy(torch.full((x.d.B,), -1, dtype=torch.int32))
    status = x.done(x.L.dart_evict(C.byref(x.d), C.byref(e), *pools[0], *pools[1], w, w_out, kept, most, left, ws, n, x.status, None))
    got = ([x.pool_back(p, like) for p, like in zip(pools, c.four if four else (c.k_pool, c.v_pool))],
           None if out is None else x.buf.back(w_out, torch.float32, weights.shape),
           x.buf.back(kept, torch.int32, (x.d.B, x.d.Hkv, most)) if keep else None, x.buf.back(left, torch.int32, (x.d.B,)), status)
    x.buf.free()
    return got
