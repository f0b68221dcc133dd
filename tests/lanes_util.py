"""The attention and rotation kernels, and the host code that launches them, built for the CPU (tests/lanes): every
buffer lies between guard pages, so that an access out of bounds ends the process, and a library call is a call.

The sources are compiled as they are but for three things that are not C++: launches, the declaration of the
workgroup's dynamic memory, and a pointer's address space."""
import ctypes as C
import hashlib
import os
import re
import shutil
import subprocess

import torch

import attend_util as A
import paper_2502_11494_amd as D
from paper_2502_11494_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LANES = os.path.join(ROOT, "tests", "lanes")
OUT = os.path.join(ROOT, "_build", "lanes")
LAUNCH = re.compile(r"(k_\w+<[^;]*?>)<<<(.*?)>>>\((.*?)\);", re.S)


def replaced(text, old, new, times):
    assert text.count(old) == times, (old, text.count(old))
    return text.replace(old, new)


def sources():
    """name -> text of what is compiled."""
    csrc = os.path.join(ROOT, "paper_2502_11494_amd", "csrc")
    read = lambda name: open(os.path.join(csrc, name)).read()  # noqa: E731
    api = read("attend_api.hip")
    count = api.count("<<<")
    api, done = LAUNCH.subn(r"lanes_launch(__PRETTY_FUNCTION__, \2, [=] { \1(\3); });", api)
    assert count == done == 6 and "<<<" not in api
    kernels = replaced(read("k_attend.hpp"), "extern __shared__ __align__(16) unsigned char lds[];",
                       "unsigned char* const lds = lanes_lds();", 2)
    kernels = replaced(kernels, "(__attribute__((address_space(3))) i16x4*)", "", 1)
    return {"attend_api.cpp": replaced(api, '"../../include/dart.h"', '"dart.h"', 1), "k_attend.hpp": kernels,
            "k_rotate.hpp": read("k_rotate.hpp"), "cache.hpp": read("cache.hpp"), "common.hpp": read("common.hpp")}


def build():
    """The library; compiled if the sources changed."""
    files = sources()
    own = [os.path.join(LANES, "lanes.cpp"), os.path.join(LANES, "hip", "hip_runtime.h"), os.path.join(ROOT, "include", "dart.h")]
    h = hashlib.sha256(("-O3 -march=native" + "".join(files[k] for k in sorted(files))).encode() + b"".join(open(p, "rb").read() for p in own)).hexdigest()
    lib, stamp = os.path.join(OUT, "liblanes.so"), os.path.join(OUT, "stamp")
    if os.path.exists(lib) and os.path.exists(stamp) and open(stamp).read() == h:
        return lib
    shutil.rmtree(OUT, ignore_errors=True)
    os.makedirs(OUT)
    for name, text in files.items():
        with open(os.path.join(OUT, name), "w") as f:
            f.write(text)
    subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O3", "-march=native", "-g", "-fPIC", "-shared", "-Wno-pass-failed", "-Wno-psabi",
                    "-ffp-contract=off", "-fsanitize=bounds", "-fsanitize-trap=bounds", "-I", LANES, "-I", OUT, "-I",
                    os.path.join(ROOT, "include"), os.path.join(OUT, "attend_api.cpp"), os.path.join(LANES, "lanes.cpp"), "-o", lib],
                   check=True)
    with open(stamp, "w") as f:
        f.write(h)
    return lib


_lib = None


def lib():
    global _lib
    if _lib is None:
        L, ref = C.CDLL(build()), binding.lib()
        L.lanes_alloc.restype, L.lanes_alloc.argtypes = C.c_void_p, [C.c_size_t, C.c_size_t, C.c_int]
        L.lanes_free.argtypes = [C.c_void_p]
        L.lanes_launched.restype = C.c_char_p
        for name in ("dart_attend", "dart_attend_workspace_bytes", "dart_norm_rotate", "dart_norm_rotate_append"):
            f, like = getattr(L, name), getattr(ref, name)
            f.argtypes, f.restype = like.argtypes, like.restype
        _lib = L
    return _lib


class Buffers:
    """Copies of tensors between guard pages, each of exactly its tensor's size."""

    def __init__(self, at_end):
        self.at_end, self.held = at_end, []

    def room(self, n, alignment=16):
        p = lib().lanes_alloc(n, alignment, self.at_end)
        self.held.append(p)
        return p

    def copy(self, t):
        t = t.contiguous()
        n = t.numel() * t.element_size()
        p = self.room(n, 4 if t.dtype == torch.int32 else 8 if t.dtype == torch.int64 else 16)
        C.memmove(p, t.data_ptr(), n)
        return p

    def back(self, p, dtype, shape):
        t = torch.empty(shape, dtype=dtype)
        C.memmove(t.data_ptr(), p, t.numel() * t.element_size())
        return t

    def free(self):
        for p in self.held:
            lib().lanes_free(p)
        self.held = []


def descriptor(c, buf, *, table=None, kv=None, cu=None, max_q=None, max_kv=None, packed=None, group_cu=None, prefix=None, max_prefix=None,
               ld=0, n_pages=None):
    """ld: entries of a table's row beyond its width (the table is a view of a wider one)."""
    d = D.DartCache()
    pages, Hkv, page, width = c.k_pool.shape
    packed = any(x != 1 for x in c.n) if packed is None else packed

    def wide(t):
        if ld == 0:
            return buf.copy(t), t.shape[1], 0
        # the row stride is ld more than the width; the last row ends at the guard page
        base = torch.full((t.shape[0], t.shape[1] + ld), 1 << 30, dtype=torch.int32)
        base[:, :t.shape[1]] = t
        return buf.copy(base.flatten()[:base.numel() - ld]), base.shape[1], t.shape[1]

    d.B, d.Hq, d.Hkv, d.d, d.dtype, d.T = len(c.n), c.Hq, Hkv, width, A.KIND[c.dtype], c.T
    d.max_q, d.max_kv = max(c.n) if max_q is None else max_q, max(c.kv) if max_kv is None else max_kv
    d.cu_q = buf.copy(c.cu if cu is None else cu) if packed else None
    d.kv_len = buf.copy(torch.tensor(c.kv, dtype=torch.int32) if kv is None else kv)
    d.pages, d.pages_ld, d.pages_n = wide(c.table if table is None else table)
    d.n_pages, d.page_size = pages if n_pages is None else n_pages, page
    d.row_ld, d.head_ld, d.page_ld = ((width, page * width, Hkv * page * width) if c.order == "heads" else
                                      (Hkv * width, width, page * Hkv * width))
    if c.group_of is not None:
        d.groups = len(c.group_of)
        first = torch.tensor([sum(c.group_of[:i]) for i in range(d.groups + 1)], dtype=torch.int32)
        d.group_cu = buf.copy(first if group_cu is None else group_cu)
        d.prefix_len = buf.copy(torch.tensor(c.prefix if prefix is None else prefix, dtype=torch.int32))
        d.prefix_pages, d.prefix_ld, d.prefix_n = wide(c.front)
        d.max_prefix = max(c.prefix) if max_prefix is None else max_prefix
    return d


def stored(c, pool):
    return pool.contiguous() if c.order == "heads" else pool.transpose(1, 2).contiguous()


def attend(c, *, scale, causal=True, at_end=True, back=False, **how):
    """out [T, Hq, d], lse, the status word and the launches."""
    L, buf = lib(), Buffers(at_end)
    L.lanes_order(int(back))
    d = descriptor(c, buf, **how)
    k, v, q = buf.copy(stored(c, c.k_pool)), buf.copy(stored(c, c.v_pool)), buf.copy(c.q)
    width, size = c.Hq * d.d, c.q.element_size()
    out, lse, status = buf.room(c.T * width * size), buf.room(c.T * c.Hq * 4, 4), buf.copy(torch.zeros(1, dtype=torch.int32))
    need = L.dart_attend_workspace_bytes(C.byref(d))
    assert need > 0
    ws = buf.room(need, 256)
    L.lanes_forget()
    rc = L.dart_attend(C.byref(d), q, width, k, v, scale, int(causal), out, width, lse, ws, need, status, None)
    assert rc == D.DART_OK, rc
    got = (buf.back(out, c.dtype, (c.T, c.Hq, d.d)), buf.back(lse, torch.float32, (c.T, c.Hq)), int(buf.back(status, torch.int32, 1)),
           L.lanes_launched().decode())
    buf.free()
    return got


def append(c, rotation, q, k, v, pos, *, at_end=True, back=False, **how):
    """Rotation and append for the tokens of a case: q_out, k_pool, v_pool, the L1 norms, the status word and the launches."""
    L, buf = lib(), Buffers(at_end)
    L.lanes_order(int(back))
    d = descriptor(c, buf, **how)
    r, width, Hkv = rotation(buf), c.Hq * d.d, d.Hkv
    k_pool, v_pool = buf.copy(stored(c, c.k_pool)), buf.copy(stored(c, c.v_pool))
    rows = [buf.copy(x) for x in (q, k, v)]
    out, l1, status = buf.room(c.T * width * q.element_size()), buf.room(c.T * 4, 4), buf.copy(torch.zeros(1, dtype=torch.int32))
    L.lanes_forget()
    rc = L.dart_norm_rotate_append(C.byref(r), C.byref(d), rows[0], width, rows[1], Hkv * d.d, rows[2], Hkv * d.d, buf.copy(pos), c.T, out,
                                   width, None, 0, l1, k_pool, v_pool, status, None)
    assert rc == D.DART_OK, rc
    shape = stored(c, c.k_pool).shape
    pools = [buf.back(p, c.dtype, shape) for p in (k_pool, v_pool)]
    if c.order == "rows":
        pools = [p.transpose(1, 2) for p in pools]
    got = (buf.back(out, c.dtype, (c.T, width)), *pools, buf.back(l1, torch.float32, (c.T,)), int(buf.back(status, torch.int32, 1)),
           L.lanes_launched().decode())
    buf.free()
    return got
