"""Inputs for the tests of the attention calls and their definition in 64 bits, on the CPU.

Every row of a pool that no sequence owns holds NaN, and so does every unused place of a row's
padding: whatever a kernel reads that it should not use shows in its results."""
from __future__ import annotations

import dataclasses
from typing import List, Optional

import torch

import paper_2502_11494_amd as D

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
KIND = {torch.bfloat16: D.DART_BF16, torch.float32: D.DART_F32}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half the spacing, relative


@dataclasses.dataclass
class Case:
    n: List[int]
    kv: List[int]               # keys of each sequence, the call's tokens among them
    Hq: int
    Hkv: int
    d: int
    page: int
    dtype: torch.dtype
    order: str = "heads"        # pages hold heads of rows, or rows of heads
    cu: Optional[torch.Tensor] = None
    table: Optional[torch.Tensor] = None
    k_pool: Optional[torch.Tensor] = None
    v_pool: Optional[torch.Tensor] = None
    group_of: Optional[List[int]] = None   # sequences of each group
    prefix: Optional[List[int]] = None
    front: Optional[torch.Tensor] = None
    q: Optional[torch.Tensor] = None
    spread: float = 1.0

    @property
    def T(self):
        return sum(self.n)


def make(n, kv, Hq, Hkv, d, page, dtype, order="heads", groups=None, prefix=None, seed=0, spread=1.0, pad=0):
    """pad: elements between the rows of q beyond their width."""
    g = torch.Generator().manual_seed(seed)
    t = TYPES[dtype]
    c = Case(list(n), list(kv), Hq, Hkv, d, page, t, order, group_of=groups, prefix=prefix, spread=spread)
    c.cu = torch.tensor([sum(c.n[:i]) for i in range(len(c.n) + 1)], dtype=torch.int32)
    counts = [-(-x // page) for x in c.kv]
    fronts = [-(-x // page) for x in (prefix or [])]
    pages = sum(counts) + sum(fronts) + 2
    perm = torch.randperm(pages, generator=g)
    shape = (pages, Hkv, page, d) if order == "heads" else (pages, page, Hkv, d)
    c.k_pool = torch.full(shape, float("nan"), dtype=t)
    c.v_pool = torch.full(shape, float("nan"), dtype=t)
    if order == "rows":
        c.k_pool, c.v_pool = c.k_pool.transpose(1, 2), c.v_pool.transpose(1, 2)
    at = 0

    def fill(lengths, counts):
        nonlocal at
        table = torch.full((len(lengths), max(1, max(counts, default=0))), pages - 1, dtype=torch.int32)
        for b, (x, m) in enumerate(zip(lengths, counts)):
            table[b, :m] = perm[at:at + m]
            at += m
            where = torch.arange(x)
            p, r = table[b].long()[where // page], where % page
            c.k_pool[p, :, r] = torch.randn((x, Hkv, d), generator=g).to(t)
            c.v_pool[p, :, r] = torch.randn((x, Hkv, d), generator=g).to(t)
        return table

    c.table = fill(c.kv, counts)
    if prefix:
        c.front = fill(prefix, fronts)
    rows = torch.full((max(c.T, 1), Hq * d + pad), float("nan"), dtype=t)
    rows[:c.T, :Hq * d] = (torch.randn((c.T, Hq * d), generator=g) * spread).to(t)
    c.q = rows[:c.T, :Hq * d]
    return c


def keys_of(c, pool, table, count, h):
    where = torch.arange(count)
    return pool[table.long()[where // c.page], h, where % c.page].double()


def reference(c, scale, causal):
    """out, lse, and how far a kernel of the stated arithmetic may be from each: [T, Hq, d], [T, Hq]."""
    r = c.Hq // c.Hkv
    out = torch.zeros((c.T, c.Hq, c.d), dtype=torch.float64)
    lse = torch.full((c.T, c.Hq), -float("inf"), dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    u = 2.0 ** -24
    group = [g for g, m in enumerate(c.group_of or []) for _ in range(m)]
    q = c.q.double().reshape(c.T, c.Hq, c.d)
    for b, (n, kv) in enumerate(zip(c.n, c.kv)):
        if n == 0:
            continue
        front = c.prefix[group[b]] if group else 0
        i = torch.arange(n)
        last = kv - n + i if causal else torch.full((n,), kv - 1)
        seen = torch.cat((torch.ones((n, front), dtype=torch.bool), torch.arange(kv)[None] <= last[:, None]), 1)
        if front + kv == 0:
            continue
        for h in range(c.Hkv):
            k, v = keys_of(c, c.k_pool, c.table[b], kv, h), keys_of(c, c.v_pool, c.table[b], kv, h)
            if front:
                k = torch.cat((keys_of(c, c.k_pool, c.front[group[b]], front, h), k))
                v = torch.cat((keys_of(c, c.v_pool, c.front[group[b]], front, h), v))
            for j in range(h * r, (h + 1) * r):
                t0 = int(c.cu[b])
                x = q[t0:t0 + n, j]
                s = (x @ k.T * scale).masked_fill(~seen, -float("inf"))
                some = seen.any(1)
                m = torch.where(some, s.amax(1), 0.0)
                p = torch.exp(s - m[:, None])
                l = p.sum(1)
                safe = torch.where(some, l, 1.0)
                # a score: a 32-bit sum of d products and the scaling; its error is the relative error of its
                # exponential, beside that of the exponent's own product (relative to |s| + |m|) and of the function
                e = ((c.d + 4) * u * (x.abs() @ k.abs().T) * abs(scale) + 4 * u * (s.abs() + m.abs()[:, None]) + 4 * u)
                e = torch.where(seen, e, 0.0)
                weight = UNIT[torch.bfloat16] if c.dtype == torch.bfloat16 else 0.0
                total = front + kv + 64  # additions of the longest chain, the joins of partial sums among them
                y = p @ v / safe[:, None]
                size = p @ v.abs() / safe[:, None]
                pe = (p * e)
                tol = (pe @ v.abs() / safe[:, None] + (pe.sum(1) / safe)[:, None] * y.abs()
                       + (weight + 2 * total * u) * size + UNIT[c.dtype] * y.abs())
                out[t0:t0 + n, j] = torch.where(some[:, None], y, 0.0)
                lse[t0:t0 + n, j] = torch.where(some, m + torch.log(safe), -float("inf"))
                out_tol[t0:t0 + n, j] = 1.01 * tol + 1e-37
                lse_tol[t0:t0 + n, j] = 1.01 * (pe.sum(1) / safe + 2 * total * u + 8 * u * (1 + m.abs() + torch.log(safe)))
    return out, lse, out_tol, lse_tol


def pool_to_gpu(pool, order):
    if order == "rows":
        return pool.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    return pool.contiguous().cuda()


def to_gpu(t):
    """A copy on the GPU with the same strides (and the same padding between rows)."""
    base = torch.full((t.shape[0], max(t.stride(0), 1) if t.shape[0] > 1 else t.shape[1]), float("nan"), dtype=t.dtype)
    base[:, :t.shape[1]] = t
    return base.cuda()[:, :t.shape[1]]


def cache_of(c, k_pool, *, table=None, kv=None, cu=None, max_q=None, max_kv=None, packed=None):
    """The descriptor of a case on the GPU."""
    packed = any(x != 1 for x in c.n) if packed is None else packed
    more = {}
    if c.group_of is not None:
        more = dict(group_cu=torch.tensor([sum(c.group_of[:i]) for i in range(len(c.group_of) + 1)],
                                          dtype=torch.int32).cuda(),
                    prefix_pages=c.front.cuda(), prefix_len=torch.tensor(c.prefix, dtype=torch.int32).cuda(),
                    max_prefix=max(c.prefix))
    kv = torch.tensor(c.kv, dtype=torch.int32) if kv is None else kv
    return D.make_cache(c.Hq, k_pool, (c.table if table is None else table).cuda(), kv.cuda(),
                        max(c.kv) if max_kv is None else max_kv, T=c.T, max_q=max_q or max(c.n),
                        cu_q=(c.cu if cu is None else cu).cuda() if packed else None, **more)


def attend(c, *, scale, causal=True, want_lse=True, status=None, ws_fill=None, out_pad=0, k_pool=None, v_pool=None,
           stream=None, **how):
    """The kernels' out [T, Hq, d] and lse on the CPU."""
    k_pool = pool_to_gpu(c.k_pool, c.order) if k_pool is None else k_pool
    v_pool = pool_to_gpu(c.v_pool, c.order) if v_pool is None else v_pool
    cache = cache_of(c, k_pool, **how)
    ws = D.alloc_attend_workspace(cache)
    ws.fill_(255 if ws_fill is None else ws_fill)  # what a workspace holds before a call is nobody's business
    width = c.Hq * c.d
    room = torch.full((c.T, width + out_pad), 7.0, dtype=c.dtype, device="cuda")
    lse = torch.full((c.T, c.Hq), 7.0, device="cuda") if want_lse else None
    q = to_gpu(c.q)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())  # for what the lines above write
    D.dart_attend(cache, q, k_pool, v_pool, room[:, :width], ws, scale=scale, causal=causal, lse=lse,
                  status=status, stream=stream)
    torch.cuda.synchronize()
    assert bool((room[:, width:] == 7.0).all())
    return room[:, :width].cpu().view(c.T, c.Hq, c.d), None if lse is None else lse.cpu()


def check(c, got, *, scale, causal=True):
    out, lse = got
    want, want_lse, tol, lse_tol = reference(c, scale, causal)
    assert torch.isfinite(out.float()).all(), "a result is not finite"
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), f"out: {float((err / tol).max()):.3g} times what the arithmetic allows"
    if lse is not None:
        empty = want_lse == -float("inf")
        assert torch.equal(lse == -float("inf"), empty)
        off = (lse.double() - want_lse).abs()[~empty]
        assert bool((off <= lse_tol[~empty]).all()), f"lse: off by {float(off.max()):.3g}"
