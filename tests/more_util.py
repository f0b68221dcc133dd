"""Caches held in 4 bits, gathered weights and eviction by their definitions in 64 bits, on the CPU, for the cases of
attend_util.  Rows that no sequence owns are NaN in both forms of a pool."""
import torch

import attend_util as A

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def pack(x):
    """(codes, scales) of rows [..., d]: for each value the nearest of the grid, a tie the even code."""
    d = x.shape[-1]
    y = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    unit = torch.zeros(top.shape, dtype=torch.int64)
    for e in range(252):  # the smallest power that leaves the largest value under 7 units
        unit += (top >= 7 * 2.0 ** (e - 127)).long()
    z = y.abs() / torch.exp2(unit.double() - 127)[..., None]
    off = (z[..., None] - GRID).abs()
    least = off.amin(-1, keepdim=True)
    near = off == least
    even = torch.tensor([1, 0] * 4, dtype=torch.bool)
    pick = torch.where((near.sum(-1, keepdim=True) > 1), near & even, near)
    code = torch.argmax(pick.to(torch.int8), -1) + 8 * torch.signbit(y).long()
    bad = ~torch.isfinite(y).all(-1)
    code = torch.where(bad[..., None], 0, code).flatten(-2)
    scale = torch.where(bad, 255, unit)
    return (code[..., ::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


def unpack(pool, d):
    codes, scales = pool
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = GRID[code & 7] * torch.where(code > 7, -1.0, 1.0)
    power = torch.exp2(scales.double() - 127).masked_fill(scales == 255, float("nan"))
    return (v * power.repeat_interleave(32, -1))[..., :d]


def hold(c, sort=None):
    """The case with its pools held in 4 bits (c.four), and as rows of what the codes stand for."""
    c.four = None
    held = []
    for name in ("k_pool", "v_pool"):
        x = getattr(c, name)
        four = tuple(t.contiguous() for t in pack(x))
        if c.order == "rows":
            four = tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in four)
        held.append(four)
        y = unpack(four, c.d).to(c.dtype)
        setattr(c, name, y.transpose(1, 2).contiguous().transpose(1, 2) if c.order == "rows" else y)
    c.four = tuple(held)
    return c


def make(*a, four=True, **k):
    c = A.make(*a, **k)
    c.four = None
    return hold(c) if four else c


def places(c, b, count=None, table=None):
    """Pages and rows of the keys of sequence b."""
    at = torch.arange(c.kv[b] if count is None else count)
    return (c.table[b] if table is None else table).long()[at // c.page], at % c.page


def gathered(c, lse, old, *, scale, causal, carry):
    """Weights [pages, Hkv, page] after the call and how far a kernel of the stated arithmetic may be from them."""
    r, u = c.Hq // c.Hkv, 2.0 ** -24
    w, tol = old.double().clone(), torch.zeros(old.shape, dtype=torch.float64)
    q = c.q.double().reshape(c.T, c.Hq, c.d)
    lse = lse.double()

    def add(tokens, last, table, count, fresh):
        page, row = places(c, None, count, table)
        j = torch.arange(count)
        for h in range(c.Hkv):
            k = A.keys_of(c, c.k_pool, table, count, h)
            total = torch.where(j >= fresh, 0.0, carry * old[page, h, row].double()) if carry else torch.zeros(count, dtype=torch.float64)
            size = total.abs()
            for x in range(h * r, (h + 1) * r):
                s = q[tokens, x] @ k.T * scale
                g = lse[tokens, x][:, None]
                seen = (j[None] <= last[:, None]) & (g > -float("inf"))
                p = torch.where(seen, torch.exp(s - g), 0.0)
                # a score: a 32-bit sum of d products; the exponent: two roundings of its terms' size; the function itself
                e = (c.d + 4) * u * (q[tokens, x].abs() @ k.abs().T) * abs(scale) + 4 * u * (s.abs() + g.abs()) + 4 * u
                total = total + p.sum(0)
                size = size + p.sum(0)
                tol[page, h, row] += torch.where(seen, p * e, 0.0).sum(0)
            w[page, h, row] = total
            tol[page, h, row] += (len(tokens) * r + 8) * u * size

    first = 0
    for g, (members, count) in enumerate(zip(c.group_of or [], c.prefix or [])):
        tokens = torch.arange(int(c.cu[first]), int(c.cu[first + members]))
        first += members
        if len(tokens) and count:
            add(tokens, torch.full((len(tokens),), count - 1), c.front[g], count, count)
    for b, (n, kv) in enumerate(zip(c.n, c.kv)):
        if n == 0 or kv == 0:
            continue
        i = torch.arange(n)
        add(i + int(c.cu[b]), kv - n + i if causal else torch.full((n,), kv - 1), c.table[b], kv, kv - n)
    return w, 1.01 * tol + 1e-37


def check_gathered(c, got, lse, old, **how):
    w, tol = gathered(c, lse, old, **how)
    same = tol <= 1e-37
    assert torch.equal(got[same].double(), w[same]), "weights that no token gives to changed"
    err = (got.double() - w).abs()
    assert bool((err <= tol).all()), f"{float((err / tol).max()):.3g} times what the arithmetic allows"


def budget_of(kv, budget, ratio, first, recent):
    return min(kv, max(budget or kv * ratio[0] // ratio[1], first + recent))


def evicted(c, weights, *, budget=0, ratio=(0, 1), first=0, recent=0):
    """Kept places [B][Hkv] (lists) and lengths."""
    kept, left = [], []
    for b, kv in enumerate(c.kv):
        keep = budget_of(kv, budget, ratio, first, recent)
        page, row = places(c, b)
        per = []
        for h in range(c.Hkv):
            w = weights[page, h, row].tolist()
            w = [(-float("inf"), 0) if x != x else (x, 1) for x in w]
            order = sorted(range(first, kv - recent), key=lambda j: (w[j], -j), reverse=True) if keep < kv else []
            per.append(sorted(list(range(first)) + list(range(kv - recent, kv)) + order[:keep - first - recent]) if keep < kv else
                       list(range(kv)))
        kept.append(per)
        left.append(keep)
    return kept, left


def check_evicted(c, got, weights, out="other", **how):
    """got: pools, weights_out, kept, left, on the CPU."""
    pools, w_out, kept, left = got
    want, lens = evicted(c, weights, **how)
    assert left.tolist() == lens, (left.tolist(), lens)
    before = c.four if c.four is not None else (c.k_pool, c.v_pool)
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    for b, n in enumerate(lens):
        page, row = places(c, b)
        for h in range(c.Hkv):
            src = torch.tensor(want[b][h], dtype=torch.long)
            if kept is not None:
                assert kept[b, h, :n].tolist() == want[b][h], (b, h)
                assert bool((kept[b, h, n:] == -1).all())
            for have, old in zip(pools, before):
                for x, y in zip(have if isinstance(have, tuple) else (have,), old if isinstance(old, tuple) else (old,)):
                    if n:
                        assert torch.equal(bits(x[page[:n], h, row[:n]]), bits(y[page[src], h, row[src]])), (b, h)
            if w_out is not None and n:
                assert torch.equal(bits(w_out[page[:n], h, row[:n]]), bits(weights[page[src], h, row[src]])), (b, h)
    # rows that no sequence owns, and those behind a sequence's last key, are as they were
    for have, old in zip(pools, before):
        for x, y in zip(have if isinstance(have, tuple) else (have,), old if isinstance(old, tuple) else (old,)):
            owned = torch.zeros((x.shape[0], x.shape[2]), dtype=torch.bool)
            for b in range(len(lens)):
                owned[places(c, b)] = True
            free = ~owned
            assert torch.equal(bits(x.transpose(1, 2)[free]), bits(y.transpose(1, 2)[free]))
