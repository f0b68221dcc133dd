"""The operators on a cache held in 4 bits and on the eviction of its keys, as cases to measure: keys and
values written to 4-bit pages and read back as rows (`append`), attention over such pages (`attend`), the
attention weight that each key of a cache has gathered (`weights`), and eviction of the keys that gathered
least (`evict`).

With `own` false every case runs in its plain form, elementary torch operations in 32 bits; with `own` true
through the framework's entry points.  Token counts and widths are those of the package's own workloads:
576-token images, 2880-token multi-crop images, ragged batches of 1024..16384 tokens of which 11.1 % are kept, 64
frames of 144 tokens; hidden sizes 4096 (32 heads of 128), 3584 (28 heads, 4 key/value heads) and their relatives.

A block of 32 values of a head (the last one filled up with zeros) is held as 32 codes of 4 bits, sign and one of 0,
0.5, 1, 1.5, 2, 3, 4, 6, and a byte e that stands for 2^(e - 127): the smallest that leaves the largest value under 7.
Value 2i of a row lies in the low half of its byte i.  A block with an infinity or NaN has e = 255 and is NaN."""
import itertools
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    app = dict(op="append", d=128, before_lo=0, before_hi=0)
    att = dict(op="attend", d=128, dtype="bf16", causal=True, groups=0, prefix=0)
    wei = dict(op="weights", d=128, causal=True, bits=16, kv_lo=0, kv_hi=0, carry=0.0)
    evi = dict(op="evict", d=128, dtype="bf16", first=4)
    return [
        # a step of 32 running answers, each with its own context: the calls' latency
        dict(app, name="append_step", dtype="bf16", B=32, n_lo=1, n_hi=1, Hkv=4, page=16, before_lo=113, before_hi=1818),
        # eight multi-crop images, as many key heads as query heads
        dict(app, name="append_crops", dtype="bf16", B=8, n_lo=2880, n_hi=2880, Hkv=32, page=64),
        # the retained tokens of a ragged batch in 32 bits, heads that end inside a block
        dict(app, name="append_retained_f32", dtype="f32", B=32, n_lo=113, n_hi=1818, Hkv=12, d=80, page=16),
        # a single answer over one reduced image and its prompt: latency
        dict(att, name="attend_one_token", B=1, n_lo=1, n_hi=1, kv_lo=131, kv_hi=131, Hq=32, Hkv=32, page=16),
        # a step of 32 answers over unreduced ragged contexts: the cache is read once
        dict(att, name="attend_step_ragged", B=32, n_lo=1, n_hi=1, kv_lo=1024, kv_hi=16384, Hq=28, Hkv=4, page=16),
        # a step of 64 answers about one video
        dict(att, name="attend_video_answers", B=64, n_lo=1, n_hi=1, kv_lo=19, kv_hi=412, Hq=28, Hkv=4, page=16, groups=1,
             prefix=9216),
        # the last quarter of two videos' tokens, over the three quarters before
        dict(att, name="attend_video_chunk", B=2, n_lo=2304, n_hi=2304, kv_lo=6912, kv_hi=6912, Hq=28, Hkv=4, page=64),
        # what a step of 32 answers adds to the weights of keys held in 4 bits
        dict(wei, name="weights_step", dtype="bf16", bits=4, B=32, n_lo=1, n_hi=1, kv_lo=1024, kv_hi=16384, Hq=28, Hkv=4, page=16,
             carry=0.98),
        # one image and its prompt in 32 bits
        dict(wei, name="weights_image_f32", dtype="f32", B=1, n_lo=637, n_hi=637, Hq=32, Hkv=32, page=64),
        # two whole videos, before the first eviction
        dict(wei, name="weights_video", dtype="bf16", B=2, n_lo=9216, n_hi=9216, Hq=28, Hkv=4, page=64),
        # one image and its prompt, cut to 192 keys
        dict(evi, name="evict_image", B=1, kv_lo=637, kv_hi=637, budget=192, permille=0, recent=32, Hkv=32, page=64),
        # a ragged batch, cut to 11.1 % of each sequence
        dict(evi, name="evict_ragged", B=32, kv_lo=1024, kv_hi=16384, budget=0, permille=111, recent=64, Hkv=4, page=16),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads, kv = rng.choice([(32, 32), (28, 4), (64, 8), (40, 40), (16, 2), (12, 12), (28, 28), (8, 1)])
    d = rng.choice([128, 128, 128, 64, 80, 96, 256])
    c = dict(op=rng.choice(["append", "attend", "weights", "evict"]), Hkv=kv, d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
             page=rng.choice([16, 32, 64, 256]))
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "append":
        B = _log(rng, 1, 48)
        hi = _log(rng, 1, max(1, min(9216, 180_000_000 // (kv * d * size * B))))
        c.update(B=B, n_lo=_log(rng, 1, hi), n_hi=hi, before_lo=0, before_hi=rng.choice([0, 37, 700]))
        return c
    if c["op"] == "evict":
        B = _log(rng, 1, 48)
        hi = _log(rng, 40, max(64, min(16384, 250_000_000 // (kv * d * size * B))))
        c.update(B=B, kv_lo=max(1, hi // rng.choice([1, 2, 9])), kv_hi=hi, first=rng.choice([0, 4, 5]), recent=rng.choice([0, 1, 32, 64]),
                 budget=0, permille=0)
        if rng.random() < 0.5:
            c["permille"] = rng.randint(60, 700)
        else:
            c["budget"] = max(c["first"] + c["recent"] + 1, _log(rng, 8, hi))
        return c
    c.update(Hq=heads, causal=rng.random() < 0.8, groups=0, prefix=0)
    B = _log(rng, 1, 64)
    kind = rng.choice(["step", "few", "prompt"])
    n_hi = 1 if kind == "step" else _log(rng, 2, 24) if kind == "few" else _log(rng, 25, 4096)
    if c["op"] == "attend" and rng.random() < 0.4:
        c["groups"] = rng.choice([g for g in (1, 2, 4) if g <= B])
        B = c["groups"] * max(1, B // c["groups"])
        c["prefix"] = _log(rng, 33, 12000)
    kv_hi = rng.choice([0, _log(rng, 1, 16384)])
    # the scores of the plain form, and the pages, stay well under the largest listed case's
    while B * heads * n_hi * (c["prefix"] + kv_hi + n_hi) > 900_000_000 or B * kv * d * size * (kv_hi + n_hi) > 900_000_000:
        if n_hi > 1 and n_hi >= kv_hi:
            n_hi = max(1, n_hi // 2)
        elif kv_hi > 64:
            kv_hi //= 2
        else:
            B = max(max(1, c["groups"]), B // 2 // max(1, c["groups"]) * max(1, c["groups"]))
    c.update(B=B, n_lo=max(1, rng.randint(1, n_hi)), n_hi=n_hi, kv_lo=kv_hi // rng.choice([1, 2, 9]), kv_hi=kv_hi)
    if c["op"] == "weights":
        del c["groups"], c["prefix"]
        c.update(bits=rng.choice([4, 16]), carry=rng.choice([0.0, 0.98, 1.0]))
    return c


def _between(lo, hi, n, salt):
    """n lengths of lo..hi, the same in every run: they are part of the case, not of its inputs."""
    r = random.Random(1000003 * salt + 1009 * hi + 31 * lo + n)
    return [r.randint(lo, hi) for _ in range(n)]


def _lengths(case):
    """New tokens and keys cached before them, for each sequence."""
    if case["op"] == "evict":
        return [0] * case["B"], _between(case["kv_lo"], case["kv_hi"], case["B"], 2)
    n = _between(case["n_lo"], case["n_hi"], case["B"], 1)
    lo, hi = (case["kv_lo"], case["kv_hi"]) if "kv_lo" in case else (case["before_lo"], case["before_hi"])
    return n, _between(lo, hi, case["B"], 2)


def _offsets(n):
    return list(itertools.accumulate(n, initial=0))


def _budget(case, keys):
    """Keys that a sequence of so many keeps."""
    k = case["budget"] or keys * case["permille"] // 1000
    return min(keys, max(k, case["first"] + case["recent"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]
    B, Hkv, d, page = (case[k] for k in ("B", "Hkv", "d", "page"))
    groups, prefix = case.get("groups", 0), case.get("prefix", 0)
    n, before = _lengths(case)
    cu = _offsets(n)
    T, total = cu[-1], [x + y for x, y in zip(n, before)]

    def normal(*shape, by=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * by).to(t)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def tables(counts, at, perm):
        """A page table [len(counts), max(counts)]: pages perm[at:], in any order; unused places hold page 0."""
        table = torch.zeros((len(counts), max(1, max(counts))), dtype=torch.int32)
        for b, m in enumerate(counts):
            table[b, :m] = perm[at:at + m]
            at += m
        return table, at

    counts = [-(-x // page) for x in total]
    front = [-(-prefix // page)] * groups
    pages = sum(counts) + sum(front) + 3
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    table, at = tables(counts, 0, perm)
    s = dict(case, T=T, kind=t, n=n, total=total, max_n=max(n), cu=ints(cu), table=table.cuda(), kv_len=ints(total), max_kv=max(total),
             pages=pages)
    if groups:
        s["front"] = tables(front, at, perm)[0].cuda()
        s["group_cu"] = ints([i * (B // groups) for i in range(groups + 1)])
        s["front_len"] = ints([prefix] * groups)
    four = case["op"] in ("append", "attend") or case.get("bits") == 4
    pools = 1 if case["op"] == "weights" else 2
    if case["op"] == "append":  # empty pages, and the rows of a layer's fused projection
        wide = -(-d // 32) * 32
        s["pools"] = [(torch.zeros((pages, Hkv, page, wide // 2), dtype=torch.uint8, device="cuda"),
                       torch.zeros((pages, Hkv, page, wide // 32), dtype=torch.uint8, device="cuda")) for _ in range(2)]
        # (some elements of a head are larger than the others, as keys have them)
        rows = normal(T, 2 * Hkv, d) * (1 + 7 * (torch.arange(d, device="cuda") % 29 == 3)).to(t)
        s["k"], s["v"] = rows.view(T, -1)[:, :Hkv * d], rows.view(T, -1)[:, Hkv * d:]
        s["k_out"], s["v_out"] = (torch.empty((T, Hkv * d), dtype=t, device="cuda") for _ in range(2))
    else:
        s["pools"] = [_packed(normal(pages, Hkv, page, d).float()) if four else normal(pages, Hkv, page, d) for _ in range(pools)]
    if case["op"] in ("attend", "weights"):
        s["q"] = normal(T, case["Hq"] * d, by=1.5)
        s["scale"] = d ** -0.5
    if case["op"] == "attend":
        s["out"] = torch.empty((T, case["Hq"] * d), dtype=t, device="cuda")
        s["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device="cuda")
    if case["op"] == "weights":
        s["weights"] = torch.rand((pages, Hkv, page), generator=g, device="cuda")
        s["lse"] = torch.cat([_lse(s, b) for b in range(B)])  # as attention leaves it
    if case["op"] == "evict":
        # gathered weights: a few keys have most of it, some have none at all
        w = torch.exp(2 * torch.randn((pages, Hkv, page), generator=g, device="cuda"))
        s["weights"] = w * (torch.rand(w.shape, generator=g, device="cuda") > 0.03)
        s["most"] = max(_budget(case, x) for x in total)
        s["weights_out"] = torch.zeros_like(s["weights"])
        s["kept"] = torch.zeros((B, Hkv, s["most"]), dtype=torch.int32, device="cuda")
        s["left"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["row_of"] = _row_map(s, [_budget(case, x) for x in total])
    if own:
        import paper_2502_11494_amd as D
        more = dict(T=T, max_q=s["max_n"], cu_q=None if n == [1] * B else s["cu"])
        if groups:
            more.update(group_cu=s["group_cu"], prefix_pages=s["front"], prefix_len=s["front_len"], max_prefix=prefix)
        Hq = case.get("Hq", Hkv)
        if four:
            kind = D.DART_BF16 if case["dtype"] == "bf16" else D.DART_F32
            s["cache"] = D.make_cache_4bit(Hq, d, kind, s["pools"][0], s["table"], s["kv_len"], s["max_kv"], **more)
        else:
            s["cache"] = D.make_cache(Hq, s["pools"][0], s["table"], s["kv_len"], s["max_kv"], **more)
        if case["op"] == "attend":
            s["ws"] = D.alloc_attend_4bit_workspace(s["cache"])
        if case["op"] == "weights":
            s["ws"] = D.alloc_attend_weights_workspace(s["cache"])
        if case["op"] == "evict":
            s["eviction"] = D.make_eviction(budget=case["budget"], ratio=(case["permille"], 1000), first=case["first"],
                                            recent=case["recent"])
            s["ws"] = D.alloc_evict_workspace(s["cache"], s["eviction"])
    return s


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)


def _own(s):
    import paper_2502_11494_amd as D
    if s["op"] == "append":
        D.dart_append_4bit(s["cache"], s["k"], s["v"], *s["pools"])
        D.dart_read_4bit(s["cache"], *s["pools"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    if s["op"] == "attend":
        D.dart_attend_4bit(s["cache"], s["q"], *s["pools"], s["out"], s["ws"], scale=s["scale"], causal=s["causal"], lse=s["lse"])
        return s["out"], s["lse"]
    if s["op"] == "weights":
        D.dart_attend_weights(s["cache"], s["q"], s["pools"][0], s["lse"], s["weights"], s["ws"], scale=s["scale"],
                              causal=s["causal"], carry=s["carry"])
        return s["weights"]
    D.dart_evict(s["cache"], s["eviction"], *s["pools"], s["weights"], s["left"], s["ws"], weights_out=s["weights_out"], kept=s["kept"])
    return *s["pools"], s["weights_out"], s["kept"], s["left"]


# ---- plain forms ---------------------------------------------------------------------------

def _packed(x):
    """Codes and scales of rows [..., d].  Values are compared with the borders in 64 bits."""
    d = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -d % 32)).unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    e = (e - 3 + (m >= 0.875)).clamp(-127, 125)
    e = torch.where(top > 0, e, -127)
    y = x.abs().double() * torch.exp2(-e.double())[..., None]
    code = ((y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5))
    code += 8 * torch.signbit(x)
    good = torch.isfinite(top)
    code = torch.where(good[..., None], code, 0).flatten(-2)
    return (code[..., ::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(good, e + 127, 255).to(torch.uint8)


def _unpacked(pool, d):
    """Rows in 32 bits of (codes, scales)."""
    codes, scales = pool
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device="cuda")
    # (a byte's two values by one look-up)
    two = torch.stack((grid.repeat(16), grid.repeat_interleave(16)), -1)
    y = two[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    power = torch.exp2(torch.arange(256, device="cuda").double() - 127).float()
    power[255] = math.nan
    return (y * power[scales.int()][..., None]).flatten(-2)[..., :d]


def _rows_of(pool, table, d):
    """[rows of the table, heads, keys, d] in 32 bits."""
    if isinstance(pool, tuple):
        x = _unpacked(tuple(p[table.long()] for p in pool), d)
    else:
        x = pool[table.long()].float()
    return x.transpose(1, 2).flatten(2, 3)


def _places(s):
    """Page and row of every token of the call."""
    token = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu"], token, right=True) - 1
    place = s["kv_len"][b] - s["cu"][b + 1] + token
    return s["table"][b, torch.div(place, s["page"], rounding_mode="floor")].long(), place % s["page"]


def _plain_append(s):
    page, row = _places(s)
    out = []
    for x, pool in ((s["k"], s["pools"][0]), (s["v"], s["pools"][1])):
        for held, new in zip(pool, _packed(x.float().view(s["T"], s["Hkv"], s["d"]))):
            held[page, :, row] = new
        out.append(_unpacked(tuple(p[page, :, row] for p in pool), s["d"]).flatten(1).to(s["kind"]))
    return tuple(out)


def _plain_attend(s):
    B, Hq, Hkv, d, m, T = s["B"], s["Hq"], s["Hkv"], s["d"], s["max_n"], s["T"]
    r, groups, cu = Hq // Hkv, s["groups"], s["cu"].long()
    at = cu[:-1, None] + torch.arange(m, device="cuda")
    real = at < cu[1:, None]
    q = s["q"].float().view(T, Hkv, r, d)[at.clamp(max=T - 1)]                     # [B, m, Hkv, r, d]
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, m * r, d) * s["scale"]
    k, v = (_rows_of(p, s["table"], d) for p in s["pools"])
    key = torch.arange(k.shape[2], device="cuda")
    last = s["kv_len"].long()[:, None] - 1
    if s["causal"]:
        last = last + 1 - (cu[1:] - cu[:-1])[:, None] + torch.arange(m, device="cuda")
    seen = (key <= last.expand(B, m)[..., None]) & (key < s["kv_len"][:, None, None])  # [B, m, keys]
    w = torch.matmul(q, k.transpose(-1, -2)).view(B, Hkv, m, r, -1)
    w = w.masked_fill(~seen[:, None, :, None, :], -math.inf).view(B, Hkv, m * r, -1)
    most = w.amax(-1, keepdim=True)
    if groups:
        S = B // groups
        fk, fv = (_rows_of(p, s["front"], d)[:, :, :s["prefix"]] for p in s["pools"])
        fq = q.view(groups, S, Hkv, m * r, d).transpose(1, 2).reshape(groups, Hkv, S * m * r, d)
        fw = torch.matmul(fq, fk.transpose(-1, -2))
        fm = fw.amax(-1, keepdim=True)
        most = torch.maximum(most, fm.view(groups, Hkv, S, m * r, 1).transpose(1, 2).reshape(B, Hkv, m * r, 1))
    most = most.masked_fill(most == -math.inf, 0.0)
    w = torch.exp(w - most)
    total, out = w.sum(-1, keepdim=True), torch.matmul(w, v)
    if groups:
        fw = torch.exp(fw - most.view(groups, S, Hkv, m * r, 1).transpose(1, 2).reshape(groups, Hkv, S * m * r, 1))
        ft, fo = fw.sum(-1, keepdim=True), torch.matmul(fw, fv)
        total = total + ft.view(groups, Hkv, S, m * r, 1).transpose(1, 2).reshape(B, Hkv, m * r, 1)
        out = out + fo.view(groups, Hkv, S, m * r, d).transpose(1, 2).reshape(B, Hkv, m * r, d)
    out = torch.where(total > 0, out / total, 0.0).view(B, Hkv, m, r, d).permute(0, 2, 1, 3, 4)
    lse = (most + torch.log(total)).view(B, Hkv, m, r).permute(0, 2, 1, 3)
    return out[real].reshape(T, Hq * d).to(s["kind"]), lse[real].reshape(T, Hq)


def _scores(s, b, dtype, h=None):
    """Scores of sequence b, [key heads, tokens, query heads of a key head, keys], -infinity where not seen."""
    Hq, Hkv, d, n, kv = s["Hq"], s["Hkv"], s["d"], s["n"][b], s["total"][b]
    t0 = sum(s["n"][:b])
    heads = slice(None) if h is None else slice(h, h + 1)
    q = s["q"][t0:t0 + n].to(dtype).view(n, Hkv, -1, d)[:, heads].permute(1, 0, 2, 3)
    k = _rows_of(s["pools"][0], s["table"][b:b + 1], d)[0, heads, :kv].to(dtype)
    w = torch.matmul(q.reshape(k.shape[0], -1, d), k.transpose(-1, -2)) * s["scale"]
    w = w.view(k.shape[0], n, Hq // Hkv, kv)
    if s["causal"] and n > 1:  # token i does not see what comes after it
        w.masked_fill_(torch.ones((n, kv), dtype=torch.bool, device="cuda").triu(kv - n + 1)[:, None], -math.inf)
    return w


def _lse(s, b):
    """[tokens, heads] of sequence b, in 64 bits from 32-bit scores."""
    heads = [None] if s["n"][b] * s["Hq"] * s["total"][b] < 50_000_000 else range(s["Hkv"])
    x = torch.cat([torch.logsumexp(_scores(s, b, torch.float32, h).double(), -1) for h in heads])
    return x.transpose(0, 1).reshape(s["n"][b], -1).float()


def _plain_weights(s):
    if s["max_n"] == 1:  # a step: all sequences at once
        q = s["q"].float().view(s["B"], s["Hkv"], -1, s["d"]) * s["scale"]
        k = _rows_of(s["pools"][0], s["table"], s["d"])
        w = torch.exp(torch.matmul(q, k.transpose(-1, -2)) - s["lse"].view(s["B"], s["Hkv"], -1, 1)).sum(-2)
        key = torch.arange(k.shape[2], device="cuda")
        b, j = torch.nonzero(key < s["kv_len"][:, None], as_tuple=True)
        page, row, new = s["table"][b, j // s["page"]].long(), j % s["page"], j == s["kv_len"][b] - 1
        old = s["weights"][page, :, row]
        s["weights"][page, :, row] = torch.where(new[:, None], 0.0, old * s["carry"]) + w[b, :, j]
        return s["weights"]
    at = 0
    for b, (n, kv) in enumerate(zip(s["n"], s["total"])):
        lse = s["lse"][at:at + n].view(n, s["Hkv"], -1).transpose(0, 1)
        at += n
        w = torch.exp(_scores(s, b, torch.float32) - lse[..., None]).sum((1, 2))
        j = torch.arange(kv, device="cuda")
        page, row = s["table"][b, j // s["page"]].long(), j % s["page"]
        old = s["weights"][page, :, row]
        s["weights"][page, :, row] = torch.where((j >= kv - n)[:, None], 0.0, old * s["carry"]) + w.t()
    return s["weights"]


def _row_map(s, keep):
    """For all kept keys of the batch: sequence, place among the kept (plain data of the case)."""
    b = torch.repeat_interleave(torch.arange(s["B"]), torch.tensor(keep))
    i = torch.arange(len(b)) - torch.tensor(_offsets(keep))[b]
    return b.cuda(), i.cuda(), torch.tensor(keep, dtype=torch.int32, device="cuda")


def _plain_evict(s):
    page, Hkv = s["page"], s["Hkv"]
    b, i, keep = s["row_of"]
    kv = s["kv_len"].long()[:, None]
    w = s["weights"][s["table"].long()].transpose(1, 2).flatten(2)               # [B, Hkv, keys]
    key = torch.arange(w.shape[2], device="cuda")
    held = (key < s["first"]) | (key >= kv - s["recent"])
    w = torch.where(held[:, None], math.inf, w).masked_fill((key >= kv)[:, None], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    key = key.expand_as(order)
    chosen = torch.where(key < keep[:, None, None], order, key.shape[-1])        # (past the budget: behind all keys)
    chosen = torch.sort(chosen, -1).values[..., :s["most"]].int()
    s["kept"][b, :, i] = chosen[b, :, i]
    s["left"].copy_(keep)
    src, head = chosen[b, :, i].long(), torch.arange(Hkv, device="cuda")
    page_from, row_from = s["table"].long()[b[:, None], src // page], src % page
    page_to, row_to = s["table"].long()[b, i // page][:, None], (i % page)[:, None]
    for pool, out in ((s["pools"][0], s["pools"][0]), (s["pools"][1], s["pools"][1]), (s["weights"], s["weights_out"])):
        out[page_to, head, row_to] = pool[page_from, head, row_from]
    return *s["pools"], s["weights_out"], s["kept"], s["left"]


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    n, before = _lengths(case)
    T, e = sum(n), 2 if case["dtype"] == "bf16" else 4
    Hkv, d = case["Hkv"], case["d"]
    row4 = -(-d // 32) * 17  # bytes of a head in 4 bits
    total = sum(n) + sum(before)
    if case["op"] == "append":  # rows in, pages, rows out
        return {"bytes": 2 * T * Hkv * (2 * d * e + row4), "flops": 4 * T * Hkv * d}
    if case["op"] == "evict":
        keep = [_budget(case, x) for x in before]
        moved = sum(k - min(k, case["first"]) for k, x in zip(keep, before) if k < x)
        return {"bytes": Hkv * (4 * total + moved * (4 * d * e + 8) + 4 * sum(keep)), "flops": Hkv * total}
    if case["causal"]:
        seen = sum(x * y + x * (x + 1) // 2 for x, y in zip(n, before))
    else:
        seen = sum(x * (x + y) for x, y in zip(n, before))
    Hq = case["Hq"]
    if case["op"] == "weights":
        row = row4 if case["bits"] == 4 else d * e
        return {"bytes": T * Hq * (d * e + 4) + total * Hkv * (row + (8 if case["carry"] else 4)), "flops": 2 * d * Hq * seen}
    keys = total + case["groups"] * case["prefix"]
    seen += T * case["prefix"]
    return {"bytes": 2 * T * Hq * d * e + T * Hq * 4 + 2 * keys * Hkv * row4, "flops": 4 * d * Hq * seen}


# ---- the same from the definitions, in 64 bits ----------------------------------------------

def _value(codes, scales, d):
    """What codes and scales stand for: (-1)^s (1 + m/2) 2^(e - 1), m/2 for e = 0, times the block's power of two."""
    c = torch.stack((codes % 16, torch.div(codes, 16, rounding_mode="floor")), -1).flatten(-2).long()
    sign, e, m = c // 8, c // 2 % 4, c % 2
    size = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * torch.exp2(e.double() - 1))
    power = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), scales.double() - 127).repeat_interleave(32, -1)
    return ((1 - 2 * sign) * size * power)[..., :d]


def exact(case, seed):
    s = prepare(case, seed)
    n, before = _lengths(case)
    T, Hkv, d, cu, page = s["T"], s["Hkv"], s["d"], _offsets(n), s["page"]
    if case["op"] == "append":
        out = []
        for x in (s["k"], s["v"]):
            y = torch.zeros((T, Hkv, -(-d // 32) * 32), dtype=torch.float64, device="cuda")
            y[..., :d] = x.double().view(T, Hkv, d)
            blocks = y.view(T, Hkv, -1, 32)
            unit = torch.full(blocks.shape[:-1], 2.0 ** -127, dtype=torch.float64, device="cuda")
            top = blocks.abs().amax(-1)
            for _ in range(260):  # the smallest power of two that leaves the largest under 7
                unit = torch.where((top >= 7 * unit) & (unit < 2.0 ** 125), 2 * unit, unit)
            z = blocks / unit[..., None]
            step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0))
            z = (torch.round(z / step) * step).clamp(-6, 6) * unit[..., None]  # (round takes ties to even)
            out.append(z.flatten(-2)[..., :d].reshape(T, -1))
        return tuple(out)
    if case["op"] == "evict":
        keep = [_budget(case, x) for x in before]
        pools, w = [p.clone() for p in s["pools"]], s["weights_out"].double()
        table, weights = s["table"].cpu(), s["weights"].cpu()
        if sum(before) * Hkv > 3_000_000:
            return None
        for b in range(case["B"]):
            at = torch.arange(before[b])
            pg, row = table[b].long()[at // page], at % page
            for h in range(Hkv):
                worth = weights[pg, h, row].tolist()
                middle = range(case["first"], before[b] - case["recent"])
                short = before[b] - keep[b]
                gone = set(sorted(middle, key=lambda j: (worth[j], -j))[:short])
                left = torch.tensor([j for j in range(before[b]) if j not in gone], dtype=torch.long)
                s["kept"][b, h, :keep[b]] = left.int().cuda()
                to = pg[:keep[b]], h, row[:keep[b]]
                for p, old in zip(pools, s["pools"]):
                    p[to] = old[pg[left], h, row[left]]
                w[to] = s["weights"][pg[left], h, row[left]].double()
        return *(p.double() for p in pools), w, s["kept"], torch.tensor(keep, dtype=torch.int32, device="cuda")
    r, Hq = case["Hq"] // Hkv, case["Hq"]

    def rows_of(pool, table, count, h):
        at = torch.arange(count, device="cuda")
        where = table.long()[at // page], h, at % page
        return _value(pool[0][where], pool[1][where], d) if isinstance(pool, tuple) else pool[where].double()

    if 8 * d * Hq * T * max(case.get("prefix", 0) + x + y for x, y in zip(n, before)) > 2e14:
        return None
    if case["op"] == "weights":
        w = s["weights"].double()
        for b in range(case["B"]):
            at = torch.arange(before[b] + n[b], device="cuda")
            for h in range(Hkv):
                k = rows_of(s["pools"][0], s["table"][b], before[b] + n[b], h)
                where = s["table"][b].long()[at // page], h, at % page
                total = w[where] * case["carry"]
                total[before[b]:] = 0
                for j in range(h * r, (h + 1) * r):
                    z = s["q"][cu[b]:cu[b + 1], j * d:(j + 1) * d].double() @ k.t() * s["scale"]
                    p = torch.exp(z - s["lse"][cu[b]:cu[b + 1], j].double()[:, None])
                    if case["causal"]:
                        p = p.tril(before[b])
                    total += p.sum(0)
                w[where] = total
        return w
    out = torch.zeros((T, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    per = case["B"] // case["groups"] if case["groups"] else 1
    for b in range(case["B"]):
        for h in range(Hkv):
            k, v = (rows_of(p, s["table"][b], before[b] + n[b], h) for p in s["pools"])
            if case["groups"]:
                k, v = (torch.cat((rows_of(p, s["front"][b // per], case["prefix"], h), x)) for p, x in zip(s["pools"], (k, v)))
            hidden = None
            if case["causal"]:
                hidden = torch.ones((n[b], k.shape[0]), dtype=torch.bool, device="cuda").triu(k.shape[0] - n[b] + 1)
            for j in range(h * r, (h + 1) * r):
                z = s["q"][cu[b]:cu[b + 1], j * d:(j + 1) * d].double() @ k.t() * s["scale"]
                if hidden is not None:
                    z[hidden] = -math.inf
                lse[cu[b]:cu[b + 1], j] = torch.logsumexp(z, -1)
                out[cu[b]:cu[b + 1], j] = torch.softmax(z, -1) @ v
    return out.reshape(T, -1), lse
