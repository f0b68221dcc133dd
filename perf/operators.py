"""The attention operators around the reduction step, as cases to measure: the head norm and
position rotation of queries and keys (`rotate`), the same pass appending keys and values to a
paged cache (`append`), attention over that cache (`attend`), and attention of a batch whose
sequences share long prefixes (`prefix`).

With `own` false every case runs in its plain form, elementary torch operations in 32 bits; with
`own` true through the framework's entry points.  Token counts and widths are those of the
package's own workloads: 576-token images, 2880-token multi-crop images, ragged batches of
1024..16384 tokens of which 11.1 % are kept, 64 frames of 144 tokens; hidden sizes 4096 (32
heads of 128), 3584 (28 heads, 4 key/value heads) and their relatives."""
import itertools
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def listed():
    base = dict(d=128, norm=False, planes=1, interleaved=False, rot=128)
    rows = dict(base, op="rotate", B=1)
    app = dict(base, op="append", before_lo=0, before_hi=0)
    att = dict(op="attend", d=128, causal=True, groups=0, prefix=0)
    pre = dict(op="prefix", d=128, causal=True)
    return [
        # one new token of a 4096-wide decoder layer: the call's latency
        dict(rows, name="rotate_one_token", dtype="bf16", n_lo=1, n_hi=1, Hq=32, Hkv=32),
        # one 576-token image in 32 bits, with head norms and neighbouring pairs
        dict(rows, name="rotate_image_f32", dtype="f32", n_lo=576, n_hi=576, Hq=32, Hkv=32,
             norm=True, interleaved=True),
        # four videos before the step: time, height and width planes of position ids
        dict(rows, name="rotate_video_planes", dtype="bf16", B=4, n_lo=9216, n_hi=9216, Hq=28, Hkv=4,
             planes=3),
        # a step of 32 running answers, each with its own context
        dict(app, name="append_step", dtype="bf16", B=32, n_lo=1, n_hi=1, Hq=28, Hkv=4, page=16,
             norm=True, before_lo=113, before_hi=1818),
        # the retained tokens of a ragged batch, written to their pages after the step
        dict(app, name="append_retained", dtype="bf16", B=32, n_lo=113, n_hi=1818, Hq=28, Hkv=4, page=16,
             planes=3),
        # eight multi-crop images before the step, as many key heads as query heads
        dict(app, name="append_crops", dtype="bf16", B=8, n_lo=2880, n_hi=2880, Hq=32, Hkv=32, page=64),
        # a single answer over one reduced image and its prompt: latency
        dict(att, name="attend_one_token", dtype="bf16", B=1, n_lo=1, n_hi=1, kv_lo=131, kv_hi=131, Hq=32,
             Hkv=32, page=16),
        # a step of 32 answers over unreduced ragged contexts: the cache is read once
        dict(att, name="attend_step_ragged", dtype="bf16", B=32, n_lo=1, n_hi=1, kv_lo=1024, kv_hi=16384,
             Hq=28, Hkv=4, page=16),
        # one image and its prompt through a layer in 32 bits
        dict(att, name="attend_image_f32", dtype="f32", B=1, n_lo=637, n_hi=637, kv_lo=0, kv_hi=0, Hq=32,
             Hkv=32, page=64),
        # prefill of two whole videos in a layer before the step
        dict(att, name="attend_video_prefill", dtype="bf16", B=2, n_lo=9216, n_hi=9216, kv_lo=0, kv_hi=0,
             Hq=28, Hkv=4, page=64),
        # a step of 64 answers about one video
        dict(pre, name="prefix_video_step", dtype="bf16", B=64, n_lo=1, n_hi=1, kv_lo=19, kv_hi=412, Hq=28,
             Hkv=4, page=16, groups=1, prefix=9216),
        # eight prompts about each of four multi-crop images, before the first answer token
        dict(pre, name="prefix_crop_prompts", dtype="bf16", B=32, n_lo=9, n_hi=71, kv_lo=0, kv_hi=0, Hq=32,
             Hkv=32, page=64, groups=4, prefix=2880),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads, kv = rng.choice([(32, 32), (28, 4), (64, 8), (40, 40), (16, 2), (12, 12), (28, 28), (8, 1)])
    d = rng.choice([128, 128, 128, 64, 80, 96, 256])
    c = dict(op=rng.choice(["rotate", "append", "attend", "prefix"]), Hq=heads, Hkv=kv, d=d,
             dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if c["op"] in ("rotate", "append"):
        B = _log(rng, 1, 48)
        width = (heads + 2 * kv) * d * (2 if c["dtype"] == "bf16" else 4)
        top = max(1, min(9216, 300_000_000 // (width * B)))
        hi = _log(rng, 1, top)
        c.update(B=B, n_lo=_log(rng, 1, hi), n_hi=hi, norm=rng.random() < 0.5, planes=rng.choice([1, 1, 3]),
                 interleaved=rng.random() < 0.3, rot=rng.choice([d, d, d // 2]))
        if c["op"] == "append":
            c.update(page=rng.choice([16, 32, 64, 256]), before_lo=0, before_hi=rng.choice([0, 37, 700]))
        return c
    c.update(page=rng.choice([16, 32, 64, 256]), causal=rng.random() < 0.8, groups=0, prefix=0)
    B = _log(rng, 1, 64)
    kind = rng.choice(["step", "few", "prompt"])
    n_hi = 1 if kind == "step" else _log(rng, 2, 24) if kind == "few" else _log(rng, 25, 4096)
    if c["op"] == "prefix":
        c["groups"] = rng.choice([g for g in (1, 2, 4) if g <= B])
        B = c["groups"] * max(1, B // c["groups"])
        c["prefix"] = _log(rng, 33, 12000)
    kv_hi = rng.choice([0, _log(rng, 1, 16384)])
    # the scores of the plain form, and the pages, stay well under the largest listed case's
    while B * heads * n_hi * (c["prefix"] + kv_hi + n_hi) > 1_500_000_000 or B * kv * d * (kv_hi + n_hi) > 600_000_000:
        if n_hi > 1 and n_hi >= kv_hi:
            n_hi = max(1, n_hi // 2)
        elif kv_hi > 64:
            kv_hi //= 2
        else:
            B = max(max(1, c["groups"]), B // 2 // max(1, c["groups"]) * max(1, c["groups"]))
    c.update(B=B, n_lo=max(1, rng.randint(1, n_hi)), n_hi=n_hi, kv_lo=kv_hi // rng.choice([1, 2, 9]), kv_hi=kv_hi)
    return c


def _between(lo, hi, n, salt):
    """n lengths of lo..hi, the same in every run: they are part of the case, not of its inputs."""
    r = random.Random(1000003 * salt + 1009 * hi + 31 * lo + n)
    return [r.randint(lo, hi) for _ in range(n)]


def _lengths(case):
    """New tokens and keys cached before them, for each sequence."""
    n = _between(case["n_lo"], case["n_hi"], case["B"], 1)
    lo, hi = (case["kv_lo"], case["kv_hi"]) if "kv_lo" in case else (case.get("before_lo", 0), case.get("before_hi", 0))
    return n, _between(lo, hi, case["B"], 2)


def _offsets(n):
    return list(itertools.accumulate(n, initial=0))


def _sections(case):
    """Pairs of a head that follow each plane: a quarter, then the rest in two (16, 24, 24 for 64 pairs)."""
    half = case["rot"] // 2
    if case["planes"] == 1:
        return [half]
    t, h = half // 4, (half - half // 4) // 2
    return [t, h, half - t - h]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]
    B, Hq, Hkv, d = (case[k] for k in ("B", "Hq", "Hkv", "d"))
    n, before = _lengths(case)
    cu = _offsets(n)
    T = cu[-1]

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

    s = dict(case, T=T, kind=t, max_n=max(n), cu=ints(cu))
    if case["op"] in ("rotate", "append"):
        rows = normal(T, (Hq + 2 * Hkv) * d)  # a layer's fused projection, of which q, k and v are views
        s["q"] = rows[:, :Hq * d]
        s["k"] = rows[:, Hq * d:(Hq + Hkv) * d]
        s["v"] = rows[:, (Hq + Hkv) * d:]
        # carried position ids: ascending with gaps, as the retained tokens have them
        first = torch.cat([torch.arange(x) * 9 + y for x, y in zip(n, before)]).cuda()
        s["pos"] = torch.stack([torch.div(first, p + 1, rounding_mode="floor") for p in range(case["planes"])])
        s["pos"] += torch.randint(0, 9, s["pos"].shape, generator=g, device="cuda")
        half = case["rot"] // 2
        s["inv_freq"] = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
        s["sections"] = _sections(case)
        s["qw"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(t) if case["norm"] else None
        s["kw"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(t) if case["norm"] else None
        s["q_out"] = torch.empty((T, Hq * d), dtype=t, device="cuda")
        s["k_out"] = torch.empty((T, Hkv * d), dtype=t, device="cuda")
        s["l1"] = torch.empty(T, dtype=torch.float32, device="cuda")
    else:
        s["q"] = normal(T, Hq * d, by=1.5)
        s["scale"] = d ** -0.5
        s["out"] = torch.empty((T, Hq * d), dtype=t, device="cuda")
        s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
    if case["op"] != "rotate":
        page, groups = case["page"], case.get("groups", 0)
        total = [x + y for x, y in zip(n, before)]
        counts = [-(-x // page) for x in total]
        front = [-(-case.get("prefix", 0) // page)] * groups
        pages = sum(counts) + sum(front) + 3
        perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
        table, at = tables(counts, 0, perm)
        s["table"], s["kv_len"], s["max_kv"], s["n_pages"] = table.cuda(), ints(total), max(total), pages
        s["k_pool"] = normal(pages, Hkv, page, d)
        s["v_pool"] = normal(pages, Hkv, page, d)
        if groups:
            s["front"] = tables(front, at, perm)[0].cuda()
            s["group_cu"] = ints([i * (B // groups) for i in range(groups + 1)])
            s["front_len"] = ints([case["prefix"]] * groups)
    if own:
        import paper_2502_11494_amd as D
        kind = D.DART_BF16 if case["dtype"] == "bf16" else D.DART_F32
        if case["op"] in ("rotate", "append"):
            s["rotation"] = D.make_rotation(Hq, Hkv, d, kind, s["inv_freq"], interleaved=case["interleaved"],
                                            sections=s["sections"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS)
        if case["op"] != "rotate":
            more = {}
            if case.get("groups"):
                more = dict(group_cu=s["group_cu"], prefix_pages=s["front"], prefix_len=s["front_len"],
                            max_prefix=case["prefix"])
            s["cache"] = D.make_cache(Hq, s["k_pool"], s["table"], s["kv_len"], s["max_kv"], T=T, max_q=s["max_n"],
                                      cu_q=None if s["max_n"] == 1 else s["cu"], **more)
        if case["op"] in ("attend", "prefix"):
            s["ws"] = D.alloc_attend_workspace(s["cache"])
    return s


def run(s):
    if own:
        return _own(s)
    if s["op"] == "rotate":
        return _plain_rotate(s)
    if s["op"] == "append":
        return _plain_append(s)
    return _plain_attend(s)


def _own(s):
    import paper_2502_11494_amd as D
    if s["op"] == "rotate":
        D.dart_norm_rotate(s["rotation"], s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], l1_out=s["l1"])
        return s["q_out"], s["k_out"], s["l1"]
    if s["op"] == "append":
        D.dart_norm_rotate_append(s["rotation"], s["cache"], s["q"], s["k"], s["v"], s["pos"], s["q_out"],
                                  s["k_pool"], s["v_pool"], l1_out=s["l1"])
        return s["q_out"], s["k_pool"], s["v_pool"], s["l1"]
    D.dart_attend(s["cache"], s["q"], s["k_pool"], s["v_pool"], s["out"], s["ws"], scale=s["scale"],
                  causal=s["causal"], lse=s["lse"])
    return s["out"], s["lse"]


# ---- plain forms ---------------------------------------------------------------------------

def _rotated(x, heads, weight, s):
    """Heads of x normed, rotated and rounded once: [T, heads, d].  The angle alone is taken in 64 bits: a
    position times a frequency has no 32-bit product that is good to 32 bits as an angle."""
    T, d, rot = s["T"], s["d"], s["rot"]
    y = x.float().view(T, heads, d)
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    plane = torch.repeat_interleave(torch.arange(len(s["sections"]), device="cuda"),
                                    torch.tensor(s["sections"], device="cuda"), output_size=rot // 2)
    angle = s["pos"][plane].t().double() * s["inv_freq"].double()
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if s["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * c - b * n, b * c + a * n), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(s["kind"])


def _plain_rotate(s):
    q = _rotated(s["q"].reshape(s["T"], -1), s["Hq"], s["qw"], s)
    k = _rotated(s["k"].reshape(s["T"], -1), s["Hkv"], s["kw"], s)
    return q.flatten(1), k.flatten(1), k.float().abs().sum((1, 2))


def _plain_append(s):
    q, k, l1 = _plain_rotate(s)
    token = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu"], token, right=True) - 1
    place = s["kv_len"][b] - s["cu"][b + 1] + token
    page, inside = s["table"][b, torch.div(place, s["page"], rounding_mode="floor")].long(), place % s["page"]
    s["k_pool"][page, :, inside] = k.view(s["T"], s["Hkv"], s["d"])
    s["v_pool"][page, :, inside] = s["v"].reshape(s["T"], s["Hkv"], s["d"])
    return q, s["k_pool"], s["v_pool"], l1


def _paged(pool, table):
    """[rows of the table, heads, keys, d] in 32 bits."""
    x = pool[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1]).float()


def _plain_attend(s):
    B, Hq, Hkv, d, m, T = s["B"], s["Hq"], s["Hkv"], s["d"], s["max_n"], s["T"]
    r, groups, cu = Hq // Hkv, s["groups"], s["cu"].long()
    at = cu[:-1, None] + torch.arange(m, device="cuda")
    real = at < cu[1:, None]
    q = s["q"].float().view(T, Hkv, r, d)[at.clamp(max=T - 1)]                     # [B, m, Hkv, r, d]
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, m * r, d) * s["scale"]
    k, v = _paged(s["k_pool"], s["table"]), _paged(s["v_pool"], s["table"])
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
        fk, fv = _paged(s["k_pool"], s["front"])[:, :, :s["prefix"]], _paged(s["v_pool"], s["front"])[:, :, :s["prefix"]]
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


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    n, before = _lengths(case)
    T, e = sum(n), 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    if case["op"] in ("rotate", "append"):
        values = (Hq + Hkv * (2 if case["op"] == "append" else 1)) * d
        return {"bytes": 2 * T * values * e + T * (8 * case["planes"] + 4), "flops": T * (Hq + Hkv) * d * (7 if case["norm"] else 3)}
    keys = sum(x + y for x, y in zip(n, before)) + case["groups"] * case["prefix"]
    if case["causal"]:
        seen = sum(x * y + x * (x + 1) // 2 for x, y in zip(n, before))
    else:
        seen = sum(x * (x + y) for x, y in zip(n, before))
    seen += T * case["prefix"]
    return {"bytes": 2 * T * Hq * d * e + T * Hq * 4 + 2 * keys * Hkv * d * e, "flops": 4 * d * Hq * seen}


# ---- the same from the definitions, in 64 bits ----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    n, before = _lengths(case)
    T, Hq, Hkv, d, cu = s["T"], s["Hq"], s["Hkv"], s["d"], _offsets(n)
    if case["op"] in ("attend", "prefix"):
        page, r = case["page"], Hq // Hkv
        if 8 * d * Hq * T * max(case["prefix"] + x + y for x, y in zip(n, before)) > 2e14:
            return None
        out = torch.zeros((T, Hq, d), dtype=torch.float64, device="cuda")
        lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
        per = case["B"] // case["groups"] if case["groups"] else 1

        def rows_of(pool, table, count, h):
            at = torch.arange(count, device="cuda")
            return pool[table.long()[at // page], h, at % page].double()

        for b in range(case["B"]):
            for h in range(Hkv):
                k = rows_of(s["k_pool"], s["table"][b], before[b] + n[b], h)
                v = rows_of(s["v_pool"], s["table"][b], before[b] + n[b], h)
                if case["groups"]:
                    k = torch.cat((rows_of(s["k_pool"], s["front"][b // per], case["prefix"], h), k))
                    v = torch.cat((rows_of(s["v_pool"], s["front"][b // per], case["prefix"], h), v))
                hidden = None
                if case["causal"]:  # token i does not see what comes after it
                    hidden = torch.ones((n[b], k.shape[0]), dtype=torch.bool, device="cuda").triu(k.shape[0] - n[b] + 1)
                for j in range(h * r, (h + 1) * r):
                    z = s["q"][cu[b]:cu[b + 1], j * d:(j + 1) * d].double() @ k.t() * s["scale"]
                    if hidden is not None:
                        z[hidden] = -math.inf
                    lse[cu[b]:cu[b + 1], j] = torch.logsumexp(z, -1)
                    out[cu[b]:cu[b + 1], j] = torch.softmax(z, -1) @ v
        return out.reshape(T, -1), lse
    half = s["rot"] // 2
    planes = [p for p, count in enumerate(s["sections"]) for _ in range(count)]

    def turn(x, w):
        x = x.double().reshape(T, -1, d).clone()
        if w is not None:
            x = w.double() * x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + half)
            z = torch.polar(torch.ones(T, dtype=torch.float64, device="cuda"), s["pos"][planes[i]].double() * float(s["inv_freq"][i]))
            z = torch.complex(x[:, :, a], x[:, :, b]) * z[:, None]
            x[:, :, a], x[:, :, b] = z.real, z.imag
        return x

    q, k = turn(s["q"], s["qw"]), turn(s["k"], s["kw"])
    # the norm is that of the keys as they are stored, so their rounding belongs to its definition
    l1 = k.to(s["kind"]).double().abs().sum((1, 2)) if case["dtype"] == "f32" else None
    if case["op"] == "rotate":
        return q.reshape(T, -1), k.reshape(T, -1), l1
    kp, vp, v = s["k_pool"].double(), s["v_pool"].double(), s["v"].double().reshape(T, Hkv, d)
    page = case["page"]
    for b in range(case["B"]):
        place = torch.arange(before[b], before[b] + n[b], device="cuda")
        where = s["table"][b].long()[place // page] * page + place % page
        for pool, rows in ((kp, k), (vp, v)):
            flat = pool.transpose(1, 2).reshape(-1, Hkv, d)
            flat[where] = rows[cu[b]:cu[b + 1]]
            pool.copy_(flat.view(-1, page, Hkv, d).transpose(1, 2))
    return q.reshape(T, -1), kp, vp, l1
