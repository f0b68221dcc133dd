"""Two attention layers around the reduction step, and answers about what it kept.

A batch of sequences (text, vision tokens, text) goes through the attention of one layer: queries
and keys are normed and turned by three planes of position ids, keys and values go to the layer's
pages, and the L1 norms of the key rows come out beside them.  The step ranks the vision tokens by those
norms, keeps the budget, and shortens the sequences.  The next layer runs on the shortened sequences
with their carried position ids, into pages of its own; they are the shared prefixes of the questions
that follow: one prompt each, then answer tokens one at a time.

    python examples/answers_about_a_reduced_image.py

The weights are random: this shows the calls and their order, not a model."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_11494_amd as D  # noqa: E402
from paper_2502_11494_amd import workloads as W  # noqa: E402


class Layer:
    """The attention of a decoder layer: projections, head norms, pages."""

    def __init__(self, width, Hq, Hkv, d, n_pages, page, g):
        self.Hq, self.Hkv, self.d, self.page = Hq, Hkv, d, page
        self.w = (torch.randn((width, (Hq + 2 * Hkv) * d), generator=g, device="cuda") / width ** 0.5).bfloat16()
        self.back = (torch.randn((Hq * d, width), generator=g, device="cuda") / (Hq * d) ** 0.5).bfloat16()
        self.k_pool = torch.empty((n_pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda")
        self.v_pool = torch.empty_like(self.k_pool)
        half = d // 2
        t, h = half // 4, (half - half // 4) // 2
        inv_freq = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
        weight = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        self.rotation = D.make_rotation(Hq, Hkv, d, D.DART_BF16, inv_freq, sections=[t, h, half - t - h],
                                        q_weight=weight, k_weight=weight)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, x, pos, cache, keys=False):
        """x [T, width] -> x + attention; the key rows and their L1 norms with `keys`."""
        T = x.shape[0]
        rows = x @ self.w
        nq, nk = self.Hq * self.d, self.Hkv * self.d
        q, k, v = rows[:, :nq], rows[:, nq:nq + nk], rows[:, nq + nk:]
        k_rows = torch.empty((T, nk), dtype=x.dtype, device="cuda") if keys else None
        l1 = torch.empty(T, dtype=torch.float32, device="cuda") if keys else None
        D.dart_norm_rotate_append(self.rotation, cache, q, k, v, pos, q, self.k_pool, self.v_pool, k_out=k_rows,
                                  l1_out=l1, status=self.status)
        out = torch.empty((T, nq), dtype=x.dtype, device="cuda")
        D.dart_attend(cache, q, self.k_pool, self.v_pool, out, D.alloc_attend_workspace(cache), scale=self.d ** -0.5,
                      status=self.status)
        return x + out @ self.back, k_rows, l1


def pages_for(counts, first):
    """A page table for sequences of so many pages, numbered from `first` on."""
    table = torch.zeros((len(counts), max(counts)), dtype=torch.int32)
    for b, n in enumerate(counts):
        table[b, :n] = torch.arange(first, first + n)
        first += n
    return table.cuda(), first


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def main(images=2, N=576, width=1024, keep=64, Hq=8, Hkv=2, d=64, questions=3, prompt=11, answer=4, page=16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = W.image_batch(B=images, N=N, D=width, K=keep, P=8, n_centroids=max(8, N // 9))
    sq = W.sequences_around(w, seed=1, before=(5, 9), after=(3, 7), n_kv=0)
    rows, lens = sq.H.shape[0], [int(x) for x in sq.seq_cu[1:] - sq.seq_cu[:-1]]
    x = torch.from_numpy(sq.H.view("int16")).view(torch.bfloat16).cuda()
    pos = torch.from_numpy(sq.pos).cuda()

    # ---- a layer before the step, over whole sequences
    counts = [-(-n // page) for n in lens]
    table, n_pages = pages_for(counts, 0)
    first = Layer(width, Hq, Hkv, d, n_pages, page, g)
    cache = D.make_cache(Hq, first.k_pool, table, ints(lens), max(lens), T=rows, max_q=max(lens), cu_q=ints(sq.seq_cu.tolist()))
    x, k_rows, l1 = first.run(x, pos, cache, keys=True)

    # ---- the step: vision tokens ranked by the norms of the keys just made (good to 2^-20 of their value)
    cu, span = torch.from_numpy(w.cu).cuda(), torch.from_numpy(sq.span_start).cuda()
    total = int(w.cu[-1])
    desc = D.make_desc(images, width, 8, D.DART_BF16, K=keep, cu_seqlens=cu, total_N=total, max_N=N, span_start=span, X_rows=rows)
    ws = D.alloc_workspace(desc)
    vision = torch.cat([torch.arange(int(s), int(s) + N) for s in sq.span_start]).cuda()
    kept = torch.empty(images * keep, dtype=torch.int32, device="cuda")
    D.dart_reduce_with_norms(desc, x, None, kept, ws, l1[vision].contiguous(), 2.0 ** -20, crit=k_rows, crit_D=Hkv * d,
                             crit_ld=k_rows.stride(0))
    left = rows - total + images * keep
    short = torch.empty((left, width), dtype=x.dtype, device="cuda")
    short_pos = torch.empty((3, left), dtype=torch.int64, device="cuda")
    short_cu, row_map = torch.empty(images + 1, dtype=torch.int32, device="cuda"), torch.empty(left, dtype=torch.int32, device="cuda")
    D.dart_compact_sequences(desc, torch.from_numpy(sq.seq_cu).cuda(), kept, [(x, short)], short_cu, row_map, ws, pos=pos,
                             pos_out=short_pos)
    assert D.dart_device_status(desc, ws) == D.DART_OK

    # ---- the next layer, on the shortened sequences with the position ids they carry
    lens = [n - N + keep for n in lens]
    counts = [-(-n // page) for n in lens]
    prefix_table, used = pages_for(counts, 0)
    B = images * questions
    own_pages = [-(-(prompt + answer) // page)] * B
    own_table, n_pages = pages_for(own_pages, used)
    second = Layer(width, Hq, Hkv, d, n_pages, page, g)
    cache = D.make_cache(Hq, second.k_pool, prefix_table, ints(lens), max(lens), T=left, max_q=max(lens), cu_q=short_cu)
    prefix_out, _, _ = second.run(short, short_pos, cache)

    # ---- questions about each: the shortened sequence is their shared prefix
    shared = dict(group_cu=ints([i * questions for i in range(images + 1)]), prefix_pages=prefix_table,
                  prefix_len=ints(lens), max_prefix=max(lens))
    at = short_pos.amax() + 1
    state = (0.5 * torch.randn((B * prompt, width), generator=g, device="cuda")).bfloat16()
    outputs = []
    for step in range(answer + 1):
        n = prompt if step == 0 else 1
        done = prompt + step if step else prompt
        place = torch.arange(done - n, done, device="cuda").repeat(B) + at
        cache = D.make_cache(Hq, second.k_pool, own_table, ints([done] * B), done, T=B * n, max_q=n,
                             cu_q=ints([i * n for i in range(B + 1)]) if n > 1 else None, **shared)
        state, _, _ = second.run(state, place.expand(3, -1), cache)
        outputs.append(state)
        state = torch.tanh(state.view(B, n, width)[:, -1])  # (what a model would sample, embed and feed back)
    torch.cuda.synchronize()
    assert int(first.status) == 0 and int(second.status) == 0
    return dict(first=first, second=second, kept=kept, l1=l1, k_rows=k_rows, vision=vision, short=short, short_pos=short_pos,
                row_map=row_map, prefix_out=prefix_out, lens=lens, outputs=outputs, prefix_table=prefix_table, own_table=own_table,
                questions=questions, prompt=prompt, w=w)


if __name__ == "__main__":
    r = main()
    print(f"{r['w'].B} images of {int(r['w'].lengths[0])} tokens, {r['kept'].numel() // r['w'].B} kept of each; "
          f"prefixes of {r['lens']} tokens; {len(r['outputs'])} steps of {r['questions']} questions each, "
          f"last hidden states {tuple(r['outputs'][-1].shape)}")
