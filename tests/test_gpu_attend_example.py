"""The example's path through the calls, against a plain statement of the same two layers in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_rows(layer, x, pos):
    """Queries, keys and values of rows x, as the calls define them, each rounded once."""
    Hq, Hkv, d = layer.Hq, layer.Hkv, layer.d
    rows = (x @ layer.w).double().cpu()
    q, k, v = rows[:, :Hq * d].view(-1, Hq, d), rows[:, Hq * d:(Hq + Hkv) * d].view(-1, Hkv, d), rows[:, (Hq + Hkv) * d:].view(-1, Hkv, d)
    half = d // 2
    sections = list(layer.rotation.sections)[:3]
    plane = [p for p, n in enumerate(sections) for _ in range(n)]
    freq = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().double()
    theta = pos.cpu()[plane].t().double() * freq
    c, s = theta.cos()[:, None], theta.sin()[:, None]

    def turned(y):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        return torch.cat((y[..., :half] * c - y[..., half:] * s, y[..., half:] * c + y[..., :half] * s), -1).bfloat16().double()

    return turned(q), turned(k), v


def plain_attention(q, k, v, before, d):
    """Causal attention of q's tokens, `before` keys lying before them."""
    r = q.shape[1] // k.shape[1]
    s = torch.einsum("nhd,khd->hnk", q, k.repeat_interleave(r, 1)) / d ** 0.5
    hidden = torch.ones(q.shape[0], k.shape[0], dtype=torch.bool).triu(before + 1)
    return torch.einsum("hnk,khd->nhd", torch.softmax(s.masked_fill(hidden, -float("inf")), -1), v.repeat_interleave(r, 1))


def test_the_example_computes_what_it_says():
    import answers_about_a_reduced_image as E
    r = E.main(images=2, N=200, width=256, keep=40, Hq=4, Hkv=2, d=64, questions=3, prompt=7, answer=2, page=16)
    w = r["w"]
    # the norms are those of the stored keys, and the retained sets those of an exact ranking by them
    k = r["k_rows"][r["vision"]]
    exact = k.double().abs().sum(1)
    assert bool(((r["l1"][r["vision"]].double() - exact).abs() <= 2.0 ** -20 * exact).all())
    kept = r["kept"].cpu().numpy().reshape(w.B, -1)
    # (the step saw the hidden states after the first layer; its rows in the shortened sequences are bit copies)
    assert all((np.diff(kept[b]) > 0).all() and kept[b].max() < 200 for b in range(w.B))
    for b in range(w.B):
        norms = exact[b * 200:(b + 1) * 200].cpu().numpy()
        assert set(np.argsort(-norms, kind="stable")[:8].tolist()) <= set(kept[b].tolist()), "the pivots are kept"
    # the second layer: prefixes, then the questions' prompts over them
    second, lens = r["second"], r["lens"]
    start = np.concatenate([[0], np.cumsum(lens)])
    at = int(r["short_pos"].max()) + 1
    width = r["short"].shape[1]
    g_state = r["outputs"]
    for b in range(w.B):
        rows = slice(int(start[b]), int(start[b + 1]))
        q, kk, v = plain_rows(second, r["short"][rows], r["short_pos"][:, rows])
        out = plain_attention(q, kk, v, 0, second.d).reshape(lens[b], -1)
        want = r["short"][rows].double().cpu() + out @ second.back.double().cpu()
        got = r["prefix_out"][rows].double().cpu()
        assert float((got - want).norm() / want.norm()) < 5e-3
        # an answer token's attention sees the prefix and its own keys: read the pages back and state it plainly
        for j in range(b * 3, b * 3 + 3):
            done = 7 + 2
            own_k = torch.cat([second.k_pool[int(p)].transpose(0, 1) for p in r["own_table"][j]])[:done].double().cpu()
            own_v = torch.cat([second.v_pool[int(p)].transpose(0, 1) for p in r["own_table"][j]])[:done].double().cpu()
            x = torch.tanh(g_state[1].view(-1, width)[j:j + 1])
            q, k1, v1 = plain_rows(second, x, torch.full((3, 1), at + done - 1))
            assert float((own_k[-1:] - k1).abs().max()) < 0.1 and float((own_v[-1:] - v1).abs().max()) < 0.05
            out = plain_attention(q, torch.cat((kk, own_k)), torch.cat((v, own_v)), lens[b] + done - 1, second.d).reshape(1, -1)
            want = x.double().cpu() + out @ second.back.double().cpu()
            got = g_state[2].view(-1, width)[j:j + 1].double().cpu()
            assert float((got - want).norm() / want.norm()) < 1e-2
