"""Position planes of every number, and one plane broadcast to several."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A
from test_gpu_norm_rotate import definition, inputs, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sections", [[64], [20, 44], [0, 64], [64, 0], [16, 24, 24], [1, 0, 63], [8, 16, 24, 16], [1, 0, 0, 63], [0, 0, 0, 64]])
@pytest.mark.parametrize("interleaved", [False, True])
def test_planes(dtype, sections, interleaved):
    T, planes = 61, len(sections)
    rows, _, inv_freq, _, _, _ = inputs(T, 4, 2, 128, 128, 1, dtype, False, seed=planes)
    pos = torch.randint(0, 16384, (planes, T), generator=torch.Generator().manual_seed(7))
    q, k = rows[:, :512], rows[:, 512:768]
    r = D.make_rotation(4, 2, 128, A.KIND[rows.dtype], inv_freq.cuda(), interleaved=interleaved, sections=sections)
    out = [torch.empty((T, n), dtype=rows.dtype, device="cuda") for n in (512, 256)]
    wide = torch.full((planes, T + 5), -1, dtype=torch.int64)  # (planes further apart than their tokens)
    wide[:, 2:T + 2] = pos
    for ids in (pos.cuda(), wide.cuda()[:, 2:T + 2]):
        D.dart_norm_rotate(r, q.cuda(), k.cuda(), ids if planes > 1 else ids[0], *out)
        torch.cuda.synchronize()
        for got, src, heads in ((out[0], q, 4), (out[1], k, 2)):
            want, tol = definition(src, heads, 128, 128, pos, sections, inv_freq, interleaved, None, 1.0)
            within(got.cpu().view(T, heads, 128), want, tol, rows.dtype)


@pytest.mark.parametrize("planes", [2, 3, 4])
@pytest.mark.parametrize("T", [1, 50, 1500])
def test_one_plane_expanded_is_as_many_copies(planes, T):
    rows, _, inv_freq, _, _, _ = inputs(T, 4, 2, 64, 64, 1, "bf16", False, seed=3)
    pos = torch.randint(0, 16384, (T,), generator=torch.Generator().manual_seed(8)).cuda()
    sections = [8] * (planes - 1) + [32 - 8 * (planes - 1)]
    r = D.make_rotation(4, 2, 64, D.DART_BF16, inv_freq.cuda(), sections=sections)
    got = []
    for ids in (pos.expand(planes, -1).contiguous(), pos.expand(planes, -1)):
        q, k = (torch.empty((T, n), dtype=rows.dtype, device="cuda") for n in (256, 128))
        D.dart_norm_rotate(r, rows[:, :256].cuda(), rows[:, 256:384].cuda(), ids, q, k)
        got.append((q, k))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
