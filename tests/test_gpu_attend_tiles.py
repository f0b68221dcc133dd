"""Tiles and head widths that the prefixes of the other tests do not reach: eight waves of rows over a prefix, alone and with own keys
in the same tiles; heads of 80, 96, 192 and 256; 32-bit heads over 128, whose prefixes and own keys take a launch each."""
import pytest
import torch

import attend_util as A

pytestmark = pytest.mark.gpu


def wide_enough(c, rows_of_an_owner, max_keys):
    """The rule for eight waves of rows (bf16, heads of up to 128)."""
    return c.T * (c.Hq // c.Hkv) // 256 * c.Hkv >= 384 and rows_of_an_owner > 128 and max_keys >= 1024


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 32, 64), (32, 32, 128), (36, 36, 80), (28, 4, 128), (40, 40, 96)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("own", ["few keys", "many keys"])
def test_widest_tiles_over_prefixes(Hq, Hkv, d, causal, own):
    n = [500, 1, 700, 450, 0, 600, 513, 800]
    kv = [x + i % 5 * 13 for i, x in enumerate(n)]
    c = A.make(n, kv, Hq, Hkv, d, 32, "bf16", groups=[3, 0, 4, 1], prefix=[1100, 7, 64, 0], seed=d)
    assert wide_enough(c, c.T * (Hq // Hkv) // 4, 1100)
    max_kv = 900 if own == "few keys" else 2000
    assert wide_enough(c, 800 * (Hq // Hkv), max_kv) == (own == "many keys")
    A.check(c, A.attend(c, scale=d ** -0.5, causal=causal, max_kv=max_kv), scale=d ** -0.5, causal=causal)


def test_values_that_are_no_numbers_in_the_widest_tiles_with_a_prefix():
    n = [500, 300, 700, 450, 100, 600, 513, 800]
    c = A.make(n, n, 32, 32, 64, 32, "bf16", groups=[5, 3], prefix=[1100, 64], seed=9)
    assert wide_enough(c, c.T // 2, 1100) and wide_enough(c, 800, 2000)
    want, want_lse, tol, lse_tol = A.reference(c, 0.125, True)
    c.v_pool[int(c.table[2, 333 // 32]), 5, 333 % 32] = float("nan")   # an own key of sequence 2
    c.v_pool[int(c.front[1, 1]), 9, 7] = float("inf")                  # a key of the second prefix
    out, lse = A.attend(c, scale=0.125, max_kv=2000)
    ok = torch.ones((c.T, 32), dtype=torch.bool)
    ok[int(c.cu[2]) + 333:int(c.cu[3]), 5] = False
    ok[int(c.cu[5]):, 9] = False
    assert bool(((out.double() - want).abs() <= tol)[ok].all()) and bool(((lse.double() - want_lse).abs() <= lse_tol).all())
    assert torch.isnan(out[int(c.cu[2]) + 333:int(c.cu[3]), 5].float()).all()
    assert bool((out[int(c.cu[5]):, 9].float() == float("inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 80), (6, 2, 96), (4, 2, 192), (8, 2, 256), (14, 1, 256), (3, 3, 40)])
def test_prefixes_of_heads_of_every_width(dtype, Hq, Hkv, d):
    for n, groups, prefix in (([1] * 9, [4, 2, 3], [700, 0, 65]), ([5, 1, 0, 33, 2, 1, 70, 1, 8], [4, 0, 2, 3], [1, 9, 1300, 64]),
                              ([40, 130, 1, 70] * 2, [8], [333])):
        kv = [a + b for a, b in zip(n, [0, 3, 64, 100, 17, 0, 31, 250, 9])]
        c = A.make(n, kv, Hq, Hkv, d, 16, dtype, groups=groups, prefix=prefix, seed=d)
        for causal in (True, False):
            A.check(c, A.attend(c, scale=d ** -0.5, causal=causal), scale=d ** -0.5, causal=causal)


def test_uneven_groups():
    """The tile of the prefixes is chosen for the groups' average; one group has nearly all the sequences."""
    for dtype in ("bf16", "f32"):
        c = A.make([1] * 64, [1 + i % 7 for i in range(64)], 4, 4, 128, 16, dtype, groups=[61, 1, 1, 1], prefix=[900, 3, 0, 300], seed=11)
        A.check(c, A.attend(c, scale=0.09), scale=0.09)
