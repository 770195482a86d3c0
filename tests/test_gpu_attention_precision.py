"""How near attention over a paged cache comes to 64 bits over whole outputs, where single errors average: root mean squares, which a
product in fewer bits than the type's would exceed many times over.

Bounds by arithmetic, relative to the outputs' root mean square.  A rounding to a type of half step u errs by u / sqrt(3) at the most in the
mean of squares (evenly spread over +-u).
 * 16-bit types: one rounding of every probability and one of the result, u sqrt(2 / 3); independent roundings of probabilities err in the
   output as the probabilities' own spread over the values does, so no factor is added.
 * fp32 parts of every type: a score is a sum of hd products, hd roundings (at random, so sqrt(hd)) of partial sums of up to sqrt(hd) for
   standard normal entries, over sqrt(hd): sqrt(hd) 2^-24, twice for its own and the maximum's; 16 x 2^-24 for the difference, its scaling and the
   exponential at exponents of up to ten; sums over n keys: at most n / 4 additions in a row, at random sqrt(n) / 2 roundings, for the sum of
   probabilities and for the product with the values."""
import math

import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu


def attend(cache, q, cu, past, max_new, share=False):
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, q.shape[1], q.shape[0], len(cu) - 1, max_new, share))
    return binding.radix_paged_attention(cache, 0, q, CU.i32(cu), CU.i32(past), max_new, ws, find_shared=share)


def queries(seed, N, hq, hd, dtype):
    return torch.randn((N, hq, hd), generator=torch.Generator().manual_seed(seed)).to(CU.DT[dtype]).cuda()


@pytest.mark.parametrize("dtype,hd", [("f32", 4), ("f32", 64), ("f32", 128), ("bf16", 128), ("f16", 128)])
@pytest.mark.parametrize("past,news", [([300, 40, 700], [1, 1, 1]), ([300, 40, 700], [9, 12, 16]), ([300, 40, 700], [70, 130, 33]), ([6000], [1]),
                                       ([6000], [60])])
@pytest.mark.parametrize("share", [False, True])
def test_root_mean_square_errors(dtype, hd, past, news, share):
    lens = [p + n for p, n in zip(past, news)]
    cache = CU.random_cache(5, lens, 2, hd, 16, dtype)
    if share:
        cache.page_table[1:, :16] = cache.page_table[0, :16]
    cu = CU.ragged(news)
    q = queries(6, cu[-1], 4, hd, dtype)
    o = attend(cache, q, cu, past, max(news), share).cpu().double()
    ref, _ = CU.attention_ref(cache, 0, q, cu, past)
    err = ((o - ref).square().mean() / ref.square().mean()).sqrt().item()
    fp32 = (2 * math.sqrt(hd) + 16 + 2 * math.sqrt(max(lens)) / 2) * 2.0 ** -24
    rounded = CU.HALF_STEP[dtype] * math.sqrt(2 / 3) if dtype != "f32" else 2.0 ** -24
    assert err <= fp32 + rounded, f"{err:.3g} of {fp32 + rounded:.3g}"


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_rows_whose_best_key_leads_take_its_value(dtype, n):
    # entries of 20: a score of standard deviation 400, off by 2^-24 * 132 * |q||k| / sqrt(hd) <= 0.5; a lead of 20 leaves others e^-19 a key
    cache = CU.random_cache(3, [70 + n] * 4, 1, 128, 16, dtype, scale=20.0)
    q = queries(4, 4 * n, 2, 128, dtype) * 20
    out = attend(cache, q, CU.ragged([n] * 4), [70] * 4, n).cpu().double()
    led = 0
    for b in range(4):
        k, v = (CU.rows_of(cache, 0, b, 70 + n, kind)[:, 0] for kind in (0, 1))
        for i in range(n):
            s = q[b * n + i].cpu().double() @ k[:71 + i].T / math.sqrt(128)
            top = torch.topk(s, 2, dim=1)
            for h in range(2):
                if top.values[h, 0] - top.values[h, 1] > 20:
                    led += 1
                    want = v[top.indices[h, 0]]
                    others = 110 * math.exp(-19) * 2 * 110          # weights times differences of values (5.5 times 20 each)
                    assert ((out[b * n + i, h] - want).abs() <= 2 * CU.HALF_STEP[dtype] * want.abs() + others).all()
    assert led >= 4 * n
