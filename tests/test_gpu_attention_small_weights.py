"""fp16 attention over a paged cache where one key outweighs every other by 2^24 and more, and the others together still count: each
weight lies below what fp16 holds without losing bits, or holds at all, next to a weight of 1."""
import math

import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,max_new", [(1, 1), (12, 12), (40, 40), (1, 40)])            # 2 rows, 24, 80; and 2 beside a kernel for many
@pytest.mark.parametrize("keys", [2000, 131072])
@pytest.mark.parametrize("bits", [20.3, 24.6, 25.2, 30.0])
def test_many_small_weights_beside_a_large_one(n, max_new, keys, bits):
    page = 256
    pages = -(-keys // page)
    cache = binding.alloc_cache(1, 1, 128, page, pages, torch.float16, 1, pages)
    cache.pages.zero_()
    cache.page_table.copy_(torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1))
    cache.pages[0, 777 // page, 0, 0, 777 % page, 0] = 16.0
    per_log2 = 16.0 * math.log2(math.e) / math.sqrt(128)                    # of the leading key's score, by q[0]
    q = torch.zeros((n, 2, 128), dtype=torch.float16, device="cuda")
    q[:, 0, 0], q[:, 1, 0] = bits / per_log2, (bits + 0.4) / per_log2
    v = torch.linspace(0.25, 2.0, 128).half()
    cache.pages[0, :, 1] = v.cuda()
    cache.pages[0, 777 // page, 1, 0, 777 % page] = 0.0
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, 2, n, 1, max_new))
    past = keys - n
    out = binding.radix_paged_attention(cache, 0, q, CU.i32([0, n]), CU.i32([past]), max_new, ws).cpu().double()
    w = torch.exp2(-q[:, :, 0].cpu().double() * per_log2)                   # weight of every other key
    others = (past + torch.arange(n, dtype=torch.float64))[:, None] * w
    want = (others / (1 + others))[:, :, None] * v.double()
    # Half a step of fp16 on the weight and on the result; 2^-19 for the score (128 exact products) and its exponential; sums of equal
    # terms: a lane of four wavefronts adds up at most a sixteenth of the keys one after the other, half a step of fp32 each time, on
    # both sides of the quotient (4 more levels where parts are joined).
    # A weight times 2^15 below 2^-14 is off by half a step of those numbers, 2^-25: 2^-40 of the leading one, for every other key.
    rel = 2 * 2.0 ** -11 + 2.0 ** -19 + 2 * (keys / 16 + 64) * 2.0 ** -25
    tol = rel * want + keys * 2.0 ** -40 * v.double() + 2.0 ** -25          # (results below 2^-14: half a step of those)
    err = (out - want).abs()
    assert (err <= tol).all(), f"off by up to {(err / want).max().item():.3g} of the result, {rel:.3g} allowed"
