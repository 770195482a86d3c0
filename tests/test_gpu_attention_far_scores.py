"""Attention over a paged cache where scores are so large that a rounding of one is a whole power of two or many: finite inputs give
finite outputs, and the key that leads by more than anything else could weigh is the answer, exactly."""
import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu

# entries whose products stay in fp32's range: 128 c^2 is 2^23 to 2^39 for bf16 and fp32, up to 2^38 for fp16, and far above for bf16 and fp32
SIZES = {"f16": [300.0, 1000.0, 6000.0, 20000.0, 50000.0], "bf16": [300.0, 6000.0, 1e5, 3e9, 1e15], "f32": [300.0, 6000.0, 1e5, 3e9, 1e15]}


def attend(cache, q, cu, past, max_new, share=False):
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, q.shape[1], q.shape[0], len(cu) - 1, max_new, share))
    ws.fill_(0xFF)
    return binding.radix_paged_attention(cache, 0, q, CU.i32(cu), CU.i32(past), max_new, ws, find_shared=share)


@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 128), ("f32", 128), ("f32", 20)])
@pytest.mark.parametrize("news", [[1, 1, 1], [12, 9, 1], [70, 40, 1]])                  # 2, then up to 24, then up to 140 rows
@pytest.mark.parametrize("past", [40, 3000])                                            # whole, and split over workgroups
def test_one_key_leads_by_more_than_scores_resolve(dtype, hd, news, past):
    for i, size in enumerate(SIZES[dtype]):
        g = torch.Generator().manual_seed(i)
        lens = [past + n for n in news]
        cache = CU.random_cache(i, lens, 1, hd, 32, dtype)
        table, want = cache.page_table.tolist(), []
        for b in range(len(news)):
            # keys of a tenth of the size, one of them (which every new token sees) at full size: it leads by 0.9 of its score at the least
            at = torch.arange(lens[b])
            pages = torch.tensor(table[b])[at // 32]
            sign = torch.randint(0, 2, (lens[b], 1), generator=g) * 0.2 - 0.1
            keys = (sign * size * (1 + torch.rand((lens[b], hd), generator=g) / 16)).to(CU.DT[dtype])
            best = (past * (b + 1)) // 4
            keys[best] = torch.full((hd,), size * (1 + 0.37 * b)).to(CU.DT[dtype])
            cache.pages[0, pages.cuda(), 0, 0, (at % 32).cuda()] = keys.cuda()
            want.append(cache.pages[0, table[b][best // 32], 1, 0, best % 32].expand(news[b], 2, hd))
        q = (size * (1 + torch.rand((sum(news), 2, 1), generator=g) / 4)).to(CU.DT[dtype]).expand(-1, -1, hd).contiguous().cuda()
        if dtype == "f16" and size > 40000:
            q = q.clamp(max=60000)
            cache.pages[0, :, 0].clamp_(-60000, 60000)
        out = attend(cache, q, CU.ragged(news), [past] * len(news), max(news))
        assert torch.isfinite(out).all(), size
        assert torch.equal(out, torch.cat(want)), size


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_and_over_common_pages(dtype):
    for i, size in enumerate(SIZES[dtype][:4]):
        cache = CU.random_cache(i, [700] * 6, 1, 128, 16, dtype)
        cache.page_table[1:, :40] = cache.page_table[0, :40]
        table = cache.page_table.tolist()
        cache.pages[0, :, 0] = 0.0
        cache.pages[0, table[0][100 // 16], 0, 0, 100 % 16] = size
        for b in (1, 4):
            cache.pages[0, table[b][650 // 16], 0, 0, 650 % 16] = size * 1.5
        g = torch.Generator().manual_seed(i)
        q = (size * (0.5 + torch.rand((6, 2, 1), generator=g) / 4)).to(CU.DT[dtype]).expand(-1, -1, 128).contiguous().cuda()
        out = attend(cache, q, CU.ragged([1] * 6), [699] * 6, 1, share=True)
        for b in range(6):
            at = 650 if b in (1, 4) else 100
            assert torch.equal(out[b], cache.pages[0, table[b][at // 16], 1, 0, at % 16].expand(2, 128)), (size, b)
