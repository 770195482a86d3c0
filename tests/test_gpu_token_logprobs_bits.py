"""How a row of logits is summed depends on the number of rows, the vocabulary, the type and the row's address modulo 16, and on nothing
else: equal rows have equal results, bit for bit, wherever they stand in the call."""
import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,v", [(40, 20011), (1100, 5003)])                 # rows in several workgroups, and in one
@pytest.mark.parametrize("pad", [5, 1, 2, 4])                                # with 5, fp32 rows begin on 16-byte borders
def test_equal_rows_have_equal_bits(dtype, n, v, pad):
    g = torch.Generator().manual_seed(n)
    row = (torch.randn(v, generator=g) * 3).to(CU.DT[dtype]).cuda()
    whole = torch.zeros((n, v + pad), dtype=CU.DT[dtype], device="cuda")
    x = whole[:, :v]
    x.copy_(row.expand(n, v))
    given = torch.full((n, 1), 77, dtype=torch.int32, device="cuda")
    ws = binding.alloc_workspace(binding.radix_token_logprobs_workspace_bytes(n, v, 1, 3))
    out = binding.radix_token_logprobs(x, given, ws, top_k=3)
    period = 16 // whole.element_size()                                      # rows whose addresses agree modulo 16
    for t in out:
        for r in range(period):
            same = t[r::period].view(torch.int32)
            assert torch.equal(same, same[:1].expand_as(same))
