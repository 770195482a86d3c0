"""Calls on another stream than the current one do not write into memory that tensors of the current stream have just left: its kernels
may not be done with it."""
import pytest
import torch

from paper_2601_15013_amd import binding, harness, synth
from tests import cache_util as CU

pytestmark = pytest.mark.gpu

CFG = synth.ModelConfig("f32s", 1, 256, 4, 2, 64, 768, 1000, "f32", max_pos=512)


@pytest.fixture(scope="module")
def have():
    model = harness.upload_model(synth.SynthWeights(CFG, 3), lm_head_mode=1)
    cache = binding.alloc_cache(1, 2, 64, 16, 40, torch.float32, 3, 8)
    ws = binding.alloc_workspace(1 << 26)
    yield model, cache, ws
    model.close()


def outputs(x):
    return x if isinstance(x, tuple) else (x,)


def calls(m, c, ws):
    """name -> call on a stream, inputs made."""
    cu, past, given = CU.i32([0, 7]), CU.i32([-1]), CU.i32([[1]] * 9)
    q, x, hidden = (torch.zeros(shape, device="cuda") for shape in ((7, 4, 64), (9, 500), (9, CFG.d)))
    none, tok, nowhere, zeros = CU.i32([0, 0, 0]), CU.i32([1] * 7), CU.i32([7]), CU.i32([0] * 3)
    maps = binding.radix_build_index(tok, None, cu, ws)
    return {"extend": lambda s: binding.radix_cache_extend(c, none, ws, stream=s),
            "compact": lambda s: binding.radix_cache_compact(c, ws, stream=s),
            "attention": lambda s: binding.radix_paged_attention(c, 0, q, cu, past, 7, ws, stream=s),
            "extend_forward": lambda s: binding.radix_extend_forward(m, c, tok, cu, 7, ws, slots=nowhere, stream=s),
            "token_logprobs": lambda s: binding.radix_token_logprobs(x, given, ws, top_k=3, stream=s),
            "build_index": lambda s: binding.radix_build_index(tok, None, cu, ws, stream=s)[:3],
            "prefill": lambda s: binding.radix_prefill_forward(m, tok, None, cu, 7, *maps[:2], maps[3], ws, stream=s),
            "prefill_nodedup": lambda s: binding.radix_prefill_forward_nodedup(m, tok, None, cu, 7, ws, stream=s),
            "lm_head": lambda s: binding.radix_lm_head(m, hidden, None, ws, stream=s),
            "select_rows": lambda s: binding.radix_index_select_rows(x, zeros, stream=s),
            "score_tokens": lambda s: binding.radix_score_tokens(m, hidden, None, given, ws, top_k=3, stream=s)}


@pytest.mark.parametrize("name", ["extend", "compact", "attention", "extend_forward", "token_logprobs", "score_tokens", "build_index", "prefill",
                                  "prefill_nodedup", "lm_head", "select_rows"])
def test_memory_that_the_current_stream_left_is_not_written(have, name):
    call, side = calls(*have)[name], torch.cuda.Stream()
    shapes = [(t.shape, t.dtype) for t in outputs(call(None))]
    torch.cuda.synchronize()
    left = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(8)]
    places = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in left]
    del left
    side.wait_stream(torch.cuda.current_stream())
    got = outputs(call(side))
    torch.cuda.synchronize()
    for t in got:
        assert all(t.data_ptr() >= end or t.data_ptr() + t.numel() * t.element_size() <= begin for begin, end in places)
