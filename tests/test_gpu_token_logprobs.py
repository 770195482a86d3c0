"""Log-probabilities, entropy and likeliest tokens of rows of logits on the GPU against 64 bits.

Tolerance by arithmetic: a lane adds up at most vocab / 64 + 64 terms one after the other (fewer where a row is split), so that the sums
are off by no more than (vocab / 64 + 64) 2^-24 relative to sums of magnitudes; every term e^d by |d| 2^-23 + 2^-22 relative, weighted by
itself; x - m and the two last subtractions by a rounding each."""
import math

import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu


def ask(x, given, k, status=None):
    n, v = x.shape
    ws = binding.alloc_workspace(binding.radix_token_logprobs_workspace_bytes(n, v, given.shape[1] if given is not None else 0, k))
    ws.fill_(0xFF)
    return binding.radix_token_logprobs(x, given, ws, top_k=k, status=status)


def check(x, given, k):
    lp, ent, ids, tlp = (t.cpu() for t in ask(x, given, k))
    d = x.cpu().double()
    m = d.amax(1, keepdim=True)
    ref = torch.log_softmax(d, 1)
    p = ref.exp()
    spread = torch.where(p > 0, p * (d - m).abs(), 0.0).sum(1, keepdim=True)              # mean of |x - m|
    rel = (x.shape[1] / 64 + 64) * 2.0 ** -24 + 2.0 ** -22
    tol = rel + spread * 2.0 ** -23 + 2.0 ** -22

    def near(got, want, extra):
        want = want.expand_as(got)
        same = (got == want.float()) | (got.isnan() & want.isnan())          # (2^129 rounds to an infinite fp32)
        ok = same | ((got.double() - want).abs() <= tol + extra + want.abs() * 2.0 ** -22)
        assert ok.all(), (got[~ok], want[~ok])

    if given is not None:
        t = given.cpu().long()
        want = torch.where(t >= 0, ref.gather(1, t.clamp(min=0)), 0.0)
        near(lp, want, torch.where(want.isfinite(), want.abs(), 0.0) * 2.0 ** -22)
    h = -torch.where(p > 0, p * ref, 0.0).sum(1, keepdim=True)
    near(ent[:, None], h, spread * (rel + 2.0 ** -21))
    if k:
        order = torch.sort(d, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids.long(), order)
        near(tlp, ref.gather(1, order), 0.0)


def logits(seed, n, v, dtype, pad=0, scale=2.5, at=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((n, v + pad), generator=g) * scale + at).to(CU.DT[dtype]).cuda()
    return x[:, :v]


def tokens(seed, n, v, g):
    return torch.randint(0, v, (n, g), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,v", [(1, 1), (3, 2), (1, 63), (5, 257), (2, 1000), (7, 4096), (1, 8191), (3, 16385), (1, 151936), (9, 32000), (40, 50257), (300, 12289)])
def test_rows_of_many_lengths(dtype, n, v):
    k = min(5, v)
    check(logits(n + v, n, v, dtype), tokens(v, n, v, 2), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad", [1, 3, 5, 8, 100])
def test_rows_that_start_anywhere(dtype, pad):
    check(logits(pad, 6, 9000 + pad, dtype, pad), tokens(1, 6, 9000, 1), 3)
    whole = logits(pad, 6, 9000, dtype, 64)
    check(torch.as_strided(whole, (6, 8900), whole.stride(), pad), tokens(1, 6, 8900, 1), 3)       # and the first one off its line


@pytest.mark.parametrize("dtype,n,v", [("f32", 1, 3000001), ("bf16", 2, 1 << 20), ("f16", 1100, 4097)])
def test_long_rows_and_many_given_tokens(dtype, n, v):
    check(logits(v, n, v, dtype), tokens(v, n, v, 200 if n < 10 else 65), 7)


@pytest.mark.parametrize("k", [1, 2, 16, 31, 32])
@pytest.mark.parametrize("n,v", [(1, 40000), (600, 3000), (2, 33)])
def test_numbers_of_alternatives(k, n, v):
    check(logits(k, n, v, "f32"), None, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ["equal", "rising", "falling", "two values", "peaks at the ends", "zeros of both signs"])
@pytest.mark.parametrize("n,v", [(1, 20000), (700, 5003)])
def test_orders_and_ties(dtype, case, n, v):
    i = torch.arange(v, dtype=torch.float32)
    row = {"equal": torch.full((v,), 1.5), "rising": i / 700, "falling": -i / 700, "two values": (i % 7 == 3).float(),
           "peaks at the ends": torch.where((i < 3) | (i > v - 4), 9.0, 0.0), "zeros of both signs": torch.where(i % 2 == 0, -0.0, 0.0)}[case]
    x = row.expand(n, v).contiguous().to(CU.DT[dtype]).cuda()
    check(x, tokens(2, n, v, 1), 32)


def test_ruled_out_tokens():
    x = logits(1, 64, 30000, "f32")
    x[::2, torch.randperm(30000)[:29000].cuda()] = -math.inf
    x[1, :] = -math.inf
    x[1, 777] = 3.0                                                          # one token left: certain
    x[3, :] = -math.inf
    x[3, [5, 9]] = -1.0
    check(x, tokens(5, 64, 30000, 3), 2)
    lp, ent, ids, tlp = ask(x, CU.i32([[777, 778]] * 64), 4)
    assert lp[1].tolist() == [0.0, -math.inf] and ent[1].item() == 0.0
    assert ids[1].tolist() == [777, 0, 1, 2] and tlp[1].tolist() == [0.0] + [-math.inf] * 3        # then the ruled-out ones, lowest id first
    assert ids[3].tolist() == [5, 9, 0, 1] and abs(ent[3].item() - math.log(2)) < 1e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [8, 600])
@pytest.mark.parametrize("first", [False, True])
def test_tokens_masked_with_the_lowest_value_of_the_type(dtype, n, first):
    # differences of logits beyond the type's range, all at the start of a row (its first maximum is the mask's) or anywhere
    x = logits(3, n, 20000, dtype)
    low, high = torch.finfo(x.dtype).min, torch.finfo(x.dtype).max
    if first:
        x[:, :19000] = low
    else:
        x[:, torch.randperm(20000, generator=torch.Generator().manual_seed(1))[:15000].cuda()] = low
    x[1] = low                                                               # nothing but masked: all alike
    x[2] = low
    x[2, 19999] = high
    x[3, 5] = high
    check(x, tokens(5, n, 20000, 3), 4)


@pytest.mark.parametrize("n", [1, 600])
def test_rows_without_a_distribution(n):
    x = logits(1, n + 3, 9000, "f32")
    x[0] = -math.inf
    x[1, 100] = math.inf
    x[2, 100] = math.nan
    lp, ent, ids, tlp = ask(x, tokens(3, n + 3, 9000, 1), 3)
    assert lp[:3].isnan().all() and ent[:3].isnan().all() and tlp[:3].isnan().all()
    assert ids[0].tolist() == [0, 1, 2] and ids[1, 0].item() == 100
    y = x[2].clone()
    y[100] = -math.inf
    assert ids[2].tolist() == torch.sort(y, descending=True, stable=True).indices[:3].tolist()
    assert lp[3:].isfinite().all() and ent[3:].isfinite().all()


def test_a_row_of_nan_orders_its_ids():
    x = torch.full((2, 300), math.nan, device="cuda")
    x[1, 250] = -math.inf
    x[1, 40] = 1.0
    ids = ask(x, None, 4)[2].tolist()
    assert ids == [[0, 1, 2, 3], [40, 250, 0, 1]]


@pytest.mark.parametrize("at", [-3e4, 1e3, 1e6])
def test_entropy_of_rows_far_from_zero(at):
    # logits with an offset are rounded as inputs; what is asked about is the rows as they are
    check(logits(4, 5, 20000, "f32", at=at), tokens(1, 5, 20000, 1), 1)


def test_no_token_and_tokens_out_of_range():
    x = logits(1, 4, 500, "f32")
    status = CU.status_word()
    lp = ask(x, CU.i32([[-1, 3], [499, -7], [0, 0], [2, 2]]), 0, status)[0]
    assert lp[0, 0] == 0 and lp[1, 1] == 0 and int(status) == 0 and (lp[2:] < 0).all()
    lp = ask(x, CU.i32([[1], [500], [2], [2147483647]]), 0, status)[0]
    assert int(status) == -7 and lp[1].isnan() and lp[3].isnan() and lp[0].isfinite()


def test_rows_beyond_32_bits():
    whole = torch.empty((2 << 30) + 70000, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(whole, (3, 60001), (1 << 30, 1), 3)
    x.copy_(torch.randn((3, 60001), device="cuda") * 3)
    check(x, tokens(1, 3, 60001, 2), 4)


def test_entropy_alone_and_nothing_at_all():
    x = logits(1, 4, 500, "f32")
    lp, ent, ids, tlp = ask(x, None, 0)
    assert lp.shape == (4, 0) and ids.shape == (4, 0) and ent.isfinite().all()
    assert ask(x[:0], None, 2)[2].shape == (0, 2)


def test_replays_from_a_graph():
    x, given = logits(1, 3, 40000, "bf16"), tokens(1, 3, 40000, 1)
    ws = binding.alloc_workspace(binding.radix_token_logprobs_workspace_bytes(3, 40000, 1, 4))
    want = [t.clone() for t in binding.radix_token_logprobs(x, given, ws, top_k=4)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = binding.radix_token_logprobs(x, given, ws, top_k=4)
    for i in range(3):
        for t in got:
            t.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
