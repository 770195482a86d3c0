"""Attention of new tokens over a paged cache on the GPU against softmax in 64 bits, with tolerances that count the roundings."""
import math
import random

import pytest
import torch

from paper_2601_15013_amd import binding
from tests import cache_util as CU

pytestmark = pytest.mark.gpu

BAD_CU, BAD_PAGE, BAD_SLOT = -6, -11, -13


def attend(cache, q, cu, past, max_new, slots=None, layer=0, status=None, out=None, stream=None, share=False):
    B = len(cu) - 1
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, q.shape[1], q.shape[0], B, max_new, share))
    ws.fill_(0xFF)                                          # NaN and -1 everywhere: nothing of it may be relied on
    return binding.radix_paged_attention(cache, layer, q, CU.i32(cu), CU.i32(past), max_new, ws, slots=None if slots is None else CU.i32(slots),
                                         status=status, out=out, stream=stream, find_shared=share)


def queries(seed, N, hq, hd, dtype, fused_with=0):
    g = torch.Generator().manual_seed(seed)
    row = torch.randn((N, (hq + fused_with) * hd), generator=g).to(CU.DT[dtype]).cuda()
    return row[:, :hq * hd].view(N, hq, hd)


def check(past, news, hq, kv, hd, page, dtype, seed=1, fused_with=0, layers=1, max_new=None):
    lens = [p + n for p, n in zip(past, news)]
    cache = CU.random_cache(seed, lens, kv, hd, page, dtype, layers=layers, poison=True)
    cu = CU.ragged(news)
    q = queries(seed + 1, cu[-1], hq, hd, dtype, fused_with)
    status = CU.status_word()
    o = attend(cache, q, cu, past, max_new or max(news), layer=layers - 1, status=status).cpu().double()
    assert int(status) == 0
    ref, a = CU.attention_ref(cache, layers - 1, q, cu, past)
    tol = CU.attention_tolerance(dtype, ref, a, hd, max(lens))
    err = (o - ref).abs()
    worst = (err / tol).max().item() if err.numel() else 0.0
    assert torch.isfinite(o).all() and worst <= 1.0, f"worst error is {worst:.2f} of what arithmetic allows"


TYPES_16 = ["bf16", "f16"]


@pytest.mark.parametrize("dtype", TYPES_16)
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("hq,kv", [(8, 8), (8, 2), (5, 1), (12, 4), (16, 1)])
def test_single_tokens_over_ragged_lengths(dtype, page, hq, kv):
    check([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 700], [1] * 14, hq, kv, 128, page, dtype)


@pytest.mark.parametrize("dtype", TYPES_16)
@pytest.mark.parametrize("hq,kv,news", [(8, 2, [4, 3, 1, 2]), (32, 4, [4, 4, 1, 3]), (24, 1, [1, 1, 1, 1]), (5, 5, [16, 9, 1, 15]), (5, 5, [17, 32, 31, 1])])
def test_a_few_tokens_at_a_time(dtype, hq, kv, news):
    check([0, 30, 129, 517], news, hq, kv, 128, 32, dtype)


@pytest.mark.parametrize("dtype", TYPES_16)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,kv", [(4, 4), (8, 2), (6, 2), (7, 1), (16, 2)])
def test_chunks_behind_a_cached_prefix(dtype, page, hq, kv):
    check([0, 0, 5, 64, 100, 257], [70, 129, 64, 33, 1, 200], hq, kv, 128, page, dtype, fused_with=2)


@pytest.mark.parametrize("dtype", TYPES_16)
def test_chunks_and_single_tokens_in_one_batch(dtype):
    check([900, 0, 64, 2, 0, 333, 70], [1, 150, 1, 40, 0, 1, 2], 8, 2, 128, 32, dtype, layers=2)


@pytest.mark.parametrize("hd", [4, 32, 64, 68, 80, 128])
@pytest.mark.parametrize("hq,kv,page", [(4, 2, 16), (6, 1, 64), (3, 3, 256)])
def test_fp32(hd, hq, kv, page):
    check([0, 3, 16, 200, 0, 50], [1, 1, 20, 37, 0, 5], hq, kv, hd, page, "f32", fused_with=1)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 128), ("f32", 64)])
def test_one_long_sequence_is_split_over_the_chip(dtype, hd):
    check([9000], [1], 4, 1, hd, 64, dtype)


@pytest.mark.parametrize("dtype", TYPES_16)
def test_a_chunk_behind_a_long_prefix_is_split(dtype):
    check([5000, 100], [40, 33], 4, 1, 128, 16, dtype)


def test_a_bound_on_new_tokens_that_is_not_reached_changes_the_kernel_only():
    check([100, 40, 7], [1, 1, 1], 8, 2, 128, 16, "f16", max_new=500)


def test_large_scores_and_rows_without_weight():
    # scores of +-1e4: one key takes everything; and keys of -inf
    cache = CU.random_cache(3, [70, 70], 1, 128, 16, "bf16", scale=20.0)
    q = queries(4, 2, 2, 128, "bf16") * 20
    cu, past = [0, 1, 2], [69, 69]
    o = attend(cache, q, cu, past, 1).cpu().double()
    ref, a = CU.attention_ref(cache, 0, q, cu, past)
    # a score of s is off by 2^-24 * 132 * |q||k| / sqrt(hd) <= 0.4 here, so only rows whose best key leads by 20 are compared
    for b in range(2):
        k = CU.rows_of(cache, 0, b, 70, 0)[:, 0]
        for h in range(2):
            s = (k @ q[b, h].cpu().double()) / 128 ** 0.5
            top = torch.topk(s, 2).values
            if top[0] - top[1] > 20:
                v = CU.rows_of(cache, 0, b, 70, 1)[s.argmax(), 0]
                assert torch.allclose(o[b, h], v, rtol=2 ** -7, atol=1e-5)
    assert torch.isfinite(o).all()


def test_keys_that_are_masked_may_hold_anything():
    # infinities and NaN among the later tokens' keys reach nothing; scores of -inf are no part of a row
    cache = CU.random_cache(9, [90], 1, 128, 16, "f16")
    page, slot = cache.page_table[0, 85 // 16].item(), 85 % 16
    q = queries(2, 40, 2, 128, "f16")
    clean = attend(cache, q, [0, 40], [50], 40).clone()
    cache.pages[0, page, 0, 0, slot] = float("nan")                          # key of position 85: token 35 and later see it
    out = attend(cache, q, [0, 40], [50], 40)
    assert torch.equal(out[:35], clean[:35])
    assert torch.isnan(out[35:]).all()


@pytest.mark.parametrize("dtype,hd,n", [("bf16", 128, 1), ("f16", 128, 40), ("f32", 32, 2)])
@pytest.mark.parametrize("long", [60, 3000])
def test_rows_whose_scores_are_all_infinitely_low(dtype, hd, n, long):
    # keys of -inf under positive queries leave a row nothing: zeros; one finite key takes all the weight
    cache = CU.random_cache(9, [long + n, long + n], 1, hd, 16, dtype)
    finite = cache.pages[:, cache.page_table[1, 1].item(), 0, :, 5].clone()
    cache.pages[:, :, 0] = -math.inf
    cache.pages[:, cache.page_table[1, 1].item(), 0, :, 5] = finite
    q = queries(2, 2 * n, 2, hd, dtype).abs() + 0.1
    out = attend(cache, q, [0, n, 2 * n], [long, long], n)
    v = cache.pages[0, cache.page_table[1, 1].item(), 1, 0, 5]
    assert (out[:n] == 0).all() and torch.equal(out[n:], v.expand_as(out[n:]))


def test_sequences_without_a_place_give_zeros_and_rows_behind_the_last_stay():
    cache = CU.random_cache(5, [40, 40, 40], 2, 128, 16, "bf16")
    q = queries(6, 9, 4, 128, "bf16")
    status = CU.status_word()
    out = torch.full_like(q, 7.0)
    attend(cache, q, [0, 2, 5, 7], [38, -1, 30], 3, out=out, status=status)
    assert int(status) == 0 and (out[7:] == 7).all() and (out[2:5] == 0).all()
    ref, a = CU.attention_ref(cache, 0, q[:7], [0, 2, 5, 7], [38, -1, 30])
    assert ((out[:7].cpu().double() - ref).abs() <= CU.attention_tolerance("bf16", ref, a, 128, 40)).all()


@pytest.mark.parametrize("max_new", [1, 60])
@pytest.mark.parametrize("cu,past,slots,code,zeros", [([0, 1, 2], [39, 39], [0, 3], BAD_SLOT, [1]), ([0, 1, 2], [1000, 39], [0, 1], BAD_PAGE, [0]),
                                                      ([0, 1, 2], [2147483647, 39], [0, 1], BAD_PAGE, [0]),
                                                      ([0, 1, 9], [39, 20], [0, 1], BAD_CU, []), ([-1, 1, 2], [39, 39], [0, 1], BAD_CU, [])])
def test_what_cannot_be_is_reported(cu, past, slots, code, zeros, max_new):
    cache = CU.random_cache(5, [40, 40, 40], 2, 128, 16, "bf16")
    q = queries(6, 4, 4, 128, "bf16")
    status, out = CU.status_word(), torch.full_like(queries(6, 4, 4, 128, "bf16"), 7.0)
    attend(cache, q, cu, past, max_new, slots=slots, status=status, out=out)
    assert int(status) == code
    for i in zeros:
        assert (out[i] == 0).all()
    assert (out[2:] == 7).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 60), ("f32", 3)])
def test_an_entry_that_is_no_page_is_read_as_page_0_and_reported(dtype, n):
    cache = CU.random_cache(5, [80], 1, 128, 16, dtype)
    q = queries(6, n, 2, 128, dtype)
    for bad in (-1, cache.pages.shape[1], 2147483647):
        cache.page_table[0, 1] = bad
        status = CU.status_word()
        out = attend(cache, q, [0, n], [80 - n], n, status=status)
        assert int(status) == BAD_PAGE
        cache.page_table[0, 1] = 0
        assert torch.equal(out, attend(cache, q, [0, n], [80 - n], n))


def test_slots_shared_pages_and_the_same_slot_twice():
    cache = CU.random_cache(8, [300, 64], 2, 128, 64, "f16")
    cache.page_table[1, 0] = cache.page_table[0, 0]                          # a shared page
    q = queries(9, 4, 4, 128, "f16")
    cu, past, slots = [0, 1, 3, 4], [299, 62, 200], [0, 1, 0]
    out = attend(cache, q, cu, past, 2, slots=slots).cpu().double()
    ref, a = CU.attention_ref(cache, 0, q, cu, past, slots)
    assert ((out - ref).abs() <= CU.attention_tolerance("f16", ref, a, 128, 300)).all()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
def test_many_sequences(dtype, hd):
    rng = random.Random(4)
    news = [rng.choice([0, 1, 1, 1, 2, 40]) for _ in range(300)]
    past = [rng.randint(0, 90) for _ in news]
    check(past, news, 2, 1, hd, 16, dtype)


@pytest.mark.parametrize("B", [63, 64, 65, 128, 200, 256, 257])
@pytest.mark.parametrize("dtype,most", [("bf16", 1), ("bf16", 100), ("f32", 3)])
def test_numbers_of_sequences_around_the_plan(B, dtype, most):
    # a few long ones, which are split, anywhere among short and empty ones
    rng = random.Random(B)
    news = [rng.choice([0, 1, 1, most]) for _ in range(B)]
    past = [rng.choice([0, 3, 20, 20, 20, 900 if rng.random() < 0.2 else 40]) for _ in news]
    past[-1], news[-1] = 1500, 1
    past[B // 2], news[B // 2] = 2500, most
    check(past, news, 4, 2, 128 if dtype != "f32" else 32, 32, dtype)


def forks(seed, past, news, groups, kv, hd, page, dtype):
    """A cache in which the sequences of every (first, count, pages) group begin with the first one's pages."""
    cache = CU.random_cache(seed, [p + n for p, n in zip(past, news)], kv, hd, page, dtype, poison=True)
    for first, count, pages in groups:
        cache.page_table[first + 1:first + count, :pages] = cache.page_table[first, :pages]
    return cache


def check_forks(past, news, groups, hq, kv, hd, page, dtype, slots=None, max_new=None):
    cache = forks(3, past, news, groups, kv, hd, page, dtype)
    cu = CU.ragged(news)
    q = queries(4, cu[-1], hq, hd, dtype)
    status = CU.status_word()
    o = attend(cache, q, cu, past, max_new or max(news), status=status, share=True).cpu().double()
    assert int(status) == 0
    ref, a = CU.attention_ref(cache, 0, q, cu, past)
    tol = CU.attention_tolerance(dtype, ref, a, hd, max(p + n for p, n in zip(past, news)))
    worst = ((o - ref).abs() / tol).max().item()
    assert torch.isfinite(o).all() and worst <= 1.0, f"worst error is {worst:.2f} of what arithmetic allows"


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("hq,kv", [(4, 4), (8, 2), (3, 1), (8, 1), (9, 1)])
def test_neighbours_that_begin_with_the_same_pages(dtype, hd, page, hq, kv):
    # 1280 common keys (two, then nine sequences: more than a block), 512, 256 (the least), 240 (too few); one apart in between
    past = [1300, 1281, 600, 1400, 1290, 1280, 1283, 1300, 1500, 1281, 1282, 1290, 520, 513, 700, 260, 256, 257, 250, 249]
    news = [1] * len(past)
    groups = [(0, 2, 1280 // page), (3, 9, 1280 // page), (12, 3, 512 // page), (15, 3, 256 // page)]
    if page == 16:
        groups.append((18, 2, 15))
    check_forks(past, news, groups, hq, kv, hd, page, dtype)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 32)])
def test_forks_with_several_new_tokens_of_different_number(dtype, hd):
    past = [700, 690, 800, 640, 900, 901, 902, 903, 904, 905]
    news = [2, 2, 3, 3, 1, 1, 4, 4, 4, 9]
    check_forks(past, news, [(0, 10, 40)], 2, 1, hd, 16, dtype)
    check_forks(past, news, [(0, 10, 40)], 4, 2, hd, 16, dtype)


@pytest.mark.parametrize("dtype", TYPES_16)
def test_forks_beside_chunks(dtype):
    past = [2000, 2001, 2002, 100, 0, 2100, 2200, 2300, 2301, 2302]
    news = [1, 1, 1, 90, 200, 1, 1, 1, 1, 1]
    check_forks(past, news, [(0, 3, 60), (5, 5, 60)], 8, 2, 128, 32, dtype)


@pytest.mark.parametrize("B", [2, 65, 300, 1030])
def test_many_forks_of_a_few_prompts(B):
    rng = random.Random(B)
    past, groups, b = [], [], 0
    while b < B:
        n = min(B - b, rng.choice([1, 2, 3, 7, 40]))
        pages = rng.choice([16, 17, 30])
        past += [16 * pages + rng.randint(0, 40) for _ in range(n)]
        groups.append((b, n, pages))
        b += n
    check_forks(past, [1] * B, groups, 4, 2, 128, 16, "bf16")


def test_a_long_common_prefix_is_split_and_so_is_the_rest():
    check_forks([9000, 12000, 8200, 8192], [1] * 4, [(0, 4, 128)], 4, 1, 128, 64, "f16")


def test_forks_that_are_not_cached_or_out_of_range():
    # a sequence without a place, a slot out of range and a bad row range between the others
    cache = forks(3, [600] * 5, [1] * 5, [(0, 5, 30)], 2, 128, 16, "bf16")
    q = queries(4, 5, 4, 128, "bf16")
    status, out = CU.status_word(), torch.full_like(queries(4, 5, 4, 128, "bf16"), 7.0)
    attend(cache, q, [0, 1, 2, 3, 4, 5], [600, -1, 600, 600, 600], 1, slots=[0, 1, 2, 9, 4], status=status, out=out, share=True)
    assert int(status) == BAD_SLOT and (out[1] == 0).all() and (out[3] == 0).all()
    ref, a = CU.attention_ref(cache, 0, q, [0, 1, 2, 3, 4, 5], [600, -1, 600, -1, 600], [0, 1, 2, 3, 4])
    assert ((out.cpu().double() - ref).abs() <= CU.attention_tolerance("bf16", ref, a, 128, 601)).all()
    status.zero_()
    out.fill_(7.0)
    attend(cache, q, [0, 1, 2, 2, 9, 5], [600] * 5, 1, status=status, out=out, share=True)
    assert int(status) == BAD_CU and torch.isfinite(out).all() and (out[2:] == 7).all()


def test_the_same_slot_many_times_and_a_bad_entry_in_the_common_part():
    cache = CU.random_cache(8, [700], 2, 128, 16, "f16")
    q = queries(9, 6, 4, 128, "f16")
    cu, past, slots = [0, 1, 2, 3, 4, 5, 6], [699, 698, 600, 699, 500, 300], [0] * 6
    out = attend(cache, q, cu, past, 1, slots=slots, share=True)
    ref, a = CU.attention_ref(cache, 0, q, cu, past, slots)
    assert ((out.cpu().double() - ref).abs() <= CU.attention_tolerance("f16", ref, a, 128, 700)).all()
    cache.page_table[0, 5] = -1
    status = CU.status_word()
    out = attend(cache, q, cu, past, 1, slots=slots, share=True, status=status)
    assert int(status) == BAD_PAGE
    cache.page_table[0, 5] = 0
    assert torch.equal(out, attend(cache, q, cu, past, 1, slots=slots, share=True))


def test_results_do_not_depend_on_the_run():
    cache = CU.random_cache(5, [4000, 900, 30], 2, 128, 32, "bf16")
    q = queries(6, 3, 8, 128, "bf16")
    first = attend(cache, q, [0, 1, 2, 3], [3999, 899, 29], 1)
    for _ in range(3):
        assert torch.equal(attend(cache, q, [0, 1, 2, 3], [3999, 899, 29], 1), first)


@pytest.mark.parametrize("n", [1, 50])
def test_replays_of_two_graphs_that_share_a_workspace(n):
    cache = CU.random_cache(5, [2000, 300], 2, 128, 32, "bf16")
    qs = [queries(s, 2 * n, 4, 128, "bf16") for s in (1, 2)]
    cu, past = CU.i32([0, n, 2 * n]), CU.i32([2000 - n, 300 - n])
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, 4, 2 * n, 2, n))
    outs = [torch.empty_like(q) for q in qs]
    want = [binding.radix_paged_attention(cache, 0, q, cu, past, n, ws).clone() for q in qs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for q, o in zip(qs, outs):
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            binding.radix_paged_attention(cache, 0, q, cu, past, n, ws, out=o)
        graphs.append(graph)
    for i in range(4):
        for o in outs:
            o.fill_(float(i))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_offsets_beyond_32_bits():
    # one layer of 4.5 GB: pages behind the first 2^32 bytes, 2^31 elements
    page, n_pages = 256, 35000
    pages = torch.empty((1, n_pages, 2, 1, page, 128), dtype=torch.bfloat16, device="cuda")
    assert pages.numel() * 2 > 1 << 32
    cache = binding.Cache(pages, torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
                          CU.i32([[n_pages - 1, n_pages - 2, 3], [n_pages // 2, n_pages - 3, 1]]), CU.i32([0, 0]))
    for p in (n_pages - 1, n_pages - 2, n_pages // 2, n_pages - 3):
        pages[0, p].copy_(torch.randn(pages[0, p].shape, device="cuda"))
    past, news = [300, 200], [1, 64]
    k, v = (torch.randn((65, 1, 128), device="cuda").bfloat16() for _ in range(2))
    binding.radix_cache_append(cache, 0, k, v, CU.i32(CU.ragged(news)), CU.i32(past))
    assert torch.equal(pages[0, n_pages - 2, 0, 0, 300 - 256], k[0, 0]) and torch.equal(pages[0, n_pages - 3, 1, 0, 7], v[64, 0])
    q = queries(1, 65, 2, 128, "bf16")
    out = attend(cache, q, CU.ragged(news), past, 64).cpu().double()
    few = {n: cache.pages[:, list(n)] for n in [(n_pages - 1, n_pages - 2, n_pages // 2, n_pages - 3)]}
    small = binding.Cache(next(iter(few.values())).contiguous(), CU.i32([0] * 4), CU.i32([[0, 1], [2, 3]]), CU.i32([0, 0]))
    ref, a = CU.attention_ref(small, 0, q, CU.ragged(news), past)
    assert ((out - ref).abs() <= CU.attention_tolerance("bf16", ref, a, 128, 301)).all()


@pytest.mark.parametrize("hq,kv", [(33, 1), (64, 1), (128, 2)])
def test_groups_of_more_than_32_heads(hq, kv):
    check([0, 700, 64, 3], [1, 1, 2, 5], hq, kv, 128, 32, "bf16")
    check([0, 700, 64, 3], [1, 1, 1, 1], hq, kv, 128, 32, "f16")


@pytest.mark.parametrize("dtype,hd,n", [("bf16", 128, 1), ("f16", 128, 70), ("f32", 20, 3)])
@pytest.mark.parametrize("long", [100, 3000])
def test_strided_outputs_leave_what_lies_between(dtype, hd, n, long):
    cache = CU.random_cache(5, [long + n, 40 + n], 2, hd, 16, dtype)
    q = queries(6, 2 * n, 6, hd, dtype, fused_with=3)
    rows = torch.full((2 * n, 8 * hd), 7.0, dtype=q.dtype, device="cuda")
    out = rows[:, hd:7 * hd].view(2 * n, 6, hd)
    want = attend(cache, q, [0, n, 2 * n], [long, 40], n)
    attend(cache, q, [0, n, 2 * n], [long, 40], n, out=out)
    assert torch.equal(out, want) and (rows[:, :hd] == 7).all() and (rows[:, 7 * hd:] == 7).all()


@pytest.mark.parametrize("share", [False, True])
def test_65535_sequences_most_of_them_empty(share):
    B, live = 65535, [0, 1, 2, 700, 701, 40000, 65533, 65534]
    cache = CU.random_cache(5, [300] * len(live), 2, 128, 16, "bf16")
    news, slots = [0] * B, [-5] * B                                          # a slot that nobody asks for is not looked at
    for i, b in enumerate(live):
        news[b], slots[b] = 1, i
    q = queries(6, len(live), 4, 128, "bf16")
    status = CU.status_word()
    out = attend(cache, q, CU.ragged(news), [299] * B, 1, slots=slots, status=status, share=share)
    assert int(status) == 0 and torch.equal(out, attend(cache, q, list(range(len(live) + 1)), [299] * len(live), 1))


def test_two_calls_at_once_and_a_replayed_search():
    cache = forks(3, [700] * 8, [1] * 8, [(0, 8, 40)], 2, 128, 16, "bf16")
    qs = [queries(s, 8, 4, 128, "bf16") for s in (1, 2)]
    cu, past = CU.i32(list(range(9))), CU.i32([700] * 8)
    wss = [binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, 4, 8, 8, 1, True)) for _ in qs]
    want = [binding.radix_paged_attention(cache, 0, q, cu, past, 1, ws, find_shared=True) for q, ws in zip(qs, wss)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(5):
        got = [binding.radix_paged_attention(cache, 0, q, cu, past, 1, ws, stream=s, find_shared=True) for q, ws, s in zip(qs, wss, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want[0])
    streams[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(streams[0]), torch.cuda.graph(graph, stream=streams[0]):
        binding.radix_paged_attention(cache, 0, qs[0], cu, past, 1, wss[0], out=out, find_shared=True)
    for i in range(3):
        out.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])
    # the sequences grow, and one of them leaves the others, between replays
    cache.page_table[3, 0] = cache.page_table[3, 41]
    past.copy_(CU.i32([690, 700, 640, 650, 660, 700, 700, 655]))
    graph.replay()
    torch.cuda.synchronize()
    ref, a = CU.attention_ref(cache, 0, qs[0], list(range(9)), past.tolist())
    assert ((out.cpu().double() - ref).abs() <= CU.attention_tolerance("bf16", ref, a, 128, 701)).all()


def test_a_stream_of_its_own():
    cache = CU.random_cache(5, [500], 2, 128, 32, "bf16")
    q = queries(6, 1, 4, 128, "bf16")
    want = attend(cache, q, [0, 1], [499], 1)
    ws = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(cache, 4, 1, 1, 1))
    cu, past, out = CU.i32([0, 1]), CU.i32([499]), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.radix_paged_attention(cache, 0, q, cu, past, 1, ws, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
