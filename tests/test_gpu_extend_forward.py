"""Forwards over a cache, as they are used: prompts in chunks, prefixes shared by forks, generation token by token - against the fp64
oracle's forward of whole sequences, with the tolerances of the plain forward (1e-4 with fp32 weights, 2e-2 with bf16 weights)."""
import numpy as np
import pytest
import torch

from oracle import forward as oracle_forward
from paper_2601_15013_amd import binding, harness, synth
from tests import cache_util as CU
from tests import gpu_util as U
from tests.test_gpu_forward import SMALL_BF16, TOL_BF16, TOL_F32

pytestmark = pytest.mark.gpu

F32 = synth.ModelConfig("f32s", 2, 256, 4, 2, 64, 768, 1000, "f32", max_pos=512)
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Live:
    """A model, a cache and the tokens that went into every slot."""

    def __init__(self, cfg, seed, page, n_pages=80, slots=8, max_pages=24, **kw):
        self.cfg, self.w = cfg, synth.SynthWeights(cfg, seed)
        self.model = harness.upload_model(self.w, **kw)
        self.cache = binding.alloc_cache(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, page, n_pages, TYPES[self.model.compute_dtype], slots, max_pages)
        self.cache.pages.fill_(float("nan"))                                 # a row that no token wrote must reach nothing
        self.tokens = {s: [] for s in range(slots)}
        self.tol = TOL_F32 if cfg.dtype == "f32" else TOL_BF16
        self.page_ws = binding.alloc_workspace(binding.radix_cache_workspace_bytes(self.cache, slots))

    def step(self, new, ws=None):
        """new: {slot: tokens}; returns the hidden states, after checking them against the oracle."""
        slots, lens = list(new), [len(t) for t in new.values()]
        tok = np.concatenate([np.asarray(t, dtype=np.int32) for t in new.values()])
        if ws is None:
            ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(self.model, self.cache, len(tok), len(slots), max(lens)))
            ws.fill_(0xFF)
        y = binding.radix_extend_forward(self.model, self.cache, torch.from_numpy(tok).cuda(), CU.i32(CU.ragged(lens)), max(lens), ws,
                                         slots=CU.i32(slots))
        assert binding.radix_device_status(ws) == 0
        for s, t in new.items():
            self.tokens[s] += list(t)
        full = [np.asarray(self.tokens[s], dtype=np.int32) for s in slots]
        cu = np.asarray(CU.ragged([len(t) for t in full]), dtype=np.int32)
        ref = oracle_forward.forward_nodedup(self.cfg, self.w.embed, self.w.layers, self.w.gf, np.concatenate(full), cu)
        want = np.concatenate([ref[cu[b + 1] - n:cu[b + 1]] for b, n in enumerate(lens)])
        err = U.rel_err(y.cpu().numpy(), want)
        assert err <= self.tol, err
        return y

    def fork(self, parents, children):
        binding.radix_cache_fork(self.cache, CU.i32(parents), CU.i32(children), self.page_ws)
        for p, c in zip(parents, children):
            self.tokens[c] = list(self.tokens[p])

    def cut(self, slots, keep):
        binding.radix_cache_free(self.cache, CU.i32(slots), keep_lens=CU.i32(keep))
        for s, k in zip(slots, keep):
            self.tokens[s] = self.tokens[s][:k]


def words(rng, cfg, n):
    return rng.integers(0, cfg.vocab, n).tolist()


VARIANTS = [(F32, 16, {}), (F32, 64, {}), (SMALL_BF16, 16, {}), (SMALL_BF16, 64, dict(hilo_layers=1)),
            (SMALL_BF16, 32, dict(hilo_layers=-1, fold_norms=1))]


@pytest.mark.parametrize("cfg,page,kw", VARIANTS)
def test_prompts_in_chunks_forks_and_steps_back(cfg, page, kw):
    live, rng = Live(cfg, 71, page, **kw), np.random.default_rng(page)
    live.step({0: words(rng, cfg, 70), 3: words(rng, cfg, 1)})               # two prompts begin
    live.step({0: words(rng, cfg, 37), 3: words(rng, cfg, 90), 5: words(rng, cfg, 3)})
    live.step({5: words(rng, cfg, 1), 0: words(rng, cfg, 1), 3: words(rng, cfg, 1)})
    live.fork([0, 0, 3], [1, 2, 4])
    live.step({1: words(rng, cfg, 5), 2: words(rng, cfg, 40), 4: words(rng, cfg, 1), 0: words(rng, cfg, 1)})
    live.cut([2, 1], [50, 3])                                                # into pages that are shared
    live.step({2: words(rng, cfg, 30), 1: words(rng, cfg, 2), 0: words(rng, cfg, 2), 4: words(rng, cfg, 2)})
    binding.radix_cache_free(live.cache, CU.i32([0]))
    live.tokens[0] = []
    binding.radix_cache_compact(live.cache, live.page_ws)
    live.step({s: words(rng, cfg, 1) for s in (1, 2, 3, 4, 5)})
    live.step({0: words(rng, cfg, 20), 4: words(rng, cfg, 1)})
    live.model.close()


@pytest.mark.parametrize("cfg", [F32, SMALL_BF16])
def test_one_workspace_for_steps_of_all_sizes(cfg):
    live, rng = Live(cfg, 79, 16), np.random.default_rng(6)
    ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(live.model, live.cache, 200, 8, 120))
    for news in [{0: 90, 1: 1, 2: 0, 3: 33}, {0: 1, 1: 0, 2: 1, 3: 1}, {5: 0, 0: 8, 3: 5}, {0: 1}, {2: 120, 0: 1}, {6: 2, 7: 2}]:
        live.step({s: words(rng, cfg, n) for s, n in news.items()}, ws)
    live.model.close()


def test_workspaces_for_larger_bounds_hold_any_smaller_call():
    live = Live(synth.ModelConfig("gen", 3, 256, 4, 2, 128, 320, 2048, "bf16", max_pos=1024), 80, 16, lm_head_mode=1)
    last = []
    for B in (1, 20, 128, 700):
        for N in (1, 128, 1024, 5000):
            sizes = [binding.radix_extend_workspace_bytes(live.model, live.cache, N, B, new) for new in (1, 2, 4, 8, 16, 17, 64, 4000)]
            assert sizes == sorted(sizes)
            assert all(x <= y for b, n, small in last if b <= B and n <= N for x, y in zip(small, sizes))
            last.append((B, N, sizes))
    for k in (0, 1, 32):
        sizes = [binding.radix_score_tokens_workspace_bytes(live.model, n, 1, k) for n in (0, 1, 2, 15, 16, 17, 500, 512, 513, 9000)]
        assert sizes == sorted(sizes)
    live.model.close()


def test_the_first_step_is_the_plain_forward():
    # with nothing cached it is the same forward, up to the attention's order of sums
    live, rng = Live(SMALL_BF16, 72, 64, hilo_layers=-1), np.random.default_rng(1)
    news = {0: words(rng, SMALL_BF16, 130), 1: words(rng, SMALL_BF16, 1), 2: words(rng, SMALL_BF16, 77)}
    y = live.step(news)
    tok = torch.tensor(sum(news.values(), []), dtype=torch.int32).cuda()
    cu = CU.i32(CU.ragged([len(t) for t in news.values()]))
    ws = binding.alloc_workspace(binding.radix_workspace_bytes(live.model, tok.numel(), 3))
    plain = binding.radix_prefill_forward_nodedup(live.model, tok, None, cu, 130, ws)
    assert U.rel_err(y.cpu().numpy(), plain.cpu().numpy().astype(np.float64)) <= TOL_BF16 / 4
    live.model.close()


@pytest.mark.parametrize("cfg,lm_head_mode", [(F32, 1), (synth.ModelConfig("gen", 3, 256, 4, 2, 128, 320, 2048, "bf16", max_pos=1024), 1)])
def test_generation_from_forks_of_one_prompt(cfg, lm_head_mode):
    """The whole path: a prompt once, forks of it, greedy continuation by the likeliest token, its probability against the oracle's."""
    live, rng = Live(cfg, 73, 16, lm_head_mode=lm_head_mode), np.random.default_rng(5)
    live.step({0: words(rng, cfg, 45)})
    live.fork([0, 0], [1, 2])
    new = {0: words(rng, cfg, 1), 1: words(rng, cfg, 6), 2: words(rng, cfg, 1)}
    ws = binding.alloc_workspace(binding.radix_score_tokens_workspace_bytes(live.model, 3, 2, 4))
    for _ in range(6):
        y = live.step(new)
        last = np.cumsum([len(t) for t in new.values()]) - 1
        given = CU.i32([[7, -1]] * 3)
        lp, ent, ids, tlp = binding.radix_score_tokens(live.model, y, CU.i32(last.tolist()), given, ws, top_k=4)
        assert binding.radix_device_status(ws) == 0
        full = [np.asarray(live.tokens[s], dtype=np.int32) for s in new]
        cu = np.asarray(CU.ragged([len(t) for t in full]), dtype=np.int32)
        hidden = oracle_forward.forward_nodedup(cfg, live.w.embed, live.w.layers, live.w.gf, np.concatenate(full), cu)
        logits = torch.from_numpy(oracle_forward.lm_head_logits(hidden, live.w.embed, rows=cu[1:] - 1))
        ref = torch.log_softmax(logits, 1)
        # an error e of every logit moves a log-probability and the entropy's mean by at most 2 e and 2 e (1 + max |x - m|)
        e = live.tol * float(logits.square().mean().sqrt())
        assert (lp[:, 0].cpu() - ref[:, 7]).abs().max() <= 2 * e and (lp[:, 1] == 0).all()
        assert (ent.cpu() + (ref.exp() * ref).sum(1)).abs().max() <= 2 * e * (1 + float(ref.abs().max()))
        assert (tlp.cpu() - torch.topk(ref, 4).values).abs().max() <= 2 * e
        assert (ref.gather(1, ids.cpu().long()) - tlp.cpu()).abs().max() <= 2 * e
        new = {s: [int(ids[i, 0])] for i, s in enumerate(new)}
    live.model.close()


def test_scoring_whole_documents_in_row_blocks():
    live, rng = Live(F32, 74, 16, lm_head_mode=1), np.random.default_rng(5)
    hidden = torch.randn((1100, F32.d), device="cuda")
    given = torch.randint(0, F32.vocab, (1100, 1), dtype=torch.int32, device="cuda")
    ws = binding.alloc_workspace(binding.radix_score_tokens_workspace_bytes(live.model, 1100, 1, 2))
    lp, ent, ids, tlp = binding.radix_score_tokens(live.model, hidden, None, given, ws, top_k=2)
    assert binding.radix_device_status(ws) == 0
    ws2 = binding.alloc_workspace(binding.radix_lm_head_workspace_bytes(live.model, 1100))
    logits = binding.radix_lm_head(live.model, hidden, None, ws2)
    ref = torch.log_softmax(logits.double(), 1)
    assert (lp - ref.gather(1, given.long())).abs().max() < 1e-5
    assert (ent + (ref.exp() * ref).sum(1)).abs().max() < 1e-4
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :2]
    assert torch.equal(ids.long(), order)
    rows = torch.randperm(1100, device="cuda")[:700].int()
    by_rows = binding.radix_score_tokens(live.model, hidden, rows, given[rows.long()].contiguous(), ws, top_k=2)
    assert torch.equal(by_rows[2], ids[rows.long()]) and (by_rows[0] - lp[rows.long()]).abs().max() < 1e-5
    # rows and tokens out of range are reported; a model without a head refuses
    binding.radix_score_tokens(live.model, hidden, CU.i32([0, 1100]), None, ws, top_k=1)
    assert binding.radix_device_status(ws) == -7
    binding.radix_score_tokens(live.model, hidden, CU.i32([0]), CU.i32([[F32.vocab]]), ws)
    assert binding.radix_device_status(ws) == -7
    assert binding.radix_score_tokens(live.model, hidden, CU.i32([]), None, ws, top_k=1)[2].shape == (0, 1)
    assert binding.radix_device_status(ws) == 0
    with pytest.raises(binding.RadixError) as err:
        binding.radix_score_tokens(live.model, hidden, None, given, binding.alloc_workspace(4096))
    assert err.value.code == -4
    for wrong in (hidden.view(-1), hidden[:, :-1].contiguous(), hidden.view(550, 2, -1)):
        with pytest.raises(TypeError):
            binding.radix_score_tokens(live.model, wrong, None, None, ws, top_k=1)
    live.model.close()
    bare = harness.upload_model(live.w)
    with pytest.raises(binding.RadixError) as err:
        binding.radix_score_tokens(bare, hidden, None, given, ws)
    assert err.value.code == -3
    bare.close()


def test_a_step_without_room_changes_nothing_and_the_next_one_works():
    live, rng = Live(F32, 75, 16, n_pages=8, max_pages=6), np.random.default_rng(5)
    live.step({0: words(rng, F32, 60), 1: words(rng, F32, 20)})              # 4 + 2 pages of 8
    before = [t.clone() for t in (live.cache.page_refs, live.cache.page_table, live.cache.seq_lens, live.cache.pages.nan_to_num(7.0))]

    def refused(new, code):
        tok = torch.tensor(sum(new.values(), []), dtype=torch.int32).cuda()
        ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(live.model, live.cache, tok.numel(), len(new), 64))
        binding.radix_extend_forward(live.model, live.cache, tok, CU.i32(CU.ragged([len(t) for t in new.values()])), 64, ws, slots=CU.i32(list(new)))
        assert binding.radix_device_status(ws) == code
        now = (live.cache.page_refs, live.cache.page_table, live.cache.seq_lens, live.cache.pages.nan_to_num(7.0))
        assert all(torch.equal(a, b) for a, b in zip(before, now))

    refused({2: words(rng, F32, 30), 1: words(rng, F32, 20)}, -12)           # 2 + 1 pages
    refused({0: words(rng, F32, 40)}, -12)                                   # longer than a row of the table
    refused({9: words(rng, F32, 1)}, -13)
    tok = torch.tensor(words(rng, F32, 5), dtype=torch.int32).cuda()
    ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(live.model, live.cache, 5, 1, 5))
    binding.radix_extend_forward(live.model, live.cache, tok, CU.i32([0, 4]), 5, ws)       # does not end at N
    assert binding.radix_device_status(ws) == -6
    binding.radix_extend_forward(live.model, live.cache, tok, CU.i32([0, 5]), 4, ws)       # longer than max_new says
    assert binding.radix_device_status(ws) == -6
    now = (live.cache.page_refs, live.cache.page_table, live.cache.seq_lens, live.cache.pages.nan_to_num(7.0))
    assert all(torch.equal(a, b) for a, b in zip(before, now))
    live.step({1: words(rng, F32, 20), 0: words(rng, F32, 1)})
    live.model.close()


def test_no_position_behind_the_rope_table():
    cfg = synth.ModelConfig("short", 1, 256, 4, 2, 64, 768, 1000, "f32", max_pos=20)
    live, rng = Live(cfg, 76, 16), np.random.default_rng(5)
    live.step({0: words(rng, cfg, 19)})
    live.step({0: words(rng, cfg, 1)})
    ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(live.model, live.cache, 1, 1, 1))
    binding.radix_extend_forward(live.model, live.cache, CU.i32([3]), CU.i32([0, 1]), 1, ws)
    assert binding.radix_device_status(ws) == -12 and live.cache.seq_lens[0].item() == 20
    live.model.close()


def test_refusals():
    live = Live(F32, 77, 16)
    ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(live.model, live.cache, 4, 2, 4))
    tok, cu = CU.i32([1, 2, 3, 4]), CU.i32([0, 2, 4])

    def code(cache=live.cache, ws=ws, tok=tok, cu=cu, new=4):
        with pytest.raises(binding.RadixError) as err:
            binding.radix_extend_forward(live.model, cache, tok, cu, new, ws)
        return err.value.code

    ints = (2, 16, 10)                                                       # kv heads, page size, pages
    for layers, kv, hd, dt in [(3, 2, 64, torch.float32), (2, 4, 64, torch.float32), (2, 2, 32, torch.float32), (2, 2, 128, torch.float16)]:
        other = binding.alloc_cache(layers, kv, hd, ints[1], ints[2], dt, 4, 4)
        assert code(cache=other) == -9
    assert code(ws=binding.alloc_workspace(4096)) == -4
    assert code(new=0) == -2
    assert code(cache=binding.alloc_cache(2, 2, 64, 16, 10, torch.float32, 1, 4)) == -2      # two sequences, one slot
    with pytest.raises(ValueError):
        binding.radix_extend_forward(live.model, live.cache, tok, cu, 4, ws, slots=CU.i32([0]))
    with pytest.raises(TypeError):
        binding.radix_extend_forward(live.model, live.cache, tok.long(), cu, 4, ws)
    assert binding.radix_extend_forward(live.model, live.cache, CU.i32([]), CU.i32([0]), 0, ws).shape == (0, F32.d)
    assert live.cache.seq_lens.tolist() == [0] * 8
    live.model.close()


def test_decoding_steps_replay_from_a_graph():
    cfg = synth.ModelConfig("gen", 3, 256, 4, 2, 128, 320, 2048, "bf16", max_pos=1024)
    live, rng = Live(cfg, 78, 16, lm_head_mode=1), np.random.default_rng(5)
    live.step({0: words(rng, cfg, 40), 1: words(rng, cfg, 17)})
    model, cache = live.model, live.cache
    tok, cu, given = CU.i32([3, 4]), CU.i32([0, 1, 2]), None
    ws = binding.alloc_workspace(binding.radix_extend_workspace_bytes(model, cache, 2, 2, 1))
    ws2 = binding.alloc_workspace(binding.radix_score_tokens_workspace_bytes(model, 2, 0, 1))
    y = torch.empty((2, cfg.d), device="cuda")

    def decode():
        binding.radix_extend_forward(model, cache, tok, cu, 1, ws, out=y)
        ids = binding.radix_score_tokens(model, y, None, given, ws2, top_k=1)[2]
        tok.copy_(ids[:, 0])
        return ids

    state = [t.clone() for t in (cache.page_refs, cache.page_table, cache.seq_lens, cache.pages, tok)]
    eager = [(decode()[:, 0].tolist(), y.clone()) for _ in range(12)]        # crosses page borders
    for t, s in zip((cache.page_refs, cache.page_table, cache.seq_lens, cache.pages, tok), state):
        t.copy_(s)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ids = decode()
    for want, hidden in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert ids[:, 0].tolist() == want and torch.equal(y, hidden)
        assert binding.radix_device_status(ws) == 0
    assert cache.seq_lens.tolist()[:2] == [52, 29]
    live.model.close()
