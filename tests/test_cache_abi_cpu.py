"""Host-visible argument errors of the paged cache's, the paged attention's and the log-probabilities' entries: refused before anything
is launched (no GPU needed), and workspace sizes that grow with what they are asked for."""
import ctypes as C
import os

import pytest

from paper_2601_15013_amd import binding

FAKE = C.c_void_p(0x1000)              # never dereferenced: every call below fails its host checks
NULL, BAD_SIZE, UNSUPPORTED, TOO_SMALL, MISALIGNED = -1, -2, -3, -4, -5
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2601_15013_amd import build
        build.build()
    return binding.load_library()


def cache(**kw):
    good = dict(n_layers=2, n_kv_heads=4, head_dim=128, page_size=16, n_pages=100, dtype=1, max_seqs=8, max_pages=10, pages=0x1000,
                page_refs=0x1000, page_table=0x1000, seq_lens=0x1000)
    return C.byref(binding.radix_cache(**dict(good, **kw)))


BAD_SHAPES = [(dict(n_layers=0), BAD_SIZE), (dict(n_kv_heads=-1), BAD_SIZE), (dict(head_dim=0), BAD_SIZE), (dict(n_pages=0), BAD_SIZE),
              (dict(max_seqs=0), BAD_SIZE), (dict(max_pages=0), BAD_SIZE), (dict(dtype=3), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
              (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED),
              (dict(dtype=0, head_dim=66), UNSUPPORTED), (dict(dtype=0, head_dim=132), UNSUPPORTED), (dict(max_pages=1 << 27), BAD_SIZE), (dict(max_seqs=262145), UNSUPPORTED),
              (dict(n_pages=(1 << 28) + 1), UNSUPPORTED), (dict(n_kv_heads=65535, page_size=256), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_SHAPES)
def test_shapes_of_a_cache(lib, kw, code):
    n = C.c_size_t()
    assert lib.radix_cache_bytes(cache(**kw), C.byref(n)) == code
    assert lib.radix_cache_workspace_bytes(cache(**kw), 4, C.byref(n)) == code
    assert lib.radix_cache_reset(cache(**kw), None) == code
    assert lib.radix_cache_append(cache(**kw), 0, FAKE, 512, FAKE, 512, FAKE, FAKE, None, 1, 1, None, None) == code
    assert lib.radix_paged_attention_workspace_bytes(cache(**kw), 8, 4, 1, 4, 0, C.byref(n)) == code


@pytest.mark.parametrize("field", ["pages", "page_refs", "page_table", "seq_lens"])
def test_missing_arrays(lib, field):
    c = cache(**{field: None})
    assert lib.radix_cache_reset(c, None) == NULL
    assert lib.radix_cache_extend(c, None, FAKE, 1, FAKE, FAKE, BIG, None, None) == NULL
    assert lib.radix_cache_free(c, FAKE, None, 1, None, None) == NULL
    assert lib.radix_paged_attention(c, 0, FAKE, 1024, 8, FAKE, FAKE, None, 1, 1, 1, 0, FAKE, 1024, FAKE, BIG, None, None) == NULL


def test_sizes(lib):
    n = C.c_size_t()
    assert lib.radix_cache_bytes(cache(), C.byref(n)) == 0 and n.value == 2 * 100 * 2 * 4 * 16 * 128 * 2
    assert lib.radix_cache_bytes(cache(dtype=0, head_dim=4, page_size=256), C.byref(n)) == 0 and n.value == 2 * 100 * 2 * 4 * 256 * 4 * 4
    assert lib.radix_cache_bytes(cache(n_pages=200000, n_layers=36), C.byref(n)) == 0 and n.value == 36 * 200000 * 2 * 4 * 16 * 128 * 2
    assert lib.radix_cache_bytes(None, C.byref(n)) == NULL and lib.radix_cache_bytes(cache(), None) == NULL
    sizes = []
    for k in (0, 1, 50, 1000, 65535):
        assert lib.radix_cache_workspace_bytes(cache(), k, C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
    assert lib.radix_cache_workspace_bytes(cache(), -1, C.byref(n)) == BAD_SIZE
    assert lib.radix_cache_workspace_bytes(cache(), 65536, C.byref(n)) == UNSUPPORTED


@pytest.mark.parametrize("share", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_the_attention_workspace_grows_with_its_bounds(lib, dtype, share):
    n = C.c_size_t()

    def size(N, B, new):
        assert lib.radix_paged_attention_workspace_bytes(cache(dtype=dtype), 8, N, B, new, share, C.byref(n)) == 0
        return n.value

    for grow in ([(1, 1, 1), (8, 8, 1), (100, 100, 1), (2000, 2000, 1), (2100, 2100, 1), (4000, 4000, 1)], [(200, 10, 1), (200, 10, 8), (200, 10, 17), (200, 10, 100), (200, 10, 200)],
                 [(100, 1, 100), (1000, 1, 100), (1000, 1, 1000), (1000, 9, 1000)]):
        sizes = [size(*g) for g in grow]
        assert sizes == sorted(sizes)
    assert lib.radix_paged_attention_workspace_bytes(cache(), 6, 4, 1, 4, 0, C.byref(n)) == BAD_SIZE         # 4 kv heads do not divide 6
    assert lib.radix_paged_attention_workspace_bytes(cache(), 8, 1 << 29, 1, 4, 0, C.byref(n)) == UNSUPPORTED
    assert lib.radix_paged_attention_workspace_bytes(cache(), 8, -1, 1, 4, 0, C.byref(n)) == BAD_SIZE
    assert lib.radix_paged_attention_workspace_bytes(None, 8, 1, 1, 4, 0, C.byref(n)) == NULL


@pytest.mark.parametrize("share", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("heads", [4, 8, 16, 32, 64, 256])
def test_a_workspace_for_larger_bounds_holds_any_smaller_call(lib, dtype, share, heads):
    n = C.c_size_t()
    news = [0, 1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 200, 5000]
    last = {}
    for B in (0, 1, 2, 50, 127, 128, 600, 3000, 60000):
        for N in (0, 1, 50, 128, 700, 9000, 70000):
            sizes = []
            for new in news:
                assert lib.radix_paged_attention_workspace_bytes(cache(dtype=dtype), heads, N, B, new, share, C.byref(n)) == 0
                sizes.append(n.value)
            assert sizes == sorted(sizes), (B, N)
            for other, small in last.items():
                if other[0] <= B and other[1] <= N:
                    assert all(x <= y for x, y in zip(small, sizes)), (other, (B, N))
            last[B, N] = sizes


def test_page_calls_refuse(lib):
    c = cache()
    odd = C.c_void_p(0x1010)
    for call in (lambda n=2, a=FAKE, b=FAKE, ws=FAKE, sz=BIG: lib.radix_cache_fork(c, a, b, n, ws, sz, None, None),
                 lambda n=2, a=FAKE, b=FAKE, ws=FAKE, sz=BIG: lib.radix_cache_copy_pages(c, a, b, n, ws, sz, None, None),
                 lambda n=2, a=FAKE, b=FAKE, ws=FAKE, sz=BIG: lib.radix_cache_extend(c, None, a, n, b, ws, sz, None, None)):
        assert call(n=-1) == BAD_SIZE and call(n=65536) == UNSUPPORTED
        assert call(a=None) == NULL and call(b=None) == NULL and call(ws=None) == NULL
        assert call(ws=odd) == MISALIGNED and call(sz=300) == TOO_SMALL
        assert call(n=0) == 0                                                # nothing to do
    assert lib.radix_cache_extend(c, None, FAKE, 9, FAKE, FAKE, BIG, None, None) == BAD_SIZE           # 8 slots
    assert lib.radix_cache_free(c, None, None, 2, None, None) == NULL
    assert lib.radix_cache_free(c, FAKE, None, -2, None, None) == BAD_SIZE
    assert lib.radix_cache_free(c, FAKE, None, 0, None, None) == 0
    assert lib.radix_cache_compact(c, None, FAKE, BIG, None, None) == NULL
    assert lib.radix_cache_compact(c, FAKE, FAKE, 300, None, None) == TOO_SMALL
    assert lib.radix_cache_reset(cache(pages=0x1008), None) == MISALIGNED


def test_append_refuses(lib):
    def call(layer=0, k=FAKE, ks=512, v=FAKE, vs=512, cu=FAKE, past=FAKE, B=1, N=4, **kw):
        return lib.radix_cache_append(cache(**kw), layer, k, ks, v, vs, cu, past, None, B, N, None, None)

    assert call(layer=2) == BAD_SIZE and call(layer=-1) == BAD_SIZE and call(B=-1) == BAD_SIZE and call(N=-1) == BAD_SIZE
    assert call(ks=511) == BAD_SIZE and call(vs=8) == BAD_SIZE and call(ks=-512) == BAD_SIZE
    assert call(ks=516) == MISALIGNED and call(k=C.c_void_p(0x1008)) == MISALIGNED and call(v=C.c_void_p(0x1002)) == MISALIGNED
    assert call(k=None) == NULL and call(v=None) == NULL and call(cu=None) == NULL and call(past=None) == NULL
    assert call(B=65536) == UNSUPPORTED and call(N=1 << 24) == UNSUPPORTED
    assert call(N=0) == 0 and call(B=0) == 0


def test_paged_attention_refuses(lib):
    def call(layer=0, q=FAKE, qs=1024, hq=8, cu=FAKE, past=FAKE, B=1, N=4, new=4, out=FAKE, os_=1024, ws=FAKE, sz=BIG, **kw):
        return lib.radix_paged_attention(cache(**kw), layer, q, qs, hq, cu, past, None, B, N, new, 1, out, os_, ws, sz, None, None)

    assert call(layer=2) == BAD_SIZE and call(layer=-1) == BAD_SIZE and call(hq=6) == BAD_SIZE and call(hq=0) == BAD_SIZE
    assert call(B=-1) == BAD_SIZE and call(N=-1) == BAD_SIZE and call(new=-1) == BAD_SIZE and call(new=0) == BAD_SIZE
    assert call(qs=1020) == BAD_SIZE and call(os_=1016) == BAD_SIZE and call(qs=1028) == MISALIGNED and call(os_=1028) == MISALIGNED
    assert call(q=C.c_void_p(0x1008)) == MISALIGNED and call(out=C.c_void_p(0x1004)) == MISALIGNED and call(ws=C.c_void_p(0x1010)) == MISALIGNED
    for name in ("q", "cu", "past", "out", "ws"):
        assert call(**{name: None}) == NULL
    assert call(sz=4096) == TOO_SMALL and call(B=65536) == UNSUPPORTED and call(N=1 << 28) == UNSUPPORTED
    assert call(dtype=0, head_dim=4, qs=32, os_=32, N=1 << 27, new=1 << 27) == UNSUPPORTED                 # 2^26 blocks of 16 rows
    assert call(N=0) == 0 and call(B=0) == 0


def test_logprobs_refuse(lib):
    def call(x=FAKE, dt=0, stride=100, n=4, vocab=100, given=FAKE, g=1, k=2, lp=FAKE, ids=FAKE, tlp=FAKE, ws=FAKE, sz=BIG):
        return lib.radix_token_logprobs(x, dt, stride, n, vocab, given, g, k, lp, FAKE, ids, tlp, ws, sz, None, None)

    assert call(n=-1) == BAD_SIZE and call(vocab=0) == BAD_SIZE and call(g=-1) == BAD_SIZE and call(k=-1) == BAD_SIZE
    assert call(n=1 << 24) == UNSUPPORTED
    assert call(vocab=20, k=21) == BAD_SIZE and call(k=33) == UNSUPPORTED and call(dt=5) == UNSUPPORTED and call(stride=99) == BAD_SIZE
    for name in ("x", "given", "lp", "ids", "tlp", "ws"):
        assert call(**{name: None}) == NULL
    assert call(x=C.c_void_p(0x1002)) == MISALIGNED and call(ws=C.c_void_p(0x1010)) == MISALIGNED and call(sz=256) == TOO_SMALL
    assert call(n=0) == 0
    n = C.c_size_t()
    sizes = []
    for rows in (1, 2, 15, 16, 100, 5000):
        assert lib.radix_token_logprobs_workspace_bytes(rows, 50000, 1, 5, C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes)
    assert lib.radix_token_logprobs_workspace_bytes(1, 50000, 1, 5, None) == NULL


def test_model_calls_refuse_without_a_model(lib):
    n = C.c_size_t()
    assert lib.radix_extend_workspace_bytes(None, cache(), 4, 1, 4, C.byref(n)) == NULL
    assert lib.radix_extend_forward(None, cache(), FAKE, FAKE, None, 1, 4, 4, FAKE, FAKE, BIG, None) == NULL
    assert lib.radix_score_tokens_workspace_bytes(None, 4, 1, 1, C.byref(n)) == NULL
    assert lib.radix_score_tokens(None, FAKE, 4, None, 4, FAKE, 1, 0, FAKE, None, None, None, FAKE, BIG, None) == NULL


def test_the_new_status_codes_have_texts(lib):
    texts = {binding.radix_status_string(c) for c in (-11, -12, -13)}
    assert len(texts) == 3 and "unknown status" not in texts


def test_the_binding_struct_follows_the_header(lib):
    from tests.test_abi_cpu import _header_struct_fields
    assert [f[0] for f in binding.radix_cache._fields_] == _header_struct_fields("radix_cache")
