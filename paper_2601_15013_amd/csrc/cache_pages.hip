// Pages of a key/value cache: giving them out, storing rows in them, copying, sharing, releasing and moving them.
//
// The pool has no list of free pages: a page is free where page_refs is 0, and whoever needs pages gets the free ones of the
// lowest numbers, in the order of the request.  So the result of a call is a function of the state before it, whatever order the
// workgroups ran in.  (Reference counts are changed by atomic additions, which commute.)
//
// The calls that decide (extend, fork, compact, the check of a copy) run in one workgroup, because they are all or nothing: they
// look at everything (but for the entries of a fork's full pages, which are checked as they are copied), write nothing, then either write
// all of it or only report.  What they decide leaves as a list of moves
// (source page, destination page, rows), and a second launch over the chip copies.
#include "block_scan.h"
#include "common.h"
#include "kernels.h"

namespace {

// Numbers, in ascending order, the pages p of [from, to) for which pick(page_refs[p]) holds, and calls put(p, number) for them
// until `want` are found.  Returns how many were (at most `want`).  4096 pages a step; cnt: [2][64] in LDS.
template <typename Pick, typename Put>
__device__ __forceinline__ int number_pages(const int32_t* __restrict__ refs, int from, int to, int want, int (*cnt)[64], Pick pick,
                                            Put put) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0, par = 0;
    int r[4];
    auto fetch = [&](long long base) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long p = base + u * PT + (int)threadIdx.x;
            r[u] = p < to ? refs[p] : 0;
        }
    };
    if (from < to && want > 0) fetch(from);
    for (long long base = from; base < to && found < want; base += 4 * PT, par ^= 1) {
        unsigned long long hit[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long p = base + u * PT + (int)threadIdx.x;
            hit[u] = __ballot(p < to && pick(r[u]));
        }
        if (base + 4 * PT < to) fetch(base + 4 * PT);
        const int mine_of = lane == 0 ? __popcll(hit[0]) : lane == 1 ? __popcll(hit[1]) : lane == 2 ? __popcll(hit[2]) : __popcll(hit[3]);
        if (lane < 4) cnt[par][lane * 16 + wave] = mine_of;
        __syncthreads();
        const int mine = cnt[par][lane];                    // lane = 16 u + wavefront: the order of the pages
        const int incl = wave_inclusive(mine);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int before = __shfl(incl - mine, u * 16 + wave, 64);
            const int n = found + before + __popcll(hit[u] & ((1ull << lane) - 1ull));
            if ((hit[u] >> lane & 1ull) && n < want) put((int)(base + u * PT + (int)threadIdx.x), n);
        }
        found += __shfl(incl, 63, 64);
    }
    return found < want ? found : want;
}

// Slots that a call has met, a bit each, in LDS (in global memory every look was a round trip of a microsecond).
struct Marks {
    uint32_t bits[CACHE_MAX_SLOTS / 32];
    __device__ __forceinline__ void clear(int slots) {
        for (int i = threadIdx.x; i < (slots + 31) / 32; i += PT) bits[i] = 0;
    }
    __device__ __forceinline__ bool set(int slot) {         // whether it was set before
        return atomicOr(&bits[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1u;
    }
    __device__ __forceinline__ bool has(int slot) const { return bits[slot >> 5] >> (slot & 31) & 1u; }
};

__device__ __forceinline__ int pages_of(int tokens, int page_size) { return (tokens + page_size - 1) / page_size; }

// The sequence of entry r of a list that `first` (exclusive sums, n + 1 entries) describes.
__device__ __forceinline__ int owner_of(const int32_t* first, int n, int r) {
    int lo = 0, hi = n - 1;             // first[lo] <= r < first[hi + 1]
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= r) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ------------------------------------------------------------------ extend
// Bound by the latency of its steps, one after the other: 32 sequences 4.6 us (fork 6.2, compact of 300 pages 5.3), and in a large pool by the
// walk over the counts from page 0 to the last page that it takes: 14 us more behind 65 000 pages in use, 226 behind a million.
// Sequence b of the call gets room for cu[b + 1] - cu[b] more tokens.  Where its last page is partly filled and shared (a fork
// that was shortened), the new tokens must not reach the others: it gets a page of its own, with the rows that it has.
__global__ __launch_bounds__(PT) void cache_extend_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ cu,
                                                          int B, int limit, int32_t* __restrict__ past, int32_t* __restrict__ ws, PageWs L,
                                                          const int32_t* gate, int32_t* status) {
    __shared__ long long part[PT / 64];
    __shared__ int cnt[2][64];
    __shared__ int bad, n_moves;
    __shared__ Marks met;
    const int tid = threadIdx.x, P = c.page_size;
    int32_t *list = ws + L.list, *first = ws + L.first, *shared = ws + L.shared;
    if (tid == 0) { bad = gate ? *gate : 0; n_moves = 0; }
    met.clear(c.max_seqs);
    __syncthreads();
    long long run = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
        const int b = b0 + tid;
        int need = 0, err = 0, own = 0;
        if (b < B) {
            const int s = slots ? slots[b] : b;
            const long long from = cu[b], to = cu[b + 1], n = to - from;
            if (from < 0 || n < 0 || (b == 0 && from != 0)) err = RADIX_ERR_BAD_CU_SEQLENS;
            else if (s < 0 || s >= c.max_seqs || met.set(s)) err = RADIX_ERR_BAD_SLOT;
            else {
                const int len = c.lens[s];
                if (len < 0 || len > (long long)c.max_pages * P) err = RADIX_ERR_BAD_PAGE;
                else if (len + n > limit) err = RADIX_ERR_OUT_OF_PAGES;
                else {
                    if (n > 0 && len % P != 0) {
                        const int p = c.table[(size_t)s * c.max_pages + len / P];
                        if (p < 0 || p >= c.n_pages) err = RADIX_ERR_BAD_PAGE;
                        else own = c.refs[p] > 1;
                    }
                    need = pages_of(len + (int)n, P) - pages_of(len, P) + own;
                }
            }
            if (err) { atomicMin(&bad, err); need = 0; own = 0; }
        }
        long long total;
        const long long before = block_exclusive(need, &total, part) + run;
        if (b < B) {
            first[b] = before > c.n_pages ? c.n_pages : (int)before;        // more than the pool holds: refused below
            shared[b] = own;
        }
        run += total;
    }
    if (tid == 0) first[B] = run > c.n_pages ? c.n_pages : (int)run;
    __syncthreads();
    if (bad == 0 && run <= c.n_pages) {
        const int got = number_pages(c.refs, 0, c.n_pages, (int)run, cnt, [](int r) { return r == 0; }, [&](int p, int n) { list[n] = p; });
        if (got < run && tid == 0) bad = RADIX_ERR_OUT_OF_PAGES;
    } else if (tid == 0 && bad == 0) {
        bad = RADIX_ERR_OUT_OF_PAGES;
    }
    __syncthreads();
    if (bad != 0) {
        if (tid == 0) { set_status(status, bad); ws[0] = 0; }
        for (int b = tid; b < B; b += PT) past[b] = -1;
        return;
    }
    for (int r = tid; r < (int)run; r += PT) {
        const int b = owner_of(first, B, r), s = slots ? slots[b] : b, len = c.lens[s], page = list[r];
        int32_t* row = c.table + (size_t)s * c.max_pages;
        const int at = r - first[b] - shared[b];
        if (at < 0) {
            const int m = atomicAdd(&n_moves, 1), old = row[len / P];
            ws[L.src + m] = old; ws[L.dst + m] = page; ws[L.rows + m] = len % P;
            atomicSub(&c.refs[old], 1);
            row[len / P] = page;
        } else {
            row[pages_of(len, P) + at] = page;
        }
        atomicExch(&c.refs[page], 1);
    }
    __syncthreads();
    if (tid == 0) ws[0] = n_moves;
    for (int b = tid; b < B; b += PT) {
        const int s = slots ? slots[b] : b, len = c.lens[s];
        past[b] = len;
        c.lens[s] = len + (cu[b + 1] - cu[b]);
    }
}

// ------------------------------------------------------------------ fork
// children[i] (empty) becomes a copy of parents[i]: full pages shared (by the second launch), a partly filled last page copied.
__global__ __launch_bounds__(PT) void cache_fork_kernel(CacheView c, const int32_t* __restrict__ parents,
                                                        const int32_t* __restrict__ children, int n, int32_t* __restrict__ ws, PageWs L,
                                                        int32_t* status) {
    __shared__ long long part[PT / 64];
    __shared__ int cnt[2][64];
    __shared__ int bad;
    __shared__ Marks is_child, is_parent;
    const int tid = threadIdx.x, P = c.page_size;
    int32_t *list = ws + L.list, *first = ws + L.first;
    auto ok_slot = [&](int s) { return s >= 0 && s < c.max_seqs; };
    if (tid == 0) bad = 0;
    is_child.clear(c.max_seqs);
    is_parent.clear(c.max_seqs);
    __syncthreads();
    long long run = 0;
    for (int i0 = 0; i0 < n; i0 += PT) {
        const int i = i0 + tid;
        int need = 0, err = 0;
        if (i < n) {
            const int p = parents[i], s = children[i];
            if (!ok_slot(p) || !ok_slot(s)) err = RADIX_ERR_BAD_SLOT;
            else {
                if (is_child.set(s)) err = RADIX_ERR_BAD_SLOT;                      // the same child twice
                is_parent.set(p);
                const int len = c.lens[p];
                if (c.lens[s] != 0) err = RADIX_ERR_BAD_SLOT;                       // the child holds something
                else if (len < 0 || len > (long long)c.max_pages * P) err = RADIX_ERR_BAD_PAGE;
                else if (len % P != 0) {
                    const int page = c.table[(size_t)p * c.max_pages + len / P];
                    if (page < 0 || page >= c.n_pages) err = RADIX_ERR_BAD_PAGE; else need = 1;
                }
            }
            if (err) { atomicMin(&bad, err); need = 0; }
        }
        long long total;
        const long long before = block_exclusive(need, &total, part) + run;
        if (i < n) first[i] = (int)before;
        run += total;
    }
    if (tid == 0) first[n] = (int)run;
    __syncthreads();
    for (int i = tid; i < n; i += PT)                                               // a child that is a parent, too
        if (ok_slot(children[i]) && is_parent.has(children[i])) atomicMin(&bad, (int)RADIX_ERR_BAD_SLOT);
    __syncthreads();
    if (bad == 0 && run <= c.n_pages) {
        const int got = number_pages(c.refs, 0, c.n_pages, (int)run, cnt, [](int r) { return r == 0; }, [&](int p, int k) { list[k] = p; });
        if (got < run && tid == 0) bad = RADIX_ERR_OUT_OF_PAGES;
    } else if (tid == 0 && bad == 0) {
        bad = RADIX_ERR_OUT_OF_PAGES;
    }
    __syncthreads();
    if (bad != 0) {
        if (tid == 0) { set_status(status, bad); ws[0] = 0; ws[1] = 0; }
        return;
    }
    for (int i = tid; i < n; i += PT) {
        const int p = parents[i], s = children[i], len = c.lens[p], m = first[i];
        if (first[i + 1] > m) {
            const int page = list[m];
            ws[L.src + m] = c.table[(size_t)p * c.max_pages + len / P];
            ws[L.dst + m] = page;
            ws[L.rows + m] = len % P;
            c.table[(size_t)s * c.max_pages + len / P] = page;
            c.refs[page] = 1;
        }
        c.lens[s] = len;
    }
    if (tid == 0) { ws[0] = (int)run; ws[1] = 1; }
}

// ------------------------------------------------------------------ compact
// U pages are used: those numbered U or more move, in ascending order, into the free pages below U.
__global__ __launch_bounds__(PT) void cache_compact_kernel(CacheView c, int32_t* __restrict__ n_used, int32_t* __restrict__ ws, PageWs L) {
    __shared__ long long part[PT / 64];
    __shared__ int cnt[2][64];
    const int tid = threadIdx.x;
    int32_t *map = ws + L.map, *src = ws + L.src, *dst = ws + L.dst, *rows = ws + L.rows;
    long long mine = 0, total;
    for (long long p0 = 0; p0 < c.n_pages; p0 += 8 * PT) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const long long p = p0 + u * PT + tid;
            mine += p < c.n_pages ? c.refs[p] != 0 : 0;
        }
    }
    block_exclusive(mine, &total, part);
    const int U = (int)total;
    for (int p = U + tid; p < c.n_pages; p += PT) map[p] = -1;
    __syncthreads();
    const int holes = number_pages(c.refs, 0, U, U, cnt, [](int r) { return r == 0; }, [&](int p, int k) { dst[k] = p; });
    __syncthreads();
    const int moved = number_pages(c.refs, U, c.n_pages, holes, cnt, [](int r) { return r != 0; }, [&](int p, int k) { src[k] = p; });
    __syncthreads();
    for (int m = tid; m < moved; m += PT) {
        const int from = src[m], to = dst[m];
        map[from] = to;
        rows[m] = c.page_size;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (tid == 0) { ws[0] = moved; ws[1] = U; *n_used = U; }
}

// ------------------------------------------------------------------ check of a list of copies
__global__ __launch_bounds__(PT) void cache_copy_check_kernel(CacheView c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                              int n, int32_t* __restrict__ ws, PageWs L, int32_t* status) {
    __shared__ int bad;
    const int tid = threadIdx.x;
    int32_t* mark = ws + L.map;
    auto ok = [&](int p) { return p >= 0 && p < c.n_pages; };
    if (tid == 0) bad = 0;
    for (int i = tid; i < n; i += PT) {
        if (ok(src[i])) atomicExch(&mark[src[i]], 0);
        if (ok(dst[i])) atomicExch(&mark[dst[i]], 0);
    }
    __syncthreads();
    for (int i = tid; i < n; i += PT) {
        if (!ok(src[i]) || !ok(dst[i])) { bad = 1; continue; }
        if (atomicOr(&mark[dst[i]], 1) & 1) bad = 1;                // two copies to one page
        atomicOr(&mark[src[i]], 2);
    }
    __syncthreads();
    for (int i = tid; i < n; i += PT)
        if (ok(dst[i]) && (atomicOr(&mark[dst[i]], 0) & 2)) bad = 1;        // copied to and copied from
    __syncthreads();
    if (tid == 0) {
        ws[0] = bad ? 0 : n;
        if (bad) set_status(status, RADIX_ERR_BAD_PAGE);
    }
}

// ------------------------------------------------------------------ moves
// The copies of a call, and beside them what it does to the table.  A wavefront copies one piece (one head's keys or values of one
// layer of a page: consecutive bytes) of 16-byte vectors, eight in flight per lane; the pieces are dealt to the wavefronts in turn.
// Bound by HBM.  2.3 GB pool, 0.56 GB moved: 210 us, 5.4 TB/s read and written (217 without the non-temporal accesses; a copy of 4 GB
// by torch runs at 4.8).  Rows of 32 forks over 28 layers (69 MB, much of it read from cache): 19 us.
enum { TABLE_NONE = 0, TABLE_FORK = 1, TABLE_REMAP = 2 };
template <int TABLE>
__global__ __launch_bounds__(256) void cache_move_kernel(CacheView c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                         const int32_t* __restrict__ rows, const int32_t* __restrict__ ws, int table_blocks,
                                                         const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                                                         const int32_t* __restrict__ map, int32_t* status) {
    if ((int)blockIdx.x < table_blocks) {
        if (TABLE == TABLE_FORK) {
            if (ws[1] == 0) return;                                         // the call was refused
            const int p = parents[blockIdx.x], s = children[blockIdx.x];
            const int full = c.lens[s] / c.page_size;
            const int32_t* from = c.table + (size_t)p * c.max_pages;
            int32_t* to = c.table + (size_t)s * c.max_pages;
            for (int j = threadIdx.x; j < full; j += 256) {
                const int page = from[j];
                to[j] = page;
                if (page >= 0 && page < c.n_pages) atomicAdd(&c.refs[page], 1);
                else set_status(status, RADIX_ERR_BAD_PAGE);
            }
        }
        if (TABLE == TABLE_REMAP) {
            const size_t n = (size_t)c.max_seqs * c.max_pages;
            for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)table_blocks * 256) {
                const int page = c.table[i];
                if (page < ws[1]) continue;                                 // stays, or no page
                const int to = page < c.n_pages ? map[page] : -1;
                if (to >= 0) c.table[i] = to; else set_status(status, RADIX_ERR_BAD_PAGE);
            }
        }
        return;
    }
    const int lane = threadIdx.x & 63;
    const int pieces = 2 * c.n_kv_heads;
    const long long units = (long long)ws[0] * c.n_layers * pieces;
    const long long step = (long long)(gridDim.x - table_blocks) * 4;
    const size_t row_vecs = (size_t)c.piece_bytes / c.page_size / 16;
    for (long long u = (long long)(blockIdx.x - table_blocks) * 4 + (threadIdx.x >> 6); u < units; u += step) {
        const int piece = (int)(u % pieces);
        const int m = (int)(u / pieces / c.n_layers), layer = (int)(u / pieces % c.n_layers);
        const size_t at = (size_t)layer * c.layer_bytes + (size_t)piece * c.piece_bytes;
        const u32x4* s = reinterpret_cast<const u32x4*>(c.pages + at + (size_t)src[m] * c.page_bytes);
        u32x4* d = reinterpret_cast<u32x4*>(c.pages + at + (size_t)dst[m] * c.page_bytes);
        const int vecs = (int)((rows ? rows[m] : c.page_size) * row_vecs);
        int v = lane;
        for (; v + 7 * 64 < vecs; v += 8 * 64) {
            u32x4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = __builtin_nontemporal_load(s + v + 64 * k);
#pragma unroll
            for (int k = 0; k < 8; ++k) __builtin_nontemporal_store(x[k], d + v + 64 * k);
        }
        for (; v < vecs; v += 64) d[v] = s[v];
    }
}

// ------------------------------------------------------------------ free
// Entries of the pages from ceil(keep / page) on leave the table, each by exchange, so that a slot listed twice loses a page once.
__global__ __launch_bounds__(256) void cache_free_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ keep,
                                                         int32_t* status) {
    const int s = slots[blockIdx.x];
    if (s < 0 || s >= c.max_seqs) {
        if (threadIdx.x == 0) set_status(status, RADIX_ERR_BAD_SLOT);
        return;
    }
    int k = keep ? keep[blockIdx.x] : 0;
    k = k < 0 ? 0 : k;
    const long long from = ((long long)k + c.page_size - 1) / c.page_size;
    for (long long j = from + threadIdx.x; j < c.max_pages; j += 256) {
        int32_t* entry = &c.table[(size_t)s * c.max_pages + j];
        if (*entry == -1) continue;                                         // (most are)
        const int page = atomicExch(entry, -1);
        if (page == -1) continue;
        if (page < 0 || page >= c.n_pages) { set_status(status, RADIX_ERR_BAD_PAGE); continue; }
        if (atomicSub(&c.refs[page], 1) <= 0) {                             // nobody held it: leave it free
            atomicAdd(&c.refs[page], 1);
            set_status(status, RADIX_ERR_BAD_PAGE);
        }
    }
    if (threadIdx.x == 0) atomicMin(&c.lens[s], k);
}

__global__ __launch_bounds__(256) void cache_reset_kernel(CacheView c) {
    const size_t entries = (size_t)c.max_seqs * c.max_pages, step = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += step) c.table[i] = -1;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)c.n_pages; i += step) c.refs[i] = 0;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)c.max_seqs; i += step) c.lens[i] = 0;
}

// ------------------------------------------------------------------ append
// One wavefront per new token: its keys and values of all heads are two runs of 16-byte vectors; each head's part goes to its piece.
// Bound by HBM: 21 200 tokens of 8 heads of 128, fp16: 31 us, 5.6 TB/s read and written (36 with one vector in flight and plain loads).
// 64 tokens: 3.7 us, a launch.
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, int layer, const char* __restrict__ k, const char* __restrict__ v,
                                                           size_t k_stride, size_t v_stride, const int32_t* __restrict__ cu,
                                                           const int32_t* __restrict__ past, const int32_t* __restrict__ slots, int B, int N,
                                                           int32_t* status) {
    const int lane = threadIdx.x & 63;
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= N) return;
    const int b = sequence_of(cu, B, i, lane);
    const int from = cu[b], to = cu[b + 1];
    if (from < 0 || from > to || to > N || i < from) { if (lane == 0) set_status(status, RADIX_ERR_BAD_CU_SEQLENS); return; }
    if (i >= to) return;                                    // behind the last sequence
    const int done = past[b];
    if (done < 0) return;
    const int s = slots ? slots[b] : b;
    if (s < 0 || s >= c.max_seqs) { if (lane == 0) set_status(status, RADIX_ERR_BAD_SLOT); return; }
    const long long p = (long long)done + (i - from);
    int page = -1;
    if (p < (long long)c.max_pages * c.page_size) page = c.table[(size_t)s * c.max_pages + p / c.page_size];
    if (page < 0 || page >= c.n_pages) { if (lane == 0) set_status(status, RADIX_ERR_BAD_PAGE); return; }
    const size_t row_bytes = c.piece_bytes / c.page_size;
    const int row_vecs = (int)(row_bytes / 16), vecs = c.n_kv_heads * row_vecs;
    char* base = c.pages + (size_t)layer * c.layer_bytes + (size_t)page * c.page_bytes + (size_t)(p % c.page_size) * row_bytes;
    const u32x4* ks = reinterpret_cast<const u32x4*>(k + (size_t)i * k_stride);
    const u32x4* vs = reinterpret_cast<const u32x4*>(v + (size_t)i * v_stride);
    for (int e0 = lane; e0 < 2 * vecs; e0 += 4 * 64) {      // four vectors in flight
        u32x4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = e0 + 64 * u;
            if (e < 2 * vecs) y[u] = __builtin_nontemporal_load(e < vecs ? ks + e : vs + (e - vecs));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = e0 + 64 * u, x = e < vecs ? e : e - vecs, piece = (e < vecs ? 0 : c.n_kv_heads) + x / row_vecs;
            if (e < 2 * vecs) *reinterpret_cast<u32x4*>(base + (size_t)piece * c.piece_bytes + (size_t)(x % row_vecs) * 16) = y[u];
        }
    }
}

__global__ __launch_bounds__(256) void paged_positions_kernel(const int32_t* __restrict__ cu, const int32_t* __restrict__ past, int B,
                                                              int N, int32_t* __restrict__ pos) {
    const int lane = threadIdx.x & 63;
    const int i0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 64;              // 64 tokens a wavefront
    if (i0 >= N) return;
    const int i = i0 + lane;
    int lo = sequence_of(cu, B, i0, lane), hi = B - 1;                      // of its own token every lane searches from there
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid + 1] > i) hi = mid; else lo = mid + 1;
    }
    if (i < N) pos[i] = past[lo] < 0 ? 0 : past[lo] + (i - cu[lo]);
}

unsigned move_blocks(const CacheView& c, long long moves) {
    const long long b = (moves * c.n_layers * 2 * c.n_kv_heads + 3) / 4;
    return (unsigned)(b < 1 ? 1 : (b > 4096 ? 4096 : b));
}

}  // namespace

void launch_cache_reset(const CacheView& c, hipStream_t stream) {
    const size_t most = (size_t)c.max_seqs * c.max_pages + (size_t)c.n_pages;
    const size_t blocks = (most + 1023) / 1024;
    hipLaunchKernelGGL(cache_reset_kernel, dim3((unsigned)(blocks > 2048 ? 2048 : blocks)), dim3(256), 0, stream, c);
}

void launch_cache_extend(const CacheView& c, const int32_t* slots, const int32_t* cu, int B, int limit, int32_t* past, int32_t* ws,
                         const int32_t* gate, int32_t* status, hipStream_t stream) {
    const PageWs L = page_ws_layout(c.n_pages, B);
    hipLaunchKernelGGL(cache_extend_kernel, dim3(1), dim3(PT), 0, stream, c, slots, cu, B, limit, past, ws, L, gate, status);
    hipLaunchKernelGGL(cache_move_kernel<TABLE_NONE>, dim3(move_blocks(c, B)), dim3(256), 0, stream, c, ws + L.src, ws + L.dst, ws + L.rows,
                       ws, 0, nullptr, nullptr, nullptr, status);
}

void launch_cache_fork(const CacheView& c, const int32_t* parents, const int32_t* children, int n, int32_t* ws, int32_t* status,
                       hipStream_t stream) {
    const PageWs L = page_ws_layout(c.n_pages, n);
    hipLaunchKernelGGL(cache_fork_kernel, dim3(1), dim3(PT), 0, stream, c, parents, children, n, ws, L, status);
    hipLaunchKernelGGL(cache_move_kernel<TABLE_FORK>, dim3(move_blocks(c, n) + (unsigned)n), dim3(256), 0, stream, c, ws + L.src, ws + L.dst,
                       ws + L.rows, ws, n, parents, children, nullptr, status);
}

void launch_cache_free(const CacheView& c, const int32_t* slots, const int32_t* keep, int n, int32_t* status, hipStream_t stream) {
    hipLaunchKernelGGL(cache_free_kernel, dim3((unsigned)n), dim3(256), 0, stream, c, slots, keep, status);
}

void launch_cache_compact(const CacheView& c, int32_t* n_used, int32_t* ws, int32_t* status, hipStream_t stream) {
    const PageWs L = page_ws_layout(c.n_pages, 0);
    hipLaunchKernelGGL(cache_compact_kernel, dim3(1), dim3(PT), 0, stream, c, n_used, ws, L);
    const size_t entries = (size_t)c.max_seqs * c.max_pages;
    const unsigned tb = (unsigned)(entries / 2048 > 1024 ? 1024 : entries / 2048 + 1);
    hipLaunchKernelGGL(cache_move_kernel<TABLE_REMAP>, dim3(move_blocks(c, c.n_pages / 2) + tb), dim3(256), 0, stream, c, ws + L.src,
                       ws + L.dst, ws + L.rows, ws, (int)tb, nullptr, nullptr, ws + L.map, status);
}

void launch_cache_copy(const CacheView& c, const int32_t* src, const int32_t* dst, int n, int32_t* ws, int32_t* status,
                       hipStream_t stream) {
    const PageWs L = page_ws_layout(c.n_pages, 0);
    hipLaunchKernelGGL(cache_copy_check_kernel, dim3(1), dim3(PT), 0, stream, c, src, dst, n, ws, L, status);
    hipLaunchKernelGGL(cache_move_kernel<TABLE_NONE>, dim3(move_blocks(c, n)), dim3(256), 0, stream, c, src, dst, nullptr, ws, 0, nullptr,
                       nullptr, nullptr, status);
}

void launch_cache_append(const CacheView& c, int layer, const void* k, const void* v, size_t k_stride, size_t v_stride,
                         const int32_t* cu, const int32_t* past, const int32_t* slots, int B, int N, int32_t* status,
                         hipStream_t stream) {
    hipLaunchKernelGGL(cache_append_kernel, dim3((unsigned)ceil_div(N, 4)), dim3(256), 0, stream, c, layer, (const char*)k, (const char*)v,
                       k_stride, v_stride, cu, past, slots, B, N, status);
}

void launch_paged_positions(const int32_t* cu, const int32_t* past, int B, int N, int32_t* pos, hipStream_t stream) {
    hipLaunchKernelGGL(paged_positions_kernel, dim3((unsigned)ceil_div(N, 256)), dim3(256), 0, stream, cu, past, B, N, pos);
}
