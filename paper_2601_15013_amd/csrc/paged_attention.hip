// Causal attention of new tokens over a paged key/value cache: a chunk of a prompt, one token of a decoding sequence, or both in
// one batch.  o[i, h] = sum over the positions p <= pos(i) of softmax_p(q[i, h] . K[p, h / group] / sqrt(hd)) V[p, h / group], where the
// new tokens' own keys and values are in the cache already.
//
// Softmax runs online (running maximum m and sum l in fp32, one pass over the keys); the fp32 accumulators of a row are rescaled when
// m grows.  Probabilities are rounded to the operand type for the second product: the sum l is taken before that rounding, so a row's
// error stays at half a step of the type on each term.
//
// Rows are (token, query head of a group) pairs of one kv head, so that a key tile is read once for the whole group, whatever its
// size.  Two kernels:
//  few rows   (decoding): bound by the cache's bytes.  A wavefront owns whole key tiles and keeps everything in registers: no LDS and no
//             barrier on the way, the next tile in flight while one is multiplied.
//  many rows  (chunks): bound by the matrix and vector units.  Four wavefronts of 32 rows share key tiles in LDS.
// Long key ranges are split over workgroups where a batch has few blocks; a last launch joins the parts in the order of the keys.
#include "block_scan.h"
#include "common.h"
#include "gemm_async.h"
#include "kernels.h"

namespace {

constexpr int FEW_TARGET = 1024, MANY_TARGET = 512;      // workgroups that a batch is split for
constexpr int MANY_ROWS = 128, MANY_TILE = 64;
constexpr int MAX_HD = 128;

struct PagedArgs {
    CacheView c;
    PagedShape s;
    PagedLayout L;
    const int32_t *cu, *past, *slots;
    int layer;
    const int32_t* plan;
    float *few_acc, *few_ml, *many_acc, *many_ml;
};

// What a sequence of the batch has, from device data that may be anything: `from` .. `from + n` lies in [0, N), and len <= what the
// table's row can hold.  len = 0: nothing to attend to (zeros).
struct PagedSeq { int from, n, len, past, row, err; };
__device__ __forceinline__ PagedSeq paged_seq(const CacheView& c, const PagedShape& s, const int32_t* cu, const int32_t* past,
                                              const int32_t* slots, int b) {
    PagedSeq q;
    const int from = cu[b], to = cu[b + 1];
    const int p = past[b], row = slots ? slots[b] : b;
    q.err = 0;
    q.from = from; q.n = 0; q.len = 0; q.past = 0; q.row = 0;
    if (from < 0 || to < from || to > s.N || (long long)to - from > s.max_new) { q.from = 0; q.err = RADIX_ERR_BAD_CU_SEQLENS; return q; }
    q.n = to - from;
    if (p < 0 || q.n == 0) return q;
    if (row < 0 || row >= c.max_seqs) { q.err = RADIX_ERR_BAD_SLOT; return q; }
    if ((long long)p + q.n > (long long)c.max_pages * c.page_size) { q.err = RADIX_ERR_BAD_PAGE; return q; }
    q.row = row;
    q.past = p;
    q.len = p + q.n;
    return q;
}

// ------------------------------------------------------------------ the plan (one workgroup)
__global__ __launch_bounds__(PT) void paged_plan_kernel(CacheView c, PagedShape s, PagedLayout L, const int32_t* __restrict__ cu,
                                                        const int32_t* __restrict__ past, const int32_t* __restrict__ slots,
                                                        int32_t* __restrict__ plan, int32_t* status) {
    __shared__ long long part[PT / 64];
    const int tid = threadIdx.x, group = s.n_q_heads / c.n_kv_heads;
    auto shape_of = [&](int b, bool& few, int& blocks, int& tiles) -> int {
        const PagedSeq q = paged_seq(c, s, cu, past, slots, b);
        const int rows = q.n * group;
        few = !L.many || rows <= L.few_rows;
        blocks = few ? ceil_div(rows, L.few_rows) : ceil_div(rows, MANY_ROWS);
        tiles = few ? ceil_div(q.len, L.few_tile) : ceil_div(q.len, MANY_TILE);
        return q.err;
    };
    long long few_work = 0, many_work = 0, total;
    for (int b = tid; b < s.B; b += PT) {
        bool few; int blocks, tiles;
        const int err = shape_of(b, few, blocks, tiles);
        if (err) set_status(status, err);
        (few ? few_work : many_work) += (long long)blocks * tiles * c.n_kv_heads;
    }
    block_exclusive(few_work, &total, part);
    // tiles of a split: even shares of the work for the target number of workgroups, no less than 256 keys
    const long long least_few = 256 / L.few_tile, least_many = 256 / MANY_TILE;
    const long long few_len = max(least_few, (total + FEW_TARGET - 1) / FEW_TARGET);
    block_exclusive(many_work, &total, part);
    const long long many_len = max(least_many, (total + MANY_TARGET - 1) / MANY_TARGET);
    long long run_items = 0, run_slots = 0, run_units = 0;               // few in the low half, many in the high half
    for (int b0 = 0; b0 < s.B; b0 += PT) {
        const int b = b0 + tid;
        bool few = true; int blocks = 0, tiles = 0, splits = 1;
        if (b < s.B) {
            shape_of(b, few, blocks, tiles);
            splits = (int)((tiles + (few ? few_len : many_len) - 1) / (few ? few_len : many_len));
            splits = splits < 1 ? 1 : splits;
        }
        const long long units = (long long)blocks * c.n_kv_heads, items = units * splits;
        const int sh = few ? 0 : 32;
        long long ti, ts, tu;
        const long long i0 = run_items + block_exclusive(items << sh, &ti, part);
        const long long s0 = run_slots + block_exclusive((splits > 1 ? items : 0) << sh, &ts, part);
        const long long u0 = run_units + block_exclusive(splits > 1 ? units : 0, &tu, part);
        if (b < s.B) {
            plan[L.item_few + b] = (int)(i0 & 0xffffffffLL);
            plan[L.item_many + b] = (int)(i0 >> 32);
            plan[L.slot_few + b] = (int)(s0 & 0xffffffffLL);
            plan[L.slot_many + b] = (int)(s0 >> 32);
            plan[L.unit + b] = (int)u0;
            plan[L.splits + b] = splits;
        }
        run_items += ti; run_slots += ts; run_units += tu;
    }
    if (tid == 0) {
        plan[L.item_few + s.B] = (int)(run_items & 0xffffffffLL);
        plan[L.item_many + s.B] = (int)(run_items >> 32);
        plan[L.unit + s.B] = (int)run_units;
    }
}

// A work item: the kv head, block and tile range of a sequence; `slot` of its partial result where the block is split.
// Items of a sequence: kv heads fastest, so that consecutive workgroups - and with them the eight XCDs - take different heads, and
// the blocks of one head, which read the same keys, meet in one L2; then the splits; then the blocks, the last (longest) first.
struct PagedItem { int b, kvh, blk, split, splits, slot; };
__device__ __forceinline__ bool paged_item(const PagedArgs& a, size_t item_at, size_t slot_at, long long max_slots, int item, int lane, PagedItem& w) {
    const int32_t* first = a.plan + item_at;
    if (item >= first[a.s.B]) return false;
    w.b = __builtin_amdgcn_readfirstlane(sequence_of(first, a.s.B, item, lane));
    const int begin = first[w.b], in = item - begin, items = first[w.b + 1] - begin;
    w.splits = a.plan[a.L.splits + w.b];
    w.kvh = in % a.c.n_kv_heads;
    w.split = in / a.c.n_kv_heads % w.splits;
    w.blk = items / a.c.n_kv_heads / w.splits - 1 - in / a.c.n_kv_heads / w.splits;
    w.slot = a.plan[slot_at + w.b] + in;
    return in >= 0 && w.blk >= 0 && (w.splits == 1 || (w.slot >= 0 && w.slot < max_slots));    // (sums over a malformed cu may wrap)
}

// A table entry is fetched well before it is needed and checked where it is: one that is no page becomes page 0 and is reported.
__device__ __forceinline__ int checked_page(const CacheView& c, int p, int32_t* status) {
    if (p >= 0 && p < c.n_pages) return p;
    set_status(status, RADIX_ERR_BAD_PAGE);
    return 0;
}

__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// ------------------------------------------------------------------ few rows
// One block of rows of one kv head; wavefront w takes key tiles w, w + 4, ... of the item's range.  Scores are formed transposed,
// S^T = K Q^T, so that a lane owns a row (column r = lane % 16) and four keys of every 16; which key stands in which row of K is free,
// and is chosen such that the lane ends up with just the keys that the second product O^T = V^T P^T wants from it.
//
// 16-bit: tiles of 32 keys, v_mfma_f32_16x16x32.  Lane (r, g) fetches K[8 (r / 4) + r % 4 (+ 4)][32 ks + 8 g ..] for S^T and, for O^T,
// 16 bytes of each of its keys 8 g .. 8 g + 7: eight elements 8 r .. 8 r + 7 of eight keys, an 8 x 8 square that 32 byte permutes turn
// into what the A operand wants (eight keys of one element).  So V needs no LDS to be transposed.
template <int DT, int NT> struct FewTile {
    static constexpr int KEYS = 32, NA = 8;                                   // NA: accumulators (of four) of a lane per 16 rows
    typedef typename Op<DT>::T T;
    typedef typename Op<DT>::V8 V8;
    V8 q[NT][4];
    struct K { u32x4 k[2][4]; };
    struct V { u32x4 v[8]; };
    struct Where { int pk, pv; };                                             // pages of this lane's keys
    __device__ __forceinline__ void load_q(const T* row, int nt, bool valid, int hd, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            uint4 x = {0, 0, 0, 0};
            if (valid) x = *reinterpret_cast<const uint4*>(row + 32 * ks + 8 * g);
            q[nt][ks] = *reinterpret_cast<V8*>(&x);
        }
    }
    static __device__ __forceinline__ Where where(const CacheView& c, const int32_t* table, int t, int last, int lane) {
        const int kk = min(32 * t + 8 * ((lane & 15) >> 2), last), kv = min(32 * t + 8 * (lane >> 4), last);
        return {table[kk >> c.page_shift], table[kv >> c.page_shift]};
    }
    // rows past the end of the sequence are replaced by its last one: what lies behind it in the page is never read
    static __device__ __forceinline__ void load_k(K& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  int32_t* status) {
        const int r = lane & 15, g = lane >> 4, k0 = 32 * t + 8 * (r >> 2) + (r & 3), mask = c.page_size - 1;
        const char* kp = base + (size_t)checked_page(c, w.pk, status) * c.page_bytes + 16 * g;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t row = (uint32_t)(min(k0 + 4 * kb, last) & mask) * 256u;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) x.k[kb][ks] = *reinterpret_cast<const u32x4*>(kp + row + 64 * ks);
        }
    }
    static __device__ __forceinline__ void load_v(V& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  int32_t* status) {
        const int r = lane & 15, v0 = 32 * t + 8 * (lane >> 4), mask = c.page_size - 1;
        const char* vp = base + (size_t)checked_page(c, w.pv, status) * c.page_bytes + (size_t)c.n_kv_heads * c.piece_bytes + 16 * r;
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = *reinterpret_cast<const u32x4*>(vp + (uint32_t)(min(v0 + i, last) & mask) * 256u);
    }
    // s[u]: score of key 8 g + u of the tile
    __device__ __forceinline__ void scores(const K& x, int nt, float (&s)[8]) const {
        f32x4 a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) a[kb] = Op<DT>::mfma16(*reinterpret_cast<const V8*>(&x.k[kb][ks]), q[nt][ks], a[kb]);
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u] = a[u >> 2][u & 3];
    }
    static constexpr int N_KEYS = 8;                                          // keys of a lane per tile
    static __device__ __forceinline__ int key_of(int t, int u, int lane) { return 32 * t + 8 * (lane >> 4) + u; }
    struct Vt { V8 v[8]; };
    static __device__ __forceinline__ void transpose(const V& x, Vt& y) {
        #pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t o[4];
#pragma unroll
            for (int d = 0; d < 4; ++d)
                o[d] = __builtin_amdgcn_perm(x.v[2 * d + 1][e / 2], x.v[2 * d][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            y.v[e] = *reinterpret_cast<V8*>(o);
        }
    }
    // acc[4 e + i]: element 8 (4 g + i) + e of row r
    static __device__ __forceinline__ void accumulate(const Vt& y, const float (&p)[8], f32x4 (&acc)[8]) {
        V8 pp;
#pragma unroll
        for (int u = 0; u < 8; ++u) pp[u] = (T)p[u];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = Op<DT>::mfma16(y.v[e], pp, acc[e]);
    }
    static __device__ __forceinline__ int element_of(int a, int i, int lane) { return 8 * (4 * (lane >> 4) + i) + a; }
};

// fp32: tiles of 16 keys, v_mfma_f32_16x16x4.  Step (j, u) of the first product takes element 16 j + 4 g + u of a row, so that a lane
// reads four consecutive elements at a time; step e of the second takes key 4 g + e, the lane's own.
template <int HC> struct FewTileF32 {                                         // head_dim <= 64 HC, a multiple of 4
    static constexpr int KEYS = 16, NA = 4 * HC, NJ = 4 * HC;
    typedef float T;
    f32x4 q[1][NJ];
    struct K { f32x4 k[NJ]; };
    struct V { f32x4 v[4][HC]; };
    struct Where { int pk, pv; };
    __device__ __forceinline__ void load_q(const float* row, int, bool valid, int hd, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            q[0][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (valid && 16 * j + 4 * g < hd) q[0][j] = *reinterpret_cast<const f32x4*>(row + 16 * j + 4 * g);
        }
    }
    static __device__ __forceinline__ Where where(const CacheView& c, const int32_t* table, int t, int last, int lane) {
        const int p = table[min(16 * t, last) >> c.page_shift];                             // pages hold a multiple of 16 keys
        return {p, p};
    }
    static __device__ __forceinline__ void load_k(K& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  int32_t* status) {
        const int g = lane >> 4;
        const float* kr = reinterpret_cast<const float*>(base + (size_t)checked_page(c, w.pk, status) * c.page_bytes) +
                          (size_t)(min(16 * t + (lane & 15), last) & (c.page_size - 1)) * hd;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            x.k[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (16 * j + 4 * g < hd) x.k[j] = *reinterpret_cast<const f32x4*>(kr + 16 * j + 4 * g);
        }
    }
    static __device__ __forceinline__ void load_v(V& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  int32_t* status) {
        const int r = lane & 15, g = lane >> 4;
        const float* vp = reinterpret_cast<const float*>(base + (size_t)checked_page(c, w.pv, status) * c.page_bytes +
                                                         (size_t)c.n_kv_heads * c.piece_bytes);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float* vr = vp + (size_t)(min(16 * t + 4 * g + e, last) & (c.page_size - 1)) * hd;
#pragma unroll
            for (int h = 0; h < HC; ++h) {
                x.v[e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (64 * h + 4 * r < hd) x.v[e][h] = *reinterpret_cast<const f32x4*>(vr + 64 * h + 4 * r);
            }
        }
    }
    __device__ __forceinline__ void scores(const K& x, int, float (&s)[4]) const {
        f32x4 a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int u = 0; u < 4; ++u) a[u & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[j][u], q[0][j][u], a[u & 1], 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = a[0][u] + a[1][u];
    }
    static constexpr int N_KEYS = 4;
    static __device__ __forceinline__ int key_of(int t, int u, int lane) { return 16 * t + 4 * (lane >> 4) + u; }
    typedef V Vt;                                                             // one element of one key is what an operand holds
    static __device__ __forceinline__ void transpose(const V& x, Vt& y) { y = x; }
    // acc[4 h + u][i]: element 64 h + 4 (4 g + i) + u of row r
    static __device__ __forceinline__ void accumulate(const Vt& x, const float (&p)[4], f32x4 (&acc)[4 * HC]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < HC; ++h)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    acc[4 * h + u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[e][h][u], p[e], acc[4 * h + u], 0, 0, 0);
    }
    static __device__ __forceinline__ int element_of(int a, int i, int lane) { return 64 * (a >> 2) + 4 * (4 * (lane >> 4) + i) + (a & 3); }
};

template <typename Tile, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 2 : 1) void paged_few_kernel(PagedArgs a, const typename Tile::T* __restrict__ q,
                                                           typename Tile::T* __restrict__ out, int32_t* status) {
    typedef typename Tile::T T;
    constexpr int NA = Tile::NA;
    constexpr int ROWS = 16 * NT, PITCH = MAX_HD + 4;
    __shared__ float so[4][ROWS][PITCH];
    __shared__ float sm[4][ROWS], sl[4][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15;
    PagedItem w;
    if (!paged_item(a, a.L.item_few, a.L.slot_few, a.L.few_slots, blockIdx.x, lane, w)) return;
    const PagedSeq sq = paged_seq(a.c, a.s, a.cu, a.past, a.slots, w.b);
    const int hd = a.c.head_dim, group = a.s.n_q_heads / a.c.n_kv_heads, rows = sq.n * group;
    const int row0 = w.blk * ROWS, last = sq.len - 1;
    // the item's tiles: its share of those up to the last position that a row of the block sees
    const int last_row = min(row0 + ROWS, rows) - 1;
    const int tiles = sq.len > 0 ? (sq.past + last_row / group) / Tile::KEYS + 1 : 0;
    const int t0 = (int)((long long)tiles * w.split / w.splits), t1 = (int)((long long)tiles * (w.split + 1) / w.splits);
    const int32_t* table = a.c.table + (size_t)sq.row * a.c.max_pages;
    const char* base = a.c.pages + (size_t)a.layer * a.c.layer_bytes + (size_t)w.kvh * a.c.piece_bytes;

    Tile tile;
    int limit[NT];                                          // last position that this lane's rows see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + 16 * nt + r, j = min(row, last_row) / group, h = w.kvh * group + min(row, last_row) % group;
        limit[nt] = sq.past + j;
        tile.load_q(q + (size_t)(sq.from + j) * a.s.q_stride + (size_t)h * hd, nt, row <= last_row, hd, lane);
    }
    f32x4 acc[NT][NA];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = -INFINITY; l[nt] = 0.f;
#pragma unroll
        for (int e = 0; e < NA; ++e) acc[nt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float sc = 1.4426950408889634f / sqrtf((float)hd);
    // One tile's registers: the next keys are asked for as soon as the scores are formed, the next values as soon as this tile's are
    // turned, so that a tile is on its way nearly all the time; two wavefronts per SIMD keep 128 KB per CU in flight.
    typename Tile::K xk;
    typename Tile::V xv;
    typename Tile::Where at = {};
    int t = t0 + wave;
    if (t < t1) {
        at = Tile::where(a.c, table, t, last, lane);
        Tile::load_k(xk, a.c, base, at, t, last, hd, lane, status);
        Tile::load_v(xv, a.c, base, at, t, last, hd, lane, status);
        if (t + 4 < t1) at = Tile::where(a.c, table, t + 4, last, lane);
    }
    for (; t < t1; t += 4) {
        float s[NT][Tile::N_KEYS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) tile.scores(xk, nt, s[nt]);
        typename Tile::Where next = {};
        if (t + 8 < t1) next = Tile::where(a.c, table, t + 8, last, lane);
        if (t + 4 < t1) Tile::load_k(xk, a.c, base, at, t + 4, last, hd, lane, status);
        float alpha[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < Tile::N_KEYS; ++u) {
                if (Tile::key_of(t, u, lane) > limit[nt]) s[nt][u] = -INFINITY;
                top = fmaxf(top, s[nt][u]);
            }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m[nt], top), m_use = finite_or_zero(m_new);   // a row may see no key of the tile
            alpha[nt] = __builtin_amdgcn_exp2f((m[nt] - m_use) * sc);
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < Tile::N_KEYS; ++u) {
                s[nt][u] = __builtin_amdgcn_exp2f(fmaf(s[nt][u], sc, -m_use * sc));
                sum += s[nt][u];
            }
            l[nt] = fmaf(l[nt], alpha[nt], sum);
            m[nt] = m_new;
        }
        typename Tile::Vt vt;
        Tile::transpose(xv, vt);
        if (t + 4 < t1) Tile::load_v(xv, a.c, base, at, t + 4, last, hd, lane, status);
        at = next;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < NA; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][e][i] *= alpha[nt];
            Tile::accumulate(vt, s[nt], acc[nt]);
        }
    }

    // ---- the four wavefronts' parts, joined in their order
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float lt = l[nt];
        lt += __shfl_xor(lt, 16, 64);
        lt += __shfl_xor(lt, 32, 64);
        if (lane < 16) { sm[wave][16 * nt + r] = m[nt] * sc; sl[wave][16 * nt + r] = lt; }     // m in units of the exponent of two
#pragma unroll
        for (int e = 0; e < NA; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) so[wave][16 * nt + r][Tile::element_of(e, i, lane)] = acc[nt][e][i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * (MAX_HD / 4); i += 256) {
        const int row = i / (MAX_HD / 4), e = i % (MAX_HD / 4) * 4;
        if (row0 + row > last_row || e >= hd) continue;
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, sm[k][row]);
        const float use = finite_or_zero(top);
        float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = __builtin_amdgcn_exp2f(sm[k][row] - use);
            sum = fmaf(f, sl[k][row], sum);
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] = fmaf(f, so[k][row][e + u], o[u]);
        }
        if (w.splits > 1) {
            const size_t at = (size_t)w.slot * ROWS + row;
            *reinterpret_cast<f32x4*>(a.few_acc + at * MAX_HD + e) = f32x4{o[0], o[1], o[2], o[3]};
            if (e == 0) { a.few_ml[2 * at] = top; a.few_ml[2 * at + 1] = sum; }
        } else {
            const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);        // no key at all: zeros; a NaN stays one
            const int grow = row0 + row;
            T* op = out + (size_t)(sq.from + grow / group) * a.s.out_stride + (size_t)(w.kvh * group + grow % group) * hd + e;
            T y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = from_f32<T>(o[u] * inv);
            if (sizeof(T) == 4) *reinterpret_cast<uint4*>(op) = *reinterpret_cast<uint4*>(y);
            else *reinterpret_cast<uint2*>(op) = *reinterpret_cast<uint2*>(y);
        }
    }
}

// ------------------------------------------------------------------ many rows (16-bit, head_dim 128)
// 128 rows of one kv head, 32 per wavefront; key tiles of 64 go global -> LDS without passing registers, two stages.  A wavefront
// fills 16 rows of a tile, which lie in one page (pages hold a multiple of 16 keys).  The products are formed as in the full-layout
// kernel: S^T = K Q^T with 32x32x16 matrix instructions, so that a lane owns one row; O^T = V^T P^T with V^T read by transposing reads.
typedef __attribute__((ext_vector_type(4))) short s16x4;

template <int DT>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(PagedArgs a, const typename Op<DT>::T* __restrict__ q,
                                                            typename Op<DT>::T* __restrict__ out, int32_t* status) {
    typedef typename Op<DT>::T T;
    typedef typename Op<DT>::V8 V8;
    typedef typename Op<DT>::V4 V4;
    constexpr int HD = MAX_HD, BKV = MANY_TILE;
    __shared__ uint4 Ks[2][BKV * 16];                        // chunk (8 elements) ^= key & 15
    __shared__ uint4 Vs[2][BKV * 16];                        // chunk ^= (key & 3) << 2
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;
    PagedItem w;
    if (!paged_item(a, a.L.item_many, a.L.slot_many, a.L.many_slots, blockIdx.x, lane, w)) return;
    const PagedSeq sq = paged_seq(a.c, a.s, a.cu, a.past, a.slots, w.b);
    const int group = a.s.n_q_heads / a.c.n_kv_heads, rows = sq.n * group;
    const int row0 = w.blk * MANY_ROWS, last_row = min(row0 + MANY_ROWS, rows) - 1;
    const int tiles = sq.len > 0 ? (sq.past + last_row / group) / BKV + 1 : 0;
    const int t0 = (int)((long long)tiles * w.split / w.splits), t1 = (int)((long long)tiles * (w.split + 1) / w.splits);
    const int32_t* table = a.c.table + (size_t)sq.row * a.c.max_pages;
    const char* base = a.c.pages + (size_t)a.layer * a.c.layer_bytes + (size_t)w.kvh * a.c.piece_bytes;
    const int last = sq.len - 1;

    // the wavefront's rows and the positions that its first and last one see
    const int wrow = row0 + 32 * wave;
    const int qmin = sq.past + min(wrow, last_row) / group;
    const int qmax = wrow <= last_row ? sq.past + min(wrow + 31, last_row) / group : -1;
    const int my_row = min(wrow + n, last_row), my_tok = my_row / group, my_head = w.kvh * group + my_row % group;
    const int limit = sq.past + my_tok;

    const int lrow = lane >> 4, lpc = lane & 15;
    auto page_of = [&](int t) { return table[min(t * BKV + 16 * wave, last) >> a.c.page_shift]; };
    auto issue = [&](int t, int entry, int stage) {
        const int page = checked_page(a.c, __builtin_amdgcn_readfirstlane(entry), status);
        const char* kb = base + (size_t)page * a.c.page_bytes;
        const char* vb = kb + (size_t)a.c.n_kv_heads * a.c.piece_bytes;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int rr = 16 * wave + 4 * j + lrow;
            const uint32_t rb = (uint32_t)(min(t * BKV + rr, last) & (a.c.page_size - 1)) * 256u;
            dma16(kb, rb + 16u * (uint32_t)(lpc ^ (rr & 15)), lds_addr(&Ks[stage][(16 * wave + 4 * j) * 16]));
            dma16(vb, rb + 16u * (uint32_t)(lpc ^ ((rr & 3) << 2)), lds_addr(&Vs[stage][(16 * wave + 4 * j) * 16]));
        }
    };
    int page_next = 0;
    if (t0 < t1) {
        issue(t0, page_of(t0), 0);
        if (t0 + 1 < t1) page_next = page_of(t0 + 1);
    }
    V8 qf[8];
    {
        const uint4* qp = reinterpret_cast<const uint4*>(q + (size_t)(sq.from + my_tok) * a.s.q_stride + (size_t)my_head * HD);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
            uint4 v = qp[ks * 2 + g];
            qf[ks] = *reinterpret_cast<V8*>(&v);
        }
    }
    f32x16 o[4];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const float sc = 1.4426950408889634f / sqrtf((float)HD);
    const int tr_e = (lane >> 2) & 3, tr_a = lane & 3, tr_half = (lane >> 4) & 1;
    const uint32_t tr_key0 = (uint32_t)(4 * g + tr_e) * 256u + (uint32_t)(tr_a & 1) * 8u;
    const int tr_chunk0 = 2 * tr_half + (tr_a >> 1);

    for (int t = t0; t < t1; ++t) {
        const int st = (t - t0) & 1, kv0 = t * BKV;
        wait_vmcnt<0>();                                     // this wavefront's share of tile t has landed
        __syncthreads();                                     // everybody's has, and everybody is done with tile t - 1
        if (t + 1 < t1) issue(t + 1, page_next, st ^ 1);
        if (t + 2 < t1) page_next = page_of(t + 2);
        if (kv0 > qmax) continue;                            // the whole tile is in this wavefront's future
        f32x16 s[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
        {
            uint4 kf[16];
            auto read_k = [&](int u) {
                const int key = (u & 1) * 32 + n;
                kf[u] = Ks[st][key * 16 + (((u >> 1) * 2 + g) ^ (key & 15))];
            };
#pragma unroll
            for (int u = 0; u < 4; ++u) read_k(u);
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                if (u + 4 < 16) read_k(u + 4 < 16 ? u + 4 : 0);
                s[u & 1] = Op<DT>::mfma(*reinterpret_cast<V8*>(&kf[u]), qf[u >> 1], s[u & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        s16x4 vlo[16], vhi[16];
        auto read_v = [&](int u) {
            const char* vt = (const char*)&Vs[st][0];
            const int kk = u >> 2, b = u & 3;
            const uint32_t off = tr_key0 + (uint32_t)kk * 4096u + (uint32_t)(((4 * b + tr_chunk0) ^ (tr_e << 2)) << 4);
            vlo[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + off));
            vhi[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + off + 2048u));
        };
#pragma unroll
        for (int u = 0; u < 4; ++u) read_v(u);
        __builtin_amdgcn_sched_barrier(0);
        if (kv0 + BKV - 1 > qmin) {                          // register e of block kb is key kv0 + 32 kb + 8 (e / 4) + 4 g + e % 4
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (kv0 + kb * 32 + 8 * (e >> 2) + 4 * g + (e & 3) > limit) s[kb][e] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m_run, top), m_use = finite_or_zero(m_new);
        const float neg_mc = -m_use * sc;
        float psum = 0.f;
        V8 pf[4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][e], sc, neg_mc));
                psum += p;
                pf[kb * 2 + (e >> 3)][e & 7] = (T)p;
            }
        if (__any(m_new != m_run)) {                         // some row of the wavefront saw a new maximum
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_use) * sc);
            l_run *= alpha;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[b][e] *= alpha;
        }
        l_run += psum;
        m_run = m_new;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            if (u + 4 < 16) read_v(u + 4 < 16 ? u + 4 : 0);
            union { struct { s16x4 lo, hi; } p; V8 v; } cvt;
            cvt.p.lo = vlo[u];
            cvt.p.hi = vhi[u];
            o[u & 3] = Op<DT>::mfma(cvt.v, pf[u >> 2], o[u & 3]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // register e of block b is element 32 b + 8 (e / 4) + 4 g + e % 4
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    if (wrow + n > last_row) return;
    if (w.splits > 1) {
        const size_t at = (size_t)w.slot * MANY_ROWS + 32 * wave + n;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<f32x4*>(a.many_acc + at * HD + b * 32 + q4 * 8 + g * 4) =
                    f32x4{o[b][q4 * 4], o[b][q4 * 4 + 1], o[b][q4 * 4 + 2], o[b][q4 * 4 + 3]};
        if (g == 0) { a.many_ml[2 * at] = m_run * sc; a.many_ml[2 * at + 1] = l_tot; }
        return;
    }
    const float inv = l_tot > 0.f ? 1.0f / l_tot : (l_tot == 0.f ? 0.f : l_tot);
    T* op = out + (size_t)(sq.from + my_tok) * a.s.out_stride + (size_t)my_head * HD;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            V4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (T)(o[b][q4 * 4 + j] * inv);
            *reinterpret_cast<V4*>(op + b * 32 + q4 * 8 + g * 4) = v;
        }
}

// ------------------------------------------------------------------ join
// A wavefront joins the parts of one row of a split block, in the order of the keys; a lane owns two elements.
template <typename T>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, T* __restrict__ out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int hd = a.c.head_dim, group = a.s.n_q_heads / a.c.n_kv_heads;
    const int32_t* first = a.plan + a.L.unit;
    const int units = first[a.s.B];
    for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int b = __builtin_amdgcn_readfirstlane(sequence_of(first, a.s.B, unit, lane));
        const PagedSeq sq = paged_seq(a.c, a.s, a.cu, a.past, a.slots, b);
        const int rows = sq.n * group, splits = a.plan[a.L.splits + b];
        const bool few = !a.L.many || rows <= a.L.few_rows;
        const int block = few ? a.L.few_rows : MANY_ROWS;
        const int in = unit - first[b], kvh = in % a.c.n_kv_heads, back = in / a.c.n_kv_heads;
        const int blocks = ceil_div(rows, block), blk = blocks - 1 - back;
        const int row = blk * block + (int)blockIdx.y * 4 + wave;
        if ((int)blockIdx.y * 4 + wave >= block || row >= rows) continue;
        const float* acc = few ? a.few_acc : a.many_acc;
        const float* ml = few ? a.few_ml : a.many_ml;
        const size_t slot0 = (size_t)a.plan[(few ? a.L.slot_few : a.L.slot_many) + b] + (size_t)back * splits * a.c.n_kv_heads + kvh;
        auto at = [&](int k) { return (slot0 + (size_t)k * a.c.n_kv_heads) * block + (row - blk * block); };
        float top = -INFINITY;
        for (int k = lane; k < splits; k += 64) top = fmaxf(top, ml[2 * at(k)]);
        top = wave_max(top);
        const float use = finite_or_zero(top);
        float sum = 0.f, o0 = 0.f, o1 = 0.f;
        const int e = 2 * lane < hd ? 2 * lane : hd - 2;
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            const size_t i = at(k);
            const float f = __builtin_amdgcn_exp2f(ml[2 * i] - use);
            sum = fmaf(f, ml[2 * i + 1], sum);
            o0 = fmaf(f, acc[i * MAX_HD + e], o0);
            o1 = fmaf(f, acc[i * MAX_HD + e + 1], o1);
        }
        const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);
        T* op = out + (size_t)(sq.from + row / group) * a.s.out_stride + (size_t)(kvh * group + row % group) * hd;
        if (2 * lane < hd) { op[e] = from_f32<T>(o0 * inv); op[e + 1] = from_f32<T>(o1 * inv); }
    }
}

}  // namespace

PagedLayout paged_layout(const CacheView& c, int dtype, const PagedShape& s) {
    PagedLayout L;
    const int group = s.n_q_heads / c.n_kv_heads;
    const long long most_rows = (long long)s.max_new * group;
    L.few_rows = dtype == RADIX_F32 || most_rows <= 16 ? 16 : 32;
    L.few_tile = dtype == RADIX_F32 ? 16 : 32;
    L.many = dtype != RADIX_F32 && most_rows > L.few_rows;
    const long long N = s.N, B = s.B, kv = c.n_kv_heads;
    // blocks of sequence b: at most rows / block + 1, and none without tokens
    const long long few_blocks = dtype == RADIX_F32 ? N * group / 16 + B : B, many_blocks = L.many ? N * group / MANY_ROWS + B : 0;
    L.few_items = few_blocks * kv + FEW_TARGET;
    L.many_items = L.many ? many_blocks * kv + MANY_TARGET : 0;
    // a block is split into ceil(tiles / length) > 1 parts, fewer than 2 tiles / length, and the lengths add up to the target
    L.few_slots = 2 * FEW_TARGET;
    L.many_slots = L.many ? 2 * MANY_TARGET : 0;
    L.units = FEW_TARGET + (L.many ? MANY_TARGET : 0);
    if (L.units > (few_blocks + many_blocks) * kv) L.units = (few_blocks + many_blocks) * kv;
    size_t w = 64;
    L.item_few = w; w += (size_t)B + 1;
    L.item_many = w; w += (size_t)B + 1;
    L.unit = w; w += (size_t)B + 1;
    L.slot_few = w; w += (size_t)B;
    L.slot_many = w; w += (size_t)B;
    L.splits = w; w += (size_t)B;
    L.total_words = w;
    size_t off = align_up(w * 4, 256);
    auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes, 256); return o; };
    L.few_acc = take((size_t)L.few_slots * L.few_rows * MAX_HD * 4);
    L.few_ml = take((size_t)L.few_slots * L.few_rows * 8);
    L.many_acc = take((size_t)L.many_slots * MANY_ROWS * MAX_HD * 4);
    L.many_ml = take((size_t)L.many_slots * MANY_ROWS * 8);
    L.total = off;
    return L;
}

void launch_paged_plan(const CacheView& c, const PagedShape& s, const PagedLayout& L, const int32_t* cu, const int32_t* past,
                       const int32_t* slots, void* ws, int32_t* status, hipStream_t stream) {
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(PT), 0, stream, c, s, L, cu, past, slots, (int32_t*)ws, status);
}

int launch_paged_attention(const CacheView& c, int dtype, int layer, const PagedShape& s, const PagedLayout& L, const void* q,
                           const int32_t* cu, const int32_t* past, const int32_t* slots, void* out, void* ws, int32_t* status,
                           hipStream_t stream) {
    char* w = (char*)ws;
    PagedArgs a = {c, s, L, cu, past, slots, layer, (const int32_t*)ws, (float*)(w + L.few_acc), (float*)(w + L.few_ml),
                   (float*)(w + L.many_acc), (float*)(w + L.many_ml)};
    if (L.few_items > 0x7FFFFFFFLL || L.many_items > 0x7FFFFFFFLL) return RADIX_ERR_UNSUPPORTED;
    const dim3 few((unsigned)L.few_items), many((unsigned)L.many_items), block(256);
    const int join_rows = L.many ? MANY_ROWS : L.few_rows;
    const dim3 join((unsigned)(L.units > 1024 ? 1024 : L.units), (unsigned)ceil_div(join_rows, 4));
    if (dtype == RADIX_F32) {
        if (c.head_dim <= 64)
            hipLaunchKernelGGL((paged_few_kernel<FewTileF32<1>, 1>), few, block, 0, stream, a, (const float*)q, (float*)out, status);
        else
            hipLaunchKernelGGL((paged_few_kernel<FewTileF32<2>, 1>), few, block, 0, stream, a, (const float*)q, (float*)out, status);
        hipLaunchKernelGGL(paged_join_kernel<float>, join, block, 0, stream, a, (float*)out);
        return RADIX_OK;
    }
#define RADIX_PAGED(DT)                                                                                                                  \
    do {                                                                                                                                 \
        typedef Op<DT>::T T;                                                                                                             \
        if (L.few_rows == 16) hipLaunchKernelGGL((paged_few_kernel<FewTile<DT, 1>, 1>), few, block, 0, stream, a, (const T*)q, (T*)out, status); \
        else hipLaunchKernelGGL((paged_few_kernel<FewTile<DT, 2>, 2>), few, block, 0, stream, a, (const T*)q, (T*)out, status);           \
        if (L.many) hipLaunchKernelGGL(paged_many_kernel<DT>, many, block, 0, stream, a, (const T*)q, (T*)out, status);                   \
        hipLaunchKernelGGL(paged_join_kernel<T>, join, block, 0, stream, a, (T*)out);                                                     \
    } while (0)
    if (dtype == RADIX_BF16) RADIX_PAGED(RADIX_BF16); else RADIX_PAGED(RADIX_F16);
#undef RADIX_PAGED
    return RADIX_OK;
}
