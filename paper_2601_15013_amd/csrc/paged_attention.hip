// Causal attention of new tokens over a paged key/value cache: a chunk of a prompt, one token of a decoding sequence, or both in
// one batch.  o[i, h] = sum over the positions p <= pos(i) of softmax_p(q[i, h] . K[p, h / group] / sqrt(hd)) V[p, h / group], where the
// new tokens' own keys and values are in the cache already.
//
// Softmax runs online (running maximum m and sum l in fp32, one pass over the keys); the fp32 accumulators of a row are rescaled when
// m grows.  Probabilities are rounded to the operand type for the second product: the sum l is taken before that rounding, so a row's
// error stays at half a step of the type on each term.  fp16 has no exponents for that below 2^-14, and many small weights beside a large
// one add up: there p, l and the accumulators are kept times 2^15, up to which the type goes, so that a weight is rounded by half a step down
// to 2^-29 and by 2^-40 below.  The factor drops out of the quotient.
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

// Most workgroups that the work of few rows / of many rows is split for.
constexpr int FEW_TARGET = 1536, FEW_TARGET_EVEN = 512, MANY_TARGET = 512;
constexpr int MANY_ROWS = 128, MANY_TILE = 64;
constexpr int MAX_HD = 128;
constexpr long long SHARE_BLOCKS = 8192;                 // most blocks of a batch that is searched for common pages: room for their parts

// Up to PLAN_INLINE sequences every workgroup works out the plan by itself, 64 of them at a time; more are planned by a launch of
// their own.  A plan launch took 8 us, a third of a short sequence's call.
constexpr int PLAN_INLINE = 256;

struct PagedArgs {
    CacheView c;
    PagedShape s;
    PagedLayout L;
    const int32_t *cu, *past, *slots;
    int layer;
    int32_t* plan;
    float *few_acc, *few_ml, *many_acc, *many_ml;
};

// What a sequence of the batch has, from device data that may be anything: `from` .. `from + n` lies in [0, N), and len = past + n <=
// what the table's row can hold.  len = 0: nothing to attend to (zeros).
struct PagedSeq { int from, n, len, row, err; };
__device__ __forceinline__ PagedSeq paged_seq(const CacheView& c, const PagedShape& s, const int32_t* cu, const int32_t* past,
                                              const int32_t* slots, int b) {
    const int from = cu[b], to = cu[b + 1];
    const int p = past[b], row = slots ? slots[b] : b;
    PagedSeq q = {0, 0, 0, 0, 0};
    if (from < 0 || to < from || to > s.N || (long long)to - from > s.max_new) { q.err = RADIX_ERR_BAD_CU_SEQLENS; return q; }
    q.from = from;
    q.n = to - from;
    if (p < 0 || q.n == 0) return q;
    if (row < 0 || row >= c.max_seqs) { q.err = RADIX_ERR_BAD_SLOT; return q; }
    if ((long long)p + q.n > (long long)c.max_pages * c.page_size) { q.err = RADIX_ERR_BAD_PAGE; return q; }
    q.row = row;
    q.len = p + q.n;
    return q;
}

// How a sequence is cut: by which kernel, into how many blocks of rows, and tiles of keys up to its last position.
struct PagedCut { bool few; int blocks, tiles; };
__device__ __forceinline__ PagedCut paged_cut(const CacheView& c, const PagedShape& s, const PagedLayout& L, const PagedSeq& q) {
    const int rows = q.n * (s.n_q_heads / c.n_kv_heads);
    PagedCut k;
    k.few = !L.many || rows <= L.few_rows;
    k.blocks = k.few ? (rows + L.few_rows - 1) >> (L.few_rows == 16 ? 4 : 5) : (rows + MANY_ROWS - 1) / MANY_ROWS;
    k.tiles = (q.len >> 4) + ((q.len & 15) != 0);                // of 16 keys
    k.tiles = k.few ? (L.few_tile == 16 ? k.tiles : (k.tiles + 1) >> 1) : (k.tiles + 3) >> 2;
    return k;
}
// Tiles of a split: an even share of the work for the target number of workgroups, and no less than pays for writing and joining the
// parts: 256 keys with few rows, 1024 with many, whose parts of 64 KB cost what six tiles do.  With few rows, which are bound by memory
// and want to be even, a sequence is cut into ceil(tiles / length) parts, with many into floor(tiles / length).
// (The sum of the work is a float: its rounding is covered by the factor, so that the parts of split blocks are fewer than twice the
// target, or than the target, for which there is room.)
__device__ __forceinline__ int split_length(float work, int target, int least) {
    const int share = (int)ceilf(work * (1.0001f / (float)target));
    return share > least ? share : least;
}
__device__ __forceinline__ int few_length(float work, const PagedLayout& L) { return split_length(work, L.few_target, 256 / L.few_tile); }
__device__ __forceinline__ int many_length(float work) { return split_length(work, MANY_TARGET, 1024 / MANY_TILE); }
__device__ __forceinline__ int splits_of(const PagedCut& k, int few_len, int many_len) {
    const unsigned length = k.few ? few_len : many_len;
    const int n = (int)(((unsigned)k.tiles + (k.few ? length - 1 : 0)) / length);
    return n > 1 ? n : 1;
}
// Entries of the join for a split sequence: some rows of a kv head each, which all lie in one block.  With few parts eight rows are joined
// side by side, with more of them one after the other.
constexpr int JOIN_ALONE = 8;
__device__ __forceinline__ int join_step(int splits) { return splits > JOIN_ALONE ? 1 : 8; }
__device__ __forceinline__ int join_rows(bool few, int splits) { return join_step(splits) * (few ? 1 : splits > JOIN_ALONE ? 8 : 4); }
__device__ __forceinline__ int join_entries(bool few, int rows, int kv, int splits) {
    const int step = join_rows(few, splits);
    return splits <= 1 ? 0 : (rows + step - 1) / step * kv;
}

// ------------------------------------------------------------------ sequences that begin with the same pages
// Forks of one prompt hold the same pages, and decoding them one by one reads those once per sequence while most of a 16-row tile is
// empty.  So sequences that stand next to each other in the batch and begin with the same pages form a cluster: their rows share tiles
// over the common keys (all of them before any new token: nothing is masked), then each walks its own keys; the join brings both
// together.  32 query heads over 8 kv heads, 64 tokens behind 3840 common and 160 own keys: 105 us one by one, 59 with the search for
// clusters (12 of them its two launches, which a forward makes once for all its layers); 256 tokens of 16 heads behind 2048 and 32:
// 180 and 72.  Nothing in common: 167 and 179.
//
// One wavefront per sequence: full pages that it has in common with the one before it.
__global__ __launch_bounds__(256) void paged_common_kernel(CacheView c, PagedShape s, PagedLayout L, const int32_t* __restrict__ cu,
                                                           const int32_t* __restrict__ past, const int32_t* __restrict__ slots,
                                                           int32_t* __restrict__ plan) {
    const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= s.B) return;
    int n = 0;
    if (b > 0) {
        const PagedSeq q = paged_seq(c, s, cu, past, slots, b), p = paged_seq(c, s, cu, past, slots, b - 1);
        if (q.len > 0 && p.len > 0 && q.n == p.n && 2 * q.n * (s.n_q_heads / c.n_kv_heads) <= L.few_rows) {
            const int32_t *x = c.table + (size_t)q.row * c.max_pages, *y = c.table + (size_t)p.row * c.max_pages;
            const int limit = min(q.len, p.len) - q.n, pages = limit >> c.page_shift;
            for (n = 0; n < pages; n += 64) {
                const unsigned long long differ = __ballot(n + lane < pages && x[n + lane] != y[n + lane]);
                if (differ) { n += __ffsll((long long)differ) - 1; break; }
            }
            n = min(n, pages);
        }
    }
    if (lane == 0) plan[L.common + b] = n;
}

// Largest v of this and the threads before it, or `carry`; all threads of the workgroup call.
__device__ __forceinline__ int block_max(int v, int carry, int* part /* [PT / 64] in LDS */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v = max(v, u);
    }
    __syncthreads();
    if (lane == 63) part[wave] = v;
    __syncthreads();
    v = max(v, carry);
    for (int w = 0; w < wave; ++w) v = max(v, part[w]);
    return v;
}

// ------------------------------------------------------------------ the plan as a launch of its own (one workgroup)
// Entry 2 b of the list of items is what the cluster that sequence b leads has in common, entry 2 b + 1 the sequence's own keys.
__global__ __launch_bounds__(PT) void paged_plan_kernel(CacheView c, PagedShape s, PagedLayout L, const int32_t* __restrict__ cu,
                                                        const int32_t* __restrict__ past, const int32_t* __restrict__ slots,
                                                        int32_t* __restrict__ plan, int32_t* status) {
    __shared__ long long part[PT / 64];
    __shared__ float work[2][PT / 64];
    __shared__ int top[PT / 64];
    __shared__ int carry;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, group = s.n_q_heads / c.n_kv_heads;
    int32_t *common = plan + L.common, *lead = plan + L.lead, *shared = plan + L.shared, *members = plan + L.members;
    // clusters: runs of sequences that have enough in common with the one before, cut where a block's rows are full
    const int tile_shift = L.few_tile == 16 ? 4 : 5, enough = 256;
    auto goes_on = [&](int b) { return b > 0 && b < s.B && (long long)common[b] << c.page_shift >= enough; };
    if (tid == 0) carry = 0;
    for (int b0 = 0; b0 < s.B; b0 += PT) {
        const int b = b0 + tid;
        __syncthreads();
        const int begin = block_max(L.share && b < s.B && !goes_on(b) ? b : 0, carry, top);         // first sequence of the run
        __syncthreads();
        if (tid == PT - 1) carry = begin;
        if (b < s.B) {
            lead[b] = -1;
            shared[b] = members[b] = 0;
            if (L.share) {
                const int rows = (cu[b + 1] - cu[b]) * group, fit = rows > 0 && 2 * rows <= L.few_rows ? L.few_rows / rows : 1;
                const int at = (b - begin) % fit, first = b - at;
                int n = 1, pages = 0x7FFFFFFF;
                while (n < fit && goes_on(first + n)) { pages = min(pages, common[first + n]); ++n; }
                if (n > 1) {
                    lead[b] = first;
                    shared[b] = (pages << c.page_shift) >> tile_shift;              // whole tiles
                    if (at == 0) members[b] = n;
                }
            }
        }
    }
    __syncthreads();
    float few_work = 0.f, many_work = 0.f;
    for (int b = tid; b < s.B; b += PT) {
        const PagedSeq q = paged_seq(c, s, cu, past, slots, b);
        const PagedCut k = paged_cut(c, s, L, q);
        if (q.err) set_status(status, q.err);
        const float w = ((float)k.blocks * (float)(k.tiles - shared[b]) + (members[b] ? (float)shared[b] : 0.f)) * (float)c.n_kv_heads;
        few_work += k.few ? w : 0.f;
        many_work += k.few ? 0.f : w;
    }
    few_work = wave_sum(few_work);
    many_work = wave_sum(many_work);
    if (lane == 0) { work[0][wave] = few_work; work[1][wave] = many_work; }
    __syncthreads();
    few_work = many_work = 0.f;
    for (int w = 0; w < PT / 64; ++w) { few_work += work[0][w]; many_work += work[1][w]; }
    const int few_len = few_length(few_work, L), many_len = many_length(many_work);
    long long run_items = 0, run_slots = 0, run_rows = 0;               // few in the low half, many in the high half
    for (int b0 = 0; b0 < s.B; b0 += PT) {
        const int b = b0 + tid;
        PagedCut k = {true, 0, 0};
        int rows = 0, splits = 1, splits_shared = 0, parts = 0;         // parts: of a row of the sequence, the common ones included
        if (b < s.B) {
            const PagedSeq q = paged_seq(c, s, cu, past, slots, b);
            k = paged_cut(c, s, L, q);
            k.tiles -= shared[b];
            splits = parts = splits_of(k, few_len, many_len);
            if (lead[b] >= 0) parts += splits_of({true, 1, shared[b]}, few_len, many_len);
            if (members[b]) splits_shared = parts - splits;
            rows = q.n * group;
        }
        const long long items = (long long)k.blocks * c.n_kv_heads * splits, items_shared = (long long)splits_shared * c.n_kv_heads;
        const int sh = k.few ? 0 : 32;
        long long ti, ts, tr;
        const long long i0 = run_items + block_exclusive((items << sh) + items_shared, &ti, part);
        const long long s0 = run_slots + block_exclusive(((parts > 1 ? items : 0) << sh) + items_shared, &ts, part);
        const long long r0 = run_rows + block_exclusive(join_entries(k.few, rows, c.n_kv_heads, parts), &tr, part);
        if (b < s.B) {
            const int few_at = (int)(i0 & 0xffffffffLL), slot_at = (int)(k.few ? s0 & 0xffffffffLL : s0 >> 32);
            plan[L.item_few + 2 * b] = few_at;
            plan[L.item_few + 2 * b + 1] = few_at + (int)items_shared;
            plan[L.item_many + b] = (int)(i0 >> 32);
            plan[L.slot + 2 * b] = slot_at;
            plan[L.slot + 2 * b + 1] = slot_at + (k.few ? (int)items_shared : 0);
            plan[L.splits + 2 * b] = splits_shared;
            plan[L.splits + 2 * b + 1] = splits;
            plan[L.join + b] = (int)r0;
        }
        run_items += ti; run_slots += ts; run_rows += tr;
    }
    if (tid == 0) {
        plan[L.item_few + 2 * s.B] = (int)(run_items & 0xffffffffLL);
        plan[L.item_many + s.B] = (int)(run_items >> 32);
        plan[L.join + s.B] = (int)run_rows;
    }
}

// One entry of the batch's list of items (those of many rows first): its sequence, the entry's number within the sequence, the
// sequence's splits and where its partial results begin.  By a wavefront.
// first: first tile.  common: keys that a cluster shares; its members' rows then stand one after the other as those of one sequence would.
struct PagedFound { PagedSeq q; bool few, common, apart; int in, blocks, splits, slot, first; };       // apart: its results are parts
// From the lists in the workspace.
__device__ __forceinline__ bool paged_listed(const PagedArgs& a, int index, int lane, PagedFound& f) {
    const int32_t* many = a.plan + a.L.item_many;
    const int n_many = many[a.s.B];
    int b, e;
    if (index < n_many) {
        b = __builtin_amdgcn_readfirstlane(sequence_of(many, a.s.B, index, lane));
        e = 2 * b + 1;
        f.in = index - many[b];
    } else {
        const int32_t* few = a.plan + a.L.item_few;
        index -= n_many;
        if (index >= few[2 * a.s.B]) return false;
        e = __builtin_amdgcn_readfirstlane(sequence_of(few, 2 * a.s.B, index, lane));
        b = e >> 1;
        f.in = index - few[e];
    }
    f.common = (e & 1) == 0;
    f.splits = a.plan[a.L.splits + e];
    f.slot = a.plan[a.L.slot + e];
    f.q = paged_seq(a.c, a.s, a.cu, a.past, a.slots, b);
    const PagedCut k = paged_cut(a.c, a.s, a.L, f.q);
    f.few = k.few;
    f.blocks = k.blocks;
    const int shared = a.plan[a.L.shared + b];
    f.first = f.common ? 0 : shared;
    f.apart = f.splits > 1 || shared > 0;
    if (f.common) {
        const int n = f.q.n * a.plan[a.L.members + b];
        f.blocks = 1;
        f.q.len = shared * a.L.few_tile;
        f.q.n = n <= a.s.N - f.q.from ? n : 0;
        if (n * (a.s.n_q_heads / a.c.n_kv_heads) > a.L.few_rows || f.q.n == 0 || f.splits < 1) return false;
    }
    return true;
}
// Worked out on the spot, 64 sequences at a time; the first 64, which are often all, stay in registers between the passes.  Workgroup 0
// reports what cannot be and leaves the join its lists.
__device__ __forceinline__ bool paged_planned(const PagedArgs& a, int index, int lane, PagedFound& f, int32_t* plan, int32_t* status) {
    const int kv = a.c.n_kv_heads, group = a.s.n_q_heads / kv;
    const bool writer = blockIdx.x == 0 && threadIdx.x < 64;
    PagedSeq q;
    PagedCut k;
    auto fetch = [&](int b) {
        q = {0, 0, 0, 0, 0};
        k = {true, 0, 0};
        if (b < a.s.B) {
            q = paged_seq(a.c, a.s, a.cu, a.past, a.slots, b);
            k = paged_cut(a.c, a.s, a.L, q);
        }
    };
    const int last = (a.s.B - 1) & ~63;
    float few_work = 0.f, many_work = 0.f;
#pragma unroll 1
    for (int b0 = last; b0 >= 0; b0 -= 64) {
        fetch(b0 + lane);
        if (writer && q.err) set_status(status, q.err);
        const float w = (float)k.blocks * (float)k.tiles * (float)kv;
        few_work += k.few ? w : 0.f;
        many_work += k.few ? 0.f : w;
    }
    const int few_len = few_length(wave_total(few_work), a.L);
    int many_len = 1;
    bool few = true;
    if (a.L.many) {
        many_len = many_length(wave_total(many_work));
        int n_many = 0;
#pragma unroll 1
        for (int b0 = last; b0 >= 0; b0 -= 64) {
            if (last > 0) fetch(b0 + lane);
            n_many += k.few ? 0 : k.blocks * kv * splits_of(k, 1, many_len);
        }
        n_many = wave_total(n_many);
        few = index >= n_many;
        if (few) index -= n_many;
    }
    int at = 0, at_few = 0, at_many = 0, at_join = 0;
    bool found = false;
    f.common = false;
    f.first = 0;
#pragma unroll 1
    for (int b0 = 0; b0 <= last; b0 += 64) {
        if (b0 > 0) fetch(b0 + lane);
        const int splits = splits_of(k, few_len, many_len);
        const int items = k.blocks * kv * splits, parts = splits > 1 ? items : 0;
        const int mine = k.few == few ? items : 0;
        const int incl = wave_inclusive(mine) + at;
        const int few_parts = wave_inclusive(k.few ? parts : 0) + at_few;
        int many_parts = at_many;
        if (a.L.many) many_parts += wave_inclusive(k.few ? 0 : parts);
        const int slot = (k.few ? few_parts : many_parts) - parts;
        if (writer) {                                       // (in the form of the plan's own launch: no sequence leads a cluster)
            const int joins = join_entries(k.few, q.n * group, kv, splits), join_incl = wave_inclusive(joins) + at_join;
            if (b0 + lane < a.s.B) {
                plan[a.L.join + b0 + lane + 1] = join_incl;
                plan[a.L.slot + 2 * (b0 + lane) + 1] = slot;
                plan[a.L.splits + 2 * (b0 + lane) + 1] = splits;
                plan[a.L.lead + b0 + lane] = -1;
                if (b0 + lane == 0) plan[a.L.join] = 0;
            }
            at_join = __builtin_amdgcn_readlane(join_incl, 63);
        }
        const unsigned long long hit = __ballot(index < incl && index >= incl - mine);
        if (hit && !found) {
            const int l = __ffsll((long long)hit) - 1;
            found = true;
            f.few = __builtin_amdgcn_readlane((int)k.few, l) != 0;
            f.in = index - __builtin_amdgcn_readlane(incl - mine, l);
            f.blocks = __builtin_amdgcn_readlane(k.blocks, l);
            f.splits = __builtin_amdgcn_readlane(splits, l);
            f.apart = f.splits > 1;
            f.slot = __builtin_amdgcn_readlane(slot, l);
            f.q.from = __builtin_amdgcn_readlane(q.from, l);
            f.q.n = __builtin_amdgcn_readlane(q.n, l);
            f.q.len = __builtin_amdgcn_readlane(q.len, l);
            f.q.row = __builtin_amdgcn_readlane(q.row, l);
            if (!writer) break;
        }
        at = __builtin_amdgcn_readlane(incl, 63);
        at_few = __builtin_amdgcn_readlane(few_parts, 63);
        at_many = __builtin_amdgcn_readlane(many_parts, 63);
    }
    return found;
}
// (sums over a malformed cu_seqlens may have wrapped: nothing leaves the lists' room)
__device__ __forceinline__ bool paged_find(const PagedArgs& a, int lane, PagedFound& f, int32_t* status) {
    const bool found = a.s.B > PLAN_INLINE || a.L.share ? paged_listed(a, blockIdx.x, lane, f) : paged_planned(a, blockIdx.x, lane, f, a.plan, status);
    if (!found) return false;
    const long long items = (long long)f.blocks * a.c.n_kv_heads * f.splits;
    return f.in >= 0 && f.in < items && (!f.apart || (f.slot >= 0 && f.slot + items <= (f.few ? a.L.few_slots : a.L.many_slots)));
}

// A work item: the kv head, block and split of a sequence; `slot` of its partial result where the block is split.
// Items of a sequence: kv heads fastest, so that consecutive workgroups - and with them the eight XCDs - take different heads, and
// the blocks of one head, which read the same keys, meet in one L2; then the splits; then the blocks, the last (longest) first.
struct PagedItem { PagedSeq q; int kvh, blk, split, splits, slot, first; bool common, apart; };
__device__ __forceinline__ PagedItem paged_item(const PagedArgs& a, const PagedFound& f) {
    auto u = [](int x) { return __builtin_amdgcn_readfirstlane(x); };        // the same in all lanes, which not every path tells
    const int kv = a.c.n_kv_heads, in = u(f.in), splits = u(f.splits), rest = in / kv;
    PagedItem w;
    w.q = {u(f.q.from), u(f.q.n), u(f.q.len), u(f.q.row), 0};
    w.kvh = in - rest * kv;
    w.splits = splits;
    w.split = rest % splits;
    w.blk = u(f.blocks) - 1 - rest / splits;
    w.slot = u(f.slot) + in;
    w.first = u(f.first);
    w.common = u((int)f.common) != 0;
    w.apart = u((int)f.apart) != 0;
    return w;
}

// A table entry is fetched well before it is needed and checked where it is: one that is no page becomes page 0 and is noted in `bad`.
__device__ __forceinline__ uint32_t checked_page(const CacheView& c, int p, uint32_t& bad) {
    const bool ok = (uint32_t)p < (uint32_t)c.n_pages;
    bad |= ok ? 0u : 1u;
    return ok ? (uint32_t)p : 0u;
}
__device__ __forceinline__ const char* page_at(const CacheView& c, const char* base, int p, uint32_t& bad) {
    return base + (uint64_t)checked_page(c, p, bad) * (uint32_t)c.page_bytes;        // pages are smaller than 2^31 bytes
}

// Tiles are dealt to the parts evenly, the first ones one more where it does not come out.
__device__ __forceinline__ int part_begin(int tiles, int part, int parts) {
    const int per = (int)((unsigned)tiles / (unsigned)parts), more = tiles - per * parts;
    return part * per + min(part, more);
}

// Probabilities of an operand type are kept times 2^WEIGHT_BITS.
template <typename T> constexpr float WEIGHT_BITS = 0.f;
template <> constexpr float WEIGHT_BITS<f16_t> = 15.f;

// A score (in units of the exponent of two) below it is rounded in fp32 by 2^-13 at the most, which changes p by a sixth of half a step of fp16.
constexpr float FAR = 4096.f;

__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// ------------------------------------------------------------------ few rows
// One block of rows of one kv head; wavefront w takes key tiles w, w + 4, ... of the item's range.  Scores are formed transposed,
// S^T = K Q^T, so that a lane owns a row (column r = lane % 16) and four keys of every 16; which key stands in which row of K is free,
// and is chosen such that the lane ends up with just the keys that the second product O^T = V^T P^T wants from it.
//
// 16-bit: tiles of 32 keys, v_mfma_f32_16x16x32.  Lane (r, g) fetches K[8 (r / 4) + r % 4 (+ 4)][32 ks + 8 g ..] for S^T and, for O^T,
// 16 bytes of each of its keys 8 g .. 8 g + 7: eight elements 8 r .. 8 r + 7 of eight keys, an 8 x 8 square that 32 byte permutes turn
// into what the A operand wants (eight keys of one element).  So V needs no LDS to be transposed.
//
// Measured, kernel alone: 64 tokens behind 500 to 4000 keys, 32 heads over 8, bf16 (593 MB): 97 us, 6.1 TB/s; one token behind 131071 keys,
// fp16 (537 MB): 83 us, 6.5 TB/s; one behind 200 keys: 7.8 us.
template <int DT, int NT> struct FewTile {
    static constexpr int KEYS = 32, NA = 8, WAVES = NT == 1 ? 3 : 2;          // NA: accumulators (of four) of a lane per 16 rows; WAVES: per SIMD
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
    // Eight keys in a row lie in one page, so one address and offsets will do.  Rows past the end of the sequence, which its last page may
    // have, are loaded with the others and have no part: their scores are masked, their values cleared.  A sequence's keys and values are
    // read once: non-temporal loads, with which a plain loop reads 6.9 TB/s of a large buffer, 6.1 without.  KEEP: common ones, which other
    // clusters read too, stay in L2 (70 -> 59 us for 64 tokens behind 3840 common keys); not in batches that hold chunks as well.
    template <bool KEEP> static __device__ __forceinline__ u32x4 fetch(const char* p) {
        const u32x4* v = reinterpret_cast<const u32x4*>(p);
        if constexpr (KEEP) return *v;
        return __builtin_nontemporal_load(v);
    }
    template <bool KEEP> static __device__ __forceinline__ void load_k(K& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  uint32_t& bad) {
        const int r = lane & 15, k0 = 32 * t + 8 * (r >> 2) + (r & 3);
        const char* p = page_at(c, base, w.pk, bad) + ((uint32_t)(k0 & (c.page_size - 1)) * 256u + 16u * (lane >> 4));
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) x.k[kb][ks] = fetch<KEEP>(p + 1024 * kb + 64 * ks);
    }
    template <bool KEEP> static __device__ __forceinline__ void load_v(V& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  uint32_t& bad) {
        const int v0 = 32 * t + 8 * (lane >> 4);
        const char* p = page_at(c, base + (size_t)c.n_kv_heads * c.piece_bytes, w.pv, bad) +
                        ((uint32_t)(v0 & (c.page_size - 1)) * 256u + 16u * (lane & 15));
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = fetch<KEEP>(p + 256 * i);
    }
    static __device__ __forceinline__ void clear_past(V& x, int t, int last, int lane) {
        if (32 * t + 31 <= last) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (32 * t + 8 * (lane >> 4) + i > last) x.v[i] = u32x4{0, 0, 0, 0};
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
    // acc[e][i]: element 8 (4 g + i) + e of row r
    static __device__ __forceinline__ void accumulate(const V& x, const float (&p)[NT][8], f32x4 (&acc)[NT][8]) {
        V8 pp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < 8; ++u) pp[nt][u] = (T)p[nt][u];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u32x4 o;
#pragma unroll
            for (int d = 0; d < 4; ++d)
                o[d] = __builtin_amdgcn_perm(x.v[2 * d + 1][e / 2], x.v[2 * d][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            const V8 vt = *reinterpret_cast<V8*>(&o);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][e] = Op<DT>::mfma16(vt, pp[nt], acc[nt][e]);
            __builtin_amdgcn_sched_barrier(0);                                // (or all eight squares are turned first, in 28 more registers)
        }
    }
    static __device__ __forceinline__ int element_of(int a, int i, int lane) { return 8 * (4 * (lane >> 4) + i) + a; }
};

// fp32: tiles of 16 keys, v_mfma_f32_16x16x4.  Step (j, u) of the first product takes element 16 j + 4 g + u of a row, so that a lane
// reads four consecutive elements at a time; step e of the second takes key 4 g + e, the lane's own.  8 sequences of 1 to 60 tokens
// behind 100 to 450, 4 heads of 64 over 2: 10.2 us.
template <int HC> struct FewTileF32 {                                         // head_dim <= 64 HC, a multiple of 4
    static constexpr int KEYS = 16, NA = 4 * HC, NJ = 4 * HC, WAVES = 3;
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
    template <bool KEEP> static __device__ __forceinline__ void load_k(K& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  uint32_t& bad) {
        const int g = lane >> 4;
        const float* kr = reinterpret_cast<const float*>(page_at(c, base, w.pk, bad)) +
                          (size_t)(min(16 * t + (lane & 15), last) & (c.page_size - 1)) * hd;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            x.k[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (16 * j + 4 * g < hd) x.k[j] = *reinterpret_cast<const f32x4*>(kr + 16 * j + 4 * g);
        }
    }
    template <bool KEEP> static __device__ __forceinline__ void load_v(V& x, const CacheView& c, const char* base, Where w, int t, int last, int hd, int lane,
                                                  uint32_t& bad) {
        const int r = lane & 15, g = lane >> 4;
        const float* vp = reinterpret_cast<const float*>(page_at(c, base + (size_t)c.n_kv_heads * c.piece_bytes, w.pv, bad));
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
    static __device__ __forceinline__ void clear_past(V&, int, int, int) {}      // (loads of rows past the end take the last row instead)
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
    // acc[4 h + u][i]: element 64 h + 4 (4 g + i) + u of row r
    static __device__ __forceinline__ void accumulate(const V& x, const float (&p)[1][4], f32x4 (&acc)[1][4 * HC]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < HC; ++h)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    acc[0][4 * h + u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[e][h][u], p[0][e], acc[0][4 * h + u], 0, 0, 0);
    }
    static __device__ __forceinline__ int element_of(int a, int i, int lane) { return 64 * (a >> 2) + 4 * (4 * (lane >> 4) + i) + (a & 3); }
};

template <typename Tile, int NT> struct FewShared {
    float o[4][16 * NT][MAX_HD + 4];
    float m[4][16 * NT], l[4][16 * NT];
};
template <typename Tile, int NT, bool KEEP>
__device__ __forceinline__ void few_rows(const PagedArgs& a, const PagedItem& w, const typename Tile::T* __restrict__ q,
                                         typename Tile::T* __restrict__ out, FewShared<Tile, NT>& sh, int32_t* status) {
    typedef typename Tile::T T;
    constexpr int NA = Tile::NA, ROWS = 16 * NT;
    auto &so = sh.o;
    auto &sm = sh.m, &sl = sh.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15;
    const PagedSeq& sq = w.q;
    const int past = sq.len - sq.n;                         // (len = 0: unused)
    const int hd = a.c.head_dim, group = a.s.n_q_heads / a.c.n_kv_heads, rows = sq.n * group;
    const int row0 = w.blk * ROWS, last = sq.len - 1;
    // the item's tiles: its share of those up to the last position that a row of the block sees
    const int last_row = min(row0 + ROWS, rows) - 1;
    const int tiles = w.common ? sq.len / Tile::KEYS : sq.len > 0 ? (past + last_row / group) / Tile::KEYS + 1 : 0;
    const int t0 = w.first + part_begin(tiles - w.first, w.split, w.splits), t1 = w.first + part_begin(tiles - w.first, w.split + 1, w.splits);
    const int32_t* table = a.c.table + (size_t)sq.row * a.c.max_pages;
    const char* base = a.c.pages + (size_t)a.layer * a.c.layer_bytes + (size_t)w.kvh * a.c.piece_bytes;

    Tile tile;
    int limit[NT];                                          // last position that this lane's rows see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + 16 * nt + r, j = min(row, last_row) / group, h = w.kvh * group + min(row, last_row) % group;
        limit[nt] = w.common ? last : past + j;
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
    // used, so that a tile is on its way nearly all the time; three wavefronts per SIMD keep 192 KB per CU in flight.
    typename Tile::K xk;
    typename Tile::V xv;
    typename Tile::Where at = {};
    uint32_t bad = 0;
    int t = t0 + wave;
    if (t < t1) {
        at = Tile::where(a.c, table, t, last, lane);
        Tile::template load_k<KEEP>(xk, a.c, base, at, t, last, hd, lane, bad);
        Tile::template load_v<KEEP>(xv, a.c, base, at, t, last, hd, lane, bad);
        if (t + 4 < t1) at = Tile::where(a.c, table, t + 4, last, lane);
    }
    for (; t < t1; t += 4) {
        float s[NT][Tile::N_KEYS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) tile.scores(xk, nt, s[nt]);
        typename Tile::Where next = {};
        if (t + 8 < t1) next = Tile::where(a.c, table, t + 8, last, lane);
        if (t + 4 < t1) Tile::template load_k<KEEP>(xk, a.c, base, at, t + 4, last, hd, lane, bad);
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
                s[nt][u] = __builtin_amdgcn_exp2f(fmaf(s[nt][u] - m_use, sc, WEIGHT_BITS<T>));
                sum += s[nt][u];
            }
            l[nt] = fmaf(l[nt], alpha[nt], sum);
            m[nt] = m_new;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < NA; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][e][i] *= alpha[nt];
        Tile::clear_past(xv, t, last, lane);
        Tile::accumulate(xv, s, acc);
        if (t + 4 < t1) Tile::template load_v<KEEP>(xv, a.c, base, at, t + 4, last, hd, lane, bad);
        at = next;
    }
    if (bad) set_status(status, RADIX_ERR_BAD_PAGE);

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
        if (w.apart) {
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
// Bound as that one is, by how far matrix instructions, softmax arithmetic and LDS reads overlap: chunks of 900 to 1100 tokens behind
// 2000 to 8000, 32 heads over 8, fp16: 430 to 458 us by the card, 789 to 740 TFLOP/s.
typedef __attribute__((ext_vector_type(4))) short s16x4;

struct ManyShared {
    uint4 K[2][MANY_TILE * 16];                              // chunk (8 elements) ^= key & 15
    uint4 V[2][MANY_TILE * 16];                              // chunk ^= (key & 3) << 2
};
template <int DT>
__device__ __forceinline__ void many_rows(const PagedArgs& a, const PagedItem& w, const typename Op<DT>::T* __restrict__ q,
                                          typename Op<DT>::T* __restrict__ out, ManyShared& sh, int32_t* status) {
    typedef typename Op<DT>::T T;
    typedef typename Op<DT>::V8 V8;
    typedef typename Op<DT>::V4 V4;
    constexpr int HD = MAX_HD, BKV = MANY_TILE;
    auto &Ks = sh.K, &Vs = sh.V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;
    const PagedSeq& sq = w.q;
    const int past = sq.len - sq.n;                          // (len = 0: unused)
    const int group = a.s.n_q_heads / a.c.n_kv_heads, rows = sq.n * group;
    const int row0 = w.blk * MANY_ROWS, last_row = min(row0 + MANY_ROWS, rows) - 1;
    const int tiles = sq.len > 0 ? (past + last_row / group) / BKV + 1 : 0;
    const int t0 = part_begin(tiles, w.split, w.splits), t1 = part_begin(tiles, w.split + 1, w.splits);
    const int32_t* table = a.c.table + (size_t)sq.row * a.c.max_pages;
    const char* base = a.c.pages + (size_t)a.layer * a.c.layer_bytes + (size_t)w.kvh * a.c.piece_bytes;
    const int last = sq.len - 1;

    // the wavefront's rows and the positions that its first and last one see
    const int wrow = row0 + 32 * wave;
    const int qmin = past + min(wrow, last_row) / group;
    const int qmax = wrow <= last_row ? past + min(wrow + 31, last_row) / group : -1;
    const int my_row = min(wrow + n, last_row), my_tok = my_row / group, my_head = w.kvh * group + my_row % group;
    const int limit = past + my_tok;

    const int lrow = lane >> 4, lpc = lane & 15;
    uint32_t bad = 0;
    auto page_of = [&](int t) { return table[min(t * BKV + 16 * wave, last) >> a.c.page_shift]; };
    auto issue = [&](int t, int entry, int stage) {
        const char* kb = page_at(a.c, base, __builtin_amdgcn_readfirstlane(entry), bad);
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
        // (s - m) sc + WEIGHT_BITS by one fused operation, s sc - mc with mc = m sc - WEIGHT_BITS rounded.  The rounding is common to a row's keys and drops out, but where
        // it reaches whole powers of two the largest p would leave the type, or all of them vanish: beyond FAR the difference is taken first.
        // (Four chunks behind 2000 to 8000 keys: 440 us without the question, 443 with it, 455 with the difference in every tile.)
        float neg_mc = fmaf(-m_use, sc, WEIGHT_BITS<T>);
        if (__builtin_expect(__any(fabsf(neg_mc) > FAR), 0)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[kb][e] -= m_use;
            neg_mc = WEIGHT_BITS<T>;
        }
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
    if (bad) set_status(status, RADIX_ERR_BAD_PAGE);
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

// ------------------------------------------------------------------ the kernels
template <typename Tile, int NT>
__global__ __launch_bounds__(256, Tile::WAVES) void paged_few_kernel(PagedArgs a, const typename Tile::T* __restrict__ q,
                                                                         typename Tile::T* __restrict__ out, int32_t* status) {
    __shared__ FewShared<Tile, NT> sh;
    PagedFound f;
    if (!paged_find(a, threadIdx.x & 63, f, status)) return;
    const PagedItem w = paged_item(a, f);
    if (w.common) few_rows<Tile, NT, true>(a, w, q, out, sh, status);
    else few_rows<Tile, NT, false>(a, w, q, out, sh, status);
}

// Both kinds of items in one launch: the blocks of many rows first, whose work is the longer.
template <int DT>
__global__ __launch_bounds__(256, 2) void paged_mixed_kernel(PagedArgs a, const typename Op<DT>::T* __restrict__ q,
                                                             typename Op<DT>::T* __restrict__ out, int32_t* status) {
    __shared__ union { ManyShared many; FewShared<FewTile<DT, 1>, 1> few; } sh;
    PagedFound f;
    if (!paged_find(a, threadIdx.x & 63, f, status)) return;
    const PagedItem w = paged_item(a, f);
    if (__builtin_amdgcn_readfirstlane((int)f.few)) few_rows<FewTile<DT, 1>, 1, false>(a, w, q, out, sh.few, status);
    else many_rows<DT>(a, w, q, out, sh.many, status);
}

// Joins the parts of split blocks; workgroups take entries in turn.  Groups of 32 lanes, four elements a lane: with few parts a group joins a row by itself, with more
// the eight groups take every eighth part of one row and their sums are added in order.  Bound by latency: 5.1 us for 64 sequences, 4.5 for
// one in 64 parts; one wavefront a row, parts one after the other, took 6.2 and 13.7, and 47 where chunks were split.
struct JoinArgs {
    const int32_t *cu, *first, *splits, *slot, *lead;
    const char* ws;
    uint32_t few_acc, few_ml, many_acc, many_ml;             // bytes from ws
    int B, N, max_new, kv, group, hd, few_rows, few_slots, many_slots, out_stride;
    bool many;
};
template <typename T>
__global__ __launch_bounds__(256) void paged_join_kernel(JoinArgs a, T* __restrict__ out) {
    __shared__ f32x4 so[8][MAX_HD / 4];
    __shared__ float sl[8], sm[4];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 5, e = threadIdx.x & 31;
    const int entries = a.first[a.B];
#pragma unroll 1
    for (int index = blockIdx.x; index < entries; index += gridDim.x) {
        int kv = a.kv, group = a.group;
        asm volatile("" : "+s"(kv), "+s"(group));          // what their divisions need is made anew: held over the loop it would not fit
        const int b = __builtin_amdgcn_readfirstlane(sequence_of(a.first, a.B, index, lane));
        const int in = index - a.first[b], own = a.splits[2 * b + 1], slot = a.slot[2 * b + 1], from = a.cu[b], n = a.cu[b + 1] - from;
        if (from < 0 || n <= 0 || n > a.max_new || from > a.N - n) continue;
        const int rows = n * group, lead = a.lead[b], before = lead >= 0 ? a.splits[2 * lead] : 0, splits = before + own;
        const bool few = !a.many || rows <= a.few_rows, together = splits > JOIN_ALONE;
        const int block = few ? a.few_rows : MANY_ROWS, blocks = (rows + block - 1) / block;
        const int step = join_step(splits), count = join_rows(few, splits);
        const int kvh = in % kv, row0 = in / kv * count, end = min(row0 + count, rows), room = few ? a.few_slots : a.many_slots;
        if (in < 0 || row0 >= rows || slot < 0 || slot + (long long)blocks * kv * own > room) continue;
        // parts 0 .. before - 1: those of the cluster, where the sequence's rows begin at row (b - lead) * rows
        const int lead_slot = lead >= 0 ? a.slot[2 * lead] : 0, lead_row = lead >= 0 ? (b - lead) * rows : 0;
        if (lead_slot < 0 || lead_slot + (long long)kv * before > room || lead_row < 0 || lead_row + rows > (lead >= 0 ? block : rows)) continue;
        const float* acc = reinterpret_cast<const float*>(a.ws + (few ? a.few_acc : a.many_acc));
        const float* ml = reinterpret_cast<const float*>(a.ws + (few ? a.few_ml : a.many_ml));
        // 32 bits hold any place in the parts' room; places in vector registers: there are plenty
        int own_at = (slot + (blocks - 1 - row0 / block) * own * kv + kvh) * block, lead_at = (lead_slot + kvh) * block + lead_row;
        int before_v = before, stride_v = kv * block;
        asm volatile("" : "+v"(own_at), "+v"(lead_at), "+v"(before_v), "+v"(stride_v));
#pragma unroll 1
        for (int r0 = row0; r0 < end; r0 += step) {
            const int row = together ? r0 : r0 + part;
            const bool active = row < end;
            auto at = [&](int k) { return (k < before_v ? lead_at + k * stride_v : own_at + (k - before_v) * stride_v) + (row & (block - 1)); };
            float top = -INFINITY, sum = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            auto add = [&](int k, float use) {
                const int i = at(k);
                const float w = __builtin_amdgcn_exp2f(ml[2 * i] - use);
                const f32x4 x = *reinterpret_cast<const f32x4*>(acc + i * MAX_HD + 4 * e);  // (elements from head_dim on: unused)
                sum = fmaf(w, ml[2 * i + 1], sum);
#pragma unroll
                for (int u = 0; u < 4; ++u) o[u] = fmaf(w, x[u], o[u]);
            };
            if (together) {
                for (int k = threadIdx.x; k < splits; k += 256) top = fmaxf(top, ml[2 * at(k)]);
                top = wave_max(top);
                __syncthreads();                            // the row before is through with LDS
                if (lane == 0) sm[threadIdx.x >> 6] = top;
                __syncthreads();
                const float use = finite_or_zero(fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])));
#pragma unroll 8
                for (int k = part; k < splits; k += 8) add(k, use);
                so[part][e] = o;
                if (e == 0) sl[part] = sum;
                __syncthreads();
                sum = 0.f;
                o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    sum += sl[p];
                    o += so[p][e];
                }
            } else if (active) {
#pragma unroll 4
                for (int k = 0; k < splits; ++k) top = fmaxf(top, ml[2 * at(k)]);
                const float use = finite_or_zero(top);
#pragma unroll 4
                for (int k = 0; k < splits; ++k) add(k, use);
            }
            if (active && (!together || part == 0) && 4 * e < a.hd) {
                const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);
                T* op = out + (size_t)(from + row / group) * a.out_stride + (size_t)(kvh * group + row % group) * a.hd + 4 * e;
                T y[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) y[u] = from_f32<T>(o[u] * inv);
                if (sizeof(T) == 4) *reinterpret_cast<uint4*>(op) = *reinterpret_cast<uint4*>(y);
                else *reinterpret_cast<uint2*>(op) = *reinterpret_cast<uint2*>(y);
            }
        }
    }
}

}  // namespace

PagedLayout paged_layout(const CacheView& c, int dtype, const PagedShape& s) {
    PagedLayout L;
    const int group = s.n_q_heads / c.n_kv_heads;
    const long long most_rows = (long long)s.max_new * group;
    // 16 rows a block, or 32 where the whole batch fits that: then no sequence needs the other kernel.  (Sequences of one token in a batch
    // with chunks: 84 us in blocks of 32 rows, 61 in blocks of 16, whose wavefronts leave room for a second one per SIMD.)
    L.few_rows = dtype != RADIX_F32 && most_rows > 16 && most_rows <= 32 ? 32 : 16;
    L.few_tile = dtype == RADIX_F32 ? 16 : 32;
    L.many = dtype != RADIX_F32 && most_rows > L.few_rows;
    const long long N = s.N, B = s.B, kv = c.n_kv_heads;
    // blocks of sequence b: at most rows / block + 1, and none without tokens
    const long long few_blocks = dtype == RADIX_F32 ? N * group / 16 + B : (B < N ? B : N), many_blocks = L.many ? N * group / MANY_ROWS + B : 0;
    // (ceil(x) < 2 x where it is more than one)
    // With few blocks all parts are of about one length, and two workgroups a CU that are done together beat any more; many blocks of
    // different lengths even out in more parts.  One token behind 131071 keys, 8 kv heads: 88.9 us in 512 parts, 92.9 in 768, 94 in 1024
    // and more; 64 tokens behind 500 to 4000 keys: 121 us for 512, 111 for 1024, 106.6 for 1536, 107.8 for 2048.
    L.few_target = few_blocks * kv < FEW_TARGET_EVEN / 2 ? FEW_TARGET_EVEN : FEW_TARGET;
    // clusters (two sequences at the least have to fit a block): what of them is not split is a part all the same
    const long long shared_blocks = B * kv < SHARE_BLOCKS ? B * kv : SHARE_BLOCKS;
    L.share = s.find_shared && B > 1 && B * kv <= SHARE_BLOCKS && 2 * group <= L.few_rows;
    L.few_slots = 2 * FEW_TARGET + (s.find_shared ? 2 * shared_blocks : 0);
    L.many_slots = L.many ? MANY_TARGET : 0;
    L.items = few_blocks * kv * (L.share ? 2 : 1) + FEW_TARGET + (L.many ? many_blocks * kv + MANY_TARGET : 0);
    // entries of the join: a row at the least; none where a row of the table holds no more than one part (few_length, many_length)
    L.joins = (long long)c.max_pages * c.page_size <= 256 ? 0 : N * s.n_q_heads;
    size_t w = 64;
    auto words = [&](size_t n) { const size_t o = w; w += n; return o; };
    L.item_few = words(2 * (size_t)B + 1);
    L.item_many = words((size_t)B + 1);
    L.join = words((size_t)B + 1);
    L.slot = words(2 * (size_t)B);
    L.splits = words(2 * (size_t)B);
    L.common = words((size_t)B);
    L.lead = words((size_t)B);
    L.shared = words((size_t)B);
    L.members = words((size_t)B);
    size_t off = align_up(w * 4, 256);
    auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes, 256); return o; };
    // 16 rows a block, or 32: room for either from 17 rows on, so that the size grows with max_new (32 is for 17 to 32 rows only)
    const size_t few_room = (size_t)L.few_slots * (dtype != RADIX_F32 && most_rows > 16 ? 32 : 16);
    L.few_acc = take(few_room * MAX_HD * 4);
    L.few_ml = take(few_room * 8);
    L.many_acc = take((size_t)L.many_slots * MANY_ROWS * MAX_HD * 4);
    L.many_ml = take((size_t)L.many_slots * MANY_ROWS * 8);
    L.total = off;
    return L;
}

void launch_paged_plan(const CacheView& c, const PagedShape& s, const PagedLayout& L, const int32_t* cu, const int32_t* past,
                       const int32_t* slots, void* ws, int32_t* status, hipStream_t stream) {
    if (L.share)
        hipLaunchKernelGGL(paged_common_kernel, dim3((unsigned)ceil_div(s.B, 4)), dim3(256), 0, stream, c, s, L, cu, past, slots, (int32_t*)ws);
    if (L.share || s.B > PLAN_INLINE)
        hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(PT), 0, stream, c, s, L, cu, past, slots, (int32_t*)ws, status);
}

int launch_paged_attention(const CacheView& c, int dtype, int layer, const PagedShape& s, const PagedLayout& L, const void* q,
                           const int32_t* cu, const int32_t* past, const int32_t* slots, void* out, void* ws, int32_t* status,
                           hipStream_t stream) {
    char* w = (char*)ws;
    PagedArgs a = {c, s, L, cu, past, slots, layer, (int32_t*)ws, (float*)(w + L.few_acc), (float*)(w + L.few_ml),
                   (float*)(w + L.many_acc), (float*)(w + L.many_ml)};
    if (L.items > MAX_BLOCKS) return RADIX_ERR_UNSUPPORTED;
    const JoinArgs j = {cu, a.plan + L.join, a.plan + L.splits, a.plan + L.slot, a.plan + L.lead, w, (uint32_t)L.few_acc, (uint32_t)L.few_ml,
                        (uint32_t)L.many_acc, (uint32_t)L.many_ml, s.B, s.N, s.max_new,
                        c.n_kv_heads, s.n_q_heads / c.n_kv_heads, c.head_dim, L.few_rows, (int)L.few_slots, (int)L.many_slots, (int)s.out_stride,
                        L.many != 0};
    const dim3 grid((unsigned)L.items), block(256), join((unsigned)(L.joins > 1024 ? 1024 : L.joins));
#define RADIX_PAGED(KERNEL, T)                                                                                       \
    do {                                                                                                             \
        hipLaunchKernelGGL((KERNEL), grid, block, 0, stream, a, (const T*)q, (T*)out, status);                       \
        if (L.joins > 0) hipLaunchKernelGGL((paged_join_kernel<T>), join, block, 0, stream, j, (T*)out);                              \
    } while (0)
#define RADIX_PAGED_16(DT)                                                                                           \
    do {                                                                                                             \
        typedef Op<DT>::T T;                                                                                         \
        if (L.many) RADIX_PAGED(paged_mixed_kernel<DT>, T);                                                          \
        else if (L.few_rows == 16) RADIX_PAGED((paged_few_kernel<FewTile<DT, 1>, 1>), T);                            \
        else RADIX_PAGED((paged_few_kernel<FewTile<DT, 2>, 2>), T);                                                  \
    } while (0)
    if (dtype == RADIX_F32) {
        if (c.head_dim <= 64) RADIX_PAGED((paged_few_kernel<FewTileF32<1>, 1>), float);
        else RADIX_PAGED((paged_few_kernel<FewTileF32<2>, 1>), float);
    } else if (dtype == RADIX_BF16) RADIX_PAGED_16(RADIX_BF16);
    else RADIX_PAGED_16(RADIX_F16);
#undef RADIX_PAGED_16
#undef RADIX_PAGED
    return RADIX_OK;
}
