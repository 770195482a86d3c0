// What a scorer, a reranker or a sampler wants of a row of logits x[0 .. vocab): log-probabilities of given tokens, the entropy of the
// distribution and its k likeliest tokens, in one pass over the row.
//
// With m = max x, S = sum e^(x - m), T = sum (x - m) e^(x - m):  log p(t) = (x_t - m) - log S,  entropy = log S - T / S.
// (m, S, T) are kept online in fp32; to a larger maximum m' they become S a and a (T + (m - m') S) with a = e^(m - m').  T is kept about m
// and not about 0, so that the entropy is no difference of large numbers where all logits are large.
//
// The k likeliest are ordered by value, equal ones by id (a 64-bit key holds both, so no two are equal).  A wavefront keeps a list of
// candidates in LDS and the k-th best value so far: what does not exceed that is dropped by one comparison with the maximum of 16
// values; the rest is appended and the list cut back to k when it is long.  No order of arrival enters the result.
//
// Bound by the row's bytes: 16-byte non-temporal loads, one turn of 16 elements a lane ahead; a row is split over several workgroups where
// there are few rows, whose parts a second launch joins.  2048 rows of 151936 fp32 logits: 199 us, 6.3 TB/s (range checks in every turn
// cost 15 us more, plain loads 33); 8 rows: 9.8 us and 5.5 for the join.
#include "common.h"
#include "kernels.h"

namespace {

typedef unsigned long long u64;
constexpr float LOG2E = 1.4426950408889634f;
// Differences below it count as it in the sums of d e^d: e^d is 0 there, and d may be -inf or so large (a mask of the type's lowest value)
// that a multiple of it is, which would make a NaN of 0 d.
constexpr float FAR = -1e4f;
template <int N> struct Count { static constexpr int value = N; };
constexpr int LIST = 1120;              // 64 kept entries and a batch of 16 for every lane fit

__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// Larger for larger x; a NaN comes last.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);            // -0 counts as 0
    const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return x != x ? 0u : o;
}
// Equal values: larger for the lower id.  Never 0.
__device__ __forceinline__ u64 key_of(float x, int id) { return ((u64)ordered(x) << 32) | (0xFFFFFFFFu - (uint32_t)id); }
// A bound (an ordered value) that at least k lanes' x reach, so that no value below it is among the k largest; the largest one whose lower
// 16 bits are 0.  0 where fewer than k lanes have one above -inf.
__device__ __forceinline__ uint32_t bound_of(float x, int k) {
    const uint32_t o = ordered(x);
    uint32_t bound = 0;
    if (__popcll(__ballot(x > -INFINITY)) < k) return 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t next = bound | (1u << bit);
        if (__popcll(__ballot(o >= next)) >= k) bound = next;
    }
    return bound;
}
__device__ __forceinline__ float value_of(u64 key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ int id_of(u64 key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }
__device__ __forceinline__ u64 read_lane(u64 v, int l) {
    return ((u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, l);
}
// How many of the first n lanes hold a larger key than this one.
__device__ __forceinline__ int rank_of(u64 key, int n) {
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += read_lane(key, j) > key;
    return rank;
}
// The k largest of buf[0 .. c) in descending order, by one wavefront; returns how many there are.  While more than 64 are left: the k-th
// largest of the lanes' maxima is no larger than the k-th largest key, so what lies below it goes; with k <= 32 at least half does.
__device__ int cut_list(u64* buf, int c, int k, int lane) {
    while (c > 64) {
        u64 top = 0;
        for (int i = lane; i < c; i += 64) top = buf[i] > top ? buf[i] : top;
        const int rank = rank_of(top, 64);
        const u64 bound = read_lane(top, __ffsll((long long)__ballot(rank == k - 1)) - 1);
        int kept = 0;
        for (int i0 = 0; i0 < c; i0 += 64) {
            const u64 key = i0 + lane < c ? buf[i0 + lane] : 0;
            const u64 keep = __ballot(key >= bound);
            wave_order();
            if (key >= bound) buf[kept + __popcll(keep & ((1ull << lane) - 1ull))] = key;
            kept += __popcll(keep);
            wave_order();
        }
        c = kept;
    }
    const u64 key = lane < c ? buf[lane] : 0;
    const int rank = rank_of(key, c);
    wave_order();
    if (lane < c && rank < k) buf[rank] = key;
    wave_order();
    return c < k ? c : k;
}

struct Stat { float m, s, t; };
__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    auto add = [&](Stat x, Stat& r) {
        const float d = x.m == m ? 0.f : x.m - m;             // also where both are -inf
        const float f = __builtin_amdgcn_exp2f(d * LOG2E);
        r.s += f * x.s;
        r.t += f * fmaf(fmaxf(d, FAR), x.s, x.t);
    };
    Stat r = {m, 0.f, 0.f};
    add(a, r);
    add(b, r);
    return r;
}

struct Answer {
    const int32_t* given;
    int n_given, k, vocab;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_ids, *status;
};
// The logits of a row's given tokens, one a lane, asked for before the rest of the row is through.
struct Given { int token; float x; };
template <typename T> __device__ __forceinline__ Given ask_given(const Answer& a, const T* x, size_t row, int j) {
    Given g = {-1, 0.f};
    if (j < a.n_given) g.token = a.given[row * a.n_given + j];
    if (g.token >= 0 && g.token < a.vocab) g.x = to_f32<T>(x[g.token]);
    return g;
}
// The row's results from its statistics and its sorted list, by one wavefront.
template <typename T>
__device__ __forceinline__ void answer(const Answer& a, const T* x, size_t row, Stat st, const u64* list, int n, Given g, int lane) {
    const float ls = st.s > 0.f ? logf(st.s) : NAN;           // no finite logit, or a NaN or +inf among them: no distribution
    for (int j = lane; j < a.n_given; j += 64) {
        if (j >= 64) g = ask_given<T>(a, x, row, j);
        float y = 0.f;                                        // token < 0: none
        if (g.token >= a.vocab) { set_status(a.status, RADIX_ERR_BAD_TOKEN); y = NAN; }
        else if (g.token >= 0) y = (g.x - st.m) - ls;
        a.logprobs[row * a.n_given + j] = y;
    }
    if (lane == 0 && a.entropy) a.entropy[row] = ls - st.t / st.s;
    for (int j = lane; j < a.k; j += 64) {
        const u64 key = j < n ? list[j] : 0;
        a.top_ids[row * a.k + j] = j < n ? id_of(key) : -1;
        a.top_logprobs[row * a.k + j] = j < n ? (value_of(key) - st.m) - ls : -INFINITY;
    }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(256) void token_logprobs_kernel(const T* __restrict__ logits, size_t ld, int splits, int per, Answer a,
                                                             Stat* __restrict__ part_stat, u64* __restrict__ part_list) {
    constexpr int V = 16 / sizeof(T), U = 16 / V;             // elements of a vector, vectors of a thread per turn
    typedef __attribute__((ext_vector_type(V))) T Vec;
    __shared__ u64 lists[4][TOP ? LIST : 1];
    __shared__ Stat stats[4];
    __shared__ int counts[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t row = blockIdx.x / (unsigned)splits;
    const int split = (int)(blockIdx.x % (unsigned)splits);
    const T* x = logits + row * ld;
    // aligned vectors between a head and a tail of fewer than V elements each, which split 0 takes
    const int to_line = (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T);
    const int head = to_line < a.vocab ? to_line : a.vocab;
    const int vecs = (a.vocab - head) / V, tail = a.vocab - head - vecs * V;
    const Vec* xv = reinterpret_cast<const Vec*>(x + head);
    const int v0 = split * per * U * 256 < vecs ? split * per * U * 256 : vecs, v1 = v0 + per * U * 256 < vecs ? v0 + per * U * 256 : vecs;
    u64* list = lists[wave];
    int n = 0;                                                // entries of this wavefront's list
    float thr = 0.f;
    bool full = false;                                        // the list holds k entries of values >= thr, of lower ids than what comes
    float m = -INFINITY, s = 0.f, t = 0.f;

    // NE elements of every lane (valid ones only), of ids id(e) that grow from turn to turn
    auto take = [&](auto ne, const float (&e)[16], auto valid, auto id) {
        constexpr int NE = decltype(ne)::value;
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < NE; ++u) top = fmaxf(top, e[u]);                    // invalid ones are -inf
        if (__any(top > m)) {
            const float mn = fmaxf(m, top), d = m == mn ? 0.f : m - mn, f = __builtin_amdgcn_exp2f(d * LOG2E);
            t = f * fmaf(fmaxf(d, FAR), s, t);
            s *= f;
            m = mn;
        }
        const float use = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int u = 0; u < NE; ++u) {
            const float d = e[u] - use, p = __builtin_amdgcn_exp2f(d * LOG2E);
            s += p;
            t = fmaf(fmaxf(d, FAR), p, t);
        }
        if constexpr (TOP) {
            if (full && !__any(top > thr)) return;
            if (!full && n == 0) {                            // a first bound, from the lanes' maxima
                const uint32_t bound = bound_of(top, a.k);
#pragma unroll
                for (int u = 0; u < NE; ++u) {
                    const bool keep = valid(u) && ordered(e[u]) >= bound;
                    const u64 in = __ballot(keep);
                    if (keep) list[n + __popcll(in & ((1ull << lane) - 1ull))] = key_of(e[u], id(u));
                    n += __popcll(in);
                }
            } else {
#pragma unroll
                for (int u = 0; u < NE; ++u) {
                    const bool keep = valid(u) && (!full || e[u] > thr);
                    const u64 in = __ballot(keep);
                    if (keep) list[n + __popcll(in & ((1ull << lane) - 1ull))] = key_of(e[u], id(u));
                    n += __popcll(in);
                }
            }
            wave_order();
            if (n > 64 || (!full && n >= a.k)) {
                n = cut_list(list, n, a.k, lane);
                full = n == a.k && (list[n - 1] >> 32) != 0;  // (not while a NaN is among them: everything else comes before it)
                if (full) thr = value_of(list[n - 1]);
                wave_order();
            }
        }
    };
    auto take_edge = [&](int from, int count) {               // `count` single elements, by wavefront 0 of split 0
        float e[16];
        e[0] = lane < count ? to_f32<T>(x[from + lane]) : -INFINITY;
        take(Count<1>{}, e, [&](int) { return lane < count; }, [&](int) { return from + lane; });
    };
    const bool edges = split == 0 && wave == 0;
    if (edges && head > 0) take_edge(0, head);
    Vec next[U];
    auto fetch = [&](int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = base + u * 256 + (int)threadIdx.x;
            next[u] = __builtin_nontemporal_load(xv + (v < v1 ? v : v1 - 1));
        }
    };
    if (v0 < v1) fetch(v0);
    auto turn = [&](int base, auto whole) {                   // whole: every lane's vectors are in the range
        float e[16];
        auto in = [&](int u) { return decltype(whole)::value != 0 || base + u / V * 256 + (int)threadIdx.x < v1; };
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const float y = to_f32<T>(next[u / V][u % V]);
            e[u] = in(u) ? y : -INFINITY;
        }
        if (base + U * 256 < v1) fetch(base + U * 256);
        take(Count<16>{}, e, in, [&](int u) { return head + (base + u / V * 256 + (int)threadIdx.x) * V + u % V; });
    };
    int base = v0;
    for (; base + U * 256 <= v1; base += U * 256) turn(base, Count<1>{});
    if (base < v1) turn(base, Count<0>{});
    if (edges && tail > 0) take_edge(head + vecs * V, tail);

    // ---- the wavefront's, then the workgroup's: lanes and wavefronts are joined in a fixed tree
    Stat st = {m, s, t};
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const Stat other = {__shfl_xor(st.m, o, 64), __shfl_xor(st.s, o, 64), __shfl_xor(st.t, o, 64)};
        st = lane & o ? join(other, st) : join(st, other);
    }
    if constexpr (TOP) n = cut_list(list, n, a.k, lane);
    if (lane == 0) { stats[wave] = st; counts[wave] = n; }
    __syncthreads();
    if (wave != 0) return;
    st = join(join(stats[0], stats[1]), join(stats[2], stats[3]));
    if constexpr (TOP) {
        for (int w = 1; w < 4; ++w) {                         // at most 4 k <= 128 entries
            const int c = counts[w];
            if (lane < c) list[n + lane] = lists[w][lane];
            n += c;
        }
        wave_order();
        n = cut_list(list, n, a.k, lane);
    }
    if (splits == 1) {
        answer<T>(a, x, row, st, list, n, ask_given<T>(a, x, row, lane), lane);
    } else {
        const size_t at = row * splits + split;
        if (lane == 0) part_stat[at] = st;
        if (TOP && lane < a.k) part_list[at * a.k + lane] = lane < n ? list[lane] : 0;
    }
}

template <typename T>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(const T* __restrict__ logits, size_t ld, int splits, Answer a,
                                                                 const Stat* __restrict__ part_stat, const u64* __restrict__ part_list) {
    __shared__ u64 list[64 * 32];
    const int lane = threadIdx.x;
    const size_t row = blockIdx.x;
    const Given g = ask_given<T>(a, logits + row * ld, row, lane);
    Stat st = {-INFINITY, 0.f, 0.f};                          // at most 64 splits: one a lane
    if (lane < splits) st = part_stat[row * splits + lane];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const Stat other = {__shfl_xor(st.m, o, 64), __shfl_xor(st.s, o, 64), __shfl_xor(st.t, o, 64)};
        st = lane & o ? join(other, st) : join(st, other);
    }
    int n = 0;
    if (a.k > 0) {
        const int c = splits * a.k;
        for (int i0 = 0; i0 < c; i0 += 256) {
            u64 key[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) key[u] = i0 + 64 * u + lane < c ? part_list[row * c + i0 + 64 * u + lane] : 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const u64 in = __ballot(key[u] != 0);
                if (key[u] != 0) list[n + __popcll(in & ((1ull << lane) - 1ull))] = key[u];
                n += __popcll(in);
            }
        }
        wave_order();
        n = cut_list(list, n, a.k, lane);
    }
    answer<T>(a, logits + row * ld, row, st, list, n, g, lane);
}

}  // namespace

// Turns (of 4096 elements) of a workgroup, and workgroups of a row: four a CU for the whole chip, no more than 64 a row.
static void shape_of(int n_rows, int vocab, int* per, int* splits) {
    const int turns = vocab / 4096 + (vocab % 4096 != 0), wanted = n_rows < 1024 ? 1024 / n_rows : 1, most = wanted < 64 ? wanted : 64;
    *per = (turns + most - 1) / most;
    *splits = (turns + *per - 1) / *per;
}

size_t token_logprobs_ws_bytes(int n_rows, int k) {
    const size_t parts = n_rows < 16 ? 64 * (size_t)(n_rows > 0 ? n_rows : 1) : 1024;      // of any number of rows up to n_rows
    return align_up(parts * sizeof(Stat), 256) + align_up(parts * k * 8, 256);
}

void launch_token_logprobs(const void* logits, int dtype, size_t ld, int n_rows, int vocab, const int32_t* given, int n_given, int k,
                           float* logprobs, float* entropy, int32_t* top_ids, float* top_logprobs, void* ws, int32_t* status,
                           hipStream_t stream) {
    int per, splits;
    shape_of(n_rows, vocab, &per, &splits);
    const Answer a = {given, n_given, k, vocab, logprobs, entropy, top_logprobs, top_ids, status};
    Stat* ps = (Stat*)ws;
    u64* pl = (u64*)((char*)ws + align_up((size_t)n_rows * splits * sizeof(Stat), 256));
    const dim3 grid((unsigned)n_rows * (unsigned)splits);
#define RADIX_LOGPROBS(T)                                                                                                              \
    do {                                                                                                                               \
        if (k > 0) hipLaunchKernelGGL((token_logprobs_kernel<T, true>), grid, dim3(256), 0, stream, (const T*)logits, ld, splits, per, a, ps, pl); \
        else hipLaunchKernelGGL((token_logprobs_kernel<T, false>), grid, dim3(256), 0, stream, (const T*)logits, ld, splits, per, a, ps, pl);  \
        if (splits > 1)                                                                                                                \
            hipLaunchKernelGGL(token_logprobs_join_kernel<T>, dim3((unsigned)n_rows), dim3(64), 0, stream, (const T*)logits, ld, splits, a, ps, pl); \
    } while (0)
    if (dtype == RADIX_F32) RADIX_LOGPROBS(float);
    else if (dtype == RADIX_BF16) RADIX_LOGPROBS(bf16_t);
    else RADIX_LOGPROBS(f16_t);
#undef RADIX_LOGPROBS
}
