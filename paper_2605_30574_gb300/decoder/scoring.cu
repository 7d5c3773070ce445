// What a row of logits says, in one pass over it, for logits x [row][V] of
// fp32, bf16 or fp16 at a temperature T (z = x / T):
//
//   token scores   log p of a given token, the entropy of p = softmax(z), and
//                  the K largest log p with their tokens
//   distillation   the divergence of p from a teacher's K alternatives, and its
//                  gradient with respect to x
//
// A row is shared by a cluster of 1 to 16 CTAs, which trade their parts through
// distributed shared memory: no workspace, no second launch, and sums in a
// fixed order.  Both are bound by HBM: the scores read x once, the
// distillation reads it once and writes the gradient once.  512 rows of 151936
// fp32: scores with 20 alternatives 54.9 us (5.7 TB/s), divergence from 32 69 (4.5),
// with its gradient 114 (5.5).  bf16 has twice the elements to a byte, and their
// exponentials and sums come to as much: scores of 2047 rows of 100003 with 64
// alternatives 98 us (74 with none), divergence and gradient of 1999 146.
//
// Gradients are contiguous; where that leaves a row on another 16-byte alignment
// than its logits have, they go out element by element: 512 x 151936 at odd starts
// 136 us in fp32 and 89 in bf16, for 113 and 64.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../csrc/per_device.h"
#include "../csrc/tc_ptx.cuh"
#include "attention.cuh"
#include "decoder.h"

namespace cg = cooperative_groups;
namespace tc = splice::tc;

namespace {

using decoder::bulk_load;
using decoder::ex2;

constexpr int kMaxTop = 128, kMaxCluster = 16, kMaxWarps = 16;
constexpr unsigned kErrRow = 256;
constexpr float kNone = -INFINITY;
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <class T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// 16 bytes of a row.
template <class T>
struct alignas(16) Word {
    static constexpr int N = 16 / sizeof(T);
    T x[N];
};

// A row as its elements before the first 16-byte boundary, whole 16-byte words,
// and the elements behind the last.
template <class T>
struct Row {
    const T* x;
    int head, words, tail;
    __device__ Row(const T* row, int V) : x(row) {
        head = min(V, int((16u - unsigned(reinterpret_cast<uintptr_t>(row) & 15u)) % 16u / unsigned(sizeof(T))));
        words = (V - head) / Word<T>::N;
        tail = V - head - words * Word<T>::N;
    }
    __device__ const Word<T>* body() const { return reinterpret_cast<const Word<T>*>(x + head); }
    __device__ int at(int word) const { return head + word * Word<T>::N; }
};

// The largest of a warp's; NaN is passed over.
__device__ __forceinline__ float max_of_warp(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// sum e^(z - m) and sum e^(z - m) (x - m) of elements whose largest x is m, in
// fp32.  Elements of -inf weigh nothing; a NaN or +inf makes s NaN (m passes
// over NaN).  Differences x - m come before the product with 1 / T: masks of
// the type's lowest value stay finite.
struct Sums {
    float m, s, t;

    // of a warp
    __device__ __forceinline__ Sums joined(float c) const {
        Sums a = *this;
        a.shift(max_of_warp(m), c);
#pragma unroll
        for (int off = 16; off > 0; off /= 2) {
            a.s += __shfl_xor_sync(0xffffffffu, a.s, off);
            a.t += __shfl_xor_sync(0xffffffffu, a.t, off);
        }
        return a;
    }
    __device__ __forceinline__ void shift(float to, float c) {
        if (m != kNone && m != to) {                // (-inf: s is 0, or NaN)
            const float by = m - to, f = ex2(by * c);
            t = f == 0.f ? 0.f : f * fmaf(by, s, t);    // (by may be the type's lowest value)
            s *= f;
        }
        m = to;
    }
};

// A lane's sums, of the even and of the odd elements of its words.
struct LaneSums {
    float m = kNone;
    float2 s = {0.f, 0.f}, t = {0.f, 0.f};

    // `most`: the largest of the elements that follow
    __device__ __forceinline__ void rise(float most, float c) {
        if (most > m) {
            if (m != kNone) {
                const float by = m - most, f = ex2(by * c);
                t.x = f == 0.f ? 0.f : f * fmaf(by, s.x, t.x);
                t.y = f == 0.f ? 0.f : f * fmaf(by, s.y, t.y);
                s.x *= f;
                s.y *= f;
            }
            m = most;
        }
    }
    __device__ __forceinline__ float2 minus_ref() const {
        const float r = m == kNone ? 0.f : -m;
        return make_float2(r, r);
    }
    template <bool WITH_T>
    __device__ __forceinline__ void add(float2 x, float2 minus, float2 c) {
        const float2 by = __fadd2_rn(x, minus), y = __fmul2_rn(by, c), e = make_float2(ex2(y.x), ex2(y.y));
        s = __fadd2_rn(s, e);
        // (0 times -inf is not wanted)
        if constexpr (WITH_T) t = __ffma2_rn(e, make_float2(fmaxf(by.x, -3.0e38f), fmaxf(by.y, -3.0e38f)), t);
    }
    __device__ __forceinline__ Sums both() const { return Sums{m, s.x + s.y, t.x + t.y}; }
};

// (NaN is passed over; pairs of two bytes each take one instruction)
template <class T>
__device__ __forceinline__ float largest(const Word<T>& w) {
    if constexpr (sizeof(T) == 2) {
        using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
        const T2 *v = reinterpret_cast<const T2*>(&w), m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
        return to_float(__hmax(m.x, m.y));
    } else {
        return fmaxf(fmaxf(w.x[0], w.x[1]), fmaxf(w.x[2], w.x[3]));
    }
}

template <bool WITH_T, class T>
__device__ __forceinline__ void add_word(LaneSums& sums, const Word<T>& w, float2 minus, float2 c) {
#pragma unroll
    for (int e = 0; e < Word<T>::N; e += 2) sums.add<WITH_T>(make_float2(to_float(w.x[e]), to_float(w.x[e + 1])), minus, c);
}

// ---- the K largest ----
//
// An element as one key: larger values first, then lower indices (-0 as +0; no
// NaN).  0: none.
using Key = unsigned long long;
__device__ __forceinline__ Key make_key(float x, int i) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return Key(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | uint32_t(~i);
}
__device__ __forceinline__ float key_value(Key k) {
    const uint32_t b = uint32_t(k >> 32);
    return k == 0 ? kNone : __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int key_index(Key k) { return int(~uint32_t(k)); }

// The n-th largest of the lanes' values, n from 1 on.
__device__ __forceinline__ float nth_of_lanes(float x, int n, int lane) {
#pragma unroll
    for (int w = 2; w <= 32; w *= 2) {
#pragma unroll
        for (int j = w / 2; j > 0; j /= 2) {
            const bool desc = w == 32 || (lane & w) == 0, low = (lane & j) == 0;
            const float o = __shfl_xor_sync(0xffffffffu, x, j);
            x = low == desc ? fmaxf(x, o) : fminf(x, o);
        }
    }
    return __shfl_sync(0xffffffffu, x, n - 1);
}

struct ScoreParams {
    const void* x;
    long stride;
    int V, K;
    float inv_T, c;             // 1 / T; log2(e) / T
    const int64_t* tokens;      // or NULL
    float *logprobs, *entropy, *top;
    int64_t* ids;
    int buckets;                // of a thread
};

constexpr int kBuckets = 32;          // of a thread's words, by the order in which it takes them
constexpr int kCandidates = 1024;

// The ordered bits of a value above -inf, 0 for the others and NaN.
__device__ __forceinline__ uint32_t order_of(float x) { return x > kNone ? uint32_t(make_key(x, 0) >> 32) : 0u; }

// The K largest of a CTA's slice (words w0 to w1 and an edge element of the first
// threads), or all above -inf if there are fewer, as keys in any order: the K-th's
// value by four rounds of 8 bits, then the larger ones, then the first of its
// equals.  Returns how many; all threads take part.
template <class T>
__device__ __noinline__ int select(const ScoreParams& P, const Row<T>& in, int w0, int w1, int edge, float edge_x, Key* s_out, int* s_count) {
    constexpr int N = Word<T>::N;
    __shared__ int s_bins[256], s_warp[kMaxWarps + 1];
    __shared__ uint32_t s_prefix;
    __shared__ int s_left;
    const int tid = threadIdx.x, threads = int(blockDim.x), warp = tid >> 5, lane = tid & 31;
    const Word<T>* body = in.body();
    auto each = [&](auto&& f) {
        if (edge >= 0) f(edge_x, edge);
        for (int w = w0 + tid; w < w1; w += threads) {
            const Word<T> v = body[w];
#pragma unroll
            for (int e = 0; e < N; ++e) f(to_float(v.x[e]), in.at(w) + e);
        }
    };
    uint32_t prefix = 0;
    int left = P.K;             // how many are wanted of those that begin with prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += threads) s_bins[b] = 0;
        __syncthreads();
        each([&](float x, int) {
            const uint32_t o = order_of(x);
            if (o != 0 && (shift == 24 || o >> (shift + 8) == prefix)) atomicAdd(&s_bins[o >> shift & 255u], 1);
        });
        __syncthreads();
        if (tid == 0) {
            int b = 255, above = 0;
            while (b > 0 && above + s_bins[b] < left) above += s_bins[b--];
            s_prefix = prefix << 8 | uint32_t(b);
            s_left = left - above;
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
        __syncthreads();
    }
    // (prefix 0: fewer than K above -inf)
    if (tid == 0) *s_count = 0;
    __syncthreads();
    each([&](float x, int i) {
        if (order_of(x) > prefix) s_out[atomicAdd(s_count, 1)] = make_key(x, i);
    });
    __syncthreads();
    int at = *s_count;
    __syncthreads();
    if (prefix == 0) return at;
    // equals, in the order of the row: edge elements before the words, words a
    // round of the threads at a time, those behind them
    const int end = at + left;
    auto round = [&](int n, auto&& put) {        // n: this thread's
        int before = n;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += o;
        }
        if (lane == 31) s_warp[warp] = before;
        __syncthreads();
        int sum = 0, from = 0;
        for (int w = 0; w < threads / 32; ++w) {
            if (w == warp) from = sum;
            sum += s_warp[w];
        }
        put(at + from + before - n);
        at += sum;
        __syncthreads();
    };
    const bool is_edge = edge >= 0 && order_of(edge_x) == prefix;
    auto edges = [&](bool mine) {
        round(mine ? 1 : 0, [&](int p) {
            if (mine && p < end) s_out[p] = make_key(edge_x, edge);
        });
    };
    edges(is_edge && edge < in.at(w0));
    for (int base = w0; base < w1 && at < end; base += threads) {
        const int w = base + tid;
        unsigned is = 0;
        Word<T> v;
        if (w < w1) {
            v = body[w];
#pragma unroll
            for (int e = 0; e < N; ++e) is |= order_of(to_float(v.x[e])) == prefix ? 1u << e : 0u;
        }
        round(__popc(is), [&](int p) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (is >> e & 1u) {
                    if (p < end) s_out[p] = make_key(to_float(v.x[e]), in.at(w) + e);
                    ++p;
                }
        });
    }
    if (at < end) edges(is_edge && edge >= in.at(w0));
    return min(at, end);
}

// A thread takes its CTA's words in turn, four at a time: the softmax sums are
// its own, with its own running maximum.  For the K largest it keeps no more than
// the largest element of each of up to 32 buckets of its words.  Once the slice is
// through, each warp has ceil(K / warps) lanes whose largest elements are at least
// so and so large, so the least of those, over the warps, is no larger than the
// K-th of all; the few buckets that reach it are listed and read again (from L2),
// a word to a thread, and the elements that do, 1.5 K or so, are ranked by counting.
// (Each thread reading its own buckets, one after another, and a rank to a thread
// took 1.25 to 1.4 times as long in all.)  Rows with more candidates than there is
// room for (equal elements; an order that leaves a warp only small ones) take
// `select`, a radix selection by further reads.
template <class T, bool TOP>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) score_kernel(const ScoreParams P) {
    constexpr int N = Word<T>::N, U = 4;
    extern __shared__ __align__(16) float s_bucket[];       // [bucket][thread]
    __shared__ Sums s_sums[kMaxWarps], s_cta[kMaxCluster];
    __shared__ float s_known[kMaxWarps];
    __shared__ int s_count, s_listed;
    __shared__ Key s_cand[TOP ? kCandidates : 1];
    __shared__ int s_list[TOP ? kCandidates : 1];
    const int tid = threadIdx.x, threads = int(blockDim.x), warp = tid >> 5, lane = tid & 31, warps = threads >> 5;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int log2_C = __popc(C - 1);       // (C is a power of two)
    const long row = blockIdx.x >> log2_C;
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (TOP && tid == 0) s_count = s_listed = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
    const int w0 = int(long(in.words) * rank >> log2_C), w1 = int(long(in.words) * (rank + 1) >> log2_C);
    const float c = P.c;
    const float2 c2 = make_float2(c, c);
    const Word<T>* body = in.body();
    const int per_look = threads * U, looks = (w1 - w0 + per_look - 1) / per_look;
    int log2_bucket = 0;            // of the looks to a bucket
    while (looks > kBuckets << log2_bucket) ++log2_bucket;
    LaneSums sums;
    // the slice's edge elements, one to a thread: those before the row's first
    // word, those behind its last
    const int heads = rank == 0 ? in.head : 0, tails = rank == C - 1 ? in.tail : 0;
    const int edge = tid < heads ? tid : tid < heads + tails ? P.V - in.tail + tid - heads : -1;
    float edge_x = kNone;
    if (edge >= 0) {
        edge_x = to_float(in.x[edge]);
        sums.rise(edge_x, c);
        sums.add<true>(make_float2(edge_x, kNone), sums.minus_ref(), c2);
    }
    const int64_t token = rank == 0 && P.tokens ? P.tokens[row] : 0;       // (on its way until it is needed)
    float bucket = kNone;
    int in_bucket = 0;
    float* s_mine = s_bucket + tid;
    Key* s_inbox = reinterpret_cast<Key*>(s_bucket + P.buckets * threads);      // of the cluster's keys
    auto take = [&](const Word<T>(&words)[U]) {
        float most = largest(words[0]);
#pragma unroll
        for (int u = 1; u < U; ++u) most = fmaxf(most, largest(words[u]));
        sums.rise(most, c);
        const float2 minus = sums.minus_ref();
#pragma unroll
        for (int u = 0; u < U; ++u) add_word<true>(sums, words[u], minus, c2);
        if constexpr (TOP) {
            bucket = fmaxf(bucket, most);
            if (++in_bucket == 1 << log2_bucket) {
                *s_mine = bucket;
                s_mine += threads;
                bucket = kNone;
                in_bucket = 0;
            }
        }
    };
    int base = w0 + tid;
    for (; base - tid + per_look <= w1; base += per_look) {
        Word<T> words[U];
#pragma unroll
        for (int u = 0; u < U; ++u) words[u] = body[base + u * threads];
        take(words);
    }
    if (base - tid < w1) {
        Word<T> words[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int w = base + u * threads;
            if (w < w1) words[u] = body[w];
            else
#pragma unroll
                for (int e = 0; e < N; ++e) words[u].x[e] = from_float<T>(kNone);
        }
        take(words);
    }
    if (TOP && in_bucket) *s_mine = bucket;

    const float token_x = rank == 0 && warp == 0 && token >= 0 && token < P.V ? to_float(in.x[token]) : NAN;

    // lanes, warps, CTAs
    const Sums mine = sums.both().joined(c);
    if (lane == 0) s_sums[warp] = mine;
    int found = 0;              // of the CTA's largest, above -inf, in any order
    if constexpr (TOP) {
        // the warps whose every lane has elements
        const int full = min(warps, (w1 - w0) / 32), share = full > 0 ? (P.K + full - 1) / full : 33;
        if (share <= 32) {
            const float known = share == 1 ? mine.m : nth_of_lanes(sums.m, share, lane);
            if (lane == 0) s_known[warp] = known;
        }
        __syncthreads();
        float bound = -3.4028235e38f;       // (what is above -inf)
        if (share <= 32) {
            float least = s_known[0];
            for (int w = 1; w < full; ++w) least = fminf(least, s_known[w]);
            bound = fmaxf(bound, least);
        }
        unsigned reach = 0;
#pragma unroll 8
        for (int b = 0; b << log2_bucket < looks; ++b) reach |= s_bucket[b * threads + tid] >= bound ? 1u << b : 0u;
        if (reach) {
            int at = atomicAdd(&s_listed, __popc(reach));
            for (; reach && at < kCandidates; reach &= reach - 1) s_list[at++] = ((__ffs(reach) - 1) << log2_bucket) * per_look + tid;
        }
        if (edge_x >= bound) {
            const int at = atomicAdd(&s_count, 1);
            if (at < kCandidates) s_cand[at] = make_key(edge_x, edge);
        }
        __syncthreads();
        // (more listed: there are more candidates than that, too)
        const int listed = s_listed, log2_span = log2_bucket + 2, all = listed <= kCandidates ? listed << log2_span : 0;
        static_assert(U == 4);
        for (int base = tid; base < all; base += U * threads) {
            Word<T> words[U];
            int w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = base + u * threads;
                w[u] = i < all ? w0 + s_list[i >> log2_span] + (i & ((1 << log2_span) - 1)) * threads : w1;
                if (w[u] < w1) words[u] = body[w[u]];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (w[u] >= w1 || !(largest(words[u]) >= bound)) continue;
                unsigned is = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) is |= to_float(words[u].x[e]) >= bound ? 1u << e : 0u;
                int at = atomicAdd(&s_count, __popc(is));
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (is >> e & 1u && at < kCandidates) s_cand[at] = make_key(to_float(words[u].x[e]), in.at(w[u]) + e);
                    at += is >> e & 1u;
                }
            }
        }
        __syncthreads();
        found = listed <= kCandidates ? s_count : kCandidates + 1;
        if (found > kCandidates) found = select<T>(P, in, w0, w1, edge, edge_x, s_cand, &s_count);
    } else {
        __syncthreads();
    }
    // The candidates' ranks by counting: four to as many lanes as there are, up to
    // eight, as reading the others is what it costs.  (A bitonic sort takes longer.)
    auto ranked = [&](auto&& put) {
        constexpr int B = 4;
        const int groups = (found + B - 1) / B;
        int log2 = 0;
        while (log2 < 3 && groups << (log2 + 1) <= threads) ++log2;
        for (int base = 0; base < groups << log2; base += threads) {
            const int g = (base + tid) >> log2, part = tid & ((1 << log2) - 1);
            Key k[B];
            int r[B] = {};
#pragma unroll
            for (int i = 0; i < B; ++i) k[i] = g * B + i < found ? s_cand[g * B + i] : 0;
#pragma unroll 4
            for (int j = part; j < found; j += 1 << log2) {
                const Key o = s_cand[j];
#pragma unroll
                for (int i = 0; i < B; ++i) r[i] += o > k[i];
            }
            // (two counts to a number)
            int two[B / 2];
#pragma unroll
            for (int i = 0; i < B / 2; ++i) two[i] = r[2 * i] | r[2 * i + 1] << 16;
            for (int off = 1 << log2 >> 1; off > 0; off /= 2)
#pragma unroll
                for (int i = 0; i < B / 2; ++i) two[i] += __shfl_xor_sync(0xffffffffu, two[i], off);
            if (part == 0)
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    const int at = i & 1 ? two[i / 2] >> 16 : two[i / 2] & 0xffff;
                    if (k[i] != 0 && at < P.K) put(at, k[i]);
                }
        }
    };
    if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (every CTA has begun)
        if (warp == 0) {
            const Sums all = (lane < warps ? s_sums[lane] : Sums{kNone, 0.f, 0.f}).joined(c);
            if (lane == 0) *cluster.map_shared_rank(&s_cta[rank], 0) = all;
        }
        if constexpr (TOP) {
            Key* to = cluster.map_shared_rank(s_inbox + rank * P.K, 0);
            ranked([&](int r, Key k) { to[r] = k; });
            for (int k = found + tid; k < P.K; k += threads) to[k] = 0;
        }
        cluster.sync();
        if (rank != 0) return;
    }
    const int parts = C > 1 ? C : warps;
    const Sums all = (lane < parts ? (C > 1 ? s_cta[lane] : s_sums[lane]) : Sums{kNone, 0.f, 0.f}).joined(c);
    const bool empty = all.m == kNone && !(all.s != all.s);
    const float log_s = logf(all.s);
    auto logprob = [&](float x) { return empty ? kNone : (x - all.m) * P.inv_T - log_s; };
    if (tid == 0) {
        if (P.tokens) P.logprobs[row] = token < 0 ? 0.f : token >= P.V ? NAN : logprob(token_x);
        P.entropy[row] = empty ? 0.f : log_s - all.t / all.s * P.inv_T;
    }
    if constexpr (TOP) {
        auto put = [&](int r, Key k) {
            P.top[row * P.K + r] = logprob(key_value(k));
            P.ids[row * P.K + r] = key_index(k);
        };
        if (C == 1) {
            ranked(put);
        } else {
            // each CTA's are in order: those of the others before a key by bisection
            for (int i = tid; i < C * P.K; i += threads) {
                const Key k = s_inbox[i];
                const int own = i / P.K;
                int r = i - own * P.K;
                if (k == 0) continue;
                for (int o = 0; o < C && r < P.K; ++o) {
                    if (o == own) continue;
                    int lo = 0, hi = P.K;
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (s_inbox[o * P.K + mid] > k) lo = mid + 1;
                        else hi = mid;
                    }
                    r += lo;
                }
                if (r < P.K) put(r, k);
            }
        }
        if (warp != 0) return;
        // fewer than K above -inf: the first of the others
        if (C > 1) {
            found = 0;
            for (int i = lane; i < C * P.K; i += 32) found += s_inbox[i] != 0;
            found = int(__reduce_add_sync(0xffffffffu, unsigned(found)));
        }
        for (int base = 0; found < P.K && base < P.V; base += 32) {
            const bool is = base + lane < P.V && !(to_float(in.x[min(base + lane, P.V - 1)]) > kNone);
            const unsigned who = __ballot_sync(0xffffffffu, is);
            const int p = found + __popc(who & ((1u << lane) - 1u));
            if (is && p < P.K) {
                P.top[row * P.K + p] = logprob(kNone);
                P.ids[row * P.K + p] = base + lane;
            }
            found += __popc(who);
        }
    }
}

// ---- distillation ----

constexpr int kWorkers = 256, kDistillThreads = kWorkers + 32;

struct DistillParams {
    const void* x;
    long stride;
    long rows;
    int V, K, rest;
    float inv_T, inv_T_low;     // 1 / T, and what its rounding left
    float c, c_low;             // log2(e) / T, the same
    float least;                // -160 / c
    const int64_t* ids;
    const float* teacher;
    const float* weight;        // or NULL
    float* loss;
    void* grad;                 // or NULL
    unsigned* err;
};

// k e^((x - ref) / T) of two logits, for a gradient of type T.  In fp32 with the
// exponent's rounding made good, which 30 below the maximum costs 1e-6 of the
// value.
template <class T>
__device__ __forceinline__ float2 weights_of(float2 x, float ref, float k, const DistillParams& P) {
    float2 by = __fadd2_rn(x, make_float2(-ref, -ref));
    if constexpr (sizeof(T) < 4) {
        const float2 y = __fmul2_rn(by, make_float2(P.c, P.c));
        return __fmul2_rn(make_float2(ex2(y.x), ex2(y.y)), make_float2(k, k));
    } else {
        // (as good as none from 2^-160 on; a NaN's row has a k of NaN)
        by = make_float2(fmaxf(by.x, P.least), fmaxf(by.y, P.least));
        const float2 y = __fmul2_rn(by, make_float2(P.c, P.c)), minus_y = make_float2(-y.x, -y.y);
        const float2 e = __fmul2_rn(make_float2(ex2(y.x), ex2(y.y)), make_float2(k, k));
        const float2 low = __ffma2_rn(by, make_float2(P.c_low, P.c_low), __ffma2_rn(by, make_float2(P.c, P.c), minus_y));
        return __ffma2_rn(e, __fmul2_rn(low, make_float2(0.69314718f, 0.69314718f)), e);
    }
}

// 8 bytes to another CTA of the cluster, which count on its barrier.  (A store and
// an arrival that releases it wait for all that the thread has written before, its
// gradients among it: 2 us.)
__device__ __forceinline__ void store_async(uint32_t to, float2 v, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to), "f"(v.x), "f"(v.y),
                 "r"(bar)
                 : "memory");
}

// A wait for what other CTAs of the cluster send.
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort, unsigned* err, unsigned code) {
    const uint64_t t0 = tc::globaltimer_ns();
    for (uint32_t i = 1;; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((i & 63u) == 0) {
            if (*abort) return false;
            if (tc::globaltimer_ns() - t0 > 1000000000ull) {
                *abort = 1;
                atomicOr(err, code);
                return false;
            }
        }
    }
}

// Sums of two floats each: a pair's value is x + y, y the smaller.  (fp64, on this
// part, takes 50 clocks an operation.)
__device__ __forceinline__ float2 exact_sum(float a, float b) {            // Knuth's
    const float s = __fadd_rn(a, b), t = __fadd_rn(s, -a);
    return make_float2(s, __fadd_rn(__fadd_rn(a, -__fadd_rn(s, -t)), __fadd_rn(b, -t)));
}
__device__ __forceinline__ float2 pair_sum(float2 a, float2 b) {
    const float2 s = exact_sum(a.x, b.x);
    return exact_sum(s.x, __fadd_rn(s.y, __fadd_rn(a.y, b.y)));
}

// log x as a pair, to 1e-9: 2 atanh(u) of u = (m - 1) / (m + 1), m the mantissa
// between sqrt(1/2) and sqrt(2), by its series; u's first term and quotient's rest
// exactly, the terms from u^3 on in fp32.
__device__ __forceinline__ float2 log_pair(float x) {
    if (!(x > 0.f)) return make_float2(x == 0.f ? -INFINITY : NAN, 0.f);
    if (x > 3.4e38f) return make_float2(INFINITY, 0.f);
    const bool small = x < 1.2e-38f;
    if (small) x *= 18446744073709551616.f;         // 2^64
    const int b = __float_as_int(x);
    int e = (b >> 23) - 127 - (small ? 64 : 0);
    float m = __int_as_float((b & 0x7fffff) | 0x3f800000);
    if (m > 1.41421356f) {
        m *= 0.5f;
        ++e;
    }
    const float num = m - 1.f;                      // (exact)
    const float2 den = exact_sum(m, 1.f);
    const float u = num / den.x, rest = __fadd_rn(fmaf(-u, den.x, num), -u * den.y) / den.x, v = u * u;
    float p = 1.f / 13.f;
    p = fmaf(p, v, 1.f / 11.f);
    p = fmaf(p, v, 1.f / 9.f);
    p = fmaf(p, v, 1.f / 7.f);
    p = fmaf(p, v, 1.f / 5.f);
    p = fmaf(p, v, 1.f / 3.f);
    // (ln 2 in two: e times the first is exact)
    const float2 whole = exact_sum(float(e) * 0.693145752f, 2.f * u);
    return exact_sum(whole.x, __fadd_rn(whole.y, fmaf(float(e), 1.42860677e-6f, fmaf(2.f * u * v, p, 2.f * rest))));
}

// What warp kWorkers / 32 makes of a row's teacher before the row is taken.
struct Teacher {
    alignas(16) int id[kMaxTop];        // -1: none
    float q[kMaxTop], z[kMaxTop];       // probabilities; logits, before the temperature
    float log_q[kMaxTop];               // and log q, less `shift`
    float sum[kMaxTop];                 // of all mentions of the token, at its first; -1: not the first
    float most, e;                      // the tokens' largest logit, and sum of e^(z - most)
    float all, rest;                    // the teacher's sum, and what is left of 1
    bool none;                          // whether it says nothing of the row
    float norm;                         // shift is log(norm)
    unsigned edges;                     // which of the first 8 elements, and of the 8 before the last word's end, are the teacher's
};

__device__ __forceinline__ void workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkers) : "memory"); }

// Clusters stay and take row after row.  A CTA's slice of a row comes into shared
// memory by one bulk copy: the sums are taken from it, and once the cluster has the
// row's, the gradient is made from the same copy and the next row's slice asked for
// in its place; the warp behind the workers' reads the next row's teacher.  The
// other CTAs of an SM work under a CTA's copy and exchange.  (A cluster for each
// row, gone when it was done: 1.7 times as long.  A slice in eight pieces, each
// replaced by the next row's as soon as it is used: 1.15 times, as the
// instructions of eight loops cost more than the copies' earlier start gives.)
//
// The teacher's tokens are taken out of the slice (-inf) before it is summed up
// and put in their own way, so the sum of all others is a sum and not a
// difference.
template <class T, bool GRAD, int J>
__global__ void __launch_bounds__(kDistillThreads, 4) distill_kernel(const DistillParams P) {
    constexpr int N = Word<T>::N;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[3];
    __shared__ Teacher s_teacher[2];
    __shared__ float2 s_warps[kWorkers / 32], s_cta[2][kMaxCluster];       // largest x, sum of the others' e^
    __shared__ volatile int s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int log2_C = __popc(C - 1);       // (C is a power of two)
    const long row0 = blockIdx.x >> log2_C, step = gridDim.x >> log2_C;
    const uint32_t bar0 = tc::smem_u32(bars);
    const Word<T>* slice = reinterpret_cast<const Word<T>*>(smem);
    T* flat = reinterpret_cast<T*>(smem);
    const float c = P.c;
    const float2 c2 = make_float2(c, c);
    if (tid == 0) {
        for (int i = 0; i < 3; ++i) tc::mbar_init(bar0 + 8u * i, 1);
        s_abort = 0;
        tc::fence_mbar_init();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // this CTA's part of a row: words, from w0 on
    struct Part {
        Row<T> in;
        int w0, nw;
    };
    auto part_of = [&](long row) {
        const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
        const int w0 = int(long(in.words) * rank >> log2_C);
        return Part{in, w0, int(long(in.words) * (rank + 1) >> log2_C) - w0};
    };
    // a slice, by one thread (an empty one just arrives)
    auto ask = [&](const Part& p) {
        tc::mbar_arrive_expect_tx(bar0, uint32_t(p.nw) * 16u);
        if (p.nw > 0) bulk_load(tc::smem_u32(slice), p.in.body() + p.w0, uint32_t(p.nw) * 16u, bar0);
    };
    // The teacher of a row, J alternatives to a lane, in three steps, each
    // a row ahead of the next so that none waits for memory: what is given for it,
    // its tokens' logits, and what it comes to.
    int64_t asked[J];
    float given[J], q[J], z[J];
    int id[J];
    bool poison = false;
    auto ask_teacher = [&](long row) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = j * 32 + lane;
            asked[j] = -1;
            given[j] = kNone;
            if (k < P.K && row < P.rows) {
                asked[j] = P.ids[row * P.K + k];
                given[j] = P.teacher[row * P.K + k];
            }
        }
    };
    auto look_up = [&](long row) {
        const T* x = static_cast<const T*>(P.x) + row * P.stride;
        poison = false;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            poison |= asked[j] >= P.V;
            id[j] = asked[j] >= 0 && asked[j] < P.V ? int(asked[j]) : -1;
            z[j] = id[j] >= 0 ? to_float(x[id[j]]) : kNone;
            q[j] = id[j] >= 0 ? given[j] : kNone;
        }
    };
    auto teach = [&](long row, Teacher& t) {
        const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
        unsigned edges = 0;
        bool first[J];
        float top = kNone, most = kNone;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (id[j] >= 0 && id[j] < in.head) edges |= 1u << id[j];
            if (id[j] >= P.V - in.tail) edges |= 256u << (id[j] - (P.V - in.tail));
            t.id[j * 32 + lane] = id[j];
            top = fmaxf(top, q[j]);
            // first of its 32, and not among those before
            first[j] = false;
            {
                const unsigned same = __match_any_sync(0xffffffffu, id[j]);
                first[j] = id[j] >= 0 && (same & ((1u << lane) - 1u)) == 0;
            }
        }
        __syncwarp();
#pragma unroll
        for (int j = 1; j < J; ++j) {
            for (int k = 0; k < j * 32; k += 4) {
                const int4 four = *reinterpret_cast<const int4*>(t.id + k);
                first[j] = first[j] && four.x != id[j] && four.y != id[j] && four.z != id[j] && four.w != id[j];
            }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            t.z[j * 32 + lane] = z[j];
            most = fmaxf(most, z[j]);
        }
        const bool outside = __any_sync(0xffffffffu, poison);
        edges = __reduce_or_sync(0xffffffffu, edges);
#pragma unroll
        for (int off = 16; off > 0; off /= 2) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
        }
        if (P.rest || top == kNone) top = 0.f;
        float sum = 0.f, e = 0.f, sizes = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const float log_q = t.log_q[j * 32 + lane] = q[j] - top;
            q[j] = expf(log_q);
            sum += q[j];
            if (q[j] > 0.f) sizes = fmaf(q[j], 1.f + fabsf(log_q), sizes);
            if (first[j]) e += ex2((z[j] - (most == kNone ? 0.f : most)) * c);
        }
#pragma unroll
        for (int off = 16; off > 0; off /= 2) {
            sum += __shfl_xor_sync(0xffffffffu, sum, off);
            e += __shfl_xor_sync(0xffffffffu, e, off);
            sizes += __shfl_xor_sync(0xffffffffu, sizes, off);
        }
        // (NaN for a row with a token outside the vocabulary)
        float2 all = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (!P.rest && sum != 0.f) q[j] /= sum;
            if (outside) q[j] = NAN;
            all = pair_sum(all, make_float2(q[j], 0.f));
            t.q[j * 32 + lane] = q[j];
        }
#pragma unroll
        for (int off = 16; off > 0; off /= 2)
            all = pair_sum(all, make_float2(__shfl_xor_sync(0xffffffffu, all.x, off), __shfl_xor_sync(0xffffffffu, all.y, off)));
        // What is left of 1 is no weight up to what rounding makes of K log
        // probabilities whose sum is 1: each is off by some 2^-24 of itself and of
        // the row's log sum, its exponential by 2^-23.  (Whole distributions of 2 to
        // 128 tokens: left at up to 2.9 x 2^-23 sum q (1 + |log q|), in fp32.)
        const float left = pair_sum(make_float2(1.f, 0.f), make_float2(-all.x, -all.y)).x, least = 0x1p-21f * sizes;
        __syncwarp();
        bool again = false, any = outside;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            again |= id[j] >= 0 && !first[j];
            any |= P.rest ? id[j] >= 0 : q[j] != 0.f;
        }
        again = __any_sync(0xffffffffu, again);
        any = __any_sync(0xffffffffu, any);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float own = q[j];
            for (int k = j * 32 + lane + 1; again && k < P.K; ++k)
                if (t.id[k] == id[j]) own += t.q[k];
            t.sum[j * 32 + lane] = first[j] ? own : -1.f;
        }
        if (lane == 0) {
            t.most = most;
            t.e = e;
            t.edges = edges;
            t.norm = P.rest || sum == 0.f ? 1.f : sum;
            t.all = all.x;
            t.rest = P.rest && any && (left > least || left != left) ? left : 0.f;
            t.none = !any;
        }
    };
    // of sums with their largest x, over a warp (-inf: a sum of 0, or NaN)
    auto together = [&](float2 v) {
        float m = v.x;
#pragma unroll
        for (int off = 16; off > 0; off /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
        if (v.x != kNone && v.x != m) v.y *= ex2((v.x - m) * c);
#pragma unroll
        for (int off = 16; off > 0; off /= 2) v.y += __shfl_xor_sync(0xffffffffu, v.y, off);
        return make_float2(m, v.y);
    };

    if (tid == 0 && row0 < P.rows) ask(part_of(row0));         // (it has made the barriers itself)
    if (warp == kWorkers / 32 && row0 < P.rows) {
        ask_teacher(row0);
        look_up(row0);
        ask_teacher(row0 + step);
        teach(row0, s_teacher[0]);
        look_up(row0 + step);
        ask_teacher(row0 + 2 * step);
    }
    if (C > 1) cluster.sync();                // every CTA has begun
    else __syncthreads();

    // What a row's gradient goes by: p_j = e^((x_j - ref) / T) / s; the gradient of
    // a token that is not the teacher's is out e^((x_j - out_ref) / T), of one that
    // is (all p_j - q_j); all times scale.  Where the others lie far below ref they
    // go by their own largest logit: what the rest gives them is q_rest times their
    // shares of it, and does not vanish where p_rest does.  Else p_rest is taken from
    // the same sum as s: an error in it then counts p_rest - q_rest times in the loss.
    struct Stats {
        float2 others;              // an x, and the others' sum of e^ from there
        float ref, s, inv_s, all, out_ref, out, scale;
    };
    __shared__ Stats s_stats;
    uint32_t turn = 0, round = 0;        // row by row, and every other
    // (once every CTA's sums are here)
    auto stats_of = [&](const Teacher& t, float weight) {
        const float2 others = together(lane < C ? s_cta[turn][lane] : make_float2(kNone, 0.f));
        const float m = fmaxf(others.x, t.most);
        Stats a;
        a.ref = m == kNone ? 0.f : m;
        // (-inf: a sum of 0, or NaN)
        const float2 f = weights_of<float>(make_float2(others.x, t.most), a.ref, 1.f, P);
        const bool far = f.x < 0x1p-24f;
        a.others = far ? others : make_float2(a.ref, others.y * f.x);
        a.s = others.y * f.x + t.e * f.y;
        a.inv_s = a.s == 0.f ? 0.f : 1.f / a.s;
        a.all = P.rest ? 1.f : t.all;
        a.out_ref = a.ref;
        a.out = a.all * a.inv_s;
        if (t.rest != 0.f && others.y > 0.f) {      // (of 0: nothing to share it)
            if (far) a.out_ref = others.x;
            a.out = (far ? f.x * a.inv_s : a.inv_s) - t.rest / a.others.y;
        }
        if (t.rest != t.rest) a.out = t.rest;
        a.scale = t.none ? 0.f : weight * P.inv_T;
        return a;
    };
    auto exchanged = [&]() { return wait_cluster(bar0 + 8u * (1 + turn), round, &s_abort, P.err, kErrRow); };

    if (warp < kWorkers / 32) {
        for (long row = row0; row < P.rows; row += step) {
            const Part p = part_of(row), next = part_of(min(row + step, P.rows - 1));
            const bool more = row + step < P.rows;
            const Teacher& t = s_teacher[turn];
            const float weight = P.weight ? P.weight[row] : 1.f;
            const int first_word = p.in.at(p.w0);
            // the slice's edge elements, one to a thread: those before the row's
            // first word, those behind its last
            const int heads = rank == 0 ? p.in.head : 0, tails = rank == C - 1 ? p.in.tail : 0;
            const int edge = tid < heads ? tid : tid < heads + tails ? P.V - p.in.tail + tid - heads : -1;
            // the teacher's tokens out
            float edge_x = kNone;
            if (edge >= 0 && !(t.edges >> (tid < heads ? edge : 8 + tid - heads) & 1u)) edge_x = to_float(p.in.x[edge]);
            if (tc::mbar_wait(bar0, turn, &s_abort, P.err, kErrRow) && tid < P.K) {
                const int at = t.id[tid] - first_word;
                if (t.id[tid] >= 0 && at >= 0 && at < p.nw * N) flat[at] = from_float<T>(kNone);
            }
            workers_sync();
            // the sum of all others
            LaneSums sums;
            if (edge >= 0) {
                sums.rise(edge_x, c);
                sums.add<false>(make_float2(edge_x, kNone), sums.minus_ref(), c2);
            }
            for (int w = tid; w < p.nw; w += 2 * kWorkers) {
                const Word<T> a = slice[w], b = slice[min(w + kWorkers, p.nw - 1)];
                const bool two = w + kWorkers < p.nw;
                sums.rise(two ? fmaxf(largest(a), largest(b)) : largest(a), c);
                const float2 minus = sums.minus_ref();
                add_word<false>(sums, a, minus, c2);
                if (two) add_word<false>(sums, b, minus, c2);
            }
            if constexpr (!GRAD) {
                tc::fence_proxy_async_smem();
                workers_sync();
                if (tid == 0 && more) ask(next);
            }
            const float2 mine = together(make_float2(sums.m, sums.s.x + sums.s.y));
            if (lane == 0) s_warps[warp] = mine;
            workers_sync();
            // to every CTA of the cluster
            if (warp == 0) {
                const float2 part = together(lane < kWorkers / 32 ? s_warps[lane] : make_float2(kNone, 0.f));
                const uint32_t to = tc::smem_u32(&s_cta[turn][rank]), bar = bar0 + 8u * (1 + turn);
                if (lane == 0) tc::mbar_arrive_expect_tx(bar, uint32_t(C) * 8u);
                if (lane < C) store_async(tc::map_cta(to, uint32_t(lane)), part, tc::map_cta(bar, uint32_t(lane)));
            }
            if constexpr (GRAD) {
                // (by one warp: the others would take the issue slots of CTAs that work)
                if (warp == 0) {
                    exchanged();
                    const Stats a = stats_of(t, weight);
                    if (lane == 0) s_stats = a;
                }
                workers_sync();
                const Stats a = s_stats;
                T* out = static_cast<T*>(P.grad) + row * P.V;
                const bool words_out = (reinterpret_cast<uintptr_t>(out + p.in.head) & 15u) == 0;
                const float k = a.out * a.scale;
                if (a.scale == 0.f) {        // a row that is left out
                    if (words_out) {
                        for (int w = tid; w < p.nw; w += kWorkers) reinterpret_cast<uint4*>(out + first_word)[w] = make_uint4(0, 0, 0, 0);
                    } else {
                        for (int w = tid; w < p.nw * N; w += kWorkers) out[first_word + w] = from_float<T>(0.f);
                    }
                } else if (words_out) {
#pragma unroll 4
                    for (int w = tid; w < p.nw; w += kWorkers) {
                        const Word<T> v = slice[w];
                        Word<T> g;
#pragma unroll
                        for (int e = 0; e < N; e += 2) {
                            const float2 two = weights_of<T>(make_float2(to_float(v.x[e]), to_float(v.x[e + 1])), a.out_ref, k, P);
                            g.x[e] = from_float<T>(two.x);
                            g.x[e + 1] = from_float<T>(two.y);
                        }
                        reinterpret_cast<Word<T>*>(out + first_word)[w] = g;
                    }
                } else {
                    for (int w = tid; w < p.nw * N; w += kWorkers)
                        out[first_word + w] = from_float<T>(weights_of<T>(make_float2(to_float(flat[w]), 0.f), a.out_ref, k, P).x);
                }
                tc::fence_proxy_async_smem();
                workers_sync();
                if (tid == 0 && more) ask(next);
                if (edge >= 0) out[edge] = from_float<T>(a.scale == 0.f ? 0.f : weights_of<T>(make_float2(edge_x, 0.f), a.out_ref, k, P).x);
            }
            if (__syncthreads_or(s_abort)) {         // (a wait ran out; the copy on its way lands first)
                volatile int no_abort = 0;
                if (tid == 0 && more) tc::mbar_wait(bar0, turn ^ 1u, &no_abort, P.err, kErrRow);
                break;
            }
            round ^= turn;
            turn ^= 1u;
        }
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        // (no CTA leaves while another may send it something)
        if (C > 1) cluster.sync();
        return;
    }

    // The teacher's warp, a row behind and a row ahead: the gradients of the last
    // row's tokens, which the workers have written as any others', are put right;
    // the next row's teacher; this one's loss.
    Stats last{};
    auto put_right = [&](long row, const Teacher& t) {
        if (!GRAD || last.scale == 0.f) return;
        const Part p = part_of(row);
        const int first_word = p.in.at(p.w0);
        T* out = static_cast<T*>(P.grad) + row * P.V;
        for (int k = lane; k < P.K; k += 32) {
            const int i = t.id[k];
            const bool here = (i >= first_word && i < first_word + p.nw * N) || (rank == 0 && i < p.in.head) ||
                              (rank == C - 1 && i >= P.V - p.in.tail);
            const float sum = t.sum[k];
            if (i >= 0 && here && sum != -1.f)
                out[i] = from_float<T>(fmaf(last.scale * last.all, weights_of<T>(make_float2(t.z[k], 0.f), last.ref, last.inv_s, P).x,
                                            -last.scale * sum));
        }
    };
    for (long row = row0; row < P.rows; row += step) {
        const Teacher& t = s_teacher[turn];
        const float weight = P.weight ? P.weight[row] : 1.f;
        if (row > row0) put_right(row - step, s_teacher[turn ^ 1u]);
        __syncwarp();
        if (row + step < P.rows) {
            teach(row + step, s_teacher[turn ^ 1u]);
            look_up(row + 2 * step);
            ask_teacher(row + 3 * step);
        }
        exchanged();
        const Stats a = last = stats_of(t, weight);
        if (rank == 0) {
            // in pairs, as the terms are small differences of log probabilities; the
            // four logarithms by a lane each
            const float2 mine = log_pair(lane == 0 ? a.s : lane == 1 ? a.others.y : lane == 2 ? t.rest : t.norm);
            auto of = [&](int from) {
                return make_float2(__shfl_sync(0xffffffffu, mine.x, from), __shfl_sync(0xffffffffu, mine.y, from));
            };
            auto minus = [](float2 a) { return make_float2(-a.x, -a.y); };
            const float2 log_s = of(0), log_others = of(1), log_rest = of(2), log_norm = of(3);
            // (an infinity's rest would be NaN)
            auto plus = [](float2 a, float2 b) {
                const float2 x = pair_sum(a, b);
                return fabsf(x.x) < INFINITY ? x : make_float2(a.x + b.x, 0.f);
            };
            float2 total = make_float2(0.f, 0.f);
            const float no_number = a.s - a.s;      // NaN in a row with NaN or +inf, else 0
            // q (log q - log p) of log p = (x - ref) / T + log_w - log s; p is 0 where
            // x is -inf or no token has any
            auto add = [&](float q, float2 log_q, float x, float2 log_w, bool none) {
                const float2 by = exact_sum(x, -a.ref);
                const float z = by.x * P.inv_T, v = q * P.inv_T;
                float2 y;
                if (none) {
                    y = make_float2(q * INFINITY + no_number, 0.f);
                } else if (!(fabsf(z) < INFINITY)) {
                    // (a mask of the type's lowest value: past fp32, its product with q perhaps not)
                    y = make_float2((fabsf(by.x) < INFINITY ? -v * by.x : v * a.ref - v * x) + no_number, 0.f);
                } else {
                    const float2 log_p = pair_sum(pair_sum(make_float2(z, fmaf(by.x, P.inv_T, -z) + fmaf(by.y, P.inv_T, by.x * P.inv_T_low)), log_w), minus(log_s));
                    const float2 d = pair_sum(log_q, minus(log_p));
                    y = make_float2(q * d.x, fmaf(q, d.x, -(q * d.x)) + q * d.y);
                }
                total = plus(total, y);
            };
            for (int k = lane; k < P.K; k += 32)
                if (t.q[k] != 0.f)
                    add(t.q[k], pair_sum(make_float2(t.log_q[k], 0.f), minus(log_norm)), t.z[k], make_float2(0.f, 0.f), a.s == 0.f || t.z[k] == kNone);
            if (lane == 0 && t.rest > 0.f) add(t.rest, log_rest, a.others.x, log_others, a.others.y == 0.f);
#pragma unroll
            for (int off = 16; off > 0; off /= 2)
                total = plus(total, make_float2(__shfl_xor_sync(0xffffffffu, total.x, off), __shfl_xor_sync(0xffffffffu, total.y, off)));
            if (lane == 0) P.loss[row] = weight == 0.f ? 0.f : (total.x + total.y) * weight;
        }
        if (__syncthreads_or(s_abort)) break;
        round ^= turn;
        turn ^= 1u;
        if (row + step >= P.rows) put_right(row, s_teacher[turn ^ 1u]);
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (C > 1) cluster.sync();
}

template <class Kernel, class Params>
int launch(Kernel kernel, long ctas, int threads, size_t smem, int cluster, const Params& P, cudaStream_t st, bool early = true) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return int(cudaLaunchKernelEx(&cfg, kernel, P));
}

// Clusters of more than 8 CTAs have to be allowed, and dynamic shared memory of
// more than 48 KB.
template <class Kernel>
cudaError_t allow(splice::PerDevice<bool>& kept, Kernel kernel, size_t smem) {
    bool set = false;
    return kept.get(&set, [&](int, bool* done) {
        *done = true;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        return e;
    });
}

// CTAs that share a row: as many as leave one to an SM, of 16384 elements at least
// and with 256 alternatives in all at most, which one of them merges.  (151936 fp32,
// 20 alternatives: 20 rows in twos, fours and eights 11.3, 9.4 and 9.8 us; 80 rows
// alone, in twos and fours 13.5, 13.9 and 16; 512 rows 54, 62 and 72; one row with
// 128 in twos and eights 11.7 and 22.9.)
int score_cluster(long rows, long V, int K) {
    int C = 1;
    while (C < kMaxCluster && rows * 2 * C <= 152 && V >= 32768L * C && 2 * C * K <= 256) C *= 2;
    return C;
}

// Warps of a CTA: 16 where it has an SM to itself and enough to read, or half of
// one and much, else 8.  (Slices of 76, 100, 152, 200 KB with an SM each, 8 and 16
// warps: 8.8 and 9.6 us, 9.7 and 10.1, 9.9 and 9.4, 11.7 and 10.8; 200 rows of 200
// and 608 KB: 14.9 and 17.2, 35.4 and 27.4; 512 rows of 608 KB: 54 and 60.)
int score_warps(long ctas, long slice_bytes) {
    return ctas <= 152 && slice_bytes >= 112 * 1024 || ctas <= 304 && slice_bytes >= 400 * 1024 ? 16 : 8;
}

template <class T, bool TOP>
int scores(ScoreParams P, long rows, cudaStream_t st) {
    static splice::PerDevice<bool> kept;
    const cudaError_t e = allow(kept, score_kernel<T, TOP>, kBuckets * kMaxWarps * 32 * 4 + kMaxCluster * kMaxTop * sizeof(Key));
    if (e != cudaSuccess) return int(e);
    const int C = score_cluster(rows, P.V, P.K), warps = score_warps(rows * C, P.V * long(sizeof(T)) / C);
    P.buckets = int(std::min(P.V / (Word<T>::N * 4L * 32 * warps * C) + 1, long(kBuckets)));
    const size_t smem = TOP ? size_t(P.buckets) * warps * 32 * 4 + (C > 1 ? size_t(C) * P.K * sizeof(Key) : 0) : 0;
    return launch(score_kernel<T, TOP>, rows * C, 32 * warps, smem, C, P, st);
}

template <class T>
int scores(const ScoreParams& P, long rows, cudaStream_t st) {
    return P.K ? scores<T, true>(P, rows, st) : scores<T, false>(P, rows, st);
}

// Bytes of a CTA's slice with four, two and one CTA to an SM.
constexpr int kClasses = 3;
constexpr size_t kSlices[kClasses] = {49 * 1024, 104 * 1024, 216 * 1024}, kSliceMax = kSlices[kClasses - 1];

size_t slice_bytes(long V, size_t size, int C) { return (size_t(V) * size / 16 / C + 1) * 16; }

int distill_cluster(long rows, long V, size_t size) {
    int C = 1;
    while (C < kMaxCluster && slice_bytes(V, size, C) > kSlices[0]) C *= 2;
    while (C < kMaxCluster && rows * C < 304 && V >= 8192L * C) C *= 2;
    return C;
}

// Clusters of 1, 2, 4, 8 and 16 CTAs that are resident together.
struct Clusters {
    int n[5][kClasses];
};

template <class T, bool GRAD, int J>
int distill(DistillParams P, cudaStream_t st) {
    static splice::PerDevice<Clusters> kept;
    Clusters clusters;
    const cudaError_t e = kept.get(&clusters, [](int, Clusters* r) {
        auto kernel = distill_kernel<T, GRAD, J>;
        cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSliceMax));
        if (err == cudaSuccess) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        for (int i = 0; i < 5 * kClasses && err == cudaSuccess; ++i) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(1u << (i / kClasses));
            cfg.blockDim = dim3(kDistillThreads);
            cfg.dynamicSmemBytes = kSlices[i % kClasses];
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 1u << (i / kClasses);
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            err = cudaOccupancyMaxActiveClusters(&r->n[i / kClasses][i % kClasses], kernel, &cfg);
        }
        return err;
    });
    if (e != cudaSuccess) return int(e);
    const int C = distill_cluster(P.rows, P.V, sizeof(T));
    const size_t bytes = slice_bytes(P.V, sizeof(T), C);
    if (bytes > kSliceMax) return int(cudaErrorInvalidValue);
    int log2 = 0;
    while (1 << log2 < C) ++log2;
    int size = 0;
    while (bytes > kSlices[size]) ++size;
    const long n = std::min(P.rows, long(std::max(1, clusters.n[log2][size])));
    // Clusters that stay have to be resident all at once.  Set up while another
    // kernel's CTAs leave they do not fit as they would on an empty GPU, and the
    // last begin when the first have ended (190 us in place of 115): only few come
    // before their time.
    return launch(distill_kernel<T, GRAD, J>, n * C, kDistillThreads, kSlices[size], C, P, st, n * C <= 152);
}

template <class T, bool GRAD>
int distill(const DistillParams& P, cudaStream_t st) {
    return P.K <= 32 ? distill<T, GRAD, 1>(P, st) : P.K <= 64 ? distill<T, GRAD, 2>(P, st) : distill<T, GRAD, 4>(P, st);
}

template <class T>
int distill(const DistillParams& P, cudaStream_t st) {
    return P.grad ? distill<T, true>(P, st) : distill<T, false>(P, st);
}

}  // namespace

extern "C" {

// dtype: 0 fp32, 1 bf16, 2 fp16 logits [rows][V], rows `stride` elements apart;
// tokens int64 [rows] or NULL; K <= 128 alternatives, in top and ids [rows][K].
// Returns a cudaError_t.
int decoder_token_scores(const void* x, int dtype, long stride, long rows, long V, const void* tokens, int K, double inv_T,
                         void* logprobs, void* entropy, void* top, void* ids, void* stream) {
    if (rows < 1 || rows > (1L << 27) || V < 1 || V > (1L << 30) || K < 0 || K > kMaxTop || K > V || !(inv_T > 0.0))
        return int(cudaErrorInvalidValue);
    const ScoreParams P{x, stride, int(V), K, float(inv_T), float(inv_T * kLog2e), static_cast<const int64_t*>(tokens), static_cast<float*>(logprobs),
                        static_cast<float*>(entropy), static_cast<float*>(top), static_cast<int64_t*>(ids), 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == 0) return scores<float>(P, rows, st);
    if (dtype == 1) return scores<__nv_bfloat16>(P, rows, st);
    if (dtype == 2) return scores<__half>(P, rows, st);
    return int(cudaErrorInvalidValue);
}

// The longest row that decoder_distill takes: what 8 CTAs hold.
long decoder_distill_vocab(int dtype) { return long((kSliceMax / 16 - 1) * 8 * (dtype == 0 ? 4 : 8)); }

// ids int64, teacher fp32 [rows][K]; weight fp32 [rows] or NULL; loss fp32
// [rows]; grad [rows][V] contiguous, of the logits' type, or NULL.  Returns a
// cudaError_t.
int decoder_distill(const void* x, int dtype, long stride, long rows, long V, const void* ids, const void* teacher, int K,
                    const void* weight, int rest, double inv_T, void* loss, void* grad, void* stream) {
    if (rows < 1 || rows > (1L << 27) || V < 1 || V > decoder_distill_vocab(dtype) || K < 1 || K > kMaxTop || !(inv_T > 0.0))
        return int(cudaErrorInvalidValue);
    const float c = float(inv_T * kLog2e);
    const DistillParams P{x, stride, rows, int(V), K, rest, float(inv_T), float(inv_T - double(float(inv_T))), c, float(inv_T * kLog2e - double(c)), -160.f / c, static_cast<const int64_t*>(ids), static_cast<const float*>(teacher),
                          static_cast<const float*>(weight), static_cast<float*>(loss), grad, decoder::error_word()};
    if (!P.err) return int(cudaErrorInvalidValue);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == 0) return distill<float>(P, st);
    if (dtype == 1) return distill<__nv_bfloat16>(P, st);
    if (dtype == 2) return distill<__half>(P, st);
    return int(cudaErrorInvalidValue);
}

}  // extern "C"
