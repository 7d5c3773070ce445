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
// distillation reads it once and writes the gradient once.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

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
#ifndef SCORE_CTAS
#define SCORE_CTAS 512
#endif
#ifndef DISTILL_KB
#define DISTILL_KB 80
#endif
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

// sum e^(z - m) and sum e^(z - m) (x - m) of elements whose largest x is m, in
// fp32.  Elements of -inf weigh nothing; a NaN or +inf makes s NaN (m passes
// over NaN).  Differences x - m come before the product with 1 / T: masks of
// the type's lowest value stay finite.
struct Sums {
    float m, s, t;

    __device__ __forceinline__ void join(const Sums& o, float c) {
        const float to = fmaxf(m, o.m);
        Sums a = *this, b = o;
        a.shift(to, c);
        b.shift(to, c);
        m = to;
        s = a.s + b.s;
        t = a.t + b.t;
    }
    __device__ __forceinline__ void shift(float to, float c) {
        if (m == kNone || m == to) return;          // (-inf: s is 0, or NaN)
        const float by = m - to, f = ex2(by * c);
        t = f == 0.f ? 0.f : f * fmaf(by, s, t);    // (by may be the type's lowest value)
        s *= f;
    }
    __device__ __forceinline__ Sums from(int lane_mask) const {
        Sums o;
        o.m = __shfl_xor_sync(0xffffffffu, m, lane_mask);
        o.s = __shfl_xor_sync(0xffffffffu, s, lane_mask);
        o.t = __shfl_xor_sync(0xffffffffu, t, lane_mask);
        return o;
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

template <class T>
__device__ __forceinline__ float largest(const Word<T>& w) {
    float m = to_float(w.x[0]);
#pragma unroll
    for (int e = 1; e < Word<T>::N; ++e) m = fmaxf(m, to_float(w.x[e]));
    return m;
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

// 32 R keys over a warp, the p-th in lane p % 32's element p / 32.
template <int R>
struct Keys {
    Key k[R];

    template <int J>
    __device__ __forceinline__ void exchange(int lane, int up_bit) {
        // descending where position & up_bit is 0 (up_bit 0: everywhere)
        if constexpr (J >= 32) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r & (J / 32)) continue;
                const int q = r | (J / 32);
                const bool desc = ((r * 32 + lane) & up_bit) == 0;
                const Key a = k[r], b = k[q];
                const bool swap = desc ? a < b : a > b;
                k[r] = swap ? b : a;
                k[q] = swap ? a : b;
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool desc = ((r * 32 + lane) & up_bit) == 0, low = (lane & J) == 0;
                const Key o = __shfl_xor_sync(0xffffffffu, k[r], J);
                if (low == desc ? o > k[r] : o < k[r]) k[r] = o;
            }
        }
    }
    template <int J>
    __device__ __forceinline__ void tidy(int lane, int up_bit) {
        exchange<J>(lane, up_bit);
        if constexpr (J > 1) tidy<J / 2>(lane, up_bit);
    }
    template <int W>
    __device__ __forceinline__ void sort_by(int lane) {
        tidy<W / 2>(lane, W == 32 * R ? 0 : W);
        if constexpr (W < 32 * R) sort_by<W * 2>(lane);
    }
    __device__ __forceinline__ void sort(int lane) { sort_by<2>(lane); }
    // The 32 R largest of this and another, both in order.
    __device__ __forceinline__ void merge(const Keys& o, int lane) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Key b = __shfl_xor_sync(0xffffffffu, o.k[R - 1 - r], 31);
            if (b > k[r]) k[r] = b;
        }
        tidy<16 * R>(lane, 0);
    }
    __device__ __forceinline__ void put(Key* to, int lane) const {
#pragma unroll
        for (int r = 0; r < R; ++r) to[r * 32 + lane] = k[r];
    }
    __device__ __forceinline__ void get(const Key* from, int lane) {
#pragma unroll
        for (int r = 0; r < R; ++r) k[r] = from[r * 32 + lane];
    }
    __device__ __forceinline__ Key nth(int n) const {
        Key v = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (n / 32 == r) v = __shfl_sync(0xffffffffu, k[r], n % 32);
        return v;
    }
};

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

// The largest float below x (x finite), -inf for -inf.
__device__ __forceinline__ float below(float x) {
    const int b = __float_as_int(x);
    if (x == kNone) return x;
    return __int_as_float(x > 0.f ? b - 1 : x == 0.f ? int(0x80000001u) : b + 1);
}

struct ScoreParams {
    const void* x;
    long stride;
    int V, K;
    float inv_T, c;             // 1 / T; log2(e) / T
    const int64_t* tokens;      // or NULL
    float *logprobs, *entropy, *top;
    int64_t* ids;
};

// The CTA looks at four words of each lane at a time (two for R = 4, for the
// buffers' sake).  The softmax sums are a lane's own, with its own running
// maximum.  For the K largest, a lane puts the places of its elements above a
// bound into the warp's buffer (in any order), and from there they go, 32 R
// sorted at a time, into the warp's sorted list.  The bound is the larger of
// the list's K-th and what the CTA's warps know together: each has ceil(K /
// warps) lanes whose largest elements are at least so and so large, so the least
// of those is no larger than the K-th of all.  That is brought up to date after
// 1, 2, 4, ... looks; without it, each warp by its own list, most looks of a
// warp found candidates.  The bound stays as it is during a look, and a warp's
// looks go up the row, so an element that equals the list's K-th comes behind it.
template <class T, int R>
struct ScoreShape {
    static constexpr int N = Word<T>::N, U = R == 4 ? 2 : 4;
    // of a buffer: what a flush leaves, and a look's (a list fits in, at the end)
    static constexpr int CAP = 32 * R + 32 * U * N;
    static_assert(CAP >= 2 * 32 * R);
    static size_t smem(int warps, int cluster) { return R ? size_t(warps * CAP) * 4 + size_t(cluster) * 32 * R * sizeof(Key) : 0; }
};

template <class T, int R>
__global__ void __launch_bounds__(32 * kMaxWarps) score_kernel(const ScoreParams P) {
    using Shape = ScoreShape<T, R>;
    constexpr int N = Shape::N, U = Shape::U, CAP = Shape::CAP;
    constexpr bool TOP = R > 0;
    constexpr int RR = TOP ? R : 1;
    extern __shared__ __align__(16) int s_places[];
    __shared__ Sums s_sums[kMaxWarps], s_cta[kMaxCluster];
    __shared__ volatile float s_known[kMaxWarps];
    __shared__ int s_held[kMaxWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = int(blockDim.x) >> 5;
    Key *s_keys = reinterpret_cast<Key*>(s_places), *s_lists = s_keys + warps * CAP / 2;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const long row = long(blockIdx.x) / C;
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (lane == 0) s_held[warp] = 0;
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
    const int w0 = int(long(in.words) * rank / C), w1 = int(long(in.words) * (rank + 1) / C);
    const float c = P.c;
    const float2 c2 = make_float2(c, c);
    LaneSums sums;
    Keys<RR> list;
#pragma unroll
    for (int r = 0; r < RR; ++r) list.k[r] = 0;
    int* buf = s_places + warp * CAP;
    float bound = kNone, own = kNone;
    // the warps whose every lane has elements, and the lanes of each that the
    // bound goes by (more than there are: no bound)
    const int full = min(warps, (w1 - w0) / 32), share = full > 0 ? (P.K + full - 1) / full : 33;

    auto offer = [&](float x, int i) {
        if (x > bound) buf[atomicAdd(&s_held[warp], 1)] = i;
    };
    // the buffer's last 32 R into the list, until no more than `left` are in it
    auto flush = [&](int left) {
        __syncwarp();
        int held = *const_cast<volatile int*>(&s_held[warp]);
        if (held <= left) return;
        while (held > left) {
            Keys<RR> batch;
            const int from = max(0, held - 32 * RR);
#pragma unroll
            for (int r = 0; r < RR; ++r) {
                const int b = from + r * 32 + lane, i = b < held ? buf[b] : -1;
                batch.k[r] = i >= 0 ? make_key(to_float(in.x[i]), i) : 0;
            }
            held = from;
            batch.sort(lane);
            list.merge(batch, lane);
        }
        own = key_value(list.nth(P.K - 1));
        if (lane == 0) s_held[warp] = held;
        __syncwarp();
    };
    // elements that are not in words: before the first, behind the last
    auto single = [&](int i, bool is) {
        const float x = is ? to_float(in.x[i]) : kNone;
        sums.rise(x, c);
        if (is) sums.add<true>(make_float2(x, kNone), sums.minus_ref(), c2);
        if constexpr (TOP) {
            if (is) offer(x, i);
        }
    };

    if (rank == 0 && warp == 0) single(lane, lane < in.head);
    const Word<T>* body = in.body();
    int look = 0;
    for (int base = w0; base < w1 || look == 0; base += 32 * warps * U, ++look) {
        Word<T> words[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int w = base + u * 32 * warps + int(threadIdx.x);
            if (w < w1) words[u] = body[w];
            else
#pragma unroll
                for (int e = 0; e < N; ++e) words[u].x[e] = from_float<T>(kNone);
        }
        float top[U], most = kNone;
#pragma unroll
        for (int u = 0; u < U; ++u) most = fmaxf(most, top[u] = largest(words[u]));
        sums.rise(most, c);
        const float2 minus = sums.minus_ref();
#pragma unroll
        for (int u = 0; u < U; ++u) add_word<true>(sums, words[u], minus, c2);
        if constexpr (TOP) {
            if ((look & (look + 1)) == 0 && share <= 32) {
                const float mine = nth_of_lanes(sums.m, share, lane);
                if (lane == 0) s_known[warp] = mine;
                if (look == 0) __syncthreads();
                float least = lane < full ? s_known[lane] : INFINITY;
#pragma unroll
                for (int off = kMaxWarps / 2; off > 0; off /= 2) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, off));
                bound = below(__shfl_sync(0xffffffffu, least, 0));
            }
            bound = fmaxf(bound, own);
            if (__any_sync(0xffffffffu, most > bound)) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (top[u] > bound) {
#pragma unroll
                        for (int e = 0; e < N; ++e) offer(to_float(words[u].x[e]), in.at(base + u * 32 * warps + int(threadIdx.x)) + e);
                    }
                }
                flush(32 * RR - 1);
            }
        }
    }
    if (rank == C - 1 && warp == 0) {
        bound = fmaxf(bound, own);
        single(P.V - in.tail + lane, lane < in.tail);
    }

    // lanes, warps, CTAs
    Sums mine = sums.both();
#pragma unroll
    for (int off = 16; off > 0; off /= 2) mine.join(mine.from(off), c);
    if (lane == 0) s_sums[warp] = mine;
    // the lists of a power of two of places, pairs at a time
    auto merge_all = [&](Key* at, int step, int n) {
        for (int half = n / 2; half > 0; half /= 2) {
            __syncthreads();
            if (warp < half) {
                Keys<RR> o;
                o.get(at + (warp + half) * step, lane);
                list.merge(o, lane);
                if (half > 1) list.put(at + warp * step, lane);
            }
        }
    };
    if constexpr (TOP) {
        flush(0);
        __syncwarp();
        list.put(s_keys + warp * (CAP / 2), lane);
        merge_all(s_keys, CAP / 2, warps);
    }
    __syncthreads();
    if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (every CTA has begun)
        if (warp == 0) {
            if (lane == 0) {
                Sums all = s_sums[0];
                for (int w = 1; w < warps; ++w) all.join(s_sums[w], c);
                *cluster.map_shared_rank(&s_cta[rank], 0) = all;
            }
            if constexpr (TOP) list.put(cluster.map_shared_rank(s_lists + rank * 32 * RR, 0), lane);
        }
        cluster.sync();
        if (rank != 0) return;
        if constexpr (TOP) {
            if (warp < C) list.get(s_lists + warp * 32 * RR, lane);
            merge_all(s_lists, 32 * RR, C);
        }
    }
    if (warp != 0) return;
    const int parts = C > 1 ? C : warps;
    Sums all = lane < parts ? (C > 1 ? s_cta[lane] : s_sums[lane]) : Sums{kNone, 0.f, 0.f};
#pragma unroll
    for (int off = 16; off > 0; off /= 2) all.join(all.from(off), c);
    const bool empty = all.m == kNone && !(all.s != all.s);
    const float log_s = logf(all.s);
    auto logprob = [&](float x) { return empty ? kNone : (x - all.m) * P.inv_T - log_s; };
    if (lane == 0) {
        if (P.tokens) {
            const int64_t tok = P.tokens[row];
            P.logprobs[row] = tok < 0 ? 0.f : tok >= P.V ? NAN : logprob(to_float(in.x[tok]));
        }
        P.entropy[row] = empty ? 0.f : log_s - all.t / all.s * P.inv_T;
    }
    if constexpr (TOP) {
        int found = 0;
#pragma unroll
        for (int r = 0; r < RR; ++r) {
            const int p = r * 32 + lane;
            const Key k = list.k[r];
            found += __popc(__ballot_sync(0xffffffffu, k != 0));
            if (p < P.K && k != 0) {
                P.top[row * P.K + p] = logprob(key_value(k));
                P.ids[row * P.K + p] = key_index(k);
            }
        }
        // fewer than K above -inf: the first of the others
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

constexpr int kPieces = 4;            // copies that a CTA's slice arrives in
constexpr int kDistillThreads = 256;

struct DistillParams {
    const void* x;
    long stride;
    int V, K, rest;
    float inv_T, c, c_low;      // 1 / T; log2(e) / T, and what its rounding left
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

// A CTA's slice of the row comes into shared memory by bulk copies and stays
// there: the sums are taken from it, and once the cluster has the row's, the
// gradient is made from the same copy.  The teacher's tokens are taken out of the
// slice (-inf) before it is summed up and put in their own way, so the sum of all
// others is a sum and not a difference.  Everything that needs the teacher alone
// is done under the copies; the CTAs of other rows on the SM fill the waits.
template <class T>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams P) {
    constexpr int N = Word<T>::N;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_bar;
    __shared__ float2 s_warps[kDistillThreads / 32], s_cta[kMaxCluster];       // largest x, sum of the others' e^
    __shared__ __align__(16) int s_id[kMaxTop];
    __shared__ float s_q[kMaxTop];
    __shared__ float2 s_ids;                // the same of the teacher's tokens
    __shared__ float s_all[2];              // the teacher's sum, and its rest
    __shared__ volatile int s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const long row = long(blockIdx.x) / C;
    const uint32_t bar = tc::smem_u32(&s_bar);
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (tid == 0) {
        tc::mbar_init(bar, 1);
        s_abort = 0;
        tc::fence_mbar_init();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
    const int w0 = int(long(in.words) * rank / C), nw = int(long(in.words) * (rank + 1) / C) - w0;
    const float c = P.c, weight = P.weight ? P.weight[row] : 1.f;
    // the slice's edge elements, one to a thread: those before the row's first
    // word, those behind its last
    const int heads = rank == 0 ? in.head : 0, tails = rank == C - 1 ? in.tail : 0;
    const int edge = tid < heads ? tid : tid < heads + tails ? P.V - in.tail + tid - heads : -1;
    const Word<T>* slice = reinterpret_cast<const Word<T>*>(smem);
    T* flat = reinterpret_cast<T*>(smem);
    T* out = P.grad ? static_cast<T*>(P.grad) + row * P.V : nullptr;
    const bool words_out = out && (reinterpret_cast<uintptr_t>(out + in.head) & 15u) == 0;

    if (weight == 0.f) {         // a row that is left out
        if (rank == 0 && tid == 0) P.loss[row] = 0.f;
        if (out) {
            if (edge >= 0) out[edge] = from_float<T>(0.f);
            const int lo = in.at(w0), n = nw * N;
            if (words_out) {
                for (int w = tid; w < nw; w += kDistillThreads) reinterpret_cast<uint4*>(out + lo)[w] = make_uint4(0, 0, 0, 0);
            } else {
                for (int i = tid; i < n; i += kDistillThreads) out[lo + i] = from_float<T>(0.f);
            }
        }
        __syncwarp();
        if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        return;
    }
    if (tid == 0) {              // (it has made the barrier itself)
        tc::mbar_arrive_expect_tx(bar, uint32_t(nw) * 16u);
        for (int i = 0; i < kPieces; ++i) {
            const int lo = int(long(nw) * i / kPieces), n = int(long(nw) * (i + 1) / kPieces) - lo;
            if (n > 0) bulk_load(tc::smem_u32(slice + lo), in.body() + w0 + lo, uint32_t(n) * 16u, bar);
        }
    }

    // The teacher is warp 0's, four alternatives to a lane: tokens, their logits,
    // weights, and what they add to the sums.
    constexpr int J = kMaxTop / 32;
    const int first_word = in.at(w0);
    int id[J];
    float q[J], z[J];
    bool lead[J];                       // a token's first mention
    if (warp == 0) {
        bool poison = false;
        float top = kNone, top_z = kNone;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = j * 32 + lane;
            id[j] = -1;
            q[j] = z[j] = kNone;
            if (k < P.K) {
                const int64_t asked = P.ids[row * P.K + k];
                q[j] = P.teacher[row * P.K + k];
                poison |= asked >= P.V;
                if (asked >= 0 && asked < P.V) id[j] = int(asked);
                if (id[j] >= 0) z[j] = to_float(in.x[id[j]]);
                else q[j] = kNone;
            }
            s_id[k] = id[j];
            top = fmaxf(top, q[j]);
            top_z = fmaxf(top_z, z[j]);
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < J; ++j) lead[j] = id[j] >= 0;
        for (int k = 0; k < P.K; k += 4) {
            const int4 four = *reinterpret_cast<const int4*>(s_id + k);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int before = j * 32 + lane - k;      // how many of the four come before it
                lead[j] = lead[j] && !((before > 0 && four.x == id[j]) || (before > 1 && four.y == id[j]) || (before > 2 && four.z == id[j]) ||
                                       (before > 3 && four.w == id[j]));
            }
        }
        poison = __any_sync(0xffffffffu, poison);
#pragma unroll
        for (int off = 16; off > 0; off /= 2) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            top_z = fmaxf(top_z, __shfl_xor_sync(0xffffffffu, top_z, off));
        }
        if (P.rest || top == kNone) top = 0.f;
        float sum = 0.f, e = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            q[j] = expf(q[j] - top);
            sum += q[j];
            if (lead[j]) e += ex2((z[j] - (top_z == kNone ? 0.f : top_z)) * c);
        }
#pragma unroll
        for (int off = 16; off > 0; off /= 2) {
            sum += __shfl_xor_sync(0xffffffffu, sum, off);
            e += __shfl_xor_sync(0xffffffffu, e, off);
        }
        // in fp64 what is left of 1 (NaN for a row with a token outside the vocabulary)
        double q_all = 0.0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (!P.rest && sum != 0.f) q[j] /= sum;
            if (poison) q[j] = NAN;
            q_all += double(q[j]);
            s_q[j * 32 + lane] = q[j];
        }
#pragma unroll
        for (int off = 16; off > 0; off /= 2) q_all += __shfl_xor_sync(0xffffffffu, q_all, off);
        if (lane == 0) {
            s_ids = make_float2(top_z, e);
            s_all[0] = float(q_all);
            s_all[1] = P.rest ? float(1.0 - q_all > 0.0 || q_all != q_all ? 1.0 - q_all : 0.0) : 0.f;
        }
    }
    float edge_x = edge >= 0 ? to_float(in.x[edge]) : kNone;
    const bool landed = tc::mbar_wait(bar, 0, &s_abort, P.err, kErrRow);
    if (warp == 0 && landed) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (id[j] >= first_word && id[j] < first_word + nw * N) flat[id[j] - first_word] = from_float<T>(kNone);
    }
    __syncthreads();
    if (edge >= 0)
        for (int k = 0; k < P.K; ++k)
            if (s_id[k] == edge) edge_x = kNone;

    // the sum of all other tokens
    LaneSums sums;
    const float2 c2 = make_float2(c, c);
    if (edge >= 0) {
        sums.rise(edge_x, c);
        sums.add<false>(make_float2(edge_x, kNone), sums.minus_ref(), c2);
    }
#pragma unroll 2
    for (int w = tid; w < nw; w += kDistillThreads) {
        const Word<T> v = slice[w];
        sums.rise(largest(v), c);
        add_word<false>(sums, v, sums.minus_ref(), c2);
    }
    // of sums with their largest x, over `n` lanes (-inf: a sum of 0, or NaN)
    auto together = [&](float2 v, int n) {
        float m = v.x;
        for (int off = n / 2; off > 0; off /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
        if (v.x != kNone && v.x != m) v.y *= ex2((v.x - m) * c);
        for (int off = n / 2; off > 0; off /= 2) v.y += __shfl_xor_sync(0xffffffffu, v.y, off);
        return make_float2(m, v.y);
    };
    const float2 mine = together(make_float2(sums.m, sums.s.x + sums.s.y), 32);
    if (lane == 0) s_warps[warp] = mine;
    if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (every CTA has begun)
    __syncthreads();
    // to every CTA of the cluster
    if (warp == 0) {
        const float2 part = together(lane < kDistillThreads / 32 ? s_warps[lane] : make_float2(kNone, 0.f), 32);
        if (lane < C) *cluster.map_shared_rank(&s_cta[rank], lane) = part;
    }
    if (C > 1) cluster.sync();
    else __syncthreads();
    const float2 others = together(lane < C ? s_cta[lane] : make_float2(kNone, 0.f), 32), ids = s_ids;
    const float m = fmaxf(others.x, ids.x), ref = m == kNone ? 0.f : m;
    const float s_rest = others.x == kNone ? others.y : others.y * ex2((others.x - ref) * c);
    const float s_all_ids = ids.x == kNone ? ids.y : ids.y * ex2((ids.x - ref) * c), s_sum = s_rest + s_all_ids;
    // p_j = e_j / s_sum; the gradient of a token that is not the teacher's is
    // f p_j, of one that is (all p_j - q_j)
    const float q_rest = s_all[1], all = P.rest ? 1.f : s_all[0], inv_s = s_sum == 0.f ? 0.f : 1.f / s_sum;
    const float f = !P.rest ? all : s_rest == 0.f ? 1.f : 1.f - q_rest * s_sum / s_rest;

    if (out) {
        const float scale = weight * P.inv_T, k = f * inv_s * scale;
        if (words_out) {
#pragma unroll 2
            for (int w = tid; w < nw; w += kDistillThreads) {
                const Word<T> v = slice[w];
                Word<T> g;
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float2 two = weights_of<T>(make_float2(to_float(v.x[e]), to_float(v.x[e + 1])), ref, k, P);
                    g.x[e] = from_float<T>(two.x);
                    g.x[e + 1] = from_float<T>(two.y);
                }
                reinterpret_cast<Word<T>*>(out + first_word)[w] = g;
            }
        } else {
            for (int i = tid; i < nw * N; i += kDistillThreads)
                out[first_word + i] = from_float<T>(weights_of<T>(make_float2(to_float(flat[i]), 0.f), ref, k, P).x);
        }
        if (edge >= 0) out[edge] = from_float<T>(weights_of<T>(make_float2(edge_x, 0.f), ref, k, P).x);
        __syncthreads();
        if (warp == 0) {
            // the teacher's tokens, each by its first mention in the CTA that has it
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int i = id[j];
                const bool here = (i >= first_word && i < first_word + nw * N) || (rank == 0 && i < in.head) || (rank == C - 1 && i >= P.V - in.tail);
                if (!lead[j] || !here) continue;
                float sum = 0.f;
                for (int n = j * 32 + lane; n < P.K; ++n)
                    if (s_id[n] == i) sum += s_q[n];
                out[i] = from_float<T>(fmaf(scale * all, weights_of<T>(make_float2(z[j], 0.f), ref, inv_s, P).x, -scale * sum));
            }
        }
    }
    if (rank == 0 && warp == 0) {
        // in fp64: the terms are small differences of log probabilities
        const double log_s = s_sum == 0.f ? 0.0 : log(double(s_sum));
        double total = 0.0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (q[j] != 0.f)
                total += double(q[j]) * (log(double(q[j])) - (s_sum == 0.f ? -INFINITY : (double(z[j]) - double(ref)) * double(P.inv_T) - log_s));
        }
#pragma unroll
        for (int off = 16; off > 0; off /= 2) total += __shfl_xor_sync(0xffffffffu, total, off);
        if (lane == 0) {
            if (q_rest > 0.f) total += double(q_rest) * (log(double(q_rest)) - (log(double(s_rest)) - log_s));
            P.loss[row] = float(total * double(weight));
        }
    }
}

template <class Kernel, class Params>
int launch(Kernel kernel, long ctas, int threads, size_t smem, int cluster, const Params& P, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
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

// CTAs that share a row: as many as fill the GPU, of 4096 elements at least.
int score_cluster(long rows, long V) {
    int C = 1;
    while (C < kMaxCluster && rows * C < SCORE_CTAS && V >= 8192L * C) C *= 2;
    return C;
}

template <class T, int R>
int scores(const ScoreParams& P, long rows, cudaStream_t st) {
    using Shape = ScoreShape<T, R>;
    static splice::PerDevice<bool> kept;
    const cudaError_t e = allow(kept, score_kernel<T, R>, Shape::smem(kMaxWarps, kMaxCluster));
    if (e != cudaSuccess) return int(e);
    const int C = score_cluster(rows, P.V), warps = rows * C < 304 ? 16 : 8;
    return launch(score_kernel<T, R>, rows * C, 32 * warps, Shape::smem(warps, C), C, P, st);
}

template <class T>
int scores(const ScoreParams& P, long rows, cudaStream_t st) {
    if (P.K == 0) return scores<T, 0>(P, rows, st);
    if (P.K <= 32) return scores<T, 1>(P, rows, st);
    if (P.K <= 64) return scores<T, 2>(P, rows, st);
    return scores<T, 4>(P, rows, st);
}

// Bytes of a CTA's slice at the most.
constexpr size_t kSliceMax = 216 * 1024;

size_t slice_bytes(long V, size_t size, int C) { return (size_t(V) * size / 16 / C + 1) * 16; }

int distill_cluster(long rows, long V, size_t size) {
    int C = 1;
    while (C < kMaxCluster && slice_bytes(V, size, C) > DISTILL_KB * 1024) C *= 2;
    while (C < kMaxCluster && rows * C < 456 && V >= 8192L * C) C *= 2;
    return C;
}

template <class T>
int distill(const DistillParams& P, long rows, cudaStream_t st) {
    static splice::PerDevice<bool> kept;
    const cudaError_t e = allow(kept, distill_kernel<T>, kSliceMax);
    if (e != cudaSuccess) return int(e);
    const int C = distill_cluster(rows, P.V, sizeof(T));
    const size_t bytes = slice_bytes(P.V, sizeof(T), C);
    if (bytes > kSliceMax) return int(cudaErrorInvalidValue);
    return launch(distill_kernel<T>, rows * C, kDistillThreads, bytes, C, P, st);
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
                        static_cast<float*>(entropy), static_cast<float*>(top), static_cast<int64_t*>(ids)};
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
    const DistillParams P{x, stride, int(V), K, rest, float(inv_T), c, float(inv_T * kLog2e - double(c)), -160.f / c, static_cast<const int64_t*>(ids), static_cast<const float*>(teacher),
                          static_cast<const float*>(weight), static_cast<float*>(loss), grad, decoder::error_word()};
    if (!P.err) return int(cudaErrorInvalidValue);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == 0) return distill<float>(P, rows, st);
    if (dtype == 1) return distill<__nv_bfloat16>(P, rows, st);
    if (dtype == 2) return distill<__half>(P, rows, st);
    return int(cudaErrorInvalidValue);
}

}  // extern "C"
