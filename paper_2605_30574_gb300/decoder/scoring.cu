// What a row of logits says, in one pass over it, for logits x [row][V] of
// fp32, bf16 or fp16 at a temperature T (z = x / T):
//
//   token scores   log p of a given token, the entropy of p = softmax(z), and
//                  the K largest log p with their tokens
//   distillation   the divergence of p from a teacher's K alternatives, and its
//                  gradient with respect to x
//
// A row is shared by a cluster of 1 to 8 CTAs, which trade their parts through
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

constexpr int kMaxTop = 128, kMaxCluster = 8;
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

    __device__ __forceinline__ void rise(float to, float c) {
        if (to > m) {
            shift(to, c);
            m = to;
        }
    }
    // (m at least x already; ref: m, or 0 while m is -inf)
    __device__ __forceinline__ void add(float x, float ref, float c) {
        const float by = x - ref, e = ex2(by * c);
        s += e;
        t = fmaf(e, fmaxf(by, -3.0e38f), t);
    }
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

// A warp looks at 512 elements at a time, 16 to a lane (256 for R = 4, for its
// buffer's sake).  The softmax sums are
// a lane's own, with its own running maximum.  For the K largest, the elements
// above a bound go to the warp's buffer, and from there, 32 R sorted at a time,
// into its sorted list.  The bound is the larger of the list's K-th and what
// the CTA's warps know together: each has ceil(K / warps) lanes whose largest
// elements are at least so and so large, so the least of those is no larger
// than the K-th of all.  That is read and brought up to date after 1, 2, 4,
// ... looks, and without it (each warp by its list alone) most looks of a warp
// find candidates.
// The bound stays as it is during a look, and looks go up the row, so an
// element that equals the list's K-th comes behind it.
template <class T, int R, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) score_kernel(const ScoreParams P) {
    constexpr int N = Word<T>::N, U = (R == 4 ? 8 : 16) / N;
    constexpr int CAP = 32 * R + 32 * U * N;      // (what a flush leaves, and a look's)
    constexpr bool TOP = R > 0;
    constexpr int RR = TOP ? R : 1;
    __shared__ Sums s_sums[WARPS], s_cta[kMaxCluster];
    __shared__ Key s_keys[TOP ? WARPS * CAP : 1], s_lists[TOP ? kMaxCluster * 32 * RR : 1];
    __shared__ volatile float s_known[WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const long row = long(blockIdx.x) / C;
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
    const int w0 = int(long(in.words) * rank / C), w1 = int(long(in.words) * (rank + 1) / C);
    const float c = P.c;
    Sums sums{kNone, 0.f, 0.f};
    Keys<RR> list;
#pragma unroll
    for (int r = 0; r < RR; ++r) list.k[r] = 0;
    Key* buf = s_keys + warp * CAP;
    int held = 0;
    float bound = kNone, own = kNone;
    const int share = TOP ? (P.K + WARPS - 1) / WARPS : 1;

    auto offer = [&](float x, int i) {
        const bool in_it = x > bound;
        const unsigned who = __ballot_sync(0xffffffffu, in_it);
        if (in_it) buf[held + __popc(who & ((1u << lane) - 1u))] = make_key(x, i);
        held += __popc(who);
    };
    // the buffer's last 32 R into the list, until no more than `left` are in it
    auto flush = [&](int left) {
        while (held > left) {
            Keys<RR> batch;
            const int from = max(0, held - 32 * RR);
            __syncwarp();
#pragma unroll
            for (int r = 0; r < RR; ++r) batch.k[r] = from + r * 32 + lane < held ? buf[from + r * 32 + lane] : 0;
            __syncwarp();
            held = from;
            batch.sort(lane);
            list.merge(batch, lane);
        }
        own = key_value(list.nth(P.K - 1));
    };

    // the elements before the first word
    if (rank == 0 && warp == 0) {
        const float x = lane < in.head ? to_float(in.x[lane]) : kNone;
        sums.rise(x, c);
        if (lane < in.head) sums.add(x, sums.m == kNone ? 0.f : sums.m, c);
        if constexpr (TOP) offer(x, lane);
    }
    const Word<T>* body = in.body();
    int look = 0;
    for (int base = w0 + warp * 32 * U; base < w1 || look == 0; base += WARPS * 32 * U, ++look) {
        Word<T> words[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int w = base + u * 32 + lane;
            if (w < w1) words[u] = body[w];
            else
#pragma unroll
                for (int e = 0; e < N; ++e) words[u].x[e] = from_float<T>(kNone);
        }
        float most = kNone;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, to_float(words[u].x[e]));
        sums.rise(most, c);
        const float ref = sums.m == kNone ? 0.f : sums.m;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) sums.add(to_float(words[u].x[e]), ref, c);
        if constexpr (TOP) {
            if ((look & (look + 1)) == 0) {
                const float mine = nth_of_lanes(sums.m, share, lane);
                if (lane == 0) s_known[warp] = mine;
                if (look == 0) __syncthreads();
                float least = s_known[lane % WARPS];
#pragma unroll
                for (int off = WARPS / 2; off > 0; off /= 2) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, off));
                bound = below(least);
            }
            bound = fmaxf(bound, own);
            if (__any_sync(0xffffffffu, most > bound)) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < N; ++e) offer(to_float(words[u].x[e]), in.at(base + u * 32 + lane) + e);
                if (held >= 32 * RR) flush(32 * RR - 1);
            }
        }
    }
    // and those behind the last
    if (rank == C - 1 && warp == 0) {
        const int i = P.V - in.tail + lane;
        const float x = lane < in.tail ? to_float(in.x[i]) : kNone;
        sums.rise(x, c);
        if (lane < in.tail) sums.add(x, sums.m == kNone ? 0.f : sums.m, c);
        if constexpr (TOP) {
            bound = fmaxf(bound, own);
            offer(x, i);
        }
    }

    // lanes, warps, CTAs
#pragma unroll
    for (int off = 16; off > 0; off /= 2) sums.join(sums.from(off), c);
    if (lane == 0) s_sums[warp] = sums;
    if constexpr (TOP) {
        flush(0);
        __syncwarp();
        list.put(buf, lane);
    }
    __syncthreads();
    if constexpr (TOP) {
#pragma unroll
        for (int half = WARPS / 2; half > 0; half /= 2) {
            if (warp < half) {
                Keys<RR> o;
                o.get(s_keys + (warp + half) * CAP, lane);
                list.merge(o, lane);
                if (half > 1) list.put(buf, lane);
            }
            if (half > 1) __syncthreads();
        }
    }
    if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (every CTA has begun)
        if (warp == 0) {
            if (lane == 0) {
                Sums all = s_sums[0];
                for (int w = 1; w < WARPS; ++w) all.join(s_sums[w], c);
                *cluster.map_shared_rank(&s_cta[rank], 0) = all;
            }
            if constexpr (TOP) list.put(cluster.map_shared_rank(s_lists + rank * 32 * RR, 0), lane);
        }
        cluster.sync();
        if (rank != 0) return;
    }
    if (warp != 0) return;
    Sums all = C > 1 ? s_cta[0] : s_sums[0];
    for (int i = 1; i < (C > 1 ? C : WARPS); ++i) all.join(C > 1 ? s_cta[i] : s_sums[i], c);
    if constexpr (TOP) {
        for (int i = 1; i < C; ++i) {
            Keys<RR> o;
            o.get(s_lists + i * 32 * RR, lane);
            list.merge(o, lane);
        }
    }
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

constexpr int kParts = 8;             // pieces that a CTA's slice arrives in
constexpr int kDistillThreads = 256;

struct DistillParams {
    const void* x;
    long stride;
    int V, K, rest;
    float inv_T, c, c_low;      // 1 / T; log2(e) / T, and what its rounding left
    const int64_t* ids;
    const float* teacher;
    const float* weight;        // or NULL
    float* loss;
    void* grad;                 // or NULL
    unsigned* err;
};

// Sums a value of each thread, or takes the largest, in a fixed order.
template <class V, class Op>
__device__ __forceinline__ V over_block(V v, Op op, V* s) {
#pragma unroll
    for (int off = 16; off > 0; off /= 2) v = op(v, __shfl_xor_sync(0xffffffffu, v, off));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < kDistillThreads / 32; ++w) v = op(v, s[w]);
    __syncthreads();
    return v;
}

// e^(by / T) of a difference of logits, for a gradient of type T.  In fp32 with
// the exponent's rounding made good, which 30 below the maximum costs 1e-6 of
// the value (5 instructions of a pass that waits for memory).
template <class T>
__device__ __forceinline__ float weight_of(float by, const DistillParams& P) {
    if constexpr (sizeof(T) < 4) return ex2(by * P.c);
    const float y = by * P.c, e = ex2(y);
    const float low = fmaf(by, P.c_low, fmaf(by, P.c, -y));
    return y < -150.f ? 0.f : fmaf(e, low * 0.69314718f, e);
}

// A CTA's slice of the row comes into shared memory by bulk copies, all asked
// for at the start, and stays there: the sums are taken piece by piece as they
// land, and once the cluster has the row's, the gradient is made from the same
// copy.  The teacher's tokens are taken out of the slice (-inf) before it is
// summed up and put in their own way, so the sum of all others is a sum and not
// a difference.
template <class T>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams P) {
    constexpr int N = Word<T>::N;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kParts];
    __shared__ float2 s_cta[kMaxCluster];
    __shared__ int64_t s_id[kMaxTop];
    __shared__ float s_q[kMaxTop], s_f[kDistillThreads / 32];
    __shared__ double s_d[kDistillThreads / 32];
    __shared__ volatile int s_abort;
    const int tid = threadIdx.x;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const long row = long(blockIdx.x) / C;
    const uint32_t bar0 = tc::smem_u32(bars);
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < kParts; ++i) tc::mbar_init(bar0 + 8u * i, 1);
        s_abort = 0;
        tc::fence_mbar_init();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();

    const Row<T> in(static_cast<const T*>(P.x) + row * P.stride, P.V);
    const int w0 = int(long(in.words) * rank / C), nw = int(long(in.words) * (rank + 1) / C) - w0;
    const int per = (nw + kParts - 1) / kParts;              // words of a piece
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
    if (tid == 0) {
        for (int i = 0; i < kParts; ++i) {
            const int n = min(per, nw - i * per);
            if (n <= 0) break;
            tc::mbar_arrive_expect_tx(bar0 + 8u * i, uint32_t(n) * 16u);
            bulk_load(tc::smem_u32(slice + i * per), in.body() + w0 + i * per, uint32_t(n) * 16u, bar0 + 8u * i);
        }
    }

    // the teacher's tokens
    int64_t id = -1;
    float q = 0.f, z = kNone;           // (z: x, before the temperature)
    bool poison = false;
    if (tid < P.K) {
        id = P.ids[row * P.K + tid];
        q = P.teacher[row * P.K + tid];
        poison = id >= P.V;
        if (id >= P.V) id = -1;
        if (id >= 0) z = to_float(in.x[id]);
        s_id[tid] = id;
    }
    __syncthreads();
    bool first = id >= 0;               // a token's first mention
    for (int j = 0; first && j < tid; ++j) first = s_id[j] != id;
    float edge_x = edge >= 0 ? to_float(in.x[edge]) : kNone;
    if (edge >= 0)
        for (int j = 0; j < P.K; ++j)
            if (s_id[j] == edge) edge_x = kNone;
    const int place = id >= 0 ? int(id) - in.at(w0) : -1;     // in the slice's words
    const bool here = place >= 0 && place < nw * N;

    // the sum of all other tokens
    Sums sums{kNone, 0.f, 0.f};
    sums.rise(edge_x, c);
    if (edge >= 0) sums.add(edge_x, sums.m == kNone ? 0.f : sums.m, c);
    bool ok = true;
    for (int i = 0; i < kParts && i * per < nw; ++i) {
        const int lo = i * per, hi = min(nw, lo + per);
        ok = ok && tc::mbar_wait(bar0 + 8u * i, 0, &s_abort, P.err, kErrRow);
        if (here && ok && place >= lo * N && place < hi * N) flat[place] = from_float<T>(kNone);
        __syncthreads();
        for (int w = lo + tid; w < hi; w += kDistillThreads) {
            const Word<T> v = slice[w];
            float most = kNone;
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, to_float(v.x[e]));
            if (most > sums.m) {
                if (sums.m != kNone) sums.s *= ex2((sums.m - most) * c);
                sums.m = most;
            }
            const float ref = sums.m == kNone ? 0.f : sums.m;
#pragma unroll
            for (int e = 0; e < N; ++e) sums.s += ex2((to_float(v.x[e]) - ref) * c);
        }
    }
    const float most = over_block(fmaxf(sums.m, z), [](float a, float b) { return fmaxf(a, b); }, s_f);
    auto add = [](float a, float b) { return a + b; };
    if (sums.m != kNone && sums.m != most) sums.s *= ex2((sums.m - most) * c);
    float2 mine = make_float2(most, over_block(sums.s, add, s_f));
    // over the cluster: every CTA gets every part
    float m = mine.x, s_rest = mine.y;
    if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (every CTA has begun)
        if (tid < C) *cluster.map_shared_rank(&s_cta[rank], tid) = mine;
        cluster.sync();
        for (int i = 0; i < C; ++i) m = fmaxf(m, s_cta[i].x);
        s_rest = 0.f;
        for (int i = 0; i < C; ++i) s_rest += s_cta[i].x == kNone || s_cta[i].x == m ? s_cta[i].y : s_cta[i].y * ex2((s_cta[i].x - m) * c);
    }
    const float ref = m == kNone ? 0.f : m;
    const float e_id = id >= 0 ? weight_of<T>(z - ref, P) : 0.f;
    const float s_all = s_rest + over_block(first ? e_id : 0.f, add, s_f);

    // the teacher's weights
    const bool asked = id >= 0 && (q > kNone || q != q);
    if (P.rest) {
        q = asked ? expf(q) : 0.f;
    } else {
        const float top = over_block(asked ? q : kNone, [](float a, float b) { return fmaxf(a, b); }, s_f);
        q = asked ? expf(q - top) : 0.f;
        const float sum = over_block(q, add, s_f);
        if (asked) q /= sum;
    }
    if (poison) q = NAN;
    if (tid < P.K) s_q[tid] = q;
    auto add_d = [](double a, double b) { return a + b; };
    // (NaN for a row with a token outside the vocabulary)
    const double q_all = over_block(double(q), add_d, s_d);
    const float q_rest = P.rest ? float(1.0 - q_all > 0.0 || q_all != q_all ? 1.0 - q_all : 0.0) : 0.f;
    // p_j = e_j / s_all; the gradient of a token that is not the teacher's is
    // f p_j, of one that is (all p_j - q_j)
    const float all = P.rest ? 1.f : float(q_all), inv_s = s_all == 0.f ? 0.f : 1.f / s_all;
    const float f = !P.rest ? all : s_rest == 0.f ? 1.f : 1.f - q_rest * s_all / s_rest;

    if (rank == 0) {
        // in fp64: the terms are small differences of log probabilities
        const double log_s = s_all == 0.f ? 0.0 : log(double(s_all));
        double term = 0.0;
        if (q != 0.f && tid < P.K)
            term = double(q) * (log(double(q)) - (s_all == 0.f ? -INFINITY : (double(z) - double(ref)) * double(P.inv_T) - log_s));
        double total = over_block(term, add_d, s_d);
        if (tid == 0) {
            if (q_rest > 0.f) total += double(q_rest) * (log(double(q_rest)) - (log(double(s_rest)) - log_s));
            P.loss[row] = float(total * double(weight));
        }
    }
    if (out) {
        const float scale = weight * P.inv_T, k = f * inv_s * scale;
        const int lo = in.at(w0);
        if (words_out) {
            for (int w = tid; w < nw; w += kDistillThreads) {
                const Word<T> v = slice[w];
                Word<T> g;
#pragma unroll
                for (int e = 0; e < N; ++e) g.x[e] = from_float<T>(weight_of<T>(to_float(v.x[e]) - ref, P) * k);
                reinterpret_cast<Word<T>*>(out + lo)[w] = g;
            }
        } else {
            for (int i = tid; i < nw * N; i += kDistillThreads) out[lo + i] = from_float<T>(weight_of<T>(to_float(flat[i]) - ref, P) * k);
        }
        if (edge >= 0) out[edge] = from_float<T>(weight_of<T>(edge_x - ref, P) * k);
        __syncthreads();
        const bool on_edge = id >= 0 && ((rank == 0 && id < in.head) || (rank == C - 1 && id >= P.V - in.tail));
        if (first && (here || on_edge)) {
            float sum = 0.f;
            for (int j = tid; j < P.K; ++j)
                if (s_id[j] == id) sum += s_q[j];
            out[id] = from_float<T>(scale * (all * e_id * inv_s - sum));
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

// CTAs that share a row: as many as fill the GPU, of 4096 elements at least.
int score_cluster(long rows, long V) {
    int C = 1;
    while (C < kMaxCluster && rows * C < 1216 && V >= 8192L * C) C *= 2;
    return C;
}

template <class T>
int scores(const ScoreParams& P, long rows, cudaStream_t st) {
    const int C = score_cluster(rows, P.V);
    const long ctas = rows * C;
    constexpr int W = 8;
    if (P.K == 0) return launch(score_kernel<T, 0, W>, ctas, 32 * W, 0, C, P, st);
    if (P.K <= 32) return launch(score_kernel<T, 1, W>, ctas, 32 * W, 0, C, P, st);
    if (P.K <= 64) return launch(score_kernel<T, 2, W>, ctas, 32 * W, 0, C, P, st);
    return launch(score_kernel<T, 4, W>, ctas, 32 * W, 0, C, P, st);
}

// Bytes of a CTA's slice at the most.
constexpr size_t kSliceMax = 216 * 1024;

size_t slice_bytes(long V, size_t size, int C) { return (size_t(V) * size / 16 / C + 1) * 16; }

int distill_cluster(long rows, long V, size_t size) {
    int C = 1;
    while (C < kMaxCluster && slice_bytes(V, size, C) > 56 * 1024) C *= 2;
    while (C < kMaxCluster && rows * C < 456 && V >= 8192L * C) C *= 2;
    return C;
}

template <class T>
int distill(const DistillParams& P, long rows, cudaStream_t st) {
    static splice::PerDevice<bool> kept;
    bool set = false;
    const cudaError_t e = kept.get(&set, [](int, bool* done) {
        *done = true;
        return cudaFuncSetAttribute(distill_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSliceMax));
    });
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

// The longest row that decoder_distill takes.
long decoder_distill_vocab(int dtype) { return long((kSliceMax / 16 - 1) * kMaxCluster * (dtype == 0 ? 4 : 8)); }

// ids int64, teacher fp32 [rows][K]; weight fp32 [rows] or NULL; loss fp32
// [rows]; grad [rows][V] contiguous, of the logits' type, or NULL.  Returns a
// cudaError_t.
int decoder_distill(const void* x, int dtype, long stride, long rows, long V, const void* ids, const void* teacher, int K,
                    const void* weight, int rest, double inv_T, void* loss, void* grad, void* stream) {
    if (rows < 1 || rows > (1L << 27) || V < 1 || V > decoder_distill_vocab(dtype) || K < 1 || K > kMaxTop || !(inv_T > 0.0))
        return int(cudaErrorInvalidValue);
    const float c = float(inv_T * kLog2e);
    const DistillParams P{x, stride, int(V), K, rest, float(inv_T), c, float(inv_T * kLog2e - double(c)), static_cast<const int64_t*>(ids), static_cast<const float*>(teacher),
                          static_cast<const float*>(weight), static_cast<float*>(loss), grad, decoder::error_word()};
    if (!P.err) return int(cudaErrorInvalidValue);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == 0) return distill<float>(P, rows, st);
    if (dtype == 1) return distill<__nv_bfloat16>(P, rows, st);
    if (dtype == 2) return distill<__half>(P, rows, st);
    return int(cudaErrorInvalidValue);
}

}  // extern "C"
