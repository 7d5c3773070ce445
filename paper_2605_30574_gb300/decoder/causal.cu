// Causal attention of one sequence over itself, for the prefill: q [T][Hq][d],
// k, v [Hkv][T][d], out [T][Hq][d], all bf16; scores, sums and outputs in fp32,
// probabilities rounded to bf16 for their product with V (a tensor-core
// operand).
//
// A CTA takes 128 rows of one query head, on tcgen05, over key blocks of 64:
// S = Q K^T into one of two TMEM slots, softmax by four warps (a thread per
// row), P over S in its slot as the A operand of P V, O in TMEM.  The next
// block's Q K^T is issued before a block's softmax is waited for, and two CTAs
// share an SM (d <= 128), so that MMAs of one run under the softmax of the
// other; that softmax, 64 exponentials per thread and block at a quarter of a
// warp per clock, is the bound.  Tiles of many blocks come first, the heads of a
// kv head next to one another.  O is rescaled where a row's maximum grows, so
// that the largest weight is 1 exactly (left up to 2^8 behind, 7% faster but 3%
// further from 64 bits).  32 heads of 128, 8 for keys, against the flash kernel
// that torch picks: 256 tokens 7.2 us, 16.2; 1024 22.9, 53.4; 4096 143, 427; no
// further from 64 bits at any size.
//
// With the rows' log sums (LSE), for the gradients of attention_grad.cu: a batch,
// queries that are the last T of Tk positions, any strides, and P in two bf16 terms:
// 4096 tokens 173 us.  The second term makes the output the exact one's rounding
// (off by 1.5e-3 to 1.6e-3 of its size at 32 to 2000 keys, for 1.7e-3 to 2.0e-3); the
// gradients, whose delta takes it, gain no more than 2% of their error.  Few tiles share their keys over a cluster, whose CTAs trade
// maxima, sums and outputs through distributed shared memory: one row of 4196 keys
// 22.5 us, and 62 without.
//
// Every wait is bounded, as in gemm.cu.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
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

using decoder::ex2;
using decoder::mma_f16_ts;
using decoder::tma_load_4d;
using decoder::tmem_ld32_done;

constexpr int kRows = 128, kBN = 64, kThreads = 192;     // softmax: warps 0-3
constexpr int kLoadWarp = 4, kMmaWarp = 5, kMaxShares = 4;
constexpr unsigned kErrLoad = 16, kErrMma = 32, kErrOut = 64, kErrDrain = 128;

template <int D>
struct Cfg {
    static constexpr int PANELS = D / 64;
    static constexpr uint32_t Q_BYTES = kRows * D * 2, KV_BYTES = kBN * D * 2;
    static constexpr uint32_t OFF_K = Q_BYTES, OFF_V = OFF_K + 2 * KV_BYTES, BYTES = OFF_V + 2 * KV_BYTES;
    static constexpr int CTAS = D == 256 ? 1 : 2;        // per SM, by TMEM (and no third by shared memory)
    static constexpr uint32_t SMEM = (BYTES + 1024 > 80 * 1024 ? BYTES + 1024 : 80 * 1024);
    static constexpr uint32_t COL_O = 2 * kBN;
    static constexpr uint32_t TMEM = D == 256 ? 512 : 256;
    // what the CTAs of a cluster trade, in the operands' room
    static constexpr uint32_t OFF_STATS = D * kRows * 4;
    static_assert(OFF_STATS + kMaxShares * kRows * 8 <= BYTES && D / 16 % kMaxShares == 0);
    static_assert(COL_O + D <= TMEM && CTAS * TMEM <= 512 && (CTAS + 1) * (SMEM + 1024) > 228 * 1024);
};

template <int D, bool LSE>
__global__ void __launch_bounds__(kThreads, Cfg<D>::CTAS)
    causal_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                  const __grid_constant__ CUtensorMap tm_v, __nv_bfloat16* out, float* lse, int T, int Tk, int Hq, int G,
                  int heads, int shares, float scale_log2, unsigned* err) {
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[15];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    const uint32_t sbase = (tc::smem_u32(smem_raw) + 1023) & ~1023u, bar0 = tc::smem_u32(bars);
    const uint32_t qfull = bar0, pvdone = bar0 + 8, drain = bar0 + 16;
    auto kfull = [&](int i) { return bar0 + 24 + 8u * i; };
    auto vfull = [&](int i) { return bar0 + 40 + 8u * i; };
    auto kempty = [&](int i) { return bar0 + 56 + 8u * i; };
    auto vempty = [&](int i) { return bar0 + 72 + 8u * i; };
    auto sfull = [&](int i) { return bar0 + 88 + 8u * i; };
    auto pfull = [&](int i) { return bar0 + 104 + 8u * i; };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int share = LSE && shares > 1 ? int(cluster.block_rank()) : 0, item = LSE ? int(blockIdx.x) / shares : int(blockIdx.x);
    const int at = item % heads, head = at % Hq, batch = at / Hq;
    const int row0 = ((T + kRows - 1) / kRows - 1 - item / heads) * kRows;
    const int shift = Tk - T;            // row i sees the keys up to i + shift
    const int all = max(0, (min(Tk, row0 + kRows + shift) + kBN - 1) / kBN);
    const int first = LSE ? all * share / shares : 0, nblk = LSE ? all * (share + 1) / shares - first : all;    // this CTA's

    if (threadIdx.x == 0) {
        for (int i = 0; i < 13; ++i) tc::mbar_init(bar0 + 8u * i, 1);
        for (int i = 0; i < 2; ++i) tc::mbar_init(pfull(i), kRows);
        s_abort = 0;
        tc::fence_mbar_init();
        tc::prefetch_tmap(&tm_q);
        tc::prefetch_tmap(&tm_k);
        tc::prefetch_tmap(&tm_v);
    }
    if (warp == kMmaWarp) {
        tc::tmem_alloc(tc::smem_u32(&s_tmem), C::TMEM);
        tc::tmem_relinquish();
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    // (a programmatic dependent of what precedes it, as the other kernels are)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = s_tmem;
    float m = 0.f, l = 0.f;     // a row's maximum (log2), and sum
    bool ok = true;

    if (warp == kLoadWarp) {
        const bool leader = tc::elect_one();
        const int hk = head / G;
        if (leader) {
            tc::mbar_arrive_expect_tx(qfull, C::Q_BYTES);
#pragma unroll
            for (int p = 0; p < C::PANELS; ++p) tma_load_4d(sbase + p * (kRows * 128), &tm_q, p * 64, row0, head, batch, qfull);
        }
        int j = 0;
        for (; j < nblk; ++j) {
            const int s = j & 1;
            const uint32_t phase = (uint32_t(j >> 1) & 1u) ^ 1u;
            if (!__all_sync(0xffffffffu, tc::mbar_wait(kempty(s), phase, &s_abort, err, kErrLoad))) break;
            if (leader) {
                tc::mbar_arrive_expect_tx(kfull(s), C::KV_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p)
                    tma_load_4d(sbase + C::OFF_K + s * C::KV_BYTES + p * (kBN * 128), &tm_k, p * 64, (first + j) * kBN, hk, batch, kfull(s));
            }
            if (!__all_sync(0xffffffffu, tc::mbar_wait(vempty(s), phase, &s_abort, err, kErrLoad))) break;
            if (leader) {
                tc::mbar_arrive_expect_tx(vfull(s), C::KV_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p)
                    tma_load_4d(sbase + C::OFF_V + s * C::KV_BYTES + p * (kBN * 128), &tm_v, p * 64, (first + j) * kBN, hk, batch, vfull(s));
            }
        }
        // Every copy issued must land before the CTA may exit.  (A broken-off
        // round's own K block has had the second of the wait that ran out.)
        volatile int no_abort = 0;
        tc::mbar_wait(qfull, 0, &no_abort, err, kErrDrain);
        for (int i = max(0, j - 2); i < j; ++i) {
            tc::mbar_wait(kfull(i & 1), uint32_t(i >> 1) & 1u, &no_abort, err, kErrDrain);
            tc::mbar_wait(vfull(i & 1), uint32_t(i >> 1) & 1u, &no_abort, err, kErrDrain);
        }
        // So must the commits arrive: the last P V's comes after the stages',
        // but nothing says that two commits arrive in their order.
        ok = j == nblk;
        for (int i = max(0, j - 2); ok && i < j; ++i)
            ok = tc::mbar_wait(kempty(i & 1), uint32_t(i >> 1) & 1u, &s_abort, err, kErrDrain) &&
                 tc::mbar_wait(vempty(i & 1), uint32_t(i >> 1) & 1u, &s_abort, err, kErrDrain);
    } else if (warp == kMmaWarp) {
        const bool leader = tc::elect_one();
        constexpr uint32_t idesc_qk = tc::idesc_bf16_f32(kRows, kBN, false), idesc_pv = tc::idesc_bf16_f32(kRows, D, true);
        bool any = false;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(qfull, 0, &s_abort, err, kErrMma));
        for (int j = -1; ok && j < nblk; ++j) {
            if (j + 1 < nblk) {
                // S of block j + 1, once P V of block j - 1 has read P from
                // its slot (under the softmax of block j)
                const int s = (j + 1) & 1;
                ok = __all_sync(0xffffffffu, tc::mbar_wait(kfull(s), uint32_t((j + 1) >> 1) & 1u, &s_abort, err, kErrMma)) &&
                     (j < 1 || __all_sync(0xffffffffu, tc::mbar_wait(pvdone, uint32_t(j - 1) & 1u, &s_abort, err, kErrMma)));
                if (!ok) break;
                tc::tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t a = tc::sw128_desc(sbase + (kk / 4) * (kRows * 128) + (kk % 4) * 32, 16, 1024);
                        const uint64_t b = tc::sw128_desc(sbase + C::OFF_K + s * C::KV_BYTES + (kk / 4) * (kBN * 128) + (kk % 4) * 32, 16, 1024);
                        tc::mma_f16_ss(tmem + s * kBN, a, b, idesc_qk, kk > 0 ? 1u : 0u);
                    }
                    tc::mma_commit(sfull(s));
                    tc::mma_commit(kempty(s));
                }
                any = true;
            }
            if (j < 0) continue;
            const int s = j & 1;
            const uint32_t phase = uint32_t(j >> 1) & 1u;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(vfull(s), phase, &s_abort, err, kErrMma)) &&
                 __all_sync(0xffffffffu, tc::mbar_wait(pfull(s), phase, &s_abort, err, kErrMma));
            if (!ok) break;
            tc::tc_fence_after();
            if (leader) {
#pragma unroll
                for (int kk = 0; kk < kBN / 16; ++kk) {
                    const uint64_t b = tc::sw128_desc(sbase + C::OFF_V + s * C::KV_BYTES + kk * 16 * 128, kBN * 128, 1024);
                    mma_f16_ts(tmem + C::COL_O, tmem + s * kBN + kk * 8, b, idesc_pv, j > 0 || kk > 0 ? 1u : 0u);
                    if constexpr (LSE) mma_f16_ts(tmem + C::COL_O, tmem + s * kBN + 32 + kk * 8, b, idesc_pv, 1u);
                }
                tc::mma_commit(vempty(s));
                tc::mma_commit(pvdone);
            }
        }
        if (!ok && any && leader) {
            // let the MMAs already issued finish before TMEM is freed
            tc::mma_commit(drain);
            volatile int no_abort = 0;
            tc::mbar_wait(drain, 0, &no_abort, err, kErrDrain);
        }
    } else {
        const int row = row0 + warp * 32 + lane;
        const uint32_t mine = tmem + (uint32_t(warp * 32) << 16);
        m = nblk ? 0.f : -INFINITY;
        // A positive scale goes in with the exponent's fma, past the masking and
        // the maximum; one of zero or below would make NaN or +inf of a masked
        // score and turn the order round, so it goes in first.
        const bool scale_first = !(scale_log2 > 0.f);
        const float scale_later = scale_first ? 1.f : scale_log2;
        for (int j = 0; j < nblk; ++j) {
            const int s = j & 1;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(sfull(s), uint32_t(j >> 1) & 1u, &s_abort, err, kErrOut));
            if (!ok) break;
            tc::tc_fence_after();
            float v[2][32];
            tmem_ld32_done(mine + s * kBN, v[0]);
            tmem_ld32_done(mine + s * kBN + 32, v[1]);
            if (scale_first) {
#pragma unroll
                for (int i = 0; i < kBN; ++i) v[i >> 5][i & 31] *= scale_log2;
            }
            if ((first + j + 1) * kBN > row0 + shift + 1) {          // the diagonal's blocks
                const int last = row + shift - (first + j) * kBN;      // this row's last key in the block
#pragma unroll
                for (int i = 0; i < kBN; ++i)
                    if (i > last) v[i >> 5][i & 31] = -INFINITY;
            }
            float top = v[0][0];
#pragma unroll
            for (int i = 1; i < kBN; ++i) top = fmaxf(top, v[i >> 5][i & 31]);
            top *= scale_later;
            if (j == 0) {
                m = top;
            } else if (__any_sync(0xffffffffu, top > m)) {
                const float to = fmaxf(m, top), alpha = ex2(m - (to == -INFINITY ? 0.f : to));
                m = to;
                l *= alpha;
                // O is at rest: the last P V issued is the previous block's
                ok = __all_sync(0xffffffffu, tc::mbar_wait(pvdone, uint32_t(j - 1) & 1u, &s_abort, err, kErrOut));
                if (!ok) break;
                tc::tc_fence_after();
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    tmem_ld32_done(mine + C::COL_O + c, o);
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] *= alpha;
                    tc::tmem_st32(mine + C::COL_O + c, o);
                }
                tc::tmem_wait_st();
            }
            // a row whose every score so far is -inf has no weights yet
            const float ref = m == -INFINITY ? 0.f : m;
            // (the weights as they are used, rounded: their sum then makes up
            // for part of the rounding.  LSE: as they are, and used in two
            // terms of bf16)
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t pk[16], low[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float a = ex2(fmaf(v[half][2 * i], scale_later, -ref)), b = ex2(fmaf(v[half][2 * i + 1], scale_later, -ref));
                    const __nv_bfloat162 p2 = __floats2bfloat162_rn(a, b);
                    pk[i] = *reinterpret_cast<const uint32_t*>(&p2);
                    if constexpr (LSE) {
                        low[i] = decoder::pack_bf16(a - __low2float(p2), b - __high2float(p2));
                        part[i & 3] += a + b;
                    } else {
                        part[i & 3] += __low2float(p2) + __high2float(p2);
                    }
                }
                if constexpr (LSE) decoder::tmem_st16(mine + s * kBN + 32 + half * 16, low);
                decoder::tmem_st16(mine + s * kBN + half * 16, pk);
            }
            l += (part[0] + part[1]) + (part[2] + part[3]);
            tc::tmem_wait_st();
            // Each warp sees each of pvdone's phases (long complete by now):
            // one that went on without could take the last but one for the
            // last, as a wait tells a phase by its parity.
            if (j > 0) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(pvdone, uint32_t(j - 1) & 1u, &s_abort, err, kErrOut));
                if (!ok) break;
            }
            tc::tc_fence_before();
            tc::mbar_arrive(pfull(s));
        }
        if (ok && nblk) ok = __all_sync(0xffffffffu, tc::mbar_wait(pvdone, uint32_t(nblk - 1) & 1u, &s_abort, err, kErrOut));
        if (ok) tc::tc_fence_after();
        if (ok && shares == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;   // (no weights at all: zeros)
            if constexpr (LSE) {
                if (row < T) lse[size_t(at) * T + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
            uint4* dst = reinterpret_cast<uint4*>(out + ((size_t(batch) * T + row) * Hq + head) * D);
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                float o[32];
                if (nblk) {
                    tmem_ld32_done(mine + C::COL_O + c, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                }
                if (row < T) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __nv_bfloat162 p2 = __floats2bfloat162_rn(o[8 * i + 2 * e] * inv, o[8 * i + 2 * e + 1] * inv);
                            w[e] = *reinterpret_cast<const uint32_t*>(&p2);
                        }
                        dst[c / 8 + i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
        }
    }
    __syncwarp();
    if constexpr (LSE) {
        if (shares > 1) {
            // The rows' maxima and sums go to all, their outputs 16 columns at a time
            // round the shares: [from share][part][16][128] fp32.  (No CTA of the
            // cluster has a copy or an MMA in flight any more.)
            constexpr int UNITS = D / 16, UNIT = 16 * kRows;
            float* inbox = reinterpret_cast<float*>(smem_raw + (sbase - tc::smem_u32(smem_raw)));
            float2* stats = reinterpret_cast<float2*>(inbox) + C::OFF_STATS / 8;
            const int parts = UNITS / shares, r = warp * 32 + lane, row = row0 + r;
            const uint32_t mine = tmem + (uint32_t(warp * 32) << 16) + C::COL_O;
            const bool takes = warp < kLoadWarp && ok;
            cluster.sync();
            if (takes) {
                for (int to = 0; to < shares; ++to) cluster.map_shared_rank(stats, to)[share * kRows + r] = make_float2(m, l);
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    float o[16];
                    decoder::tmem_ld16_done(mine + u * 16, o);
                    float* box = cluster.map_shared_rank(inbox, u % shares) + (share * parts + u / shares) * UNIT + r;
#pragma unroll
                    for (int e = 0; e < 16; ++e) box[e * kRows] = nblk ? o[e] : 0.f;
                }
            }
            cluster.sync();
            if (takes && row < T) {
                float most = -INFINITY, sum = 0.f, by[kMaxShares];
                for (int from = 0; from < shares; ++from) most = fmaxf(most, stats[from * kRows + r].x);
#pragma unroll
                for (int from = 0; from < kMaxShares; ++from) {
                    if (from >= shares) break;
                    const float2 s = stats[from * kRows + r];
                    by[from] = s.x == -INFINITY ? 0.f : ex2(s.x - most);
                    sum += by[from] * s.y;
                }
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                if (share == 0) lse[size_t(at) * T + row] = sum == 0.f ? -INFINITY : (most + log2f(sum)) * 0.6931471805599453f;
                for (int part = 0; part < parts; ++part) {
                    float o[16] = {};
#pragma unroll
                    for (int from = 0; from < kMaxShares; ++from) {
                        if (from >= shares) break;
                        const float* box = inbox + (from * parts + part) * UNIT + r;
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = fmaf(by[from], box[e * kRows], o[e]);
                    }
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = decoder::pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
                    uint4* dst = reinterpret_cast<uint4*>(out + ((size_t(batch) * T + row) * Hq + head) * D + (part * shares + share) * 16);
                    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == kMmaWarp) tc::tmem_dealloc(tmem, C::TMEM);
}

// CTAs that share a tile's blocks of keys: as many as there are places for, of two
// blocks at least.  (32 heads of 128, one CTA and in twos and fours: 1 row of 512
// keys 11, 9.8 and 9.3 us, of 4196 62, 35 and 22.5, in eights no less; 400 rows of 4196, 128 tiles,
// 72, 57 and 66; 1024 rows, 256 tiles, 28.5, 26 and 46.)
int shares_of(long items, int blocks, int places) {
    int s = 1;
    while (s < kMaxShares && items * 2 * s <= places && blocks >= 4 * s) s *= 2;
    return s;
}

template <int D, bool LSE>
int launch(const decoder::Operand& q, const decoder::Operand& k, const decoder::Operand& v, void* out, float* lse, int B, int Tq, int Tk,
           int Hq, int Hkv, float scale, cudaStream_t st) {
    using C = Cfg<D>;
    static splice::PerDevice<int> kept;
    int sms = 0;
    const cudaError_t e = kept.get(&sms, [](int dev, int* n) {
        const cudaError_t err = cudaFuncSetAttribute(causal_kernel<D, LSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(C::SMEM));
        return err == cudaSuccess ? cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev) : err;
    });
    if (e != cudaSuccess) return int(e);
    unsigned* err = decoder::error_word();
    CUtensorMap mq, mk, mv;
    if (!err || !decoder::operand_map(&mq, q, D, Tq, Hq, B, kRows) || !decoder::operand_map(&mk, k, D, Tk, Hkv, B, kBN) ||
        !decoder::operand_map(&mv, v, D, Tk, Hkv, B, kBN))
        return int(cudaErrorInvalidValue);
    cudaLaunchConfig_t cfg = {};
    const unsigned items = unsigned((Tq + kRows - 1) / kRows) * unsigned(Hq) * unsigned(B);
    const int shares = LSE ? shares_of(items, (Tk + kBN - 1) / kBN, C::CTAS * sms) : 1;
    cfg.gridDim = dim3(items * unsigned(shares));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute a[2];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    a[1].id = cudaLaunchAttributeClusterDimension;
    a[1].val.clusterDim.x = unsigned(shares);
    a[1].val.clusterDim.y = a[1].val.clusterDim.z = 1;
    cfg.attrs = a;
    cfg.numAttrs = shares > 1 ? 2 : 1;
    return int(cudaLaunchKernelEx(&cfg, causal_kernel<D, LSE>, mq, mk, mv, static_cast<__nv_bfloat16*>(out), lse, Tq, Tk, Hq, Hq / Hkv,
                                  Hq * B, shares, scale * 1.4426950408889634f, err));
}

template <bool LSE>
int launch(const decoder::Operand& q, const decoder::Operand& k, const decoder::Operand& v, void* out, float* lse, long B, long Tq, long Tk,
           int Hq, int Hkv, int d, float scale, cudaStream_t st) {
    if (d == 64) return launch<64, LSE>(q, k, v, out, lse, int(B), int(Tq), int(Tk), Hq, Hkv, scale, st);
    if (d == 128) return launch<128, LSE>(q, k, v, out, lse, int(B), int(Tq), int(Tk), Hq, Hkv, scale, st);
    if (d == 256) return launch<256, LSE>(q, k, v, out, lse, int(B), int(Tq), int(Tk), Hq, Hkv, scale, st);
    return int(cudaErrorInvalidValue);
}

}  // namespace

extern "C" {

// See the head of this file; 16-byte aligned.  Returns a cudaError_t.
int decoder_causal(const void* q, const void* k, const void* v, void* out, long T, int Hq, int Hkv, int d, float scale,
                   void* stream) {
    if (T < 1 || T > (1 << 20) || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return int(cudaErrorInvalidValue);
    const decoder::Operand oq{q, long(Hq) * d, d, T * Hq * d}, ok{k, d, T * d, T * Hkv * d}, ov{v, d, T * d, T * Hkv * d};
    return launch<false>(oq, ok, ov, out, nullptr, 1, T, T, Hq, Hkv, d, scale, static_cast<cudaStream_t>(stream));
}

// The same for B sequences whose queries are the last Tq positions of the Tk
// (Tq above Tk: the first rows see nothing), with the rows' log sums: q
// [B][Tq][Hq][d], k, v [B][Hkv][Tk][d] of any strides that are multiples of 8
// elements (q row, head, batch, k row, head, batch, v row, head, batch; NULL:
// contiguous), out
// [B][Tq][Hq][d] contiguous, lse fp32 [B][Hq][Tq] (natural log of the sum of
// e^(scale q . k), -inf for a row that sees nothing).
int decoder_attention(const void* q, const void* k, const void* v, const long* strides, void* out, void* lse, long B, long Tq,
                      long Tk, int Hq, int Hkv, int d, float scale, void* stream) {
    if (!decoder::attention_takes(B, Tq, Tk, Hq, Hkv)) return int(cudaErrorInvalidValue);
    const long of_q[3] = {long(Hq) * d, d, Tq * Hq * d}, of_k[3] = {d, Tk * d, Tk * Hkv * d};
    auto operand = [&](const void* p, int i) {
        const long* s = strides ? strides + 3 * i : i == 0 ? of_q : of_k;
        return decoder::Operand{p, s[0], s[1], s[2]};
    };
    const decoder::Operand oq = operand(q, 0), ok = operand(k, 1), ov = operand(v, 2);
    return launch<true>(oq, ok, ov, out, static_cast<float*>(lse), B, Tq, Tk, Hq, Hkv, d, scale, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
