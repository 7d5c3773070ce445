// The gradients of causal attention (causal.cu) with respect to queries, keys
// and values.  With P = exp(scale Q K^T - lse), which is computed again from the
// row's log sum, and delta = rowsum(dO * O):
//
//   dV = P^T dO      dP = dO V^T      dS = P * (dP - delta)
//   dK = scale dS^T Q                 dQ = scale dS K
//
// dK and dV sum over rows, dQ over keys.  Each is the sum of one CTA (or, in a
// fixed order, of the CTAs of one cluster) in TMEM: no atomics, so the same
// inputs give the same bits, and the sums over the query heads that share a kv
// head are taken there too.  The price is that S and dP are computed twice:
// seven products in place of five.
//
// Both passes are one kernel.  A CTA holds 128 rows of a fixed pair of operands
// (F1, F2) and streams blocks of another pair (X1, X2) past them:
//
//            F1  F2   X1  X2    P -> sum with X2    dS -> sum with X1
//   kKeys    K   V    Q   dO    dV                  dK
//   kQueries Q   dO   K   V     -                   dQ
//
// S = F1 X1^T and dP = F2 X2^T (128 x 64, fp32 in TMEM, two slots each), the
// element operations by two warpgroups that take every other block (a thread
// per row), P and dS rounded to bf16 over their slots as the A operands of the
// second products.  One warp issues all MMAs in the order dV(j) dK(j) S(j+2)
// dP(j+2): S(j+2) waits for dV(j)'s reading of its slot under dK(j), dP(j+2)
// for dK(j)'s under S(j+2).
//
// 256 dims: blocks of 32, and dK and dV, which do not fit in TMEM together, in
// a launch each.
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
using decoder::Operand;
using decoder::pack_bf16;
using decoder::tma_load_4d;
using decoder::tmem_ld32_done;
using decoder::tmem_st16;

constexpr int kRows = 128, kThreads = 320, kLoadWarp = 8, kMmaWarp = 9, kMaxStages = 4, kMaxShares = 8;
constexpr unsigned kErrLoad = 512, kErrMma = 1024, kErrOut = 2048, kErrDrain = 4096;
enum Pass { kKeys, kValuesOnly, kKeysOnly, kQueries };     // (both, dV, dK; dQ)

template <int D, int PASS>
struct Cfg {
    static constexpr bool BY_KEYS = PASS != kQueries, OUT_P = PASS == kKeys || PASS == kValuesOnly, OUT_S = PASS != kValuesOnly;
    static constexpr bool DP = OUT_S;                      // whether dP is needed
    static constexpr int BX = D == 256 ? 32 : 64, PANELS = D / 64;
    static constexpr int STAGES = D == 256 ? 3 : 4;
    static constexpr uint32_t F_BYTES = kRows * D * 2, X_BYTES = BX * D * 2;
    static constexpr uint32_t STAT_BYTES = BY_KEYS ? 2 * BX * 4 : 0;
    static constexpr uint32_t OFF_F2 = F_BYTES, OFF_X = OFF_F2 + (DP ? F_BYTES : 0);
    static constexpr uint32_t OFF_STAT = OFF_X + STAGES * 2 * X_BYTES, BYTES = OFF_STAT + STAGES * STAT_BYTES;
    static constexpr int OUTS = (OUT_P ? 1 : 0) + (OUT_S ? 1 : 0);
    static constexpr int COLS = OUTS * D / 2;              // a warpgroup's columns of the sums
    static constexpr int UNITS = COLS / 16;
    // TMEM columns
    static constexpr uint32_t COL_S = 0, COL_DP = 128, COL_SUM = 256, COL_S_SUM = COL_SUM + (OUT_P ? D : 0);
    static_assert(COL_S_SUM + (OUT_S ? D : 0) <= 512);
    static constexpr uint32_t inbox(int shares) { return uint32_t(shares) * 2 * ((UNITS + shares - 1) / shares) * 16 * kRows * 4; }
    // (more than half of an SM's, so that no two CTAs of these kernels share one:
    // each takes all of TMEM, and CTAs of two clusters that wait for one
    // another's would wait for ever)
    static constexpr uint32_t smem(int shares) {
        const uint32_t in = shares > 1 ? inbox(shares) : 0, all = (BYTES > in ? BYTES : in) + 1024;
        return all > 116 * 1024 ? all : 116 * 1024;
    }
    static_assert(smem(kMaxShares) <= 227 * 1024 - 512);
};

struct GradParams {
    const float *lse2, *delta;      // [B Hq][Tpad]: log2 of the row's sum (+inf where it has no weights), delta
    __nv_bfloat16 *p_sum, *s_sum;   // outputs
    long p_row, p_head, p_batch, s_row, s_head, s_batch;
    int Tq, Tk, Tpad, Hq, Hkv, B;
    int tiles;                      // of 128 fixed rows
    int shares;
    float scale, scale_log2;
    unsigned* err;
};

template <int D, int PASS>
__global__ void __launch_bounds__(kThreads, 1)
    grad_kernel(const __grid_constant__ CUtensorMap tm_f1, const __grid_constant__ CUtensorMap tm_f2,
                const __grid_constant__ CUtensorMap tm_x1, const __grid_constant__ CUtensorMap tm_x2, const GradParams P) {
    using C = Cfg<D, PASS>;
    constexpr int BX = C::BX, ST = C::STAGES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 15];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = tc::smem_u32(smem), bar0 = tc::smem_u32(bars);
    auto full = [&](int i) { return bar0 + 8u * i; };
    auto empty = [&](int i) { return bar0 + 8u * (kMaxStages + i); };
    const uint32_t bar1 = bar0 + 8u * 2 * kMaxStages;
    auto s_full = [&](int i) { return bar1 + 8u * i; };
    auto dp_full = [&](int i) { return bar1 + 8u * (2 + i); };
    auto p_ready = [&](int i) { return bar1 + 8u * (4 + i); };
    auto ds_ready = [&](int i) { return bar1 + 8u * (6 + i); };
    auto p_taken = [&](int i) { return bar1 + 8u * (8 + i); };
    auto ds_taken = [&](int i) { return bar1 + 8u * (10 + i); };
    const uint32_t f_full = bar1 + 8u * 12, sums = bar1 + 8u * 13, drain = bar1 + 8u * 14;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int share = P.shares > 1 ? int(cluster.block_rank()) : 0;

    // this CTA's fixed rows, and the blocks that pass by: by keys the blocks of
    // rows that see them, of all heads of the group; by queries the blocks of
    // keys that they see
    const int item = int(blockIdx.x) / P.shares, shift = P.Tk - P.Tq, G = P.Hq / P.Hkv;
    const int heads = C::BY_KEYS ? P.Hkv : P.Hq;
    const int head = item % heads, batch = item / heads % P.B;
    const int tile = C::BY_KEYS ? item / (heads * P.B) : P.tiles - 1 - item / (heads * P.B);    // long ones first
    const int row0 = tile * kRows;
    int first, per;      // a head's blocks
    if (C::BY_KEYS) {
        first = max(0, row0 - shift) / BX;
        per = max(0, (P.Tq + BX - 1) / BX - first);
    } else {
        first = 0;
        per = max(0, (min(P.Tk, row0 + kRows + shift) + BX - 1) / BX);
    }
    const long all = long(per) * (C::BY_KEYS ? G : 1);
    const int j0 = int(all * share / P.shares), n = int(all * (share + 1) / P.shares) - j0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * kMaxStages + 15; ++i) tc::mbar_init(bar0 + 8u * i, 1);
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(p_ready(i), kRows);
            tc::mbar_init(ds_ready(i), kRows);
        }
        s_abort = 0;
        tc::fence_mbar_init();
        tc::prefetch_tmap(&tm_f1);
        tc::prefetch_tmap(&tm_f2);
        tc::prefetch_tmap(&tm_x1);
        tc::prefetch_tmap(&tm_x2);
    }
    if (warp == kMmaWarp) {
        tc::tmem_alloc(tc::smem_u32(&s_tmem), 512);
        tc::tmem_relinquish();
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    // By keys: a programmatic dependent of what makes the rows' statistics.  By
    // queries: of the pass by keys, which it neither needs nor disturbs; its
    // CTAs start as that one's leave (all of them have begun by then, and with
    // that the statistics are there), and end after it.
    if constexpr (C::BY_KEYS) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = s_tmem;
    bool ok = true;

    if (warp == kLoadWarp) {
        const bool leader = tc::elect_one();
        if (n > 0 && leader) {
            tc::mbar_arrive_expect_tx(f_full, C::DP ? 2 * C::F_BYTES : C::F_BYTES);
#pragma unroll
            for (int p = 0; p < C::PANELS; ++p) {
                tma_load_4d(sbase + p * (kRows * 128), &tm_f1, p * 64, row0, head, batch, f_full);
                if (C::DP) tma_load_4d(sbase + C::OFF_F2 + p * (kRows * 128), &tm_f2, p * 64, row0, head, batch, f_full);
            }
        }
        int j = 0;
        for (; j < n; ++j) {
            const int s = j % ST;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(empty(s), (uint32_t(j / ST) & 1u) ^ 1u, &s_abort, P.err, kErrLoad));
            if (!ok) break;
            if (leader) {
                const int at = (first + (j0 + j) % per) * BX;
                const int x_head = C::BY_KEYS ? head * G + (j0 + j) / per : head / G;
                const uint32_t to = sbase + C::OFF_X + uint32_t(s) * 2 * C::X_BYTES;
                tc::mbar_arrive_expect_tx(full(s), 2 * C::X_BYTES + C::STAT_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p) {
                    tma_load_4d(to + p * (BX * 128), &tm_x1, p * 64, at, x_head, batch, full(s));
                    tma_load_4d(to + C::X_BYTES + p * (BX * 128), &tm_x2, p * 64, at, x_head, batch, full(s));
                }
                if constexpr (C::BY_KEYS) {
                    const long stat = (long(batch) * P.Hq + x_head) * P.Tpad + at;
                    const uint32_t st = sbase + C::OFF_STAT + uint32_t(s) * C::STAT_BYTES;
                    decoder::bulk_load(st, P.lse2 + stat, BX * 4, full(s));
                    decoder::bulk_load(st + BX * 4, P.delta + stat, BX * 4, full(s));
                }
            }
        }
        // Every copy issued must land before the CTA may exit, and the commits
        // on the stages' barriers must arrive.
        volatile int no_abort = 0;
        if (n > 0) tc::mbar_wait(f_full, 0, &no_abort, P.err, kErrDrain);
        for (int i = max(0, j - ST); i < j; ++i) tc::mbar_wait(full(i % ST), uint32_t(i / ST) & 1u, &no_abort, P.err, kErrDrain);
        for (int i = max(0, j - ST); ok && i < j; ++i)
            ok = tc::mbar_wait(empty(i % ST), uint32_t(i / ST) & 1u, &s_abort, P.err, kErrDrain);
    } else if (warp == kMmaWarp) {
        const bool leader = tc::elect_one();
        constexpr uint32_t idesc_s = tc::idesc_bf16_f32(kRows, BX, false), idesc_sum = tc::idesc_bf16_f32(kRows, D, true);
        auto wait = [&](uint32_t bar, uint32_t phase) {
            return __all_sync(0xffffffffu, tc::mbar_wait(bar, phase & 1u, &s_abort, P.err, kErrMma));
        };
        // F X^T of block j into its slot
        auto first_product = [&](int j, uint32_t off_f, uint32_t off_x, uint32_t col, uint32_t done) {
            const uint32_t x = sbase + C::OFF_X + uint32_t(j % ST) * 2 * C::X_BYTES + off_x;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t a = tc::sw128_desc(sbase + off_f + (kk / 4) * (kRows * 128) + (kk % 4) * 32, 16, 1024);
                const uint64_t b = tc::sw128_desc(x + (kk / 4) * (BX * 128) + (kk % 4) * 32, 16, 1024);
                tc::mma_f16_ss(tmem + col + uint32_t(j & 1) * 64, a, b, idesc_s, kk > 0 ? 1u : 0u);
            }
            tc::mma_commit(done);
        };
        // the slot's bf16 times X, added up
        auto second_product = [&](int j, uint32_t off_x, uint32_t col, uint32_t sum) {
            const uint32_t x = sbase + C::OFF_X + uint32_t(j % ST) * 2 * C::X_BYTES + off_x;
#pragma unroll
            for (int kk = 0; kk < BX / 16; ++kk)
                mma_f16_ts(tmem + sum, tmem + col + uint32_t(j & 1) * 64 + kk * 8, tc::sw128_desc(x + kk * 16 * 128, BX * 128, 1024), idesc_sum,
                           j > 0 || kk > 0 ? 1u : 0u);
        };
        bool any = false;
        ok = n == 0 || wait(f_full, 0);
        // (j runs two behind the first products)
        for (int j = -2; ok && j < n; ++j) {
            const int s = j & 1;
            const uint32_t phase = uint32_t(j >> 1);
            if (j >= 0) {
                if constexpr (C::OUT_P) {
                    ok = wait(p_ready(s), phase);
                    if (!ok) break;
                    tc::tc_fence_after();
                    if (leader) {
                        second_product(j, C::X_BYTES, C::COL_S, C::COL_SUM);
                        tc::mma_commit(p_taken(s));
                    }
                }
                if constexpr (C::OUT_S) {
                    ok = wait(ds_ready(s), phase);
                    if (!ok) break;
                    tc::tc_fence_after();
                    if (leader) {
                        second_product(j, 0, C::COL_DP, C::COL_S_SUM);
                        tc::mma_commit(ds_taken(s));
                    }
                }
                if (leader) tc::mma_commit(empty(j % ST));
            }
            if (j + 2 >= n) continue;
            const int next = j + 2;
            ok = wait(full(next % ST), uint32_t(next / ST));
            // (a slot's S has been read once its dS is there)
            if constexpr (C::OUT_P) ok = ok && (j < 0 || wait(p_taken(s), phase));
            if (!ok) break;
            tc::tc_fence_after();
            if (leader) first_product(next, 0, 0, C::COL_S, s_full(s));
            any = true;
            if constexpr (C::DP) {
                ok = j < 0 || wait(ds_taken(s), phase);
                if (!ok) break;
                tc::tc_fence_after();
                if (leader) first_product(next, C::OFF_F2, C::X_BYTES, C::COL_DP, dp_full(s));
            }
        }
        if (ok && n > 0) {
            if (leader) tc::mma_commit(sums);
            // the commits that nothing else waits for
            for (int j = max(0, n - 2); ok && j < n; ++j) {
                if constexpr (C::OUT_P) ok = wait(p_taken(j & 1), uint32_t(j >> 1));
                if constexpr (C::OUT_S) ok = ok && wait(ds_taken(j & 1), uint32_t(j >> 1));
            }
        }
        if (!ok && any && leader) {
            // let the MMAs already issued finish before TMEM is freed
            tc::mma_commit(drain);
            volatile int no_abort = 0;
            tc::mbar_wait(drain, 0, &no_abort, P.err, kErrDrain);
        }
    } else {
        const int wg = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + r;
        const uint32_t mine = tmem + (uint32_t((warp & 3) * 32) << 16);
        const uint32_t s_col = mine + C::COL_S + uint32_t(wg) * 64, dp_col = mine + C::COL_DP + uint32_t(wg) * 64;
        float row_lse = INFINITY, row_delta = 0.f;
        if constexpr (!C::BY_KEYS) {
            const long stat = (long(batch) * P.Hq + head) * P.Tpad + row;
            // (a row of one key: its weight is 1, whatever the scores are)
            row_lse = row + shift == 0 ? INFINITY : __ldcg(P.lse2 + stat);
            row_delta = __ldcg(P.delta + stat);
        }
        for (int j = wg; j < n; j += 2) {
            const uint32_t phase = uint32_t(j >> 1) & 1u;
            const int at = (first + (j0 + j) % per) * BX;
            // columns that the row's key is seen from, or the row sees: from lo, to hi
            int lo = 0, hi = BX, single = -1;
            bool masked;
            if constexpr (C::BY_KEYS) {
                masked = shift + at < row0 + kRows - 1;
                lo = row - shift - at;
                single = -(shift + at);
            } else {
                masked = at + BX > row0 + shift + 1;
                hi = row + shift + 1 - at;
            }
            const float* stat = reinterpret_cast<const float*>(smem + C::OFF_STAT + (j % ST) * C::STAT_BYTES);
            if constexpr (C::BY_KEYS) ok = __all_sync(0xffffffffu, tc::mbar_wait(full(j % ST), uint32_t(j / ST) & 1u, &s_abort, P.err, kErrOut));
            ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(s_full(wg), phase, &s_abort, P.err, kErrOut));
            if (!ok) break;
            tc::tc_fence_after();
            float p[BX / 32][32];
#pragma unroll
            for (int b = 0; b < BX / 32; ++b) {
                tmem_ld32_done(s_col + b * 32, p[b]);
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    float l[4] = {row_lse, row_lse, row_lse, row_lse};
                    if constexpr (C::BY_KEYS) *reinterpret_cast<float4*>(l) = *reinterpret_cast<const float4*>(stat + b * 32 + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[b][i + e] = ex2(fmaf(p[b][i + e], P.scale_log2, -l[e]));
                }
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (b * 32 + i < lo || b * 32 + i >= hi) p[b][i] = 0.f;
                }
                if constexpr (C::OUT_P) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack_bf16(p[b][2 * i], p[b][2 * i + 1]);
                    // (over S: columns 0-15 are read by now, as are 0-31 of the second half's 16-31)
                    tmem_st16(s_col + b * 16, w);
                }
            }
            if constexpr (C::OUT_P) {
                tc::tmem_wait_st();
                tc::tc_fence_before();
                tc::mbar_arrive(p_ready(wg));
            }
            if constexpr (C::OUT_S) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(dp_full(wg), phase, &s_abort, P.err, kErrOut));
                if (!ok) break;
                tc::tc_fence_after();
#pragma unroll
                for (int b = 0; b < BX / 32; ++b) {
                    float d[32];
                    tmem_ld32_done(dp_col + b * 32, d);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        float l[4] = {row_delta, row_delta, row_delta, row_delta};
                        if constexpr (C::BY_KEYS) *reinterpret_cast<float4*>(l) = *reinterpret_cast<const float4*>(stat + BX + b * 32 + i);
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[i + e] = p[b][i + e] * (d[i + e] - l[e]);
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (p[b][i] == 0.f || b * 32 + i == single) d[i] = 0.f;
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack_bf16(d[2 * i], d[2 * i + 1]);
                    tmem_st16(dp_col + b * 16, w);
                }
                tc::tmem_wait_st();
                tc::tc_fence_before();
                tc::mbar_arrive(ds_ready(wg));
            }
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(sums, 0, &s_abort, P.err, kErrOut));
        tc::tc_fence_after();
        // Sums out: a warpgroup's columns are one of two sums, or half of the one.
        // All lanes of a warp take part in the TMEM loads.
        if (P.shares == 1 && ok) {
            const bool of_p = C::OUT_P && (wg == 0 || !C::OUT_S), in = row < (C::BY_KEYS ? P.Tk : P.Tq);
            const int c0 = C::OUTS == 2 ? 0 : wg * C::COLS;
            __nv_bfloat16* out = of_p ? P.p_sum + batch * P.p_batch + head * P.p_head + row * P.p_row
                                      : P.s_sum + batch * P.s_batch + head * P.s_head + row * P.s_row;
            const float by = of_p ? 1.f : P.scale;
            uint4* dst = reinterpret_cast<uint4*>(out + c0);
#pragma unroll
            for (int c = 0; c < C::COLS; c += 32) {
                float o[32];
                if (n > 0) {
                    tmem_ld32_done(mine + C::COL_SUM + wg * C::COLS + c, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                }
                if (in) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[c / 8 + i] = make_uint4(pack_bf16(o[8 * i] * by, o[8 * i + 1] * by), pack_bf16(o[8 * i + 2] * by, o[8 * i + 3] * by),
                                                    pack_bf16(o[8 * i + 4] * by, o[8 * i + 5] * by), pack_bf16(o[8 * i + 6] * by, o[8 * i + 7] * by));
                }
            }
        }
    }
    __syncwarp();
    if (P.shares > 1) {
        // The sums, 16 columns at a time, go round the shares: each adds up its
        // part of everyone's in share order.  No CTA of the cluster has a copy
        // or an MMA in flight any more, so the operands' room is their inbox:
        // [from share][warpgroup][part][16][128] fp32.
        float* inbox = reinterpret_cast<float*>(smem);
        const int parts = (C::UNITS + P.shares - 1) / P.shares;
        constexpr int UNIT = 16 * kRows;
        const int wg = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + r;
        const uint32_t mine = tmem + (uint32_t((warp & 3) * 32) << 16) + C::COL_SUM + wg * C::COLS;
        cluster.sync();
        if (warp < 8 && ok) {
#pragma unroll
            for (int c = 0; c < C::COLS; c += 32) {
                float o[32];
                if (n > 0) {
                    tmem_ld32_done(mine + c, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int u = c / 16 + h;
                    float* box = cluster.map_shared_rank(inbox, u % P.shares) + size_t((share * 2 + wg) * parts + u / P.shares) * UNIT + r;
#pragma unroll
                    for (int e = 0; e < 16; ++e) box[e * kRows] = o[h * 16 + e];
                }
            }
        }
        cluster.sync();
        if (warp < 8 && ok && row < (C::BY_KEYS ? P.Tk : P.Tq)) {
            const bool of_p = C::OUT_P && (wg == 0 || !C::OUT_S);
            const int c0 = C::OUTS == 2 ? 0 : wg * C::COLS;
            __nv_bfloat16* out = of_p ? P.p_sum + batch * P.p_batch + head * P.p_head + row * P.p_row
                                      : P.s_sum + batch * P.s_batch + head * P.s_head + row * P.s_row;
            const float by = of_p ? 1.f : P.scale;
            for (int u = share, part = 0; u < C::UNITS; u += P.shares, ++part) {
                float sum[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e] = 0.f;
                for (int from = 0; from < P.shares; ++from) {
                    const float* box = inbox + size_t((from * 2 + wg) * parts + part) * UNIT + r;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[e] += box[e * kRows];
                }
                uint4* dst = reinterpret_cast<uint4*>(out + c0 + u * 16);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    dst[i] = make_uint4(pack_bf16(sum[8 * i] * by, sum[8 * i + 1] * by), pack_bf16(sum[8 * i + 2] * by, sum[8 * i + 3] * by),
                                        pack_bf16(sum[8 * i + 4] * by, sum[8 * i + 5] * by), pack_bf16(sum[8 * i + 6] * by, sum[8 * i + 7] * by));
            }
        }
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == kMmaWarp) tc::tmem_dealloc(tmem, 512);
    // (what follows on the stream waits for this grid alone)
    if constexpr (!C::BY_KEYS) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The rows' statistics: log2 of the sum of weights, and delta.  A warp per
// (row, head), rows behind the last as rows without weights.
template <int D>
__global__ void __launch_bounds__(256)
    stats_kernel(const Operand dout, const Operand out, const float* lse, float* lse2, float* delta, int Tq, int Tpad, int Hq, long units) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int V = D / 32;
    struct alignas(2 * V) Vec {
        __nv_bfloat16 x[V];
    };
    const int lane = threadIdx.x & 31;
    const long unit = long(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (unit >= units) return;
    const int head = int(unit % Hq);
    const long rest = unit / Hq, batch = rest / Tpad;
    const int row = int(rest % Tpad);
    float sum = 0.f;
    if (row < Tq) {
        const auto at = [&](const Operand& o) {
            return reinterpret_cast<const Vec*>(static_cast<const __nv_bfloat16*>(o.p) + batch * o.batch + head * o.head + row * o.row)[lane];
        };
        const Vec a = at(dout), b = at(out);
#pragma unroll
        for (int i = 0; i < V; ++i) sum = fmaf(__bfloat162float(a.x[i]), __bfloat162float(b.x[i]), sum);
#pragma unroll
        for (int off = 16; off > 0; off /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    }
    if (lane == 0) {
        const long to = (batch * Hq + head) * Tpad + row;
        const float l = row < Tq ? lse[(batch * Hq + head) * Tq + row] : -INFINITY;
        lse2[to] = l == -INFINITY ? INFINITY : l * 1.4426950408889634f;
        delta[to] = sum;
    }
}

// CTAs that share an item's blocks (host arithmetic only): the longest share
// no longer than half as much again as an SM's part of all blocks, as long as
// a share keeps 4.  (Rows whose blocks grow with the position: the last tile's
// are the most, the average over the tiles half of it and more.)
int shares_of(long longest, long total, int sms) {
    int s = 1;
    while (s < kMaxShares && longest >= 8L * s && longest * 2 * sms > 3L * total * s) s *= 2;
    return s;
}

template <int D, int PASS>
int launch(const CUtensorMap (&maps)[4], GradParams p, long longest, long total, cudaStream_t st) {
    using C = Cfg<D, PASS>;
    static splice::PerDevice<int> kept;
    int sms = 0;
    const cudaError_t e = kept.get(&sms, [](int dev, int* n) {
        cudaError_t err = cudaFuncSetAttribute(grad_kernel<D, PASS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(C::smem(kMaxShares)));
        if (err == cudaSuccess) err = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
        return err;
    });
    if (e != cudaSuccess) return int(e);
    p.shares = shares_of(longest, total, sms);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(p.tiles) * unsigned(C::BY_KEYS ? p.Hkv : p.Hq) * unsigned(p.B) * unsigned(p.shares));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::smem(p.shares);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(p.shares);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return int(cudaLaunchKernelEx(&cfg, grad_kernel<D, PASS>, maps[0], maps[1], maps[2], maps[3], p));
}

struct Args {
    Operand dout, q, k, v, out;
    const float* lse;
    float* stats;
    __nv_bfloat16 *dq, *dk, *dv;
    int B, Tq, Tk, Hq, Hkv;
    float scale;
};

int padded(int T) { return (T + kRows - 1) / kRows * kRows; }

template <int D>
int backward(const Args& a, cudaStream_t st) {
    constexpr int BX = Cfg<D, kQueries>::BX;
    const int Tpad = padded(a.Tq), shift = a.Tk - a.Tq, G = a.Hq / a.Hkv;
    const long rows = long(a.B) * a.Hq * Tpad;
    float *lse2 = a.stats, *delta = a.stats + rows;
    {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned((rows + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        const int e = int(cudaLaunchKernelEx(&cfg, stats_kernel<D>, a.dout, a.out, a.lse, lse2, delta, a.Tq, Tpad, a.Hq, rows));
        if (e != 0) return e;
    }
    CUtensorMap fixed_k, fixed_v, fixed_q, fixed_o, block_k, block_v, block_q, block_o;
    if (!decoder::operand_map(&fixed_k, a.k, D, a.Tk, a.Hkv, a.B, kRows) || !decoder::operand_map(&fixed_v, a.v, D, a.Tk, a.Hkv, a.B, kRows) ||
        !decoder::operand_map(&fixed_q, a.q, D, a.Tq, a.Hq, a.B, kRows) || !decoder::operand_map(&fixed_o, a.dout, D, a.Tq, a.Hq, a.B, kRows) ||
        !decoder::operand_map(&block_k, a.k, D, a.Tk, a.Hkv, a.B, BX) || !decoder::operand_map(&block_v, a.v, D, a.Tk, a.Hkv, a.B, BX) ||
        !decoder::operand_map(&block_q, a.q, D, a.Tq, a.Hq, a.B, BX) || !decoder::operand_map(&block_o, a.dout, D, a.Tq, a.Hq, a.B, BX))
        return int(cudaErrorInvalidValue);
    GradParams p{};
    p.lse2 = lse2;
    p.delta = delta;
    p.Tq = a.Tq;
    p.Tk = a.Tk;
    p.Tpad = Tpad;
    p.Hq = a.Hq;
    p.Hkv = a.Hkv;
    p.B = a.B;
    p.scale = a.scale;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.err = decoder::error_word();
    if (!p.err) return int(cudaErrorInvalidValue);
    // by keys
    p.p_sum = a.dv;
    p.s_sum = a.dk;
    p.p_row = p.s_row = D;
    p.p_head = p.s_head = long(a.Tk) * D;
    p.p_batch = p.s_batch = long(a.Hkv) * a.Tk * D;
    p.tiles = (a.Tk + kRows - 1) / kRows;
    const int blocks = (a.Tq + BX - 1) / BX;
    long longest = 0, total = 0;
    for (int t = 0; t < p.tiles; ++t) {
        const long n = long(G) * std::max(0, blocks - std::max(0, t * kRows - shift) / BX);
        longest = std::max(longest, n);
        total += n;
    }
    total *= long(a.Hkv) * a.B;
    const CUtensorMap by_keys[4] = {fixed_k, fixed_v, block_q, block_o};
    int e;
    if constexpr (D == 256) {
        e = launch<D, kValuesOnly>(by_keys, p, longest, total, st);
        if (e == 0) e = launch<D, kKeysOnly>(by_keys, p, longest, total, st);
    } else {
        e = launch<D, kKeys>(by_keys, p, longest, total, st);
    }
    if (e != 0) return e;
    // by queries
    p.s_sum = a.dq;
    p.s_row = long(a.Hq) * D;
    p.s_head = D;
    p.s_batch = long(a.Tq) * a.Hq * D;
    p.tiles = Tpad / kRows;
    longest = total = 0;
    for (int t = 0; t < p.tiles; ++t) {
        const long n = std::max(0, (std::min(a.Tk, (t + 1) * kRows + shift) + BX - 1) / BX);
        longest = std::max(longest, n);
        total += n;
    }
    total *= long(a.Hq) * a.B;
    const CUtensorMap by_queries[4] = {fixed_q, fixed_o, block_k, block_v};
    return launch<D, kQueries>(by_queries, p, longest, total, st);
}

}  // namespace

extern "C" {

// Bytes of scratch that decoder_attention_backward needs.
long decoder_attention_scratch(long B, long Tq, int Hq) { return 8 * B * Hq * ((Tq + kRows - 1) / kRows * kRows); }

// Gradients of decoder_attention: dout, q [B][Tq][Hq][d], k, v [B][Hkv][Tk][d]
// and out [B][Tq][Hq][d] of any strides that are multiples of 8 elements (row,
// head, batch of each in this order), lse as that gives it; dq [B][Tq][Hq][d],
// dk, dv [B][Hkv][Tk][d] contiguous; all bf16 and 16-byte aligned.  Returns a
// cudaError_t.
int decoder_attention_backward(const void* dout, const void* q, const void* k, const void* v, const void* out, const void* lse,
                               const long* strides, void* scratch, void* dq, void* dk, void* dv, long B, long Tq, long Tk, int Hq,
                               int Hkv, int d, float scale, void* stream) {
    if (!decoder::attention_takes(B, Tq, Tk, Hq, Hkv)) return int(cudaErrorInvalidValue);
    auto operand = [&](const void* p, int i) { return Operand{p, strides[3 * i], strides[3 * i + 1], strides[3 * i + 2]}; };
    const Args a{operand(dout, 0), operand(q, 1), operand(k, 2), operand(v, 3), operand(out, 4), static_cast<const float*>(lse),
                 static_cast<float*>(scratch), static_cast<__nv_bfloat16*>(dq), static_cast<__nv_bfloat16*>(dk),
                 static_cast<__nv_bfloat16*>(dv), int(B), int(Tq), int(Tk), Hq, Hkv, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d == 64) return backward<64>(a, st);
    if (d == 128) return backward<128>(a, st);
    if (d == 256) return backward<256>(a, st);
    return int(cudaErrorInvalidValue);
}

}  // extern "C"
