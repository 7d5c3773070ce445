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
// S = F1 X1^T and dP = F2 X2^T go to TMEM in fp32; four warpgroups, a thread per
// row and each with 32 of a block's columns, make P and dS of them, rounded to
// bf16 over their columns as the A operands of the second products (two with 64
// columns each took 1.9 times as long).  One warp issues all MMAs, blocks are of
// 128 (an MMA of 64 columns reads its A operand twice as often, and takes 48
// clocks in place of 32).
//
// What bounds the loop is shared memory, 128 bytes a clock: an SS MMA of 128 x
// 128 x 16 reads 8 KB in its 64 clocks, and a block's arrival writes 64 KB.  So
//
// * by queries, Q and dO stay in TMEM, as A operands (256 dims: Q only);
// * by keys, where a row of S is a key and lse and delta go by column, they are
//   not read from shared memory (a broadcast of 16 bytes takes as long as 512
//   different ones: 1024 clocks a block) but come with the products: S - lse /
//   scale is one more MMA, of ones with the three bf16 terms of the number.
//
// By keys, TMEM is full with a slot each for S and dP and the two sums (128
// dims); the order is dV(j) S(j+1) dK(j) dP(j+1), so that P(j+1) is made under
// dK(j) and dP(j+1), dS(j+1) under dV(j+1) and S(j+2).  By queries it is S(j+1)
// dQ(j) dP(j+1), or S(j+1) dP(j+1) dQ(j) where TMEM has a second slot for dP.
//
// 256 dims: blocks of 64, and dK and dV, which do not fit in TMEM together, in
// a launch each.
//
// 32 heads of 128, 8 for keys: 4096 positions 335 us in a row of calls of its own,
// 355 among others (1.03 and 0.97 PFLOP/s of the five products that the gradients
// are, 1.44 and 1.36 of the seven), 1024 49 and 52; 4 x 100 rows of 4196 136.  The
// loops take 84% (by keys) and 81% of the tensor cores' rate; a CTA's
// operands in, and its sums out, the time of 8 blocks more.
//
// P, dS and the outputs in bf16, 1.7e-3 of their size each, make errors of 2.3e-3;
// an fp32 product of P and dS has the outputs' 1.7e-3 alone, at tf32's half rate or
// of two bf16 terms each (ten products for seven).  delta has the error of an output
// in bf16 besides, which rows of few keys show: dQ and dK of 2, 6, 17 and 28
// positions would be off by 4.7e-3, 4.4e-3, 3.0e-3 and 2.4e-3.  dS sums to 0 over a
// row; so where the 32 keys of a thread by queries, or of a warp by keys, are all
// that there are, the sum that it has all the same, times P, is taken from it: 2.3e-3
// to 2.7e-3, in 14.6 us for 12.7 (8 heads of 64).  From 33 keys on it is not: 2.6e-3
// to 2.7e-3 at 33 to 40, 2.5e-3 to 2.6e-3 at 64 to 256, 2.4e-3 from 1000 on (means of
// 4 inputs; single ones of few rows up to 2.9e-3).
//
// Every wait is bounded, as in gemm.cu.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

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
using decoder::tmem_ld16_done;
using decoder::tmem_ld32_done;
using decoder::tmem_st16;
using decoder::tmem_st8;

constexpr int kRows = 128, kMaxStages = 4, kMaxShares = 8, kFew = 32;
constexpr unsigned kErrLoad = 512, kErrMma = 1024, kErrOut = 2048, kErrDrain = 4096;
// S - lse / scale, times the scale, has to be finite, and lse for a scale of 0:
// below this the scores make no difference.
constexpr float kLeastScale = 9.094947e-13f;               // 2^-40
enum Pass { kKeys, kValuesOnly, kKeysOnly, kQueries };     // (both, dV, dK; dQ)

template <int D, int PASS>
struct Cfg {
    static constexpr bool BY_KEYS = PASS != kQueries, OUT_P = PASS == kKeys || PASS == kValuesOnly, OUT_S = PASS != kValuesOnly;
    static constexpr int BX = D == 256 || (D == 128 && PASS == kKeys) ? 64 : 128, PANELS = D / 64;
    // warpgroups of the element operations, 32 columns of a block each; then the
    // warps that load and that issue
    static constexpr int WGS = BX / 32, LOAD_WARP = 4 * WGS, MMA_WARP = LOAD_WARP + 1, THREADS = 32 * (MMA_WARP + 1);
    // which of the fixed operands are in TMEM; whether P and dS have columns of
    // their own there (else they are written over S and dP, one slot each but
    // two of S for P alone)
    static constexpr bool T1 = D == 256 || (PASS == kKeys) == (D == 128), T2 = PASS == kQueries && D < 256;
    static constexpr bool P_OWN = PASS == kKeys, DS_OWN = OUT_S && D < 256;
    static constexpr int NS = OUT_S ? 1 : 2, ND = OUT_S ? 1 : 0;
    // rings of X1 and X2.  S(j + 1) is issued before a block's sums: three blocks
    // of X1 are then in use or on their way.
    static constexpr int R1 = D == 128 && PASS == kKeys ? 4 : D == 64 || PASS == kQueries ? 3 : 2;
    static constexpr int R2 = D == 128 && PASS == kKeys ? 4 : D == 64 ? 3 : 2;
    static constexpr uint32_t F_BYTES = kRows * D * 2, X_BYTES = BX * D * 2;
    // the rows' numbers come with X1: see stats_kernel; ONES meets them
    static constexpr uint32_t AUG_BYTES = BY_KEYS ? BX * 32 : 0, ONES_BYTES = BY_KEYS ? kRows * 32 + 128 : 0;
    static constexpr int F_LOADS = (T1 ? 0 : 1) + (OUT_S && !T2 ? 1 : 0);
    static constexpr uint32_t OFF_F2 = T1 ? 0 : F_BYTES, OFF_X1 = OFF_F2 + (OUT_S && !T2 ? F_BYTES : 0), OFF_X2 = OFF_X1 + R1 * X_BYTES;
    static constexpr uint32_t OFF_AUG = OFF_X2 + R2 * X_BYTES, OFF_ONES = OFF_AUG + R1 * AUG_BYTES, BYTES = OFF_ONES + ONES_BYTES;
    static constexpr int OUTS = (OUT_P ? 1 : 0) + (OUT_S ? 1 : 0);
    static constexpr int COLS = OUTS * D / WGS;            // a warpgroup's columns of the sums
    static constexpr int UNITS = COLS / 16;
    // TMEM columns
    static constexpr uint32_t COL_DP = NS * BX, COL_P = COL_DP + ND * BX, COL_DS = COL_P + (P_OWN ? BX / 2 : 0);
    static constexpr uint32_t COL_F1 = COL_DS + (DS_OWN ? BX / 2 : 0), COL_F2 = COL_F1 + (T1 ? D / 2 : 0);
    static constexpr uint32_t COL_SUM = COL_F2 + (T2 ? D / 2 : 0), COL_S_SUM = COL_SUM + (OUT_P ? D : 0);
    static_assert(COL_S_SUM + (OUT_S ? D : 0) <= 512);
    static constexpr uint32_t inbox(int shares) { return uint32_t(shares) * ((WGS * UNITS + shares - 1) / shares) * 16 * kRows * 4; }
    // (so much of an SM's that no CTA of these kernels shares one with another, or
    // with one of causal.cu: each takes all of TMEM, and CTAs of two clusters that
    // wait for one another's would wait for ever)
    static constexpr uint32_t smem(int shares) {
        const uint32_t in = shares > 1 ? inbox(shares) : 0, all = (BYTES > in ? BYTES : in) + 1024;
        return all > 150 * 1024 ? all : 150 * 1024;
    }
    static_assert(smem(kMaxShares) <= 227 * 1024 - 512);
};

// An operand without swizzle: 8 rows of 16 bytes of K at a time, `k_bytes` to
// the next 16 bytes of K, `rows_bytes` to the next 8 rows.
__device__ __forceinline__ uint64_t plain_desc(uint32_t saddr, uint32_t k_bytes, uint32_t rows_bytes) {
    return uint64_t((saddr >> 4) & 0x3FFFu) | uint64_t(k_bytes >> 4) << 16 | uint64_t(rows_bytes >> 4) << 32 | uint64_t(1) << 46;
}

// A ring's stage, and the parity of its round.
template <int N>
struct Ring {
    int s = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++s == N) {
            s = 0;
            phase ^= 1u;
        }
    }
};

struct GradParams {
    // [B Hq][Tpad]: log2 of the row's sum (+inf where it has no weights), delta;
    // the same for an MMA
    const float *lse2, *delta;
    const uint8_t* aug;
    Operand f1, f2;                 // the fixed operands that go to TMEM
    __nv_bfloat16 *p_sum, *s_sum;   // outputs
    long p_row, p_head, p_batch, s_row, s_head, s_batch;
    int Tq, Tk, Tpad, Hq, Hkv, B;
    int tiles;                      // of 128 fixed rows
    int shares;
    bool leads;                     // whether this pass is the first
    float scale, scale_log2;        // scale_log2 by keys: not below kLeastScale
    unsigned* err;
};

// (FEW: no more than kFew keys)
template <int D, int PASS, bool FEW>
__global__ void __launch_bounds__(Cfg<D, PASS>::THREADS, 1)
    grad_kernel(const __grid_constant__ CUtensorMap tm_f1, const __grid_constant__ CUtensorMap tm_f2,
                const __grid_constant__ CUtensorMap tm_x1, const __grid_constant__ CUtensorMap tm_x2, const GradParams P) {
    using C = Cfg<D, PASS>;
    constexpr int BX = C::BX, NS = C::NS;
    extern __shared__ uint8_t smem_raw[];
    constexpr int kBars = 4 * kMaxStages + 10;
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = tc::smem_u32(smem), bar0 = tc::smem_u32(bars);
    auto x1_full = [&](int i) { return bar0 + 8u * i; };
    auto x1_empty = [&](int i) { return bar0 + 8u * (kMaxStages + i); };
    auto x2_full = [&](int i) { return bar0 + 8u * (2 * kMaxStages + i); };
    auto x2_empty = [&](int i) { return bar0 + 8u * (3 * kMaxStages + i); };
    const uint32_t bar1 = bar0 + 8u * 4 * kMaxStages;
    auto p_ready = [&](int i) { return bar1 + 8u * i; };
    const uint32_t ds_ready = bar1 + 8u * 2, s_read = bar1 + 8u * 3, dp_read = bar1 + 8u * 4;      // (arrivals of all threads, up to here)
    const uint32_t s_full = bar1 + 8u * 5, dp_full = bar1 + 8u * 6, f_full = bar1 + 8u * 7, sums = bar1 + 8u * 8, drain = bar1 + 8u * 9;
    // A product's one commit (a second one right behind it waits for the first:
    // 300 clocks) tells all that it frees: the last that reads a block of X1 or X2
    // that its stage is empty, and with that what it has read or made besides.
    // Block j's S, dP and sums are complete with:
    auto s_done = [&](int j, uint32_t& phase) { return C::OUT_S ? (phase = j, s_full) : (phase = j / C::R1, x1_empty(j % C::R1)); };
    auto dp_done = [&](int j, uint32_t& phase) { return C::OUT_P ? (phase = j, dp_full) : (phase = j / C::R2, x2_empty(j % C::R2)); };
    auto p_done = [&](int j, uint32_t& phase) { return phase = j / C::R2, x2_empty(j % C::R2); };
    auto ds_done = [&](int j, uint32_t& phase) { return phase = j / C::R1, x1_empty(j % C::R1); };
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
        // (how many arrive: an issue or a commit, or all threads of the warpgroups)
        constexpr int kAll = C::WGS * kRows;
        for (int i = 0; i < kBars; ++i) {
            const uint32_t bar = bar0 + 8u * i;
            const bool threads = bar >= p_ready(0) && bar <= dp_read;
            tc::mbar_init(bar, threads ? kAll : bar == f_full ? (C::T1 || C::T2 ? kAll : 0) + (C::F_LOADS > 0 ? 1 : 0) : 1);
        }
        s_abort = 0;
        tc::fence_mbar_init();
        tc::prefetch_tmap(&tm_f1);
        tc::prefetch_tmap(&tm_f2);
        tc::prefetch_tmap(&tm_x1);
        tc::prefetch_tmap(&tm_x2);
    }
    if constexpr (C::BY_KEYS) {
        // [8 rows][8 of K], ones in the first three of K, and as many zeros, in turn
        uint4* ones = reinterpret_cast<uint4*>(smem + C::OFF_ONES);
        for (int i = threadIdx.x; i < int(C::ONES_BYTES / 16); i += C::THREADS)
            ones[i] = i & 8 ? make_uint4(0, 0, 0, 0) : make_uint4(0x3f803f80u, 0x3f80u, 0, 0);
        tc::fence_proxy_async_smem();
    }
    if (warp == C::MMA_WARP) {
        tc::tmem_alloc(tc::smem_u32(&s_tmem), 512);
        tc::tmem_relinquish();
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = s_tmem;
    bool ok = true;
    // The pass that leads is a programmatic dependent of what makes the rows'
    // statistics, and of nothing else (that has waited for all that is before): the
    // fixed operands are asked for first.  The others are dependents of the one
    // before them, which they neither need nor disturb: their CTAs start as that
    // one's leave (all of them have begun by then, and with that the statistics are
    // there), and end after it.
    auto statistics_are_there = [&]() {
        if (P.leads) asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    };

    // One lane of its warp loads and one issues, all of the loop: with every lane
    // in it, and each copy and MMA under a test for the one, an MMA took 35 to 50
    // clocks to issue in place of 10, a wait on a complete barrier 140, and the
    // whole backward pass 1.2 times as long.
    if (warp == C::LOAD_WARP) {
        const bool leader = tc::elect_one();
        if (!leader || n == 0) statistics_are_there();
        if (leader && n > 0) {
            auto wait = [&](uint32_t bar, uint32_t phase) { return tc::mbar_wait(bar, phase, &s_abort, P.err, kErrLoad); };
            if constexpr (C::F_LOADS > 0) {
                tc::mbar_arrive_expect_tx(f_full, C::F_LOADS * C::F_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p) {
                    if (!C::T1) tma_load_4d(sbase + p * (kRows * 128), &tm_f1, p * 64, row0, head, batch, f_full);
                    if (C::OUT_S && !C::T2) tma_load_4d(sbase + C::OFF_F2 + p * (kRows * 128), &tm_f2, p * 64, row0, head, batch, f_full);
                }
            }
            statistics_are_there();
            int j1 = 0, j2 = 0;      // blocks asked for
            int block = j0 % per, x_head = C::BY_KEYS ? head * G + j0 / per : head / G;
            Ring<C::R1> r1;
            Ring<C::R2> r2;
            for (; j2 < n; ++j2) {
                const int at = (first + block) * BX;
                ok = wait(x1_empty(r1.s), r1.phase ^ 1u);
                if (!ok) break;
                const uint32_t to1 = sbase + C::OFF_X1 + uint32_t(r1.s) * C::X_BYTES, bar1 = x1_full(r1.s);
                tc::mbar_arrive_expect_tx(bar1, C::X_BYTES + C::AUG_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p) tma_load_4d(to1 + p * (BX * 128), &tm_x1, p * 64, at, x_head, batch, bar1);
                if constexpr (C::BY_KEYS)
                    decoder::bulk_load(sbase + C::OFF_AUG + uint32_t(r1.s) * C::AUG_BYTES, P.aug + ((long(batch) * P.Hq + x_head) * P.Tpad + at) * 32,
                                       C::AUG_BYTES, bar1);
                r1.next();
                ++j1;
                ok = wait(x2_empty(r2.s), r2.phase ^ 1u);
                if (!ok) break;
                const uint32_t to2 = sbase + C::OFF_X2 + uint32_t(r2.s) * C::X_BYTES, bar2 = x2_full(r2.s);
                tc::mbar_arrive_expect_tx(bar2, C::X_BYTES);
#pragma unroll
                for (int p = 0; p < C::PANELS; ++p) tma_load_4d(to2 + p * (BX * 128), &tm_x2, p * 64, at, x_head, batch, bar2);
                r2.next();
                if (++block == per) {
                    block = 0;
                    x_head += C::BY_KEYS ? 1 : 0;
                }
            }
            // Every copy issued must land before the CTA may exit, and the commits
            // on the stages' barriers must arrive.
            volatile int no_abort = 0;
            tc::mbar_wait(f_full, 0, &no_abort, P.err, kErrDrain);
            for (int i = max(0, j1 - C::R1); i < j1; ++i) tc::mbar_wait(x1_full(i % C::R1), uint32_t(i / C::R1) & 1u, &no_abort, P.err, kErrDrain);
            for (int i = max(0, j2 - C::R2); i < j2; ++i) tc::mbar_wait(x2_full(i % C::R2), uint32_t(i / C::R2) & 1u, &no_abort, P.err, kErrDrain);
            for (int i = max(0, j1 - C::R1); ok && i < j1; ++i) ok = wait(x1_empty(i % C::R1), uint32_t(i / C::R1) & 1u);
            for (int i = max(0, j2 - C::R2); ok && i < j2; ++i) ok = wait(x2_empty(i % C::R2), uint32_t(i / C::R2) & 1u);
        }
    } else if (warp == C::MMA_WARP) {
        statistics_are_there();
        if (tc::elect_one() && n > 0) {
            constexpr uint32_t idesc_s = tc::idesc_bf16_f32(kRows, BX, false), idesc_sum = tc::idesc_bf16_f32(kRows, D, true);
            const uint64_t f1 = tc::sw128_desc(sbase, 16, 1024), f2 = tc::sw128_desc(sbase + C::OFF_F2, 16, 1024);
            const uint64_t x1 = tc::sw128_desc(sbase + C::OFF_X1, 16, 1024), x2 = tc::sw128_desc(sbase + C::OFF_X2, 16, 1024);
            const uint64_t x1_mn = tc::sw128_desc(sbase + C::OFF_X1, BX * 128, 1024), x2_mn = tc::sw128_desc(sbase + C::OFF_X2, BX * 128, 1024);
            const uint64_t ones = plain_desc(sbase + C::OFF_ONES, 128, 256), augs = plain_desc(sbase + C::OFF_AUG, 128, 256);
            auto wait = [&](uint32_t bar, uint32_t phase) {
                const bool is = tc::mbar_wait(bar, phase & 1u, &s_abort, P.err, kErrMma);
                tc::tc_fence_after();
                return is;
            };
            // F X^T into a slot (descriptor units of 16 bytes), F by descriptor or in
            // TMEM; by keys with the rows' numbers, from the half `core` of them
            auto first_product = [&](auto in_tmem, uint32_t to, uint64_t f, uint32_t f_tmem, uint64_t x, int aug, int core) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint64_t b = x + uint64_t((kk / 4) * (BX * 8) + (kk % 4) * 2);
                    if constexpr (decltype(in_tmem)::value)
                        mma_f16_ts(to, f_tmem + kk * 8, b, idesc_s, kk > 0 ? 1u : 0u);
                    else
                        tc::mma_f16_ss(to, f + uint64_t((kk / 4) * (kRows * 8) + (kk % 4) * 2), b, idesc_s, kk > 0 ? 1u : 0u);
                }
                if constexpr (C::BY_KEYS) tc::mma_f16_ss(to, ones + uint64_t(core * 8), augs + uint64_t(aug) * (C::AUG_BYTES >> 4), idesc_s, 1u);
            };
            // bf16 in columns of their own, or 16 at the start of each 32 of a slot,
            // times X, added up
            auto second_product = [&](auto own, uint32_t sum, uint32_t slot, uint64_t x, bool add) {
#pragma unroll
                for (int kk = 0; kk < BX / 16; ++kk)
                    mma_f16_ts(sum, slot + (decltype(own)::value ? kk * 8 : (kk / 2) * 32 + (kk % 2) * 8), x + uint64_t(kk * 128), idesc_sum,
                               add || kk > 0 ? 1u : 0u);
            };
            constexpr uint32_t XSTEP = C::X_BYTES >> 4;
            // the stages of each product's operand, in the order of its blocks
            Ring<C::R1> s_ring, ss_ring, aug_ring;
            Ring<C::R2> dp_ring, sp_ring;
            auto make_s = [&](int j) {
                const int s = s_ring.s;
                if (!wait(x1_full(s), s_ring.phase)) return false;
                uint32_t phase, bar = C::OUT_P && !C::P_OWN ? p_done(j - NS, phase) : (phase = j - 1, s_read);
                if (j >= (C::OUT_P && !C::P_OWN ? NS : 1) && !wait(bar, phase)) return false;
                first_product(std::bool_constant<C::T1>(), tmem + uint32_t(j % NS) * BX, f1, tmem + C::COL_F1, x1 + uint64_t(s) * XSTEP, s, 0);
                tc::mma_commit(s_done(j, phase));
                s_ring.next();
                return true;
            };
            auto make_dp = [&](int j) {
                const int s = dp_ring.s;
                if (!wait(x2_full(s), dp_ring.phase)) return false;
                uint32_t phase, bar = C::DS_OWN ? (phase = j - 1, dp_read) : ds_done(j - 1, phase);
                if (j > 0 && !wait(bar, phase)) return false;
                first_product(std::bool_constant<C::T2>(), tmem + C::COL_DP, f2, tmem + C::COL_F2, x2 + uint64_t(s) * XSTEP, aug_ring.s, 1);
                tc::mma_commit(dp_done(j, phase));
                dp_ring.next();
                aug_ring.next();
                return true;
            };
            auto sum_p = [&](int j) {
                const int s = sp_ring.s;
                if (!wait(p_ready(j % NS), j / NS)) return false;
                if (C::OUT_P && !C::OUT_S && !wait(x2_full(s), sp_ring.phase)) return false;     // (else dP has waited)
                second_product(std::bool_constant<C::P_OWN>(), tmem + C::COL_SUM, tmem + (C::P_OWN ? C::COL_P : uint32_t(j % NS) * BX),
                               x2_mn + uint64_t(s) * XSTEP, j > 0);
                tc::mma_commit(x2_empty(s));
                sp_ring.next();
                return true;
            };
            auto sum_s = [&](int j) {
                const int s = ss_ring.s;
                if (!wait(ds_ready, j)) return false;
                second_product(std::bool_constant<C::DS_OWN>(), tmem + C::COL_S_SUM, tmem + (C::DS_OWN ? C::COL_DS : C::COL_DP),
                               x1_mn + uint64_t(s) * XSTEP, j > 0);
                tc::mma_commit(x1_empty(s));
                ss_ring.next();
                return true;
            };
            const bool any = ok = wait(f_full, 0);
            ok = ok && make_s(0);
            if constexpr (C::OUT_S) ok = ok && make_dp(0);
            for (int j = 0; ok && j < n; ++j) {
                const bool more = j + 1 < n;
                if constexpr (PASS == kKeys) {
                    ok = (!more || make_s(j + 1)) && sum_p(j) && (!more || make_dp(j + 1)) && sum_s(j);
                } else if constexpr (PASS == kValuesOnly) {
                    ok = (!more || make_s(j + 1)) && sum_p(j);
                } else if constexpr (C::DS_OWN) {
                    ok = (!more || (make_s(j + 1) && make_dp(j + 1))) && sum_s(j);
                } else {
                    ok = (!more || make_s(j + 1)) && sum_s(j) && (!more || make_dp(j + 1));
                }
            }
            if (ok) tc::mma_commit(sums);
            if (!ok && any) {
                // let the MMAs already issued finish before TMEM is freed
                tc::mma_commit(drain);
                volatile int no_abort = 0;
                tc::mbar_wait(drain, 0, &no_abort, P.err, kErrDrain);
            }
        }
    } else {
        const int wg = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + r;
        const uint32_t mine = tmem + (uint32_t((warp & 3) * 32) << 16);
        auto wait = [&](uint32_t bar, int phase) {
            const bool is = __all_sync(0xffffffffu, tc::mbar_wait(bar, uint32_t(phase) & 1u, &s_abort, P.err, kErrOut));
            tc::tc_fence_after();
            return is;
        };
        if constexpr (C::T1 || C::T2) {
            // the fixed operands' rows into TMEM, a part of the dims to a warpgroup
            const bool in = row < (C::BY_KEYS ? P.Tk : P.Tq);
            auto keep = [&](const Operand& o, uint32_t col) {
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(o.p) + batch * o.batch + head * o.head + row * o.row);
#pragma unroll
                for (int u = 0; u < D / 16 / C::WGS; ++u) {
                    const int at = wg * (D / 16 / C::WGS) + u;
                    const uint4 none = make_uint4(0, 0, 0, 0), a = in ? src[2 * at] : none, b = in ? src[2 * at + 1] : none;
                    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                    tmem_st8(mine + col + at * 8, w);
                }
            };
            if constexpr (C::T1) keep(P.f1, C::COL_F1);
            if constexpr (C::T2) keep(P.f2, C::COL_F2);
            tc::tmem_wait_st();
            tc::tc_fence_before();
            tc::mbar_arrive(f_full);
        }
        statistics_are_there();
        float row_lse = INFINITY, row_delta = 0.f;
        if constexpr (!C::BY_KEYS) {
            const long stat = (long(batch) * P.Hq + head) * P.Tpad + row;
            // (a row of one key: its weight is 1, whatever the scores are)
            row_lse = row + shift == 0 ? INFINITY : __ldcg(P.lse2 + stat);
            row_delta = __ldcg(P.delta + stat);
        }
        for (int j = 0; j < n; ++j) {
            const int at = (first + (j0 + j) % per) * BX + wg * 32;
            const uint32_t s_col = mine + uint32_t(j % NS) * BX + wg * 32, dp_col = mine + C::COL_DP + wg * 32;
            // columns that the row's key is seen from, or the row sees: from lo, to hi
            int lo = 0, hi = 32, single = -1;
            bool masked;
            if constexpr (C::BY_KEYS) {
                masked = shift + at < row0 + kRows - 1;
                lo = row - shift - at;
                single = -(shift + at);
            } else {
                masked = at + 32 > row0 + shift + 1;
                hi = row + shift + 1 - at;
            }
            uint32_t phase, bar = s_done(j, phase);
            ok = wait(bar, phase);
            if (!ok) break;
            float p[32];
            uint32_t w[16];
            tmem_ld32_done(s_col, p);
            if constexpr (!C::OUT_P || C::P_OWN) {
                tc::tc_fence_before();
                tc::mbar_arrive(s_read);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) p[i] = ex2(C::BY_KEYS ? p[i] * P.scale_log2 : fmaf(p[i], P.scale_log2, -row_lse));
            if (masked) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < lo || i >= hi) p[i] = 0.f;
            }
            if constexpr (C::OUT_P) {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
                if constexpr (C::P_OWN) {
                    bar = p_done(j - 1, phase);
                    ok = j == 0 || wait(bar, phase);
                    if (!ok) break;
                }
                tmem_st16(C::P_OWN ? mine + C::COL_P + wg * 16 : s_col, w);
                tc::tmem_wait_st();
                tc::tc_fence_before();
                tc::mbar_arrive(p_ready(j % NS));
            }
            if constexpr (C::OUT_S) {
                bar = dp_done(j, phase);
                ok = wait(bar, phase);
                if (!ok) break;
                float d[32];
                tmem_ld32_done(dp_col, d);
                if constexpr (C::DS_OWN) {
                    tc::tc_fence_before();
                    tc::mbar_arrive(dp_read);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) d[i] = p[i] * (C::BY_KEYS ? d[i] : d[i] - row_delta);
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (p[i] == 0.f || i == single) d[i] = 0.f;
                }
                if constexpr (FEW && C::BY_KEYS) {
                    // (the first warp's keys are all that there are; a column's sum
                    // to the lane of its number)
                    if ((warp & 3) == 0) {
                        float t[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) t[i] = (lane & 16 ? d[i + 16] : d[i]) + __shfl_xor_sync(0xffffffffu, lane & 16 ? d[i] : d[i + 16], 16);
#pragma unroll
                        for (int half = 8; half > 0; half /= 2)
#pragma unroll
                            for (int i = 0; i < half; ++i)
                                t[i] = (lane & half ? t[i + half] : t[i]) + __shfl_xor_sync(0xffffffffu, lane & half ? t[i] : t[i + half], half);
#pragma unroll
                        for (int i = 0; i < 32; ++i) d[i] = fmaf(-p[i], __shfl_sync(0xffffffffu, t[0], i), d[i]);
                    }
                } else if constexpr (FEW) {
                    float sum = 0.f;        // (all keys are the first warpgroup's)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum += d[i];
#pragma unroll
                    for (int i = 0; i < 32; ++i) d[i] = fmaf(-p[i], sum, d[i]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16(d[2 * i], d[2 * i + 1]);
                if constexpr (C::DS_OWN) {
                    bar = ds_done(j - 1, phase);
                    ok = j == 0 || wait(bar, phase);
                    if (!ok) break;
                }
                tmem_st16(C::DS_OWN ? mine + C::COL_DS + wg * 16 : dp_col, w);
                tc::tmem_wait_st();
                tc::tc_fence_before();
                tc::mbar_arrive(ds_ready);
            }
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(sums, 0, &s_abort, P.err, kErrOut));
        tc::tc_fence_after();
    }
    __syncwarp();
    // Sums out, 16 columns at a time.  With shares, the columns go round them:
    // each adds up its part of everyone's in share order.  No CTA of the
    // cluster has a copy or an MMA in flight any more then, so the operands'
    // room is their inbox: [from share][part][16][128] fp32.
    const int wg = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + r;
    const uint32_t mine = tmem + (uint32_t((warp & 3) * 32) << 16) + C::COL_SUM + wg * C::COLS;
    const int parts = (C::WGS * C::UNITS + P.shares - 1) / P.shares, u0 = wg * C::UNITS;
    constexpr int UNIT = 16 * kRows;
    float* inbox = reinterpret_cast<float*>(smem);
    const bool takes = warp < C::LOAD_WARP && ok;
    if (P.shares > 1) {
        cluster.sync();
        if (takes) {
#pragma unroll
            for (int u = 0; u < C::UNITS; ++u) {
                float o[16];
                tmem_ld16_done(mine + u * 16, o);
                float* box = cluster.map_shared_rank(inbox, (u0 + u) % P.shares) + size_t(share * parts + (u0 + u) / P.shares) * UNIT + r;
#pragma unroll
                for (int e = 0; e < 16; ++e) box[e * kRows] = n > 0 ? o[e] : 0.f;
            }
        }
        cluster.sync();
    }
    if (takes) {
        // (a warpgroup's columns are of one sum)
        const int c0 = wg * C::COLS;
        const bool of_p = C::OUT_P && c0 < D;
        __nv_bfloat16* out = of_p ? P.p_sum + batch * P.p_batch + head * P.p_head + row * P.p_row + c0
                                  : P.s_sum + batch * P.s_batch + head * P.s_head + row * P.s_row + (C::OUT_P ? c0 - D : c0);
        const float by = of_p ? 1.f : P.scale;
        const bool in = row < (C::BY_KEYS ? P.Tk : P.Tq);
#pragma unroll
        for (int u = 0; u < C::UNITS; ++u) {
            if ((u0 + u) % P.shares != share) continue;
            float o[16];
            if (P.shares > 1) {
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0.f;
                for (int from = 0; from < P.shares; ++from) {
                    const float* box = inbox + size_t(from * parts + (u0 + u) / P.shares) * UNIT + r;
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] += box[e * kRows];
                }
            } else {
                tmem_ld16_done(mine + u * 16, o);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = n > 0 || P.shares > 1 ? o[e] * by : 0.f;
            if (in) {
                uint4* dst = reinterpret_cast<uint4*>(out + u * 16);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    dst[i] = make_uint4(pack_bf16(o[8 * i], o[8 * i + 1]), pack_bf16(o[8 * i + 2], o[8 * i + 3]),
                                        pack_bf16(o[8 * i + 4], o[8 * i + 5]), pack_bf16(o[8 * i + 6], o[8 * i + 7]));
            }
        }
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == C::MMA_WARP) tc::tmem_dealloc(tmem, 512);
    // (what follows on the stream waits for this grid alone)
    if (!P.leads) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A number as three bf16 whose sum has all 24 bits of it (an infinity as the first).
__device__ __forceinline__ uint4 three_terms(float x) {
    const float a = __bfloat162float(__float2bfloat16_rn(x)), ra = isinf(a) ? 0.f : x - a;
    const float b = __bfloat162float(__float2bfloat16_rn(ra)), rb = ra - b;
    return make_uint4(pack_bf16(a, b), pack_bf16(rb, 0.f), 0, 0);
}

// The rows' statistics: log2 of the sum of weights, and delta; and as an MMA by
// keys takes them, per 8 rows [2][8 rows][8 bf16]: the terms of -lse2 / scale
// and of -delta.  A row without weights has a number there that makes its
// weights 0, but no infinity, which would meet zeros.  A warp takes 8 rows of a
// head, 16 bytes to a lane, all asked for at once; rows behind the last are rows
// without weights.
template <int D>
__global__ void __launch_bounds__(256)
    stats_kernel(const Operand dout, const Operand out, const float* lse, float* lse2, float* delta, uint8_t* aug, float scale_log2, int Tq, int Tpad,
                 int Hq, long units) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int LANES = D / 8, AT_ONCE = 32 / LANES, N = 8 / AT_ONCE;      // lanes to a row, rows of a load
    const int lane = threadIdx.x & 31, part = lane % LANES;
    const long unit = long(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (unit >= units) return;
    const int groups = Tpad / 8, row0 = int(unit % groups) * 8;
    const long at = unit / groups, batch = at / Hq, head = at % Hq;
    auto load = [&](const Operand& o, int row) {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(o.p) + batch * o.batch + head * o.head + row * o.row;
        return row < Tq ? reinterpret_cast<const uint4*>(p)[part] : make_uint4(0, 0, 0, 0);
    };
    uint4 a[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = row0 + i * AT_ONCE + lane / LANES;
        a[i] = load(dout, row);
        b[i] = load(out, row);
    }
    float mine = 0.f;           // delta of row row0 + lane % 8
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float sum = 0.f;
        const __nv_bfloat162 *x = reinterpret_cast<const __nv_bfloat162*>(&a[i]), *y = reinterpret_cast<const __nv_bfloat162*>(&b[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 u = __bfloat1622float2(x[e]), v = __bfloat1622float2(y[e]);
            sum = fmaf(u.x, v.x, fmaf(u.y, v.y, sum));
        }
#pragma unroll
        for (int off = LANES / 2; off > 0; off /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        const int r = lane % 8;
        const float from = __shfl_sync(0xffffffffu, sum, r % AT_ONCE * LANES);
        if (r / AT_ONCE == i) mine = from;
    }
    if (lane >= 16) return;
    const int row = row0 + lane % 8;
    const float l = row < Tq ? lse[at * Tq + row] : -INFINITY, l2 = l * 1.4426950408889634f;
    const bool none = l == -INFINITY;
    uint4* terms = reinterpret_cast<uint4*>(aug + (at * Tpad + row0) * 32);
    if (lane < 8) {
        lse2[at * Tpad + row] = none ? INFINITY : l2;
        delta[at * Tpad + row] = mine;
        terms[lane] = three_terms(none ? (scale_log2 > 0.f ? -1e30f : 1e30f) : -l2 / scale_log2);
    } else {
        terms[lane] = three_terms(-mine);
    }
}

// What one pass has to do: items, the blocks of the longest and of all.
struct Work {
    long items, longest, total;
};

// CTAs that share an item's blocks (host arithmetic only), for the least time in
// blocks: the longest share, or everything shared out evenly, and once more a CTA's
// own time (operands in, sums out, with shares traded: 8 blocks' and 15) where an
// SM gets a second.  32 / 8 heads of 128 by keys, alone, in twos and fours: 1024
// positions 73, 50, 60 us; 1500 107, 78, 98; 2048 146, 119, 142; 3000 234, 219,
// 263; 4096 340, 361, 417 (of both passes).
int shares_of(const Work& w, int sms) {
    int best = 1;
    double least = 0;
    for (int s = 1; s <= kMaxShares && (s == 1 || w.longest >= 2L * s); s *= 2) {
        const double own = s > 1 ? 15 : 8, ctas = double(w.items) * s, longest = double(w.longest) / s + own;
        const double time = ctas <= sms ? longest : std::max(longest, (double(w.total) + ctas * own) / sms) + own;
        if (s == 1 || time < least) {
            least = time;
            best = s;
        }
    }
    return best;
}

template <int D, int PASS, bool FEW>
int launch(const CUtensorMap (&maps)[4], GradParams p, const Work& w, bool leads, cudaStream_t st) {
    using C = Cfg<D, PASS>;
    static splice::PerDevice<int> kept;
    int sms = 0;
    const cudaError_t e = kept.get(&sms, [](int dev, int* n) {
        cudaError_t err = cudaFuncSetAttribute(grad_kernel<D, PASS, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(C::smem(kMaxShares)));
        if (err == cudaSuccess) err = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
        return err;
    });
    if (e != cudaSuccess) return int(e);
    p.shares = shares_of(w, sms);
    p.leads = leads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(w.items * p.shares));
    cfg.blockDim = dim3(C::THREADS);
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
    return int(cudaLaunchKernelEx(&cfg, grad_kernel<D, PASS, FEW>, maps[0], maps[1], maps[2], maps[3], p));
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
    constexpr int BX = Cfg<D, kQueries>::BX, BXK = Cfg<D, D == 256 ? kKeysOnly : kKeys>::BX;      // (of keys, of queries)
    const int Tpad = padded(a.Tq), shift = a.Tk - a.Tq, G = a.Hq / a.Hkv;
    const long rows = long(a.B) * a.Hq * Tpad;
    float *lse2 = a.stats, *delta = a.stats + rows;
    uint8_t* aug = reinterpret_cast<uint8_t*>(a.stats + 2 * rows);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const float by_keys_scale = std::fabs(scale_log2) >= kLeastScale ? scale_log2 : scale_log2 < 0.f ? -kLeastScale : kLeastScale;
    {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned((rows / 8 + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        const int e = int(cudaLaunchKernelEx(&cfg, stats_kernel<D>, a.dout, a.out, a.lse, lse2, delta, aug, by_keys_scale, a.Tq, Tpad, a.Hq, rows / 8));
        if (e != 0) return e;
    }
    // (a map of 128 rows serves as the fixed operand's and as the blocks')
    CUtensorMap fixed_k, fixed_v, fixed_q, fixed_o, block_k, block_v, block_q, block_o;
    auto maps = [&](CUtensorMap* fixed, CUtensorMap* block, const Operand& o, int T, int H, int rows) {
        if (!decoder::operand_map(fixed, o, D, T, H, a.B, kRows)) return false;
        *block = *fixed;
        return rows == kRows || decoder::operand_map(block, o, D, T, H, a.B, rows);
    };
    if (!maps(&fixed_k, &block_k, a.k, a.Tk, a.Hkv, BX) || !maps(&fixed_v, &block_v, a.v, a.Tk, a.Hkv, BX) ||
        !maps(&fixed_q, &block_q, a.q, a.Tq, a.Hq, BXK) || !maps(&fixed_o, &block_o, a.dout, a.Tq, a.Hq, BXK))
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
    p.scale_log2 = by_keys_scale;
    p.aug = aug;
    p.f1 = a.k;
    p.f2 = a.v;
    p.err = decoder::error_word();
    if (!p.err) return int(cudaErrorInvalidValue);
    // by keys
    p.p_sum = a.dv;
    p.s_sum = a.dk;
    p.p_row = p.s_row = D;
    p.p_head = p.s_head = long(a.Tk) * D;
    p.p_batch = p.s_batch = long(a.Hkv) * a.Tk * D;
    p.tiles = (a.Tk + kRows - 1) / kRows;
    const int blocks = (a.Tq + BXK - 1) / BXK;
    Work keys{long(p.tiles) * a.Hkv * a.B, 0, 0}, queries{long(Tpad / kRows) * a.Hq * a.B, 0, 0};
    for (int t = 0; t < p.tiles; ++t) {
        const long n = long(G) * std::max(0, blocks - std::max(0, t * kRows - shift) / BXK);
        keys.longest = std::max(keys.longest, n);
        keys.total += n * a.Hkv * a.B;
    }
    for (int t = 0; t < Tpad / kRows; ++t) {
        const long n = std::max(0, (std::min(a.Tk, (t + 1) * kRows + shift) + BX - 1) / BX);
        queries.longest = std::max(queries.longest, n);
        queries.total += n * a.Hq * a.B;
    }
    // The pass of the longer items leads: the other's fill the SMs that it leaves.
    // (Blocks by keys of 128 dims are half as long.)
    const bool keys_lead = keys.longest * BXK >= queries.longest * BX;
    const CUtensorMap by_keys[4] = {fixed_k, fixed_v, block_q, block_o};
    GradParams r = p;           // by queries
    r.scale_log2 = scale_log2;
    r.f1 = a.q;
    r.f2 = a.dout;
    r.s_sum = a.dq;
    r.s_row = long(a.Hq) * D;
    r.s_head = D;
    r.s_batch = long(a.Tq) * a.Hq * D;
    r.tiles = Tpad / kRows;
    const CUtensorMap by_queries[4] = {fixed_q, fixed_o, block_k, block_v};
    auto passes = [&](auto few) {
        constexpr bool FEW = decltype(few)::value;
        int e = 0;
        if (!keys_lead) e = launch<D, kQueries, FEW>(by_queries, r, queries, true, st);
        if constexpr (D == 256) {
            if (e == 0) e = launch<D, kValuesOnly, false>(by_keys, p, keys, keys_lead, st);
            if (e == 0) e = launch<D, kKeysOnly, FEW>(by_keys, p, keys, false, st);
        } else {
            if (e == 0) e = launch<D, kKeys, FEW>(by_keys, p, keys, keys_lead, st);
        }
        if (keys_lead && e == 0) e = launch<D, kQueries, FEW>(by_queries, r, queries, false, st);
        return e;
    };
    return a.Tk <= kFew ? passes(std::true_type()) : passes(std::false_type());
}

}  // namespace

extern "C" {

// Bytes of scratch that decoder_attention_backward needs.
long decoder_attention_scratch(long B, long Tq, int Hq) { return 40 * B * Hq * ((Tq + kRows - 1) / kRows * kRows); }

// Gradients of decoder_attention: dout, q, out [B][Tq][Hq][d] and k, v
// [B][Hkv][Tk][d] of any strides that are multiples of 8 elements (row, head,
// batch of each in this order; NULL: contiguous), lse as that gives it; dq
// [B][Tq][Hq][d], dk, dv [B][Hkv][Tk][d] contiguous; all bf16 and 16-byte
// aligned.  Returns a cudaError_t.
int decoder_attention_backward(const void* dout, const void* q, const void* out, const void* k, const void* v, const void* lse,
                               const long* strides, void* scratch, void* dq, void* dk, void* dv, long B, long Tq, long Tk, int Hq,
                               int Hkv, int d, float scale, void* stream) {
    if (!decoder::attention_takes(B, Tq, Tk, Hq, Hkv)) return int(cudaErrorInvalidValue);
    const long of_q[3] = {long(Hq) * d, d, Tq * Hq * d}, of_k[3] = {d, Tk * d, Tk * Hkv * d};
    auto operand = [&](const void* p, int i) {
        const long* s = strides ? strides + 3 * i : i < 3 ? of_q : of_k;
        return Operand{p, s[0], s[1], s[2]};
    };
    const Args a{operand(dout, 0), operand(q, 1), operand(k, 3), operand(v, 4), operand(out, 2), static_cast<const float*>(lse),
                 static_cast<float*>(scratch), static_cast<__nv_bfloat16*>(dq), static_cast<__nv_bfloat16*>(dk),
                 static_cast<__nv_bfloat16*>(dv), int(B), int(Tq), int(Tk), Hq, Hkv, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d == 64) return backward<64>(a, st);
    if (d == 128) return backward<128>(a, st);
    if (d == 256) return backward<256>(a, st);
    return int(cudaErrorInvalidValue);
}

}  // extern "C"
