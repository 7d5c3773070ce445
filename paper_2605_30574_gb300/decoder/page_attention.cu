// Attention of each sequence's newest tokens over its pages of a cache in 4 bits.
//
//   out_i = sum_j p_ij v_j,  p_ij = softmax over j of scale q_i . k_j,
//   j <= pos_i = length - new + i,  j > pos_i - window
//
// A step reads every key and value once for the G = Hq / Hkv query rows of a kv head
// (times its new tokens): 138 bytes to 512 G flops at 128 dims, so HBM is the bound,
// and what a kernel may spend on making operands of 4-bit codes is about three
// instructions of a lane to an element.  Products therefore take the codes as they
// are: a nibble n = c + 8, masked in place, is the fp16 number n 2^-24 (bits 0 to 3) or
// 16 n 2^-24 (bits 4 to 7).  In order of what each measured, at 512 sequences of 4224
// tokens, 32 / 8 heads of 128 (2.4 GB; 355 us at the copy rate, now 379):
//
//  * Scores: S[key][row], keys on the 16-row side of m16n8k16, eight rows on the other
//    (or twice eight).  q is scaled to 2^14 by a power of two and rounded to fp16 (all
//    of bf16's bits down to 2^-28 of the row's largest), with 1/16 where the code comes
//    16-fold.  Groups of 32 are added up in fp32 by their ratios, from -8 sum q r, which
//    takes the 8 out of c + 8 and is one product more, of the ratios and sum q in three
//    fp16 terms.
//  * Output: O[dim][row].  P as the fp16 operand has V's scales in it, so it is taken
//    relative to the largest of (score + E of the value's row), and not of the score:
//    then no product of a weight and a scale is above 2^15, and one that is rounded or
//    lost below fp16's normal range is 2^-29 of the largest.  That reference is two
//    numbers, a score and the rest: in one, E would be lost in scores from 2^24 on (1.3%
//    faster with 8 new tokens, 4% with 16, as fast with one).  Codes have their 8
//    subtracted (exactly): O would otherwise carry it through sums of thousands of keys.
//    Subtracting the weights' sums by the tensor core instead, 417 us for 398.  The
//    second nibble of a byte is taken off the first's sum, not masked out of it: 376 for
//    386.
//  * The transposition from S's layout to an operand is movmatrix; a key's four lanes and
//    a row's eight are those of both.
//  * Up to four rows to a kv head: two heads to a product, four columns each, with zeros
//    for the other's in q and in P, so that the softmax is done once for both: 417 for
//    482 (306 -> 261 instructions for 16 keys of a head).  More than eight rows: sixteen
//    columns, as the codes are made operands once: 64 rows 52 us for 56, 18 rows 57 for 59.
//  * Keys come through a ring in shared memory, 16 bytes by cp.async to a lane; bulk copies
//    took 25 instructions each, one after another, 681 us against 623.  A stage is 32
//    keys, or 16 of two heads: 482 against 562 with 16.
//  * What is not needed in the loop over the keys is in shared memory (Walk): at 168
//    registers the loop then spills and recomputes nothing (286 -> 276 instructions); 16
//    warps of 128 registers, 415 us for 388.
//
// What bounds it now is HBM, 94% of its copy rate, and close behind it issue: 65% of all
// slots, the ALU 60% (profile).
//
// Work: all (sequence, kv head, tile of rows, stage of keys) in one line, an even share to
// each warp, whatever the sequences' lengths, which only the device knows.  (Short tiles:
// an even share of the tiles, not cut, to each CTA; see launch.)  A tile whose
// keys fall to several warps leaves a state (m, l, O) per warp; a CTA joins its warps', and
// a second kernel the CTAs', in their order: the same inputs give the same bits.  131072
// tokens of one sequence: 36 us, 12 of which are set-up, joins and the SMs' uneven speed
// (their last warps end 8 us apart); all in the second kernel it was 109.
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "../csrc/per_device.h"
#include "../csrc/tc_ptx.cuh"
#include "decoder.h"
#include "pages.cuh"

namespace decoder {
namespace {

using splice::tc::smem_u32;

constexpr unsigned kFull = 0xffffffffu;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -3e38f;         // the reference of rows that have seen nothing
constexpr int kMinWarps = 4;            // warps to a CTA that are given keys, at least
// Tiles are apart where they have so many stages to a warp at most, and so many more to
// the one that has most than on the line (see launch).
constexpr int kMost = 16, kMore = 3;

struct Args {
    PageLayer c;
    PageRows s;
    const __nv_bfloat16* q;
    long q_token, q_head;
    __nv_bfloat16* out;
    int G, window;
    int apart;              // warps to a tile, each tile's to one CTA; 0: all on one line
    float scale;
    float *states, *joined; // of warps [each][columns][d + 4], and of CTAs [each][2][columns][d + 4]
    int4* begun;            // per CTA: the tile whose keys begin with it and go on
};

// A warp's products have 8 NT columns: rows of one kv head, or of P heads next to each
// other, 8 / P of each.
template <int D_, int NT_, int P_>
struct Shape {
    static constexpr int D = D_, NT = NT_, P = P_, kI = D / 32;
    static constexpr int kCols = 8 * NT, kRows = kCols / P;         // (rows of a head, to a tile)
    static constexpr int kKeys = 32 / P;                            // keys to a stage: two runs of 16, or of two heads
    // stages that a tile's begin and end take as long as (200 sequences of 1 to 9000 tokens: 50
    // us; with 2 for 4 57, with 7 52)
    static constexpr int kBegin = D == 256 ? 2 : 2 * P;
    static constexpr int kLeast = 32 / kKeys;                       // stages to a warp, at least
    // warps to an SM, all of one CTA: as many as their registers allow
    static constexpr int kWarps = D == 256 ? 8 : D == 128 ? (NT == 2 ? 8 : 12) : NT == 2 ? 12 : 16;
    static constexpr int kThreads = 32 * kWarps;
    // a stage of a warp's ring: where its parts are
    static constexpr int kStages = D == 256 ? 2 : D == 128 ? 3 : 4;
    static constexpr int kV = 16 * D, kKr = 32 * D, kVr = kKr + 32 * kI, kE = kKr + 64 * kI, kBytes = kE + 64;
    static constexpr int kRest = 4 * kI + 4;                        // copies of 16 bytes that bring ratios and exponents
    static constexpr int kQ = P * NT * kI * 512;                    // q as operands
    static constexpr int kWarpBytes = kStages * kBytes + kQ, kSmem = kWarps * kWarpBytes;
    static_assert(kSmem <= 224 * 1024 && kStages * kBytes >= kCols * (D + 4) * 4);
};
constexpr int kJoin = 128;              // threads of a CTA that joins states

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// x 2^d, d at most 0.  A sum of weights is taken so: its reference goes by the values' sizes
// too, and may rise by 200 bits where it does not become nothing (keys of zeros next to one
// of large values).
__device__ __forceinline__ float lowered(float x, float d) { return x * ex2(fmaxf(d, -100.f)) * ex2(fminf(d + 100.f, 0.f)); }

__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma0(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Bytes of a and b (numbers 4 to 7) by the selector's digits; with 8 in a digit, the
// byte's sign.
__device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t select) {
    uint32_t y;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(y) : "r"(a), "r"(b), "r"(select));
    return y;
}

__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const uint32_t&>(h);
}

__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
    const __half2 h = __hadd2(reinterpret_cast<const __half2&>(a), reinterpret_cast<const __half2&>(b));
    return reinterpret_cast<const uint32_t&>(h);
}

__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    const __half2 h = __hmul2(reinterpret_cast<const __half2&>(a), reinterpret_cast<const __half2&>(b));
    return reinterpret_cast<const uint32_t&>(h);
}

// `N` bytes of shared memory at their own alignment, as words.
template <int N>
__device__ __forceinline__ void lds(uint32_t* x, uint32_t from) {
    if constexpr (N == 2) {
        uint16_t y;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(from));
        x[0] = y;
    }
    if constexpr (N == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x[0]) : "r"(from));
    if constexpr (N == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(from));
    if constexpr (N >= 16)
#pragma unroll
        for (int i = 0; i < N / 16; ++i)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[4 * i]), "=r"(x[4 * i + 1]), "=r"(x[4 * i + 2]), "=r"(x[4 * i + 3])
                         : "r"(from + 16 * i));
}

// a / b, of numbers that rarely need 64 bits.
__device__ __forceinline__ long quotient(long a, long b) {
    return (a | b) >> 32 ? a / b : long(uint32_t(a) / uint32_t(b));
}

// The sequences' shares of the line of work.  All of a sequence's tiles count as many
// stages of keys, and kBegin more (none where tiles are apart), as the one that sees most.
struct Seq {
    int first, new_, base, length, tiles, blocks;       // (its first row of q, its rows; the first one's position)
    bool broken;                                        // (it is longer than its pages are)
};

template <class S, bool kApart>
__device__ __forceinline__ Seq sequence(const Args& A, int b) {
    Seq q;
    const int from = A.s.starts[b], to = A.s.starts[b + 1], length = A.s.lengths[b];
    const long room = long(A.s.width) << A.c.log_page;
    q.first = max(0, min(from, A.s.rows));
    q.new_ = max(0, min(to, A.s.rows) - q.first);
    q.broken = length > room;
    q.length = int(min(long(max(0, length)), room));    // (no more keys than there are places, whatever it says)
    q.base = q.length - (to - from) + (q.first - from);
    q.tiles = int((long(q.new_) * A.G + S::kRows - 1) / S::kRows);
    int blocks = q.length / S::kKeys + (q.length % S::kKeys != 0);
    if (A.window) blocks = min(blocks, int((long(A.window) + (S::kRows + A.G - 2) / A.G + 2 * S::kKeys - 2) / S::kKeys));
    q.blocks = max(1, blocks) + (kApart ? 0 : S::kBegin);
    return q;
}

template <class S>
__device__ __forceinline__ long tiles_of(const Args& A, const Seq& q) { return long(q.tiles) * (A.c.hkv / S::P); }

template <class S>
__device__ __forceinline__ long size_of(const Args& A, const Seq& q) { return tiles_of<S>(A, q) * q.blocks; }

__device__ __forceinline__ void sts16(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void cp16(uint32_t to, const uint8_t* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// What a warp does with its share, in shared memory: between two tiles it is all that a
// warp knows, so that the loop over the keys has the registers.
template <class S>
struct Walk {
    long x, end, begin, at, item_at;            // on the line: where it is, its share, its sequence's begin, its tile's
    long origin, each, longer;                  // where the shares begin, their stages, and how many have one more
    int b, line, first, new_, base, head, tile, rows;
    int worker;                                 // of the first share
    int pos[S::kCols];                          // of the columns' rows
    int ids[64];                                // pages of the sequence, two times 32 places
};

// Rows' states joined, 8 lanes to a row: O for the reference m + size, at D and D + 2, and the
// sum l, at D + 1.
template <int D>
struct State {
    static constexpr int kVec = D / 32;         // by four elements
    float m = kNone, l = 0.f, size = 0.f;
    float4 o[kVec] = {};

    __device__ __forceinline__ void add(const float* from) {
        const int lane = threadIdx.x & 7;
        float4 y[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[i] = reinterpret_cast<const float4*>(from)[lane + 8 * i];
        const float4 it = *reinterpret_cast<const float4*>(from + D);
        const float above = (it.x - m) + (it.z - size), down = fminf(-above, 0.f), its = fminf(above, 0.f);
        const float f = ex2(down), fy = ex2(its);
        l = lowered(l, down) + lowered(it.y, its);
        if (above > 0.f) m = it.x, size = it.z;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            o[i] = make_float4(o[i].x * f + y[i].x * fy, o[i].y * f + y[i].y * fy, o[i].z * f + y[i].z * fy, o[i].w * f + y[i].w * fy);
    }
    __device__ __forceinline__ void keep(float* to) const {
        const int lane = threadIdx.x & 7;
#pragma unroll
        for (int i = 0; i < kVec; ++i) reinterpret_cast<float4*>(to)[lane + 8 * i] = o[i];
        if (lane == 0) *reinterpret_cast<float4*>(to + D) = make_float4(m, l, size, 0.f);
    }
    __device__ __forceinline__ void write(__nv_bfloat16* to) const {
        const int lane = threadIdx.x & 7;
        const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(o[i].x * f, o[i].y * f), b = __floats2bfloat162_rn(o[i].z * f, o[i].w * f);
            *reinterpret_cast<uint2*>(to + 4 * (lane + 8 * i)) = make_uint2(reinterpret_cast<const uint32_t&>(a), reinterpret_cast<const uint32_t&>(b));
        }
    }
};

// The row of out of a tile's row.
template <class S>
__device__ __forceinline__ size_t row_of(const Args& A, const int4& info, int mine, int row) {
    const int r = (info.y & 0xffffff) * S::kRows + row, token = r / A.G;
    return (size_t(info.x + token) * A.c.hkv + (info.z & 0x3fffffff) + mine) * A.G + r - token * A.G;
}

// (Two kernels: one for both takes 381 us for 375, and 7.0 for 6.7 of a short sequence.)
template <class S, bool kApart>
__global__ void __launch_bounds__(S::kThreads, 1) attention_kernel(const Args A) {
    constexpr int D = S::D, NT = S::NT, P = S::P, kI = S::kI, kThreads = S::kThreads, R = S::kRows;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long before[kThreads + 1];       // work before each run of sequences
    __shared__ long sums[kThreads / 32];
    __shared__ float* places[S::kWarps][2];     // states of tiles that go on here, and that go on behind this warp
    __shared__ Walk<S> walks[S::kWarps];
    __shared__ int4 runs[S::kWarps + 1];        // tiles that warps share: the one that goes on here, and each warp's that goes on
    wait_for_previous();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp_in = threadIdx.x / 32;
    const int run = (A.s.batch + kThreads - 1) / kThreads;
    {
        long mine = 0;
        for (int b = threadIdx.x * run; b < min(A.s.batch, int(threadIdx.x + 1) * run); ++b) {
            const Seq q = sequence<S, kApart>(A, b);
            mine += kApart ? tiles_of<S>(A, q) : size_of<S>(A, q);
        }
        long x = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long y = __shfl_up_sync(kFull, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp_in] = x;
        __syncthreads();
        for (int w = 0; w < warp_in; ++w) x += sums[w];
        before[threadIdx.x + 1] = x;
        if (threadIdx.x == 0) before[0] = 0;
        __syncthreads();
    }
    const long total = before[kThreads];
    // few keys: one CTA, or four warps and more of as many as there are shares for
    const long shares = max(1L, quotient(total, S::kLeast));
    const int active = kApart                ? S::kWarps
                       : shares <= S::kWarps ? int(shares)
                                             : int(max(long(kMinWarps), min(long(S::kWarps), quotient(shares + gridDim.x - 1, gridDim.x))));
    const int worker0 = active * blockIdx.x;
    Walk<S>& walk = walks[warp_in];
    if (lane == 0) {
        // who gets equal parts of all stages: a warp; or, apart, of all tiles: some of a CTA's
        const int slot = kApart ? warp_in / A.apart : 0;
        const long workers = kApart ? long(S::kWarps / A.apart) * gridDim.x : min(shares, long(active) * gridDim.x);
        long worker = kApart ? long(slot) * gridDim.x + blockIdx.x : worker0 + warp_in;
        walk.each = quotient(total, workers), walk.longer = total - walk.each * workers;
        walk.origin = walk.worker = 0;
        long from = walk.each * worker + min(worker, walk.longer), many = walk.each + (worker < walk.longer);
        if (worker >= workers || (!kApart && warp_in >= active)) from = many = 0;
        int lo = 0;                              // the run of sequences that it is in
        for (int step = 256; step; step /= 2)
            if (lo + step < kThreads && before[lo + step] <= from) lo += step;
        walk.at = before[lo];
        walk.b = min(lo * run, A.s.batch - 1);
        if (kApart) {
            // the tiles' stages, on a line that begins with their first one's sequence, and
            // the warp's part of them
            long skipped = from - walk.at, stages = 0;
            int b = walk.b;
            for (bool found = false; many && b < A.s.batch; ++b) {
                const Seq q = sequence<S, kApart>(A, b);
                const long n = tiles_of<S>(A, q), taken = min(many, max(0L, n - skipped));
                if (!found && taken) walk.b = b, walk.origin = skipped * q.blocks, found = true;
                skipped = max(0L, skipped - n);
                stages += taken * q.blocks;
                many -= taken;
            }
            walk.at = 0;
            walk.each = stages / A.apart, walk.longer = stages % A.apart;
            worker = warp_in - slot * A.apart;
            walk.worker = worker0 + slot * A.apart;
            from = walk.origin + walk.each * worker + min(worker, walk.longer), many = walk.each + (worker < walk.longer);
        }
        walk.x = walk.begin = from;
        walk.end = from + many;
        runs[1 + warp_in].x = -1;
        if (warp_in == 0) runs[0].x = -1;
        places[warp_in][0] = places[warp_in][1] = reinterpret_cast<float*>(smem + warp_in * S::kWarpBytes);
    }
    __syncthreads();

    // the warp's ring, and what a lane copies of a stage: 16 bytes of every 512 of the
    // codes, and of the rest its share: of K's ratios, V's, and the exponents, 2 kI, 2 kI
    // and 4 lanes' worth (past 32: a second time)
    const uint32_t ring = smem_u32(smem) + warp_in * S::kWarpBytes, ring_end = ring + S::kStages * S::kBytes;
    const uint32_t q_at = ring_end + 16 * lane;
    constexpr int kMore = S::kRest > 32 ? 2 : 1;
    auto rest_kind = [&](int m) { return lane + 32 * m < 2 * kI ? 0 : lane + 32 * m < 4 * kI ? 1 : 2; };
    auto rest_row = [&](int m) { return lane + 32 * m < 4 * kI ? kI : 2; };
    const int log_blocks = A.c.log_page - (P == 2 ? 4 : 5);     // (below 0: pages of 16, two to a stage)
    const int in_page = log_blocks > 0 ? (1 << log_blocks) - 1 : 0;
    const bool small = log_blocks < 0;
    // (kept in registers: as constants they are made anew for every product)
    uint32_t centre[2];                          // -136 and -128, times 2^-24
#pragma unroll
    for (int i = 0; i < 2; ++i) asm volatile("mov.b32 %0, %1;" : "=r"(centre[i]) : "r"(i ? 0x80808080u : 0x80888088u));

    while (walk.x < walk.end) {
        const long x = walk.x;
        long at = walk.at;
        int b = walk.b;
        Seq sq = sequence<S, kApart>(A, b);
        while (at + size_of<S>(A, sq) <= x) {
            at += size_of<S>(A, sq);
            if (++b >= A.s.batch) break;         // (lengths that changed under the call)
            sq = sequence<S, kApart>(A, b);
        }
        if (b >= A.s.batch) break;
        const long rel = x - at;
        const int item = int(quotient(rel, sq.blocks)), j0 = int(rel - long(item) * sq.blocks);
        const int j1 = int(min(long(sq.blocks), j0 + (walk.end - x)));
        const int group = item / sq.tiles, head = group * P, tile = item - group * sq.tiles;
        const int rows = int(min(long(R), long(sq.new_) * A.G - long(tile) * R));
        const int base = sq.base, begin = kApart ? 0 : S::kBegin;
        const int first_pos = base + tile * R / A.G, last_pos = base + (tile * R + rows - 1) / A.G;
        // (positions and windows may be close to 2^31)
        const int kb0 = A.window && first_pos >= A.window ? (first_pos - A.window + 1) / S::kKeys : 0;
        const int kb_end = min(kb0 + j1 - begin, last_pos < 0 ? 0 : last_pos / S::kKeys + 1);
        int kb = kb0 + max(0, j0 - begin), kb_in = kb;
        __syncwarp();
        if (lane == 0) {
            walk.x = x + (j1 - j0), walk.at = at, walk.item_at = x - j0;
            walk.b = b, walk.line = sq.blocks, walk.first = sq.first, walk.new_ = sq.new_, walk.base = base;
            walk.head = head, walk.tile = tile, walk.rows = rows;
        }
        // ---- stages on their way: the numbers of 64 pages in the walk ----
        auto place = [&](int at) { return small ? 2 * at : at >> log_blocks; };
        auto look_up = [&](const int* table, int first) {
            const int i = first + lane;
            walk.ids[i & 63] = i < A.s.width ? __ldg(table + i) : -1;
        };
        {
            const int* table = A.s.table + size_t(b) * A.s.width;
            look_up(table, place(kb) & ~31);
            look_up(table, (place(kb) & ~31) + 32);
        }
        __syncwarp();
        // (q on its way meanwhile: columns are a head's rows, 8 / P or 8 NT of them)
        uint32_t raw[NT][kI][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int col = P == 2 ? g & 3 : 8 * n + g, r = tile * R + col, token = r / A.G;
            const __nv_bfloat16* p = A.q + (sq.first + (col < rows ? token : 0)) * A.q_token +
                                     ((head + (P == 2 ? g >> 2 : 0)) * A.G + (col < rows ? r - token * A.G : 0)) * A.q_head;
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const uint4 y = __ldg(reinterpret_cast<const uint4*>(p + 32 * i + 8 * t));
                raw[n][i][0] = y.x, raw[n][i][1] = y.y, raw[n][i][2] = y.z, raw[n][i][3] = y.w;
            }
        }
        const uint8_t *k_in, *late_in, *rest_in[kMore];         // (late: the stage's second half)
        bool broken = sq.broken;                 // (or with a page that is none of the cache's)
        auto locate = [&]() {
            const int i = place(kb_in);
            if ((i & 31) == 0) {
                __syncwarp();
                look_up(A.s.table + size_t(walk.b) * A.s.width, i + 32);
                __syncwarp();
            }
            auto checked = [&](int at) {
                const int page = walk.ids[at & 63];
                if (page >= 0 && page < A.c.pages) return uint32_t(page);
                broken = true;
                return 0u;
            };
            const uint32_t page = checked(i);
            uint32_t late = page;
            if (small) late = 32 * kb_in + 16 <= last_pos ? checked(i + 1) : page;
            const uint32_t page_rows = 1u << A.c.log_page, both = page_rows * A.c.hkv;      // (of keys or values, of a page)
            const uint32_t slot = S::kKeys * (kb_in & in_page), row = page_rows * walk.head;
            const uint8_t* codes = A.c.codes + 16 * lane;
            k_in = codes + uint64_t(page) * (both * D) + (row + slot) * (D / 2);
            late_in = P == 2 ? k_in + page_rows * (D / 2) : small ? codes + uint64_t(late) * (both * D) + row * (D / 2) : k_in + 8 * D;
#pragma unroll
            for (int m = 0; m < kMore; ++m) {
                const int kind = rest_kind(m), each_row = rest_row(m), j = lane + 32 * m - 2 * kI * kind;
                const bool second = j >= each_row;               // (of the stage's second half)
                rest_in[m] = (kind < 2 ? A.c.ratios + (kind ? both * kI : 0) : A.c.exponents) + 16 * j +
                             uint64_t(second ? late : page) * (both * (kind < 2 ? 2 * kI : 2)) +
                             int64_t(int(row + slot) + (second ? (P == 2 ? int(page_rows) - 16 : small ? -16 : 0) : 0)) * each_row;
            }
        };
        uint32_t in_at = ring, out_at = ring;
        auto fill = [&]() {
            if (kb_in < kb_end) {
                const uint32_t values = (uint32_t(A.c.hkv) << A.c.log_page) * (D / 2);
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    const uint8_t* from = (j < D / 64 ? k_in : late_in) + 512 * (j % (D / 64));
                    cp16(in_at + 16 * lane + 512 * j, from);
                    cp16(in_at + 16 * lane + S::kV + 512 * j, from + values);
                }
#pragma unroll
                for (int m = 0; m < kMore; ++m)
                    if (lane + 32 * m < S::kRest) cp16(in_at + S::kKr + 16 * (lane + 32 * m), rest_in[m]);
                in_at += S::kBytes;
                if (in_at == ring_end) in_at = ring;
                if ((++kb_in & in_page) == 0) {
                    if (kb_in < kb_end) locate();
                } else {
                    k_in += S::kKeys * (D / 2);
                    late_in += S::kKeys * (D / 2);
#pragma unroll
                    for (int m = 0; m < kMore; ++m) rest_in[m] += S::kKeys * rest_row(m);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        if (kb < kb_end) locate();
#pragma unroll 1
        for (int i = 0; i < S::kStages - 1; ++i) fill();

        // ---- the rows: q as an operand, and what is known of each column ----
        uint32_t minus[P][NT][kI > 4 ? 4 : 2];
        float factor[NT][2], l[NT][2], ref[NT][2], size[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int mine = P == 2 ? g >> 2 : 0;
            uint32_t top2 = 0;
#pragma unroll
            for (int i = 0; i < kI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) top2 = __vmaxu2(top2, raw[n][i][j] & 0x7fff7fffu);
            unsigned top = max(top2 & 0xffffu, top2 >> 16);
            top = max(top, __shfl_xor_sync(kFull, top, 1));
            top = max(top, __shfl_xor_sync(kFull, top, 2));
            const int E = max(int(top >> 7), 1);
            // (2^(141 - E) in two factors; a row with infinities or NaN: NaN)
            const float up = E == 255 ? __int_as_float(0x7fffffff) : power_of(255 - E);
            const float down = power_of(E);
            uint32_t hi[kI], mid[kI], low[kI];       // -8 sum q of a group, as three fp16
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                // elements 8t + j of group i, j = 0 .. 7; pairs (j, j + 4) to an operand
                float f[8], sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    f[j] = __uint_as_float(j & 1 ? raw[n][i][j / 2] & 0xffff0000u : raw[n][i][j / 2] << 16) * up * (j & 1 ? 0x1p9f : 0x1p13f);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    raw[n][i][j] = half2_of(f[j], f[j + 4]);
                    const float2 y = __half22float2(reinterpret_cast<const __half2&>(raw[n][i][j]));
                    sum = fmaf(y.x + y.y, j & 1 ? -128.f * 0x1p-24f : -8.f * 0x1p-24f, sum);
                }
                // (a head's operand has zeros for the other's columns; a lane reads its own)
#pragma unroll
                for (int ph = 0; ph < P; ++ph) {
                    const bool zero = P == 2 && ph != mine;
                    sts16(q_at + ((ph * NT + n) * kI + i) * 512, zero ? 0 : raw[n][i][0], zero ? 0 : raw[n][i][1], zero ? 0 : raw[n][i][2],
                          zero ? 0 : raw[n][i][3]);
                }
                sum += __shfl_xor_sync(kFull, sum, 1);
                sum += __shfl_xor_sync(kFull, sum, 2);
                const __half a = __float2half_rn(sum), c = __float2half_rn(sum - __half2float(a)),
                             e = __float2half_rn(sum - __half2float(a) - __half2float(c));
                hi[i] = __half_as_ushort(a), mid[i] = __half_as_ushort(c), low[i] = __half_as_ushort(e);
            }
            // as an operand against the keys' ratios (see below)
            auto two = [](const uint32_t* y, int i) { return y[i] | y[i + 1] << 16; };
            uint32_t m[kI > 4 ? 4 : 2];
            if constexpr (kI == 2) {
                m[0] = t == 0 ? two(hi, 0) : t == 1 ? two(mid, 0) : t == 2 ? two(low, 0) : 0u;
                m[1] = 0u;
            } else if constexpr (kI == 4) {
                m[0] = t == 0 ? two(hi, 0) : t == 1 ? two(hi, 2) : t == 2 ? two(mid, 0) : two(mid, 2);
                m[1] = t == 0 ? two(low, 0) : t == 1 ? two(low, 2) : 0u;
            } else {
                auto by_t = [&](const uint32_t* y) { return t == 0 ? two(y, 0) : t == 1 ? two(y, 2) : t == 2 ? two(y, 4) : two(y, 6); };
                m[0] = by_t(hi), m[1] = by_t(mid), m[2] = by_t(low), m[3] = 0u;
            }
#pragma unroll
            for (int ph = 0; ph < P; ++ph)
#pragma unroll
                for (int j = 0; j < (kI > 4 ? 4 : 2); ++j) minus[ph][n][j] = P == 2 && ph != mine ? 0u : m[j];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                // scale S 2^(E_k - 2) 2^24 / 2^(141 - E), in bits, but for 2^(E_k + 22) (see ek)
                factor[n][c] = __shfl_sync(kFull, down, 4 * (2 * t + c)) * A.scale * (0x1p-14f * kLog2e);
                const int column = P == 2 ? 2 * t + c & 3 : 8 * n + 2 * t + c;
                if (g == 0) walk.pos[8 * n + 2 * t + c] = column < rows ? base + (tile * R + column) / A.G : -1;
                l[n][c] = 0.f;
                ref[n][c] = kNone;
                size[n][c] = 0.f;
            }
        }
        __syncwarp();
        float acc[NT][kI][2][4] = {};
        // values 2t and 2t + 1 are read in turn and back, by t: half the bank conflicts
        const uint32_t even = t & 1 ? 0x1054u : 0x5410u, odd = t & 1 ? 0x3276u : 0x7632u;

        // ---- the keys ----
        const uint32_t k_of = 4 * kI * lane, v_of = S::kV + g * 2 * kI, v0_of = v_of + (2 * t + (t & 1)) * (D / 2),
                       v1_of = v_of + (2 * t + 1 - (t & 1)) * (D / 2), e_of = S::kE + 2 * g + (P == 2 ? 32 * (t >> 1) : 0);
        // 16 keys: the stage's half, or (P = 2) both heads'
        auto block = [&](auto at_edge, const int half) {
            constexpr bool kEdge = decltype(at_edge)::value;
            const int key0 = S::kKeys * kb + 16 * half;
            const uint32_t codes_at = out_at + half * 8 * D, ratios_at = out_at + half * 16 * kI;
            uint32_t kc[P][2][kI], ratio[P][2][kI / 2], ex[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int ph = 0; ph < P; ++ph) {
                    lds<4 * kI>(kc[ph][h], codes_at + ph * 8 * D + k_of + h * 8 * (D / 2));
                    uint32_t kr[(kI + 3) / 4];
                    lds<kI>(kr, ratios_at + ph * 16 * kI + S::kKr + g * kI + 8 * h * kI);
                    // two groups' ratios as fp16 (bytes of a word, with their signs, 0, between)
#pragma unroll
                    for (int i = 0; i < kI; i += 2) ratio[ph][h][i / 2] = bytes_of(kr[i / 4], 0, i % 4 ? 0xb3a2u : 0x9180u) << 7;
                }
                lds<2>(&ex[h], out_at + e_of + 32 * half + 16 * h);
            }
            // scores: first what the codes' 8 adds to all groups
            float s[NT][4];
#pragma unroll
            for (int ph = 0; ph < P; ++ph) {
                auto mine = [&](int h) {
                    const uint32_t* r = ratio[ph][h];
                    if constexpr (kI == 2) return r[0];
                    if constexpr (kI == 4) return t & 1 ? r[1] : r[0];
                    if constexpr (kI == 8) return t & 2 ? (t & 1 ? r[3] : r[2]) : t & 1 ? r[1] : r[0];
                };
                const uint32_t ra = mine(0), rc = mine(1);
                const uint32_t r4[4] = {ra, rc, ra, rc};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (ph == 0)
                        mma0(s[n], r4, minus[ph][n][0], minus[ph][n][1]);
                    else
                        mma(s[n], r4, minus[ph][n][0], minus[ph][n][1]);
                    if constexpr (kI > 4) mma(s[n], r4, minus[ph][n][2], minus[ph][n][3]);
                }
            }
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                float part[NT][4];
#pragma unroll
                for (int ph = 0; ph < P; ++ph) {
                    const uint32_t a = kc[ph][0][i], c = kc[ph][1][i];
                    const uint32_t lo4[4] = {a & 0x000f000fu, c & 0x000f000fu, a & 0x00f000f0u, c & 0x00f000f0u};
                    const uint32_t a8 = a >> 8, c8 = c >> 8;
                    const uint32_t hi4[4] = {a8 & 0x000f000fu, c8 & 0x000f000fu, a8 & 0x00f000f0u, c8 & 0x00f000f0u};
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t qf[4];
                        lds<16>(qf, q_at + ((ph * NT + n) * kI + i) * 512);
                        if (ph == 0)
                            mma0(part[n], lo4, qf[0], qf[1]);
                        else
                            mma(part[n], lo4, qf[0], qf[1]);
                        mma(part[n], hi4, qf[2], qf[3]);
                    }
                }
                // (by the ratios of the lane's columns' head)
                const uint32_t r0 = P == 2 && t >= 2 ? ratio[P - 1][0][i / 2] : ratio[0][0][i / 2],
                               r1 = P == 2 && t >= 2 ? ratio[P - 1][1][i / 2] : ratio[0][1][i / 2];
                const __half2 ra = reinterpret_cast<const __half2&>(r0), rc = reinterpret_cast<const __half2&>(r1);
                const float fa = i & 1 ? __high2float(ra) : __low2float(ra), fc = i & 1 ? __high2float(rc) : __low2float(rc);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s[n][0] = fmaf(part[n][0], fa, s[n][0]);
                    s[n][1] = fmaf(part[n][1], fa, s[n][1]);
                    s[n][2] = fmaf(part[n][2], fc, s[n][2]);
                    s[n][3] = fmaf(part[n][3], fc, s[n][3]);
                }
            }
            // weights, of keys g and g + 8
            float ek[2], up[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ek[h] = power_of(ex[h] & 255);
                up[h] = power_of(ex[h] >> 8);
                // (infinite, of a key or value of NaN: the score is NaN.  The 2^22 of the codes is
                // here, as the row's factor may be as large as scale q)
                ek[h] = fmaf(ek[h], 0x1p22f, __fmul_rn(__fadd_rn(ek[h], up[h]), 0.f));
                up[h] *= 0x1p6f;
            }
            uint32_t w[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[4], p[4], pv[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // (rounded before the reference is taken off, which was rounded so: of two
                    // scores in the millions the one that is the reference leaves 0.  In this
                    // order both products are numbers of fp32 where the score is: S is below
                    // 2^3, ek below 2^122, the factor below scale q.  With that of the factors
                    // taken first, which may be none, 512 sequences took 1% less, and 48 with 8
                    // new tokens 1.6% more)
                    s[n][j] = __fmul_rn(__fmul_rn(s[n][j], ek[j >> 1]), factor[n][j & 1]);
                    x[j] = __fsub_rn(__fsub_rn(s[n][j], ref[n][j & 1]), size[n][j & 1]);
                }
                if (kEdge) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + g + 8 * (j >> 1), last = walk.pos[8 * n + 2 * t + (j & 1)];
                        if (key > last || (A.window && key <= last - A.window)) x[j] = -INFINITY;
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[j] = ex2(x[j]);
                    pv[j] = p[j] * up[j >> 1];
                }
                if (kEdge) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (x[j] == -INFINITY) pv[j] = 0.f;          // (whatever the value is)
                }
                // what is past the reference is found by the weights: infinite, or too large
                if (__any_sync(kFull, fmaxf(fmaxf(pv[0], pv[1]), fmaxf(pv[2], pv[3])) > 0x1p14f)) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (kEdge && x[j] == -INFINITY) s[n][j] = -INFINITY;
                    const float e[2] = {float(int(ex[0] >> 8) - 127), float(int(ex[1] >> 8) - 127)};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = fmaxf(s[n][c], s[n][2 + c]);
#pragma unroll
                        for (int o = 4; o < 32; o *= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
                        m = fmaxf(ref[n][c], m);
                        // (what the largest of score + E, the old one's too, is above the largest score)
                        float down = (ref[n][c] - m) + size[n][c];
                        float rest = fmaxf(fmaxf((s[n][c] - m) + e[0], (s[n][2 + c] - m) + e[1]), down);
#pragma unroll
                        for (int o = 4; o < 32; o *= 2) rest = fmaxf(rest, __shfl_xor_sync(kFull, rest, o));
                        down -= rest;
                        ref[n][c] = m, size[n][c] = rest;
                        l[n][c] = lowered(l[n][c], down);
                        const float f = ex2(down);
#pragma unroll
                        for (int i = 0; i < kI; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) acc[n][i][h][c] *= f, acc[n][i][h][2 + c] *= f;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        p[j] = ex2(__fsub_rn(__fsub_rn(s[n][j], ref[n][j & 1]), size[n][j & 1]));
                        pv[j] = kEdge && x[j] == -INFINITY ? 0.f : p[j] * up[j >> 1];
                    }
                }
                // (a weight is up to 2^108, of values of 2^-100)
                l[n][0] = fmaf(p[0] + p[2], 0x1p-20f, l[n][0]);
                l[n][1] = fmaf(p[1] + p[3], 0x1p-20f, l[n][1]);
                w[n][0] = transposed(half2_of(pv[0], pv[1]));
                w[n][1] = transposed(half2_of(pv[2], pv[3]));
            }
            // output
#pragma unroll
            for (int ph = 0; ph < P; ++ph) {
                uint32_t v[4][(kI + 1) / 2], vr[2][(2 * kI + 3) / 4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    lds<2 * kI>(v[2 * h], codes_at + ph * 8 * D + v0_of + h * 8 * (D / 2));
                    lds<2 * kI>(v[2 * h + 1], codes_at + ph * 8 * D + v1_of + h * 8 * (D / 2));
                    lds<2 * kI>(vr[h], ratios_at + ph * 16 * kI + S::kVr + 2 * t * kI + 8 * h * kI);
                }
                if (kEdge) {
                    // what no row sees may hold anything: its ratios are left out
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + 2 * t + (j & 1) + 8 * (j >> 1);
                        if (key > last_pos || (A.window && key <= max(0, first_pos) - A.window)) {
                            if constexpr (kI == 2) vr[j >> 1][0] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
                            if constexpr (kI > 2)
#pragma unroll
                                for (int i = 0; i < kI / 4; ++i) vr[j >> 1][(j & 1) * (kI / 4) + i] = 0;
                        }
                    }
                }
                // (a head's products add to its own columns)
                uint32_t wh[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) wh[n][h] = P == 2 && (g >> 2) != ph ? 0u : w[n][h];
#pragma unroll
                for (int i = 0; i < kI; ++i) {
                    // bytes i of two keys' ratios, as fp16
                    constexpr int kNext = kI == 2 ? 2 : 4;               // (the second key's byte 0)
                    const uint32_t sel = (i & 3) | 8 << 4 | (kNext + (i & 3)) << 8 | 8 << 12;
                    const uint32_t r0 = bytes_of(vr[0][i / 4], vr[0][kI == 2 ? 0 : kI / 4 + i / 4], sel) << 7;
                    const uint32_t r1 = bytes_of(vr[1][i / 4], vr[1][kI == 2 ? 0 : kI / 4 + i / 4], sel) << 7;
                    const uint32_t a = bytes_of(v[0][i / 2], v[1][i / 2], i & 1 ? odd : even);
                    const uint32_t c = bytes_of(v[2][i / 2], v[3][i / 2], i & 1 ? odd : even);
                    // a byte is n + 16 n', its upper nibble 16 n': the first sum less the second
                    // is what n alone gives
                    const uint32_t a8 = bytes_of(a, 0, 0x4341), c8 = bytes_of(c, 0, 0x4341);
                    const uint32_t lo4[4] = {add2(a & 0x00ff00ffu, centre[0]), add2(a & 0x00f000f0u, centre[1]),
                                             add2(c & 0x00ff00ffu, centre[0]), add2(c & 0x00f000f0u, centre[1])};
                    const uint32_t hi4[4] = {add2(a8, centre[0]), add2(a8 & 0x00f000f0u, centre[1]), add2(c8, centre[0]),
                                             add2(c8 & 0x00f000f0u, centre[1])};
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint32_t b0 = mul2(wh[n][0], r0), b1 = mul2(wh[n][1], r1);
                        mma(acc[n][i][0], lo4, b0, b1);
                        mma(acc[n][i][1], hi4, b0, b1);
                    }
                }
            }
        };
        // (stages all of whose keys all rows see, and the others)
        const int inner = A.window && last_pos >= A.window ? (last_pos - A.window) / S::kKeys + 1 : 0, inner_end = (first_pos + 1) / S::kKeys;
        for (; kb < kb_end; ++kb) {
            // (the stage is there when all but the newest kStages - 2 are; all lanes have
            // read the one before, which is filled anew)
            asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 2) : "memory");
            __syncwarp();
            fill();
            if (kb >= inner && kb < inner_end) {
                block(std::false_type(), 0);
                if (P == 1) block(std::false_type(), 1);
            } else {
#pragma unroll 1
                for (int half = 0; half < 2 / P; ++half)
                    if (S::kKeys * kb + 16 * half <= last_pos) block(std::true_type(), half);
            }
            out_at += S::kBytes;
            if (out_at == ring_end) out_at = ring;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();

        // ---- the rows' states: out, or left for the join ----
        const long item_at = walk.item_at, item_end = item_at + walk.line;
        const bool whole = item_at >= walk.begin && item_end <= walk.x;
        // (a warp's last state goes where its ring was)
        float* const state = kApart || walk.x >= walk.end ? reinterpret_cast<float*>(smem + warp_in * S::kWarpBytes)
                                                          : A.states + size_t(worker0 + warp_in) * S::kCols * (D + 4);
        if (!whole && lane == 0) {
            const int slot = item_at <= walk.begin ? 0 : 1;
            const long each = walk.each, longer = walk.longer;
            auto worker_of = [&](long at) {
                at -= walk.origin;
                return walk.worker +
                       int(at < longer * (each + 1) ? quotient(at, each + 1) : longer + quotient(at - longer * (each + 1), max(1L, each)));
            };
            places[warp_in][slot] = state;
            const int4 info = make_int4(walk.first, walk.tile | walk.rows << 24, walk.head | slot << 30, worker_of(item_end - 1));
            if (item_at >= walk.begin) runs[1 + warp_in] = info;
            if (item_at < walk.begin && warp_in == 0 && !kApart) runs[0] = info;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float sum = l[n][c];
#pragma unroll
                for (int o = 4; o < 32; o *= 2) sum += __shfl_xor_sync(kFull, sum, o);
                if (__any_sync(kFull, broken)) sum = __int_as_float(0x7fffffff);
                const int col = 8 * n + 2 * t + c, mine = P == 2 ? col >> 2 : 0, row = P == 2 ? col & 3 : col;
                if (row >= walk.rows) continue;
                const float f = whole ? (sum == 0.f ? 0.f : 0x1p-4f / sum) : 0x1p-4f;
                if (whole) {
                    const int r = walk.tile * R + row, token = r / A.G;
                    __nv_bfloat16* to = A.out + ((size_t(walk.first + token) * A.c.hkv + walk.head + mine) * A.G + r - token * A.G) * D;
#pragma unroll
                    for (int i = 0; i < kI; ++i) {
                        const __nv_bfloat162 x0 = __floats2bfloat162_rn((acc[n][i][0][c] - acc[n][i][0][2 + c]) * f, acc[n][i][0][2 + c] * (f * 0.0625f));
                        const __nv_bfloat162 x1 = __floats2bfloat162_rn((acc[n][i][1][c] - acc[n][i][1][2 + c]) * f, acc[n][i][1][2 + c] * (f * 0.0625f));
                        *reinterpret_cast<uint2*>(to + 32 * i + 4 * g) =
                            make_uint2(reinterpret_cast<const uint32_t&>(x0), reinterpret_cast<const uint32_t&>(x1));
                    }
                } else {
                    float* to = state + col * (D + 4);
#pragma unroll
                    for (int i = 0; i < kI; ++i)
                        *reinterpret_cast<float4*>(to + 32 * i + 4 * g) =
                            make_float4((acc[n][i][0][c] - acc[n][i][0][2 + c]) * f, acc[n][i][0][2 + c] * (f * 0.0625f),
                                        (acc[n][i][1][c] - acc[n][i][1][2 + c]) * f, acc[n][i][1][2 + c] * (f * 0.0625f));
                    if (g == 0) to[D] = ref[n][c], to[D + 1] = sum, to[D + 2] = size[n][c];
                }
            }
        }
    }

    // ---- tiles that several warps of the CTA share: their states in one, 8 lanes to a row ----
    __syncthreads();
    for (int u = threadIdx.x / 8; u < (active + 1) * S::kCols; u += kThreads / 8) {
        const int r = u / S::kCols, col = u - r * S::kCols;
        const int4 info = runs[r];
        const int mine = P == 2 ? col >> 2 : 0, row = P == 2 ? col & 3 : col, last = min(info.w, worker0 + active - 1);
        if (info.x < 0 || row >= info.y >> 24) continue;
        const int w0 = worker0 + max(0, r - 1);
        State<D> st;
#pragma unroll 4
        for (int w = w0; w <= last; ++w)
            st.add(places[w - worker0][r && w == w0 ? info.z >> 30 & 1 : 0] + col * (D + 4));
        if (kApart || (r && info.w < worker0 + active))
            st.write(A.out + row_of<S>(A, info, mine, row) * D);
        else
            st.keep(A.joined + ((size_t(blockIdx.x) * 2 + (r ? 1 : 0)) * S::kCols + col) * (D + 4));
    }
    if (threadIdx.x == 0 && !kApart) {
        int4 going = make_int4(-1, 0, 0, 0);
        for (int r = 1; r <= active; ++r)
            if (runs[r].x >= 0 && runs[r].w >= worker0 + active) going = runs[r], going.w /= active;
        going.w = min(going.w, int(gridDim.x) - 1);
        A.begun[blockIdx.x] = going;
    }
}

// Joins the states of a tile whose keys went to several CTAs: a block per row.
template <class S>
__global__ void __launch_bounds__(kJoin) join_kernel(const Args A) {
    constexpr int D = S::D, kEach = kJoin / 8;
    __shared__ __align__(16) float part[kEach][D + 4];
    wait_for_previous();
    const int group = threadIdx.x / 8, col = blockIdx.y, mine = S::P == 2 ? col >> 2 : 0, row = S::P == 2 ? col & 3 : col;
    const int4 info = A.begun[blockIdx.x];
    if (info.x < 0 || row >= info.y >> 24) return;
    State<D> st;
#pragma unroll 2
    for (int c = blockIdx.x + group; c <= info.w; c += kEach)
        st.add(A.joined + ((size_t(c) * 2 + (c == blockIdx.x ? 1 : 0)) * S::kCols + col) * (D + 4));
    st.keep(part[group]);
    __syncthreads();
    if (group) return;
    State<D> all;
    for (int k = 0; k < kEach && k <= info.w - int(blockIdx.x); ++k) all.add(part[k]);
    all.write(A.out + row_of<S>(A, info, mine, row) * D);
}

// The current device's multiprocessors, with the kernels' shared memory allowed.
template <class S>
cudaError_t prepared(int* sms) {
    static splice::PerDevice<int> counts;
    return counts.get(sms, [](int dev, int* n) {
        cudaError_t e = cudaFuncSetAttribute(attention_kernel<S, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(attention_kernel<S, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        return e == cudaSuccess ? cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev) : e;
    });
}

template <class S>
constexpr long scratch_of(int sms) { return sms * ((S::kWarps + 2L) * S::kCols * (S::D + 4) * 4 + 16); }

template <class S>
int launch(const Args& a, void* scratch, cudaStream_t stream) {
    int sms = 0;
    const cudaError_t e = prepared<S>(&sms);
    if (e != cudaSuccess) return int(e);
    Args A = a;
    // Tiles that are short, however long the sequences are, and even enough on the warps
    // are apart: each with warps of one CTA, as many as there are, so that there is nothing
    // to join across CTAs, and no second launch.  32 / 8 heads of 128, apart and on the line,
    // us: 300 sequences of 100 tokens 14 and 24, 1000 of them 40 and 45, 32 of 200 9.5 and 14,
    // one of 300 9.2 and 11, of 1000 14 and 11, of 4000 34 and 12; 8 of 600 11.9 and 10.7, but
    // the host's call is shorter by 2.
    // (a sequence's last tile may be begun, or each token's)
    const long R = S::kRows, rows = long(a.s.rows) * a.G, warps = long(sms) * S::kWarps;
    const long tiles = std::min((a.G + R - 1) / R * a.s.rows, (rows + a.s.batch * (R - 1)) / R) * (a.c.hkv / S::P);
    long stages = ((long(a.s.width) << a.c.log_page) + S::kKeys - 1) / S::kKeys;
    if (a.window) stages = std::min(stages, (a.window + (R + a.G - 2) / a.G + 2 * S::kKeys - 2) / S::kKeys);
    int to_tile = 1;
    for (int n = 2; n <= S::kWarps; ++n)
        if (S::kWarps % n == 0 && tiles * n <= warps && to_tile * S::kLeast < stages) to_tile = n;
    const long most = (tiles * to_tile + warps - 1) / warps * stages;       // (a warp's, times to_tile)
    if (stages <= kMost * to_tile && most * warps <= to_tile * (kMore * warps + tiles * (stages + S::kBegin))) A.apart = to_tile;
    if (!A.apart) {
        if (!scratch) return -1;
        A.states = static_cast<float*>(scratch);
        A.joined = A.states + long(sms) * S::kWarps * S::kCols * (S::D + 4);
        A.begun = reinterpret_cast<int4*>(A.joined + sms * 2L * S::kCols * (S::D + 4));
    }
    const int rc = dependent(A.apart ? attention_kernel<S, true> : attention_kernel<S, false>, dim3(unsigned(sms)), S::kThreads, S::kSmem,
                             stream, A);
    if (rc || A.apart) return rc;
    return dependent(join_kernel<S>, dim3(unsigned(sms), S::kCols), kJoin, 0, stream, A);
}

template <int D>
int run(const Args& a, void* scratch, cudaStream_t stream) {
    // By the rows of a kv head that a sequence has on average: up to four share the
    // columns with those of the next head (64 sequences of 4000 tokens, one row of 128: 60
    // us for 65; 256 with four of 64: 118 for 134; 64 with two of 256: 49 for 51), more
    // than eight take sixteen columns (24 sequences of up to 16 tokens with four rows of
    // 128: 52 for 56; of 256 they spill, 48 sequences of 8 tokens with two rows 74 for 51).
    const long rows = long(a.s.rows) * a.G, all = a.s.batch;
    if (rows <= 4 * all && a.c.hkv % 2 == 0) return launch<Shape<D, 1, 2>>(a, scratch, stream);
    if constexpr (D < 256)
        if (rows > 8 * all) return launch<Shape<D, 2, 1>>(a, scratch, stream);
    return launch<Shape<D, 1, 1>>(a, scratch, stream);
}

}  // namespace
}  // namespace decoder

using namespace decoder;

// Bytes of scratch of any call for heads of d on the current device; below 0: a CUDA
// error, negated.
extern "C" long decoder_page_attention_scratch(int d) {
    if (d != 64 && d != 128 && d != 256) return -long(cudaErrorInvalidValue);
    int sms = 0;
    const cudaError_t e = prepared<Shape<64, 1, 1>>(&sms);
    if (e != cudaSuccess) return -long(e);
    return d == 64    ? std::max(scratch_of<Shape<64, 2, 1>>(sms), scratch_of<Shape<64, 1, 1>>(sms))
           : d == 128 ? std::max(scratch_of<Shape<128, 2, 1>>(sms), scratch_of<Shape<128, 1, 1>>(sms))
                      : scratch_of<Shape<256, 1, 1>>(sms);
}

// q [rows][hq][d] (its strides: token, head) over the layer's pages; out [rows][hq][d].  -1:
// nothing is done, as it takes scratch, and there is none.
extern "C" int decoder_page_attention(const PageCache* cache, int layer, const void* q, long q_token, long q_head, const void* table,
                                      const void* starts, const void* lengths, int width, int batch, int rows, int hq, float scale, int window,
                                      void* out, void* scratch, void* stream) {
    if (!cache->valid() || layer < 0 || layer >= cache->layers || width < 1 || batch < 1 || rows < 1 || hq < 1 || hq % cache->hkv ||
        window < 0 || long(rows) * hq >= 1L << 26)
        return int(cudaErrorInvalidValue);
    Args a = {};
    a.c = cache->layer(layer);
    a.s = {static_cast<const int*>(table), static_cast<const int*>(starts), static_cast<const int*>(lengths), width, batch, rows};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.q_token = q_token, a.q_head = q_head;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.G = hq / cache->hkv, a.window = window, a.scale = scale;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cache->d == 64 ? run<64>(a, scratch, s) : cache->d == 128 ? run<128>(a, scratch, s) : run<256>(a, scratch, s);
}
