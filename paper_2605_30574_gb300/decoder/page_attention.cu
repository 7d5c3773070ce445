// Attention of each sequence's newest tokens over its pages of a cache in 4 bits.
//
//   out_i = sum_j p_ij v_j,  p_ij = softmax over j of scale q_i . k_j,
//   j <= pos_i = length - new + i,  j > pos_i - window
//
// A step reads every key and value once for the G = Hq / Hkv query rows of a kv head
// (times its new tokens): 138 bytes to 1024 G flops at 128 dims, so HBM is the bound,
// and what a kernel may spend on making operands of 4-bit codes is about three
// instructions of a lane to an element.  Products therefore take the codes as they
// are: a nibble n = c + 8, masked in place, is the fp16 number n 2^-24 (bits 0 to 3) or
// 16 n 2^-24 (bits 4 to 7), so that one shift and four ANDs make eight elements.
//
//  * Scores: S[key][row], keys on the 16-row side of m16n8k16, the rows (eight, or twice
//    eight) on the other.  q is scaled to 2^14 by a power of two and rounded to fp16 (all
//    of bf16's bits down to 2^-28 of the row's largest), with 1/16 where the code comes
//    16-fold; a group's sum starts from -8 sum q, which takes the 8 out of c + 8; groups
//    are added up in fp32 by their ratios.
//  * Output: O[dim][row].  P as the fp16 operand has V's scales in it, so it is taken
//    relative to the largest of (score + E of the value's row), and not of the score:
//    then no product of a weight and a scale is above 2^15, and one that is rounded or
//    lost below fp16's normal range is 2^-29 of the largest.  Codes have their 8
//    subtracted (exactly): O would otherwise carry it through sums of thousands of keys.
//  * The transposition from S's layout to an operand is movmatrix; a key's four lanes and
//    a row's eight are those of both.
//
// Work: all (sequence, kv head, tile of rows, 16 keys) in one line, an even share to
// each warp, whatever the sequences' lengths, which only the device knows.  A tile whose
// keys fall to several warps leaves a state (m, l, O) per warp, and a second kernel joins
// them in the warps' order: the same inputs give the same bits.
#include <cuda_fp16.h>

#include "../csrc/per_device.h"
#include "decoder.h"
#include "pages.cuh"

namespace decoder {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1e30f;         // the reference of rows that have seen nothing
constexpr float kTau = 8.f;             // how far weights may pass the reference, in bits
constexpr int kMinShare = 4;            // blocks of 16 keys to a warp, at least

struct Args {
    PageLayer c;
    PageRows s;
    const __nv_bfloat16* q;
    long q_token, q_head;
    __nv_bfloat16* out;
    int G, window;
    float scale;
    float* states;          // [worker][2][rows][d + 2]
    int4* begun;            // per worker: the tile whose keys begin with it and go on
};

template <int D>
constexpr int ctas_per_sm(int nt) { return D == 256 || nt == 2 ? 1 : 2; }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// `N` consecutive bytes at their own alignment as words (a half word: zero-extended).
template <int N>
__device__ __forceinline__ void load_bytes(uint32_t* to, const uint8_t* p) {
    if constexpr (N == 2) to[0] = *reinterpret_cast<const uint16_t*>(p);
    if constexpr (N == 4) to[0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (N == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        to[0] = x.x, to[1] = x.y;
    }
    if constexpr (N >= 16) {
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            const uint4 x = reinterpret_cast<const uint4*>(p)[i];
            to[4 * i] = x.x, to[4 * i + 1] = x.y, to[4 * i + 2] = x.z, to[4 * i + 3] = x.w;
        }
    }
}

// The sequences' shares of the line of work.  All of a sequence's tiles count as many
// blocks of 16 keys as the one that sees most.
struct Seq {
    int first, new_, length, tiles, blocks;     // (its first row of q; its tokens, its keys)
};

template <int R>
__device__ __forceinline__ Seq sequence(const Args& A, int b) {
    Seq q;
    const int first = max(0, min(A.s.starts[b], A.s.rows)), end = max(first, min(A.s.starts[b + 1], A.s.rows));
    q.first = first;
    q.new_ = end - first;
    q.length = max(0, A.s.lengths[b]);
    q.tiles = int((long(q.new_) * A.G + R - 1) / R);
    int blocks = (q.length + 15) / 16;
    if (A.window) blocks = min(blocks, int((long(A.window) + (R + A.G - 2) / A.G + 30) / 16));
    q.blocks = max(1, blocks);
    return q;
}

template <int R>
__device__ __forceinline__ long size_of(const Args& A, const Seq& q) {
    return long(q.tiles) * A.c.hkv * q.blocks;
}

// What a lane holds of a block of 16 keys: keys g and g + 8 (its words t + 4 i), and for
// the values 2t, 2t + 1, 2t + 8, 2t + 9 (its runs g + 8 i), with ratios and exponents.
template <int D>
struct Block {
    static constexpr int kI = D / 32;
    uint32_t k[2][kI], v[4][(kI + 1) / 2];
    uint32_t kr[2][(kI + 3) / 4], vr[4][(kI + 3) / 4], e[2];
};

template <int D>
__device__ __forceinline__ void fetch(const Args& A, Block<D>& x, int page, int head, int slot) {
    constexpr int kI = D / 32;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const size_t kr = page_row(A.c, page, 0, head, slot), vr = page_row(A.c, page, 1, head, slot),
                 er = exponent_row(A.c, page, head, slot);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const size_t row = kr + g + 8 * h;
        load_bytes<4 * kI>(x.k[h], A.c.codes + row * (D / 2) + t * 4 * kI);
        load_bytes<kI>(x.kr[h], A.c.ratios + row * kI);
        x.e[h] = *reinterpret_cast<const uint16_t*>(A.c.exponents + (er + g + 8 * h) * 2);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const size_t row = vr + 2 * t + (j & 1) + 8 * (j >> 1);
        load_bytes<2 * kI>(x.v[j], A.c.codes + row * (D / 2) + g * 2 * kI);
        load_bytes<kI>(x.vr[j], A.c.ratios + row * kI);
    }
}

// A row's state as it leaves the kernel: O for the reference m and the sum l.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads, ctas_per_sm<D>(NT)) attention_kernel(const Args A, int workers) {
    constexpr int kI = D / 32, R = 8 * NT;
    __shared__ long before[kThreads + 1];       // work before each run of sequences
    __shared__ long sums[kWarps];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp_in = threadIdx.x / 32;
    const int run = (A.s.batch + kThreads - 1) / kThreads;
    {
        long mine = 0;
        for (int b = threadIdx.x * run; b < min(A.s.batch, int(threadIdx.x + 1) * run); ++b) mine += size_of<R>(A, sequence<R>(A, b));
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
    const long share = max(long(kMinShare), (total + workers - 1) / workers);
    const int worker = warp_in * gridDim.x + blockIdx.x;
    long x = worker * share;
    const long end = min(total, x + share);
    if (lane == 0) A.begun[worker] = make_int4(-1, 0, 0, 0);
    if (x >= end) return;
    int lo = 0;                                  // the run of sequences that x is in
    for (int step = kThreads / 2; step; step /= 2)
        if (before[lo + step] <= x) lo += step;
    long at = before[lo];
    int b = lo * run;
    Seq sq = sequence<R>(A, b);
    while (x < end) {
        while (at + size_of<R>(A, sq) <= x) {
            at += size_of<R>(A, sq);
            if (++b >= A.s.batch) return;        // (lengths that changed under the call)
            sq = sequence<R>(A, b);
        }
        const long rel = x - at;
        const int item = int(rel / sq.blocks), j0 = int(rel - long(item) * sq.blocks);
        const int j1 = int(min(long(sq.blocks), j0 + (end - x)));
        const int head = item / sq.tiles, tile = item - head * sq.tiles;
        const long item_at = x - j0;
        x += j1 - j0;
        const int rows = int(min(long(R), long(sq.new_) * A.G - long(tile) * R));

        // ---- the rows: q as an operand, and what is known of each column ----
        uint32_t qf[NT][kI][4];
        float start[NT][kI][2], factor[NT][2], l[NT][2], ref[NT][2];
        int pos[NT][2];
        const int base = sq.length - sq.new_;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int col = 8 * n + g, r = tile * R + col, token = r / A.G;
            const __nv_bfloat16* p = A.q + (sq.first + (col < rows ? token : 0)) * A.q_token +
                                     (head * A.G + (col < rows ? r - token * A.G : 0)) * A.q_head;
            uint32_t raw[kI][4], top2 = 0;
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const uint4 y = *reinterpret_cast<const uint4*>(p + 32 * i + 8 * t);
                raw[i][0] = y.x, raw[i][1] = y.y, raw[i][2] = y.z, raw[i][3] = y.w;
#pragma unroll
                for (int j = 0; j < 4; ++j) top2 = __vmaxu2(top2, raw[i][j] & 0x7fff7fffu);
            }
            unsigned top = max(top2 & 0xffffu, top2 >> 16);
            top = max(top, __shfl_xor_sync(kFull, top, 1));
            top = max(top, __shfl_xor_sync(kFull, top, 2));
            const int E = max(int(top >> 7), kLeastExponent);
            // (a row with infinities or NaN: NaN)
            const float up = E == 255 ? __int_as_float(0x7fffffff) : power_of(268 - E);
            const float down = power_of(E < 255 ? E - 14 : 1);
            float qs[kI];
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                // elements 8t + j of group i, j = 0 .. 7; pairs (j, j + 4) to an operand
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    f[j] = __uint_as_float(j & 1 ? raw[i][j / 2] & 0xffff0000u : raw[i][j / 2] << 16) * up * (j & 1 ? 0.0625f : 1.f);
                qs[i] = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    qf[n][i][j] = half2_of(f[j], f[j + 4]);
                    const float2 y = __half22float2(reinterpret_cast<const __half2&>(qf[n][i][j]));
                    qs[i] = fmaf(y.x + y.y, j & 1 ? -128.f * 0x1p-24f : -8.f * 0x1p-24f, qs[i]);
                }
                qs[i] += __shfl_xor_sync(kFull, qs[i], 1);
                qs[i] += __shfl_xor_sync(kFull, qs[i], 2);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int from = 4 * (2 * t + c);
#pragma unroll
                for (int i = 0; i < kI; ++i) start[n][i][c] = __shfl_sync(kFull, qs[i], from);
                // S 2^(E_k - 2) 2^24 / up, in bits
                factor[n][c] = __shfl_sync(kFull, down, from) * (0x1p22f * kLog2e) * A.scale;
                const int column = 8 * n + 2 * t + c;
                pos[n][c] = column < rows ? base + (tile * R + column) / A.G : -1;
                l[n][c] = 0.f;
                ref[n][c] = kNone;
            }
        }
        float acc[NT][kI][2][4] = {};

        // ---- the keys ----
        const int first_pos = base + tile * R / A.G, last_pos = base + (tile * R + rows - 1) / A.G;
        const int kb0 = A.window ? max(0, first_pos - A.window + 1) / 16 : 0;
        const int kb_end = min(kb0 + j1, (last_pos + 16) / 16);
        const int log_blocks = A.c.log_page - 4, in_page = (1 << log_blocks) - 1;
        const int* table = A.s.table + size_t(b) * A.s.width;
        bool broken = false;                     // a page that is none of the cache's
        auto page_of = [&](int kb) {
            const int i = kb >> log_blocks;
            return kb < kb_end ? i < A.s.width ? __ldg(table + i) : -1 : 0;
        };
        auto checked = [&](int page) {
            if (page >= 0 && page < A.c.pages) return page;
            broken = true;
            return 0;
        };
        int kb = kb0 + j0;
        int next_page = page_of(kb + 1);
        Block<D> now;
        if (kb < kb_end) fetch<D>(A, now, checked(page_of(kb)), head, (kb & in_page) * 16);
        for (; kb < kb_end; ++kb) {
            Block<D> next;
            if (kb + 1 < kb_end) {
                fetch<D>(A, next, checked(next_page), head, (kb + 1 & in_page) * 16);
                next_page = page_of(kb + 2);
            }
            const bool edge = 16 * kb + 15 > first_pos || (A.window && 16 * kb <= last_pos - A.window) || rows < 1;

            // scores
            float s[NT][4] = {};
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                float part[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    part[n][0] = part[n][2] = start[n][i][0], part[n][1] = part[n][3] = start[n][i][1];
                const uint32_t a = now.k[0][i], c = now.k[1][i];
                const uint32_t lo[4] = {a & 0x000f000fu, c & 0x000f000fu, a & 0x00f000f0u, c & 0x00f000f0u};
                const uint32_t a8 = a >> 8, c8 = c >> 8;
                const uint32_t hi[4] = {a8 & 0x000f000fu, c8 & 0x000f000fu, a8 & 0x00f000f0u, c8 & 0x00f000f0u};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma(part[n], lo, qf[n][i][0], qf[n][i][1]);
                    mma(part[n], hi, qf[n][i][2], qf[n][i][3]);
                }
                const uint32_t ra = now.kr[0][i / 4], rc = now.kr[1][i / 4];
                const int sh = 8 * (i & 3);
                const float fa = __uint_as_float((((sh <= 20 ? ra << (20 - sh) : ra >> (sh - 20)) & 0x07f00000u) | 0x38000000u));
                const float fc = __uint_as_float((((sh <= 20 ? rc << (20 - sh) : rc >> (sh - 20)) & 0x07f00000u) | 0x38000000u));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s[n][0] = fmaf(part[n][0], fa, s[n][0]);
                    s[n][1] = fmaf(part[n][1], fa, s[n][1]);
                    s[n][2] = fmaf(part[n][2], fc, s[n][2]);
                    s[n][3] = fmaf(part[n][3], fc, s[n][3]);
                }
            }
            // weights, of keys g and g + 8
            float ek[2], ev[2], up[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = now.e[h] >> 8;
                ek[h] = power_of(now.e[h] & 255);
                up[h] = power_of(e);
                // (infinite, of a key or value of NaN: the score is NaN)
                ek[h] = fmaf(up[h], 0.f, fmaf(ek[h], 0.f, ek[h]));
                up[h] *= 0x1p6f;
                ev[h] = float(e - 127);
            }
            uint32_t w[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int j = 0; j < 4; ++j) s[n][j] *= factor[n][j & 1] * ek[j >> 1];
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = 16 * kb + g + 8 * (j >> 1), p = pos[n][j & 1];
                        if (key > p || (A.window && key <= p - A.window)) s[n][j] = -INFINITY;
                    }
                }
                float top[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) top[c] = fmaxf(s[n][c] + ev[0], s[n][2 + c] + ev[1]);
                if (__any_sync(kFull, top[0] > ref[n][0] + kTau || top[1] > ref[n][1] + kTau)) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
#pragma unroll
                        for (int o = 4; o < 32; o *= 2) top[c] = fmaxf(top[c], __shfl_xor_sync(kFull, top[c], o));
                        const float m = fmaxf(ref[n][c], top[c]), f = ex2(ref[n][c] - m);
                        ref[n][c] = m;
                        l[n][c] *= f;
#pragma unroll
                        for (int i = 0; i < kI; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) acc[n][i][h][c] *= f, acc[n][i][h][2 + c] *= f;
                    }
                }
                float p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = ex2(s[n][j] - ref[n][j & 1]);
                l[n][0] += p[0] + p[2];
                l[n][1] += p[1] + p[3];
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = edge && s[n][j] == -INFINITY ? 0.f : p[j] * up[j >> 1];
                w[n][0] = transposed(half2_of(p[0], p[1]));
                w[n][1] = transposed(half2_of(p[2], p[3]));
            }
            // what no row sees may hold anything: its ratios are left out
            if (edge) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = 16 * kb + 2 * t + (j & 1) + 8 * (j >> 1);
                    if (key > last_pos || (A.window && key <= first_pos - A.window))
#pragma unroll
                        for (int i = 0; i < (kI + 3) / 4; ++i) now.vr[j][i] = 0;
                }
            }
            // output
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                // bytes i of two keys' ratios, as fp16 (the third and fourth: a sign, 0)
                const int sel = (i & 3) | 8 << 4 | (4 + (i & 3)) << 8 | 12 << 12;
                const uint32_t r0 = bytes_of(now.vr[0][i / 4], now.vr[1][i / 4], sel) << 7;
                const uint32_t r1 = bytes_of(now.vr[2][i / 4], now.vr[3][i / 4], sel) << 7;
                const int pick = i & 1 ? 0x7632 : 0x5410;
                const uint32_t a = bytes_of(now.v[0][i / 2], now.v[1][i / 2], pick);
                const uint32_t c = bytes_of(now.v[2][i / 2], now.v[3][i / 2], pick);
                constexpr uint32_t k8 = 0x80088008u, k128 = 0x80808080u;        // -8 2^-24, -128 2^-24
                const uint32_t lo[4] = {add2(a & 0x000f000fu, k8), add2(a & 0x00f000f0u, k128),
                                        add2(c & 0x000f000fu, k8), add2(c & 0x00f000f0u, k128)};
                const uint32_t a8 = a >> 8, c8 = c >> 8;
                const uint32_t hi[4] = {add2(a8 & 0x000f000fu, k8), add2(a8 & 0x00f000f0u, k128),
                                        add2(c8 & 0x000f000fu, k8), add2(c8 & 0x00f000f0u, k128)};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t b0 = mul2(w[n][0], r0), b1 = mul2(w[n][1], r1);
                    mma(acc[n][i][0], lo, b0, b1);
                    mma(acc[n][i][1], hi, b0, b1);
                }
            }
            now = next;
        }

        // ---- the rows' states: out, or left for the join ----
        const bool whole = j0 == 0 && j1 == sq.blocks;
        const int slot = item_at <= worker * share ? 0 : 1;
        if (!whole && j0 == 0 && lane == 0)
            A.begun[worker] = make_int4(sq.first, tile | rows << 24, head | slot << 30, int(min(long(workers) - 1, (item_at + sq.blocks - 1) / share)));
        if (__any_sync(kFull, broken)) l[0][0] = __int_as_float(0x7fffffff);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float sum = l[n][c];
#pragma unroll
                for (int o = 4; o < 32; o *= 2) sum += __shfl_xor_sync(kFull, sum, o);
                if (__any_sync(kFull, broken)) sum = __int_as_float(0x7fffffff);
                const int col = 8 * n + 2 * t + c;
                if (col >= rows) continue;
                const float f = whole ? (sum == 0.f ? 0.f : 0x1p16f / sum) : 0x1p16f;
                if (whole) {
                    const int r = tile * R + col, token = r / A.G;
                    __nv_bfloat16* to = A.out + (size_t(sq.first + token) * A.c.hkv * A.G + head * A.G + r - token * A.G) * D;
#pragma unroll
                    for (int i = 0; i < kI; ++i) {
                        const __nv_bfloat162 x0 = __floats2bfloat162_rn(acc[n][i][0][c] * f, acc[n][i][0][2 + c] * (f * 0.0625f));
                        const __nv_bfloat162 x1 = __floats2bfloat162_rn(acc[n][i][1][c] * f, acc[n][i][1][2 + c] * (f * 0.0625f));
                        *reinterpret_cast<uint2*>(to + 32 * i + 4 * g) =
                            make_uint2(reinterpret_cast<const uint32_t&>(x0), reinterpret_cast<const uint32_t&>(x1));
                    }
                } else {
                    float* to = A.states + ((size_t(worker) * 2 + slot) * R + col) * (D + 4);
#pragma unroll
                    for (int i = 0; i < kI; ++i)
                        *reinterpret_cast<float4*>(to + 32 * i + 4 * g) =
                            make_float4(acc[n][i][0][c] * f, acc[n][i][0][2 + c] * (f * 0.0625f), acc[n][i][1][c] * f,
                                        acc[n][i][1][2 + c] * (f * 0.0625f));
                    if (g == 0) to[D] = ref[n][c], to[D + 1] = sum;
                }
            }
        }
    }
}

// Joins the states of a tile whose keys went to several workers: a block per row.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads) join_kernel(const Args A, int workers) {
    constexpr int R = 8 * NT, kVec = D / 32;
    __shared__ float part[kWarps][D + 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, col = blockIdx.y;
    for (int w0 = blockIdx.x; w0 < workers; w0 += gridDim.x) {
        const int4 x = A.begun[w0];
        const int rows = x.y >> 24, tile = x.y & 0xffffff;
        if (x.x < 0 || col >= rows) continue;
        // (the first worker's state is its second, if it did not begin with the tile)
        float m = kNone, l = 0.f, o[kVec] = {};
        for (int w = w0 + warp; w <= x.w; w += kWarps) {
            const float* from = A.states + ((size_t(w) * 2 + (w == w0 ? x.z >> 30 & 1 : 0)) * R + col) * (D + 4);
            const float mw = from[D], lw = from[D + 1], M = fmaxf(m, mw), f = ex2(m - M), fw = ex2(mw - M);
            m = M;
            l = l * f + lw * fw;
#pragma unroll
            for (int i = 0; i < kVec; ++i) o[i] = o[i] * f + from[lane + 32 * i] * fw;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kVec; ++i) part[warp][lane + 32 * i] = o[i];
        if (lane == 0) part[warp][D] = m, part[warp][D + 1] = l;
        __syncthreads();
        const int head = x.z & 0x3fffffff, r = tile * R + col, token = r / A.G;
        __nv_bfloat16* to = A.out + (size_t(x.x + token) * A.c.hkv * A.G + head * A.G + r - token * A.G) * D;
        if (threadIdx.x < D) {
            float M = kNone, sum = 0.f, y = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) M = fmaxf(M, part[k][D]);
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                const float f = ex2(part[k][D] - M);
                sum += part[k][D + 1] * f;
                y += part[k][threadIdx.x] * f;
            }
            to[threadIdx.x] = __float2bfloat16_rn(sum == 0.f ? 0.f : y / sum);
        }
    }
}

template <int D, int NT>
int launch(const Args& a, void* scratch, cudaStream_t stream, long* bytes) {
    static splice::PerDevice<int> counts;
    int sms = 0;
    const cudaError_t e = counts.get(&sms, [](int dev, int* n) { return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev); });
    if (e != cudaSuccess) return int(e);
    const int grid = sms * ctas_per_sm<D>(NT), workers = grid * kWarps;
    const long states = long(workers) * 2 * 8 * NT * (D + 4) * 4;
    if (bytes) {
        *bytes = states + long(workers) * 16;
        return 0;
    }
    Args A = a;
    A.states = static_cast<float*>(scratch);
    A.begun = reinterpret_cast<int4*>(static_cast<char*>(scratch) + states);
    attention_kernel<D, NT><<<grid, kThreads, 0, stream>>>(A, workers);
    join_kernel<D, NT><<<dim3(unsigned(sms), 8 * NT), kThreads, 0, stream>>>(A, workers);
    return int(cudaGetLastError());
}

int run(const Args& a, int d, void* scratch, cudaStream_t stream, long* bytes) {
    // Sixteen rows to a tile where there are more than eight: the codes are made
    // operands once for both halves.
    const bool two = a.G > 8 || (a.s.rows > a.s.batch && long(a.s.rows) * a.G > 8L * a.s.batch);
    if (d == 64) return two ? launch<64, 2>(a, scratch, stream, bytes) : launch<64, 1>(a, scratch, stream, bytes);
    if (d == 128) return two ? launch<128, 2>(a, scratch, stream, bytes) : launch<128, 1>(a, scratch, stream, bytes);
    return launch<256, 1>(a, scratch, stream, bytes);
}

}  // namespace
}  // namespace decoder

using namespace decoder;

// Bytes of scratch of a call with these numbers, 0 for those that it does not take;
// below 0: a CUDA error, negated.
extern "C" long decoder_page_attention_scratch(int batch, int rows, int hq, int hkv, int d) {
    if (batch < 1 || rows < 1 || hkv < 1 || hq < 1 || hq % hkv || (d != 64 && d != 128 && d != 256) || long(rows) * hq >= 1L << 26) return 0;
    Args a = {};
    a.s.batch = batch, a.s.rows = rows, a.G = hq / hkv;
    long bytes = 0;
    const int rc = run(a, d, nullptr, nullptr, &bytes);
    return rc ? -rc : bytes;
}

// q [rows][hq][d] (its strides: token, head) over the layer's pages; out [rows][hq][d].
extern "C" int decoder_page_attention(const void* codes, const void* ratios, const void* exponents, int pages, int hkv, int d, int log_page,
                                      const void* q, const long* strides, const void* table, const void* starts, const void* lengths,
                                      int width, int batch, int rows, int hq, float scale, int window, void* out, void* scratch,
                                      void* stream) {
    if (pages < 1 || log_page < 4 || log_page > 8 || width < 1 || window < 0 || decoder_page_attention_scratch(batch, rows, hq, hkv, d) <= 0)
        return int(cudaErrorInvalidValue);
    const auto bytes = [](const void* p) { return const_cast<uint8_t*>(static_cast<const uint8_t*>(p)); };
    Args a = {};
    a.c = {bytes(codes), bytes(ratios), bytes(exponents), pages, hkv, log_page};
    a.s = {static_cast<const int*>(table), static_cast<const int*>(starts), static_cast<const int*>(lengths), width, batch, rows};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.q_token = strides[0], a.q_head = strides[1];
    a.out = static_cast<__nv_bfloat16*>(out);
    a.G = hq / hkv, a.window = window, a.scale = scale;
    return run(a, d, scratch, static_cast<cudaStream_t>(stream), nullptr);
}
