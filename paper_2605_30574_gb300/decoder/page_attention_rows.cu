// Attention of many rows to a kv head over its pages: several new tokens to a sequence.
//
// The few-row kernel (page_attention.cu) makes operands of the codes in each warp, for eight
// rows.  With more rows than that it does so again and again, so here a CTA makes 64 keys
// and values at a time numbers in fp16 in shared memory, once for up to 64 rows:
// (n - 8) r, of seven bits, is exact, and is one product and sum of the masked nibble, as
// (64 + n) r - 72 r.  What is left of a key's scale is the power of two of its row, which
// the scores take, and of a value's, which its weight takes.  Weights are relative to the
// largest of (score + E of the value's row), as in the few-row kernel.
//
// A CTA's eight warps take a tile of 16 rows and part of the stage's keys each: 16 keys of
// one of two tiles, or 32 of one of four.  Rows are on the 16-row side of m16n8k16, so that
// the scores are the weights' operand as they are; keys and values come by ldmatrix,
// 16-byte chunks ordered by key to spread over the banks.  Two CTAs to an SM: one's products
// run under the other's conversion.  The warps' states of a row are joined in shared memory
// at a tile's end.
//
// Within a row of 8-element chunks c = 4i' + t' (of keys; words t' + 4 i') elements lie as
// 0, 4, 1, 5, 2, 6, 3, 7, which masks of a word give; q's rows are laid out likewise.  A
// value's chunk holds its words' runs g of two groups by turns.
#include <type_traits>

#include "../csrc/per_device.h"
#include "decoder.h"
#include "page_attention.cuh"

namespace decoder {
namespace page {
namespace {

template <int D_>
struct Many {
    static constexpr int D = D_, kI = D / 32, kKeys = 64, kRows = 64, kThreads = 256, kWarps = 8, kStages = 2;
    static constexpr int kBegin = 2;                                // stages that a tile's begin and end take as long as
    // a stage as it lies in the pages, where its parts are
    static constexpr int kV = kKeys * D / 2, kKr = kKeys * D, kVr = kKr + kKeys * kI, kE = kVr + kKeys * kI, kRaw = kE + kKeys * 2;
    // numbers: keys, values and q, rows of 2 D bytes; the keys' two powers of two; then the
    // warps' states where all that was
    static constexpr int kKeysAt = kStages * kRaw, kValuesAt = kKeysAt + kKeys * 2 * D, kQAt = kValuesAt + kKeys * 2 * D,
                         kPowersAt = kQAt + kRows * 2 * D, kUsed = kPowersAt + kKeys * 8, kStates = kWarps * 16 * (D + 4) * 4;
    static constexpr int kSmem = kUsed > kStates ? kUsed : kStates;
    static_assert(kSmem <= 100 * 1024 && kRaw % 16 == 0);
};

// What a CTA does with its share.
struct Walk {
    long x, end, begin, at, item_at;
    int b, first, head, tile, rows, broken;
    long line;
    int pos[64], ids[64];
    float factor[64];
};

__device__ __forceinline__ void ldmatrix(uint32_t* x, uint32_t from) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from));
}

__device__ __forceinline__ void ldmatrix_trans(uint32_t* x, uint32_t from) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                 : "r"(from));
}

__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    const __half2 h = __hfma2(reinterpret_cast<const __half2&>(a), reinterpret_cast<const __half2&>(b), reinterpret_cast<const __half2&>(c));
    return reinterpret_cast<const uint32_t&>(h);
}

struct Seq {
    int first, new_, length, tiles, weight;
    long line;                                  // of a tile
};

// A stage of a sequence's tiles counts by their rows: its conversion and their products.
template <class S>
__device__ __forceinline__ Seq sequence(const Args& A, int b) {
    Seq q;
    const int first = max(0, min(A.s.starts[b], A.s.rows)), end = max(first, min(A.s.starts[b + 1], A.s.rows));
    q.first = first;
    q.new_ = end - first;
    q.length = max(0, A.s.lengths[b]);
    const long rows = long(q.new_) * A.G;
    q.tiles = int((rows + S::kRows - 1) / S::kRows);
    int stages = q.length / S::kKeys + (q.length % S::kKeys != 0);
    if (A.window) stages = min(stages, int((long(A.window) + (S::kRows + A.G - 2) / A.G + 2 * S::kKeys - 2) / S::kKeys));
    q.weight = 2 + int(min(long(S::kRows), rows) + 15) / 16;
    q.line = long(max(1, stages) + S::kBegin) * q.weight;
    return q;
}

// Eight elements of a word (or four of two runs): nibbles times r16, and -72 r added.
__device__ __forceinline__ void numbers(uint32_t word, uint32_t r16, uint32_t minus, uint32_t to) {
    auto part = [&](uint32_t x) { return fma2((x & 0x00f000f0u) | 0x64006400u, r16, minus); };
    sts16(to, part(word << 4), part(word), part(word >> 4), part(word >> 8));
}

template <class S>
__global__ void __launch_bounds__(S::kThreads, 2) rows_kernel(const Args A) {
    constexpr int D = S::D, kI = S::kI, R = S::kRows, kThreads = S::kThreads;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long before[kThreads + 1];       // work before each run of sequences
    __shared__ long sums[S::kWarps];
    __shared__ Walk walk;
    wait_for_previous();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = threadIdx.x / 32;
    const int run = (A.s.batch + kThreads - 1) / kThreads;
    {
        long mine = 0;
        for (int b = threadIdx.x * run; b < min(A.s.batch, int(threadIdx.x + 1) * run); ++b) {
            const Seq q = sequence<S>(A, b);
            mine += q.line * q.tiles * A.c.hkv;
        }
        long x = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long y = __shfl_up_sync(kFull, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        for (int w = 0; w < warp; ++w) x += sums[w];
        before[threadIdx.x + 1] = x;
        if (threadIdx.x == 0) before[0] = 0;
        __syncthreads();
    }
    const long total = before[kThreads], workers = max(1L, min(long(gridDim.x), quotient(total, 8)));
    // (the first total % workers have one unit more)
    const long each = quotient(total, workers), longer = total - each * workers;
    if (threadIdx.x == 0) {
        const int worker = blockIdx.x;
        walk.x = walk.begin = worker < workers ? each * worker + min(long(worker), longer) : 0;
        walk.end = worker < workers ? walk.begin + each + (worker < longer) : 0;
        int lo = 0;
        for (int step = kThreads / 2; step; step /= 2)
            if (before[lo + step] <= walk.x) lo += step;
        walk.at = before[lo];
        walk.b = min(lo * run, A.s.batch - 1);
        A.begun[blockIdx.x] = make_int4(-1, 0, 0, 0);
    }
    __syncthreads();

    const uint32_t base_at = smem_u32(smem), keys_at = base_at + S::kKeysAt, values_at = base_at + S::kValuesAt, q_at = base_at + S::kQAt,
                   powers_at = base_at + S::kPowersAt;
    while (walk.x < walk.end) {
        const long x = walk.x, end = walk.end;
        long at = walk.at;
        int b = walk.b;
        Seq sq = sequence<S>(A, b);
        while (at + sq.line * sq.tiles * A.c.hkv <= x) {
            at += sq.line * sq.tiles * A.c.hkv;
            if (++b >= A.s.batch) break;         // (lengths that changed under the call)
            sq = sequence<S>(A, b);
        }
        if (b >= A.s.batch) break;
        const int item = int(quotient(x - at, sq.line));
        const long item_at = at + item * sq.line, item_end = min(item_at + sq.line, end);
        // (a stage is the CTA's that its first unit is)
        const int j0 = int(quotient(x - item_at + sq.weight - 1, sq.weight)), j1 = int(quotient(item_end - item_at + sq.weight - 1, sq.weight));
        const int head = item / sq.tiles, tile = item - head * sq.tiles;
        const int rows = int(min(long(R), long(sq.new_) * A.G - long(tile) * R));
        const int base = sq.length - sq.new_;
        const int first_pos = base + tile * R / A.G, last_pos = base + (tile * R + rows - 1) / A.G;
        const int kb0 = A.window ? max(0, first_pos - A.window + 1) / S::kKeys : 0;
        const int kb_end = min(kb0 + j1 - S::kBegin, (last_pos + S::kKeys) / S::kKeys);
        int kb = kb0 + max(0, j0 - S::kBegin), kb_in = kb;
        const int* table = A.s.table + size_t(b) * A.s.width;
        __syncthreads();
        if (threadIdx.x == 0) {
            walk.x = item_end, walk.at = at, walk.item_at = item_at, walk.line = sq.line;
            walk.b = b, walk.first = sq.first, walk.head = head, walk.tile = tile, walk.rows = rows, walk.broken = 0;
        }
        // ---- stages on their way: the numbers of 64 pages in the walk ----
        auto place = [&](int key) { return key >> A.c.log_page; };
        auto look_up = [&](int first) {
            const int i = first + int(threadIdx.x);
            if (threadIdx.x < 32) walk.ids[i & 63] = i < A.s.width ? __ldg(table + i) : -1;
        };
        look_up(place(kb * S::kKeys) & ~31);
        look_up((place(kb * S::kKeys) & ~31) + 32);
        __syncthreads();
        const uint32_t page_rows = 1u << A.c.log_page, both = page_rows * A.c.hkv;       // (of keys or values, of a page)
        auto fill = [&]() {
            if (kb_in < kb_end) {
                const int key0 = kb_in * S::kKeys, i = place(key0);
                if ((i & 31) == 0) {
                    __syncthreads();
                    look_up(i + 32);
                    __syncthreads();
                }
                const uint32_t raw = base_at + kb_in % S::kStages * S::kRaw;
                // a key's place in a page: rows of keys before it, or -1
                auto row_of_key = [&](int key, uint64_t* page) {
                    if (key > last_pos) return -1;
                    const int id = walk.ids[place(key) & 63];
                    if (id < 0 || id >= A.c.pages) {
                        walk.broken = 1;
                        return -1;
                    }
                    *page = uint64_t(uint32_t(id));
                    return int(page_rows * head + (key & (page_rows - 1)));
                };
                constexpr int kChunks = D / 32;  // (of 16 bytes, of a row's codes)
                uint64_t page;
                if (int(threadIdx.x) < S::kKeys * kChunks) {
                    const int key = threadIdx.x / kChunks, c = threadIdx.x % kChunks, row = row_of_key(key0 + key, &page);
                    if (row >= 0) {
                        const uint8_t* from = A.c.codes + page * (both * D) + uint32_t(row) * (D / 2) + 16 * c;
                        cp16(raw + key * (D / 2) + 16 * c, from);
                        cp16(raw + S::kV + key * (D / 2) + 16 * c, from + both * (D / 2));
                    }
                }
                constexpr int kEach = 16 / kI, kRatios = S::kKeys / kEach;       // (keys to 16 bytes of ratios)
                if (int(threadIdx.x) < 2 * kRatios) {
                    const int kv = threadIdx.x / kRatios, key = threadIdx.x % kRatios * kEach, row = row_of_key(key0 + key, &page);
                    if (row >= 0)
                        cp16(raw + (kv ? S::kVr : S::kKr) + key * kI, A.c.ratios + page * (both * 2 * kI) + (kv ? both : 0) * kI + uint32_t(row) * kI);
                }
                if (int(threadIdx.x) >= 64 && int(threadIdx.x) < 72) {
                    const int key = (threadIdx.x - 64) * 8, row = row_of_key(key0 + key, &page);
                    if (row >= 0) cp16(raw + S::kE + key * 2, A.c.exponents + page * (both * 2) + uint32_t(row) * 2);
                }
                ++kb_in;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < S::kStages; ++i) fill();

        // ---- the rows: q as numbers below 2^15, four threads to a row ----
        {
            const int row = threadIdx.x / 4, r = tile * R + row, token = r / A.G, c = threadIdx.x & 3;
            uint32_t raw[kI][4] = {}, top2 = 0;
            if (row < rows) {
                const __nv_bfloat16* p = A.q + (sq.first + token) * A.q_token + (head * A.G + r - token * A.G) * A.q_head;
#pragma unroll
                for (int i = 0; i < kI; ++i) {
                    const uint4 y = __ldg(reinterpret_cast<const uint4*>(p + 32 * i + 8 * c));
                    raw[i][0] = y.x, raw[i][1] = y.y, raw[i][2] = y.z, raw[i][3] = y.w;
                }
            }
#pragma unroll
            for (int i = 0; i < kI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) top2 = __vmaxu2(top2, raw[i][j] & 0x7fff7fffu);
            unsigned top = max(top2 & 0xffffu, top2 >> 16);
            top = max(top, __shfl_xor_sync(kFull, top, 1));
            top = max(top, __shfl_xor_sync(kFull, top, 2));
            const int E = max(int(top >> 7), kLeastExponent);
            // (a row with infinities or NaN: NaN)
            const float up = E == 255 ? __int_as_float(0x7fffffff) : power_of(268 - E);
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(j & 1 ? raw[i][j / 2] & 0xffff0000u : raw[i][j / 2] << 16) * up;
                sts16(q_at + row * 2 * D + ((4 * i + c) ^ (row & 7)) * 16, half2_of(f[0], f[4]), half2_of(f[1], f[5]), half2_of(f[2], f[6]),
                      half2_of(f[3], f[7]));
            }
            if (c == 0) {
                // (S 2^(E_k - 2) / up, in bits)
                walk.factor[row] = row < rows ? power_of(E < 255 ? E - 14 : 1) * (0.25f * kLog2e) * A.scale : 0.f;
                walk.pos[row] = row < rows ? base + token : -1;
            }
        }
        __syncthreads();
        // a warp's tile of rows and share of a stage's keys
        const int parts = rows <= 32 ? 4 : 2, mine = warp / parts, key_at = warp % parts * (64 / parts);
        const bool idle = 16 * mine >= rows;
        const int row0 = min(16 * mine, R - 16) + g;
        const float factor[2] = {walk.factor[row0], walk.factor[row0 + 8]};
        const int pos[2] = {walk.pos[row0], walk.pos[row0 + 8]};
        const uint32_t a_at = q_at + (row0 - g + (lane & 15)) * 2 * D;
        float acc[D / 8][4] = {}, l[2] = {}, ref[2] = {kNone, kNone};

        // ---- the keys ----
        for (; kb < kb_end; ++kb) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
            __syncthreads();
            const int key0 = kb * S::kKeys;
            {
                // four threads to a key and a value: 16 (8) bytes of the codes each
                const uint32_t raw = base_at + kb % S::kStages * S::kRaw;
                const int key = threadIdx.x / 4, c = threadIdx.x & 3;
                // (what no row sees may hold anything, and counts as zeros)
                const bool seen = key0 + key <= last_pos && (!A.window || key0 + key > first_pos - A.window);
                uint32_t k[kI], v[kI], kr[1], vr[1];
                lds<4 * kI>(k, raw + key * (D / 2) + c * 4 * kI);
                lds<4 * kI>(v, raw + S::kV + key * (D / 2) + c * 4 * kI);
                lds<kI>(kr, raw + S::kKr + key * kI);
                lds<kI>(vr, raw + S::kVr + key * kI);
                const uint32_t k16 = seen ? 0x2c002c00u : 0u, k72 = seen ? 0xd480d480u : 0u;      // 1 / 16, -72
                if (!seen) kr[0] = vr[0] = 0;
#pragma unroll
                for (int i = 0; i < kI; ++i) {
                    const uint32_t r = bytes_of(kr[0], 0, i | 8 << 4 | i << 8 | 8 << 12) << 7;
                    numbers(k[i], mul2(r, k16), mul2(r, k72), keys_at + key * 2 * D + ((4 * i + c) ^ (key & 7)) * 16);
                }
#pragma unroll
                for (int j = 0; j < kI; ++j) {
                    const uint32_t r = bytes_of(vr[0], 0, j % (kI / 2) ? 0xb3a2u : 0x9180u) << 7;
                    numbers(v[j], mul2(r, k16), mul2(r, k72), values_at + key * 2 * D + ((c * kI + j) ^ (key & 7)) * 16);
                }
                if (c == 0) {
                    uint32_t e[1];
                    lds<2>(e, raw + S::kE + key * 2);
                    float ek = power_of(e[0] & 255), up = power_of(e[0] >> 8);
                    // (infinite, of a key or value of NaN: the score is NaN)
                    ek = fmaf(up, 0.f, fmaf(ek, 0.f, ek));
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(powers_at + key * 8), "f"(ek), "f"(up * 0x1p6f) : "memory");
                }
            }
            __syncthreads();
            fill();
            if (idle) continue;
#pragma unroll 1
            for (int at_key = key_at; at_key < key_at + 64 / parts; at_key += 16) {
                if (key0 + at_key > last_pos) break;
                const bool edge = key0 + at_key + 15 > first_pos || (A.window && key0 + at_key <= last_pos - A.window);
                float s[2][4] = {};
#pragma unroll
                for (int c = 0; c < D / 8; c += 2) {
                    // rows lane & 15 of q, keys (lane & 7) and + 8, chunks c and c + 1
                    uint32_t a[4], y[4];
                    ldmatrix(a, a_at + ((c + (lane >> 4)) ^ (lane & 7)) * 16);
                    ldmatrix(y, keys_at + (at_key + (lane & 7) + (lane >> 4) * 8) * 2 * D + ((c + (lane >> 3 & 1)) ^ (lane & 7)) * 16);
                    mma(s[0], a, y[0], y[1]);
                    mma(s[1], a, y[2], y[3]);
                }
                // weights: rows g and g + 8, keys 2t, 2t + 1 and 8 on
                float power[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t y[4];
                    lds<16>(y, powers_at + (at_key + 8 * j + 2 * t) * 8);
#pragma unroll
                    for (int i = 0; i < 4; ++i) power[j][i] = __uint_as_float(y[i]);
                }
                float p[2][4], pv[2][4], most = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float y = fmaf(s[j][i], factor[i >> 1] * power[j][2 * (i & 1)], -ref[i >> 1]);
                        if (edge) {
                            const int key = key0 + at_key + 8 * j + 2 * t + (i & 1), last = pos[i >> 1];
                            if (key > last || (A.window && key <= last - A.window)) y = -INFINITY;
                        }
                        p[j][i] = ex2(y);
                        pv[j][i] = edge && y == -INFINITY ? 0.f : p[j][i] * power[j][2 * (i & 1) + 1];
                        most = fmaxf(most, pv[j][i]);
                        s[j][i] = edge && y == -INFINITY ? -INFINITY : s[j][i] * (factor[i >> 1] * power[j][2 * (i & 1)]);
                    }
                // what is past the reference is found by the weights: infinite, or too large
                if (__any_sync(kFull, most > 0x1p14f)) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float top = -INFINITY;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                top = fmaxf(top, s[j][2 * r + i] + float(int(__float_as_uint(power[j][2 * i + 1]) >> 23) - 133));
                        top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
                        const float m = fmaxf(ref[r], top), f = ex2(ref[r] - m);
                        ref[r] = m;
                        l[r] *= f;
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) acc[c][2 * r] *= f, acc[c][2 * r + 1] *= f;
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            p[j][i] = ex2(s[j][i] - ref[i >> 1]);
                            pv[j][i] = edge && s[j][i] == -INFINITY ? 0.f : p[j][i] * power[j][2 * (i & 1) + 1];
                        }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) l[r] += (p[0][2 * r] + p[0][2 * r + 1]) + (p[1][2 * r] + p[1][2 * r + 1]);
                const uint32_t w[4] = {half2_of(pv[0][0], pv[0][1]), half2_of(pv[0][2], pv[0][3]), half2_of(pv[1][0], pv[1][1]),
                                       half2_of(pv[1][2], pv[1][3])};
#pragma unroll
                for (int c = 0; c < D / 8; c += 2) {
                    uint32_t y[4];
                    ldmatrix_trans(y, values_at + (at_key + (lane & 15)) * 2 * D + ((c + (lane >> 4)) ^ (lane & 7)) * 16);
                    mma(acc[c], w, y[0], y[1]);
                    mma(acc[c + 1], w, y[2], y[3]);
                }
            }
        }

        // ---- the rows' states: joined here, then out, or left for the join ----
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        float* states = reinterpret_cast<float*>(smem);
        if (!idle) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float* to = states + (warp * 16 + g + 8 * r) * (D + 4);
                float sum = l[r];
                sum += __shfl_xor_sync(kFull, sum, 1);
                sum += __shfl_xor_sync(kFull, sum, 2);
                if (t == 0) to[D] = ref[r], to[D + 1] = sum;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    // chunk c: word c % kI of its quarter, element t of two runs
                    const int j = c % kI, dim = 64 * (j % (kI / 2)) + 4 * (c / kI * 2 + j / (kI / 2)) + t;
                    to[dim] = acc[c][2 * r] * 0x1p-8f;
                    to[dim + 32] = acc[c][2 * r + 1] * 0x1p-8f;
                }
            }
        }
        __syncthreads();
        const bool whole = item_at >= walk.begin && item_end == item_at + sq.line;
        const int4 info = make_int4(sq.first, tile | rows << 24, head, 0);
        for (int row = threadIdx.x / 8; row < rows; row += kThreads / 8) {
            State<D> st;
            for (int k = 0; k < parts; ++k) st.add(states + ((row / 16 * parts + k) * 16 + row % 16) * (D + 4));
            if (walk.broken) st.l = __int_as_float(0x7fffffff);
            if (whole)
                st.write(A.out + row_of<R>(A, info, 0, row) * D);
            else
                st.keep(A.joined + ((size_t(blockIdx.x) * 2 + (item_at >= walk.begin ? 1 : 0)) * R + row) * (D + 4));
        }
        if (!whole && item_at >= walk.begin && threadIdx.x == 0) {
            const long last = item_at + sq.line - 1;
            const long worker = last < longer * (each + 1) ? quotient(last, each + 1) : longer + quotient(last - longer * (each + 1), max(1L, each));
            A.begun[blockIdx.x] = make_int4(info.x, info.y, info.z, int(min(worker, long(gridDim.x) - 1)));
        }
        __syncthreads();
    }
}

template <class S>
cudaError_t prepared(int* grid) {
    static splice::PerDevice<int> counts;
    return counts.get(grid, [](int dev, int* n) {
        const cudaError_t e = cudaFuncSetAttribute(rows_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        if (e != cudaSuccess) return e;
        int sms = 0;
        const cudaError_t f = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        *n = 2 * sms;
        return f;
    });
}

template <class S>
int launch(const Args& a, void* scratch, cudaStream_t stream) {
    int grid = 0;
    const cudaError_t e = prepared<S>(&grid);
    if (e != cudaSuccess) return int(e);
    Args A = a;
    A.joined = static_cast<float*>(scratch);
    A.begun = reinterpret_cast<int4*>(A.joined + grid * 2L * S::kRows * (S::D + 4));
    const int rc = dependent(rows_kernel<S>, dim3(unsigned(grid)), S::kThreads, S::kSmem, stream, A);
    return rc ? rc : dependent(join_kernel<S::D, S::kRows, 1>, dim3(unsigned(grid), 8), kJoin, 0, stream, A);
}

template <class S>
cudaError_t scratch_of(long* bytes) {
    int grid = 0;
    const cudaError_t e = prepared<S>(&grid);
    *bytes = grid * (2L * S::kRows * (S::D + 4) * 4 + 16);
    return e;
}

}  // namespace

int many_rows(const Args& a, int d, void* scratch, cudaStream_t stream) {
    return d == 64 ? launch<Many<64>>(a, scratch, stream) : launch<Many<128>>(a, scratch, stream);
}

cudaError_t many_rows_scratch(int d, long* bytes) { return d == 64 ? scratch_of<Many<64>>(bytes) : scratch_of<Many<128>>(bytes); }

}  // namespace page
}  // namespace decoder
