// Rows into the pages of a cache in 4 bits and out of them, and pages copied.
//
// All three are bound by HBM: a row of 128 elements is 256 bytes in bf16 and 69 in a
// page, and a copied page is read and written once.  Small calls are latency: the
// search for a row's sequence, its page, the access.
//
// 16384 tokens of 8 heads of 128 with cold caches: stored in 24 us, loaded in 23 (85 MB each:
// 12.6 at the copy rate), what a row's scales cost in instructions and a warp's chain of four
// loads before its first row.  Measured on the way, 20992 tokens of ragged prompts stored and
// then loaded (109 MB each: 32.4 together): 129 with a warp to a row, 79 with eight rows on
// their way in a warp, 70 without divisions (below), 55 with rows of a page a constant apart,
// 51 with sixteen elements to a lane, 49 with CTAs of four warps for eight and a row's
// successor fetched when it is rounded.  36 layers of 340 pages copied: 254 us (1.73 GB, the
// copy rate).
#include "pages.cuh"

#include <algorithm>
#include <cstdlib>

#include "decoder.h"

namespace decoder {
namespace {

constexpr int kThreads = 128, kCopying = 256;
constexpr unsigned kFull = 0xffffffffu;

// The sequence of token `row`, starts[b] <= row < starts[b + 1], one that has tokens: 32
// places at a time, so a look or two for a batch.  row lies between the first start and
// the last.
__device__ int sequence_of(const PageRows& s, int row) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = s.batch;                    // the sequence is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned below = __ballot_sync(kFull, lane * step < n && s.starts[at] <= row);
        const int k = 31 - __clz(below | 1u);
        n = min(step, n - k * step);
        lo += k * step;
    }
    return lo;
}

// The page and slot of a token.  Page -1: no place (a position before the first), -2: a
// page that is none of the cache's, -3: nobody's token.
__device__ __forceinline__ int place_of(const PageLayer& c, const PageRows& s, int b, int row, int* slot) {
    const int first = s.starts[b], last = s.starts[b + 1], at = s.lengths[b] - (last - first) + (row - first);
    if (row < first || row >= last) return -3;
    if (at < 0) return -1;
    const int i = at >> c.log_page;
    if (i >= s.width) return -2;
    const int page = s.table[size_t(b) * s.width + i];
    *slot = at & ((1 << c.log_page) - 1);
    return page < 0 || page >= c.pages ? -2 : page;
}

// The places of tokens row .. row + n - 1, in lanes 0 .. n - 1.
__device__ __forceinline__ int places_of(const PageLayer& c, const PageRows& s, int row, int n, int* slot) {
    const int lane = threadIdx.x & 31, mine = row + lane;
    const int begin = s.starts[0], end = s.starts[s.batch];
    if (row + n <= begin || row >= end) return -3;
    int b = sequence_of(s, min(max(row, begin), end - 1));
    if (n > 1) {
        // the next 32 starts say how many sequences further (behind them a lane goes on by
        // itself)
        const int next = b + 1 + lane <= s.batch ? s.starts[b + 1 + lane] : 0x7fffffff;
        int past = 0;
#pragma unroll
        for (int step = 16; step; step /= 2)
            if (__shfl_sync(kFull, next, past + step - 1) <= mine) past += step;
        b += past;
        while (b < s.batch - 1 && s.starts[b + 1] <= mine) ++b;
    }
    return lane < n && b < s.batch ? place_of(c, s, b, mine, slot) : -3;
}

struct Rows {
    const __nv_bfloat16 *k, *v;     // (written by a load)
    long k_token, k_head, v_token, v_head;
};

// E elements of a row in each lane (8 or 16): where a lane's parts of page 0 are, and what
// is from page to page.  (A page is below 2^27 bytes.)
template <int D, int E>
struct Lane {
    static constexpr int kLanes = D / E, kI = D / 32;
    uint8_t *codes, *ratios, *exponents;
    uint32_t rows;                          // of a page: keys, or values

    __device__ __forceinline__ Lane(const PageLayer& c, int kv, int head) {
        const int w = threadIdx.x & (kLanes - 1), i = w / (32 / E), t = w % (32 / E);
        rows = uint32_t(c.hkv) << c.log_page;
        const uint32_t row = (kv ? rows : 0) + (uint32_t(head) << c.log_page);
        codes = c.codes + row * (D / 2) + (kv ? E / 2 * t * kI + 2 * i : 4 * (E / 8 * t * kI + i));     // (the first word, or run)
        ratios = c.ratios + row * kI + i;
        exponents = c.exponents + ((uint32_t(head) << c.log_page) * 2 + kv);
    }
};

// Where a lane's parts of a token are.
template <int D>
struct Place {
    uint8_t *codes, *ratio, *exponent;
    template <int E>
    __device__ __forceinline__ Place(const Lane<D, E>& at, int page, int slot) {
        const uint64_t n = uint64_t(uint32_t(page)) * at.rows;
        codes = at.codes + n * D + slot * (D / 2);
        ratio = at.ratios + n * (D / 16) + slot * (D / 32);
        exponent = at.exponents + n * 2 + slot * 2;
    }
    // (of the token i places on, in the same page)
    __device__ __forceinline__ uint8_t* codes_at(int i) const { return codes + i * (D / 2); }
    __device__ __forceinline__ uint8_t* ratio_at(int i) const { return ratio + i * (D / 32); }
    __device__ __forceinline__ uint8_t* exponent_at(int i) const { return exponent + i * 2; }
};

template <int D, int N>
__device__ __forceinline__ void quantise_and_store(const Place<D>& at, int n, const uint4* x, int kv, bool out) {
    constexpr int kLanes = D / N, kGroup = 32 / N, kI = D / 32;      // (lanes to a row, and to a group)
    const int w = threadIdx.x & (kLanes - 1);
    uint32_t raw[N / 2];
#pragma unroll
    for (int i = 0; i < N / 8; ++i) raw[4 * i] = x[i].x, raw[4 * i + 1] = x[i].y, raw[4 * i + 2] = x[i].z, raw[4 * i + 3] = x[i].w;
    // magnitudes as whole numbers: infinities are above all numbers, and NaN above those
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) top2 = __vmaxu2(top2, raw[i] & 0x7fff7fffu);
    unsigned top = max(top2 & 0xffffu, top2 >> 16);
#pragma unroll
    for (int o = 1; o < kGroup; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
    unsigned most = top;
#pragma unroll
    for (int o = kGroup; o < kLanes; o *= 2) most = max(most, __shfl_xor_sync(kFull, most, o));
    int E = most >> 7;
    const bool bad = E > kMostExponent, none = E < kLeastExponent;
    if (bad || none) E = kLeastExponent;
    // r to four significant bits, ties to even.  A quotient of 8 bits by 7 that is halfway
    // between two of them has to be found as such; x (1 / 7) is within an ulp of it, and
    // any other quotient 2^11 ulps away: so to multiples of 16 ulps first.
    uint32_t bits = __float_as_uint(__uint_as_float(top << 16) * power_of(256 - E) * (1.f / 7.f));
    bits = (bits + 8u) & ~15u;
    bits = (bits + 0x7ffffu + ((bits >> 20) & 1u)) & 0xfff00000u;
    bits = bad || none ? 0x38800000u : max(bits, 0x38800000u);         // (at least 2^-14)
    // Likewise x / s, halfway between two codes: x (1 / s) is within 2^-19 of it, while
    // quotients of 8 by 4 bits that are not halfway are 2^-10 away: the first sum rounds to
    // multiples of 2^-12, the second to whole numbers, which start at bit 0 of y.  They
    // are 1 to 15 without a bound, as 7 (1 + 2^-4) rounds to 7.
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__uint_as_float(bits) * power_of(E - 2)));
    uint32_t word[N / 8];
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
        word[k] = 0u - 0x4b400000u * 0x11111111u;            // (what all the ys add but for their codes)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t two = raw[4 * k + i / 2];
            const float v = __uint_as_float(i & 1 ? two & 0xffff0000u : two << 16);
            word[k] += __float_as_uint(__fadd_rn(fmaf(v, inv, 0x1.8p11f), 0x1.8p23f + 8.f - 0x1.8p11f)) << (4 * i);
        }
        if (bad || none) word[k] = 0x88888888u;
    }
    const int i = w / kGroup, t = w % kGroup;
    uint8_t* to = at.codes_at(n);
    int step = 4 * kI;                           // (bytes to the next word)
    if (kv) {
        // lanes of two groups trade half of their runs of four, so that each writes words:
        // the first half of the runs of the even group and the next, and the second half
        const bool odd = i & 1;
        const uint32_t mine = N == 8 ? (odd ? word[0] >> 16 : word[0] & 0xffffu) : word[odd ? N / 8 - 1 : 0];
        const uint32_t theirs = N == 8 ? (odd ? word[0] & 0xffffu : word[0] >> 16) : word[odd ? 0 : N / 8 - 1];
        const uint32_t got = __shfl_xor_sync(kFull, theirs, kGroup), first = odd ? got : mine, second = odd ? mine : got;
        word[0] = __byte_perm(first, second, 0x5410);
        if (N == 16) word[N / 8 - 1] = __byte_perm(first, second, 0x7632);
        if (odd) to += N / 4 * kI - 2;
        step = 2 * kI;
    }
    if (!out) return;
#pragma unroll
    for (int k = 0; k < N / 8; ++k) *reinterpret_cast<uint32_t*>(to + k * step) = word[k];
    if (t == 0) *at.ratio_at(n) = uint8_t((bits >> 20) - (112u << 3));
    if (w == 0) *at.exponent_at(n) = uint8_t(bad ? kBadExponent : E);
}

// What N elements are held as (a value's words still as they lie, for two groups).
template <int N>
struct Held {
    uint32_t word[N / 8];
    uint8_t ratio, exponent;
};

template <int D, int N>
__device__ __forceinline__ Held<N> read(const Place<D>& at, int n, int kv) {
    constexpr int kI = D / 32;
    Held<N> x;
    const uint8_t* codes = at.codes_at(n);
    if (kv && N == 8) {
        x.word[0] = *reinterpret_cast<const uint16_t*>(codes) | uint32_t(*reinterpret_cast<const uint16_t*>(codes + 2 * kI)) << 16;
    } else {
        const bool odd = threadIdx.x / (32 / N) & 1;
        if (kv && odd) codes += N / 4 * kI - 2;
#pragma unroll
        for (int k = 0; k < N / 8; ++k) x.word[k] = *reinterpret_cast<const uint32_t*>(codes + k * (kv ? 2 : 4) * kI);
    }
    x.ratio = *at.ratio_at(n);
    x.exponent = *at.exponent_at(n);
    return x;
}

// Lanes of two groups have read half of the runs of both, as they wrote them.
template <int N>
__device__ __forceinline__ void trade(Held<N>& x, int kv) {
    if constexpr (N == 16) {
        if (!kv) return;
        const bool odd = threadIdx.x / (32 / N) & 1;
        const uint32_t lo = __byte_perm(x.word[0], x.word[1], 0x5410), hi = __byte_perm(x.word[0], x.word[1], 0x7632);
        const uint32_t got = __shfl_xor_sync(kFull, odd ? lo : hi, 32 / N);
        x.word[0] = odd ? got : lo;
        x.word[1] = odd ? hi : got;
    }
}

template <int N>
__device__ __forceinline__ uint4 values_of(const Held<N>& x, int k) {
    // c as bf16 is (128 + n) - 136, and c s, of three bits by four, is exact
    const uint32_t scale = x.exponent == kBadExponent ? 0x7fffu : (uint32_t(x.ratio) + (112u << 3) << 4) + uint32_t(x.exponent - 129) * 128u;
    const uint32_t s2 = scale * 0x10001u, k136 = 0xc308c308u;
    uint32_t pair[4], out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // elements j and j + 4
        const uint32_t n = ((x.word[k] >> (4 * j)) & 0x000f000fu) | 0x43004300u;
        const __nv_bfloat162 c = __hadd2(reinterpret_cast<const __nv_bfloat162&>(n), reinterpret_cast<const __nv_bfloat162&>(k136));
        const __nv_bfloat162 y = __hmul2(c, reinterpret_cast<const __nv_bfloat162&>(s2));
        pair[j] = reinterpret_cast<const uint32_t&>(y);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = __byte_perm(pair[2 * (j & 1)], pair[2 * (j & 1) + 1], j < 2 ? 0x5410 : 0x7632);
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// A warp takes up to 32 tokens, whose places its lanes find at once, and as many heads of
// K or of V as fill its lanes.  N rows are on their way together: those to store from before
// the first's place is known, and another when one is rounded.
template <int D, bool Store, int N, int E>
__global__ void __launch_bounds__(kThreads) rows_kernel(PageLayer c, PageRows s, Rows x, int per_warp, unsigned kinds) {
    wait_for_previous();
    constexpr int kLanes = D / E, kHeads = 32 / kLanes;
    const unsigned group = blockIdx.x / kinds, kind = blockIdx.x - group * kinds;
    const int kv = kind >= kinds / 2, lane = threadIdx.x & 31, head = int(kind - kv * (kinds / 2)) * kHeads + lane / kLanes;
    const long first = (long(group) * (kThreads / 32) + threadIdx.x / 32) * per_warp;
    if (first >= s.rows) return;
    const int n = int(min(long(per_warp), s.rows - first));
    const bool mine = head < c.hkv;
    const long token = kv ? x.v_token : x.k_token;
    const __nv_bfloat16* p = (kv ? x.v : x.k) + (mine ? head : 0) * (kv ? x.v_head : x.k_head) + E * (lane & (kLanes - 1)) + first * token;
    const Lane<D, E> at(c, kv, mine ? head : 0);
    auto write = [&](int row, const Held<E>& x) {
#pragma unroll
        for (int k = 0; k < E / 8; ++k) reinterpret_cast<uint4*>(const_cast<__nv_bfloat16*>(p) + row * token)[k] = values_of(x, k);
    };
    uint4 data[N][E / 8];
    auto fetch = [&](int i, int from) {
#pragma unroll
        for (int k = 0; k < E / 8; ++k) data[i][k] = reinterpret_cast<const uint4*>(p + min(from + i, n - 1) * token)[k];
    };
    if (Store)
#pragma unroll
        for (int i = 0; i < N; ++i) fetch(i, 0);
    int slot = 0;
    const int page = places_of(c, s, int(first), n, &slot);
    for (int from = 0; from < n; from += N) {
        // rows of one page, one behind the other, are a constant apart
        const int page0 = __shfl_sync(kFull, page, from), slot0 = __shfl_sync(kFull, slot, from);
        const bool run = N > 1 && __all_sync(kFull, lane < from || lane >= from + N || (page == page0 && slot == slot0 + lane - from)) &&
                         page0 >= 0;
        const Place<D> first_at(at, max(page0, 0), page0 < 0 ? 0 : slot0);
        if (run) {
            if (Store) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    quantise_and_store<D, E>(first_at, i, data[i], kv, mine);
                    if (from + N < n) fetch(i, from + N);
                }
            } else {
                Held<E> held[N];
#pragma unroll
                for (int i = 0; i < N; ++i) held[i] = read<D, E>(first_at, i, kv);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    trade(held[i], kv);
                    if (mine) write(from + i, held[i]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int to = __shfl_sync(kFull, page, (from + i) & 31), in = __shfl_sync(kFull, slot, (from + i) & 31);
                const Place<D> place(at, max(to, 0), to < 0 ? 0 : in);
                if (Store) {
                    quantise_and_store<D, E>(place, 0, data[i], kv, mine && to >= 0);
                    if (from + N < n) fetch(i, from + N);
                } else {
                    // (no place: codes of 0, or a row of NaN)
                    Held<E> x = read<D, E>(place, 0, kv);
                    trade(x, kv);
                    if (to < 0) {
#pragma unroll
                        for (int k = 0; k < E / 8; ++k) x.word[k] = to == -1 ? 0x88888888u : 0u;
                        x.exponent = to == -1 ? 127 : kBadExponent;
                    }
                    if (mine && to > -3) write(from + i, x);
                }
            }
        }
    }
}

constexpr int kPairs = 448;     // pages copied by a launch: their numbers are its parameters

struct Copies {
    int src[kPairs], dst[kPairs];
};

// A block copies one page of one layer; an array's part is `bytes` long.
struct Part {
    uint8_t* base;
    unsigned bytes;
};

__global__ void __launch_bounds__(kCopying) copy_kernel(Part a, Part b, Part e, int pages, const __grid_constant__ Copies copies) {
    wait_for_previous();
    const int src = copies.src[blockIdx.x], dst = copies.dst[blockIdx.x];
    const Part parts[3] = {a, b, e};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const size_t layer = size_t(blockIdx.y) * pages, n = parts[i].bytes;
        const uint4* from = reinterpret_cast<const uint4*>(parts[i].base + (layer + src) * n);
        uint4* to = reinterpret_cast<uint4*>(parts[i].base + (layer + dst) * n);
#pragma unroll 4
        for (unsigned j = threadIdx.x; j < n / 16; j += kCopying) to[j] = from[j];
    }
}

// The kernel of a call: N rows on their way, E elements of each to a lane.
template <bool Store, int N, int E>
auto kernel_of(int d) {
    return d == 64 ? rows_kernel<64, Store, N, E> : d == 128 ? rows_kernel<128, Store, N, E> : rows_kernel<256, Store, N, E>;
}

template <bool Store>
int rows(const PageLayer& c, const PageRows& s, const Rows& x, int d, cudaStream_t stream) {
    // Tokens to a warp: as many as leave each of the 152 SMs some sixteen warps; a lone one
    // has the shortest chain of loads.
    auto kinds_of = [&](int each) { return 2L * ((c.hkv * d + 32 * each - 1) / (32 * each)); };
    auto tokens_of = [&](long kinds) { return s.rows / 16 * kinds >= 152 * 32 ? 16 : s.rows / 8 * kinds >= 152 * 16 ? 8 : 1; };
    // Sixteen elements to a lane halve what a row's scales cost, where a warp's lanes are
    // filled by a row of all heads.  Loads of more than a token to a warp are better off
    // with eight (35k tokens of 8 heads of 128: 41 us for 43; 512: 8.2 with sixteen for 10.1).
    const bool wide = c.hkv * d >= 1024 && (Store || tokens_of(kinds_of(8)) == 1);
    const long kinds = kinds_of(wide ? 16 : 8);
    const int per_warp = tokens_of(kinds);
    const long blocks = (s.rows + kThreads / 32L * per_warp - 1) / (kThreads / 32L * per_warp) * kinds;
    if (blocks >= 1L << 31) return int(cudaErrorInvalidValue);
    auto kernel = per_warp > 1 ? kernel_of<Store, 8, 8>(d) : kernel_of<Store, 1, 8>(d);
    if (wide) kernel = kernel_of<Store, 1, 16>(d);
    if constexpr (Store)
        if (wide && per_warp > 1) kernel = kernel_of<Store, 4, 16>(d);
    return dependent(kernel, dim3(unsigned(blocks)), kThreads, 0, stream, c, s, x, per_warp, unsigned(kinds));
}

}  // namespace
}  // namespace decoder

using namespace decoder;

// Rows k, v [rows][hkv][d] (each with its strides, token and head) into the layer's
// pages (out 0), or out of them (out 1).
extern "C" int decoder_page_rows(int out, const PageCache* cache, int layer, const void* k, long k_token, long k_head, const void* v,
                                 long v_token, long v_head, const void* table, const void* starts, const void* lengths, int width, int batch,
                                 int rows_, void* stream) {
    if (!cache->valid() || layer < 0 || layer >= cache->layers || width < 1 || batch < 1 || rows_ < 1) return int(cudaErrorInvalidValue);
    const PageLayer c = cache->layer(layer);
    const PageRows s = {static_cast<const int*>(table), static_cast<const int*>(starts), static_cast<const int*>(lengths), width, batch, rows_};
    const Rows x = {static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v), k_token, k_head, v_token, v_head};
    return out ? rows<false>(c, s, x, cache->d, static_cast<cudaStream_t>(stream))
               : rows<true>(c, s, x, cache->d, static_cast<cudaStream_t>(stream));
}

// What pages to copy are refused for: 1, there is no such page; 2, one is written twice, or
// written and read; 3, no memory to find out.
extern "C" int decoder_page_copy_refused(const int* src, const int* dst, int n, int pages) {
    for (int i = 0; i < n; ++i)
        if (src[i] < 0 || src[i] >= pages || dst[i] < 0 || dst[i] >= pages) return 1;
    if (n > pages) return 2;
    // what is written, hashed into at least twice the places (2^32 over the golden ratio)
    int bits = 6;
    while ((1L << bits) < 2L * n) ++bits;
    int few[512], *const places = bits <= 9 ? few : static_cast<int*>(std::malloc(sizeof(int) << bits));
    if (!places) return 3;
    std::fill(places, places + (1L << bits), -1);
    auto place_of_page = [&](int page) {
        uint32_t at = uint32_t(page) * 2654435769u >> (32 - bits);
        while (places[at] >= 0 && places[at] != page) at = (at + 1) & ((1u << bits) - 1);
        return places + at;
    };
    int refused = 0;
    for (int i = 0; i < n && !refused; ++i) {
        int* const at = place_of_page(dst[i]);
        refused = *at >= 0 ? 2 : 0;
        *at = dst[i];
    }
    for (int i = 0; i < n && !refused; ++i) refused = *place_of_page(src[i]) >= 0 ? 2 : 0;
    if (places != few) std::free(places);
    return refused;
}

// Pages src[i] to dst[i] of all layers; no dst is another's, or a src.
extern "C" int decoder_page_copy(const PageCache* cache, const int* src, const int* dst, int n, void* stream) {
    if (!cache->valid() || cache->layers > 65535 || n < 0) return int(cudaErrorInvalidValue);
    for (int i = 0; i < n; ++i)
        if (src[i] < 0 || src[i] >= cache->pages || dst[i] < 0 || dst[i] >= cache->pages) return int(cudaErrorInvalidValue);
    const unsigned rows = unsigned(cache->hkv) << cache->log_page, d = unsigned(cache->d);      // (rows of keys, and as many of values)
    const Part a = {cache->codes, rows * d}, b = {cache->ratios, rows * (d / 16)}, e = {cache->exponents, rows * 2};
    for (int at = 0; at < n; at += kPairs) {
        const int m = n - at < kPairs ? n - at : kPairs;
        Copies copies;
        for (int i = 0; i < m; ++i) copies.src[i] = src[at + i], copies.dst[i] = dst[at + i];
        const int rc = dependent(copy_kernel, dim3(unsigned(m), unsigned(cache->layers)), kCopying, 0, static_cast<cudaStream_t>(stream), a, b, e,
                                 cache->pages, copies);
        if (rc) return rc;
    }
    return 0;
}
