// Rows into the pages of a cache in 4 bits and out of them, and pages copied.
//
// All three are bound by HBM: a row of 128 elements is 256 bytes in bf16 and 69 in a
// page, and a copied page is read and written once.  Small calls are latency: the
// search for a row's sequence, its page, the access.
#include "pages.cuh"

#include "decoder.h"

namespace decoder {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kFull = 0xffffffffu;

// Where token `row` lies: its sequence b (starts[b] <= row < starts[b + 1]), or -1
// behind the last.  32 places at a time: a look or two for a batch.
__device__ int sequence_of(const PageRows& s, int row) {
    const int lane = threadIdx.x & 31;
    if (row >= s.starts[s.batch] || row < s.starts[0]) return -1;
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

// The token's page and slot.  -1: no place (a position before the first), -2: a page
// that is none of the cache's.
__device__ __forceinline__ int place_of(const PageLayer& c, const PageRows& s, int b, int row, int* slot) {
    const int first = s.starts[b], at = s.lengths[b] - (s.starts[b + 1] - first) + (row - first);
    if (at < 0) return -1;
    const int i = at >> c.log_page;
    if (i >= s.width) return -2;
    const int page = s.table[size_t(b) * s.width + i];
    *slot = at & ((1 << c.log_page) - 1);
    return page < 0 || page >= c.pages ? -2 : page;
}

struct Rows {
    const __nv_bfloat16 *k, *v;     // (written by a load)
    long k_token, k_head, v_token, v_head;
};

// Eight elements of a row in each lane; D / 8 lanes to a row.
template <int D>
__device__ __forceinline__ void quantise_and_store(const PageLayer& c, uint4 x, int kv, int page, int head, int slot) {
    constexpr int kLanes = D / 8;
    const int w = threadIdx.x & (kLanes - 1);
    const uint32_t raw[4] = {x.x, x.y, x.z, x.w};
    // magnitudes as whole numbers: infinities are above all numbers, and NaN above those
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top2 = __vmaxu2(top2, raw[i] & 0x7fff7fffu);
    unsigned top = max(top2 & 0xffffu, top2 >> 16);
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    top = max(top, __shfl_xor_sync(kFull, top, 2));
    unsigned most = top;
#pragma unroll
    for (int o = 4; o < kLanes; o *= 2) most = max(most, __shfl_xor_sync(kFull, most, o));
    int E = most >> 7;
    const bool bad = E > kMostExponent, none = E < kLeastExponent;
    if (bad || none) E = kLeastExponent;
    // r to four significant bits, ties to even: the quotient is either halfway, and
    // then exact, or further than 2^-11 from it
    float ratio = bad || none ? 0.f : __fdiv_rn(__uint_as_float(top << 16) * power_of(256 - E), 7.f);
    uint32_t bits = __float_as_uint(fmaxf(ratio, 0x1p-14f));
    bits = (bits + 0x7ffffu + ((bits >> 20) & 1u)) & 0xfff00000u;
    // x / s halfway between two codes has to be found as such, and x (1 / s) is within
    // 2^-20 of it, while quotients of 8 by 4 bits that are not halfway are 2^-10 away:
    // the first sum rounds to multiples of 2^-12, the second of 1
    const float inv = __frcp_rn(__uint_as_float(bits) * power_of(E - 2));
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
        float y = __fadd_rn(fmaf(v, inv, 0x1.8p11f), 0x1.8p23f + 8.f - 0x1.8p11f);
        y = fminf(fmaxf(y, 0x1.8p23f + 1.f), 0x1.8p23f + 15.f);
        word |= (__float_as_uint(y) & 15u) << (4 * i);
    }
    if (bad || none) word = 0x88888888u;
    const int i = w >> 2, t = w & 3;
    int at = t * (D / 32) + i;
    if (kv) {
        // lanes of two groups trade their runs of four, so that each writes a word
        const uint32_t got = __shfl_xor_sync(kFull, i & 1 ? word & 0xffffu : word >> 16, 4);
        word = i & 1 ? (word & 0xffff0000u) | got : (word & 0xffffu) | (got << 16);
        at = (2 * t + (i & 1)) * (D / 64) + (i >> 1);
    }
    if (page < 0) return;
    const size_t row = page_row(c, page, kv, head, slot);
    reinterpret_cast<uint32_t*>(c.codes + row * (D / 2))[at] = word;
    if (t == 0) c.ratios[row * (D / 32) + i] = uint8_t((bits >> 20) - (112u << 3));
    if (w == 0) c.exponents[exponent_row(c, page, head, slot) * 2 + kv] = uint8_t(bad ? kBadExponent : E);
}

template <int D>
__device__ __forceinline__ uint4 loaded(const PageLayer& c, int kv, int page, int head, int slot) {
    constexpr int kLanes = D / 8;
    const int w = threadIdx.x & (kLanes - 1), i = w >> 2, t = w & 3;
    if (page < 0) {
        const uint32_t x = page == -1 ? 0u : 0x7fff7fffu;
        return make_uint4(x, x, x, x);
    }
    const size_t row = page_row(c, page, kv, head, slot);
    const uint8_t* codes = c.codes + row * (D / 2);
    uint32_t word;
    if (kv) {
        const uint16_t* runs = reinterpret_cast<const uint16_t*>(codes);
        word = runs[2 * t * (D / 32) + i] | uint32_t(runs[(2 * t + 1) * (D / 32) + i]) << 16;
    } else {
        word = reinterpret_cast<const uint32_t*>(codes)[t * (D / 32) + i];
    }
    const int E = c.exponents[exponent_row(c, page, head, slot) * 2 + kv];
    const float ratio = __uint_as_float((uint32_t(c.ratios[row * (D / 32) + i]) + (112u << 3)) << 20);
    const float s = E == kBadExponent ? __int_as_float(0x7fffffff) : ratio * power_of(E - 2);
    uint32_t out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // (exact: three bits by four)
        const float a = (float(word >> (8 * j) & 15u) - 8.f) * s, b = (float(word >> (8 * j + 4) & 15u) - 8.f) * s;
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        out[j] = reinterpret_cast<const uint32_t&>(p);
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// A warp takes a run of tokens and as many heads of K or of V as fill its lanes.
template <int D, bool Store>
__global__ void __launch_bounds__(kThreads) rows_kernel(PageLayer c, PageRows s, Rows x, int per_warp) {
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
    const int slices = (c.hkv + kHeads - 1) / kHeads;
    const long warp = (long(blockIdx.x) * kThreads + threadIdx.x) / 32;
    const int kind = int(warp % (2 * slices)), kv = kind / slices;
    const int head = (kind - kv * slices) * kHeads + (threadIdx.x & 31) / kLanes, w = threadIdx.x & (kLanes - 1);
    const long first = warp / (2 * slices) * per_warp;
    if (first >= s.rows) return;
    const int last = int(min(long(s.rows), first + per_warp));
    const bool mine = head < c.hkv;
    const long token = kv ? x.v_token : x.k_token;
    const __nv_bfloat16* p = (kv ? x.v : x.k) + (mine ? head : 0) * (kv ? x.v_head : x.k_head) + 8 * w;
    int b = sequence_of(s, int(first));
    for (int row = int(first); row < last; ++row) {
        uint4 data = {};
        const bool out = b < 0;
        if (Store && mine) data = *reinterpret_cast<const uint4*>(p + row * token);
        if (out) return;
        while (b < s.batch && s.starts[b + 1] <= row) ++b;
        if (b >= s.batch) return;
        int slot = 0, page = place_of(c, s, b, row, &slot);
        if (Store) {
            quantise_and_store<D>(c, data, kv, mine ? page : -1, head, slot);
        } else if (mine) {
            data = loaded<D>(c, kv, page, head, slot);
            *reinterpret_cast<uint4*>(const_cast<__nv_bfloat16*>(p) + row * token) = data;
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

__global__ void __launch_bounds__(kThreads) copy_kernel(Part a, Part b, Part e, int pages, const __grid_constant__ Copies copies) {
    const int src = copies.src[blockIdx.x], dst = copies.dst[blockIdx.x];
    const Part parts[3] = {a, b, e};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const size_t layer = size_t(blockIdx.y) * pages, n = parts[i].bytes;
        const uint4* from = reinterpret_cast<const uint4*>(parts[i].base + (layer + src) * n);
        uint4* to = reinterpret_cast<uint4*>(parts[i].base + (layer + dst) * n);
#pragma unroll 4
        for (unsigned j = threadIdx.x; j < n / 16; j += kThreads) to[j] = from[j];
    }
}

template <bool Store>
int rows(const PageLayer& c, const PageRows& s, const Rows& x, int d, cudaStream_t stream) {
    const int heads = 32 / (d / 8);
    const long kinds = 2L * ((c.hkv + heads - 1) / heads);
    const int per_warp = 1;
    const long warps = (s.rows + per_warp - 1) / per_warp * kinds;
    const long blocks = (warps * 32 + kThreads - 1) / kThreads;
    if (blocks >= 1L << 31) return int(cudaErrorInvalidValue);
    const auto kernel = d == 64 ? rows_kernel<64, Store> : d == 128 ? rows_kernel<128, Store> : rows_kernel<256, Store>;
    kernel<<<unsigned(blocks), kThreads, 0, stream>>>(c, s, x, per_warp);
    return int(cudaGetLastError());
}

bool takes(int pages, int hkv, int d, int log_page, int width, int batch, int rows) {
    return pages >= 1 && hkv >= 1 && hkv <= 1024 && (d == 64 || d == 128 || d == 256) && log_page >= 4 && log_page <= 8 && width >= 1 &&
           batch >= 1 && rows >= 1;
}

}  // namespace
}  // namespace decoder

using namespace decoder;

// Rows k, v [rows][hkv][d] (strides: token and head of k, then of v) into the layer's
// pages (out 0), or out of them (out 1).
extern "C" int decoder_page_rows(int out, void* codes, void* ratios, void* exponents, int pages, int hkv, int d, int log_page,
                                 const void* k, const void* v, const long* strides, const void* table, const void* starts,
                                 const void* lengths, int width, int batch, int rows_, void* stream) {
    if (!takes(pages, hkv, d, log_page, width, batch, rows_)) return int(cudaErrorInvalidValue);
    const PageLayer c = {static_cast<uint8_t*>(codes), static_cast<uint8_t*>(ratios), static_cast<uint8_t*>(exponents), pages, hkv, log_page};
    const PageRows s = {static_cast<const int*>(table), static_cast<const int*>(starts), static_cast<const int*>(lengths), width, batch, rows_};
    const Rows x = {static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v), strides[0], strides[1], strides[2], strides[3]};
    return out ? rows<false>(c, s, x, d, static_cast<cudaStream_t>(stream)) : rows<true>(c, s, x, d, static_cast<cudaStream_t>(stream));
}

// Pages src[i] to dst[i] of all layers; no dst is another's, or a src.
extern "C" int decoder_page_copy(void* codes, void* ratios, void* exponents, int layers, int pages, int hkv, int d, int log_page,
                                 const int* src, const int* dst, int n, void* stream) {
    if (!takes(pages, hkv, d, log_page, 1, 1, 1) || layers < 1 || layers > 65535 || n < 0) return int(cudaErrorInvalidValue);
    const unsigned rows = unsigned(hkv) << log_page;        // of keys, and as many of values
    const Part a = {static_cast<uint8_t*>(codes), rows * unsigned(d)}, b = {static_cast<uint8_t*>(ratios), rows * unsigned(d / 16)},
               e = {static_cast<uint8_t*>(exponents), rows * 2};
    for (int at = 0; at < n; at += kPairs) {
        const int m = n - at < kPairs ? n - at : kPairs;
        Copies copies;
        for (int i = 0; i < m; ++i) {
            copies.src[i] = src[at + i];
            copies.dst[i] = dst[at + i];
            if (src[at + i] < 0 || src[at + i] >= pages || dst[at + i] < 0 || dst[at + i] >= pages) return int(cudaErrorInvalidValue);
        }
        copy_kernel<<<dim3(unsigned(m), unsigned(layers)), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a, b, e, pages, copies);
        const int rc = int(cudaGetLastError());
        if (rc) return rc;
    }
    return 0;
}
