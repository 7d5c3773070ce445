// Attention over the pages of a cache in 4 bits: what its two kernels share.
//
// Both take their work off a line: every tile (rows of a sequence and a kv head) is so many
// stages of keys, the line is cut into even shares, whatever the sequences' lengths, and
// a tile that is cut leaves a state (m, l, O) of its rows on either side, which are joined
// in their order.
#pragma once

#include <cuda_fp16.h>

#include "../csrc/tc_ptx.cuh"
#include "pages.cuh"

namespace decoder {
namespace page {

using splice::tc::smem_u32;

constexpr unsigned kFull = 0xffffffffu;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1e30f;         // the reference of rows that have seen nothing

// A call.  Its scratch holds the states of tiles whose keys fall to several CTAs, and the
// few-row kernel's of those that fall to several warps.
struct Args {
    PageLayer c;
    PageRows s;
    const __nv_bfloat16* q;
    long q_token, q_head;
    __nv_bfloat16* out;
    int G, window;
    float scale;
    float *states, *joined; // of warps [each][columns][d + 4], and of CTAs [each][2][columns][d + 4]
    int4* begun;            // per CTA: the tile whose keys begin with it and go on
};

constexpr int kJoin = 128;              // threads of a CTA that joins states


__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

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

__device__ __forceinline__ void sts16(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void cp16(uint32_t to, const uint8_t* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// Rows' states joined, 8 lanes to a row: O for the reference m and the sum l, at D and
// D + 1.
template <int D>
struct State {
    static constexpr int kVec = D / 32;         // by four elements
    float m = kNone, l = 0.f;
    float4 o[kVec] = {};

    __device__ __forceinline__ void add(const float* from) {
        const int lane = threadIdx.x & 7;
        float4 y[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[i] = reinterpret_cast<const float4*>(from)[lane + 8 * i];
        const float2 ml = *reinterpret_cast<const float2*>(from + D);
        const float M = fmaxf(m, ml.x), f = ex2(m - M), fy = ex2(ml.x - M);
        m = M;
        l = l * f + ml.y * fy;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            o[i] = make_float4(o[i].x * f + y[i].x * fy, o[i].y * f + y[i].y * fy, o[i].z * f + y[i].z * fy, o[i].w * f + y[i].w * fy);
    }
    __device__ __forceinline__ void keep(float* to) const {
        const int lane = threadIdx.x & 7;
#pragma unroll
        for (int i = 0; i < kVec; ++i) reinterpret_cast<float4*>(to)[lane + 8 * i] = o[i];
        if (lane == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m, l);
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

// The row of out of a tile's row; a tile has kRows of P heads each.
template <int kRows>
__device__ __forceinline__ size_t row_of(const Args& A, const int4& info, int mine, int row) {
    const int r = (info.y & 0xffffff) * kRows + row, token = r / A.G;
    return (size_t(info.x + token) * A.c.hkv + (info.z & 0x3fffffff) + mine) * A.G + r - token * A.G;
}

// Joins the states of a tile whose keys went to several CTAs, its second state of the CTA
// that it begins in and the first of those behind: blocks take its rows in turn.
template <int D, int kRows, int P>
__global__ void __launch_bounds__(kJoin) join_kernel(const Args A) {
    constexpr int kEach = kJoin / 8, kCols = kRows * P;
    __shared__ __align__(16) float part[kEach][D + 4];
    wait_for_previous();
    const int group = threadIdx.x / 8;
    const int4 info = A.begun[blockIdx.x];
    if (info.x < 0) return;
    for (int col = blockIdx.y; col < kCols; col += gridDim.y) {
        if (col % kRows >= info.y >> 24) continue;
        State<D> st;
#pragma unroll 2
        for (int c = blockIdx.x + group; c <= info.w; c += kEach)
            st.add(A.joined + ((size_t(c) * 2 + (c == blockIdx.x ? 1 : 0)) * kCols + col) * (D + 4));
        st.keep(part[group]);
        __syncthreads();
        if (group == 0) {
            State<D> all;
            for (int k = 0; k < kEach && k <= info.w - int(blockIdx.x); ++k) all.add(part[k]);
            all.write(A.out + row_of<kRows>(A, info, col / kRows, col % kRows) * D);
        }
        __syncthreads();
    }
}

// Attention of many rows to a kv head (page_attention_rows.cu), of heads of 64 and 128, and
// its scratch, by the device's multiprocessors; errors come back as CUDA's.
int many_rows(const Args& a, int d, void* scratch, cudaStream_t stream);
cudaError_t many_rows_scratch(int d, long* bytes);

}  // namespace page
}  // namespace decoder
