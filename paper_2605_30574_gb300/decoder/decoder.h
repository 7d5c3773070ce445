// Internal declarations of the decoder library.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

namespace decoder {

constexpr int kPlain = 0, kResid = 1, kSwiglu = 2;

// cuTensorMapEncodeTiled, by the driver's entry point (NULL: none).
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn();

// The current device's error word (see decoder_error).
unsigned* error_word();

// The fused projections of gemm.cu (see decoder_gemm) and the shapes they take.
bool gemm_takes(int M, int N, int K);
int gemm(int mode, const void* x, const void* w0, const void* w1, const void* h, void* y, int M, int N, int K,
         cudaStream_t stream);

// The shapes that attention with log sums and its gradients take: lengths whose
// row indices and grids stay within 32 bits.
inline bool attention_takes(long B, long Tq, long Tk, int Hq, int Hkv) {
    constexpr long kMax = 1L << 20;
    return B >= 1 && B <= 65536 && Tq >= 1 && Tq <= kMax && Tk >= 1 && Tk <= kMax && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 &&
           B * Hq <= 1L << 20 && (Tq + 127) / 128 * Hq * B < 1L << 27 && (Tk + 127) / 128 * Hkv * B < 1L << 27;
}

}  // namespace decoder
