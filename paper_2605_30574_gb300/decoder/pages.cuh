// The paged key/value cache in 4 bits: what its kernels share.
//
// A row is one token's key or value of one head, D elements in groups of 32.  With A
// its largest magnitude and E = floor(log2 A), a group's scale is s = r 2^(E - 2),
// r = (the group's largest magnitude) 2^(2 - E) / 7 to four significant bits (at least
// 2^-14), and a value is c s, c = x / s to a whole number between -7 and 7 (ties to
// even, both).  A power of two to a row lets values of any size be operands in fp16,
// and four bits of r let c s, of seven, be exact in bf16.  Rows with A below 2^-100 are
// zero (E = -100), those with A of 2^100 and more, or not finite, are NaN (byte 255).
//
// A layer of the cache is three arrays:
//   codes      [page][2][head][slot][D / 2]   c + 8 in a nibble, the low one first
//   ratios     [page][2][head][slot][D / 32]  bits 14 to 7 of r in fp16
//   exponents  [page][head][slot][2]          E + 127
// keys before values.  Within a row nibbles are ordered for the lanes that multiply
// them (page_attention.cu), so that each reads what it needs of a row at once: word
// t + 4 i of a key (8 elements of group i) lies at place t D / 32 + i, the run of four
// elements g + 8 i of a value (of group i) at place g D / 32 + i.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace decoder {

struct PageLayer {
    uint8_t *codes, *ratios, *exponents;
    int pages, hkv, log_page;
};

// A cache as its owner describes it, once for all calls.
struct PageCache {
    uint8_t *codes, *ratios, *exponents;
    int layers, pages, hkv, d, log_page;

    bool valid() const {
        return layers >= 1 && pages >= 1 && hkv >= 1 && hkv <= 1024 && (d == 64 || d == 128 || d == 256) && log_page >= 4 && log_page <= 8;
    }
    PageLayer layer(int i) const {
        const size_t rows = (size_t(pages) * hkv << log_page) * size_t(i);       // (of keys, or values, of the layers before)
        return {codes + rows * d, ratios + rows * (d / 16), exponents + rows * 2, pages, hkv, log_page};
    }
};

// Sequences: their newest tokens are rows starts[b] to starts[b + 1] of what is
// stored, loaded or attends, and end at lengths[b]; their pages are table[b].
struct PageRows {
    const int *table, *starts, *lengths;
    int width, batch, rows;     // (pages to a sequence, sequences, rows there are)
};

constexpr int kBadExponent = 255;       // a row of NaN
constexpr int kLeastExponent = 27;      // 2^-100, biased
constexpr int kMostExponent = 226;

// 2^(biased - 127).
__device__ __forceinline__ float power_of(int biased) { return __int_as_float(biased << 23); }

// Every kernel is launched as a programmatic dependent of what precedes it on the stream:
// set up while that still runs, it waits for all of it before it reads or writes.
__device__ __forceinline__ void wait_for_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <class... Params, class... Given>
inline int dependent(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t stream, const Given&... given) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return int(cudaLaunchKernelEx(&cfg, kernel, given...));
}

}  // namespace decoder
