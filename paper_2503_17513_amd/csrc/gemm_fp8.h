// What the kernels of the e4m3 products share.
#pragma once
#include "gemm_tile.h"

namespace pme {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

// v / (1 + e^-v) in ten instructions (a library exponential and a quotient are some thirty, and code that runs once comes from memory).
// e^-v = 2^h (1 + l ln 2), h the rounded product of -v and log2 e and l what the rounding left out of it.  Two roundings of an ulp, the
// exponential's and the reciprocal's, and three of half an ulp (4 2^-24 at most over 4 million values).  Below -87.3, where 1 / (1 + e^-v) is
// no normal number, 0 in place of less than 2^-119.
__device__ __forceinline__ float silu(float v) {
    const float w = __builtin_amdgcn_fmed3f(v, -88.7f, 128.f), h = w * -1.44269502f;
    const float l = fmaf(w, -1.92596303e-8f, fmaf(w, -1.44269502f, -h)), p = __builtin_amdgcn_exp2f(h);
    return v * __builtin_amdgcn_rcpf(1.f + fmaf(p, l * 0.693147181f, p));
}

// As dma16, from a buffer: dwords beyond its end arrive as zeros.
__device__ __forceinline__ void dma16_buffer(u32x4 rsrc, uint32_t voff, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds_base) : "memory");
}
// Buffer descriptor of `bytes` bytes at p.
__device__ __forceinline__ u32x4 buffer_of(const void* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xFFFFu, bytes, 0x00027000u};
}

// 16 bytes a lane from a buffer to LDS place lds + AT; dwords beyond the buffer's end arrive as zeros.  All of the offset is in the vector
// register: the range check leaves a scalar offset out.
template <int AT> __device__ __forceinline__ void dma16_to(u32x4 rsrc, uint32_t voff, uint32_t lds) {
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds), "n"(AT) : "memory", "scc");
}

// LDS swizzle of rows of 128 bytes of which 16 are read together, 16 bytes each: chunk c of row r sits at position c ^ swz16(r).
__device__ __forceinline__ int swz16(int r) { return (r >> 1) & 7; }

struct Fp8TileArgs {
    const uint8_t* qx;
    const float* sx;
    const uint8_t* qw;
    const float* sw;
    const uint8_t* qu;
    const float* su;
    int T, N, K;
    uint16_t* y;
    int64_t ldo;
    int tiles_m, tiles_n, band;
};

// Workgroup -> output tile.  Workgroups are dealt round-robin to the 8 XCDs, each with an L2 of its own: XCD x takes a contiguous share of
// the tiles in an order that walks bands of `band` rows of tiles column by column, so that what it works on at a time is a block of about
// as many rows of tokens as of weights.
__device__ __forceinline__ void fp8_tile(int wg, int tiles_m, int tiles_n, int band, int& tm, int& tn) {
    const int n = tiles_m * tiles_n, x = wg & 7, t = x * (n >> 3) + min(x, n & 7) + (wg >> 3);
    const int b = t / (band * tiles_n), first = b * band, rows = min(band, tiles_m - first), r = t - first * tiles_n;
    tm = first + r % rows;
    tn = r / rows;
}
// The band of tiles of `rows` tokens and `weights` weights, `resident` of them on a compute unit at a time.
inline int fp8_band(int tiles_m, int tiles_n, int rows, int weights, int resident) {
    const int most = tiles_m * tiles_n / 8 + 1, c = most < 32 * resident ? most : 32 * resident;
    int band = 1;
    while (band < tiles_m && (band + 1) * band * rows <= c * weights) ++band;      // band * rows <= c / band * weights, to the nearer side
    return band;
}

}  // namespace
}  // namespace pme
