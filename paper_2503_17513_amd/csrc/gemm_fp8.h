// What the kernels of the e4m3 products share.
#pragma once
#include "gemm_tile.h"

namespace pme {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ float silu(float v) { return v / (1.f + expf(-v)); }

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
    int tiles_m, tiles_n, xcd_gm;
};

}  // namespace
}  // namespace pme
