// Products of e4m3 codes with a scale for each block of 128:
//
//   p[t][n] = sum_g sx[t][g] sw[n / 128][g] sum_{k in group g} qx[t][k] qw[n][k],   y = bf16(p),
//   gated:  y = bf16( p_g / (1 + e^-p_g) p_u )  of two weight matrices.
#include "gemm_tile.h"

#include <algorithm>

namespace pme {
namespace {

__device__ __forceinline__ float silu(float v) { return v / (1.f + expf(-v)); }

// Plain-ALU kernel, one thread per output: every shape, and the cross-check of the matrix-core kernels.
template <bool GATED>
__global__ void __launch_bounds__(256)
k_fp8_gemm_generic(const uint8_t* __restrict__ qx, const float* __restrict__ sx, const uint8_t* __restrict__ qw, const float* __restrict__ sw,
                   const uint8_t* __restrict__ qu, const float* __restrict__ su, int T, int N, int K, uint16_t* __restrict__ y, int64_t ldo) {
    const int n = blockIdx.x * 16 + (threadIdx.x & 15), groups = K / 128;
    if (n >= N) return;
    // blocks of 16 tokens: the grid's y extent is capped (65535), so a workgroup walks its share of them
    for (int64_t t = (int64_t)blockIdx.y * 16 + (threadIdx.x >> 4); t < T; t += (int64_t)gridDim.y * 16) {
        auto product = [&](const uint8_t* w, const float* s) {
            float sum = 0.f;
            for (int g = 0; g < groups; ++g) {
                const uint32_t* pa = reinterpret_cast<const uint32_t*>(qx + t * K + 128 * g);
                const uint32_t* pw = reinterpret_cast<const uint32_t*>(w + (int64_t)n * K + 128 * g);
                float inner = 0.f;
                for (int p = 0; p < 32; ++p) {
                    const int va = (int)pa[p], vw = (int)pw[p];
                    inner = fmaf(__builtin_amdgcn_cvt_f32_fp8(va, 0), __builtin_amdgcn_cvt_f32_fp8(vw, 0), inner);
                    inner = fmaf(__builtin_amdgcn_cvt_f32_fp8(va, 1), __builtin_amdgcn_cvt_f32_fp8(vw, 1), inner);
                    inner = fmaf(__builtin_amdgcn_cvt_f32_fp8(va, 2), __builtin_amdgcn_cvt_f32_fp8(vw, 2), inner);
                    inner = fmaf(__builtin_amdgcn_cvt_f32_fp8(va, 3), __builtin_amdgcn_cvt_f32_fp8(vw, 3), inner);
                }
                sum = fmaf(inner, sx[t * groups + g] * s[(int64_t)(n / 128) * groups + g], sum);
            }
            return sum;
        };
        float v = product(qw, sw);
        if constexpr (GATED) v = silu(v) * product(qu, su);
        y[t * ldo + n] = f32_to_bf16_bits(v);
    }
}

}  // namespace

pme_status launch_fp8_gemm_generic(const Fp8GemmArgs& a) {
    if (a.dry) {
        if (a.plan) *a.plan = a.qu ? "k_fp8_gemm_generic<true>" : "k_fp8_gemm_generic<false>";
        return PME_OK;
    }
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)std::min<int64_t>((a.T + 15) / 16, 65535)), block(256);
    if (a.qu)
        hipLaunchKernelGGL((k_fp8_gemm_generic<true>), grid, block, 0, a.stream, a.qx, a.sx, a.qw, a.sw, a.qu, a.su, (int)a.T, (int)a.N, (int)a.K, static_cast<uint16_t*>(a.y), a.ldy);
    else
        hipLaunchKernelGGL((k_fp8_gemm_generic<false>), grid, block, 0, a.stream, a.qx, a.sx, a.qw, a.sw, a.qu, a.su, (int)a.T, (int)a.N, (int)a.K, static_cast<uint16_t*>(a.y), a.ldy);
    return hip_status(hipGetLastError());
}

}  // namespace pme
