// Products of e4m3 codes with a scale for each block of 128, for few tokens: memory-bound on the weights.
//
//   p[t][n] = sum_g sx[t][g] sw[n / 128][g] sum_{k in group g} qx[t][k] qw[n][k],   y = bf16(p), or gated bf16(silu(p_g) p_u).
//
// One workgroup owns 16 output channels (of both matrices where it is gated) and the whole of K; its waves split K into contiguous runs of
// blocks of 128, so that every weight byte is loaded exactly once, straight from HBM into registers, with several blocks of a wave in
// flight before the first use.  A block of 16 channels is two 16-byte loads a lane (lane = channel % 16 + 16 * part; 64 contiguous bytes of
// every channel a load) and one v_mfma_f32_16x16x128_f8f6f4 against the tokens' codes, whose sum is scaled into the wave's fp32
// accumulators.  The waves' partial tiles are added through LDS in the order of K.
// HALF: 8 channels, for at most 8 tokens.  Rows 8 .. 15 of the weight operand and columns 8 .. 15 of the token operand hold the next block
// of K of the same channels and tokens, so that both diagonal quarters of the instruction's result are partial sums and as many weight
// bytes enter each instruction; twice the workgroups share a narrow output.
#include "gemm_fp8.h"
#include <cstdlib>

namespace pme {
namespace {

template <int NW, int TG, int KB, bool GATED, bool HALF>
__global__ void __launch_bounds__(64 * NW)
k_fp8_gemm_decode(const uint8_t* __restrict__ qx, const float* __restrict__ sx, const uint8_t* __restrict__ qw, const float* __restrict__ sw,
                  const uint8_t* __restrict__ qu, const float* __restrict__ su, int T, int N, int K, uint16_t* __restrict__ y, int64_t ldo) {
    static_assert(!HALF || TG == 1, "8 tokens");
    constexpr int MATS = GATED ? 2 : 1, CHANNELS = HALF ? 8 : 16, SPAN = HALF ? 2 : 1;      // SPAN: blocks of K an instruction takes
    __shared__ f32x4 part[NW][MATS][64];
    // The wave's number is read into a scalar register, so that the conditions on its share of K are branches: a matrix
    // instruction takes no notice of the execution mask, and one that is only masked runs on registers nothing was loaded into.
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, kg = lane >> 4, sub = HALF ? r >> 3 : 0, rr = HALF ? r & 7 : r;
    const int n0 = blockIdx.x * CHANNELS, groups = K / 128, steps = (groups + SPAN - 1) / SPAN;
    const int S = (steps + NW - 1) / NW;               // this wave's: blocks (pairs) wave, wave + NW, ...
    const int64_t wrow = (int64_t)min(n0 + rr, N - 1) * K + kg * 16;
    const float* swr[MATS] = {sw + (int64_t)(n0 / 128) * groups};
    const uint8_t* qwr[MATS] = {qw + wrow};
    if constexpr (GATED) {
        swr[1] = su + (int64_t)(n0 / 128) * groups;
        qwr[1] = qu + wrow;
    }
    const uint8_t* xrow[TG];
    const float* sxr[TG];
#pragma unroll
    for (int g = 0; g < TG; ++g) {
        const int64_t t = min(16 * g + rr, T - 1);
        xrow[g] = qx + t * K + kg * 16;
        sxr[g] = sx + t * groups;
    }
    f32x4 acc[MATS][TG];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int g = 0; g < TG; ++g) acc[m][g] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 w[MATS][KB][2], x[TG][KB][2];
    float sc[TG][KB], sm[MATS][KB];
    // step c into slot i; a block beyond K is the last one again, with a scale of zero
    auto load = [&](auto ic, int c) {
        constexpr int i = decltype(ic)::value;
        const int kb = SPAN * (wave + NW * min(c, S - 1)) + sub, at = min(kb, groups - 1);
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) w[m][i][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(qwr[m] + (int64_t)at * 128 + 64 * h));
#pragma unroll
        for (int m = 0; m < MATS; ++m) sm[m][i] = swr[m][at];
#pragma unroll
        for (int g = 0; g < TG; ++g) {
#pragma unroll
            for (int h = 0; h < 2; ++h) x[g][i][h] = *reinterpret_cast<const u32x4*>(xrow[g] + (int64_t)at * 128 + 64 * h);
            sc[g][i] = kb < groups ? sxr[g][at] : 0.f;
        }
    };
    auto compute = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            const i32x8 wv = {(int)w[m][i][0][0], (int)w[m][i][0][1], (int)w[m][i][0][2], (int)w[m][i][0][3],
                              (int)w[m][i][1][0], (int)w[m][i][1][1], (int)w[m][i][1][2], (int)w[m][i][1][3]};
#pragma unroll
            for (int g = 0; g < TG; ++g) {
                const i32x8 xv = {(int)x[g][i][0][0], (int)x[g][i][0][1], (int)x[g][i][0][2], (int)x[g][i][0][3],
                                  (int)x[g][i][1][0], (int)x[g][i][1][1], (int)x[g][i][1][2], (int)x[g][i][1][3]};
                const f32x4 t = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                const float p = sc[g][i] * sm[m][i];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][g][e] = fmaf(t[e], p, acc[m][g][e]);
            }
        }
    };
    static_for<KB>([&](auto ic) { load(ic, decltype(ic)::value); });
    int c = 0;
    for (; c + KB < S; c += KB)
        static_for<KB>([&](auto ic) {
            compute(ic);
            load(ic, c + KB + decltype(ic)::value);
        });
    static_for<KB>([&](auto ic) {
        if (c + decltype(ic)::value < S) compute(ic);
    });
    // one group at a time through the reduction buffer
#pragma unroll
    for (int g = 0; g < TG; ++g) {
        if (g > 0) __syncthreads();                     // the previous group has been read
#pragma unroll
        for (int m = 0; m < MATS; ++m) part[wave][m][lane] = acc[m][g];
        __syncthreads();
        // element tid = 4 * lane' + e of the 16 x 16 tile: channel 4 * (lane' / 16) + e, token lane' % 16 (HALF: of the first quarter,
        // lanes' tokens 0 .. 7 and parts 0, 1; the last quarter's lane is 8 tokens and 2 parts on)
        const int ln = HALF ? ((tid >> 2) & 7) | (((tid >> 5) & 1) << 4) : tid >> 2, e = tid & 3;
        const int t = 16 * g + (ln & 15), n = n0 + 4 * (ln >> 4) + e;
        if (tid < 16 * CHANNELS / (HALF ? 2 : 1) && t < T && n < N) {
            float v[MATS];
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
                v[m] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    v[m] += part[w][m][ln][e];
                    if constexpr (HALF) v[m] += part[w][m][ln + 8 + 32][e];
                }
            }
            const float out = GATED ? v[0] / (1.f + expf(-v[0])) * v[MATS - 1] : v[0];
            y[(int64_t)t * ldo + n] = f32_to_bf16_bits(out);
        }
    }
}

template <int NW, int TG, int KB, bool GATED, bool HALF> pme_status launch_kb(const Fp8GemmArgs& a) {
    constexpr int CHANNELS = HALF ? 8 : 16;
    hipLaunchKernelGGL((k_fp8_gemm_decode<NW, TG, KB, GATED, HALF>), dim3((unsigned)((a.N + CHANNELS - 1) / CHANNELS)), dim3(64 * NW), 0, a.stream,
                       a.qx, a.sx, a.qw, a.sw, a.qu, a.su, (int)a.T, (int)a.N, (int)a.K, static_cast<uint16_t*>(a.y), a.ldy);
    return hip_status(hipGetLastError());
}

int decode_nw() { static int v = getenv("NWV") ? atoi(getenv("NWV")) : 0; return v; }
template <int TG, bool GATED, bool HALF> pme_status launch_nw(const Fp8GemmArgs& a) {
    const int64_t steps = (a.K / 128 + (HALF ? 1 : 0)) / (HALF ? 2 : 1);
    constexpr int KB = GATED || TG > 1 ? 2 : 4;      // what 128 registers hold
    const int nw = decode_nw() ? decode_nw() : steps >= 32 ? 16 : steps >= 8 ? 8 : 4;
    if (nw == 16) return launch_kb<16, TG, KB, GATED, HALF>(a);
    if (nw == 8) return launch_kb<8, TG, KB, GATED, HALF>(a);
    return launch_kb<4, TG, KB, GATED, HALF>(a);
}

template <bool GATED> pme_status launch_of(const Fp8GemmArgs& a) {
    static int hv = getenv("HALFV") ? atoi(getenv("HALFV")) : 2;
    if (a.T <= 8 && (hv == 1 || (hv == 2 && (a.N + 15) / 16 < 256))) return launch_nw<1, GATED, true>(a);
    if (a.T <= 16) return launch_nw<1, GATED, false>(a);
    return launch_nw<2, GATED, false>(a);
}

}  // namespace

pme_status launch_fp8_gemm_decode(const Fp8GemmArgs& a) {
    if (a.T > 32) return PME_ERR_UNSUPPORTED_PATH;
    if (a.dry) {
        if (a.plan) *a.plan = "k_fp8_gemm_decode";
        return PME_OK;
    }
    return a.qu ? launch_of<true>(a) : launch_of<false>(a);
}

}  // namespace pme
