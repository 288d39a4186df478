// Products of e4m3 codes with a scale for each block of 128, for few tokens: the waves of a workgroup split K.
//
//   p[t][n] = sum_g sx[t][g] sw[n / 128][g] sum_{k in group g} qx[t][k] qw[n][k],   y = bf16(p), or gated bf16(silu(p_g) p_u).
//
// A workgroup owns AR tokens and BN rows of weights (gated: BN / 2 of each matrix).  Each of its NW waves takes a contiguous NW-th of the
// blocks of K and computes the whole tile over it, from an LDS ring of its own that it fills by DMA itself: no barrier in the K loop.
// The waves' fp32 sums are added through LDS in the order of K.  The matrix instruction and what it rounds: as in gemm_fp8.hip.
//
// Bound by the weights, each read once (by DMA with nothing in registers, so that 4 waves of several K blocks each are in flight on a
// unit; tokens x features x channels, weights in the last-level cache): 16 rows of weights a workgroup spread N = 2048 over 128 units, 1 x 8192 x 2048
// 5.5 us, 3.0 TB/s, on 32 rows 6.5; gated 8 x 2048 x 8192 7.4 us, 4.6 TB/s; 8 x 14336 x 4096 11.5 us, 5.1 TB/s.  An empty launch is 1.9 of these.
// Tiles of more tokens take up to about 256 of them: 64 x 32 fills the units where 64 x 64 leaves most of them idle.
#include "gemm_fp8.h"

#include <algorithm>
#include <cstdio>
#include <string>

namespace pme {
namespace {

constexpr int fp8_kslice_group(int ar, bool gated) { return ((ar + (gated ? 2 : 1)) * 16 + 63) / 64 * 64; }      // bytes of four K blocks' scales
constexpr int fp8_kslice_ring(int ar, int bn, int nstage, bool gated) { return (nstage * (ar + bn) * 128 + 2 * fp8_kslice_group(ar, gated) + 127) / 128 * 128; }
constexpr int fp8_kslice_lds(int ar, int bn, int nw, int nstage, bool gated) {
    const int rings = nw * fp8_kslice_ring(ar, bn, nstage, gated), parts = nw * ((ar + 15) / 16) * (bn / 16) * 1024;
    return rings > parts ? rings : parts;
}

template <int AR, int BN, int NW, int NSTAGE, bool GATED>
__global__ void __launch_bounds__(64 * NW, 2)
k_fp8_gemm_kslice(const Fp8TileArgs p) {
    constexpr int FM = (AR + 15) / 16, FN = BN / 16, BO = GATED ? BN / 2 : BN, FO = BO / 16, ROWS = AR + BN;
    constexpr int CH = ROWS / 8;                                 // DMA instructions of a K block
    constexpr int STAGE = ROWS * 128, SCALES = NSTAGE * STAGE, GROUP = fp8_kslice_group(AR, GATED), RING = fp8_kslice_ring(AR, BN, NSTAGE, GATED);
    static_assert((AR == 8 || AR % 16 == 0) && BN % (GATED ? 32 : 16) == 0 && 128 % BO == 0, "whole fragments; a tile's channels have one scale a matrix");
    static_assert(AR <= 64 && (NSTAGE - 1) * CH + 2 <= 63, "one DMA for the tokens' scales; wait counts fit vmcnt");
    static_assert(NSTAGE <= 6, "a group of scales, issued four steps before its first reader, is older than the codes that the wait leaves in flight");
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn;
    fp8_tile((int)blockIdx.x, p.tiles_m, p.tiles_n, p.band, tm, tn);
    const int m0 = tm * AR, n0 = tn * BO, groups = p.K / 128;
    const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)wave * groups / NW));
    const int steps = __builtin_amdgcn_readfirstlane((int)((int64_t)(wave + 1) * groups / NW) - first);
    const int ring = wave * RING;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(PME_AS3 unsigned char*)smem + ring);

    const uint32_t lane_off = (uint32_t)(lane >> 3) * (uint32_t)p.K + (uint32_t)(((lane & 7) ^ swz16(lane >> 3)) << 4);
    const u32x4 x_buf = buffer_of(p.qx, (uint32_t)p.T * (uint32_t)p.K), w_buf = buffer_of(p.qw, (uint32_t)p.N * (uint32_t)p.K);
    const u32x4 u_buf = buffer_of(GATED ? p.qu : p.qw, (uint32_t)p.N * (uint32_t)p.K);
    // step s of this wave (beyond its last one the last of all K blocks, which nobody reads); rows beyond the last are zeros, or any
    auto issue_codes = [&](auto stage, int s) {
        const uint32_t at = lane_off + (uint32_t)(min(first + s, groups - 1) * 128);
        static_for<CH>([&](auto qc) {
            constexpr int q = decltype(qc)::value, r = 8 * q, b = r - AR;
            const uint32_t row = (uint32_t)(r < AR ? m0 + r : n0 + (b < BO ? b : b - BO)) * (uint32_t)p.K;
            // the odd blocks' rows have the other half of the swizzles
            dma16_to<decltype(stage)::value * STAGE + q * 1024>(r < AR ? x_buf : GATED && b >= BO ? u_buf : w_buf, ((q & 1) ? at ^ 64 : at) + row, lds0);
        });
    };
    // scales of steps 4 g .. 4 g + 3: sixteen bytes of every token and block of channels, those beyond the end of the array as zeros
    const uint32_t rowb = (uint32_t)groups * 4, wrow = (uint32_t)(n0 / 128) * rowb;
    const u32x4 sx_buf = buffer_of(p.sx, (uint32_t)p.T * rowb), sw_buf = buffer_of(p.sw, (uint32_t)((p.N + 127) / 128) * rowb);
    const u32x4 su_buf = buffer_of(GATED ? p.su : p.sw, (uint32_t)((p.N + 127) / 128) * rowb);
    const uint32_t srow = (uint32_t)min(m0 + min(lane, AR - 1), p.T - 1) * rowb;
    auto issue_scales = [&](int g) {
        const uint32_t at = (uint32_t)min(first + 4 * g, groups - 1) * 4, to = __builtin_amdgcn_readfirstlane(lds0 + SCALES + (g & 1) * GROUP);
        if (lane < AR) dma16_buffer(sx_buf, srow + at, to);
        if (lane == 0) {
            dma16_buffer(sw_buf, wrow + at, to + 16 * AR);
            if constexpr (GATED) dma16_buffer(su_buf, wrow + at, to + 16 * AR + 16);
        }
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int r16 = lane & 15, kg = lane >> 4, ra = AR == 8 ? r16 & 7 : r16;
    // a tile of 8 tokens repeats them over the fragment's rows: the surplus results are never stored
    const int a0 = ring + ra * 128 + ((kg ^ swz16(ra)) << 4), a1 = a0 ^ 64, b0 = ring + (AR + r16) * 128 + ((kg ^ swz16(AR + r16)) << 4), b1 = b0 ^ 64;
    auto frag = [&](int lo, int hi) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(smem + lo), b = *reinterpret_cast<const u32x4*>(smem + hi);
        return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    };

    if (steps > 0) {
        issue_scales(0);
        issue_scales(1);
        static_for<NSTAGE - 1>([&](auto st) { issue_codes(st, decltype(st)::value); });
        auto step = [&](auto uc, int s) {
            constexpr int at = decltype(uc)::value * STAGE;
            constexpr std::integral_constant<int, (decltype(uc)::value + NSTAGE - 1) % NSTAGE> prv{};
            // the fragments of the step before are in registers (their reads have been waited for): its stage, and every fourth step
            // its group of scales, can be filled again
            if (s > 0 && (s & 3) == 0) issue_scales((s >> 2) + 1);
            issue_codes(prv, s + NSTAGE - 1);
            wait_vm<(NSTAGE - 1) * CH>();
            const int sc = ring + SCALES + ((s >> 2) & 1) * GROUP + 4 * (s & 3);
            const float sw = *reinterpret_cast<const float*>(smem + sc + 16 * AR), su = GATED ? *reinterpret_cast<const float*>(smem + sc + 16 * (AR + 1)) : 0.f;
            float sx[FM];
            i32x8 a[FM], b[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                a[i] = frag(a0 + at + 2048 * i, a1 + at + 2048 * i);
                sx[i] = *reinterpret_cast<const float*>(smem + sc + 16 * (ra + 16 * i));
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) b[j] = frag(b0 + at + 2048 * j, b1 + at + 2048 * j);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const f32x4 t = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                    const float f = sx[i] * (GATED && j >= FO ? su : sw);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[e], f, acc[i][j][e]);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        };
        for (int s = 0; s < steps; s += NSTAGE)
            static_for<NSTAGE>([&](auto uc) {
                if (decltype(uc)::value == 0 || s + decltype(uc)::value < steps) step(uc, s + decltype(uc)::value);
            });
        wait_vm<0>();
    }
    __syncthreads();

    // ---- the waves' sums: element e of lane l of block (i, j) is token 16 i + l % 16, channel 16 j + 4 (l / 16) + e
    f32x4* part = reinterpret_cast<f32x4*>(smem);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) part[((wave * FM + i) * FN + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    constexpr int OUT = FM * FO * 256;
    for (int o = tid; o < OUT; o += 64 * NW) {
        const int e = o & 3, l = (o >> 2) & 63, blk = o >> 8, i = blk / FO, j = blk % FO;
        float v = 0.f, u = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            v += part[((w * FM + i) * FN + j) * 64 + l][e];
            if constexpr (GATED) u += part[((w * FM + i) * FN + j + FO) * 64 + l][e];
        }
        const int row = 16 * i + (l & 15), t = m0 + row, n = n0 + 16 * j + 4 * (l >> 4) + e;
        if (row < AR && t < p.T && n < p.N) p.y[(int64_t)t * p.ldo + n] = f32_to_bf16_bits(GATED ? silu(v) * u : v);
    }
}

template <int AR, int BN, int NW, int NSTAGE, bool GATED> pme_status launch_kslice(const Fp8GemmArgs& a) {
    if (a.dry) {
        if (a.plan) {
            // the instantiation's name as a profiler prints it
            static const std::string name = [] {
                char buf[96];
                snprintf(buf, sizeof buf, "k_fp8_gemm_kslice<%d, %d, %d, %d, %s>", AR, BN, NW, NSTAGE, GATED ? "true" : "false");
                return std::string(buf);
            }();
            *a.plan = name.c_str();
        }
        return PME_OK;
    }
    constexpr int BO = GATED ? BN / 2 : BN;
    constexpr int lds = fp8_kslice_lds(AR, BN, NW, NSTAGE, GATED);
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    const int tiles_m = (int)((a.T + AR - 1) / AR), tiles_n = (int)((a.N + BO - 1) / BO);
    auto kern = k_fp8_gemm_kslice<AR, BN, NW, NSTAGE, GATED>;
    static std::atomic<uint32_t> done;
    if (allow_dynamic_lds(kern, lds, done) != PME_OK) return PME_ERR_HIP;
    const Fp8TileArgs p{a.qx, a.sx, a.qw, a.sw, a.qu, a.su, (int)a.T, (int)a.N, (int)a.K, static_cast<uint16_t*>(a.y), a.ldy,
                        tiles_m, tiles_n, fp8_band(tiles_m, tiles_n, AR, BN, 160 * 1024 / lds)};
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * tiles_n)), dim3(64 * NW), lds, a.stream, p);
    return hip_status(hipGetLastError());
}

template <bool GATED> pme_status launch_of(const Fp8GemmArgs& a, int tile) {
    if constexpr (!GATED) switch (tile) {
        case 0: return launch_kslice<8, 16, 4, 5, GATED>(a);
        case 1: return launch_kslice<16, 16, 4, 4, GATED>(a);
    }
    switch (tile) {
        case 2: return launch_kslice<8, 32, 4, 3, GATED>(a);
        case 3: return launch_kslice<16, 32, 4, 2, GATED>(a);
        case 4: return launch_kslice<32, 32, 4, 2, GATED>(a);
        case 5: return launch_kslice<64, 32, 4, 2, GATED>(a);
    }
    return PME_ERR_UNSUPPORTED_PATH;
}

}  // namespace

pme_status launch_fp8_gemm_kslice(const Fp8GemmArgs& a, int tile) { return a.qu ? launch_of<true>(a, tile) : launch_of<false>(a, tile); }

}  // namespace pme
