// Products of e4m3 codes with a scale for each block of 128:
//
//   p[t][n] = sum_g sx[t][g] sw[n / 128][g] sum_{k in group g} qx[t][k] qw[n][k],   y = bf16(p),
//   gated:  y = bf16( p_g / (1 + e^-p_g) p_u )  of two weight matrices.
//
// v_mfma_f32_16x16x128_f8f6f4 sums a whole block of K.  It starts from zero, and its sum goes into fp32 accumulators by four FMAs a lane with
// sx sw.  Everything behind the instruction is fp32; inside, it adds eight products at a time on a grid 13 bits below the largest exponent
// among them (measured; v_mfma_f32_16x16x32_fp8_fp8 does the same, so that no form of an 8-bit product at this rate is finer): at most
// 7 2^-13 of a run's largest product, an eightieth of what a code's own rounding (2^-4) leaves.
//
// What bounds it: the instruction alone runs at 4270 TFLOP/s, with the FMAs, which share its issue slots, at 3450 (32 x 32 x 64: 3890 and
// 3360, for twice the sums in flight), registers only; 4096 x 14336 x 4096 (tokens, features, channels, here and below) runs at 2570 (187 us),
// an unscaled library product at 2690.  There the matrix pipe is busy 73 % of the cycles at a clock that power holds at 1.5 to 1.9 GHz.
#include "gemm_fp8.h"

#include <algorithm>
#include <cstdio>
#include <string>

namespace pme {
namespace {

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

// ---- Matrix-core kernel: a workgroup computes BM tokens x BN weights (gated: BN / 2 of either matrix, interleaved a wave at a time, so that
// the lane that holds g holds u), WGM x WGN waves, KS slices of them on blocks of K in turn.  Codes go to LDS by DMA, NSTAGE stages of one
// block of K a slice, chunks of 16 bytes swizzled so that a fragment's reads have no bank conflicts beyond the instruction's own; scales go
// there four blocks at a time.  The instruction's operands are exchanged (weights as rows), which leaves a lane four consecutive channels of
// a token: one sx a lane, one sw a wave.
//
// Two schedules, by what fits the registers.  AHEAD (up to 128 x 128): a step's operands are all in registers when it begins; a step costs
// one wait and one barrier.  333 x 4096 x 4096 on 64 x 128: 13.1 us, 0.29 a step, of which 0.11 are matrix instructions of its two waves a
// SIMD.  What holds the rest has not been told apart; two readings fit.  Codes arrive at 80 to 85 bytes a ns and unit on this tile (24 KB a step), on
// 128 x 128 (32 KB in 0.40), on 128 x 256 (48 in 0.62) and on the 64 x 32 tiles that split K (48 in 0.60), on 64 units as on 192.  And reading the fragments
// (64, 96 and 160 KB a step at 128 bytes a cycle of 2.4 GHz) and a constant 0.08 give 0.29, 0.40 and 0.61 on the first three; against that one, 15 %
// fewer reads (2 x 4 waves on 128 x 256) are no faster.  Nothing tried has shortened a step: rings of 5 and 6 stages, waves of twice
// the tile, two slices of K, a ninth wave that touches the codes 5 or 10 steps ahead, operands straight from L2 into registers (16 rows a load: 32 us).
// Not AHEAD (128 x 128 to 256 x 256, two workgroups a compute unit where they fit): stages in two parts, described there.  256 x 256: half the
// bytes from L2 and LDS for an operation, and with them less power: 4096 x 14336 x 4096 187 us, on 128 x 256 219, on 128 x 128 247 (AHEAD 265).
constexpr int fp8_stage(int bm, int bn, int ks) { return ks * (bm + bn) * 128; }
constexpr int fp8_scale_blocks(int bm, bool gated) { return (bm + 63) / 64 + (gated ? 2 : 1); }
constexpr int fp8_lds(int bm, int bn, int ks, int nstage, bool gated) { return nstage * fp8_stage(bm, bn, ks) + 2 * 1024 * fp8_scale_blocks(bm, gated); }

template <int BM, int BN, int WGM, int WGN, int KS, int NSTAGE, bool AHEAD, bool GATED>
__global__ void __launch_bounds__(64 * WGM * WGN * KS, 2)
k_fp8_gemm(const Fp8TileArgs p) {
    constexpr int NWW = WGM * WGN;                               // waves of a slice of K
    constexpr int WM = BM / WGM, WN = BN / WGN, FM = WM / 16, FN = WN / 16;
    constexpr int BO = GATED ? BN / 2 : BN, WO = GATED ? WN / 2 : WN, FO = WO / 16;      // output channels of the tile, of a wave, in blocks
    constexpr int ROWS = BM + BN, STAGE = fp8_stage(BM, BN, KS), SLICE = ROWS * 128;
    constexpr int CH = ROWS / 8 / NWW;                           // DMA instructions per wave and stage
    constexpr int XB = (BM + 63) / 64, SBLKS = fp8_scale_blocks(BM, GATED), GROUP = SBLKS * 1024, SCALES = NSTAGE * STAGE;
    constexpr int GS = 4 / KS;                                   // steps of a group of scales
    constexpr int DEPTH = AHEAD ? NSTAGE - 2 : NSTAGE - 1;       // stages in flight behind the one that a step's reads are from
    constexpr int DJ = AHEAD ? FN : FN - 1 < 2 ? FN - 1 : 2;     // regions of a step that carry its DMA
    constexpr int UNROLL = NSTAGE % 2 ? 2 * NSTAGE : NSTAGE;     // steps of a round, in which every place in LDS is a constant
    static_assert(KS == 1 || KS == 2, "a group of scales is whole steps, two at least");
    static_assert(ROWS / 8 % NWW == 0 && BM / 8 % NWW == 0 && BO / 8 % NWW == 0, "a DMA instruction of every wave is from one operand");
    static_assert(128 % WO == 0 && WM % 16 == 0 && WO % 16 == 0, "a wave's channels lie in one block of scales");
    static_assert(BO <= 128 || BO == 256, "a tile has the scales of one or two blocks of channels");
    static_assert(DEPTH >= 1 && GS >= DEPTH, "a group of scales is older than the codes that the wait leaves in flight");
    static_assert(FM * FN % 4 == 0 && FN % 2 == 0, "the sums in flight, and the fragments of weights, go round");

    // both lines of the arguments before anything is made of either: one latency of memory, not two in a row (0.1 to 0.2 us)
    asm volatile("" ::"s"(p.qx), "s"(p.tiles_m));
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = wave % NWW, ks = wave / NWW, wm = w / WGN, wn = w % WGN;
    int tm, tn;
    fp8_tile((int)blockIdx.x, p.tiles_m, p.tiles_n, p.band, tm, tn);
    const int m0 = tm * BM, n0 = tn * BO, groups = p.K / 128, KT = (groups + KS - 1) / KS;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(PME_AS3 unsigned char*)smem;

    // DMA of codes: block blk is rows 8 blk .. 8 blk + 7 of the wave's slice (tokens, channels, gated: the second matrix's channels);
    // lane L fills chunk position L % 8 of row L / 8, which holds chunk (L % 8) ^ swz
    // (not AHEAD: after the tokens, of every column of waves the weights of its first regions, then those of its last ones)
    constexpr int CHX = BM / 8 / NWW;
    auto block_of = [](int q) {                                  // first block of the NWW that the q-th instructions fill
        if (AHEAD || q < CHX) return NWW * q;
        const int c = (q - CHX) % WGN, h = (q - CHX) / WGN;
        return (BM + (GATED ? h * BO + c * (WN / 2) : c * WN + h * (WN / 2))) / 8;
    };
    static_assert(AHEAD || (WN / 2 / 8 == NWW && NSTAGE == 2 && KS == 1), "half the weights of a column of waves an instruction");
    static_assert(NWW % 2 == 0, "every block of a wave has the same swizzle");
    const uint32_t lane_off = (uint32_t)(lane >> 3) * (uint32_t)p.K + (uint32_t)(((lane & 7) ^ swz16(8 * w + (lane >> 3))) << 4);
    const u32x4 x_buf = buffer_of(p.qx, (uint32_t)p.T * (uint32_t)p.K), w_buf = buffer_of(p.qw, (uint32_t)p.N * (uint32_t)p.K);
    const u32x4 u_buf = buffer_of(GATED ? p.qu : p.qw, (uint32_t)p.N * (uint32_t)p.K);
    uint32_t row_off[CH];                                        // of the block's first row (rows beyond the last: zeros, or any)
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const int r = 8 * (w + block_of(q)), b = r - BM;
        row_off[q] = __builtin_amdgcn_readfirstlane((uint32_t)(r < BM ? m0 + r : n0 + (b < BO ? b : b - BO)) * (uint32_t)p.K);
    }
    const uint32_t lds_w = __builtin_amdgcn_readfirstlane(lds0 + ks * SLICE + w * 1024);
    auto issue_codes = [&](auto stage, auto qc, int kt) {        // K block beyond the last: the last again, which nobody reads
        constexpr int q = decltype(qc)::value, blk = block_of(q);
        const uint32_t at = lane_off + (uint32_t)(min(kt * KS + ks, groups - 1) * 128);
        dma16_to<decltype(stage)::value * STAGE + blk * 1024>(blk < BM / 8 ? x_buf : (GATED && blk >= (BM + BO) / 8) ? u_buf : w_buf, at + row_off[q], lds_w);
    };
    // of scales: sixteen bytes, four K blocks, of a token or of a block of channels; group g goes to place g & 1
    const uint32_t rowb = (uint32_t)groups * 4;
    const u32x4 sx_buf = buffer_of(p.sx, (uint32_t)p.T * rowb), sw_buf = buffer_of(p.sw, (uint32_t)((p.N + 127) / 128) * rowb);
    const u32x4 su_buf = buffer_of(GATED ? p.su : p.sw, (uint32_t)((p.N + 127) / 128) * rowb);
    static_assert(SBLKS <= NWW * KS, "a DMA instruction of scales a wave");
    const uint32_t srow = (uint32_t)(wave < XB ? min(m0 + min(64 * wave + lane, BM - 1), p.T - 1) : min(n0 / 128 + min(lane, 1), (p.N - 1) / 128)) * rowb;
    const uint32_t lds_s = __builtin_amdgcn_readfirstlane(lds0 + SCALES + wave * 1024);
    auto issue_scales = [&](int g) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_s + (g & 1) * GROUP), at = srow + 16 * (uint32_t)g;
        if (wave < XB) dma16_buffer(sx_buf, at, to);
        else if (wave == XB) dma16_buffer(sw_buf, at, to);
        else if (GATED && wave == XB + 1) dma16_buffer(su_buf, at, to);
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int r16 = lane & 15, kg = lane >> 4;
    // chunk 4 q + kg of a row is at position (kg ^ swz) ^ 4 q; rows 16 apart share their swizzle
    const int c0 = ks * SLICE + r16 * 128 + ((kg ^ swz16(r16)) << 4);
    const int a0 = c0 + wm * WM * 128, a1 = a0 ^ 64, b0 = c0 + (BM + wn * WO) * 128, b1 = b0 ^ 64;
    const int soff = SCALES + 16 * (wm * WM + r16), swoff = SCALES + XB * 1024 + 16 * ((n0 + wn * WO) / 128 - n0 / 128);      // the wave's block of channels
    auto frag = [&](int lo, int hi) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(smem + lo), b = *reinterpret_cast<const u32x4*>(smem + hi);
        return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    };
    auto load_a = [&](auto stage, auto ic) {
        constexpr int at = decltype(stage)::value * STAGE + 2048 * decltype(ic)::value;
        return frag(a0 + at, a1 + at);
    };
    auto load_b = [&](auto stage, auto jc) {
        constexpr int j = decltype(jc)::value, at = decltype(stage)::value * STAGE + 128 * (GATED && j >= FO ? BO + 16 * (j - FO) : 16 * j);
        return frag(b0 + at, b1 + at);
    };
    // scales of a step: of the wave's tokens, of its block of channels; then their products
    struct Scales { float x[FM], w, u; };
    struct Products { float w[FM], u[FM]; };
    auto scales_of = [&](int kt) { return ((kt / GS) & 1) * GROUP + 4 * ((kt * KS + ks) & 3); };
    auto load_scales = [&](Scales& s, int kt) {
        const int at = scales_of(kt);
        s.w = *reinterpret_cast<const float*>(smem + (at + swoff));
        if constexpr (GATED) s.u = *reinterpret_cast<const float*>(smem + (at + swoff) + 1024);
#pragma unroll
        for (int i = 0; i < FM; ++i) s.x[i] = *reinterpret_cast<const float*>(smem + (at + soff) + 256 * i);
    };
    auto products = [&](const Scales& s, int kt) {
        Products r;
        // a slice of K that has no block left in the last step works on its last block again, with a factor of zero (the scales read for it
        // are the next token's, and may be anything)
        const bool live = KS == 1 || kt * KS + ks < groups;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            r.w[i] = live ? s.x[i] * s.w : 0.f;
            if constexpr (GATED) r.u[i] = live ? s.x[i] * s.u : 0.f;
        }
        return r;
    };
    // Instruction m = j FM + i of a step, and the addition of its sum three instructions later, when it is there; the last three of a step
    // are added in the next one.
    f32x4 t[4] = {};
    auto multiply = [&](auto mc, const i32x8& wv, const i32x8& xv) {
        t[decltype(mc)::value & 3] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    };
    auto add = [&](const Products& s, auto mc) {
        constexpr int m = decltype(mc)::value, i = m % FM, j = m / FM;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[m & 3][e], GATED && j >= FO ? s.u[i] : s.w[i], acc[i][j][e]);
    };
    auto add_behind = [&](const Products& before, const Products& now, auto mc) {
        constexpr int m = decltype(mc)::value;
        if constexpr (m < 3) add(before, std::integral_constant<int, FM * FN - 3 + m>{});
        else add(now, std::integral_constant<int, m - 3>{});
    };
    Products before, now;
#pragma unroll
    for (int i = 0; i < FM; ++i) before.w[i] = before.u[i] = 0.f;

    issue_scales(0);
    issue_scales(1);
    constexpr std::integral_constant<int, 0> first{};
    Scales s;
    if constexpr (AHEAD) {
        // Every operand of a step is in registers when the step begins, while the next one's are read into others: a step's LDS reads
        // have the whole of the step before to arrive in, and nothing waits for the last of them at the barrier.
        i32x8 a[2][FM], b[2][FN];
        static_for<DEPTH + 1>([&](auto st) { static_for<CH>([&](auto qc) { issue_codes(st, qc, decltype(st)::value); }); });
        wait_vm<DEPTH * CH>();
        lds_barrier();
        load_scales(s, 0);
        static_for<FM>([&](auto ic) { a[0][decltype(ic)::value] = load_a(first, ic); });
        static_for<FN>([&](auto jc) { b[0][decltype(jc)::value] = load_b(first, jc); });
        auto step = [&](auto uc, int kt) {
            constexpr int u = decltype(uc)::value;
            constexpr std::integral_constant<int, (u + 1) % NSTAGE> nxt{};
            constexpr std::integral_constant<int, (u + NSTAGE - 1) % NSTAGE> prv{};
            // The next step's operands have landed, by this wave's DMA and then by every wave's.  This step's may still be on their way into
            // other waves' registers; those of the step before were used there: their stage can be filled again, and the place of the
            // scales before this group's.
            wait_vm<(DEPTH - 1) * CH>();
            asm volatile("s_barrier" ::: "memory");
            if (kt > 0 && kt % GS == 0) issue_scales(kt / GS + 1);
            now = products(s, kt);
            load_scales(s, kt + 1);
            static_for<FN>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                static_for<CH>([&](auto qc) {
                    if constexpr (decltype(qc)::value * DJ / CH == j) issue_codes(prv, qc, kt + NSTAGE - 1);
                });
                static_for<FM>([&](auto ic) {
                    constexpr std::integral_constant<int, j * FM + decltype(ic)::value> m{};
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m < 3) add_behind(before, now, m);
                    multiply(m, b[u & 1][j], a[u & 1][decltype(ic)::value]);
                    // the next step's fragments in the order of their use, evenly: 5 to 7 % of 128 x 128 over all of them first
                    static_for<FM + FN>([&](auto lc) {
                        constexpr int l = decltype(lc)::value;
                        if constexpr (l * FM * FN / (FM + FN) == m) {
                            if constexpr (l == 0) b[(u + 1) & 1][0] = load_b(nxt, first);
                            else if constexpr (l <= FM) a[(u + 1) & 1][l - 1] = load_a(nxt, std::integral_constant<int, l - 1>{});
                            else b[(u + 1) & 1][l - FM] = load_b(nxt, std::integral_constant<int, l - FM>{});
                        }
                    });
                    if constexpr (m >= 3) add_behind(before, now, m);
                });
            });
            before = now;
        };
        for (int kt = 0; kt < KT; kt += UNROLL)
            static_for<UNROLL>([&](auto uc) {
                if (decltype(uc)::value == 0 || kt + decltype(uc)::value < KT) step(uc, kt + decltype(uc)::value);
            });
    } else {
        // Too many registers for that: the weights' fragments come one region ahead, the next step's first operands over the last region.
        // Two stages, each in two parts: the tokens and the weights of the first half of the regions, and the weights of the other half.
        // Every part is filled again as soon as it has been read, half a step or a whole one before the step that last read it ends, and
        // has more than a step to land.
        constexpr int G1 = CHX + WGN, H = FN / 2;                // DMA instructions of the first part; its regions
        constexpr int R = H < 3 ? H : 3;                         // regions that carry its refill, all before the last one's wait
        static_assert(H >= 2, "the second part's refill is issued before the wait that counts it");
        i32x8 a[FM], b[2];
        auto issue_part = [&](auto part, auto stage, int kt, auto from, auto to) {       // instructions [from, to) of the part
            static_for<decltype(to)::value - decltype(from)::value>([&](auto qc) {
                issue_codes(stage, std::integral_constant<int, decltype(part)::value * G1 + decltype(from)::value + decltype(qc)::value>{}, kt);
            });
        };
        constexpr std::integral_constant<int, 1> second{};
        constexpr std::integral_constant<int, G1> g1{};
        constexpr std::integral_constant<int, CH - G1> g2{};
        issue_part(first, first, 0, first, g1);
        issue_part(second, first, 0, first, g2);
        issue_part(first, second, 1, first, g1);
        wait_vm<CH>();
        lds_barrier();
        load_scales(s, 0);
        static_for<FM>([&](auto ic) { a[decltype(ic)::value] = load_a(first, ic); });
        b[0] = load_b(first, first);
        auto step = [&](auto uc, int kt) {
            constexpr std::integral_constant<int, decltype(uc)::value & 1> cur{};
            constexpr std::integral_constant<int, 1 - cur> nxt{};
            if (kt > 0 && kt % GS == 0) issue_scales(kt / GS + 1);       // into the place that the last step has left
            now = products(s, kt);
            static_for<FN>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                // One part behind the newest CH instructions has landed, by this wave's DMA and then by every wave's: before region H - 1
                // the second part of this step, before the last region the first part of the next one.  What lies before the fragment
                // that this region multiplies has been read by every wave.
                if constexpr (j == H - 1 || j == FN - 1) {
                    wait_vm<CH>();
                    lds_barrier();
                }
                if constexpr (j + 1 < FN) b[(j + 1) & 1] = load_b(cur, std::integral_constant<int, j + 1>{});
                else {
                    b[0] = load_b(nxt, first);
                    load_scales(s, kt + 1);
                }
                if constexpr (j == 0) issue_part(second, nxt, kt + 1, first, g2);
                if constexpr (j >= H - 1 && j < H - 1 + R) {
                    constexpr std::integral_constant<int, (j - H + 1) * G1 / R> from{};
                    constexpr std::integral_constant<int, (j - H + 2) * G1 / R> to{};
                    issue_part(first, cur, kt + 2, from, to);
                }
                static_for<FM>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    constexpr std::integral_constant<int, j * FM + i> m{};
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m < 3) add_behind(before, now, m);
                    multiply(m, b[j & 1], a[i]);
                    if constexpr (j == FN - 1) a[i] = load_a(nxt, ic);
                    if constexpr (m >= 3) add_behind(before, now, m);
                });
            });
            before = now;
            // the additions stay in their step
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    f32x4& v = acc[i][j];
                    asm volatile("" : "+v"(v));
                }
        };
        for (int kt = 0; kt < KT; kt += UNROLL)
            static_for<UNROLL>([&](auto uc) {
                if (decltype(uc)::value == 0 || kt + decltype(uc)::value < KT) step(uc, kt + decltype(uc)::value);
            });
    }
    static_for<3>([&](auto mc) { add_behind(before, now, mc); });
    wait_vm<0>();
    lds_barrier();

    // ---- the slices of K are added in LDS: slice i % KS finishes the 16 tokens of group i
    if constexpr (KS > 1) {
        f32x4* part = reinterpret_cast<f32x4*>(smem);
        static_assert(NWW * FM * KS * FN * 1024 <= NSTAGE * STAGE, "the partial sums go through the stages");
        auto at = [&](int i, int slice, int j) { return part + ((((w * FM + i) * KS + slice) * FN + j) * 64 + lane); };
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (i % KS != ks) {
#pragma unroll
                for (int j = 0; j < FN; ++j) *at(i, ks, j) = acc[i][j];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < FM; ++i)
            if (i % KS == ks) {
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    if (s != i % KS) {
#pragma unroll
                        for (int j = 0; j < FN; ++j) acc[i][j] += *at(i, s, j);
                    }
            }
        __syncthreads();
    }

    // ---- epilogue: element e of block (i, j) is token m0 + wm WM + 16 i + r16, channel n0 + wn WO + 16 j + 4 kg + e.  A wave's outputs go
    // through LDS of its own into 16-byte pieces of rows, 16-byte chunk c of row r at position c ^ swz(r).  Only the registers' way into LDS is
    // written out; the stores are a loop, since code that runs once comes from memory (256 x 256, one K block: 7.0 us, 13.0 with all of it written out).
    constexpr int WR = WM / KS, CPS = WO / 8, RPB = WO < 128 ? 128 / WO : 1;      // the wave's rows, a row's chunks, rows of all the banks
    static_assert(FM % KS == 0 && BM * BO * 2 <= NSTAGE * STAGE, "the outputs go through the stages");
    unsigned char* slab = smem + wave * (WR * WO * 2);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        if (i % KS != ks) continue;
#pragma unroll
        for (int j = 0; j < FO; ++j) {
            f32x4 v = acc[i][j];
            if constexpr (GATED) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = silu(v[e]) * acc[i][j + FO][e];
            }
            *reinterpret_cast<u32x2*>(slab + (16 * (i / KS) + r16) * (WO * 2) + (((2 * j + (kg >> 1)) ^ ((r16 / RPB) & (CPS - 1))) << 4) + 8 * (kg & 1)) =
                u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int n = n0 + wn * WO + lane % CPS * 8;
#pragma unroll 4
    for (int row = lane / CPS; row < WR; row += 64 / CPS) {
        const int t = m0 + wm * WM + 16 * (row / 16 * KS + ks) + row % 16;
        const uint16_t* from = reinterpret_cast<const uint16_t*>(slab + row * (WO * 2) + ((lane % CPS ^ ((row % 16 / RPB) & (CPS - 1))) << 4));
        uint16_t* to = p.y + (int64_t)t * p.ldo + n;
        // 16 bytes wherever they lie: the memory system takes wide accesses at any address
        if (t < p.T && n + 8 <= p.N) __builtin_memcpy(to, from, 16);
    }
    if (n < p.N && n + 8 > p.N) {
#pragma unroll 1
        for (int row = lane / CPS; row < WR; row += 64 / CPS) {
            const int t = m0 + wm * WM + 16 * (row / 16 * KS + ks) + row % 16;
            const uint16_t* from = reinterpret_cast<const uint16_t*>(slab + row * (WO * 2) + ((lane % CPS ^ ((row % 16 / RPB) & (CPS - 1))) << 4));
            if (t < p.T)
#pragma unroll 1
                for (int e = 0; n + e < p.N; ++e) p.y[(int64_t)t * p.ldo + n + e] = from[e];
        }
    }
}

template <int BM, int BN, int WGM, int WGN, int KS, int NSTAGE, bool AHEAD, bool GATED> pme_status launch_tile(const Fp8GemmArgs& a) {
    if (a.dry) {
        if (a.plan) {
            // the instantiation's name as a profiler prints it
            static const std::string name = [] {
                char buf[96];
                snprintf(buf, sizeof buf, "k_fp8_gemm<%d, %d, %d, %d, %d, %d, %s, %s>", BM, BN, WGM, WGN, KS, NSTAGE, AHEAD ? "true" : "false", GATED ? "true" : "false");
                return std::string(buf);
            }();
            *a.plan = name.c_str();
        }
        return PME_OK;
    }
    constexpr int BO = GATED ? BN / 2 : BN;
    constexpr int lds = fp8_lds(BM, BN, KS, NSTAGE, GATED);
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    const int tiles_m = (int)((a.T + BM - 1) / BM), tiles_n = (int)((a.N + BO - 1) / BO);
    auto kern = k_fp8_gemm<BM, BN, WGM, WGN, KS, NSTAGE, AHEAD, GATED>;
    static std::atomic<uint32_t> done;
    if (allow_dynamic_lds(kern, lds, done) != PME_OK) return PME_ERR_HIP;
    const Fp8TileArgs p{a.qx, a.sx, a.qw, a.sw, a.qu, a.su, (int)a.T, (int)a.N, (int)a.K, static_cast<uint16_t*>(a.y), a.ldy,
                        tiles_m, tiles_n, fp8_band(tiles_m, tiles_n, BM, BN, 160 * 1024 / lds)};
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * tiles_n)), dim3(64 * WGM * WGN * KS), lds, a.stream, p);
    return hip_status(hipGetLastError());
}

int g_fp8_tile_override = 0;

// The tiles, and their times by tile_cost: fitted, in us, to 2600 shapes of 1 .. 4096 tokens, 256 .. 16384 features and 128 .. 14336 channels, a
// third of them gated, up to 256 tokens the geometric mean of weights from the caches and from memory (a fit's mean error is 3 to 7 %).  On
// these shapes the tile of the least estimate is 0.3 % slower in the mean than the fastest of all that were timed, 1.9 % at the 95th percentile.
struct Tile {
    int rows, weights;           // of the tile: tokens, weights (of both matrices where gated)
    double cost[8];
};
const Tile kTiles[] = {
    {8, 16, {2.696, 0.6948, 0.0376, 0.003804, 0.01109, 0.02497, 0.03937, 1.578}},
    {16, 16, {2.677, 0.6307, 0.04023, 0.009718, 0.01423, 0.03093, 0.03426, 1.634}},
    {8, 32, {2.734, 0.5718, 0.05993, 0.0001506, 0.0156, 0.03934, 0.05048, 2.667}},
    {16, 32, {2.633, 0.3302, 0.07102, 0.01027, 0.0214, 0.04488, 0.0468, 1.053}},
    {32, 32, {3.063, 0.6422, 0.09365, 0.003589, 0.02283, 0.06409, 0.04334, 0.8272}},
    {64, 32, {3.683, 1.983, 0.1344, 0.006331, 0.008033, 0.1389, 0.03713, 0.5888}},
    {64, 64, {3.328, 1.687, 0.1716, 0.0007186, 0.03206, 0.1666, 0.05376, 0.5}},
    {64, 64, {2.627, 0.4282, 0.2324, 0, 0.1255, 0.06432, 0.05639, 0.3038}},
    {64, 128, {3.056, 1.47, 0.2918, 0, 0.07068, 0.2674, 0.05896, 0.2557}},
    {128, 128, {3.697, 1.589, 0.3721, 0.02714, 0.1339, 0.4102, 0.03928, 0.2679}},
    {128, 128, {3.731, 0.402, 0.467, 0.03458, 0.2668, 0.2518, 0.02569, 0.2271}},
    {128, 256, {4.366, 2.152, 0.6234, 0.1061, 0.2853, 0.6835, 0.03302, 0.2263}},
    {256, 256, {6.545, 3.155, 1.089, 0.3802, 0.5706, 1.188, 0, 0.2507}},
};
constexpr int kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]);

template <bool GATED> pme_status launch_one(const Fp8GemmArgs& a, int id) {
    switch (id) {
        case 6: return launch_tile<64, 64, 2, 2, 2, 4, true, GATED>(a);
        case 7: return launch_tile<64, 64, 2, 2, 1, 4, true, GATED>(a);
        case 8: return launch_tile<64, 128, 2, 4, 1, 4, true, GATED>(a);
        case 9: return launch_tile<128, 128, 4, 2, 1, 4, true, GATED>(a);
        case 10: return launch_tile<128, 128, 2, 2, 1, 2, false, GATED>(a);
        case 11: return launch_tile<128, 256, 4, 2, 1, 2, false, GATED>(a);
        case 12: return launch_tile<256, 256, 4, 2, 1, 2, false, GATED>(a);
    }
    return launch_fp8_gemm_kslice(a, id);
}

int64_t tiles_of(const Tile& t, const Fp8GemmArgs& a) {
    return ((a.T + t.rows - 1) / t.rows) * ((a.N * (a.qu ? 2 : 1) + t.weights - 1) / t.weights);
}

// Tile estimated fastest, and its time.
int choose(const Fp8GemmArgs& a, double* us) {
    int best = -1;
    for (int id = 0; id < kNumTiles; ++id) {
        const Tile& t = kTiles[id];
        if (a.qu && t.weights < 32) continue;                    // a tile of 16 rows of weights has no room for two matrices
        if (t.rows > 16 && t.rows > 2 * a.T) continue;           // mostly empty rows: not what the times were fitted to
        const double c = tile_cost(t.cost, tiles_of(t, a), a.T, a.N * (a.qu ? 2 : 1), a.K);
        if (best < 0 || c < *us) best = id, *us = c;
    }
    return best;
}

// Channels [first, first + count) of a product.
Fp8GemmArgs channels_of(const Fp8GemmArgs& a, int64_t first, int64_t count) {
    Fp8GemmArgs p = a;
    p.N = count;
    p.qw = a.qw + first * a.K;
    p.sw = a.sw + first / 128 * (a.K / 128);
    if (a.qu) {
        p.qu = a.qu + first * a.K;
        p.su = a.su + first / 128 * (a.K / 128);
    }
    p.y = static_cast<uint16_t*>(a.y) + first;
    return p;
}

pme_status launch_id(const Fp8GemmArgs& a, int id) { return a.qu ? launch_one<true>(a, id) : launch_one<false>(a, id); }

}  // namespace

void set_fp8_tile_override(int id) { g_fp8_tile_override = id; }

pme_status launch_fp8_gemm_mfma(const Fp8GemmArgs& a) {
    if (g_fp8_tile_override) return launch_id(a, g_fp8_tile_override - 1);
    const int64_t mats = a.qu ? 2 : 1;
    double us = 0;
    const int id = choose(a, &us);
    // A large tile whose last round would fill few compute units: the whole rounds by it, and the channels that are left by what is fastest
    // for them, where that is estimated a twentieth better at least (gated, against the fastest tile alone: 1999 x 4096 x 14336 218 -> 212 us, 700 x 4096 x
    // 14336 97 -> 92, 2337 x 7680 x 3456 147 -> 124).
    int first_id = -1, rest_id = -1;
    int64_t first = 0;
    us *= 0.95;
    for (int k = 0; k < kNumTiles; ++k) {
        const Tile& t = kTiles[k];
        if (t.rows < 128 || t.rows > 2 * a.T) continue;
        const int64_t rounds = tiles_of(t, a) / 256, whole = rounds * 256 / ((a.T + t.rows - 1) / t.rows) * (t.weights / mats);
        if (whole <= 0 || whole >= a.N || whole % 128) continue;
        const Fp8GemmArgs bulk = channels_of(a, 0, whole), rest = channels_of(a, whole, a.N - whole);
        double both = 0;
        const int r = choose(rest, &both);
        both += tile_cost(t.cost, tiles_of(t, bulk), bulk.T, bulk.N * mats, a.K);
        if (both < us) us = both, first_id = k, rest_id = r, first = whole;
    }
    if (first_id < 0) return launch_id(a, id);
    const pme_status s = launch_id(channels_of(a, 0, first), first_id);
    if (s != PME_OK) return s;
    Fp8GemmArgs rest = channels_of(a, first, a.N - first);
    rest.plan = a.rest_plan;
    if (a.rest) *a.rest = first;
    return launch_id(rest, rest_id);
}

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
