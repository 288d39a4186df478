// 8-bit operands of the products with a scale for each block of 128 (gemm_fp8.hip): e4m3 codes and fp32 scales,
//
//   s = amax / 448 over a block (1 where amax is 0, at least 2^-126),   q = e4m3(v / s), round half to even, 448 the largest e4m3 value,
//   v / s as v times a rounded 1 / s, within 2^-22 of itself,
//
// of activations (blocks of 128 features of a token), of weights (128 x 128), and of activations that first go through the residual's
// addition and the root-mean-square norm,  h = round(x + r) in the stream's type,  v = h (mean_j h_j^2 + eps)^-1/2 w.
// Rows of codes are whole groups of 128, codes beyond d are 0, so that the product knows no ragged K.
//
// All three are bound by HBM: the values are read once, into registers, and codes, scales and h written once (kernel times and moved bytes,
// a plain copy of 1 GiB moves 5.2 to 5.8 TB/s: norm with a residual, 4096 x 4096 in bf16 23.7 us, 5.0 TB/s; 4096 x 14336 values 51 us in fp32,
// 5.8, and 34 in bf16, 5.2; 14336 x 4096 bf16 weights 34 us, 5.2), small ones by the launch and one chain load - reduction - store (one token 2.3 us).  A lane holds chunks of
// 8 consecutive values, so that a group is 16 lanes, whose largest magnitude takes four data-parallel moves; magnitudes are compared as bit
// patterns, where infinities and NaN come out largest: their group's scale and codes are NaN.
#include "gemm_tile.h"

#include <algorithm>
#include <cfloat>

namespace pme {
namespace {

constexpr int kGroup = 128;

// Eight consecutive values of a row as they lie in memory.
template <bool F32> struct Chunk;
template <> struct Chunk<true> {
    float v[8];
    __device__ __forceinline__ float get(int e) const { return v[e]; }
    __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f[e];
    }
};
template <> struct Chunk<false> {
    uint32_t v[4];
    __device__ __forceinline__ float get(int e) const { return __uint_as_float((e & 1) ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16); }
    __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) v[p] = pack_bf16(f[2 * p], f[2 * p + 1]);
    }
};
template <bool F32> using elem_t = std::conditional_t<F32, float, uint16_t>;

// Chunk c of a row of d values; values beyond d are zeros.  Rows of any alignment: the memory system takes wide accesses at any address.
template <bool F32> __device__ __forceinline__ Chunk<F32> load_chunk(const elem_t<F32>* row, int c, int d) {
    Chunk<F32> k;
    const elem_t<F32>* p = row + 8 * (int64_t)c;
    if (8 * c + 8 <= d) {
        __builtin_memcpy(&k, p, sizeof k);
    } else {
        elem_t<F32> e8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            e8[e] = 0;
            if (8 * c + e < d) e8[e] = p[e];
        }
        __builtin_memcpy(&k, e8, sizeof k);
    }
    return k;
}
template <bool F32> __device__ __forceinline__ void store_chunk(elem_t<F32>* row, int c, int d, const Chunk<F32>& k) {
    elem_t<F32>* p = row + 8 * (int64_t)c;
    if (8 * c + 8 <= d) {
        __builtin_memcpy(p, &k, sizeof k);
    } else {
        elem_t<F32> e8[8];
        __builtin_memcpy(e8, &k, sizeof k);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (8 * c + e < d) p[e] = e8[e];
    }
}

// Over the 16 lanes of a group (a row of the data-parallel moves), in every one of them.
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xF, 0xF, true));       // rotations by 1, 2, 4, 8 lanes
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true));
}
__device__ __forceinline__ float group_sum(float v) {
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x121, 0xF, 0xF, true));
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x122, 0xF, 0xF, true));
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xF, 0xF, true));
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float wave_sum(float v) {
    v = group_sum(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = group_max(v);
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    return max(a, max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }

// Scale of a block whose largest magnitude has the bits `amax`, and 1 / scale.  One Newton step each leaves the quotient and the
// reciprocal within half an ulp and what little the step's own square leaves: v times it is within two roundings, 2^-23, of v / s.
__device__ __forceinline__ void block_scale(uint32_t amax, float& s, float& inv) {
    const float a = __uint_as_float(amax);
    s = a * (1.f / 448.f);
    s = fmaf(fmaf(-448.f, s, a), 1.f / 448.f, s);
    s = amax == 0 ? 1.f : fmaxf(s, FLT_MIN);
    if (amax >= 0x7F800000u) s = __uint_as_float(0x7FC00000u);
    inv = __builtin_amdgcn_rcpf(s);
    inv = fmaf(fmaf(-s, inv, 1.f), inv, inv);
}

// Eight values over the scale as e4m3 codes.  |v * inv| exceeds 448 by roundings only, which 448 is nearest to.
__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float inv) {
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    return u32x2{(uint32_t)lo, (uint32_t)hi};
}

// Codes of chunk c of a row (every lane of the group calls), and the group's scale.
__device__ __forceinline__ void quantize_chunk(const float (&v)[8], int c, uint8_t* q, float* s) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[e]));
    float scale, inv;
    block_scale(group_max(m), scale, inv);
    *reinterpret_cast<u32x2*>(q + 8 * (int64_t)c) = codes8(v, inv);
    if ((c & 15) == 0) s[c >> 4] = scale;
}

template <bool F32> __device__ __forceinline__ const elem_t<F32>* row_of(const void* p, int64_t row, int64_t ld) { return static_cast<const elem_t<F32>*>(p) + row * ld; }

// ---- activations as they are: a workgroup takes 256 chunks of a row (two or four chunks a lane: 0 to 10 % and 5 to 60 % slower).
template <bool F32>
__global__ void __launch_bounds__(256)
k_quant_fp8(const void* __restrict__ x, int64_t rows, int d, int64_t ldx, int groups, uint8_t* __restrict__ q, float* __restrict__ s) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c >= 16 * groups) return;                   // whole groups: the lanes of one go together
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const Chunk<F32> k = load_chunk<F32>(row_of<F32>(x, row, ldx), c, d);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k.get(e);
        quantize_chunk(v, c, q + row * groups * kGroup, s + row * groups);
    }
}

// ---- residual, norm, codes.  ONE_WAVE: a wave per row, several rows a workgroup, no barrier; otherwise a workgroup per row.  The row stays
// in registers, NV chunks a lane; NV = 0: rows that do not fit are read again for the second pass (h from where the first one put it).
template <bool F32, bool WF32, bool RES, int NV, bool ONE_WAVE>
__global__ void __launch_bounds__(ONE_WAVE ? 256 : 1024)
k_rmsnorm_quant_fp8(const NormQuantArgs a) {
    __shared__ uint32_t part[2][3][16];      // by the row's parity: one barrier apart is enough
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int l = ONE_WAVE ? lane : (int)threadIdx.x, L = ONE_WAVE ? 64 : (int)blockDim.x;
    const int d = (int)a.d, groups = (int)((a.d + kGroup - 1) / kGroup), all = 16 * groups;
    constexpr int N = NV ? NV : 1;
    constexpr bool EARLY = NV > 0 && !(F32 && WF32 && NV == 4);      // the weights' registers fit too
    const int rounds = NV ? 1 : (all + L - 1) / L;
    int parity = 0;
    for (int64_t row = ONE_WAVE ? (int64_t)blockIdx.x * waves + wave : (int64_t)blockIdx.x; row < a.T; row += ONE_WAVE ? (int64_t)gridDim.x * waves : (int64_t)gridDim.x, parity ^= 1) {
        const elem_t<F32>* xr = row_of<F32>(a.x, row, a.ldx);
        const elem_t<F32>* rr = RES ? row_of<F32>(a.residual, row, a.ldr) : nullptr;
        elem_t<F32>* hr = RES ? static_cast<elem_t<F32>*>(a.h) + row * a.ldh : nullptr;
        uint8_t* q = a.qx + row * groups * kGroup;
        float* s = a.sx + row * groups;
        auto across = [&](uint32_t mine, int which, auto join) {        // over the waves of the row
            if constexpr (ONE_WAVE) return mine;
            if (lane == 0) part[parity][which][wave] = mine;
            __syncthreads();
            return join(part[parity][which], waves);
        };
        auto join_sum = [&](const uint32_t* p, int n) {
            // lane 0's order for all: every lane of the workgroup has the same bits, and takes the same branches below
            return __float_as_uint(lane_value(group_sum((lane & 15) < n ? __uint_as_float(p[lane & 15]) : 0.f), 0));
        };
        auto join_max = [&](const uint32_t* p, int n) { return group_max((lane & 15) < n ? p[lane & 15] : 0u); };

        Chunk<F32> k[N];
        Chunk<WF32> w[N];
        const elem_t<WF32>* wr = static_cast<const elem_t<WF32>*>(a.weight);
        float ss = 0.f;
        for (int r = 0; r < rounds; ++r) {
            const int c0 = r * L + l;
            Chunk<F32> t[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                k[i] = load_chunk<F32>(xr, c0 + i * L, d);
                if constexpr (RES) t[i] = load_chunk<F32>(rr, c0 + i * L, d);
            }
            if constexpr (EARLY) {       // ahead of the sum, so that the second half waits for nothing
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] = load_chunk<WF32>(wr, c0 + i * L, d);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (RES) {
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = k[i].get(e) + t[i].get(e);
                    k[i].set(f);
                    if (8 * (c0 + i * L) < d) store_chunk<F32>(hr, c0 + i * L, d, k[i]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(k[i].get(e), k[i].get(e), ss);
            }
        }
        ss = __uint_as_float(across(__float_as_uint(wave_sum(ss)), 0, join_sum));
        const float eps = a.eps, mean = ss / (float)d;
        float pre = 1.f, rms = 1.f / sqrtf(mean + eps);
        if (!(mean + eps <= FLT_MAX) || mean + eps < 1e-24f) {
            // The squares, or their mean with eps, leave fp32's range (or the row holds what is not finite): again on values times a power of
            // two that brings the larger of the largest and sqrt(eps) near 1.
            uint32_t m = 0;
            for (int r = 0; r < rounds; ++r) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if constexpr (NV == 0) k[i] = load_chunk<F32>(RES ? hr : xr, r * L + l, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) m = max(m, magnitude(k[i].get(e)));
                }
            }
            m = across(wave_max(m), 1, join_max);
            const int ex = min(max((int)(max(m, __float_as_uint(sqrtf(eps))) >> 23) - 127, -126), 126);
            pre = ldexpf(1.f, -ex);
            float sp = 0.f;
            for (int r = 0; r < rounds; ++r) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if constexpr (NV == 0) k[i] = load_chunk<F32>(RES ? hr : xr, r * L + l, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float f = k[i].get(e) * pre;
                        sp = fmaf(f, f, sp);
                    }
                }
            }
            sp = __uint_as_float(across(__float_as_uint(wave_sum(sp)), 2, join_sum));
            rms = 1.f / sqrtf(sp / (float)d + ldexpf(eps, -2 * ex));
            if (m == 0) rms = 0.f;                                        // zeros stay zeros, whatever eps
            if (m >= 0x7F800000u) rms = __uint_as_float(0x7FC00000u);
        }
        for (int r = 0; r < rounds; ++r) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = r * L + l + i * L;
                if (c >= all) continue;         // whole groups: the lanes of one go together
                if constexpr (NV == 0) k[i] = load_chunk<F32>(RES ? hr : xr, c, d);
                if constexpr (!EARLY) w[i] = load_chunk<WF32>(wr, c, d);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k[i].get(e) * pre * rms * w[i].get(e);
                quantize_chunk(v, c, q, s);
            }
        }
    }
}

// ---- weights: a workgroup per block of 128 x 128, each lane the same chunk of eight rows 16 apart.
template <bool F32>
__global__ void __launch_bounds__(256)
k_quantize_weights_fp8(const void* __restrict__ x, int64_t N, int d, int64_t ldx, uint8_t* __restrict__ q, float* __restrict__ s) {
    __shared__ uint32_t part[2][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int groups = (int)gridDim.x, c = 16 * (int)blockIdx.x + (int)(threadIdx.x & 15);
    int parity = 0;      // one barrier apart is enough for `part`
    for (int64_t b = blockIdx.y; b * kGroup < N; b += gridDim.y, parity ^= 1) {
        const int64_t r0 = b * kGroup + (threadIdx.x >> 4);
        Chunk<F32> k[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            k[i] = Chunk<F32>{};
            if (r0 + 16 * i < N) k[i] = load_chunk<F32>(row_of<F32>(x, r0 + 16 * i, ldx), c, d);
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, magnitude(k[i].get(e)));
        m = wave_max(m);
        if (lane == 0) part[parity][wave] = m;
        __syncthreads();
        m = max(max(part[parity][0], part[parity][1]), max(part[parity][2], part[parity][3]));
        float scale, inv;
        block_scale(m, scale, inv);
        if (threadIdx.x == 0) s[b * groups + blockIdx.x] = scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k[i].get(e);
            if (r0 + 16 * i < N) *reinterpret_cast<u32x2*>(q + (r0 + 16 * i) * groups * kGroup + 8 * (int64_t)c) = codes8(v, inv);
        }
    }
}

// Workgroups of a grid (along x, and along y); further rows are the same workgroups' next ones.
constexpr int64_t kMostBlocks = 1 << 20, kMostRows = 1 << 15;

template <bool F32, bool WF32, bool RES, int NV, bool ONE_WAVE> pme_status launch_norm(const NormQuantArgs& a, int waves) {
    const int64_t want = ONE_WAVE ? (a.T + waves - 1) / waves : a.T;
    hipLaunchKernelGGL((k_rmsnorm_quant_fp8<F32, WF32, RES, NV, ONE_WAVE>), dim3((unsigned)std::min(want, kMostBlocks)), dim3(64 * waves), 0, a.stream, a);
    return hip_status(hipGetLastError());
}

// A wave for rows of at most 512; otherwise the workgroup that holds the row with few chunks a lane, which have less to wait for one after
// the other (us, one / two / four chunks, norm with a residual in bf16: 1 x 2048 3.0 / 3.4 / 4.1, 512 x 4096 5.4 / 5.5 / 6.5, 4096 x 8192 47 / 44 / 45);
// rows of more than 16384 in bf16 four from 512 on, where fewer and lighter workgroups share a compute unit better (4096 x 14336 - / 87 / 80; in
// fp32, whose row takes twice the registers, - / 163 / 186).
template <bool F32, bool WF32, bool RES> pme_status norm_of(const NormQuantArgs& a) {
    const int64_t least = ((a.d + kGroup - 1) / kGroup * 16 + 63) / 64;      // waves with one chunk a lane
    if (least > 64) return launch_norm<F32, WF32, RES, 0, false>(a, 16);
    if (least == 1) return launch_norm<F32, WF32, RES, 1, true>(a, 4);
    const bool many = !F32 && a.T >= (least > 16 ? 512 : 2048);
    const int nv = least > 32 || (least > 16 && many) ? 4 : least > 8 || (least >= 4 && many) ? 2 : 1, waves = (int)((least + nv - 1) / nv);
    if (nv == 1) return launch_norm<F32, WF32, RES, 1, false>(a, waves);
    if (nv == 2) return launch_norm<F32, WF32, RES, 2, false>(a, waves);
    return launch_norm<F32, WF32, RES, 4, false>(a, waves);
}

template <bool F32, bool WF32> pme_status norm_of(const NormQuantArgs& a) { return a.residual ? norm_of<F32, WF32, true>(a) : norm_of<F32, WF32, false>(a); }

template <bool F32> pme_status quant_of(const QuantArgs& a) {
    const int64_t groups = (a.d + kGroup - 1) / kGroup;
    const dim3 grid((unsigned)((16 * groups + 255) / 256), (unsigned)std::min(a.rows, kMostRows));
    hipLaunchKernelGGL((k_quant_fp8<F32>), grid, dim3(256), 0, a.stream, a.x, a.rows, (int)a.d, a.ldx, (int)groups, a.q, a.s);
    return hip_status(hipGetLastError());
}

}  // namespace

pme_status launch_rmsnorm_quant_fp8(const NormQuantArgs& a) {
    if (a.xt == PME_F32) return a.wt == PME_F32 ? norm_of<true, true>(a) : norm_of<true, false>(a);
    return a.wt == PME_F32 ? norm_of<false, true>(a) : norm_of<false, false>(a);
}

pme_status launch_quant_fp8(const QuantArgs& a) { return a.xt == PME_F32 ? quant_of<true>(a) : quant_of<false>(a); }

pme_status launch_quantize_weights_fp8(const QuantArgs& a) {
    const dim3 grid((unsigned)((a.d + kGroup - 1) / kGroup), (unsigned)std::min((a.rows + kGroup - 1) / kGroup, kMostRows)), block(256);
    if (a.xt == PME_F32) hipLaunchKernelGGL((k_quantize_weights_fp8<true>), grid, block, 0, a.stream, a.x, a.rows, (int)a.d, a.ldx, a.q, a.s);
    else hipLaunchKernelGGL((k_quantize_weights_fp8<false>), grid, block, 0, a.stream, a.x, a.rows, (int)a.d, a.ldx, a.q, a.s);
    return hip_status(hipGetLastError());
}

}  // namespace pme
