// Products of 8-bit operands with a scale per block of 128, for one weight matrix or for rows grouped by expert.
//
//   out[m,n] = sum_b sa[m,b] sw[n/128,b] p_b[m,n],   p_b[m,n] = sum over the 128 k of block b of a[m,k] w[n,k]
//
// v_mfma_f32_16x16x128_f8f6f4 yields p_b of sixteen rows and sixteen columns; the vector ALU adds it, times its two scales, to an
// fp32 accumulator.  The instruction adds eight products at a time in fewer bits than fp32 has: what lies below 2^-13 of the power of two of
// the largest of the eight is dropped (measured; every 8-bit MFMA does), 1.4e-5 of a sum of normal values, where a bf16 output is rounded to
// 2^-9.  Products with an fp32 output are for those who go on with the sums: they multiply the codes as fp16, which holds them, on the fp16
// MFMA, whose sums are fp32 (at less than half the rate).  The W codes are the MFMA's A operand and the activations its B operand: a lane then has four consecutive n of one
// m, and the one activation scale.  Both operands are row-major, 128 bytes of a row to a step: lane l reads row l % 16, and from the row's
// eight pieces of 16 bytes the pieces l / 16 and l / 16 + 4 (the product does not care which of the 128 k is which, as long as both
// operands agree).
#include "device_util.hpp"
#include "internal.hpp"

#include <algorithm>

namespace fp4mr {
namespace {

struct Fp8Args {
    const uint8_t* a;
    const float* a_scales;
    const uint8_t* w;
    const float* w_scales;
    void* out;
    int64_t a_rows, N, K;      // a_rows: rows of A
    int64_t rows;              // rows of the output
    const int32_t* offsets;    // grouped: experts + 1 of them
    const int32_t* index;      // grouped: row of A for a row of the output, or null
    int experts;
};

// Thirty-two codes of a lane as fp16, which holds every E4M3 value.
struct Half32 {
    v8h part[4];
};
__device__ __forceinline__ Half32 to_half(const v4i (&c)[2])
{
    Half32 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const v2h lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i / 4][i % 4], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i / 4][i % 4], 1.0f, true);
        h.part[i / 2][i % 2 * 4] = lo[0];
        h.part[i / 2][i % 2 * 4 + 1] = lo[1];
        h.part[i / 2][i % 2 * 4 + 2] = hi[0];
        h.part[i / 2][i % 2 * 4 + 3] = hi[1];
    }
    return h;
}

__device__ __forceinline__ v4f mfma_half(const Half32& a, const Half32& b)
{
    v4f p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.part[i], b.part[i], p, 0, 0, 0);
    return p;
}

__device__ __forceinline__ v4f mfma_fp8(const v4i (&a)[2], const v4i (&b)[2])
{
    const v8i a8 = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
    const v8i b8 = {b[0][0], b[0][1], b[0][2], b[0][3], b[1][0], b[1][1], b[1][2], b[1][3]};
    // cbsz = blgp = 0: both operands E4M3; a scale of 2^0 for every 32
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
}

struct Rows {
    int expert, begin, end;    // rows begin .. end - 1 of the output; none: begin == end
};

// The tile-th tile of R rows: tiles never span experts, and those of an expert follow one another.  What the offsets hold is kept within
// the output, whatever it is.
__device__ __forceinline__ Rows find_rows(const Fp8Args& g, int tile, int R)
{
    const int lane = threadIdx.x & 63, T = (int)g.rows;
    int before = 0;
    for (int base = 0; base < g.experts; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0;
        if (e < g.experts) {
            lo = min(max(g.offsets[e], 0), T);
            hi = min(max(g.offsets[e + 1], lo), T);
        }
        const int tiles = (hi - lo + R - 1) / R;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int t = __shfl_up(upto, d);
            if (lane >= d) upto += t;
        }
        const uint64_t here = __ballot(tile < before + upto);
        if (here) {
            const int l = __builtin_ctzll(here);
            const int first = __shfl(lo, l) + (tile - before - __shfl(upto - tiles, l)) * R;
            return Rows{base + l, first, min(first + R, __shfl(hi, l))};
        }
        before += __shfl(upto, 63);
    }
    return Rows{0, 0, 0};
}

// Sixteen columns and 16 TM rows to a workgroup, whose waves take the blocks of K in turn.
template <bool GROUPED, bool OUT_F32, int TM, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void fp8_stream_kernel(Fp8Args g)
{
    __shared__ v4f part[WAVES][TM][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    Rows r{0, 0, 0};
    if constexpr (GROUPED) {
        r = find_rows(g, (int)blockIdx.y, 16 * TM);
    } else {
        r.begin = (int)blockIdx.y * 16 * TM;
        r.end = min(r.begin + 16 * TM, (int)g.rows);
    }
    if (r.begin >= r.end) return;
    const int KB = (int)(g.K >> 7), n0 = (int)blockIdx.x * 16, blocks_n = (int)((g.N + 127) >> 7);
    const uint8_t* w = g.w + ((int64_t)r.expert * g.N + min((int64_t)n0 + (lane & 15), g.N - 1)) * g.K + (lane >> 4) * 16;
    const float* ws = g.w_scales + ((int64_t)r.expert * blocks_n + (n0 >> 7)) * KB;
    const uint8_t* a[TM];
    const float* as[TM];
    bool none[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        int64_t row = min(r.begin + 16 * t + (lane & 15), r.end - 1);
        none[t] = false;
        if (GROUPED && g.index) {
            row = g.index[row];
            none[t] = row < 0 || row >= g.a_rows;   // (a row of zeros)
            if (none[t]) row = 0;
        }
        a[t] = g.a + row * g.K + (lane >> 4) * 16;
        as[t] = g.a_scales + row * KB;
    }
    v4f acc[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) acc[t] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int kb = wave; kb < KB; kb += WAVES) {
        const int64_t at = (int64_t)kb * 128;
        const v4i wf[2] = {*reinterpret_cast<const v4i*>(w + at), *reinterpret_cast<const v4i*>(w + at + 64)};
        const float sw = ws[kb];
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            const v4i af[2] = {*reinterpret_cast<const v4i*>(a[t] + at), *reinterpret_cast<const v4i*>(a[t] + at + 64)};
            const float s = sw * as[t][kb];
            const v4f p = OUT_F32 ? mfma_half(to_half(wf), to_half(af)) : mfma_fp8(wf, af);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(s, p[i], acc[t][i]);
        }
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < TM; t += WAVES) {
        v4f sum = part[0][t][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v][t][lane];
        const int m = r.begin + 16 * t + (lane & 15);
        if (m >= r.end) continue;
        const bool zero = GROUPED && g.index && ((uint32_t)g.index[m] >= (uint64_t)g.a_rows);
        const int64_t n = n0 + (lane >> 4) * 4, o = (int64_t)m * g.N + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i < g.N) {
                const float y = zero ? 0.0f : sum[i];
                if constexpr (OUT_F32) static_cast<float*>(g.out)[o + i] = y;
                else static_cast<__bf16*>(g.out)[o + i] = (__bf16)y;
            }
        }
    }
}

template <bool GROUPED>
hipError_t launch(const Fp8Args& g, bool out_f32, hipStream_t st)
{
    constexpr int TM = 4, WAVES = 8;
    const int64_t tiles = GROUPED ? g.rows / (16 * TM) + std::min<int64_t>(g.experts, g.rows) : (g.rows + 16 * TM - 1) / (16 * TM);
    const dim3 grid((unsigned)((g.N + 15) / 16), (unsigned)tiles);
    if (out_f32) hipLaunchKernelGGL((fp8_stream_kernel<GROUPED, true, TM, WAVES>), grid, dim3(WAVES * 64), 0, st, g);
    else hipLaunchKernelGGL((fp8_stream_kernel<GROUPED, false, TM, WAVES>), grid, dim3(WAVES * 64), 0, st, g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_gemm(const void* a, const float* a_scales, const void* w, const float* w_scales, int64_t M, int64_t N, int64_t K, void* out, bool out_f32,
                           hipStream_t st)
{
    return launch<false>(Fp8Args{static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(w), w_scales, out, M, N, K, M, nullptr, nullptr, 1}, out_f32, st);
}

hipError_t launch_fp8_grouped_gemm(const void* a, const float* a_scales, int64_t a_rows, const void* w, const float* w_scales, const int32_t* offsets,
                                   const int32_t* index, int64_t rows, int64_t experts, int64_t N, int64_t K, void* out, bool out_f32, hipStream_t st)
{
    return launch<true>(Fp8Args{static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(w), w_scales, out, a_rows, N, K, rows, offsets, index, (int)experts},
                        out_f32, st);
}

}  // namespace fp4mr
