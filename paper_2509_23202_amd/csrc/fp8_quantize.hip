// Operands of the 8-bit linear layers: E4M3 codes with one fp32 scale per 128 columns of a row (activations) or per 128 x 128 block
// (weights), behind the root-mean-square norm, behind silu(gate) * up, or of a tensor as it is.
//
//   s = max(amax, 2^-100) / 448,   code = e4m3(v * (448 / max(amax, 2^-100)))          amax: the block's largest |v|
//
// v is held in fp32 from the bf16 input to the code, which is the only rounding to fewer bits (but for the bf16 copies that a caller
// asks for).  2^-100 keeps the reciprocal finite and gives a block of zeros the code 0 and a finite scale.  amax is an integer maximum
// of the magnitudes' bit patterns, which orders infinity above every number and NaN above that: a block that holds one has the scale
// infinity or NaN, and every product with it is NaN.
#include "bf16_rows.hpp"
#include "internal.hpp"

namespace fp4mr {
namespace {

constexpr float kE4m3Max = 448.0f;

// Largest value among the sixteen lanes that hold a block of 128, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));    // quad_perm [1,0,3,2]
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true));    // quad_perm [2,3,0,1]
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xf, 0xf, true));   // row_ror 4
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xf, 0xf, true));   // row_ror 8
    return m;
}

__device__ __forceinline__ v2i codes8(const float (&v)[8], float inv)
{
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    return v2i{lo, hi};
}

// Codes of a lane's eight values of a block, and the block's scale from its first lane.
__device__ __forceinline__ void quantize8(const float (&v)[8], uint8_t* codes, float* scale, int lane)
{
    const float amax = __uint_as_float(max(max16(amax8(v)), kAmaxLeast));
    *reinterpret_cast<v2i*>(codes) = codes8(v, kE4m3Max / amax);
    if ((lane & 15) == 0) *scale = amax / kE4m3Max;
}

struct QuantArgs {
    const __bf16* x;
    int64_t x_stride, rows, K;
    uint8_t* codes;
    float* scales;
};

// Sixteen lanes to a block of 128, in the order of the outputs: 16-byte loads, a maximum in four lane exchanges, whole lines of codes.  Memory bounds it: gated 4096 x 14336 takes 47 us,
// 6.3 TB/s, what a copy reaches; 33 x 14336 takes 2.5 to 2.9, a launch's, and 4096 x 8192 as it is 21, 4.8 TB/s.  (Loads past the caches: an input is read once.)
template <bool SILU>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(QuantArgs a)
{
    const int64_t per_row = a.K / 8, total = a.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row, col = (i - row * per_row) * 8;
        const __bf16* x = a.x + row * a.x_stride + col;
        float v[8];
        widen8(load16<true>(x), v);
        if constexpr (SILU) {
            float u[8];
            widen8(load16<true>(x + a.K), u);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = silu_mul(v[j], u[j]);
        }
        quantize8(v, a.codes + i * 8, a.scales + i / 16, threadIdx.x);
    }
}

struct NormArgs {
    const __bf16* x;
    const __bf16* residual;       // or null
    const __bf16* weight;
    __bf16* residual_out;
    __bf16* norm_out;             // or null
    uint8_t* codes;
    float* scales;
    int64_t x_stride, rows;
    int K;
    float eps;
};

// A row to T threads, CH times eight values in each one's registers from the sum of squares to the codes, so that a row is read once; all of a thread's loads are on
// their way before the first is needed.  The sum is formed in the same order every time: a thread's values, a wave's lanes, the waves.  The 16-bit copies are stored past the caches
// (512 x 4096 takes 4.9 us so, 6.3 with ordinary stores; 4095 x 8192 54.7 and 56.8, on buffers in turn).  Memory bounds it: 4095 x 8192 with residual and both copies takes 50 to 55 us,
// 5.5 to 6.0 TB/s where a copy reaches 6.3; 1 x 4096 takes 2.2 to 2.7, a launch's.
template <int T, int CH, bool RESIDUAL>
__global__ __launch_bounds__(T) void fp8_rmsnorm_kernel(NormArgs a)
{
    __shared__ float part[T / 64];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63;
    v4i x[CH], r[CH], w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = min((c * T + (int)threadIdx.x) * 8, a.K - 8);      // (past the row's end its last eight again)
        x[c] = load16<false>(a.x + row * a.x_stride + col);
        if constexpr (RESIDUAL) r[c] = load16<false>(a.residual + row * a.K + col);
        w[c] = load16<false>(a.weight + col);
    }
    float v[CH][8];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * T + (int)threadIdx.x) * 8;
        widen8(x[c], v[c]);
        if constexpr (RESIDUAL) {
            float f[8];
            widen8(r[c], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = (float)(__bf16)(v[c][i] + f[i]);   // the stream that is kept is the one that is normed
            if (col < a.K) store8(a.residual_out + row * a.K + col, v[c]);
        }
        float part_sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) part_sum = fmaf(v[c][i], v[c][i], part_sum);
        sum += col < a.K ? part_sum : 0.0f;
    }
    const float rstd = row_factor<T, CH>(v, block_sum<T>(sum, part), a.K, a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * T + (int)threadIdx.x) * 8;
        if (col < a.K) {   // (whole blocks of sixteen lanes)
            float f[8];
            widen8(w[c], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * rstd * f[i];
            if (a.norm_out) store8(a.norm_out + row * a.K + col, v[c]);
            quantize8(v[c], a.codes + row * a.K + col, a.scales + row * (a.K / 128) + col / 128, lane);
        }
    }
}

struct WeightArgs {
    const __bf16* w;
    int64_t N, K;
    int blocks_n, blocks_k;
    uint8_t* codes;
    float* scales;
};

// A 128 x 128 block to a workgroup, in its threads' registers between its maximum and its codes: sixteen lanes to a row's 128, eight rows to a thread.  Memory bounds it: 57344 x 8192 takes
// 234 us, 6.0 TB/s (265 with ordinary loads and stores: both ends are read or written once).
__global__ __launch_bounds__(256) void fp8_quantize_weights_kernel(WeightArgs a)
{
    __shared__ uint32_t part[4];
    const int64_t block = blockIdx.x;
    const int64_t bk = block % a.blocks_k, en = block / a.blocks_k, expert = en / a.blocks_n, bn = en % a.blocks_n;
    const int64_t row0 = bn * 128 + threadIdx.x / 16, at = (expert * a.N + row0) * a.K + bk * 128 + (threadIdx.x % 16) * 8;
    float v[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        if (row0 + 16 * r < a.N) {
            widen8(load16<true>(a.w + at + 16 * r * a.K), v[r]);
            m = max(m, amax8(v[r]));
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(part[0], part[1]), max(part[2], part[3]));
    const float amax = __uint_as_float(max(m, kAmaxLeast)), inv = kE4m3Max / amax;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (row0 + 16 * r < a.N) __builtin_nontemporal_store(codes8(v[r], inv), reinterpret_cast<v2i*>(a.codes + at + 16 * r * a.K));
    if (threadIdx.x == 0) a.scales[block] = amax / kE4m3Max;
}

// (a launch takes fewer than 2^32 threads: very many rows in several)
constexpr int64_t kNormRows = 1 << 21;

template <int T, int CH>
hipError_t launch_norm(NormArgs a, hipStream_t st)
{
    for (int64_t left = a.rows; left > 0; left -= kNormRows) {
        const dim3 grid((unsigned)(left < kNormRows ? left : kNormRows));
        if (a.residual) hipLaunchKernelGGL((fp8_rmsnorm_kernel<T, CH, true>), grid, dim3(T), 0, st, a);
        else hipLaunchKernelGGL((fp8_rmsnorm_kernel<T, CH, false>), grid, dim3(T), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x += kNormRows * a.x_stride;
        if (a.residual) {
            a.residual += kNormRows * a.K;
            a.residual_out += kNormRows * a.K;
        }
        if (a.norm_out) a.norm_out += kNormRows * a.K;
        a.codes += kNormRows * a.K;
        a.scales += kNormRows * (a.K / 128);
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_fp8_quantize(const void* x, int64_t x_stride, int64_t rows, int64_t K, bool silu, void* codes, float* scales, hipStream_t st)
{
    const QuantArgs a{static_cast<const __bf16*>(x), x_stride, rows, K, static_cast<uint8_t*>(codes), scales};
    const int64_t blocks = (rows * K / 8 + 255) / 256, most = (int64_t)compute_units() * 64;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (silu) hipLaunchKernelGGL(fp8_quantize_kernel<true>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(fp8_quantize_kernel<false>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_fp8_rmsnorm_quantize(const void* x, int64_t x_stride, const void* residual, const void* weight, int64_t rows, int64_t K, float eps,
                                       void* codes, float* scales, void* residual_out, void* norm_out, hipStream_t st)
{
    const NormArgs a{static_cast<const __bf16*>(x), static_cast<const __bf16*>(residual), static_cast<const __bf16*>(weight), static_cast<__bf16*>(residual_out),
                     static_cast<__bf16*>(norm_out), static_cast<uint8_t*>(codes), scales, x_stride, rows, (int)K, eps};
    // Eight values to a thread while a row then has 512 threads at most (4095 x 4096: 28.5 us, with sixteen 29.4), or where there is a row or less to a compute unit (256 x 8192:
    // 4.9 and 5.0, 1 x 8192 3.1 and 3.2); else sixteen (4095 x 8192: 54.7, with eight 55.2; 1024 x 8192 16.3 and 17.0), and more where a row needs them.
    const int64_t n8 = K / 8;
    if (n8 <= 64) return launch_norm<64, 1>(a, st);
    if (n8 <= 128) return launch_norm<128, 1>(a, st);
    if (n8 <= 256) return launch_norm<256, 1>(a, st);
    if (n8 <= 512) return launch_norm<512, 1>(a, st);
    if (n8 <= 1024 && rows <= compute_units()) return launch_norm<1024, 1>(a, st);
    if (n8 <= 1024) return launch_norm<512, 2>(a, st);
    if (n8 <= 2048) return launch_norm<1024, 2>(a, st);
    if (n8 <= 4096) return launch_norm<1024, 4>(a, st);
    return launch_norm<1024, 8>(a, st);
}

hipError_t launch_fp8_quantize_weights(const void* w, int64_t experts, int64_t N, int64_t K, void* codes, float* scales, hipStream_t st)
{
    WeightArgs a{static_cast<const __bf16*>(w), N, K, (int)((N + 127) / 128), (int)(K / 128), static_cast<uint8_t*>(codes), scales};
    hipLaunchKernelGGL(fp8_quantize_weights_kernel, dim3((unsigned)(experts * a.blocks_n * a.blocks_k)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace fp4mr
