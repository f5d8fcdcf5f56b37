// Operands of the 8-bit integer layers: codes -127 .. 127 with one fp32 scale per row (a token of the activations, a channel of the weights), behind the
// root-mean-square norm, behind silu(gate) * up, or of a tensor as it is.
//
//   s = max(amax, 2^-100) / 127,   code = the integer nearest to v * (127 * (1 / max(amax, 2^-100))), ties to even         amax: the row's largest |v|
//
// v is held in fp32 from the bf16 input to the code, every operation in binary32.  For a bf16 v as it is, the code is that of the exact quotient 127 v / amax but where that lies in the middle of two codes, which may
// go to either with the roundings: with mantissas of eight bits, v = x 2^-s and amax = y (128 <= x, y <= 255, s <= 8 where the quotient is 1/2 or more) the quotient is off the middle of two codes
// by |254 x - (2k + 1) y 2^s| / (2 y 2^s), zero or at least 2^-18 and, of larger quotients, 1/510 of 2^-s, and the three roundings move it by less than 2^-21 of itself (a reciprocal below 2^-126 has 22 bits).
// amax is an integer maximum of bit patterns, which orders infinity above every number and NaN above that: a row that holds one has a scale that is not finite.
#include "bf16_rows.hpp"
#include "internal.hpp"

namespace fp4mr {
namespace {

constexpr float kTop = 127.0f;

// Codes of eight values.  Adding 1.5 * 2^23 rounds to the nearest integer, whose two's complement the sum's low byte is; the product is rounded first, as the definition has it.
__device__ __forceinline__ v2i codes8(const float (&v)[8], float inv)
{
#pragma clang fp contract(off)
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = v[i] * inv;
        b[i] = __float_as_uint(t + 12582912.0f) & 0xffu;
    }
    return v2i{(int)(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24), (int)(b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24)};
}

struct QuantArgs {
    const __bf16* x;
    int64_t x_stride, rows;
    int K;
    uint8_t* codes;
    float* scales;
};

// A row to T threads, CH times eight values in each one's registers: read once, between its statistics and its codes.  What bounds it is memory: 57344 x 8192 227 us (6.2 TB/s; a large copy reaches 6.4), gated rows of
// 4096 x 14336 50 us; of few rows the start-up and one compute unit to a row (1 x 4096 2.8 us, 33 gated ones of 14336 4.9).  Narrow rows have one load to a thread, and up to half of the threads none: 16384 rows of 1024
// columns 12.1 us (4.2 TB/s), 2560 32.2 (3.9), 4096 38.4 (5.2), 4160 41.6 (4.9), 5120 46.7 (5.4), 100000 of 256 27.0 (2.8).
template <int T, int CH, bool SILU>
__global__ __launch_bounds__(T) void int8_quantize_kernel(QuantArgs a)
{
    __shared__ uint32_t part[T / 64];
    const int64_t row = blockIdx.x;
    const __bf16* const x = a.x + row * a.x_stride;
    v4i g[CH], u[SILU ? CH : 1];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = min((c * T + (int)threadIdx.x) * 8, a.K - 8);      // (past the row's end its last eight again)
        g[c] = load16<true>(x + col);
        if constexpr (SILU) u[c] = load16<true>(x + a.K + col);
    }
    float v[CH][8];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        widen8(g[c], v[c]);
        if constexpr (SILU) {
            float f[8];
            widen8(u[c], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = silu_mul(v[c][i], f[i]);
        }
        m = max(m, amax8(v[c]));
    }
    const float amax = __uint_as_float(max(block_max<T>(m, part), kAmaxLeast)), inv = kTop * (1.0f / amax);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * T + (int)threadIdx.x) * 8;
        if (col < a.K) *reinterpret_cast<v2i*>(a.codes + row * a.K + col) = codes8(v[c], inv);
    }
    if (threadIdx.x == 0) a.scales[row] = amax / kTop;
}

// Rows that registers do not hold: read twice, the second time mostly from the caches.
template <bool SILU>
__global__ __launch_bounds__(1024) void int8_quantize_long_kernel(QuantArgs a)
{
    __shared__ uint32_t part[16];
    const int64_t row = blockIdx.x;
    const __bf16* const x = a.x + row * a.x_stride;
    auto values = [&](int col, float (&v)[8]) {
        widen8(load16<false>(x + col), v);
        if constexpr (SILU) {
            float f[8];
            widen8(load16<false>(x + a.K + col), f);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = silu_mul(v[i], f[i]);
        }
    };
    uint32_t m = 0;
    for (int col = (int)threadIdx.x * 8; col < a.K; col += 8192) {
        float v[8];
        values(col, v);
        m = max(m, amax8(v));
    }
    const float amax = __uint_as_float(max(block_max<1024>(m, part), kAmaxLeast)), inv = kTop * (1.0f / amax);
    for (int col = (int)threadIdx.x * 8; col < a.K; col += 8192) {
        float v[8];
        values(col, v);
        *reinterpret_cast<v2i*>(a.codes + row * a.K + col) = codes8(v, inv);
    }
    if (threadIdx.x == 0) a.scales[row] = amax / kTop;
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

// The same behind the norm: a row is read once and stays in registers from the sum of its squares to its codes.  The sum is formed in the same order every time: a thread's values, a wave's lanes, the waves.
// Bound by memory (4095 x 8192 with residual 43 us on buffers in turn, 134 MB in and 101 out, 5.4 TB/s; 36 where the caches have part of it), for one row by its start-up (4096 columns 2.5 us).
template <int T, int CH, bool RESIDUAL>
__global__ __launch_bounds__(T) void int8_rmsnorm_kernel(NormArgs a)
{
    __shared__ float part[T / 64];
    __shared__ uint32_t part_max[T / 64];
    const int64_t row = blockIdx.x;
    v4i x[CH], r[CH], w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = min((c * T + (int)threadIdx.x) * 8, a.K - 8);
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
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * T + (int)threadIdx.x) * 8;
        float f[8];
        widen8(w[c], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * rstd * f[i];
        if (col >= a.K) continue;          // (past the row's end its last eight were read again, perhaps after another wave has stored their sums there)
        if (a.norm_out) store8(a.norm_out + row * a.K + col, v[c]);
        m = max(m, amax8(v[c]));
    }
    const float amax = __uint_as_float(max(block_max<T>(m, part_max), kAmaxLeast)), inv = kTop * (1.0f / amax);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * T + (int)threadIdx.x) * 8;
        if (col < a.K) *reinterpret_cast<v2i*>(a.codes + row * a.K + col) = codes8(v[c], inv);
    }
    if (threadIdx.x == 0) a.scales[row] = amax / kTop;
}

// (a launch takes fewer than 2^32 threads: very many rows in several)
constexpr int64_t kRowsEach = 1 << 21;

// launch(first row, rows)
template <typename F>
hipError_t in_runs(int64_t rows, F launch)
{
    for (int64_t at = 0; at < rows; at += kRowsEach) {
        launch(at, rows - at < kRowsEach ? rows - at : kRowsEach);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int T, int CH>
hipError_t launch_quantize(const QuantArgs& q, bool silu, hipStream_t st)
{
    return in_runs(q.rows, [&](int64_t at, int64_t n) {
        QuantArgs a = q;
        a.x += at * a.x_stride;
        a.codes += at * a.K;
        a.scales += at;
        if constexpr (CH == 0) {
            if (silu) hipLaunchKernelGGL(int8_quantize_long_kernel<true>, dim3((unsigned)n), dim3(1024), 0, st, a);
            else hipLaunchKernelGGL(int8_quantize_long_kernel<false>, dim3((unsigned)n), dim3(1024), 0, st, a);
        } else {
            if (silu) hipLaunchKernelGGL((int8_quantize_kernel<T, CH, true>), dim3((unsigned)n), dim3(T), 0, st, a);
            else hipLaunchKernelGGL((int8_quantize_kernel<T, CH, false>), dim3((unsigned)n), dim3(T), 0, st, a);
        }
    });
}

template <int T, int CH>
hipError_t launch_norm(const NormArgs& q, hipStream_t st)
{
    return in_runs(q.rows, [&](int64_t at, int64_t n) {
        NormArgs a = q;
        a.x += at * a.x_stride;
        if (a.residual) {
            a.residual += at * a.K;
            a.residual_out += at * a.K;
        }
        if (a.norm_out) a.norm_out += at * a.K;
        a.codes += at * a.K;
        a.scales += at;
        if (a.residual) hipLaunchKernelGGL((int8_rmsnorm_kernel<T, CH, true>), dim3((unsigned)n), dim3(T), 0, st, a);
        else hipLaunchKernelGGL((int8_rmsnorm_kernel<T, CH, false>), dim3((unsigned)n), dim3(T), 0, st, a);
    });
}

}  // namespace

hipError_t launch_int8_quantize(const void* x, int64_t x_stride, int64_t rows, int64_t K, bool silu, void* codes, float* scales, hipStream_t st)
{
    const QuantArgs a{static_cast<const __bf16*>(x), x_stride, rows, (int)K, static_cast<uint8_t*>(codes), scales};
    // as many threads as there are pieces of eight, up to 512, then two pieces to each; longer rows need 1024 threads for their registers
    const int64_t n8 = K / 8;
    if (n8 <= 64) return launch_quantize<64, 1>(a, silu, st);
    if (n8 <= 128) return launch_quantize<128, 1>(a, silu, st);
    if (n8 <= 256) return launch_quantize<256, 1>(a, silu, st);
    if (n8 <= 512) return launch_quantize<512, 1>(a, silu, st);
    if (n8 <= 1024) return launch_quantize<512, 2>(a, silu, st);
    if (n8 <= 2048) return launch_quantize<1024, 2>(a, silu, st);
    if (n8 <= 4096) return launch_quantize<1024, 4>(a, silu, st);
    return launch_quantize<0, 0>(a, silu, st);
}

hipError_t launch_int8_rmsnorm_quantize(const void* x, int64_t x_stride, const void* residual, const void* weight, int64_t rows, int64_t K, float eps,
                                        void* codes, float* scales, void* residual_out, void* norm_out, hipStream_t st)
{
    const NormArgs a{static_cast<const __bf16*>(x), static_cast<const __bf16*>(residual), static_cast<const __bf16*>(weight), static_cast<__bf16*>(residual_out),
                     static_cast<__bf16*>(norm_out), static_cast<uint8_t*>(codes), scales, x_stride, rows, (int)K, eps};
    const int64_t n8 = K / 8;
    if (n8 <= 64) return launch_norm<64, 1>(a, st);
    if (n8 <= 128) return launch_norm<128, 1>(a, st);
    if (n8 <= 256) return launch_norm<256, 1>(a, st);
    if (n8 <= 512) return launch_norm<512, 1>(a, st);
    if (n8 <= 1024) return launch_norm<512, 2>(a, st);
    if (n8 <= 2048) return launch_norm<1024, 2>(a, st);
    if (n8 <= 4096) return launch_norm<1024, 4>(a, st);
    return launch_norm<1024, 8>(a, st);
}

}  // namespace fp4mr
