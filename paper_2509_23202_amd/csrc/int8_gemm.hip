// Products of 8-bit integer operands, for one weight matrix or for rows grouped by expert.
//
//   out[m,n] = (float(sum_k a[m,k] w[n,k]) * sa[m]) * sw[n]
//
// The sum is exact: v_mfma_i32_16x16x64_i8 adds in 32 bits, and 2^14 K is less than 2^31 for the K that the entry points take.  So no order of it, and no split of K, changes a
// bit of the result.  The W codes are the MFMA's A operand and the activations its B operand: a lane then has four consecutive n of one m.  What lies past K is
// zero in W, and may be anything in A.
#include "product_tiles.hpp"

#include <algorithm>

namespace fp4mr {
namespace {

struct Int8Args {
    const int8_t* a;
    const float* a_scales;
    const int8_t* w;
    const float* w_scales;
    void* out;
    int64_t a_rows, N, K;      // a_rows: rows of A
    int64_t rows;              // rows of the output
    const int32_t* offsets;    // grouped: experts + 1 of them
    const int32_t* index;      // grouped: row of A for a row of the output, or null
    int experts;
};

// A 64 x 64 tile to a workgroup of four waves, each 32 x 32; 64 columns of both operands in LDS to a step.
template <bool GROUPED, bool OUT_F32>
__global__ __launch_bounds__(256) void int8_simple_kernel(Int8Args g, int tiles_m, int tiles_n)
{
    __shared__ __attribute__((aligned(16))) char smem[2][64 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    ExpertTiles experts{0, 0, 0};
    if constexpr (GROUPED) {
        experts = expert_tiles(g, 0, 64);
        tiles_m = count_tiles(g, experts, 64, tiles_m);
    }
    for (int64_t tile = blockIdx.x; tile < (int64_t)tiles_m * tiles_n; tile += gridDim.x) {
    const int tm = (int)(tile / tiles_n), n0 = (int)(tile - (int64_t)tm * tiles_n) * 64;
    Rows r{0, tm * 64, min((tm + 1) * 64, (int)g.rows)};
    if constexpr (GROUPED) r = find_tile(g, experts, tm, 64);
    const bool gather = GROUPED && g.index != nullptr;
    auto a_row = [&](int m) -> int64_t {      // of A, or -1
        if (r.begin + m >= r.end) return -1;
        const int64_t row = gather ? g.index[r.begin + m] : r.begin + m;
        return row >= 0 && row < g.a_rows ? row : -1;
    };
    const int row = threadIdx.x / 4, piece = threadIdx.x % 4;
    const int64_t ar = a_row(row), wr = (int64_t)r.expert * g.N + n0 + row;
    const bool have_w = n0 + row < g.N;
    v4i acc[2][2] = {};
    for (int64_t k = 0; k < g.K; k += 64) {
        const bool in = k + piece * 16 < g.K;
        v4i x{0, 0, 0, 0}, w{0, 0, 0, 0};
        if (in && ar >= 0) x = *reinterpret_cast<const v4i*>(g.a + ar * g.K + k + piece * 16);
        if (in && have_w) w = *reinterpret_cast<const v4i*>(g.w + wr * g.K + k + piece * 16);
        __syncthreads();
        *reinterpret_cast<v4i*>(smem[0] + row * 64 + piece * 16) = x;
        *reinterpret_cast<v4i*>(smem[1] + row * 64 + piece * 16) = w;
        __syncthreads();
        v4i xf[2], wf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            xf[i] = *reinterpret_cast<const v4i*>(smem[0] + ((wave & 1) * 32 + i * 16 + (lane & 15)) * 64 + lane / 16 * 16);
            wf[i] = *reinterpret_cast<const v4i*>(smem[1] + ((wave >> 1) * 32 + i * 16 + (lane & 15)) * 64 + lane / 16 * 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = (wave & 1) * 32 + i * 16 + (lane & 15);
        if (r.begin + m >= r.end) continue;
        const int64_t from = a_row(m);
        const float sa = from >= 0 ? g.a_scales[from] : 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = n0 + (wave >> 1) * 32 + j * 16 + lane / 16 * 4 + e;
                if (n >= g.N) continue;
                const float y = (float)acc[i][j][e] * sa * g.w_scales[(int64_t)r.expert * g.N + n];
                const int64_t to = (int64_t)(r.begin + m) * g.N + n;
                if constexpr (OUT_F32) static_cast<float*>(g.out)[to] = y;
                else static_cast<__bf16*>(g.out)[to] = (__bf16)y;
            }
    }
    }
}

template <bool GROUPED, bool OUT_F32>
hipError_t launch(const Int8Args& g, hipStream_t st)
{
    const int64_t tiles_m = GROUPED ? g.rows / 64 + std::min<int64_t>(g.experts, g.rows) : (g.rows + 63) / 64, tiles_n = (g.N + 63) / 64;
    hipLaunchKernelGGL((int8_simple_kernel<GROUPED, OUT_F32>), dim3((unsigned)std::min<int64_t>(tiles_m * tiles_n, 1 << 20)), dim3(256), 0, st, g, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

}  // namespace

size_t int8_gemm_partial_bytes(int64_t M, int64_t N, int64_t K) { return 0; }

hipError_t launch_int8_gemm(const void* a, const float* a_scales, const void* w, const float* w_scales, int64_t M, int64_t N, int64_t K, void* out, bool out_f32,
                            void* partial, size_t room, hipStream_t st)
{
    const Int8Args g{static_cast<const int8_t*>(a), a_scales, static_cast<const int8_t*>(w), w_scales, out, M, N, K, M, nullptr, nullptr, 1};
    return out_f32 ? launch<false, true>(g, st) : launch<false, false>(g, st);
}

hipError_t launch_int8_grouped_gemm(const void* a, const float* a_scales, int64_t a_rows, const void* w, const float* w_scales, const int32_t* offsets,
                                    const int32_t* index, int64_t rows, int64_t experts, int64_t N, int64_t K, void* out, bool out_f32, hipStream_t st)
{
    const Int8Args g{static_cast<const int8_t*>(a), a_scales, static_cast<const int8_t*>(w), w_scales, out, a_rows, N, K, rows, offsets, index, (int)experts};
    return out_f32 ? launch<true, true>(g, st) : launch<true, false>(g, st);
}

}  // namespace fp4mr
