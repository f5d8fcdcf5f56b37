// What the quantizers to 8 bits share: bf16 rows eight values at a time, magnitudes' maxima, sums of squares, the gated activation.
#pragma once

#include "device_util.hpp"

namespace fp4mr {
namespace {

constexpr uint32_t kAmaxLeast = 27u << 23;   // 2^-100

typedef __bf16 v8b __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void widen8(const v4i& raw, float (&v)[8])
{
    const v8b t = __builtin_bit_cast(v8b, raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}

// STREAM: read once, past the caches' interest
template <bool STREAM>
__device__ __forceinline__ v4i load16(const __bf16* p)
{
    const v4i* const q = reinterpret_cast<const v4i*>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    else return *q;
}

__device__ __forceinline__ void store8(__bf16* p, const float (&v)[8])
{
    v8b t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (__bf16)v[i];
    __builtin_nontemporal_store(__builtin_bit_cast(v4i, t), reinterpret_cast<v4i*>(p));
}

__device__ __forceinline__ uint32_t amax8(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

// silu(gate) * up
__device__ __forceinline__ float silu_mul(float g, float u)
{
    return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
}

// The lane's number, taken for another one at each use: what an exchange computes from it holds no registers until the next.
__device__ __forceinline__ int own_lane()
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// Largest of the workgroup's values, in all threads.  part: T / 64 words of LDS.
template <int T>
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* part)
{
    const int lane = own_lane();
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__builtin_amdgcn_ds_bpermute((lane ^ d) << 2, (int)m));
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < T / 64; ++i) m = max(m, part[i]);
    }
    return m;
}

// The sum of the workgroup's values, in all threads and in the same order every time: a wave's lanes, the waves.  part: T / 64 words of LDS.
template <int T>
__device__ __forceinline__ float block_sum(float v, float* part)
{
    const int lane = own_lane();
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __int_as_float(__builtin_amdgcn_ds_bpermute((lane ^ d) << 2, __float_as_int(v)));
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < T / 64; ++i) v += part[i];
    }
    return v;
}

// What a row of finite numbers is multiplied with, 1 / sqrt(mean v^2 + eps).  v: the thread's pieces of eight of the row's K numbers, piece c from column (c T + thread) 8 on.  sum: of all squares.
// Where fp32 does not hold the squares (a number beyond 2^64 is enough) or only their upper bits, v is multiplied by a power of two that leaves the larger one of its largest number and sqrt(eps) below one, and the
// result is for that v.  The whole workgroup goes there or none of it.
template <int T, int CH>
__device__ __forceinline__ float row_factor(float (&v)[CH][8], float sum, int K, float eps)
{
    const float mean = sum / (float)K + eps;
    if (mean >= 0x1p-100f && mean <= 3.402823466e38f) return 1.0f / sqrtf(mean);
    __shared__ uint32_t part_max[T / 64];
    __shared__ float part[T / 64];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
        if ((c * T + (int)threadIdx.x) * 8 < K) m = max(m, amax8(v[c]));
    m = block_max<T>(m, part_max);
    const float largest = fmaxf(__uint_as_float(m), sqrtf(eps));
    if (m >= 0x7f800000u || !(largest > 0.0f && largest <= 3.402823466e38f)) return 1.0f / sqrtf(mean);       // not finite, or 0 / 0
    const int e = __builtin_amdgcn_frexp_expf(largest);
    float squares = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float of_piece = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c][i] = __builtin_amdgcn_ldexpf(v[c][i], -e);
            of_piece = fmaf(v[c][i], v[c][i], of_piece);
        }
        squares += (c * T + (int)threadIdx.x) * 8 < K ? of_piece : 0.0f;
    }
    return 1.0f / sqrtf(block_sum<T>(squares, part) / (float)K + __builtin_amdgcn_ldexpf(eps, -2 * e));
}

}  // namespace
}  // namespace fp4mr
