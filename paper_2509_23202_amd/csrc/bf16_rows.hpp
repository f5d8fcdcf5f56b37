// What the quantizers to 8 bits share: bf16 rows eight values at a time, magnitudes' maxima, the gated activation.
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

}  // namespace
}  // namespace fp4mr
