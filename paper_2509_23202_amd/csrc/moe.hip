// A router's choice of experts, and the experts' outputs added up for each token.
//
//   s = softmax(z) or sigmoid(z),  c = z where there is neither a bias nor a sum of scores to compare, else s + bias
//   of `groups` runs of experts the top_groups best ones are kept (a run counts as its largest c, or the sum of its two largest), of their experts the `top` best: (c, lower index first)
//   weight = scale s of the chosen, or scale s / sum of the chosen
//
// Which of two experts is the better one hangs on c alone.  Without a bias the order of the scores is that of the logits, which are compared as they are.  Otherwise c is formed in binary64: whole tokens would
// go elsewhere with the last bit of an exponential, and a choice could not be checked against any other arithmetic.
//
// The chosen pairs (token, place among its choices) are then sorted by expert, stably, so that an expert's rows are in the order of the tokens: counts of each expert for each run of tokens, a
// sum over the runs in front and the experts in front, and the rank within the run.  No atomic's order reaches a result.
#include "device_util.hpp"
#include "internal.hpp"

#include <algorithm>

namespace fp4mr {
namespace {

struct RouteArgs {
    const void* logits;
    int64_t stride;
    const float* bias;         // or null
    int64_t tokens;
    int experts, top, groups, top_groups;
    float scale;
    float* weights;
    int32_t* chosen;
    int32_t* offsets;
    int32_t* rows;
    int32_t* places;
    int32_t* counts;           // [runs, experts]
    int run, runs;             // tokens of a run
    bool sigmoid, renorm, sum2;
};

typedef unsigned long long u64;

// Numbers in their order as unsigned ones, zeros of both signs alike; 0: below every number.
__device__ __forceinline__ u64 order_of(double c)
{
    const long long b = __double_as_longlong(c + 0.0);
    return (u64)(b ^ (b >> 63 | (long long)(1ull << 63)));
}
__device__ __forceinline__ double of_order(u64 k)
{
    const long long b = (long long)k;
    return __longlong_as_double(b ^ (~(b >> 63) | (long long)(1ull << 63)));
}

__device__ __forceinline__ u64 wave_max(u64 v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}
template <typename F>
__device__ __forceinline__ F wave_sum(F v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// A token to a wave: expert 64 i + lane is the lane's i-th.  keys: EACH * 64 words of LDS of the wave's own, for groups.
template <int EACH, bool F32>
__device__ void route_token(const RouteArgs& a, int64_t t, u64* keys)
{
    const int lane = threadIdx.x & 63;
    double z[EACH], s[EACH];
    u64 key[EACH];
    double most = -__builtin_inf();
    bool bad = false;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = 64 * i + lane;
        z[i] = -__builtin_inf();
        if (e < a.experts) {
            if constexpr (F32) z[i] = static_cast<const float*>(a.logits)[t * a.stride + e];
            else z[i] = (float)static_cast<const __bf16*>(a.logits)[t * a.stride + e];
            bad |= z[i] != z[i] || (!a.sigmoid && z[i] == __builtin_inf()) || (a.bias && a.bias[e] != a.bias[e]);
        }
        most = fmax(most, z[i]);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmax(most, __shfl_xor(most, d));
    bad = __any(bad);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        s[i] = z[i] == -__builtin_inf() ? 0.0 : a.sigmoid ? 1.0 / (1.0 + exp(-z[i])) : exp(z[i] - most);
        sum += s[i];
    }
    if (!a.sigmoid) {
        sum = wave_sum(sum);
#pragma unroll
        for (int i = 0; i < EACH; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
    }
    const bool by_score = a.bias || (a.groups > 1 && a.sum2);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = 64 * i + lane;
        const double c = !by_score ? z[i] : a.bias && e < a.experts ? s[i] + (double)a.bias[e] : s[i];
        key[i] = z[i] == -__builtin_inf() || c == -__builtin_inf() || bad ? 0 : order_of(c);
    }
    if (a.groups > 1) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) keys[64 * i + lane] = key[i];
        __builtin_amdgcn_wave_barrier();
        const int size = a.experts / a.groups;
        u64 mark = 0;
        if (lane < a.groups) {
            u64 first = 0, second = 0;
            for (int j = 0; j < size; ++j) {
                const u64 k = keys[lane * size + j];
                second = k > first ? first : k > second ? k : second;
                first = k > first ? k : first;
            }
            mark = first == 0 || !a.sum2 ? first : order_of(second ? of_order(first) + of_order(second) : of_order(first));
        }
        u64 kept = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            const u64 best = wave_max(mark);
            if (best == 0) break;
            const int g = __builtin_ctzll(__ballot(mark == best));
            kept |= 1ull << g;
            if (lane == g) mark = 0;
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (!(kept >> (min(64 * i + lane, a.experts - 1) / size) & 1)) key[i] = 0;
        __builtin_amdgcn_wave_barrier();
    }
    int mine = -1;             // lane j: the j-th choice, and its score
    double score = 0.0;
    for (int j = 0; j < a.top; ++j) {
        u64 best = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) best = key[i] > best ? key[i] : best;
        best = wave_max(best);
        if (best == 0) break;
        int e = -1;
        double of = 0.0;
#pragma unroll
        for (int i = EACH - 1; i >= 0; --i) {
            const u64 have = __ballot(key[i] == best);
            if (have) {
                const int l = __builtin_ctzll(have);
                e = 64 * i + l;
                of = __shfl(s[i], l);
            }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (64 * i + lane == e) key[i] = 0;
        if (lane == j) {
            mine = e;
            score = of;
        }
    }
    if (a.renorm) score /= fmax(wave_sum(score), 0x1p-100);
    if (lane < a.top) {
        a.weights[t * a.top + lane] = bad ? __builtin_nanf("") : (float)(score * (double)a.scale);
        a.chosen[t * a.top + lane] = mine;
    }
}

template <int EACH, bool F32>
__global__ __launch_bounds__(256) void moe_route_kernel(RouteArgs a)
{
    __shared__ u64 keys[4][EACH * 64];
    const int wave = threadIdx.x >> 6;
    for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < a.tokens; t += (int64_t)gridDim.x * 4) route_token<EACH, F32>(a, t, keys[wave]);
}

// How often each expert was chosen in a run of tokens.
__global__ __launch_bounds__(256) void moe_count_kernel(RouteArgs a)
{
    extern __shared__ int32_t count[];
    for (int e = threadIdx.x; e < a.experts; e += 256) count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.run * a.top, end = min(first + (int64_t)a.run * a.top, a.tokens * a.top);
    for (int64_t f = first + threadIdx.x; f < end; f += 256) {
        const int e = a.chosen[f];
        if (e >= 0) atomicAdd(count + e, 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 256) a.counts[(int64_t)blockIdx.x * a.experts + e] = count[e];
}

// Where the rows of a run of tokens lie: one wave, 64 choices at a time.
__global__ __launch_bounds__(256) void moe_place_kernel(RouteArgs a)
{
    extern __shared__ int32_t at[];           // [experts]: of each expert the next row; [experts]: its rows in all
    int32_t* const total = at + a.experts;
    for (int e = threadIdx.x; e < a.experts; e += 256) {
        int before = 0, all = 0;
        for (int b = 0; b < a.runs; ++b) {
            const int n = a.counts[(int64_t)b * a.experts + e];
            before += b < (int)blockIdx.x ? n : 0;
            all += n;
        }
        at[e] = before;
        total[e] = all;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int lane = threadIdx.x;
    int front = 0;
    for (int base = 0; base < a.experts; base += 64) {
        const int e = base + lane, n = e < a.experts ? total[e] : 0;
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        if (e < a.experts) {
            at[e] += front + upto - n;
            if (blockIdx.x == 0) a.offsets[e] = front + upto - n;
        }
        front += __shfl(upto, 63);
    }
    if (blockIdx.x == 0 && lane == 0) a.offsets[a.experts] = front;
    const int64_t first = (int64_t)blockIdx.x * a.run * a.top, end = min(first + (int64_t)a.run * a.top, a.tokens * a.top);
    for (int64_t f0 = first; f0 < end; f0 += 64) {
        const int64_t f = f0 + lane;
        const int e = f < end ? a.chosen[f] : -1;
        u64 same = __ballot(e >= 0);
        for (int bit = 0; bit < 10; ++bit) {
            const u64 set = __ballot(e >> bit & 1);
            same &= e >> bit & 1 ? set : ~set;
        }
        if (e >= 0) {
            const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
            const int row = at[e] + rank;
            a.rows[row] = (int32_t)(f / a.top);
            a.places[f] = row;
            __builtin_amdgcn_wave_barrier();
            if ((same >> lane) == 1) at[e] = row + 1;
        } else if (f < end) {
            a.places[f] = -1;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

struct CombineArgs {
    const void* y;
    int64_t y_rows;
    const int32_t* places;
    const float* weights;
    const void* shared;        // or null
    void* out;
    int64_t tokens, cols;
    int top;
    bool y_f32, shared_f32, out_f32;
};

__device__ __forceinline__ float element(const void* p, int64_t i, bool f32) { return f32 ? static_cast<const float*>(p)[i] : (float)static_cast<const __bf16*>(p)[i]; }

// out[t] = shared[t] + sum_j weight[t,j] y[place[t,j]], in fp32 in the order of the choices.  A choice without a row adds its weight times zero.
__global__ __launch_bounds__(256) void moe_combine_kernel(CombineArgs a)
{
    const int64_t total = a.tokens * a.cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / a.cols, c = i - t * a.cols;
        float sum = a.shared ? element(a.shared, i, a.shared_f32) : 0.0f;
        for (int j = 0; j < a.top; ++j) {
            const int64_t row = a.places[t * a.top + j];
            const float w = a.weights[t * a.top + j];
            sum = fmaf(w, row >= 0 && row < a.y_rows ? element(a.y, row * a.cols + c, a.y_f32) : 0.0f, sum);
        }
        if (a.out_f32) static_cast<float*>(a.out)[i] = sum;
        else static_cast<__bf16*>(a.out)[i] = (__bf16)sum;
    }
}

// Tokens of a run and runs: as many runs as there are compute units at most, so that every workgroup that places rows can read all counts.
void runs_of(int64_t tokens, int& run, int& runs)
{
    const int64_t least = 16, most = 256;
    run = (int)std::max<int64_t>(least, (tokens + most - 1) / most);
    runs = (int)((tokens + run - 1) / run);
}

template <int EACH>
void route(const RouteArgs& a, bool f32, hipStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>((a.tokens + 3) / 4, 1 << 20));
    if (f32) hipLaunchKernelGGL((moe_route_kernel<EACH, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((moe_route_kernel<EACH, false>), grid, dim3(256), 0, st, a);
}

}  // namespace

size_t moe_count_bytes(int64_t tokens, int64_t experts)
{
    int run, runs;
    runs_of(tokens, run, runs);
    return (size_t)runs * experts * 4;
}

hipError_t launch_moe_route(const void* logits, int64_t stride, bool f32, const float* bias, int64_t tokens, int64_t experts, int64_t top, int64_t groups, int64_t top_groups, float scale,
                            bool sigmoid, bool renorm, bool sum2, float* weights, int32_t* chosen, int32_t* offsets, int32_t* rows, int32_t* places, void* counts, hipStream_t st)
{
    RouteArgs a{logits, stride, bias, tokens, (int)experts, (int)top, (int)groups, (int)top_groups, scale, weights, chosen, offsets, rows, places, static_cast<int32_t*>(counts), 0, 0,
                sigmoid, renorm, sum2};
    runs_of(tokens, a.run, a.runs);
    if (tokens > 0) {
        if (experts <= 64) route<1>(a, f32, st);
        else if (experts <= 128) route<2>(a, f32, st);
        else if (experts <= 256) route<4>(a, f32, st);
        else if (experts <= 512) route<8>(a, f32, st);
        else route<16>(a, f32, st);
        if (const hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(moe_count_kernel, dim3(a.runs), dim3(256), experts * 4, st, a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    hipLaunchKernelGGL(moe_place_kernel, dim3(std::max(a.runs, 1)), dim3(256), experts * 8, st, a);
    return hipGetLastError();
}

hipError_t launch_moe_combine(const void* y, int64_t y_rows, bool y_f32, const int32_t* places, const float* weights, const void* shared, bool shared_f32, int64_t tokens, int64_t top,
                              int64_t cols, void* out, bool out_f32, hipStream_t st)
{
    const CombineArgs a{y, y_rows, places, weights, shared, out, tokens, cols, (int)top, y_f32, shared_f32, out_f32};
    hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)std::min<int64_t>((tokens * cols + 255) / 256, 1 << 20)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace fp4mr
