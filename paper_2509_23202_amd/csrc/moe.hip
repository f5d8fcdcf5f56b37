// A router's choice of experts, and the experts' outputs added up for each token.
//
//   s = softmax(z) or sigmoid(z),  c = z where there is neither a bias nor a sum of scores to compare, else s + bias
//   of `groups` runs of experts the top_groups best ones are kept (a run counts as its largest c, or the sum of its two largest), of their experts the `top` best: (c, lower index first)
//   weight = scale s of the chosen, or scale s / sum of the chosen
//
// Which of two experts is the better one hangs on c alone.  Without a bias the order of the scores is that of the logits, which are compared as they are.  Otherwise the choice is that of c in binary64: else whole tokens
// would go elsewhere with the last bit of an exponential, and a choice could not be checked against any other arithmetic.  c is formed in fp32 first, and in binary64 for the few tokens whose choice fp32 leaves in doubt.
//
// The chosen pairs (token, place among its choices) are then sorted by expert, stably, so that an expert's rows are in the order of the tokens: counts of each expert for each run of tokens, a
// sum over the runs in front and the experts in front, and the rank within the run.  No atomic's order reaches a result.
//
// What bounds it: for few tokens the launches (1 token of 64 experts 2.7 us) and a chain of latencies (777 of 256 in groups 8 us, 12 with a token in doubt, the vector unit at work in a sixth of them).  For many the vector
// unit: it works in 62 % of the cycles where logits are compared (16384 tokens of 128 experts 8.0 us, 154 instructions of a wave to a token), in 77 and 79 % where scores are (of 256 with a bias 21.6 us, 456 of them; of 512
// in groups 50.6, 1160), while waves wait for half of theirs; reading the logits would take 0.7, 2.6 and 5.3.  The second launch reads all counts in every workgroup (16384 of 128 5.9 us; half of its cycles at work).
#include "bf16_rows.hpp"
#include "internal.hpp"

#include <algorithm>
#include <type_traits>

namespace fp4mr {
namespace {

typedef unsigned long long u64;

constexpr int kMaxThreads = 1024, kMaxWaves = kMaxThreads / 64;
// Threads of a workgroup at most that routes tokens: exact scores of sixteen experts to a lane take more registers than 1024 threads have.
constexpr int threads_of(int lanes, int each) { return lanes * each > 512 ? 512 : kMaxThreads; }
constexpr int kMaxRuns = 256;          // runs of tokens: a compute unit each, and few enough that every workgroup that places rows can read all counts

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
    int32_t* counts;           // [runs, wide]
    int run, runs, wide;       // tokens of a run; runs; experts rounded up to a multiple of four
    int words;                 // a power of two, for a bit to each token of a run
    bool sigmoid, renorm, sum2, alone;
    FastDiv by_size, by_top, by_fours;         // by the experts of a group, ..., a quarter of `wide`
};

// ---------------------------------------------------------------- keys: numbers in their order as unsigned ones, zeros of both signs alike; 0 is below every number
__device__ __forceinline__ uint32_t order_of(float c)
{
    const int b = __float_as_int(c + 0.0f);
    return (uint32_t)(b ^ (b >> 31 | (int)0x80000000));
}
__device__ __forceinline__ float of_order(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
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

// ---------------------------------------------------------------- over the 16 or 64 lanes of a token, in all of them
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ u64 moved(u64 v) { return (u64)moved<CTRL>((uint32_t)(v >> 32)) << 32 | moved<CTRL>((uint32_t)v); }
template <int CTRL>
__device__ __forceinline__ float moved(float v) { return __uint_as_float(moved<CTRL>(__float_as_uint(v))); }
template <int CTRL>
__device__ __forceinline__ double moved(double v) { return __builtin_bit_cast(double, moved<CTRL>(__builtin_bit_cast(u64, v))); }

// f of the values of lanes l and l ^ D, D = 16 or 32: the swap leaves one of them in every lane of each of its two results.
template <int D, typename F>
__device__ __forceinline__ uint32_t across(uint32_t v, F f)
{
    const auto p = D == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f((uint32_t)p[0], (uint32_t)p[1]);
}
template <int D, typename F>
__device__ __forceinline__ u64 across(u64 v, F f)
{
    const auto l = D == 16 ? __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false) : __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto h = D == 16 ? __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false)
                           : __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    return f((u64)(uint32_t)h[0] << 32 | (uint32_t)l[0], (u64)(uint32_t)h[1] << 32 | (uint32_t)l[1]);
}
template <int D, typename F>
__device__ __forceinline__ float across(float v, F f)
{
    return __uint_as_float(across<D>(__float_as_uint(v), [f](uint32_t x, uint32_t y) { return __float_as_uint(f(__uint_as_float(x), __uint_as_float(y))); }));
}
template <int D, typename F>
__device__ __forceinline__ double across(double v, F f)
{
    return __builtin_bit_cast(double, across<D>(__builtin_bit_cast(u64, v), [f](u64 x, u64 y) { return __builtin_bit_cast(u64, f(__builtin_bit_cast(double, x), __builtin_bit_cast(double, y))); }));
}

template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f)
{
    v = f(v, moved<0xb1>(v));       // quad_perm [1,0,3,2]
    v = f(v, moved<0x4e>(v));       // quad_perm [2,3,0,1]
    v = f(v, moved<0x141>(v));      // row_half_mirror, row_mirror: pairs of lanes exchange theirs in every step, so that a sum is the same in all of them to the last bit (a rotation's is not)
    v = f(v, moved<0x140>(v));
    if constexpr (LANES == 64) {
        v = across<16>(v, f);
        v = across<32>(v, f);
    }
    return v;
}
template <int LANES, typename T>
__device__ __forceinline__ T lanes_max(T v)
{
    return over_lanes<LANES>(v, [](T a, T b) { return a > b ? a : b; });
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_min(uint32_t v)
{
    return over_lanes<LANES>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v)
{
    return over_lanes<LANES>(v, [](double a, double b) { return a + b; });
}

// e^(x + lo), x <= 88 and lo at most a rounding of x, within two steps (0 below 2^-126): x log2 e in two parts, the first to the instruction, whose result is one step off, and the rest as a factor.
__device__ __forceinline__ float power_of_e(float x, float lo = 0.0f)
{
    const float y = x * 1.44269502f, rest = fmaf(x, 1.44269502f, -y) + x * 1.92596299e-8f;      // log2 e = 1.44269502 + 1.92596299e-8
    const float p = __builtin_amdgcn_exp2f(y);
    return fmaf(p, fmaf(rest, 0.693147182f, lo), p);
}

// How the experts are compared: a bf16 logit and the index in one word, an fp32 logit, or a score.
enum { kPacked, kLogit, kScore };

// A score in fp32, from an exponential within two steps, sums in binary64 and a reciprocal, is within 2^-20 of the score: of softmax (x = z - max) s (2^-22 + 2^-22 + 2^-23 + 2^-24) + s 2^-24 sum e^x |x| / sum e^x
// + 0.37 2^-24, where s times the quotient of sums is less than 2 (0.84 2^-20 in all), of sigmoid s (2^-22 + 2^-24 + 2^-23) + 0.28 2^-24.  With its bias, c is within 2^-20 + 2^-24 |c|.
// Two that are further apart than both errors, at most 2^-19 + 2^-23 of the larger magnitude, are in the order of their exact values (the second-order parts are in the last bit of the factor, and the difference is exact
// where it is that small).  An error grows slower than c, so one that is apart from the next is apart from all behind it; and it is a matter of the two that are compared: an expert that a bias far below the others takes
// out (-1e9, the type's lowest value) puts no token in doubt (16384 tokens, 8 of 256 experts, one of which is out so: 27 us; with one doubt for all, from the largest bias, every token was routed twice: 53).
__device__ __forceinline__ bool apart(float larger, float smaller) { return larger - smaller > fmaf(0x1.00001p-23f, fmaxf(larger, -smaller), 0x1p-19f); }

// The same of sums m of two, f >= s: within 2^-19 + 2^-24 (|f| + |s| + |m|), at most 2^-19 + 2^-23 (|m| + opposed), the lesser magnitude of the two where their signs differ.  What is beyond fp32 counts as its largest
// number, which the exact sum has passed but for a rounding.
__device__ __forceinline__ bool sums_apart(float larger, float smaller, float opposed)
{
    constexpr float MOST = 3.402823466e38f;
    const float l = __builtin_amdgcn_fmed3f(larger, -MOST, MOST), s = __builtin_amdgcn_fmed3f(smaller, -MOST, MOST);
    return l - s > fmaf(0x1.00001p-22f, fmaxf(l, -s) + opposed, 0x1p-18f);
}

// A token's LANES lanes' view of what is the same for all of them.
template <int LANES, bool F32>
struct Token {
    const RouteArgs& a;
    int lane;
    int64_t at;
    float most;                // the largest logit (softmax)
    double sum;                // of e^(z - most) over its experts (softmax)

    __device__ float logit(int e) const
    {
        if constexpr (F32) return static_cast<const float*>(a.logits)[at + e];
        else return (float)static_cast<const __bf16*>(a.logits)[at + e];
    }
    __device__ double exact_power(float z) const { return z == -__builtin_inff() ? 0.0 : exp((double)z - (double)most); }
    __device__ double exact_score(float z) const { return !a.sigmoid ? exact_power(z) / sum : z == -__builtin_inff() ? 0.0 : 1.0 / (1.0 + exp(-(double)z)); }
    // in fp32, of softmax before the division by the sum; what is below 2^-126 is 0
    __device__ float score(float z) const { return a.sigmoid ? z < -87.3f ? 0.0f : __builtin_amdgcn_rcpf(1.0f + power_of_e(fmaxf(-z, -200.0f))) : power_of_e(fmaxf(z - most, -200.0f)); }
    // the same where the last bits of z - most count too
    __device__ float weight(float z) const
    {
        if (a.sigmoid) return z < -87.3f ? 0.0f : 1.0f / (1.0f + power_of_e(fmaxf(-z, -200.0f)));
        const float x = z - most, back = x - z;
        return x > -200.0f ? power_of_e(x, (z - (x - back)) + (-most - back)) : 0.0f;      // (with what the subtraction has rounded off)
    }
};

// The wave's largest, and 1/2 at least: what hardly ever counts needs no maximum over the lanes.
__device__ __forceinline__ float largest_opposed(float opposed)
{
    return __any(opposed > 0.5f) ? __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)lanes_max<64>(__float_as_uint(opposed)))) : 0.5f;
}

// The best top_groups groups, as bits.  key: a function of the expert.  sure: stays so where scores in fp32 leave no doubt.
template <int LANES, bool EXACT, typename K>
__device__ __forceinline__ u64 best_groups(const RouteArgs& a, int lane, bool& sure, K key)
{
    typedef std::conditional_t<EXACT, u64, uint32_t> Key;
    const int size = (int)a.by_size.d;
    float opposed = 0.0f, of_wave = 0.0f;
    auto mark_of = [&](Key first, Key second) -> Key {
        if (!a.sum2 || !second) return first;
        if constexpr (!EXACT) opposed = fmaxf(opposed, fminf(of_order(first), -of_order(second)));
        return order_of(of_order(first) + of_order(second));
    };
    auto add = [](Key k, Key& first, Key& second) {
        second = k > first ? first : k > second ? k : second;
        first = k > first ? k : first;
    };
    if constexpr (LANES == 64) {
        // so many lanes to a group, of which the first has its mark; its rank among the groups says whether it is kept
        const int wide = a.groups <= 8 ? 8 : a.groups <= 16 ? 4 : a.groups <= 32 ? 2 : 1, g = lane / wide;
        Key first = 0, second = 0;
        if (g < a.groups)
            for (int j = lane & (wide - 1); j < size; j += wide) add(key(g * size + j), first, second);
        auto join = [&](Key f, Key s) {
            second = f > first ? (first > s ? first : s) : f > second ? f : second;
            first = f > first ? f : first;
        };
        if (wide > 1) join(moved<0xb1>(first), moved<0xb1>(second));
        if (wide > 2) join(moved<0x4e>(first), moved<0x4e>(second));
        if (wide > 4) join(moved<0x141>(first), moved<0x141>(second));
        const Key mark = g < a.groups ? mark_of(first, second) : 0;
        int rank = 0;
        for (int o = 0; o < a.groups; ++o) {
            Key m;
            if constexpr (EXACT) m = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(mark >> 32), o * wide) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mark, o * wide);
            else m = (uint32_t)__builtin_amdgcn_readlane((int)mark, o * wide);
            rank += m > mark || (m == mark && o < g);
        }
        const bool own = (lane & (wide - 1)) == 0 && mark != 0;
        if constexpr (!EXACT) {      // the last one that is kept and the first that is not
            of_wave = largest_opposed(opposed);
            const u64 last = __ballot(own && rank == a.top_groups - 1), out = __ballot(own && rank == a.top_groups);
            if (last && out)
                sure &= sums_apart(of_order((uint32_t)__builtin_amdgcn_readlane((int)mark, __builtin_ctzll(last))), of_order((uint32_t)__builtin_amdgcn_readlane((int)mark, __builtin_ctzll(out))), of_wave);
        }
        u64 kept = 0;
        for (u64 of = __ballot(own && rank < a.top_groups); of; of &= of - 1) kept |= 1ull << __builtin_ctzll(of) / wide;
        return kept;
    } else {
        constexpr int MARKS = 64 / LANES;
        Key mark[MARKS];
#pragma unroll
        for (int q = 0; q < MARKS; ++q) {
            const int g = q * LANES + lane;
            Key first = 0, second = 0;
            if (g < a.groups)
                for (int j = 0; j < size; ++j) add(key(g * size + j), first, second);
            mark[q] = mark_of(first, second);
        }
        if constexpr (!EXACT)
            of_wave = largest_opposed(opposed);
        u64 kept = 0;
        Key last = 0;
        for (int j = 0; j <= a.top_groups; ++j) {
            Key best = 0;
#pragma unroll
            for (int q = 0; q < MARKS; ++q) best = mark[q] > best ? mark[q] : best;
            best = lanes_max<LANES>(best);
            if (!__any(best != 0)) break;
            if (j == a.top_groups) {      // one that is left out
                if constexpr (!EXACT) sure &= best == 0 || sums_apart(of_order(last), of_order(best), of_wave);
                break;
            }
            uint32_t g = 64;
#pragma unroll
            for (int q = MARKS - 1; q >= 0; --q) g = mark[q] == best ? q * LANES + lane : g;
            g = lanes_min<LANES>(g);
            if (best != 0) {
                kept |= 1ull << g;
                last = best;
            }
#pragma unroll
            for (int q = 0; q < MARKS; ++q)
                if (q * LANES + lane == (int)g) mark[q] = 0;
        }
        return kept;
    }
}

// The lowest expert among the lanes of a token that have `best`.
template <int LANES, typename Key>
__device__ __forceinline__ uint32_t expert_of(Key of_lane, Key best, uint32_t e)
{
    if constexpr (LANES == 64) {
        const u64 have = __ballot(of_lane == best);
        if (__builtin_popcountll(have) == 1) return (uint32_t)__builtin_amdgcn_readlane((int)e, __builtin_ctzll(have));
    }
    return lanes_min<LANES>(of_lane == best ? e : 0xffffffffu);
}

template <int LANES>
__device__ __forceinline__ bool any_lane(bool v)
{
    if constexpr (LANES == 64) return __ballot(v) != 0;
    return lanes_max<LANES>((uint32_t)v) != 0;
}

// What leaves of a token: lane j has its j-th expert (or -1), and that one's logit.  Of a workgroup alone the experts are left in `count` too, else counted there.
template <int LANES, bool F32>
__device__ __forceinline__ void finish_token(const RouteArgs& a, const Token<LANES, F32>& k, int64_t t, bool real, bool bad, int mine, float of_mine, int32_t* count)
{
    float w = mine >= 0 ? k.weight(of_mine) : 0.0f;
    const float whole = fmaxf((float)k.sum, 0x1p-60f);        // (of softmax w is e^(z - max): `whole` times the score)
    if (a.renorm) w /= fmaxf(over_lanes<LANES>(w, [](float x, float y) { return x + y; }), 0x1p-60f * whole);
    else w /= whole;
    if (real && k.lane < a.top) {
        a.weights[t * a.top + k.lane] = bad ? __builtin_nanf("") : w * a.scale;
        a.chosen[t * a.top + k.lane] = mine;
        if (a.alone) count[t * a.top + k.lane] = mine;
        else if (mine >= 0) atomicAdd(count + mine, 1);
    }
}

// A token whose scores fp32 cannot tell apart, by exact scores and by a whole wave; expert 64 i + lane is the lane's i-th.  keys: room in LDS for them.
template <int EACH, bool F32>
__device__ __forceinline__ void route_exactly(const RouteArgs& a, int64_t t, u64* keys, int32_t* count)
{
    Token<64, F32> k{a, (int)threadIdx.x & 63, t * a.stride, -__builtin_inff(), 1.0};
    const int lane = k.lane;
    // (four experts' exponentials at a time, each a long chain of its own)
    auto logit = [&](int i) { return 64 * i + lane < a.experts ? k.logit(min(64 * i + lane, a.experts - 1)) : -__builtin_inff(); };
    if (!a.sigmoid) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) k.most = fmaxf(k.most, logit(i));
        k.most = of_order(lanes_max<64>(order_of(k.most)));
        double sum = 0.0;
#pragma unroll 4
        for (int i = 0; i < EACH; ++i) sum += k.exact_power(logit(i));
        k.sum = lanes_sum<64>(sum);
    }
#pragma unroll 4
    for (int i = 0; i < EACH; ++i) {
        const int e = 64 * i + lane;
        const float z = logit(i), b = a.bias ? a.bias[min(e, a.experts - 1)] : 0.0f;
        keys[e] = z == -__builtin_inff() || b == -__builtin_inff() ? 0 : order_of(k.exact_score(z) + (double)b);
    }
    __builtin_amdgcn_wave_barrier();
    u64 kept = ~0ull;
    bool sure = true;
    if (a.groups > 1) kept = best_groups<64, true>(a, lane, sure, [&](int e) { return keys[e]; });
    u64 key[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) key[i] = kept >> (fast_div(min(64 * i + lane, a.experts - 1), a.by_size) & 63) & 1 ? keys[64 * i + lane] : 0;
    int mine = -1;
    for (int j = 0; j < a.top; ++j) {
        u64 best = 0;
        uint32_t e = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            e = key[i] > best ? 64 * i + lane : e;
            best = key[i] > best ? key[i] : best;
        }
        const u64 of_lane = best;
        best = lanes_max<64>(best);
        if (best == 0) break;
        e = expert_of<64>(of_lane, best, e);
#pragma unroll
        for (int i = 0; i < EACH; ++i) key[i] = 64 * i + lane == (int)e ? 0 : key[i];
        if (lane == j) mine = (int)e;
    }
    __builtin_amdgcn_wave_barrier();
    finish_token<64, F32>(a, k, t, true, false, mine, mine >= 0 ? k.logit(mine) : 0.0f, count);
}

// The choice of a token to each LANES lanes; expert LANES i + lane is the lane's i-th.  keys: room in LDS for the token's keys.  False where fp32 leaves it in doubt: then nothing was written.
template <int LANES, int EACH, int BY, bool F32>
__device__ __forceinline__ bool route_token(const RouteArgs& a, int64_t t, bool real, u64* keys, int32_t* count)
{
    Token<LANES, F32> k{a, (int)threadIdx.x & (LANES - 1), real ? t * a.stride : 0, 0.0f, 1.0};
    const int lane = k.lane;
    float z[EACH], b[BY == kScore ? EACH : 1];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = LANES * i + lane;
        z[i] = e < a.experts ? k.logit(e) : -__builtin_inff();
        if constexpr (BY == kScore) b[i] = a.bias && e < a.experts ? a.bias[e] : 0.0f;
    }
    bool bad = false;
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        bad |= z[i] != z[i] || (!a.sigmoid && z[i] == __builtin_inff());
        if constexpr (BY == kScore) bad |= b[i] != b[i];
        most = fmaxf(most, z[i]);
    }
    bad = any_lane<LANES>(bad);
    if (!a.sigmoid) {
        k.most = of_order(lanes_max<LANES>(order_of(most)));
        if (BY == kScore || !a.renorm) {     // (else the chosen ones' weights are relative to each other)
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += (double)k.score(z[i]);
            k.sum = lanes_sum<LANES>(sum);
        }
    }

    // ---- keys
    uint32_t key[EACH];
    const float part = 1.0f / (float)k.sum;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool out = z[i] == -__builtin_inff() || bad;
        if constexpr (BY == kScore) {
            const float s = a.sigmoid ? k.score(z[i]) : k.score(z[i]) * part;
            key[i] = out || b[i] == -__builtin_inff() ? 0 : order_of(s + b[i]);
        } else if constexpr (BY == kPacked) {     // (of a bf16 the order's low half says nothing; of equal ones the first is the largest)
            key[i] = out ? 0 : (order_of(z[i]) & 0xffff0000u) | (uint32_t)(0xffff - (LANES * i + lane));
        } else {
            key[i] = out ? 0 : order_of(z[i]);
        }
    }
    bool sure = true;
    if (a.groups > 1) {
        uint32_t* const keys32 = reinterpret_cast<uint32_t*>(keys);
#pragma unroll
        for (int i = 0; i < EACH; ++i) keys32[LANES * i + lane] = BY == kPacked ? key[i] >> 16 : key[i];      // (equal groups: the lower one)
        __builtin_amdgcn_wave_barrier();
        const u64 kept = best_groups<LANES, false>(a, lane, sure, [&](int e) { return keys32[e]; });
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (!(kept >> fast_div(min(LANES * i + lane, a.experts - 1), a.by_size) & 1)) key[i] = 0;
        __builtin_amdgcn_wave_barrier();
    }

    // ---- the choice: lane j keeps the j-th, and its logit where the key has it
    int mine = -1;
    float of_mine = 0.0f, before = 3.402823466e38f;
    for (int j = 0; j < a.top; ++j) {
        uint32_t best = 0, e = 0xffffffffu;
        if constexpr (BY == kPacked) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) best = max(best, key[i]);
            best = lanes_max<LANES>(best);
            e = 0xffff - (best & 0xffff);
#pragma unroll
            for (int i = 0; i < EACH; ++i) key[i] = key[i] == best ? 0 : key[i];
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                e = key[i] > best ? LANES * i + lane : e;
                best = max(best, key[i]);
            }
            const uint32_t of_lane = best;
            best = lanes_max<LANES>(best);
            e = expert_of<LANES>(of_lane, best, e);
#pragma unroll
            for (int i = 0; i < EACH; ++i) key[i] = LANES * i + lane == (int)e ? 0 : key[i];
        }
        if (!__any(best != 0)) break;
        const float value = of_order(BY == kPacked ? (best & 0xffff0000u) | (best & 0x80000000u ? 0u : 0xffffu) : best);
        if (best != 0) {
            if constexpr (BY == kScore) sure &= apart(before, value);
            before = value;
            if (lane == j) {
                mine = (int)e;
                of_mine = value;
            }
        }
    }
    if constexpr (BY == kScore) {
        uint32_t next = 0;         // the best one that is left
#pragma unroll
        for (int i = 0; i < EACH; ++i) next = max(next, key[i]);
        next = lanes_max<LANES>(next);
        sure &= next == 0 || apart(before, of_order(next));
        of_mine = mine >= 0 ? k.logit(mine) : 0.0f;
    }

    finish_token<LANES, F32>(a, k, t, real && (BY != kScore || sure), bad, mine, of_mine, count);
    return sure;
}

// Exclusive sum over a workgroup of kMaxThreads of one number a thread, and the whole.  part: [kMaxWaves] words of LDS.
__device__ __forceinline__ int before_thread(int n, int32_t* part, int& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = n;
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, true);     // row_shr 1, 2, 4, 8: the sum within sixteen lanes
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);    // row_bcast 15 to the second and fourth sixteen, row_bcast 31 to the second half
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int front = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kMaxWaves; ++w) {
        const int of = part[w];
        front += w < wave ? of : 0;
        all += of;
    }
    return front + upto - n;
}

// The rows of few choices, all of them in LDS (kept: n of them, -1 and more behind them up to a multiple of four): a choice's row is the number of choices in front of it, an expert's first row that of lower experts.
__device__ __forceinline__ void place_few(const RouteArgs& a, const int32_t* kept, int n)
{
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    const v4u* const all = reinterpret_cast<const v4u*>(kept);       // (no expert: the largest number)
    const int fours = (n + 3) / 4, threads = blockDim.x;
    for (int x = threadIdx.x; x < n + a.experts + 1; x += threads) {
        const bool choice = x < n;
        const uint32_t e = choice ? (uint32_t)kept[x] : (uint32_t)(x - n);
        const int upto = choice ? x : 0;           // choices of the same expert count so far
        int before = 0;
#pragma unroll 4
        for (int q = 0; q < fours; ++q) {
            const v4u v = all[q];
#pragma unroll
            for (int i = 0; i < 4; ++i) before += v[i] < e || (v[i] == e && 4 * q + i < upto);
        }
        if (!choice) {
            a.offsets[x - n] = before;
        } else if ((int)e < 0) {
            a.places[x] = -1;
        } else {
            a.rows[before] = (int32_t)fast_div((uint32_t)x, a.by_top);
            a.places[x] = before;
        }
    }
}

// A run of tokens to a workgroup.  Where it is alone, it places the rows too (1 token x 4 of 64 experts 3.5 us, in two launches 6.1; 32 tokens 6.8 and 7.0; 64 tokens x 2 7.2 and 6.9, of which the host
// has one less to make).
template <int LANES, int EACH, int BY, bool F32>
__global__ __launch_bounds__(threads_of(LANES, EACH)) void moe_route_kernel(RouteArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int threads = blockDim.x, at_once = threads / LANES;
    int32_t* const count = reinterpret_cast<int32_t*>(smem);                // [experts], or alone the experts that were chosen [tokens, top]
    const int n = a.alone ? (int)a.tokens * a.top : a.experts;
    uint32_t* const doubtful = reinterpret_cast<uint32_t*>(smem + (n + 3) / 4 * 16);          // a bit to each token: the i-th in word i % words, so that they are spread over the waves
    u64* const keys = reinterpret_cast<u64*>(smem + (n + 3) / 4 * 16 + (BY == kScore ? a.words * 4 : 0));      // of each token at a time, where they are needed
    for (int i = threadIdx.x; i < (n + 3) / 4 * 4; i += threads) count[i] = a.alone ? -1 : 0;
    if constexpr (BY == kScore)
        for (int i = threadIdx.x; i < a.words; i += threads) doubtful[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.run, end = min(first + a.run, a.tokens);
    for (int64_t t0 = first; t0 < end; t0 += at_once) {
        const int64_t t = t0 + threadIdx.x / LANES;
        if (!__any(t < end)) continue;
        const bool sure = route_token<LANES, EACH, BY, F32>(a, t, t < end, keys + threadIdx.x / LANES * (LANES * EACH), count);
        if (BY == kScore && !sure && t < end && threadIdx.x % LANES == 0) atomicOr(doubtful + ((int)(t - first) & (a.words - 1)), 1u << (int)(t - first) / a.words);
    }
    if constexpr (BY == kScore) {      // (apart from the others, which have the registers for themselves then: 16384 tokens, 8 of 256 experts 32.3 -> 28.4 us in both launches, in groups 41.5 -> 35.1; without any in doubt 24.0 and 29.3)
        __syncthreads();
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        for (int w = wave; w < a.words; w += threads / 64)
            for (uint32_t bits = __builtin_amdgcn_readfirstlane(doubtful[w]); bits; bits &= bits - 1)
                route_exactly<(LANES * EACH + 63) / 64, F32>(a, first + __builtin_ctz(bits) * a.words + w, keys + wave * (64 * EACH), count);
    }
    __syncthreads();
    if (a.alone) {
        place_few(a, count, n);
    } else {
        for (int e = threadIdx.x; e < a.experts; e += threads) a.counts[(int)blockIdx.x * a.wide + e] = count[e];
    }
}

// Where the rows of a run of tokens lie, as many of its choices at a time as there are threads.  A choice's row is its expert's first one, and so many on as there are choices of that expert in front of it: in the
// runs before, in the waves before and in the lanes before.
__global__ __launch_bounds__(kMaxThreads) void moe_place_kernel(RouteArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int32_t* const part = reinterpret_cast<int32_t*>(smem);                 // [kMaxWaves]
    v2i* const sums = reinterpret_cast<v2i*>(part + kMaxWaves);             // [4 kMaxThreads]: of `shares` parts of the runs, of each expert the choices in the runs in front, and all
    int32_t* const of_wave = reinterpret_cast<int32_t*>(sums + 4 * kMaxThreads);      // [kMaxWaves, experts]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = threadIdx.x;
    const uint32_t first = (uint32_t)blockIdx.x * (uint32_t)(a.run * a.top), end = (uint32_t)min((int64_t)first + a.run * a.top, a.tokens * a.top);      // (at most 2^30)
    int e = first + x < end ? a.chosen[first + x] : -1;
    const int fours = a.wide / 4, shares = min(kMaxThreads / fours, 32), share = (int)fast_div(x, a.by_fours), four = x - share * fours;       // (experts <= kMaxThreads)
    if (share < shares) {
        v4i before{0, 0, 0, 0}, all{0, 0, 0, 0};
        const v4i* const from = reinterpret_cast<const v4i*>(a.counts) + four;
#pragma unroll 8
        for (int r = share; r < a.runs; r += shares) {
            const v4i n = from[r * fours];
            all += n;
            if (r < (int)blockIdx.x) before += n;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[share * a.wide + four * 4 + i] = v2i{before[i], all[i]};
    }
    int rank = 0;
    auto count = [&]() {       // of each wave's choices, and a choice's rank in its wave
        u64 same = __ballot(e >= 0);
        for (int bit = 0; (a.experts - 1) >> bit; ++bit) {
            const u64 set = __ballot(e >> bit & 1);
            same &= e >> bit & 1 ? set : ~set;
        }
        rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        if (e >= 0 && rank == 0) of_wave[wave * a.experts + e] = __builtin_popcountll(same);
    };
    for (int i = x; i < kMaxWaves * a.experts; i += kMaxThreads) of_wave[i] = 0;
    __syncthreads();
    count();
    int before = 0, all = 0;
    if (x < a.experts)
#pragma unroll 8
        for (int s = 0; s < shares; ++s) {
            const v2i n = sums[s * a.wide + x];
            before += n[0];
            all += n[1];
        }
    int whole;
    const int front = before_thread(all, part, whole);
    if (blockIdx.x == 0) {
        if (x < a.experts) a.offsets[x] = front;
        if (x == 0) a.offsets[a.experts] = whole;
    }
    int next = front + before;         // row of the thread's expert
    for (uint32_t f = first + x;;) {
        if (x < a.experts) {
            int n[kMaxWaves];
#pragma unroll
            for (int w = 0; w < kMaxWaves; ++w) n[w] = of_wave[w * a.experts + x];
#pragma unroll
            for (int w = 0; w < kMaxWaves; ++w) {
                of_wave[w * a.experts + x] = next;
                next += n[w];
            }
        }
        __syncthreads();
        if (e >= 0) {
            const int row = of_wave[wave * a.experts + e] + rank;
            a.rows[row] = (int32_t)fast_div(f, a.by_top);
            a.places[f] = row;
        } else if (f < end) {
            a.places[f] = -1;
        }
        f += kMaxThreads;
        if (f - x >= end) break;
        __syncthreads();
        for (int i = x; i < kMaxWaves * a.experts; i += kMaxThreads) of_wave[i] = 0;
        e = f < end ? a.chosen[f] : -1;
        __syncthreads();
        count();
        __syncthreads();
    }
}

// ---------------------------------------------------------------- the experts' outputs
struct CombineArgs {
    const void* y;
    int64_t y_rows;
    const int32_t* places;
    const float* weights;
    const void* shared;        // or null
    void* out;
    int64_t tokens, cols;
    int top;
    bool shared_f32, out_f32;
};

__device__ __forceinline__ float element(const void* p, int64_t i, bool f32) { return f32 ? static_cast<const float*>(p)[i] : (float)static_cast<const __bf16*>(p)[i]; }

// out[t] = shared[t] + sum_j weight[t,j] y[place[t,j]], in fp32 in the order of the choices.  A choice without a row adds its weight times zero.  Any number of columns, at any element; an element to a thread, whose loads of 2
// or 4 bytes and whose division bound it: 4095 tokens x 8 rows of 4097 columns 266 us, of 4096 where one of the tensors is off 16 bytes 272 (the kernel below 60).  For odd shapes; a model's rows are whole pieces.
template <bool Y_F32>
__global__ __launch_bounds__(256) void moe_combine_any_kernel(CombineArgs a)
{
    const int64_t total = a.tokens * a.cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / a.cols, c = i - t * a.cols;
        float sum = a.shared ? element(a.shared, i, a.shared_f32) : 0.0f;
        for (int j = 0; j < a.top; ++j) {
            const int64_t row = a.places[t * a.top + j];
            const float w = a.weights[t * a.top + j];
            sum = fmaf(w, row >= 0 && row < a.y_rows ? element(a.y, row * a.cols + c, Y_F32) : 0.0f, sum);
        }
        if (a.out_f32) static_cast<float*>(a.out)[i] = sum;
        else static_cast<__bf16*>(a.out)[i] = (__bf16)sum;
    }
}

__device__ __forceinline__ void load8(const void* p, int64_t i, bool f32, float (&v)[8])
{
    if (f32) {
        const v4f* const q = reinterpret_cast<const v4f*>(static_cast<const float*>(p) + i);
        const v4f lo = __builtin_nontemporal_load(q), hi = __builtin_nontemporal_load(q + 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = lo[e];
            v[4 + e] = hi[e];
        }
    } else {
        widen8(load16<true>(static_cast<const __bf16*>(p) + i), v);
    }
}

// The same for rows whose pieces of eight columns are 16-byte aligned, a piece to a thread: the loads of up to eight rows are on their way together.  A token's columns are to `wide` threads, a power of two.
// Bound by memory: 4095 tokens x 8 rows of 4096 with the shared expert's 58 us (335 MB, 5.8 TB/s; a large copy's 6.4 would be 53), all in fp32 139 (671 MB, 4.8 TB/s); of few tokens by its start-up (5 tokens 2.7 us).
template <bool Y_F32>
__global__ __launch_bounds__(256) void moe_combine_kernel(CombineArgs a, int wide)
{
    const int64_t t = (int64_t)blockIdx.x * (256 / wide) + threadIdx.x / wide;
    const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x % wide) * 8;
    if (t >= a.tokens || c >= a.cols) return;
    const int32_t* const places = a.places + t * a.top;
    const float* const weights = a.weights + t * a.top;
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    if (a.shared) load8(a.shared, t * a.cols + c, a.shared_f32, sum);
    auto add = [&](int j, auto many) {
        constexpr int MANY = many;
        float w[MANY], v[MANY][8];
        bool have[MANY];
#pragma unroll
        for (int u = 0; u < MANY; ++u) {
            const int row = places[j + u];
            w[u] = weights[j + u];
            have[u] = row >= 0 && row < a.y_rows;
            load8(a.y, (int64_t)(have[u] ? row : 0) * a.cols + c, Y_F32, v[u]);
        }
#pragma unroll
        for (int u = 0; u < MANY; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = fmaf(w[u], have[u] ? v[u][e] : 0.0f, sum[e]);
    };
    int j = 0;
    for (; j + 8 <= a.top; j += 8) add(j, std::integral_constant<int, 8>{});
    if (a.top - j >= 4) {
        add(j, std::integral_constant<int, 4>{});
        j += 4;
    }
    if (a.top - j >= 2) {
        add(j, std::integral_constant<int, 2>{});
        j += 2;
    }
    if (a.top - j >= 1) add(j, std::integral_constant<int, 1>{});
    const int64_t to = t * a.cols + c;
    if (a.out_f32) {
        v4f* const q = reinterpret_cast<v4f*>(static_cast<float*>(a.out) + to);
        __builtin_nontemporal_store(v4f{sum[0], sum[1], sum[2], sum[3]}, q);
        __builtin_nontemporal_store(v4f{sum[4], sum[5], sum[6], sum[7]}, q + 1);
    } else {
        store8(static_cast<__bf16*>(a.out) + to, sum);
    }
}

// So few are routed and placed by one workgroup.
bool alone(int64_t tokens, int64_t top) { return tokens <= 64 && tokens * top <= 128; }

FastDiv fast_div_by(uint32_t d)
{
    FastDiv f{0, 0, d};
    if (d > 1) {        // n < 2^31: with 2^l >= d, magic = ceil(2^(31 + l) / d) has 32 bits, and n times its error is less than 2^(31 + l) / d
        uint32_t l = 0;
        while ((1ull << l) < d) ++l;
        f.magic = (uint32_t)(((1ull << (31 + l)) + d - 1) / d);
        f.shift = l - 1;
    }
    return f;
}

// Tokens of a run and runs.  At least eight, a workgroup of eight waves: runs of four leave twice the counts to add (1024 tokens, 256 experts 12.1 us, with eight 10.9), of sixteen half the compute units
// idle where tokens are few (256 of 256 experts in groups 12.5, 12.3, 15.3 us).
void runs_of(int64_t tokens, int& run, int& runs)
{
    run = (int)std::max<int64_t>(8, (tokens + kMaxRuns - 1) / kMaxRuns);
    runs = (int)((tokens + run - 1) / run);
}

template <int LANES, int EACH, int BY, bool F32>
hipError_t route(const RouteArgs& a, hipStream_t st)
{
    // (alone: enough to place the rows too, at a time)
    const int64_t wanted = std::max<int64_t>(std::min<int64_t>(a.run, a.tokens) * LANES, a.alone ? a.tokens * a.top + a.experts + 1 : 1);
    const int waves = (int)std::min<int64_t>((wanted + 63) / 64, threads_of(LANES, EACH) / 64);
    const size_t lds = (size_t)((a.alone ? a.tokens * a.top : a.experts) + 3) / 4 * 16 + (BY == kScore ? a.words * 4 : 0) + (BY == kScore || a.groups > 1 ? (size_t)waves * 64 * EACH * 8 : 0);
    static LdsAttrOnce attr;
    if (const hipError_t e = attr.ensure(reinterpret_cast<const void*>(moe_route_kernel<LANES, EACH, BY, F32>), 163840)) return e;
    hipLaunchKernelGGL((moe_route_kernel<LANES, EACH, BY, F32>), dim3(std::max(a.runs, 1)), dim3(waves * 64), lds, st, a);
    return hipGetLastError();
}

// A token to a wave while the device has waves for all tokens, else to sixteen lanes, where its experts are few enough for their registers and it chooses no more than sixteen: a maximum over sixteen lanes is four
// instructions for four tokens, over a wave eight for one (both launches of 16384 tokens, 8 of 128 experts: 13.9 us, a token to a wave 20.2; of 1024 tokens 9.9, on sixteen lanes 10.5; one workgroup's 32 tokens 6.8
// on sixteen lanes, 8.6 by the wave).
template <int BY, bool F32>
hipError_t route(const RouteArgs& a, hipStream_t st)
{
    if ((a.tokens > 4096 || (a.alone && a.tokens > 16)) && a.top <= 16) {
        if (a.experts <= 64) return route<16, 4, BY, F32>(a, st);
        if (a.experts <= 128) return route<16, 8, BY, F32>(a, st);
        if (a.experts <= 256) return route<16, 16, BY, F32>(a, st);
    }
    if (a.experts <= 64) return route<64, 1, BY, F32>(a, st);
    if (a.experts <= 128) return route<64, 2, BY, F32>(a, st);
    if (a.experts <= 256) return route<64, 4, BY, F32>(a, st);
    if (a.experts <= 512) return route<64, 8, BY, F32>(a, st);
    return route<64, 16, BY, F32>(a, st);
}

}  // namespace

size_t moe_count_bytes(int64_t tokens, int64_t experts, int64_t top)
{
    if (alone(tokens, top)) return 0;
    int run, runs;
    runs_of(tokens, run, runs);
    return (size_t)runs * ((experts + 3) / 4 * 4) * 4;
}

hipError_t launch_moe_route(const void* logits, int64_t stride, bool f32, const float* bias, int64_t tokens, int64_t experts, int64_t top, int64_t groups, int64_t top_groups, float scale,
                            bool sigmoid, bool renorm, bool sum2, float* weights, int32_t* chosen, int32_t* offsets, int32_t* rows, int32_t* places, void* counts, hipStream_t st)
{
    RouteArgs a{logits, stride, bias, tokens, (int)experts, (int)top, (int)groups, (int)top_groups, scale, weights, chosen, offsets, rows, places, static_cast<int32_t*>(counts), 0, 0, 0, kMaxWaves,
                sigmoid, renorm, sum2 && groups > 1, alone(tokens, top), fast_div_by((uint32_t)(experts / groups)), fast_div_by((uint32_t)top), fast_div_by((uint32_t)(experts + 3) / 4)};
    runs_of(tokens, a.run, a.runs);
    a.wide = (int)(experts + 3) / 4 * 4;
    if (a.alone) {
        a.run = (int)tokens;
        a.runs = 1;
    }
    while (a.words * 32 < a.run) a.words *= 2;
    hipError_t e;
    if (bias || a.sum2) e = f32 ? route<kScore, true>(a, st) : route<kScore, false>(a, st);
    else e = f32 ? route<kLogit, true>(a, st) : route<kPacked, false>(a, st);
    if (e != hipSuccess || a.alone) return e;
    const size_t lds = (kMaxWaves + 8 * kMaxThreads + kMaxWaves * experts) * 4;
    static LdsAttrOnce attr;
    if ((e = attr.ensure(reinterpret_cast<const void*>(moe_place_kernel), 163840)) != hipSuccess) return e;
    hipLaunchKernelGGL(moe_place_kernel, dim3(a.runs), dim3(kMaxThreads), lds, st, a);
    return hipGetLastError();
}

hipError_t launch_moe_combine(const void* y, int64_t y_rows, bool y_f32, const int32_t* places, const float* weights, const void* shared, bool shared_f32, int64_t tokens, int64_t top,
                              int64_t cols, void* out, bool out_f32, hipStream_t st)
{
    const CombineArgs a{y, y_rows, places, weights, shared, out, tokens, cols, (int)top, shared_f32, out_f32};
    const auto odd = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; };
    if (y_rows == 0 || cols % 8 != 0 || odd(y) || odd(shared) || odd(out)) {
        const dim3 grid((unsigned)std::min<int64_t>((tokens * cols + 255) / 256, 1 << 20));
        if (y_f32) hipLaunchKernelGGL(moe_combine_any_kernel<true>, grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL(moe_combine_any_kernel<false>, grid, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    int wide = 1;
    while (wide < 256 && wide * 8 < cols) wide *= 2;
    const int64_t most = ((int64_t)1 << 22) * (256 / wide);      // tokens of a launch, which takes fewer than 2^32 threads along x
    for (int64_t first = 0; first < tokens; first += most) {
        CombineArgs c = a;
        c.tokens = std::min(tokens - first, most);
        c.places += first * top;
        c.weights += first * top;
        if (shared) c.shared = static_cast<const char*>(shared) + first * cols * (shared_f32 ? 4 : 2);
        c.out = static_cast<char*>(out) + first * cols * (out_f32 ? 4 : 2);
        const dim3 grid((unsigned)((c.tokens + 256 / wide - 1) / (256 / wide)), (unsigned)((cols / 8 + 255) / 256));
        if (y_f32) hipLaunchKernelGGL(moe_combine_kernel<true>, grid, dim3(256), 0, st, c, wide);
        else hipLaunchKernelGGL(moe_combine_kernel<false>, grid, dim3(256), 0, st, c, wide);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace fp4mr
