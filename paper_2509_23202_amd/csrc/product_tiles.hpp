// What the kernels of 8-bit products share: rows grouped by expert, operands by rows of 128 bytes in LDS, the order of tiles.
#pragma once

#include "device_util.hpp"
#include "internal.hpp"

namespace fp4mr {
namespace {

struct Rows {
    int expert, begin, end;    // rows begin .. end - 1 of the output; none: begin == end
};

// G: what a kernel is called with; it has `offsets` (experts + 1 of them), `experts`, and `rows`, the output's.
// Rows of expert base + lane, kept within the output whatever the offsets hold, and the inclusive sum over the lanes of their tiles of R rows.
struct ExpertTiles {
    int lo, hi, upto;
};
template <typename G>
__device__ __forceinline__ ExpertTiles expert_tiles(const G& g, int base, int R)
{
    const int e = base + ((int)threadIdx.x & 63), at = min(e, g.experts - 1), T = (int)g.rows;
    const int begin = g.offsets[at], end = g.offsets[at + 1];
    ExpertTiles x;
    x.lo = min(max(begin, 0), T);
    x.hi = min(max(end, x.lo), T);
    int n = e < g.experts ? (x.hi - x.lo + R - 1) / R : 0;
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xf, 0xf, true);     // row_shr 1, 2, 4, 8: the sum within sixteen lanes
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xa, 0xf, false);    // row_bcast 15 to the second and fourth sixteen, row_bcast 31 to the second half
    n += __builtin_amdgcn_update_dpp(0, n, 0x143, 0xc, 0xf, false);
    x.upto = n;
    return x;
}

// Tiles of R rows of all experts: tiles never span experts, and those of an expert follow one another.  Offsets that do not decrease make `most` at most.
// first: of the first 64 experts.
template <typename G>
__device__ __forceinline__ int count_tiles(const G& g, const ExpertTiles& first, int R, int most)
{
    int n = min(__builtin_amdgcn_readlane(first.upto, 63), most);
    for (int base = 64; base < g.experts; base += 64) n = min(n + __builtin_amdgcn_readlane(expert_tiles(g, base, R).upto, 63), most);
    return n;
}

template <typename G>
__device__ __forceinline__ Rows find_tile(const G& g, const ExpertTiles& first, int tile, int R)
{
    ExpertTiles x = first;
    for (int base = 0, before = 0;;) {
        const uint64_t here = __ballot(tile < before + x.upto);
        if (here) {
            const int l = __builtin_ctzll(here), earlier = l ? __builtin_amdgcn_readlane(x.upto, l - 1) : 0;
            const int begin = __builtin_amdgcn_readlane(x.lo, l) + (tile - before - earlier) * R;
            return Rows{base + l, begin, min(begin + R, __builtin_amdgcn_readlane(x.hi, l))};
        }
        before += __builtin_amdgcn_readlane(x.upto, 63);
        base += 64;
        if (base >= g.experts) return Rows{0, 0, 0};
        x = expert_tiles(g, base, R);
    }
}

constexpr uint32_t kOutside = (uint32_t)kFp8MaxGathered;    // an offset past every operand, to which K may be added

// What the pieces of a row are exchanged by: the sixteen rows of a fragment, which lie next to each other (X) or four by four, sixteen apart (W), have every
// pair of key and row % 2 once.
__device__ __forceinline__ int x_key(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int w_key(int row) { return ((row >> 1) & 1) | (row / 16 & 3) << 1; }

// A copy of a lane's number that the compiler takes for another one: what is computed from it stays where it is needed, once a tile, instead of in registers
// throughout the main loop.
__device__ __forceinline__ int kept_here(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// 16 or 4 bytes of every lane to LDS, the lanes' one behind the other from `to`
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t from, char* smem, int to, uint32_t offset, int uniform_offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)((lds_char*)smem + to), 16, offset, uniform_offset, 0, 0);
}
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t from, char* smem, int to, uint32_t offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)((lds_char*)smem + to), 4, offset, 0, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)(bytes > 0xffffffffll ? 0xffffffffu : (uint32_t)bytes), 0x00020000);
}

// Workgroups are dealt round-robin to the eight XCDs: each gets one contiguous range of tiles, in bands of four rows of tiles, so that those that share an
// L2 share operands.
__device__ __forceinline__ void place(int bid, int n, int tiles_m, int tiles_n, int& tm, int& tn)
{
    const int per = n >> 3, rem = n & 7, xcd = bid & 7, idx = bid >> 3;
    const int at = xcd < rem ? xcd * (per + 1) + idx : rem * (per + 1) + (xcd - rem) * per + idx;
    const int band = 4 * tiles_n, first = at / band * 4, high = min(tiles_m - first, 4), in = at % band;
    tm = first + in % high;
    tn = in / high;
}

}  // namespace
}  // namespace fp4mr
