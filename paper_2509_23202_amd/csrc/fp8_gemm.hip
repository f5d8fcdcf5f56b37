// Products of 8-bit operands with a scale per block of 128, for one weight matrix or for rows grouped by expert.
//
//   out[m,n] = sum_b sa[m,b] sw[n/128,b] p_b[m,n],   p_b[m,n] = sum over the 128 k of block b of a[m,k] w[n,k]
//
// v_mfma_f32_16x16x128_f8f6f4 yields p_b of sixteen rows and sixteen columns; the vector ALU adds it, times its two scales, to an
// fp32 accumulator.  The instruction adds eight products at a time in fewer bits than fp32 has: what lies below 2^-13 of the power of two of
// the largest of the eight is dropped (measured; every 8-bit MFMA does), 1.4e-5 of a sum of normal values, where a bf16 output is rounded to
// 2^-9.  Products with an fp32 output are for those who go on with the sums: they multiply the codes as fp16, which holds them, on the fp16
// MFMA, whose sums are fp32 (4096 x 4096 x 4096: 175 us, 0.79 PFLOP/s, where bf16 takes 63: a step of the 64-row tile, the only one with such sums, takes 0.62 us for 0.32, and the larger tiles do
// more to a step; few rows take the same time either way).  The W codes are the MFMA's A operand and the activations its B operand: a lane then has four consecutive n of one
// m, and the one activation scale.  Both operands are row-major, 128 bytes of a row to a step: lane l reads row l % 16, and from the row's
// eight pieces of 16 bytes the pieces l / 16 and l / 16 + 4 (the product does not care which of the 128 k is which, as long as both
// operands agree).
#include "product_tiles.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

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

constexpr uint32_t kPast = 0x08000000u;       // past all activations' scales (4 / 128 of kOutside), and kOutside may be added

// ---------------------------------------------------------------- few rows: weights streamed from memory
// 16 TN columns and 16 TM rows to a tile; a workgroup walks a run of tiles.  Its waves share K, each with a run of blocks; a block's codes and scales go to the
// wave's own part of LDS by direct-to-LDS loads, D blocks ahead, the next tile's behind this one's, so that what is on its way never runs dry
// and no wave waits for another but to add up a tile.  Every weight is read once for sixteen or thirty-two rows, and memory bounds it: 1 x 28672 x 4096 takes 25 us, 4.7 TB/s, 16 tokens on
// 64 experts of 4096 x 4096, four each, 93 us, 7 TB/s of those experts' weights; 1 x 4096 x 4096 takes 4.4 to 5.6 by card, three of them start-up.  K over the waves and not over
// workgroups: their sums are joined in LDS, in their order, by one launch.  A ring to a wave: tiles of 64 rows, whose waves meet at
// every block, take 33 us for the first of these.
template <int TM_, int TN_, int WAVES_, int D_>
struct Stream {
    static constexpr int TM = TM_, TN = TN_, WAVES = WAVES_, D = D_;
    static constexpr int SLOT = (TN + TM) * 2048 + 256;      // W, A, and the scales: lane t 16 + r: of row r of A fragment t, lane 63: of W
    static constexpr int LOADS = 2 * (TN + TM) + 1;
    static constexpr int PART = WAVES * TM * TN * 1024;      // partial sums, of two tiles in turn
    static constexpr int lds() { return WAVES * D * SLOT + 2 * PART; }
    static_assert(TM <= 3 && lds() <= 163840 && D * LOADS < 64, "");
};

// The scale, whichever block it is of, of a row that an index outside A stands for.
__device__ const float kZeroRowScale = 0.0f;

template <bool GROUPED, bool OUT_F32, typename C>
__global__ __launch_bounds__(C::WAVES * 64) void fp8_stream_kernel(Fp8Args g, int tiles_m, int tiles_n)
{
    constexpr int TM = C::TM, TN = C::TN, WAVES = C::WAVES, D = C::D;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int K = (int)g.K, KB = K >> 7, blocks_n = (int)((g.N + 127) >> 7);
    const bool gather = GROUPED && g.index != nullptr;
    ExpertTiles experts{0, 0, 0};
    if constexpr (GROUPED) {
        experts = expert_tiles(g, 0, 16 * TM);
        tiles_m = count_tiles(g, experts, 16 * TM, tiles_m);
    }
    const int64_t ntiles = (int64_t)tiles_m * tiles_n;
    const int tile_first = (int)(ntiles * blockIdx.x / gridDim.x), tile_end = (int)(ntiles * (blockIdx.x + 1) / gridDim.x);
    if (tile_first >= tile_end) return;
    const int each = (KB + WAVES - 1) / WAVES, kb_first = wave * each;

    // ---- loads: block `kb` of tile `at`, and what goes with the tile.  Rows that it does not have lie outside of the operands: zeros.
    const int ring = wave * D * C::SLOT;
    const int piece = (lane & 7) ^ x_key(lane / 8);               // (rows r and r + 8 of sixteen: the key of the second is the first's + 4)
    const uint32_t wo = (uint32_t)(lane / 8) * (uint32_t)K + piece * 16, wo8 = (uint32_t)(lane / 8 + 8) * (uint32_t)K + (piece ^ 4) * 16;
    __amdgpu_buffer_rsrc_t rw, rx;
    uint32_t xo[TM][2];
    const float* scale = nullptr;
    int scale_on = -1;         // 0: the same for every block
    Rows r{0, 0, 0};
    int n0 = 0, at_m = -1;
    auto locate = [&](int tile) {
        const int tm = tile / tiles_n;
        n0 = (tile - tm * tiles_n) * 16 * TN;
        if (tm != at_m) {
            at_m = tm;
            if constexpr (GROUPED) r = find_tile(g, experts, tm, 16 * TM);
            else r = Rows{0, tm * 16 * TM, min((tm + 1) * 16 * TM, (int)g.rows)};
            const int64_t x0 = gather ? 0 : r.begin, x_rows = gather ? g.a_rows : r.end - r.begin;
            rx = make_rsrc(g.a + x0 * K, x_rows * K);
            auto x_row = [&](int m) -> int64_t {      // of A, from x0; outside: x_rows
                const int64_t row = r.begin + m >= r.end ? -1 : gather ? g.index[r.begin + m] : m;
                return row >= 0 && row < x_rows ? row : x_rows;
            };
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t row = x_row(t * 16 + h * 8 + lane / 8);
                    xo[t][h] = (row < x_rows ? (uint32_t)row * (uint32_t)K : kOutside) + (piece ^ (4 * h)) * 16;
                }
            int64_t row = x_row(min(lane, 16 * TM - 1));
            const bool none = row == x_rows;
            if (none) row = 0;                        // (any: its codes are zeros, and the output's row is not stored)
            scale = g.a_scales + (x0 + row) * KB;
            if (gather && none) scale = &kZeroRowScale;
            if constexpr (GROUPED) scale_on = gather && none && lane != 63 ? 0 : -1;
        }
        rw = make_rsrc(g.w + ((int64_t)r.expert * g.N + n0) * K, (int64_t)min((int)g.N - n0, 16 * TN) * K);
        if (lane == 63) scale = g.w_scales + ((int64_t)r.expert * blocks_n + (n0 >> 7)) * KB;
    };
    int load_tile = tile_first, load_kb = 0, load_slot = 0;
    auto issue = [&]() {
        const int kb = min(kb_first + load_kb, KB - 1), to = ring + load_slot * C::SLOT;     // (past the last block: it again, with a scale of zero)
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            load_lds16(rw, smem, to + i * 2048, wo + (uint32_t)(16 * i) * (uint32_t)K, kb * 128);
            load_lds16(rw, smem, to + i * 2048 + 1024, wo8 + (uint32_t)(16 * i) * (uint32_t)K, kb * 128);
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            load_lds16(rx, smem, to + (TN + t) * 2048, xo[t][0], kb * 128);
            load_lds16(rx, smem, to + (TN + t) * 2048 + 1024, xo[t][1], kb * 128);
        }
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uintptr_t>(scale + (GROUPED ? kb & scale_on : kb))),
                                         (lds_void*)((lds_char*)smem + to + (TN + TM) * 2048), 4, 0, 0);
        load_slot = load_slot == D - 1 ? 0 : load_slot + 1;
        if (++load_kb == each) {
            load_kb = 0;
            if (++load_tile < tile_end) locate(load_tile);      // (behind the last tile: its last block again, which nobody reads)
            else load_kb = each - 1;
        }
    };
    locate(tile_first);
    const Rows r_first = r;
#pragma unroll
    for (int d = 0; d < D - 1; ++d) issue();

    // ---- products
    const int l16 = lane & 15, f_at = l16 * 128 + ((lane >> 4) ^ x_key(l16)) * 16;
    int slot = 0;
    // what the tile that is multiplied has; the loads may be a tile or more ahead
    Rows mine = r_first;
    int mine_m = tile_first / tiles_n;
    for (int tile = tile_first; tile < tile_end; ++tile) {
        v4f acc[TM][TN];
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
            for (int i = 0; i < TN; ++i) acc[t][i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int k = 0; k < each; ++k) {
            issue();
            wait_vmcnt<(D - 1) * C::LOADS>();
            asm volatile("" ::: "memory");
            const char* from = smem + ring + slot * C::SLOT;
            v4i wf[TN][2], af[TM][2];
            float sa[TM];
            auto read = [&](const char* p, v4i (&f)[2]) {
                f[0] = *reinterpret_cast<const v4i*>(p + f_at);
                f[1] = *reinterpret_cast<const v4i*>(p + (f_at ^ 64));
            };
#pragma unroll
            for (int i = 0; i < TN; ++i) read(from + i * 2048, wf[i]);
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                read(from + (TN + t) * 2048, af[t]);
                sa[t] = reinterpret_cast<const float*>(from + (TN + TM) * 2048)[t * 16 + l16];
            }
            float sw = reinterpret_cast<const float*>(from + (TN + TM) * 2048)[63];
            sw = kb_first + k < KB ? sw : 0.0f;
            wait_lgkmcnt0();      // (the slot is loaded again by the next issue but D - 2)
            asm volatile("" ::: "memory");
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                const float s = kb_first + k < KB ? sw * sa[t] : 0.0f;
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    const v4f p = OUT_F32 ? mfma_half(to_half(wf[i]), to_half(af[t])) : mfma_fp8(wf[i], af[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][i][e] = fmaf(s, p[e], acc[t][i][e]);
                }
            }
            slot = slot == D - 1 ? 0 : slot + 1;
        }
        // ---- the waves' sums in their order, and out
        v4f* const part = reinterpret_cast<v4f*>(smem + WAVES * D * C::SLOT + ((tile - tile_first) & 1) * C::PART);
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
            for (int i = 0; i < TN; ++i) part[(wave * TM * TN + t * TN + i) * 64 + lane] = acc[t][i];
        wait_lgkmcnt0();
        block_barrier();
        const int tm = tile / tiles_n, col0 = (tile - tm * tiles_n) * 16 * TN;
        if (tm != mine_m) {
            mine_m = tm;
            if constexpr (GROUPED) mine = tm == at_m ? r : find_tile(g, experts, tm, 16 * TM);
            else mine = Rows{0, tm * 16 * TM, min((tm + 1) * 16 * TM, (int)g.rows)};
        }
        for (int q = wave; q < TM * TN; q += WAVES) {
            v4f sum = part[q * 64 + lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) sum += part[(v * TM * TN + q) * 64 + lane];
            const int m = mine.begin + 16 * (q / TN) + l16, n = col0 + 16 * (q % TN) + (lane >> 4) * 4;
            if (m >= mine.end) continue;
            const int64_t o = (int64_t)m * g.N + n;
            const int have = (int)g.N - n;
            if constexpr (OUT_F32) {
                float* const to = static_cast<float*>(g.out) + o;
                if (have >= 4) __builtin_memcpy(to, &sum, 16);
                else for (int e = 0; e < have; ++e) to[e] = sum[e];
            } else {
                const __bf16 y[4] = {(__bf16)sum[0], (__bf16)sum[1], (__bf16)sum[2], (__bf16)sum[3]};
                __bf16* const to = static_cast<__bf16*>(g.out) + o;
                if (have >= 4) __builtin_memcpy(to, y, 8);      // (rows of an odd number of columns begin at any even byte)
                else
                    for (int e = 0; e < have; ++e) to[e] = e == 0 ? y[0] : e == 1 ? y[1] : y[2];
            }
        }
    }
    wait_vmcnt<0>();    // (loads to LDS past the last block)
}

// ---------------------------------------------------------------- tiles
// BM x BN to a workgroup of NWM x NWN waves, each 16 TM x 64; a workgroup walks tiles.  A stage is 128 columns of both operands' rows in LDS, eight
// rows to a 1 KB direct-to-LDS load; the sixteen-byte pieces of a row lie exchanged by a key, so that sixteen rows' reads of one piece touch
// every bank once.  A step multiplies a stage: the W fragments stay in registers, the X fragments pass through a few buffers, and the
// products of one X fragment are added to the accumulators while the next one's run.  The requests for the stage S - 1 steps on go out between the products, so many to each X fragment;
// when this tile's have all gone out, they are the next tile's, whose first stages are there before this tile's output has left.
//   Two stages (256 rows, whose stages leave no room for a third): before its last X fragment a wave has read all it needs of the stage.  There it waits for its loads of the
// next one, the workgroup meets, and the last fragment's products cover the reads of the next step's first fragments.  The eight waves have all 512 registers of a SIMD's two places,
// and the step is one loop body: unrolled it spills.
//   Four stages (64 and 128 rows): a step begins with the meeting, and four steps are one body, so that a stage's place in LDS is a constant.
//   K counts as a multiple of four blocks: the last ones' scales are zeros.  The activations' scales take the codes' way four blocks at a time (a chunk: sixteen rows and four blocks to a
// load), in a ring of chunks.  The first chunk of a tile goes out whole in front of its first codes; of chunk c + 1, a part goes out with the codes of each of the steps 4c .. 4c + 3, or
// where that is past the last chunk to a place that nobody reads: every wave has the same number of loads on their way at any step, which the waits count.  With three
// slots (two stages) chunk c + 1 overwrites chunk c - 2, last read in front of step 4c - 5, behind the meeting of step 4c - 2; four stages are ahead by two steps more and have a fourth slot.
//   The output is rounded, turned through 2 KB of LDS of each wave's own, and leaves in lines of 128 bytes.
//   What bounds them.  256 x 256: 4096 x 28672 x 4096 takes 443 to 460 us, 2.1 PFLOP/s: a step takes 1.75 to 1.85 us, in which the matrix cores are busy for 55 % at the 2.0 GHz that the
// power allows on such operands (a loop of these products in registers reaches 3.7 PFLOP/s on random codes, 5.0 on zeros; a library product with one scale
// for a tensor takes 398 us here), and the stores of a tile, 5 us of every 63, are not covered.  128 x 128 and 64 x 128: 0.50 to 0.57 and 0.32 to 0.42 us a step, 57 to 77 bytes a ns to a compute unit, which is what
// the mix of operands from L2 and from memory arrives at; without loads a step of 128 x 128 takes 0.41.
template <int TM_, int NWM_, int NWN_, int STAGES_>
struct Tile {
    static constexpr int TM = TM_, TN = 4, NWM = NWM_, NWN = NWN_, S = STAGES_, NW = NWM * NWN;
    static constexpr int BM = 16 * TM * NWM, BN = 64 * NWN;
    static constexpr int STAGE = (BM + BN) * 128, CHUNK = BM * 16, SLOTS = S == 2 ? 3 : 4;
    static constexpr int XL = BM / 8 / NW, WL = BN / 8 / NW, LPS = XL + WL + 1;   // loads of a wave for a step: X, W, scales
    static constexpr int NB = (BN + 127) / 128;
    static constexpr int padded(int blocks) { return (blocks + 3) & ~3; }               // steps of a tile
    static constexpr int out(bool f32) { return NW * 16 * 64 * (f32 ? 4 : 2); }
    static constexpr int w_room(int blocks) { return (NB * blocks + 63) / 64 * 256; }   // the scales of W of a tile
    static constexpr int lds(int blocks, bool f32) { return S * STAGE + SLOTS * CHUNK + 256 + out(f32) + 2 * w_room(blocks); }
    // blocks of K that the scales of W have room for
    static constexpr int max_blocks(bool f32) { return (163840 - lds(0, f32)) / 512 * 64 / NB; }
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && TM % 2 == 0 && BM <= 64 * NW && BM >= 64, "");
    static constexpr bool ROLLED = TM >= 8;    // (see the kernel)
    static_assert(S == (ROLLED ? 2 : 4) && (S - 1) * LPS < 64, "");
};

// EXACT: fp32 sums (the fp16 MFMA); OUT_F32: they leave as fp32.  SPLIT: a unit of work is one part of K of a tile, each of part_blocks blocks but the last, and
// what leaves is its sums, to the part's own copy of the output.
template <bool GROUPED, bool EXACT, bool OUT_F32, bool SPLIT, typename C>
__global__ __launch_bounds__(C::NW * 64) __attribute__((amdgpu_waves_per_eu(2))) void fp8_tile_kernel(Fp8Args g, int tiles_m, int tiles_n, int split_parts, int split_blocks)
{
    static_assert(!SPLIT || (OUT_F32 && !GROUPED), "");
    const int parts = SPLIT ? split_parts : 1, part_blocks = SPLIT ? split_blocks : (int)(g.K >> 7);
    constexpr int TM = C::TM, TN = C::TN, NW = C::NW, S = C::S, LPS = C::LPS;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    // places in LDS: the stages, then these
    constexpr int kChunks = S * C::STAGE, kNowhere = kChunks + C::SLOTS * C::CHUNK, kRoom = kNowhere + 256, kWScales = kRoom + C::out(OUT_F32);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave % C::NWM, wn = wave / C::NWM;
    const int K = (int)g.K, KS = K >> 7, blocks_n = (int)((g.N + 127) >> 7);

    constexpr bool KEEP = !C::ROLLED;      // (those have the registers)
    ExpertTiles experts{0, 0, 0};
    if constexpr (GROUPED) {
        experts = expert_tiles(g, 0, C::BM);
        tiles_m = count_tiles(g, experts, C::BM, tiles_m);
    }
    const int ntiles = tiles_m * tiles_n * parts;
    int tile = blockIdx.x;
    if (tile >= ntiles) return;

    // ---- the tile whose operands are requested.  Rows that it does not have lie outside of the operand: their loads bring zeros, scales too.
    const bool gather = GROUPED && g.index != nullptr;
    Rows r{0, 0, 0};
    int n0 = 0, w_side = 1, part = 0, part_k0 = 0, part_n = 0;
    auto k0 = [&]() { return SPLIT ? part_k0 : 0; };     // its blocks of K: KB() of them from k0() on
    auto KB = [&]() { return SPLIT ? part_n : KS; };
    __amdgpu_buffer_rsrc_t rx, rw, rs;
    uint32_t xo[C::XL], wo[C::WL], so[4];
    // ---- loads.  t: the step whose loads go out; its scales are a part of chunk t / 4 + 1, to slot t_slot, or where that is past the last one, nowhere.
    // (Past the last step of the last tile its codes again, into a stage that nobody reads.)
    int t = 0, t_slot = 0;
    uint32_t t_block = 0;      // of a lane, among the chunk's four, as an offset
    auto scale_block = [&](int chunk) { return 4 * chunk + (lane & 3) < KB() ? (uint32_t)(k0() + 4 * chunk + (lane & 3)) * 4 : kPast; };
    constexpr bool ROLLED = C::ROLLED;
    auto issue_scales = [&](int q, int to) {    // a part: by several waves, where there are fewer loads than waves, to the same end
        load_lds4(rs, smem, to, so[q] + t_block);
    };
    const int part_at = wave % (C::BM / 64) * 256;
    auto issue_step = [&](int stage, int q, int i) {
        const int at = (k0() + min(t, KB() - 1)) * 128;
        if (i < C::XL) load_lds16(rx, smem, stage + (i * NW + wave) * 1024, xo[i < C::XL ? i : 0], at);
        else if (i < LPS - 1) load_lds16(rw, smem, stage + C::BM * 128 + ((i - C::XL) * NW + wave) * 1024, wo[i < LPS - 1 && i >= C::XL ? i - C::XL : 0], at);
        else issue_scales(ROLLED ? 0 : q, 4 * (t >> 2) + 4 < KB() ? kChunks + t_slot * C::CHUNK + q * (C::BM / 64) * 256 + part_at : kNowhere);
    };
    auto next_slot = [](int slot) { return slot == C::SLOTS - 1 ? 0 : slot + 1; };
    // In front of a tile's first codes: where its operands are, the scales of W, the first chunk.
    auto begin_tile = [&]() {
        const int lane = kept_here((int)threadIdx.x & 63);
        int tm, tn;
        if constexpr (!SPLIT) {
            place(tile, ntiles, tiles_m, tiles_n, tm, tn);
        } else {       // (neighbours of different parts, so that with eight parts an XCD has one part of K of both operands)
            const int at = tile / parts;
            part = tile - at * parts;
            tn = at / tiles_m;
            tm = at - tn * tiles_m;
            part_k0 = part * part_blocks;
            part_n = min(part_blocks, KS - part_k0);
        }
        if constexpr (GROUPED) r = find_tile(g, KEEP ? experts : expert_tiles(g, 0, C::BM), tm, C::BM);
        else r = Rows{0, tm * C::BM, min((tm + 1) * C::BM, (int)g.rows)};
        n0 = tn * C::BN;
        const int64_t x0 = gather ? 0 : r.begin, x_rows = gather ? g.a_rows : r.end - r.begin;
        const int w_rows = min((int)g.N - n0, C::BN);
        rx = make_rsrc(g.a + x0 * K, x_rows * K);
        rs = make_rsrc(g.a_scales + x0 * KS, x_rows * KS * 4);
        rw = make_rsrc(g.w + ((int64_t)r.expert * g.N + n0) * K, (int64_t)w_rows * K);
        auto x_offset = [&](int m, int pitch) -> uint32_t {
            const int row = r.begin + m >= r.end ? -1 : gather ? g.index[r.begin + m] : m;
            return row >= 0 && row < x_rows ? (uint32_t)row * (uint32_t)pitch : kOutside;
        };
#pragma unroll
        for (int i = 0; i < C::XL; ++i) {
            const int m = (i * NW + wave) * 8 + lane / 8;
            xo[i] = x_offset(m, K) + (uint32_t)((lane & 7) ^ x_key(m)) * 16;
        }
#pragma unroll
        for (int i = 0; i < C::WL; ++i) {
            const int n = (i * NW + wave) * 8 + lane / 8;
            wo[i] = (n < w_rows ? (uint32_t)n * (uint32_t)K : kOutside) + (uint32_t)((lane & 7) ^ w_key(n)) * 16;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) so[q] = x_offset((q * (C::BM / 64) + wave % (C::BM / 64)) * 16 + lane / 4, KS * 4);

        w_side ^= 1;
        // (of one part of K: a row of the scales at a time, else all rows, which lie behind one another)
        const int have = SPLIT ? KB() : min(C::NB, blocks_n - (n0 >> 7)) * KB();
        for (int nb = 0; nb < (SPLIT ? min(C::NB, blocks_n - (n0 >> 7)) : 1); ++nb) {
            const __amdgpu_buffer_rsrc_t rsw = make_rsrc(g.w_scales + ((int64_t)r.expert * blocks_n + (n0 >> 7) + nb) * KS + k0(), (int64_t)have * 4);
            for (int i = wave * 64; i < have; i += NW * 64)
                if (i + lane < have) load_lds4(rsw, smem, kWScales + w_side * C::w_room(part_blocks) + (nb * part_blocks + i) * 4, (uint32_t)(i + lane) * 4);
        }
        t = 0;
        t_block = scale_block(0);
#pragma unroll
        for (int q = 0; q < 4; ++q) issue_scales(q, kChunks + t_slot * C::CHUNK + q * (C::BM / 64) * 256 + part_at);
        t_slot = next_slot(t_slot);
        t_block = scale_block(1);
    };
    // Behind the loads of a step.  fourth: t is now a multiple of four.
    auto next_t = [&](bool fourth) {
        ++t;
        if constexpr (ROLLED) {
            const uint32_t first = so[0];      // (part t % 4 of a chunk stays in front)
            so[0] = so[1];
            so[1] = so[2];
            so[2] = so[3];
            so[3] = first;
        }
        const bool on = fourth & (t < C::padded(KB()));
        t_slot = on ? next_slot(t_slot) : t_slot;
        t_block = on ? scale_block((t >> 2) + 1) : t_block;
    };

    // ---- fragments: row l % 16 of X; for the i-th of W, of the wave's 64 columns that which leaves a lane sixteen consecutive ones of the output
    const int l16 = lane & 15, xr = wm * TM * 16 + l16, wr = wn * 64 + l16 / 4 * 16 + l16 % 4;
    const int xf_at = xr * 128 + ((lane >> 4) ^ x_key(xr)) * 16;
    const int wf_at = C::BM * 128 + wr * 128 + ((lane >> 4) ^ w_key(wr)) * 16;    // (rows 4 i on have the same key)
    auto read = [&](int at, int more, v4i (&f)[2]) {
        f[0] = *reinterpret_cast<const v4i*>(smem + at + more);
        f[1] = *reinterpret_cast<const v4i*>(smem + (at ^ 64) + more);
    };
    const int sx_at = kChunks + (wm * TM * 64 + l16 * 4) * 4;

    begin_tile();
#pragma unroll
    for (int st = 0; st < S - 1; ++st) {
#pragma unroll
        for (int i = 0; i < LPS; ++i) issue_step(st * C::STAGE, st, i);
        next_t(st == 3);
    }
    wait_vmcnt<(S - 2) * LPS>();
    block_barrier();

    // EARLY: a step begins with the meeting that frees the stage before it and says that the next one is there, and its last fragments' products cover the reads
    // of the next step's first ones.  With two stages the meeting is in front of the last X fragment's products.
    constexpr bool EARLY = S > 2;
    constexpr int GROUPS = TM < 4 ? TM - 1 : 3, PER = (LPS + GROUPS - 1) / GROUPS, EACH_MFMA = (PER + TN - 1) / TN;   // a step's loads go out with so many X fragments
    constexpr int RING = TM < 4 ? TM : 4, AHEAD = RING / 2;                          // X fragments are read so many of them ahead
    v4i xf[RING][2], wf[TN][2];
    constexpr bool SX4 = TM <= 4;          // a lane's scales of four steps in registers, for every X fragment
    v4f sx4[SX4 ? TM : 1];
    float sx[RING];                        // or those of the fragments that were read
    int slot = 0, sw_at = kWScales + wn / 2 * part_blocks * 4;
    float sw = *reinterpret_cast<const float*>(smem + sw_at);
#pragma unroll
    for (int i = 0; i < TN; ++i) read(wf_at, i * 512, wf[i]);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        read(xf_at, j * 2048, xf[j]);
        if constexpr (!SX4) sx[j] = *reinterpret_cast<const float*>(smem + sx_at + j * 256);
    }
    if constexpr (SX4) {
#pragma unroll
        for (int j = 0; j < TM; ++j) sx4[j] = *reinterpret_cast<const v4f*>(smem + sx_at + j * 256);
    }

    for (;;) {
        const Rows here = r;       // (the loads move on to the next tile before this one is done)
        const int here_n0 = n0, here_tile = tile, here_part = part, blocks = KB();
        // p: the products of the X fragment before (and of the present one, where there are the registers)
        constexpr int P = TM >= 8 ? 1 : 2;
        v4f acc[TM][TN], p[P][TN];
        float s = 0.0f;            // their scale
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int i = 0; i < TN; ++i) acc[j][i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < TN; ++i) p[P - 1][i] = v4f{0.f, 0.f, 0.f, 0.f};

        // Step u of a chunk, 0 .. 3 (those past the last block add nothing: their scales are zeros): a constant where four steps are unrolled, so that a stage's
        // places are too, or not, where that takes more registers than there are.
        int steps = C::padded(blocks), kt = 0;
        asm volatile("" : "+s"(steps));    // (nothing that the compiler knows: every unrolled step is a block of its own to it, whose order it keeps)
        auto step = [&](auto u) {
            const int STAGE = u % S * C::STAGE, NEXT = (u + 1) % S * C::STAGE, FILL = (u + S - 1) % S * C::STAGE;
            const int Q = (u + S - 1) % 4;         // the part of a chunk that goes out
            const bool last = kt + 4 - u >= blocks;    // this is the tile's last chunk
            const int slot_next = next_slot(slot);
            const int sw_next_at = u < 3 ? sw_at + 4 * (u + 1) : last ? kWScales + w_side * C::w_room(part_blocks) + wn / 2 * part_blocks * 4 : sw_at + 16;   // (the next tile's, when the loads are there)
            auto meet = [&]() {
                wait_vmcnt<(EARLY ? S - 3 : S - 2) * LPS>();
                if constexpr (!EARLY) wait_lgkmcnt0();    // (early: what was read of the stage before has been multiplied)
                block_barrier();
            };
            if constexpr (EARLY) meet();
            Half32 wh[EXACT ? TN : 1];
            if constexpr (EXACT) {
#pragma unroll
                for (int i = 0; i < TN; ++i) wh[i] = to_half(wf[i]);
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                auto fetch = [&](int q) {     // X fragment q from the front of this stage
                    read(xf_at, q < TM ? STAGE + q * 2048 : NEXT + (q - TM) * 2048, xf[q % RING]);
                    if constexpr (!SX4) {
                        const int at = q < TM ? slot * C::CHUNK + u * 4 : u < 3 ? slot * C::CHUNK + (u + 1) * 4 : slot_next * C::CHUNK;
                        sx[q % RING] = *reinterpret_cast<const float*>(smem + sx_at + at + q % TM * 256);
                    }
                };
                if (EARLY || j + AHEAD < TM) fetch(j + AHEAD);
                float sw_next = sw;
                if (j == TM - 1) {
                    next_t(Q == 3);
                    if constexpr (!EARLY) {
                        meet();
#pragma unroll
                        for (int q = 0; q < AHEAD; ++q) fetch(TM + q);
                    }
                    sw_next = *reinterpret_cast<const float*>(smem + sw_next_at);
                }
                Half32 xh;
                if constexpr (EXACT) xh = to_half(xf[j % RING]);
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    v4f& to = acc[j == 0 ? TM - 1 : j - 1][i];
                    auto add = [&](const v4f& q) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[e] = fmaf(s, q[e], to[e]);
                    };
                    if constexpr (P == 1) add(p[0][i]);
                    if constexpr (EXACT) p[P == 1 ? 0 : j & 1][i] = mfma_half(wh[i], xh);
                    else p[P == 1 ? 0 : j & 1][i] = mfma_fp8(wf[i], xf[j % RING]);
                    if constexpr (P == 2) add(p[1 - (j & 1)][i]);
                    if (j == TM - 1) read(wf_at, NEXT + i * 512, wf[i]);
                    // (the order is kept: the additions of four products beside every MFMA, and a load or two)
#pragma unroll
                    for (int l = 0; l < EACH_MFMA; ++l)
                        if (j < GROUPS && i * EACH_MFMA + l < PER && j * PER + i * EACH_MFMA + l < LPS) issue_step(FILL, Q, j * PER + i * EACH_MFMA + l);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (SX4) {
                    s = sx4[j][(int)u] * sw;
                    if (u == 3) sx4[j] = *reinterpret_cast<const v4f*>(smem + sx_at + slot_next * C::CHUNK + j * 256);
                } else {
                    s = sx[j % RING] * sw;
                }
                if (u > 0) s = kt < blocks ? s : 0.0f;
                sw = sw_next;
                __builtin_amdgcn_sched_barrier(0);
            }
            ++kt;
            if (u == 3) {
                slot = slot_next;
                sw_at = sw_next_at;
            }
        };
        auto move_on = [&]() {     // the loads of this tile have gone out
            if (tile + (int)gridDim.x < ntiles) {
                tile += gridDim.x;
                begin_tile();
            }
        };
        if constexpr (ROLLED) {
#pragma clang loop unroll(disable)
            for (int part = 0; part < 2; ++part) {
                int to = part ? steps : steps - S + 1;
                asm volatile("" : "+s"(to));
#pragma clang loop unroll(disable)
                while (kt < to) step(kt & 3);
                if (part == 0) move_on();
            }
        } else {
            while (kt < steps) {
                const bool last = kt + 4 >= steps;
                step(std::integral_constant<int, 0>{});
#pragma unroll
                for (int j = 0; j < TM; ++j)     // (the step's products are not to be computed behind the branch)
#pragma unroll
                    for (int i = 0; i < TN; ++i) asm volatile("" : "+v"(acc[j][i]));
#pragma unroll
                for (int i = 0; i < TN; ++i) asm volatile("" : "+v"(p[P - 1][i]));
                if (last) move_on();
                if (kt < steps) step(std::integral_constant<int, 1>{});
                if (kt < steps) step(std::integral_constant<int, 2>{});
                if (kt < steps) step(std::integral_constant<int, 3>{});
            }
        }
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[TM - 1][i][e] = fmaf(s, p[P - 1][i][e], acc[TM - 1][i][e]);

        // ---- output: sixteen rows at a time through 16 x 64 elements of LDS of the wave's own, so that a row leaves as whole lines
        typedef std::conditional_t<OUT_F32, float, __bf16> Out;
        const int lane = kept_here((int)threadIdx.x & 63), l16 = lane & 15;
        constexpr int EACH = 16 / sizeof(Out), PIECES = 64 / EACH, ROWS = 64 / PIECES;     // pieces of a row; rows to a store
        auto key = [](int row) { return OUT_F32 ? row & 15 : row >> 1 & 7; };
        char* const room = smem + kRoom + wave * (C::out(OUT_F32) / NW);
        const int row0 = here.begin + wm * TM * 16 + lane / PIECES, col = here_n0 + wn * 64 + lane % PIECES * EACH, have = (int)g.N - col;
        const bool inside = here.begin + (wm + 1) * TM * 16 <= here.end && here_n0 + wn * 64 + 64 <= (int)g.N;
        Out* out = static_cast<Out*>(g.out) + ((int64_t)here_part * g.rows + row0) * g.N + col;
#pragma unroll
        for (int j = 0; j < TM; ++j) {
#pragma unroll
            for (int i = 0; i < TN; i += 8 / EACH == 2 ? 1 : 2) {
                const int piece = (lane >> 4) * (16 / EACH) + i * 4 / EACH;
                char* const to = room + l16 * (PIECES * 16) + (piece ^ key(l16)) * 16;
                if constexpr (OUT_F32) {
                    *reinterpret_cast<v4f*>(to) = acc[j][i];
                } else {
                    *reinterpret_cast<v8bf*>(to) = v8bf{(__bf16)acc[j][i][0], (__bf16)acc[j][i][1], (__bf16)acc[j][i][2], (__bf16)acc[j][i][3],
                                                        (__bf16)acc[j][i + 1][0], (__bf16)acc[j][i + 1][1], (__bf16)acc[j][i + 1][2], (__bf16)acc[j][i + 1][3]};
                }
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < 16 / ROWS; ++h) {
                const int row = h * ROWS + lane / PIECES;
                const v4i y = *reinterpret_cast<const v4i*>(room + row * (PIECES * 16) + (lane % PIECES ^ key(row)) * 16);
                // (rows of an odd number of columns begin at any even byte)
                if (inside) {
                    __builtin_memcpy(out, &y, 16);
                } else if (row0 + 16 * j + h * ROWS < here.end) {
                    if (have >= EACH) {
                        __builtin_memcpy(out, &y, 16);
                    } else {
                        const Out* const from = reinterpret_cast<const Out*>(room + row * (PIECES * 16) + (lane % PIECES ^ key(row)) * 16);
#pragma clang loop unroll(disable) vectorize(disable)
                        for (int e = 0; e < have; ++e) out[e] = from[e];
                    }
                }
                out += ROWS * g.N;
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
        if (tile == here_tile) break;
    }
    wait_vmcnt<0>();    // (loads to LDS past the last step)
}

template <bool GROUPED, bool EXACT, bool OUT_F32, bool SPLIT, typename C>
hipError_t launch_tile(const Fp8Args& g, int parts, int part_blocks, hipStream_t st)
{
    if (part_blocks > C::max_blocks(OUT_F32)) return hipErrorInvalidValue;      // (a plan keeps to it)
    static LdsAttrOnce attr;
    const hipError_t e = attr.ensure(reinterpret_cast<const void*>(fp8_tile_kernel<GROUPED, EXACT, OUT_F32, SPLIT, C>), 163840);
    if (e != hipSuccess) return e;
    const int64_t tiles_m = GROUPED ? g.rows / C::BM + std::min<int64_t>(g.experts, g.rows) : (g.rows + C::BM - 1) / C::BM, tiles_n = (g.N + C::BN - 1) / C::BN;
    const int64_t grid = std::min<int64_t>(tiles_m * tiles_n * parts, compute_units());
    hipLaunchKernelGGL((fp8_tile_kernel<GROUPED, EXACT, OUT_F32, SPLIT, C>), dim3((unsigned)grid), dim3(C::NW * 64), C::lds(part_blocks, OUT_F32), st, g, (int)tiles_m, (int)tiles_n, parts,
                       part_blocks);
    return hipGetLastError();
}

// The parts' sums in their order: for a product of few tiles and a long K, which would leave compute units idle (64 x 4096 x 14336: 50 us whole on tiles of 64 rows, 19 in parts with the sum).
template <bool OUT_F32>
__global__ __launch_bounds__(256) void fp8_join_kernel(const float* part, int parts, int64_t n, void* out)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    if (i + 4 <= n && n % 4 == 0) {
        v4f sum = *reinterpret_cast<const v4f*>(part + i);
        for (int p = 1; p < parts; ++p) sum += *reinterpret_cast<const v4f*>(part + p * n + i);
        const __bf16 y[4] = {(__bf16)sum[0], (__bf16)sum[1], (__bf16)sum[2], (__bf16)sum[3]};
        if constexpr (OUT_F32) __builtin_memcpy(static_cast<float*>(out) + i, &sum, 16);      // (an output begins at any element)
        else __builtin_memcpy(static_cast<__bf16*>(out) + i, y, 8);
    } else {
        for (int64_t e = i; e < i + 4 && e < n; ++e) {
            float sum = part[e];
            for (int p = 1; p < parts; ++p) sum += part[p * n + e];
            if constexpr (OUT_F32) static_cast<float*>(out)[e] = sum;
            else static_cast<__bf16*>(out)[e] = (__bf16)sum;
        }
    }
}

// A product in parts of K on tiles of C, and their sum.
template <bool OUT_F32, typename C>
hipError_t launch_parts(Fp8Args g, int parts, int part_blocks, void* partial, hipStream_t st)
{
    void* const out = g.out;
    g.out = partial;
    const hipError_t e = launch_tile<false, OUT_F32, true, true, C>(g, parts, part_blocks, st);
    if (e != hipSuccess) return e;
    const int64_t n = g.rows * g.N;
    hipLaunchKernelGGL(fp8_join_kernel<OUT_F32>, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, st, static_cast<const float*>(partial), parts, n, out);
    return hipGetLastError();
}

template <bool GROUPED, bool OUT_F32, typename C>
hipError_t launch_stream(const Fp8Args& g, hipStream_t st)
{
    static LdsAttrOnce attr;
    const hipError_t e = attr.ensure(reinterpret_cast<const void*>(fp8_stream_kernel<GROUPED, OUT_F32, C>), C::lds());
    if (e != hipSuccess) return e;
    const int64_t tiles_m = GROUPED ? g.rows / (16 * C::TM) + std::min<int64_t>(g.experts, g.rows) : (g.rows + 16 * C::TM - 1) / (16 * C::TM), tiles_n = (g.N + 16 * C::TN - 1) / (16 * C::TN);
    const int64_t per_cu = 163840 / C::lds(), grid = std::min<int64_t>(tiles_m * tiles_n, compute_units() * per_cu);
    hipLaunchKernelGGL((fp8_stream_kernel<GROUPED, OUT_F32, C>), dim3((unsigned)grid), dim3(C::WAVES * 64), C::lds(), st, g, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

typedef Tile<8, 2, 4, 2> Tile256;           // 256 x 256
typedef Tile<4, 2, 2, 4> Tile128;           // 128 x 128
typedef Tile<2, 2, 2, 4> Tile64;            // 64 x 128

// How a product runs.
struct Plan {
    int kind = 0;              // 0 .. 3: few rows, with 16 or 32 rows and 16 or 32 columns to a tile (bit 0: columns, bit 1: rows); 4, 5, 6: tiles of 64, 128, 256 rows
    int parts = 1, part_blocks = 0;
};

constexpr int kKinds = 7;
constexpr int kRows[kKinds] = {16, 16, 32, 32, 64, 128, 256}, kCols[kKinds] = {16, 32, 16, 32, 128, 128, 256};

// What a kind takes, microseconds on a device of `cus` compute units, as fitted to measurements on 256: rounds of tiles, each a fixed part and the steps of K (a quarter of its blocks where
// four waves share them; fp32 sums take a tile's steps twice the time), but no less than its weights take from memory: once for every row of tiles where rows are few, else once for each
// of the `sets` of weights that have rows.  Parts add the writing, reading and launch of their sum.
// The constants are a fit to all of those, not a kernel's own figures: large products run their 256-row tiles at the power limit, 1.75 to 1.85 us a step.
// Measured, each kind and number of parts forced in turn, on 183 products of 1 to 4096 rows with layers from 576 x 4096 to 28672 x 8192 and on 44 drawn ones, half of them by expert: the
// kind that is chosen takes 1.00 to 1.01 of the best one's time in the mean (on 44 more, that nothing was fitted to, 1.02 to 1.035), at worst 1.26 (256 x 1079 x 3584: 14.3 us on whole tiles, 11.3 in
// parts; 128 x 4096 x 4096: 12.8, 10.7) and by expert 1.37 to 1.46 (6240 rows of 5 experts 544 x 1664: 26 us on tiles of 128 rows, whose 254 in the mean are
// priced as one round where those experts' numbers of rows make two, 18 on tiles of 64); the others up to ten times it (1000 x 4096 x 4096: tiles of 128 rows 23.5 us, of 64 28.4, of 256 52; 905 x 1079 x
// 3584: of 64 15.5, of 128 21, of 256 47, 16 rows at a time 42; 770 rows of 52 experts 1856 x 1280: of 64 25, of 128 31, 32 rows at a time 36).
double kind_us(int kind, double rows, double tiles_m, double sets, double N, int64_t blocks, int parts, bool exact, int cus)
{
    static const double fixed[] = {0.44, 0.60, 0.66, 0.75, 0.82, 2.3, 5.6}, step[] = {0.28, 0.49, 0.46, 0.71, 0.37, 0.51, 1.5}, rate[] = {4.2e6, 10e6, 3.9e6, 7.9e6};
    const bool few = kind < 4;
    const int64_t steps = few ? (blocks + 3) / 4 : ((blocks + parts - 1) / parts + 3) / 4 * 4;
    const double rounds = std::ceil(tiles_m * std::ceil(N / kCols[kind]) * parts / (kind == 0 ? 2 * cus : cus)), work = rounds * (fixed[kind] + (double)steps * step[kind] * (exact && !few ? 2 : 1));
    const double weights = N * 128 * (double)blocks;
    if (few) return 2.1 + std::max(work, tiles_m * weights / (rate[kind] * cus / 256));
    return 2.3 + std::max(work, sets * weights / 4.8e6) + (parts > 1 ? 5.1 + parts * rows * N * 8 / 6e6 : 0.0);
}

constexpr int kMaxBlocks[2][kKinds] = {{1 << 15, 1 << 15, 1 << 15, 1 << 15, Tile64::max_blocks(false), Tile128::max_blocks(false), Tile256::max_blocks(false)},
                                       {1 << 15, 1 << 15, 1 << 15, 1 << 15, Tile64::max_blocks(true), 0, 0}};
// in parts of K: blocks of a part, whose sums leave as fp32 whatever the output is
constexpr int kMaxPartBlocks[2][kKinds] = {{0, 0, 0, 0, Tile64::max_blocks(true), Tile128::max_blocks(true), 0}, {0, 0, 0, 0, Tile64::max_blocks(true), 0, 0}};

constexpr int64_t kMostJoined = 1 << 30;     // elements of an output that is joined from parts, four to a thread

// The kind that takes least; in parts only where `room` bytes hold their sums and fewer would leave compute units idle, and up to sixteen rows one of the first two: in all of the products
// above one of those came within 2 % of every other (the whole search takes the host 0.5 us, this one 0.2 to 0.4).  Kinds of tiles take K from 512 on, where there is room for the scales of W.
Plan plan_fp8(const Fp8Args& g, bool grouped, bool out_f32, size_t room)
{
    const int64_t blocks = g.K >> 7;
    const int forced = options().fp8_variant, cus = compute_units();
    Plan best;
    best.part_blocks = (int)blocks;
    double best_us = 1e30;
    for (int kind = 0; kind < kKinds; ++kind) {
        if ((kind >= 4 && blocks < 4) || (kind >= 2 && g.rows <= 16 && !forced)) break;
        // rows of tiles; by expert: as if the rows were spread evenly over the experts, half a tile more to each than they fill
        const double active = (double)std::min<int64_t>(g.experts, g.rows);
        const double tiles_m = grouped ? active * std::max(1.0, (double)g.rows / active / kRows[kind] + 0.4) : (double)((g.rows + kRows[kind] - 1) / kRows[kind]);
        for (int parts = 1; parts <= 16; ++parts) {
            if (parts > 1 && (grouped || kind < 4 || kind > 5 || g.rows * g.N > kMostJoined || (size_t)parts * g.rows * g.N * 4 > room)) break;
            if (parts > 1 && !forced && (parts - 1) * tiles_m * std::ceil((double)g.N / kCols[kind]) >= cus) break;
            const int64_t each = parts == 1 ? blocks : ((blocks + parts - 1) / parts + 3) / 4 * 4;
            if (each > (parts > 1 ? kMaxPartBlocks : kMaxBlocks)[out_f32][kind]) continue;
            if (parts > 1 && (parts - 1) * each >= blocks) continue;      // (a part of nothing)
            const double us = kind_us(kind, (double)g.rows, tiles_m, grouped ? active : 1.0, (double)g.N, blocks, parts, out_f32, cus);
            const bool chosen = forced ? kind == (forced <= kKinds ? forced - 1 : forced <= 10 ? 4 : 5) && parts == (forced <= kKinds ? 1 : 2 << (forced - 8) % 3) : us < best_us;
            if (chosen) {
                best = Plan{kind, parts, (int)each};
                best_us = us;
            }
        }
    }
    return best;
}

template <bool GROUPED, bool OUT_F32>
hipError_t launch(const Fp8Args& g, const Plan& p, void* partial, hipStream_t st)
{
    if constexpr (!GROUPED) {
        if (p.parts > 1) {
            if (p.kind == 4) return launch_parts<OUT_F32, Tile64>(g, p.parts, p.part_blocks, partial, st);
            if constexpr (!OUT_F32) return launch_parts<OUT_F32, Tile128>(g, p.parts, p.part_blocks, partial, st);
        }
    }
    switch (p.kind) {
        case 1: return launch_stream<GROUPED, OUT_F32, Stream<1, 2, 4, 5>>(g, st);
        case 2: return launch_stream<GROUPED, OUT_F32, Stream<2, 1, 4, 5>>(g, st);
        case 3: return launch_stream<GROUPED, OUT_F32, Stream<2, 2, 4, 3>>(g, st);
        case 4: return launch_tile<GROUPED, OUT_F32, OUT_F32, false, Tile64>(g, 1, p.part_blocks, st);
        case 5: if constexpr (!OUT_F32) return launch_tile<GROUPED, false, false, false, Tile128>(g, 1, p.part_blocks, st); break;
        case 6: if constexpr (!OUT_F32) return launch_tile<GROUPED, false, false, false, Tile256>(g, 1, p.part_blocks, st); break;
        default: break;
    }
    return launch_stream<GROUPED, OUT_F32, Stream<1, 1, 4, 4>>(g, st);
}

}  // namespace

size_t fp8_gemm_partial_bytes(int64_t M, int64_t N, int64_t K, bool out_f32)
{
    const Fp8Args g{nullptr, nullptr, nullptr, nullptr, nullptr, M, N, K, M, nullptr, nullptr, 1};
    const Plan p = plan_fp8(g, false, out_f32, SIZE_MAX);
    return p.parts > 1 ? (size_t)p.parts * M * N * 4 : 0;
}

hipError_t launch_fp8_gemm(const void* a, const float* a_scales, const void* w, const float* w_scales, int64_t M, int64_t N, int64_t K, void* out, bool out_f32,
                           void* partial, size_t room, hipStream_t st)
{
    const Fp8Args g{static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(w), w_scales, out, M, N, K, M, nullptr, nullptr, 1};
    const Plan p = plan_fp8(g, false, out_f32, room);
    return out_f32 ? launch<false, true>(g, p, partial, st) : launch<false, false>(g, p, partial, st);
}

hipError_t launch_fp8_grouped_gemm(const void* a, const float* a_scales, int64_t a_rows, const void* w, const float* w_scales, const int32_t* offsets,
                                   const int32_t* index, int64_t rows, int64_t experts, int64_t N, int64_t K, void* out, bool out_f32, hipStream_t st)
{
    const Fp8Args g{static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(w), w_scales, out, a_rows, N, K, rows, offsets, index, (int)experts};
    const Plan p = plan_fp8(g, true, out_f32, 0);
    return out_f32 ? launch<true, true>(g, p, nullptr, st) : launch<true, false>(g, p, nullptr, st);
}

}  // namespace fp4mr
