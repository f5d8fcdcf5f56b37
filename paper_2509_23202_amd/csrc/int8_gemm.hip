// Products of 8-bit integer operands, for one weight matrix or for rows grouped by expert.
//
//   out[m,n] = (float(sum_k a[m,k] w[n,k]) * sa[m]) * sw[n]
//
// The sum is exact: v_mfma_i32_16x16x64_i8 adds in 32 bits, and 2^14 K is less than 2^31 for the K that the entry points take.  So no order of it, and no split of K, changes a
// bit of the result.  The W codes are the MFMA's A operand and the activations its B operand: a lane then has four consecutive n of one m.  Both operands are row-major, 128 bytes of a row to
// a step: lane l reads row l % 16, and from the row's eight pieces of 16 bytes the pieces l / 16 and l / 16 + 4, one for each of two MFMAs.  What lies past K is
// zero in W, and may be anything in A.
#include "product_tiles.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

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

typedef int v4i_any __attribute__((ext_vector_type(4), aligned(2)));

enum { kBf16, kF32, kSums };   // what leaves: the output in one of its types, or the sums of a part of K

__device__ __forceinline__ v4i mfma(const v4i& a, const v4i& b, const v4i& c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// Four consecutive values of a row, of which the row has `have`; rows of an odd number of columns begin at any element.
template <int OUT>
__device__ __forceinline__ void store4(void* out, int64_t at, const v4i& sum, float sa, const v4f& sw, int have)
{
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)sum[e] * sa * sw[e];
    if constexpr (OUT == kF32) {
        float* const to = static_cast<float*>(out) + at;
        if (have >= 4) __builtin_memcpy(to, y, 16);
        else for (int e = 0; e < have; ++e) to[e] = e == 0 ? y[0] : e == 1 ? y[1] : y[2];
    } else {
        const __bf16 b[4] = {(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
        __bf16* const to = static_cast<__bf16*>(out) + at;
        if (have >= 4) __builtin_memcpy(to, b, 8);
        else for (int e = 0; e < have; ++e) to[e] = e == 0 ? b[0] : e == 1 ? b[1] : b[2];
    }
}

// ---------------------------------------------------------------- few rows: weights streamed from memory
// 16 TN columns and 16 TM rows to a tile; a workgroup walks a run of tiles.  Its waves share K, each with a run of blocks; a block's codes go to the wave's own part of LDS by direct-to-LDS loads, D
// blocks ahead, the next tile's behind this one's, so that what is on its way never runs dry and no wave waits for another but to add up a tile.
// Bound by memory where columns are many (16 tokens, 4 of 64 experts 4096 x 4096: 28 to 34 experts' weights at 5.5 to 5.7 TB/s), else by its start-up and the last tile's sum: 1 x 4096 x 4096 6.4 us with the weights from
// memory (2.6 TB/s), 5.6 from the caches, 1 x 10240 x 8192 20.3 (4.1) and 14.8.  Loads go out for sixteen or 32 rows of X whatever there are of them: a third to a half of the load instructions.
// Four waves and three blocks each cost least at the start; two waves (16 x 32) let three workgroups share a compute unit.  Tiles of 48 and 64 rows, which read the weights once, gain where the caches have the weights
// (33 x 4096 x 14336 13.2 us against 15.8, 64 rows 17.5 against 14.7) and lose where they come from memory (48 x 16: 33 rows 18.5 against 17.1, 48 rows 21.2 against 19.1): more of what a compute unit takes in is X then.
template <int TM_, int TN_, int WAVES_, int D_>
struct Stream {
    static constexpr int TM = TM_, TN = TN_, WAVES = WAVES_, D = D_;
    static constexpr int SLOT = (TN + TM) * 2048, LOADS = 2 * (TN + TM);
    static constexpr int PART = WAVES * TM * TN * 1024;              // partial sums, of two tiles in turn
    static constexpr int SCALES = 2 * 256;                           // of a tile: of up to 64 rows, of up to 64 columns
    static constexpr int kScales = WAVES * D * SLOT + 2 * PART;      // of eight tiles: loads are D tiles ahead at most, and a wave one tile ahead of another
    static constexpr int lds() { return kScales + 8 * SCALES; }
    static_assert(TM <= 4 && TN <= 4 && D <= 5 && WAVES >= 2 && lds() <= 163840 && D * LOADS < 60, "");
};

template <bool GROUPED, int OUT, typename C>
__global__ __launch_bounds__(C::WAVES * 64) void int8_stream_kernel(Int8Args g, int tiles_m, int tiles_n)
{
    constexpr int TM = C::TM, TN = C::TN, WAVES = C::WAVES, D = C::D;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int K = (int)g.K, KB = (K + 127) >> 7;
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

    // ---- loads: block `kb` of tile `at`, and what goes with the tile.  Rows that it does not have, and what lies past K in W, are outside of the operands: zeros.
    const int ring = wave * D * C::SLOT;
    const int piece = (lane & 7) ^ x_key(lane / 8);               // (rows r and r + 8 of sixteen: the key of the second is the first's + 4)
    const uint32_t wo = (uint32_t)(lane / 8) * (uint32_t)K + piece * 16, wo8 = (uint32_t)(lane / 8 + 8) * (uint32_t)K + (piece ^ 4) * 16;
    __amdgpu_buffer_rsrc_t rw, rx;
    uint32_t xo[TM][2];
    Rows r{0, 0, 0};
    int n0 = 0, at_m = -1;
    auto locate = [&](int tile) {
        const int tm = tile / tiles_n;
        n0 = (tile - tm * tiles_n) * 16 * TN;
        const bool moved = tm != at_m;
        at_m = tm;
        if (moved) {
            if constexpr (GROUPED) r = find_tile(g, experts, tm, 16 * TM);
            else r = Rows{0, tm * 16 * TM, min((tm + 1) * 16 * TM, (int)g.rows)};
        }
        const int64_t x0 = gather ? 0 : r.begin, x_rows = gather ? g.a_rows : r.end - r.begin;
        auto x_offset = [&](int m, int pitch) -> uint32_t {      // of a row of A, from x0
            const int row = r.begin + m >= r.end ? -1 : gather ? g.index[r.begin + m] : m;
            return row >= 0 && row < x_rows ? (uint32_t)row * (uint32_t)pitch : kOutside;
        };
        if (moved) {
            rx = make_rsrc(g.a + x0 * K, x_rows * K);
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) xo[t][h] = x_offset(t * 16 + h * 8 + lane / 8, K) + (piece ^ (4 * h)) * 16;
        }
        const int w_rows = min((int)g.N - n0, 16 * TN);
        rw = make_rsrc(g.w + ((int64_t)r.expert * g.N + n0) * K, (int64_t)w_rows * K);
        const int to = C::kScales + (tile & 7) * C::SCALES;
        if (wave == 0) load_lds4(make_rsrc(g.a_scales + x0, x_rows * 4), smem, to, x_offset(min(lane, 16 * TM - 1), 4));
        if (wave == 1) load_lds4(make_rsrc(g.w_scales + (int64_t)r.expert * g.N + n0, w_rows * 4), smem, to + 256, (uint32_t)min(lane, 16 * TN - 1) * 4);
    };
    int load_tile = tile_first, load_kb = 0, load_slot = 0;
    auto issue = [&]() {
        const int k = (kb_first + load_kb) * 128, to = ring + load_slot * C::SLOT;
        const uint32_t past = k + piece * 16 < K ? 0 : kOutside, past8 = k + (piece ^ 4) * 16 < K ? 0 : kOutside;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            load_lds16(rw, smem, to + i * 2048, (wo + (uint32_t)(16 * i) * (uint32_t)K) | past, k);
            load_lds16(rw, smem, to + i * 2048 + 1024, (wo8 + (uint32_t)(16 * i) * (uint32_t)K) | past8, k);
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            load_lds16(rx, smem, to + (TN + t) * 2048, xo[t][0], k);
            load_lds16(rx, smem, to + (TN + t) * 2048 + 1024, xo[t][1], k);
        }
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
        v4i acc[TM][TN];
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
            for (int i = 0; i < TN; ++i) acc[t][i] = v4i{0, 0, 0, 0};
#pragma unroll 1
        for (int k = 0; k < each; ++k) {
            issue();
            wait_vmcnt<(D - 1) * C::LOADS>();
            asm volatile("" ::: "memory");
            const char* from = smem + ring + slot * C::SLOT;
            v4i wf[TN][2], af[TM][2];
            auto read = [&](const char* p, v4i (&f)[2]) {
                f[0] = *reinterpret_cast<const v4i*>(p + f_at);
                f[1] = *reinterpret_cast<const v4i*>(p + (f_at ^ 64));
            };
#pragma unroll
            for (int i = 0; i < TN; ++i) read(from + i * 2048, wf[i]);
#pragma unroll
            for (int t = 0; t < TM; ++t) read(from + (TN + t) * 2048, af[t]);
            wait_lgkmcnt0();      // (the slot is loaded again by the very next issue)
            asm volatile("" ::: "memory");
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < TM; ++t)
#pragma unroll
                    for (int i = 0; i < TN; ++i) acc[t][i] = mfma(wf[i][h], af[t][h], acc[t][i]);
            slot = slot == D - 1 ? 0 : slot + 1;
        }
        // ---- the waves' sums, and out
        v4i* const part = reinterpret_cast<v4i*>(smem + WAVES * D * C::SLOT + ((tile - tile_first) & 1) * C::PART);
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
        const char* const scales = smem + C::kScales + (tile & 7) * C::SCALES;
        for (int q = wave; q < TM * TN; q += WAVES) {
            v4i sum = part[q * 64 + lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) sum += part[(v * TM * TN + q) * 64 + lane];
            const int row = 16 * (q / TN) + l16, col = 16 * (q % TN) + (lane >> 4) * 4, m = mine.begin + row, n = col0 + col;
            if (m < mine.end)
                store4<OUT>(g.out, (int64_t)m * g.N + n, sum, reinterpret_cast<const float*>(scales)[row], *reinterpret_cast<const v4f*>(scales + 256 + col * 4), (int)g.N - n);
        }
    }
    wait_vmcnt<0>();    // (loads to LDS past the last block)
}

// ---------------------------------------------------------------- tiles
// BM x BN to NWM x NWN waves, each 16 TM x 16 TN; a workgroup walks tiles.  A stage is 128 columns of both operands' rows in LDS, eight rows to a 1 KB direct-to-LDS load; the sixteen-byte pieces of a row lie
// exchanged by a key, so that sixteen rows' reads of one piece touch every bank once.  A step multiplies a stage.  The loads of the stage S - 1 steps on go out in it; when a tile's have all gone out, they are the
// next tile's, whose first stages are there before this tile's output has left.
//   FEED waves beside those that multiply do nothing but load.  A wave that issues loads is held up by each (26 bytes a ns to a wave is what goes out, 105 to 145 to a compute unit from eight waves, 88 from four),
// and one that stores waits for its stores with its loads, which come back in order: so the waves that multiply neither wait for memory nor load, and a tile's output leaves under the next tile's products
// (128 x 128 with four more waves for the loads: 2048 x 4096 x 14336 130 -> 104 us, 201 x 10240 x 8192 30 -> 27).  A step begins with a meeting, which says that the next stage is there and that the stage before is
// free.  AHEAD: all fragments of the next step are read while this one's are multiplied, into a second copy of their registers; else the W fragments stay, and the X fragments pass through a few buffers.
//   Without them (256 x 256, which has no registers for more than eight waves) the waves that multiply load, and there are two stages: before its last X fragment a wave has read all it needs of the stage.  There it
// waits for its loads of the next one, the workgroup meets, and the last fragment's products cover the reads of the next step's first fragments.
// The two waves of a SIMD have different rows: one that has none in this tile leaves the other the SIMD (16384 rows dealt by a router to 64 experts 4096 x 4096, 97 tiles of which 35 are at most half full: 415 -> 399 us).
// What is left there is the weights: experts with 256 rows each take 290 us, of which reading 64 of them at 6.3 TB/s would be 170 and multiplying, as one expert's rows, 204; asking for each line a step earlier made
// it 302, rows of another pitch (K 3968 to 4352) changed nothing.
//   A tile takes S steps at least: the meeting in a step that is not one of its last S - 1 stands between a tile's output, which reads its scales, and the loads of the scales two tiles on.
template <int TM_, int TN_, int NWM_, int NWN_, int STAGES_, int FEED_, bool AHEAD_ = false>
struct Tile {
    static constexpr int TM = TM_, TN = TN_, NWM = NWM_, NWN = NWN_, S = STAGES_, NW = NWM * NWN, FEED = FEED_, LW = FEED ? FEED : NW;       // LW: waves that load
    static constexpr bool AHEAD = AHEAD_;
    static constexpr int BM = 16 * TM * NWM, BN = 16 * TN * NWN;
    static constexpr int STAGE = (BM + BN) * 128, SCALES = (BM + BN) * 4;
    static constexpr int XL = BM / 8 / LW, WL = BN / 8 / LW, LPS = XL + WL;   // loads of a wave for a step: X, W
    static constexpr int kScales = S * STAGE;                                 // of two tiles in turn
    static constexpr int kRoom = kScales + 2 * SCALES, ROOM = 512 * TN;       // for the output, of each wave
    static constexpr int lds() { return kRoom + NW * ROOM; }
    static_assert(BM % (8 * LW) == 0 && BN % (8 * LW) == 0 && BM % 64 == 0 && BN % 64 == 0 && (FEED ? S >= 3 : S == 2 && !AHEAD) && (S - 1) * LPS < 64 && lds() <= 163840, "");
};

// What the pieces of a row of W are exchanged by: a fragment has four rows in each of four runs of 4 TN.
template <int TN>
__device__ __forceinline__ int w_key_of(int row) { return (row >> 1 & 1) | (row / (4 * TN) & 3) << 1; }

// split_parts: a unit of work is one part of K of a tile, each of split_blocks times 128 columns but the last, and what leaves (OUT = kSums) is its sums, to the part's own copy of the output.
template <bool GROUPED, int OUT, typename C>
__global__ __launch_bounds__((C::NW + C::FEED) * 64) void int8_tile_kernel(Int8Args g, int tiles_m, int tiles_n, int split_parts, int split_blocks)
{
    constexpr bool SPLIT = OUT == kSums;
    static_assert(!SPLIT || !GROUPED, "");
    constexpr int TM = C::TM, TN = C::TN, NW = C::NW, S = C::S, LPS = C::LPS;
    constexpr bool FED = C::FEED > 0;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int K = (int)g.K, parts = SPLIT ? split_parts : 1;
    const bool gather = GROUPED && g.index != nullptr;
    if constexpr (GROUPED) tiles_m = count_tiles(g, expert_tiles(g, 0, C::BM), C::BM, tiles_m);
    const int ntiles = tiles_m * tiles_n * parts;
    int tile = blockIdx.x;
    if (tile >= ntiles) return;

    // ---- a tile: its rows, columns and steps, and for the waves that load where its operands are.  Rows that it does not have lie outside of the operand: their loads bring zeros.
    Rows r{0, 0, 0};
    int n0 = 0, part = 0, side = 0, k_first = 0, steps = 0;
    auto locate = [&]() {
        int tm, tn;
        if constexpr (!SPLIT) {
            place(tile, ntiles, tiles_m, tiles_n, tm, tn);
            steps = max((K + 127) / 128, S);
        } else {       // (neighbours of different parts, so that with eight parts an XCD has one part of K of both operands)
            const int at = tile / parts;
            part = tile - at * parts;
            tn = at / tiles_m;
            tm = at - tn * tiles_m;
            k_first = part * split_blocks * 128;
            steps = max((min(split_blocks * 128, K - k_first) + 127) / 128, S);     // (a part that is not the last has as many blocks, and what is past K is zeros)
        }
        if constexpr (GROUPED) r = find_tile(g, expert_tiles(g, 0, C::BM), tm, C::BM);
        else r = Rows{0, tm * C::BM, min((tm + 1) * C::BM, (int)g.rows)};
        n0 = tn * C::BN;
        side ^= 1;
    };
    __amdgpu_buffer_rsrc_t rx, rw;
    uint32_t xo[C::XL], wo[C::WL];
    int t = 0;                 // the step whose loads go out
    const int lw = FED ? wave - NW : wave;         // among the waves that load
    auto issue = [&](int stage, int i) {
        const int at = k_first + t * 128;
        if (i < C::XL) {
            load_lds16(rx, smem, stage + (i * C::LW + lw) * 1024, xo[i < C::XL ? i : 0], at);
        } else {
            const int q = i - C::XL, j = q >= 0 && q < C::WL ? q : 0;
            const int piece = (lane & 7) ^ w_key_of<TN>((j * C::LW + lw) * 8 + lane / 8);
            load_lds16(rw, smem, stage + C::BM * 128 + (j * C::LW + lw) * 1024, wo[j] | (at + piece * 16 < K ? 0u : kOutside), at);
        }
    };
    // In front of a tile's first codes: its scales too.
    auto begin_tile = [&]() {
        const int lane = kept_here((int)threadIdx.x & 63);
        locate();
        const int64_t x0 = gather ? 0 : r.begin, x_rows = gather ? g.a_rows : r.end - r.begin;
        const int w_rows = min((int)g.N - n0, C::BN);
        rx = make_rsrc(g.a + x0 * K, x_rows * K);
        rw = make_rsrc(g.w + ((int64_t)r.expert * g.N + n0) * K, (int64_t)w_rows * K);
        auto x_offset = [&](int m, int pitch) -> uint32_t {
            const int row = r.begin + m >= r.end ? -1 : gather ? g.index[r.begin + m] : m;
            return row >= 0 && row < x_rows ? (uint32_t)row * (uint32_t)pitch : kOutside;
        };
#pragma unroll
        for (int i = 0; i < C::XL; ++i) {
            const int m = (i * C::LW + lw) * 8 + lane / 8;
            xo[i] = x_offset(m, K) + (uint32_t)((lane & 7) ^ x_key(m)) * 16;
        }
#pragma unroll
        for (int i = 0; i < C::WL; ++i) {
            const int n = (i * C::LW + lw) * 8 + lane / 8;
            wo[i] = (n < w_rows ? (uint32_t)n * (uint32_t)K : kOutside) + (uint32_t)((lane & 7) ^ w_key_of<TN>(n)) * 16;
        }
        if constexpr (!SPLIT) {
            const __amdgpu_buffer_rsrc_t rs = make_rsrc(g.a_scales + x0, x_rows * 4), rsw = make_rsrc(g.w_scales + (int64_t)r.expert * g.N + n0, (int64_t)w_rows * 4);
#pragma unroll
            for (int i = 0; i < (C::BM + C::BN) / 64; i += C::LW) {
                const int q = i + lw;
                if (q < C::BM / 64) load_lds4(rs, smem, C::kScales + side * C::SCALES + q * 256, x_offset(q * 64 + lane, 4));
                else if (q < (C::BM + C::BN) / 64) load_lds4(rsw, smem, C::kScales + side * C::SCALES + q * 256, (uint32_t)((q - C::BM / 64) * 64 + lane) * 4);
            }
        }
        t = 0;
    };
    auto move_on = [&]() {     // the loads of this tile have gone out
        if (tile + (int)gridDim.x < ntiles) {
            tile += gridDim.x;
            begin_tile();
        }
    };
    auto first_stages = [&]() {
        begin_tile();
#pragma unroll
        for (int st = 0; st < S - 1; ++st) {
#pragma unroll
            for (int i = 0; i < LPS; ++i) issue(st * C::STAGE, i);
            ++t;
        }
        wait_vmcnt<(S - 2) * LPS>();
        block_barrier();
    };
    int stage = 0;             // of this step, as a place in LDS
    auto after = [](int at) { return at == (S - 1) * C::STAGE ? 0 : at + C::STAGE; };
    auto fill_of = [](int at) { return at == 0 ? (S - 1) * C::STAGE : at - C::STAGE; };     // the stage before this one, for S - 1 steps on

    if constexpr (FED) {
        if (wave >= NW) {
            first_stages();
            for (;;) {
                const int here_tile = tile, here_steps = steps;
                for (int half = 0, kt = 0; half < 2; ++half) {
                    const int to = half ? here_steps : here_steps - S + 1;
#pragma clang loop unroll(disable)
                    for (; kt < to; ++kt) {
                        wait_vmcnt<(S > 3 ? S - 3 : 0) * LPS>();
                        block_barrier();
                        const int fill = fill_of(stage);
#pragma unroll
                        for (int i = 0; i < LPS; ++i) issue(fill, i);
                        ++t;
                        stage = after(stage);
                    }
                    if (half == 0) move_on();
                }
                if (tile == here_tile) break;
            }
            wait_vmcnt<0>();    // (loads to LDS past the last step)
            return;
        }
        locate();
        block_barrier();
    } else {
        first_stages();
    }

    // ---- fragments: row l % 16 of X; for the i-th of W, of the wave's columns that which leaves a lane 4 TN consecutive ones of the output
    const int wm = wave / C::NWN, wn = wave % C::NWN;
    const int l16 = lane & 15, xr = wm * TM * 16 + l16, wr = wn * 16 * TN + l16 / 4 * 4 * TN + l16 % 4;
    const int xf_at = xr * 128 + ((lane >> 4) ^ x_key(xr)) * 16;
    const int wf_at = C::BM * 128 + wr * 128 + ((lane >> 4) ^ w_key_of<TN>(wr)) * 16;    // (rows 4 i on have the same key)
    auto read = [&](int at, int more, v4i (&f)[2]) {
        f[0] = *reinterpret_cast<const v4i*>(smem + at + more);
        f[1] = *reinterpret_cast<const v4i*>(smem + (at ^ 64) + more);
    };
    constexpr int RING = TM < 4 ? TM : 4, NEAR = RING / 2;                               // X fragments are read so many of them ahead
    v4i xf[C::AHEAD ? 2 * TM : RING][2], wf[C::AHEAD ? 2 * TN : TN][2];
#pragma unroll
    for (int i = 0; i < TN; ++i) read(wf_at, i * 512, wf[i]);
#pragma unroll
    for (int j = 0; j < (C::AHEAD ? TM : NEAR); ++j) read(xf_at, j * 2048, xf[j]);

    for (;;) {
        const Rows here = r;       // (the loads move on to the next tile before this one is done)
        const int here_n0 = n0, here_tile = tile, here_part = part, here_side = side, here_steps = steps;
        const bool without = !FED && here.begin + wm * TM * 16 >= here.end;
        v4i acc[TM][TN];
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int i = 0; i < TN; ++i) acc[j][i] = v4i{0, 0, 0, 0};
        auto step = [&]() {
            // (two stages) a step's loads go out among the products of the first three X fragments
            constexpr int SPOTS = 2 * TN * 3, EVERY = SPOTS / LPS;
            static_assert(FED || (TM > 3 && EVERY > 0), "");
            const int next = after(stage), fill = fill_of(stage);
            if constexpr (FED) block_barrier();
            auto fetch = [&](int q) { read(xf_at + (q < TM ? stage : next), q % TM * 2048, xf[q % RING]); };     // X fragment q from the front of this stage
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                if (FED || j + NEAR < TM) fetch(j + NEAR);
                if (j == TM - 1 && !FED) {
                    ++t;
                    wait_vmcnt<0>();
                    wait_lgkmcnt0();
                    block_barrier();
#pragma unroll
                    for (int q = 0; q < NEAR; ++q) fetch(TM + q);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        acc[j][i] = mfma(wf[i][h], xf[j % RING][h], acc[j][i]);
                        if (j == TM - 1 && h == 1) read(wf_at + next, i * 512, wf[i]);
                        const int spot = (j * 2 + h) * TN + i;
                        if (!FED && spot < SPOTS && spot % (EVERY ? EVERY : 1) == 0 && spot / (EVERY ? EVERY : 1) < LPS) issue(fill, spot / (EVERY ? EVERY : 1));
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
            stage = next;
        };
        // (two stages) of a wave that has no rows in this tile
        auto step_without = [&]() {
            const int next = after(stage), fill = fill_of(stage);
#pragma unroll
            for (int i = 0; i < LPS; ++i) issue(fill, i);
            ++t;
            wait_vmcnt<0>();
            block_barrier();
            stage = next;
        };
        // from the copy c of the fragments' registers, with the next step's read to the other
        auto step_ahead = [&](auto c) {
            constexpr int SPOTS = TM * 2 * TN, EVERY = SPOTS / (TM + TN);
            static_assert(!C::AHEAD || EVERY > 0, "");
            const int next = after(stage);
            block_barrier();
#pragma unroll
            for (int spot = 0; spot < SPOTS; ++spot) {
                const int q = spot / (EVERY ? EVERY : 1);
                if (spot % (EVERY ? EVERY : 1) == 0 && q < TN) read(wf_at + next, q * 512, wf[C::AHEAD ? (1 - c) * TN + q % TN : 0]);
                else if (spot % (EVERY ? EVERY : 1) == 0 && q < TM + TN) read(xf_at + next, (q - TN) * 2048, xf[C::AHEAD ? (1 - c) * TM + (q - TN) % TM : 0]);
                const int j = spot / (2 * TN), h = spot / TN % 2, i = spot % TN;
                acc[j][i] = mfma(wf[C::AHEAD ? c * TN + i : 0][h], xf[C::AHEAD ? c * TM + j : 0][h], acc[j][i]);
                __builtin_amdgcn_sched_barrier(0);
            }
            stage = next;
        };
        if constexpr (C::AHEAD) {
#pragma clang loop unroll(disable)
            for (int kt = 0; kt + 2 <= here_steps; kt += 2) {
                step_ahead(std::integral_constant<int, 0>{});
                step_ahead(std::integral_constant<int, 1>{});
            }
            if (here_steps & 1) {
                step_ahead(std::integral_constant<int, 0>{});
#pragma unroll
                for (int j = 0; j < TM; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) xf[j][h] = xf[TM + j][h];
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) wf[i][h] = wf[TN + i][h];
            }
        } else {
            int kt = 0;
#pragma clang loop unroll(disable)
            for (int half = 0; half < 2; ++half) {
                int to = FED || half ? here_steps : here_steps - S + 1;
                asm volatile("" : "+s"(to));
                if (without) {
#pragma clang loop unroll(disable)
                    for (; kt < to; ++kt) step_without();
                } else {
#pragma clang loop unroll(disable)
                    for (; kt < to; ++kt) step();
                }
                if (!FED && half == 0) move_on();
            }
            if (without) {
#pragma unroll
                for (int i = 0; i < TN; ++i) read(wf_at + stage, i * 512, wf[i]);
#pragma unroll
                for (int q = 0; q < NEAR; ++q) read(xf_at + stage, q * 2048, xf[q]);
                if (tile == here_tile) break;
                continue;
            }
        }
        // ---- output: some rows of sixteen at a time through LDS of the wave's own, so that a row leaves as whole lines
        typedef std::conditional_t<OUT == kBf16, __bf16, std::conditional_t<OUT == kF32, float, int>> Out;
        constexpr int EACH = 16 / sizeof(Out), PIECES = 16 * TN / EACH, HALVES = sizeof(Out) / 2, ROWS = 64 / PIECES;      // elements of a piece; pieces of a row; times that sixteen rows take; rows to a store
        constexpr int RUN = 4 * TN / EACH;         // pieces that a lane has of a row
        static_assert(ROWS > 0 && 16 / HALVES % ROWS == 0, "");
        const int lane = kept_here((int)threadIdx.x & 63), l16 = lane & 15;
        const float* const scales = reinterpret_cast<const float*>(smem + C::kScales + here_side * C::SCALES);
        auto key = [](int row) { return PIECES == 4 ? row >> 2 & 3 : PIECES == 8 ? row >> 1 & 7 : row & 15; };      // of a row's pieces
        char* const room = smem + C::kRoom + wave * C::ROOM;
        const int row0 = here.begin + wm * TM * 16 + lane / PIECES, col = here_n0 + wn * 16 * TN + lane % PIECES * EACH, have = (int)g.N - col;
        const bool inside = here.begin + (wm + 1) * TM * 16 <= here.end && here_n0 + (wn + 1) * 16 * TN <= (int)g.N;
        Out* out = static_cast<Out*>(g.out) + ((int64_t)here_part * g.rows + row0) * g.N + col;
        v4f sw[TN];
#pragma unroll
        for (int i = 0; i < TN; ++i) sw[i] = *reinterpret_cast<const v4f*>(scales + C::BM + wn * 16 * TN + (lane >> 4) * 4 * TN + 4 * i);
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const float sa = scales[wm * TM * 16 + 16 * j + l16];
#pragma unroll
            for (int half = 0; half < HALVES; ++half) {
                if (l16 * HALVES / 16 == half) {
                    char* const to = room + l16 % (16 / HALVES) * (PIECES * 16);
#pragma unroll
                    for (int p = 0; p < RUN; ++p) {
                        v4i y;
                        if constexpr (OUT == kSums) {
                            y = acc[j][p];
                        } else if constexpr (OUT == kF32) {
                            v4f f;
#pragma unroll
                            for (int e = 0; e < 4; ++e) f[e] = (float)acc[j][p][e] * sa * sw[p][e];
                            y = __builtin_bit_cast(v4i, f);
                        } else {
                            v8bf f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = (__bf16)((float)acc[j][2 * p + e / 4][e % 4] * sa * sw[2 * p + e / 4][e % 4]);
                            y = __builtin_bit_cast(v4i, f);
                        }
                        *reinterpret_cast<v4i*>(to + (((lane >> 4) * RUN + p) ^ key(l16)) * 16) = y;
                    }
                }
                asm volatile("" ::: "memory");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int h = 0; h < 16 / HALVES / ROWS; ++h) {
                    const int row = h * ROWS + lane / PIECES, at = 16 * j + 16 / HALVES * half + h * ROWS;
                    const char* const from = room + row * (PIECES * 16) + (lane % PIECES ^ key(row + 16 / HALVES * half)) * 16;
                    const v4i y = *reinterpret_cast<const v4i*>(from);
                    // (rows of an odd number of columns begin at any element)
                    if (inside || (row0 + at < here.end && have >= EACH)) {
                        __builtin_nontemporal_store(y, reinterpret_cast<v4i_any*>(out));
                    } else if (row0 + at < here.end) {
                        const Out* const piece = reinterpret_cast<const Out*>(from);
#pragma clang loop unroll(disable) vectorize(disable)
                        for (int e = 0; e < have; ++e) out[e] = piece[e];
                    }
                    out += ROWS * g.N;
                }
                asm volatile("" ::: "memory");
                __builtin_amdgcn_wave_barrier();
            }
        }
        if constexpr (FED) {
            tile += gridDim.x;
            if (tile >= ntiles) break;
            locate();
        } else if (tile == here_tile) {
            break;
        }
    }
    if constexpr (!FED) wait_vmcnt<0>();    // (loads to LDS past the last step)
}

template <bool GROUPED, int OUT, typename C>
hipError_t launch_tile(const Int8Args& g, int parts, int part_blocks, hipStream_t st)
{
    static LdsAttrOnce attr;
    const hipError_t e = attr.ensure(reinterpret_cast<const void*>(int8_tile_kernel<GROUPED, OUT, C>), C::lds());
    if (e != hipSuccess) return e;
    const int64_t tiles_m = GROUPED ? g.rows / C::BM + std::min<int64_t>(g.experts, g.rows) : (g.rows + C::BM - 1) / C::BM, tiles_n = (g.N + C::BN - 1) / C::BN;
    const int64_t grid = std::min<int64_t>(tiles_m * tiles_n * parts, (int64_t)compute_units() * (163840 / C::lds()));
    hipLaunchKernelGGL((int8_tile_kernel<GROUPED, OUT, C>), dim3((unsigned)grid), dim3((C::NW + C::FEED) * 64), C::lds(), st, g, (int)tiles_m, (int)tiles_n, parts, part_blocks);
    return hipGetLastError();
}

// The parts' sums added, and the output.  Four elements of a row to a thread.  A launch and what it reads: 33 x 4096 in eight parts 4 us.
template <int OUT>
__global__ __launch_bounds__(256) void int8_join_kernel(Int8Args g, const int* part, int parts)
{
    const int64_t per_row = (g.N + 3) / 4, total = g.rows * per_row, n = g.rows * g.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per_row;
        const int col = (int)(i - m * per_row) * 4, have = (int)g.N - col;
        const int* const from = part + m * g.N + col;
        v4i sum{0, 0, 0, 0};
        v4f sw{0.f, 0.f, 0.f, 0.f};
        if (have >= 4) {
            for (int p = 0; p < parts; ++p) {
                v4i q;
                __builtin_memcpy(&q, from + p * n, 16);
                sum += q;
            }
            __builtin_memcpy(&sw, g.w_scales + col, 16);
        } else {
            for (int e = 0; e < have; ++e) {
                int s = 0;
                for (int p = 0; p < parts; ++p) s += from[p * n + e];
                sum[e] = s;
                sw[e] = g.w_scales[col + e];
            }
        }
        store4<OUT>(g.out, m * g.N + col, sum, g.a_scales[m], sw, have);
    }
}

// A product in parts of K on tiles of C, and their sum.
template <int OUT, typename C>
hipError_t launch_parts(Int8Args g, int parts, int part_blocks, void* partial, hipStream_t st)
{
    Int8Args sums = g;
    sums.out = partial;
    const hipError_t e = launch_tile<false, kSums, C>(sums, parts, part_blocks, st);
    if (e != hipSuccess) return e;
    const int64_t total = g.rows * ((g.N + 3) / 4);
    hipLaunchKernelGGL(int8_join_kernel<OUT>, dim3((unsigned)std::min<int64_t>((total + 255) / 256, 1 << 20)), dim3(256), 0, st, g, static_cast<const int*>(partial), parts);
    return hipGetLastError();
}

template <bool GROUPED, int OUT, typename C>
hipError_t launch_stream(const Int8Args& g, hipStream_t st)
{
    static LdsAttrOnce attr;
    const hipError_t e = attr.ensure(reinterpret_cast<const void*>(int8_stream_kernel<GROUPED, OUT, C>), C::lds());
    if (e != hipSuccess) return e;
    const int64_t tiles_m = GROUPED ? g.rows / (16 * C::TM) + std::min<int64_t>(g.experts, g.rows) : (g.rows + 16 * C::TM - 1) / (16 * C::TM), tiles_n = (g.N + 16 * C::TN - 1) / (16 * C::TN);
    const int64_t per_cu = 163840 / C::lds(), grid = std::min<int64_t>(tiles_m * tiles_n, compute_units() * per_cu);
    hipLaunchKernelGGL((int8_stream_kernel<GROUPED, OUT, C>), dim3((unsigned)grid), dim3(C::WAVES * 64), C::lds(), st, g, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

typedef Tile<2, 2, 2, 2, 6, 4, true> Tile64;      // 64 x 64
typedef Tile<4, 2, 2, 2, 6, 4> Tile128n;          // 128 x 64
typedef Tile<4, 4, 2, 2, 4, 4> Tile128;           // 128 x 128
typedef Tile<8, 4, 1, 4, 3, 4> Tile128w;          // 128 x 256
typedef Tile<8, 4, 2, 4, 2, 0> Tile256;           // 256 x 256

// How a product runs.
struct Plan {
    int kind = 0;              // 0 .. 3: few rows; 4 .. 8: tiles
    int parts = 1, part_blocks = 0;
};

constexpr int kKinds = 9, kFew = 4, kMostParts = 8;
// a part of K has as many blocks as any of those kinds has stages
constexpr int kStages[kKinds] = {0, 0, 0, 0, Tile64::S, Tile128n::S, Tile128::S, Tile128w::S, Tile256::S}, kMostStages = 6;
static_assert(Tile64::S <= kMostStages && Tile128n::S <= kMostStages && Tile128::S <= kMostStages, "");
constexpr int kRows[kKinds] = {16, 16, 32, 32, 64, 128, 128, 128, 256}, kCols[kKinds] = {16, 32, 16, 32, 64, 64, 128, 256, 256};

// What a kind takes, microseconds on a device of `cus` compute units, as fitted to measurements on 256: a start, rounds of tiles, each a fixed part and the steps of K (a quarter of its blocks where four waves share
// them), but no less than what it reads takes from memory at `rate` TB/s: where rows are few the weights, once for the first row of tiles and `again` times for each other one (the caches have part of them), else both
// operands once, of the `sets` of weights that have rows.  Parts add the writing, reading and launch of their sum.  A product by expert runs longer and is nearer to what memory gives: it has numbers of its own.
// Measured, each kind and number of parts forced in turn, on 336 products of 1 to 4096 rows with layers from 300 x 9600 to 28672 x 4096 and on 150 drawn ones, weights from memory (450 MB of them in turn): the kind that is
// chosen takes 1.017 of the best one's time in the mean, 1.017 on 100 others too, at worst 1.26 (16 x 5001 x 2896: 8.1 us on tiles of 16 x 32, 6.4 on 16 x 16); by expert 1.04 on 66 products, and 1.05 on 51
// others, at worst 1.32: 64 experts 4096 x 4096 with 16 to 64 rows each (1024 rows 224 us on tiles of 128 x 64, 188 on 128 x 256; 4096 rows 296 and 223; dealt so unevenly that 29 and 38 experts have rows 124 and 96, 239 and
// 168).  The others take up to ten times the best one's
// (1 x 4096 x 4096: 16 x 16 5.9 us, 64 x 64 9.9, 128 x 128 19; 16 x 10240 x 8192: 64 x 64 20.3, 16 x 16 25.6; 128 x 4096 x 14336: 128 x 64 in four parts 23, in one 50; 201 x 10240 x 8192: 128 x 128 27 us, 128 x 64 37,
// 64 x 64 41, 128 x 256 50; 4096 x 4096 x 4096: 256 x 256 53 us, 128 x 256 63, 128 x 128 65, 64 x 64 100).
double kind_us(int kind, bool grouped, double rows, double tiles_m, double sets, double N, double K, int64_t blocks, int parts, int cus)
{
    static const double start[2][kKinds] = {{2.68, 2.58, 2.52, 2.66, 2.45, 3.04, 3.21, 3.88, 1.00}, {3.00, 3.16, 2.85, 3.03, 2.71, 2.56, 2.56, 2.54, 1.50}},
                        fixed[2][kKinds] = {{0.61, 0.42, 0.56, 0.75, 0.92, 1.11, 1.54, 2.05, 6.20}, {0.65, 0.42, 0.56, 0.78, 1.18, 1.74, 2.23, 3.00, 5.90}},
                        step[2][kKinds] = {{0.243, 0.485, 0.388, 0.557, 0.251, 0.344, 0.520, 1.007, 1.417}, {0.129, 0.350, 0.284, 0.328, 0.183, 0.263, 0.406, 0.854, 1.254}},
                        rate[2][kKinds] = {{3.91, 3.69, 3.98, 4.08, 4.59, 4.23, 4.34, 5.14, 3.40}, {5.9, 7.35, 6.6, 5.8, 5.9, 6.1, 5.8, 4.1, 3.9}}, again[kFew] = {0.57, 0.21, 0.45, 0.13};
    static const int per_cu[kKinds] = {2, 3, 1, 1, 1, 1, 1, 1, 1};
    const bool few = kind < kFew;
    const double steps = (double)(few ? (blocks + 3) / 4 : std::max<int64_t>((blocks + parts - 1) / parts, kStages[kind]));
    const double rounds = std::ceil(tiles_m * std::ceil(N / kCols[kind]) * parts / (per_cu[kind] * cus));
    const double bytes = few ? (sets + (grouped ? 1.0 : again[kind]) * (tiles_m - sets)) * N * K : sets * N * K + rows * K;
    const double us = start[grouped][kind] + std::max(rounds * (fixed[grouped][kind] + steps * step[grouped][kind]), bytes / (rate[grouped][kind] * 1e6 * cus / 256));
    return parts > 1 ? us + 4.6 + parts * rows * N * 8 / 7.4e6 : us;
}

// The kind that takes least; in parts only where `room` bytes hold their sums and fewer would leave compute units idle.
Plan plan_int8(const Int8Args& g, bool grouped, size_t room)
{
    const int forced = options().int8_variant, cus = compute_units();
    const int64_t blocks = (g.K + 127) / 128;
    Plan best;
    double best_us = 1e30;
    for (int kind = 0; kind < kKinds; ++kind) {
        if (forced && kind != (forced - 1) % kKinds) continue;
        // rows of tiles; by expert: as if the rows were spread evenly over the experts, half a tile more to each than they fill
        const double active = (double)std::min<int64_t>(g.experts, g.rows);
        const double tiles_m = grouped ? active * std::max(1.0, (double)g.rows / active / kRows[kind] + 0.4) : (double)((g.rows + kRows[kind] - 1) / kRows[kind]);
        const double tiles = tiles_m * std::ceil((double)g.N / kCols[kind]);
        for (int parts = 1; parts <= kMostParts; ++parts) {
            const int64_t each = std::max<int64_t>((blocks + parts - 1) / parts, kMostStages);
            if (parts > 1 && (grouped || kind < kFew || kind > kFew + 2 || (size_t)parts * g.rows * g.N * 4 > room || (parts - 1) * each >= blocks)) break;
            if (parts > 1 && !forced && (parts - 1) * tiles >= cus) break;
            if (forced && parts > 1 << (forced - 1) / kKinds) break;
            const double us = forced ? (double)-parts : kind_us(kind, grouped, (double)g.rows, tiles_m, grouped ? active : 1.0, (double)g.N, (double)g.K, blocks, parts, cus);
            if (us < best_us) {
                best = Plan{kind, parts, (int)each};
                best_us = us;
            }
        }
    }
    return best;
}

template <bool GROUPED, int OUT>
hipError_t launch(const Int8Args& g, const Plan& p, void* partial, hipStream_t st)
{
    if constexpr (!GROUPED) {
        if (p.parts > 1) {
            if (p.kind == 4) return launch_parts<OUT, Tile64>(g, p.parts, p.part_blocks, partial, st);
            if (p.kind == 5) return launch_parts<OUT, Tile128n>(g, p.parts, p.part_blocks, partial, st);
            return launch_parts<OUT, Tile128>(g, p.parts, p.part_blocks, partial, st);
        }
    }
    switch (p.kind) {
        case 1: return launch_stream<GROUPED, OUT, Stream<1, 2, 2, 3>>(g, st);
        case 2: return launch_stream<GROUPED, OUT, Stream<2, 1, 4, 3>>(g, st);
        case 3: return launch_stream<GROUPED, OUT, Stream<2, 2, 4, 3>>(g, st);
        case 4: return launch_tile<GROUPED, OUT, Tile64>(g, 1, 0, st);
        case 5: return launch_tile<GROUPED, OUT, Tile128n>(g, 1, 0, st);
        case 6: return launch_tile<GROUPED, OUT, Tile128>(g, 1, 0, st);
        case 7: return launch_tile<GROUPED, OUT, Tile128w>(g, 1, 0, st);
        case 8: return launch_tile<GROUPED, OUT, Tile256>(g, 1, 0, st);
        default: break;
    }
    return launch_stream<GROUPED, OUT, Stream<1, 1, 4, 3>>(g, st);
}

}  // namespace

size_t int8_gemm_partial_bytes(int64_t M, int64_t N, int64_t K)
{
    const Int8Args g{nullptr, nullptr, nullptr, nullptr, nullptr, M, N, K, M, nullptr, nullptr, 1};
    const Plan p = plan_int8(g, false, SIZE_MAX);
    return p.parts > 1 ? (size_t)p.parts * M * N * 4 : 0;
}

hipError_t launch_int8_gemm(const void* a, const float* a_scales, const void* w, const float* w_scales, int64_t M, int64_t N, int64_t K, void* out, bool out_f32,
                            void* partial, size_t room, hipStream_t st)
{
    const Int8Args g{static_cast<const int8_t*>(a), a_scales, static_cast<const int8_t*>(w), w_scales, out, M, N, K, M, nullptr, nullptr, 1};
    const Plan p = plan_int8(g, false, room);
    return out_f32 ? launch<false, kF32>(g, p, partial, st) : launch<false, kBf16>(g, p, partial, st);
}

hipError_t launch_int8_grouped_gemm(const void* a, const float* a_scales, int64_t a_rows, const void* w, const float* w_scales, const int32_t* offsets,
                                    const int32_t* index, int64_t rows, int64_t experts, int64_t N, int64_t K, void* out, bool out_f32, hipStream_t st)
{
    const Int8Args g{static_cast<const int8_t*>(a), a_scales, static_cast<const int8_t*>(w), w_scales, out, a_rows, N, K, rows, offsets, index, (int)experts};
    const Plan p = plan_int8(g, true, 0);
    return out_f32 ? launch<true, kF32>(g, p, nullptr, st) : launch<true, kBf16>(g, p, nullptr, st);
}

}  // namespace fp4mr
