// Products of the microscaled 4-bit form (include/lutq.h): Y = X W^T and the same by expert, on the scaled matrix instruction
// v_mfma_scale_f32_16x16x128_f8f6f4, which takes 128 columns of sixteen rows of either factor and their exponents as they are held.
//
// The instruction's first operand is the weights, so a lane's four sums are neighbours in a row of Y.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lutq.h"
#include "lutq_calib.h"
#include "lutq_layout.hpp"
#include "lutq_mx4_device.hpp"
#include "lutq_product.hpp"

namespace lutq {
namespace mx4 {

using namespace product;

lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, int64_t M, int64_t K,
                             void* codes, void* exponents, hipStream_t stream);

struct ProductParams {
    const char* x;             // row form: codes; or 16-bit values
    const char* xe;            // row form: exponents
    const char* w;             // records
    char* y;
    const int32_t* offsets;    // by expert: experts + 1; else null
    uint32_t* counters;        // K in slices: how many of a tile's are done, and
    char* partial;             // their sums
    int64_t record, expert;    // bytes of a row block's record, of an expert's weights
    int M, N, K, KT, KQ, NB;   // K tiles, quads, row blocks
    int experts;
    int slot0, slots;          // first piece of rows of this launch, and how many
    int slices;                // of K
    int bf16;                  // type of Y
    int once;                  // weights that are read once and do not stay in the caches: past them
};

// Few rows: a workgroup owns R row blocks of weights and sixteen rows of X over all of K; its wavefronts take the quads in turn, and
// their sums are added in LDS in the order of the wavefronts.  Bound by the reads of the weights, which go from memory into the operand
// registers as they lie, all of a quad asked for before X is looked at: 28672 x 4096, 62 MB, 1 row 13.0 us (4.8 TB/s), and 13 rows 14.3; smaller
// ones by the time that one load after another takes to arrive (2048 x 256, 1 row: 2.4 us).  X is asked for before the weights (4096 x 14336,
// 4 rows of bf16: 10.7 us after them, 10.0 so).
// X is read as its cache lines lie and passes through a place of the wavefront's own in LDS into the order of the operands.  (A lane per row
// would make 64 requests of every load: 4096 x 14336, 13 rows of codes 14.5 us, so 9.5; of bf16, 6144 x 4096, 8 rows, 7.5 and 6.9.)
// 16-bit values (SRC 1, 2) are quantised on the way.  ROWS 1 or 4: that many rows at a time, by the four lanes that hold a block, and the
// codes lie in LDS; 16: the values lie there, and each lane reads its block, which is half the instructions for sixteen rows, and more for
// four (4096 x 14336, 4 rows: 10.4 us and 11.1).  ROWS says what is likely; any number of rows is right.
// R = 4 is for K of one quad: a wavefront has sixteen rows of its own there, and the weights are shared in the first cache.
constexpr int kPlane = 256 + 16;                       // codes of one block of sixteen rows; the rest keeps the planes in different banks
constexpr int kStreamPlace = 16 * kPlane + 256;        // a quad's blocks, and their exponents

template <int SRC, int R, int ROWS, bool GROUPED>
__global__ __launch_bounds__(R == 1 ? 1024 : 512) void stream_kernel(const ProductParams p) {
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, i = lane & 15, o = lane >> 4;
    constexpr bool solo = R == 4;                      // every wavefront has sixteen rows of its own, and K is a quad
    const int slot = p.slot0 + (solo ? (int)blockIdx.y * waves + wave : (int)blockIdx.y);
    if (solo && !GROUPED && slot * 16 >= p.M) return;
    int expert = 0, m0 = slot * 16, m1 = min(p.M, m0 + 16);
    if constexpr (GROUPED) {
        Pieces<16> pieces{p.offsets, p.experts, p.M};
        if (slot >= pieces.count()) return;
        const auto in = pieces.find(slot);
        expert = in.expert;
        m0 = in.first + (slot - in.begin) * 16;
        m1 = min(in.end, m0 + 16);
    }
    const int rb0 = (int)blockIdx.x * R, rows = m1 - m0;
    const char* w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = p.w + expert * p.expert + min(rb0 + r, p.NB - 1) * p.record;
    char *const place = smem + wave * kStreamPlace, *const exps = place + 16 * kPlane;

    f32x4 acc[R] = {};
    for (int q = solo ? 0 : wave; q < p.KQ; q += waves) {
        const int tiles = min(4, p.KT - 4 * q);
        // X first: loads are waited for in order, and it has further to go.  Rows that do not exist stay unread, or are the last row, and what lies
        // in their places is multiplied: their sums are not stored.
        constexpr bool values = SRC != kF32 && ROWS == 16;
        u32x4 v[values ? 4 : 1][4];
        Eight<SRC == kF32 ? kF16 : SRC> few[ROWS];
        uint32_t e = 0;
        const bool word = (lane >> 2) < rows && (lane & 3) < tiles, there = o < tiles;
        auto ask_few = [&](int first) {                // lane 16 tile + 4 block + piece
            const char* from = p.x + ((int64_t)(m0 + first) * p.K + q * 512 + lane * 8) * 2;
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (first + k < rows && there) few[k].v[0] = *reinterpret_cast<const u32x4*>(from + (int64_t)k * p.K * 2);
        };
        if constexpr (SRC == kF32) {                   // (sixteen lanes take a row's sixteen blocks, four lanes its four words of exponents)
            const char* from = p.x + (int64_t)(m0 + (lane >> 4)) * (p.K / 2) + q * 256 + (lane & 15) * 16;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (4 * g + (lane >> 4) < rows && (lane & 15) < 4 * tiles) v[0][g] = *reinterpret_cast<const u32x4*>(from + (int64_t)g * 2 * p.K);
            if (word) e = *reinterpret_cast<const uint32_t*>(p.xe + (int64_t)(m0 + (lane >> 2)) * (p.K / 32) + q * 16 + (lane & 3) * 4);
        } else if constexpr (values) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (4 * g < rows)
                        v[t][g] = *reinterpret_cast<const u32x4*>(p.x + ((int64_t)min(m0 + 4 * g + o, m1 - 1) * p.K + q * 512 + min(t, tiles - 1) * 128 + i * 8) * 2);
        } else {
            ask_few(0);
        }
        uint32_t we[R];
        u32x4 wv[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r) we[r] = *reinterpret_cast<const uint32_t*>(w[r] + (int64_t)p.KT * 1024 + q * 256 + lane * 4);
        if (p.once) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < 4; ++t) wv[r][t] = __builtin_amdgcn_raw_buffer_load_b128(unbounded(w[r]), lane * 16, (4 * q + min(t, tiles - 1)) * 1024, kNonTemporal);
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < 4; ++t) wv[r][t] = __builtin_amdgcn_raw_buffer_load_b128(unbounded(w[r]), lane * 16, (4 * q + min(t, tiles - 1)) * 1024, 0);
        }
        auto multiply = [&](int t, u32x4 xv, uint32_t xe) {                    // `t` is a constant where this is called
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (t == 0) acc[r] = product<0, 0>(wv[r][0], xv, acc[r], we[r], xe);
                if (t == 1) acc[r] = product<1, 1>(wv[r][1], xv, acc[r], we[r], xe);
                if (t == 2) acc[r] = product<2, 2>(wv[r][2], xv, acc[r], we[r], xe);
                if (t == 3) acc[r] = product<3, 3>(wv[r][3], xv, acc[r], we[r], xe);
            }
        };
        if constexpr (values) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t >= tiles) break;
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (4 * g < rows) *reinterpret_cast<u32x4*>(place + (4 * g + o) * kPlane + i * 16) = v[t][g];
                between_lanes();
                Eight<SRC> block[4];
                uint32_t a = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) block[j].v[0] = *reinterpret_cast<const u32x4*>(place + i * kPlane + o * 64 + j * 16);
#pragma unroll
                for (int j = 0; j < 16; ++j) max_bits<SRC>(block[j / 4].v[0][j % 4], a);
                const uint32_t exponent = exponent_byte<SRC>(a);               // (255 makes the products NaN whatever the codes)
                u32x4 xv;
#pragma unroll
                for (int j = 0; j < 4; ++j) xv[j] = to_codes<SRC>(block[j], power_of(exponent));
                multiply(t, xv, exponent << (8 * t));
                between_lanes();
            }
            continue;
        }
        if constexpr (SRC == kF32) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (4 * g + (lane >> 4) < rows && (lane & 15) < 4 * tiles)
                    *reinterpret_cast<u32x4*>(place + (lane & 15) * kPlane + (4 * g + (lane >> 4)) * 16) = v[0][g];
            if (word)
#pragma unroll
                for (int k = 0; k < 4; ++k) exps[k * 64 + lane] = (char)(e >> (8 * k));
        } else {
            for (int first = 0; first < rows; first += ROWS) {
                if (first > 0) ask_few(first);
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    if (first + k >= rows || !there) continue;
                    uint32_t exponent;
                    const uint32_t c = quantize_eight<SRC>(few[k], exponent);
                    *reinterpret_cast<uint32_t*>(place + (lane >> 2) * kPlane + (first + k) * 16 + (lane & 3) * 4) = c;
                    if ((lane & 3) == 0) exps[((lane >> 2) & 3) * 64 + (first + k) * 4 + o] = (char)exponent;
                }
            }
        }
        between_lanes();
        const uint32_t xe = *reinterpret_cast<const uint32_t*>(exps + lane * 4);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t >= tiles) break;
            multiply(t, *reinterpret_cast<const u32x4*>(place + (4 * t + o) * kPlane + i * 16), xe);
        }
        between_lanes();
    }

    if constexpr (solo) {
        store_rows<R>([&](int r) { return acc[r]; }, p.y + ((int64_t)m0 * p.N + 16 * rb0) * 2, rows, p.NB - rb0, p.N, p.bf16);
        return;
    }
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(smem);      // [wave][row block][lane]
#pragma unroll
    for (int r = 0; r < R; ++r) sums[(wave * R + r) * 64 + lane] = acc[r];
    __syncthreads();
    for (int r = wave; r < R; r += waves) {
        f32x4 sum = sums[r * 64 + lane];
        for (int v = 1; v < waves; ++v) sum += sums[(v * R + r) * 64 + lane];
        if (i < rows && rb0 + r < p.NB) {
            const u32x2 out = {round_pair(sum[0], sum[1], p.bf16), round_pair(sum[2], sum[3], p.bf16)};
            *reinterpret_cast<u32x2*>(p.y + ((int64_t)(m0 + i) * p.N + 16 * (rb0 + r) + 4 * o) * 2) = out;
        }
    }
}

// Many rows: a workgroup of GN x GM wavefronts makes tiles of Y, 16 WN GN rows of weights times 16 WM GM rows of X, each wavefront WN x WM
// blocks of sixteen by sixteen.  K goes by in steps of two tiles (256 columns), which are copied from memory into LDS without passing
// through registers; there is room for DEPTH steps, so DEPTH - 1 are under way while one is multiplied.  The operands of one tile are read
// from LDS while the matrix instructions of the tile before run.  The exponents come the same way, a quad (two steps) at a time.  K >= 512.
//
// There are at most as many workgroups as run at once, and each takes one tile of Y after the other.  The copies run ahead across the
// tiles' borders: while one is finished and stored, the first steps of the next are under way.
//
// In LDS the weights lie as in memory, in operand order.  Of X a piece is sixteen rows of 128 bytes, whole cache lines as they are
// read (a line asked for in halves, a step apart, was fetched twice); block b of row i lies at 16 (b ^ (i >> 1)), so that the
// sixteen lanes that are served together hit all banks.
//
// Where Y has too few tiles for the device, K is cut into slices of whole quads as well.  Each slice leaves its sums in the
// workspace, and the last workgroup of a tile to finish adds them in the order of the slices.  No workgroup waits for another: the sums are
// stored past the caches that the dies do not share (sc1), complete before the workgroup counts itself, and read the same way.
template <int WN, int WM, int GN, int GM, int DEPTH> struct TileShape {
    static constexpr int kWaves = GN * GM, kThreads = 64 * kWaves;
    static constexpr int kRB = WN * GN, kMB = WM * GM;                         // pieces of sixteen rows of either factor
    static constexpr int kStep = (kRB + kMB) * 2048, kExps = (kRB + kMB) * 256;
    static constexpr int kExpPlaces = DEPTH;           // (a quad may be a single step: the last of a tile of Y)
    static constexpr int kLds = DEPTH * kStep + kExpPlaces * kExps + 16;
    static constexpr bool kSlices = WN * WM <= 8;      // (the join of slices holds four times a tile's sums)
    static constexpr int kSums = kWaves * WN * WM * 1024;                      // bytes of a tile's sums
};

template <int WN, int WM, int GN, int GM, int DEPTH, bool GROUPED, bool ONCE>
__global__ __launch_bounds__(GN * GM * 64, 2) void tile_kernel(const ProductParams p) {
    using std::integral_constant;
    using Shape = TileShape<WN, WM, GN, GM, DEPTH>;
    constexpr int kWaves = Shape::kWaves, kRB = Shape::kRB, kMB = Shape::kMB, kStep = Shape::kStep, kExps = Shape::kExps;
    constexpr int kWLoads = kRB / kWaves, kXLoads = 2 * kMB / kWaves;          // per wavefront: pieces of weights, halves of pieces of X
    constexpr int kLoads = 2 * kWLoads + kXLoads, kStores = WN / 2 * WM;
    // Of a step's copies, those that are asked for in the second half of a step; the others follow in the first half of the next, where
    // the steps are long or many enough for them to arrive in time.
    constexpr int kEarly = DEPTH > 2 || kWaves > 4 ? (2 * kLoads + 2) / 3 : kLoads;
    constexpr int kExpPieces = (kRB + kMB) / 4, kExpLoads = (kExpPieces + kWaves - 1) / kWaves;
    static_assert(kRB % kWaves == 0 && 2 * kMB % kWaves == 0 && kRB % 4 == 0 && kMB % 4 == 0, "whole loads per wavefront");
    static_assert(DEPTH == 2 || DEPTH == 4, "of any DEPTH - 2 steps half at least begin a quad");
    extern __shared__ __align__(1024) char lds[];      // DEPTH steps, then the exponents of quads, then a word
    char* const exp_places = lds + DEPTH * kStep;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, o = lane >> 4;

    const int nx = (p.NB + kRB - 1) / kRB;
    Pieces<16 * kMB> pieces{p.offsets, p.experts, p.M};
    int slots = p.slots;
    if constexpr (GROUPED) slots = min(slots, pieces.count() - p.slot0);
    const int total = slots * nx * p.slices;           // tiles of Y, each `slices` times

    struct Item { int expert, m0, m1, rb0, tile, slice, step, steps; };        // step .. steps - 1 of the whole of K
    // The tiles of an expert (without experts: all) are ordered in bands of at most kBand pieces of rows of X, so that what a die's cache holds
    // of either factor is used several times; higher ones by expert, whose weights come from memory.  (Bands of four across experts, and so:
    // 8 experts of 28672 x 4096, 2048 rows each, 1058 us and 1005; 32 of 4096 x 2304, 4099 rows, 58 and 54.  8192 rows, 8192 x 8192
    // without experts: 243 us, in bands of eight 249.)
    auto item = [&](int number) {
        constexpr int kBand = GROUPED ? 8 : 4;
        Item it;
        const int id = by_die(number, total);
        it.tile = p.slices == 1 ? id : quotient(id, p.slices);
        it.slice = id - it.tile * p.slices;
        int inside = it.tile, from = p.slot0, n = slots;                       // the tile's place among those of its expert's pieces
        typename Pieces<16 * kMB>::Found in{0, 0, p.M, 0, 0};
        if constexpr (GROUPED) {
            in = pieces.find(p.slot0 + quotient(it.tile, nx));
            from = max(in.begin, p.slot0);
            n = min(in.begin + in.pieces, p.slot0 + slots) - from;
            inside -= (from - p.slot0) * nx;
        }
        const int bands = (n + kBand - 1) / kBand, high = quotient(n + bands - 1, bands);
        const int band = quotient(inside, high * nx), left = min(high, n - band * high);
        inside -= band * high * nx;
        const int nt = quotient(inside, left);
        it.expert = in.expert;
        it.m0 = in.first + (from + band * high + inside - nt * left - in.begin) * 16 * kMB;
        it.m1 = min(in.end, it.m0 + 16 * kMB);
        it.rb0 = nt * kRB;
        it.step = 0;
        it.steps = (p.KT + 1) / 2;
        if (p.slices > 1) {                            // (up to 2^15 quads, and slices that the workspace holds: the product fits)
            it.step = 2 * quotient(it.slice * p.KQ, p.slices);
            it.steps = min(it.steps, 2 * quotient((it.slice + 1) * p.KQ, p.slices));
        }
        return it;
    };

    // Where the copies are: an item, its next step, the places they go to, and this lane's byte offsets in what the wavefront copies.  Rows
    // and row blocks past the end repeat the last.
    const int half = p.K / 2, ebytes = p.K / 32;
    const int block = (lane & 7) ^ (lane >> 4);        // of the row that this lane copies (i >> 1 of row i = 8 g + lane / 8 is 4 g + lane / 16)
    int number = (int)blockIdx.x, step = 0, steps = 0, place = 0, exp_place = 0;
    __amdgpu_buffer_rsrc_t wsrc, xsrc, esrc;
    uint32_t wfrom[kWLoads], xfrom[kXLoads], efrom[kExpLoads];
    auto aim = [&](const Item& it) {
        step = it.step;
        steps = it.steps;
        const int last_rb = p.NB - 1 - it.rb0, rows = it.m1 - it.m0;
        wsrc = unbounded(p.w + it.expert * p.expert + it.rb0 * p.record);
        xsrc = unbounded(p.x + (int64_t)it.m0 * half);
        esrc = unbounded(p.xe + (int64_t)it.m0 * ebytes);
#pragma unroll
        for (int j = 0; j < kWLoads; ++j) wfrom[j] = (uint32_t)min(wave + kWaves * j, last_rb) * (uint32_t)p.record + lane * 16;
#pragma unroll
        for (int j = 0; j < kXLoads; ++j) {
            const int c = wave + kWaves * j;           // eight rows
            xfrom[j] = (uint32_t)min(8 * c + (lane >> 3), rows - 1) * (uint32_t)half + (block ^ (4 * (c & 1))) * 16;
        }
#pragma unroll
        for (int j = 0; j < kExpLoads; ++j) {
            const int c = min(wave + kWaves * j, kExpPieces - 1);              // (the last may be copied twice)
            efrom[j] = c < kRB / 4 ? (uint32_t)min(4 * c + o, last_rb) * (uint32_t)p.record + (uint32_t)p.KT * 1024 + i * 16
                                   : (uint32_t)min(64 * (c - kRB / 4) + lane, rows - 1) * (uint32_t)ebytes;
        }
    };
    // Copy `j` of this wavefront's kLoads of a step.
    auto load_part = [&](int j) {
        char* to = lds + place * kStep;
        // An odd last step has one tile: the second is the first again, so that nothing behind the rows is touched, and
        // has exponents of zero on both sides, 2^-254 for their products, which adds nothing to an fp32 sum.
        const bool whole = 2 * step + 1 < p.KT;
        if (j < 2 * kWLoads) {
            const int c = wave + kWaves * (j >> 1), second = j & 1;
            copy16<ONCE ? kNonTemporal : 0>(wsrc, wfrom[j >> 1], step * 2048 + (second && whole ? 1024 : 0), to + c * 2048 + second * 1024);
        } else {
            const int c = wave + kWaves * (j - 2 * kWLoads);
            const uint32_t at = xfrom[j - 2 * kWLoads], from = whole ? at : at - ((block ^ (4 * (c & 1))) & 4) * 16;
            copy16(xsrc, from, step * 128, to + kRB * 2048 + c * 1024);
        }
    };
    // Exponents of the quad that begins with this step: of a row block of weights its 256 bytes, of a row of X its sixteen.  The row's last
    // quad may be short: the sixteen bytes that end with the row are taken then, so that no byte behind X is touched.
    auto load_exps = [&]() {
        if (step & 1) return;
        char* to = exp_places + exp_place * kExps;
        exp_place = exp_place == Shape::kExpPlaces - 1 ? 0 : exp_place + 1;
#pragma unroll
        for (int j = 0; j < kExpLoads; ++j) {
            const int c = min(wave + kWaves * j, kExpPieces - 1);
            if (c < kRB / 4) copy16(wsrc, efrom[j], step * 128, to + c * 1024);
            else copy16(esrc, efrom[j], min(step * 8, ebytes - 16), to + c * 1024);
        }
    };
    Item ahead = {};
    auto next = [&]() {
        place = (place + 1) % DEPTH;
        if (++step < steps) return;
        // (After the last item its last step is copied again and again, to places that nobody reads any more: as many copies are under way
        // at every step.)
        if (number + (int)gridDim.x < total) {
            number += (int)gridDim.x;
            ahead = item(number);
            aim(ahead);
        } else --step;
    };

    const int wn = wave % GN, wm = wave / GN;
    u32x4 w[WN], x[2][WM];
    uint32_t we[WN], xe[WM];
    f32x4 acc[WN][WM];
    int here = 0, exps_here = 0;                       // the places of the step and of the quad being multiplied
    const char* const wplace = lds + lane * 16 + wn * WN * 2048;
    const char* const xplace = lds + kRB * 2048 + i * 128 + wm * WM * 2048;
    const int xblock[2] = {(o ^ (i >> 1)) * 16, ((4 + o) ^ (i >> 1)) * 16};
    auto read_w = [&](int from, int h, int r) { w[r] = *reinterpret_cast<const u32x4*>(wplace + from * kStep + h * 1024 + r * 2048); };
    auto read_x = [&](int from, int h) {
#pragma unroll
        for (int b = 0; b < WM; ++b) x[h][b] = *reinterpret_cast<const u32x4*>(xplace + xblock[h] + from * kStep + b * 2048);
    };
    // A lane's word of exponents has the quad's tiles in its four bytes.  That is how the weights' lie; of X, word t of a row holds the
    // four blocks of tile t, of which this lane needs block o.
    auto read_exps = [&](int q) {
        const char* at = exp_places + exps_here * kExps;
        exps_here = exps_here == Shape::kExpPlaces - 1 ? 0 : exps_here + 1;
        const uint32_t pick = (uint32_t)o * 0x0101u + 0x0400u;
        const int missing = 4 * (q + 1) > p.KT ? 4 * (q + 1) - p.KT : 0;
#pragma unroll
        for (int r = 0; r < WN; ++r) we[r] = *reinterpret_cast<const uint32_t*>(at + (wn * WN + r) * 256 + lane * 4);
#pragma unroll
        for (int b = 0; b < WM; ++b) {
            const u32x4 e = *reinterpret_cast<const u32x4*>(at + kRB * 256 + (16 * (wm * WM + b) + i) * 16);
            const uint32_t low = __builtin_amdgcn_perm(e[1], e[0], pick), high = __builtin_amdgcn_perm(e[3], e[2], pick);
            xe[b] = __builtin_amdgcn_perm(high, low, 0x05040100u) >> (8 * missing);
        }
    };
    // The tile in the registers, half H of its step; the next one (half 1 - H, at `from`) is read meanwhile: of X into registers of
    // their own, of a row block of weights when its last product has been started.  Copies of a later step are asked for one at a
    // time between the products: together, they would keep the wavefronts from issuing anything else for a thousand cycles.
    auto multiply = [&](auto half_of_step, int from, auto before_reads, auto part) {
        constexpr int H = decltype(half_of_step)::value;
#pragma unroll
        for (int r = 0; r < WN; ++r) {
#pragma unroll
            for (int b = 0; b < WM; ++b) acc[r][b] = product<H, H>(w[r], x[H][b], acc[r][b], we[r], xe[b]);
            __builtin_amdgcn_sched_barrier(0);
            if (r == 0) {
                before_reads();
                read_x(from, 1 - H);
            }
            read_w(from, 1 - H, r);
            part(r);
        }
        // (without this the compiler moves products behind the branches and barriers that follow)
#pragma unroll
        for (int r = 0; r < WN; ++r)
#pragma unroll
            for (int b = 0; b < WM; ++b) asm volatile("" : "+v"(acc[r][b]));
    };
    // Step s of `it`; its first tile is in the registers.  `first` of an item: all copies of the steps that there is room for have been asked for,
    // and behind them kStores stores of the item before, if `stored`; those may still be under way when the next step has to be there.
    auto one_step = [&](auto first, int s, const Item& it, int first_quad, bool stored) {
        constexpr int kLate = WN / 2;
        multiply(integral_constant<int, 0>(), here, []() {}, [&](int r) {
            if (!first && r < kLate) {
#pragma unroll
                for (int j = kEarly + r * (kLoads - kEarly) / kLate; j < kEarly + (r + 1) * (kLoads - kEarly) / kLate; ++j) load_part(j);
            }
        });
        next();
        here = (here + 1) % DEPTH;
        multiply(integral_constant<int, 1>(), here, [&]() {
            // The next step is there, and nobody needs this one's place any more.  (Here and not before the first products, when the
            // operands read last may still be on their way.)
            if (first && stored) arrive<(DEPTH - 2) * kLoads + kStores>();
            else arrive<(DEPTH - 2) * kLoads>();
            __builtin_amdgcn_sched_barrier(0);
            load_exps();
        }, [&](int r) {
#pragma unroll
            for (int j = r * kEarly / WN; j < (r + 1) * kEarly / WN; ++j) load_part(j);
        });
        if (s + 1 == it.steps || (s & 1)) {
            read_exps(s + 1 == it.steps ? first_quad : s / 2 + 1);
        } else {
#pragma unroll
            for (int r = 0; r < WN; ++r) we[r] >>= 16;
#pragma unroll
            for (int b = 0; b < WM; ++b) xe[b] >>= 16;
        }
    };

    // Two wavefronts share a SIMD, and the older one is served first by itself: with the younger ones preferred they drift apart, and one
    // multiplies while the other waits for its copies to be taken (4096 rows, 28672 x 4096: 262 -> 246 us).
    if (kWaves == 8 && wave >= 4) __builtin_amdgcn_s_setprio(1);
    if (number >= total) return;
    Item it = item(number);
    aim(it);
#pragma unroll
    for (int t = 0; t < DEPTH; ++t) {
        load_exps();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) load_part(j);
        if (t < DEPTH - 1) next();
    }
    arrive<(DEPTH - 1) * kLoads>();
    read_exps(it.step / 2);
    read_x(0, 0);
#pragma unroll
    for (int r = 0; r < WN; ++r) read_w(0, 0, r);

    bool stored = false;
    for (int mine = (int)blockIdx.x;;) {
#pragma unroll
        for (int r = 0; r < WN; ++r)
#pragma unroll
            for (int b = 0; b < WM; ++b) acc[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        mine += (int)gridDim.x;
        int first_quad = 0;                            // of the next item
        if (Shape::kSlices && p.slices > 1 && mine < total) first_quad = item(mine).step / 2;
        int s = it.step;
        one_step(std::true_type(), s, it, first_quad, stored);
        for (++s; s < it.steps; ++s) one_step(std::false_type(), s, it, first_quad, false);
#pragma unroll
        for (int j = kEarly; j < kLoads; ++j) load_part(j);

        bool finished = true;
        if (Shape::kSlices && p.slices > 1) {          // the other slices of this tile
            const auto sums = unbounded(p.partial + ((int64_t)it.tile * p.slices) * Shape::kSums);
            const uint32_t at = wave * (WN * WM * 1024) + lane * 16;
#pragma unroll
            for (int r = 0; r < WN; ++r)
#pragma unroll
                for (int b = 0; b < WM; ++b) store16_shared(sums, at + (r * WM + b) * 1024, it.slice * Shape::kSums, acc[r][b]);
            arrive<0>();
            uint32_t* last = reinterpret_cast<uint32_t*>(lds + Shape::kLds - 16);
            if (threadIdx.x == 0) {
                uint32_t* count = p.counters + it.tile;
                const uint32_t n = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                *last = n + 1 == (uint32_t)p.slices;
                if (*last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            finished = __builtin_amdgcn_readfirstlane(*last);
            __syncthreads();                           // (the word is free for the next item)
            if (finished) {
                // In the order of the slices, this one from its registers, the others two ahead.
                f32x4 sum[WN][WM] = {}, even[WN][WM], odd[WN][WM];
                auto ask = [&](int z, f32x4(&to)[WN][WM]) {
                    if (z >= p.slices || z == it.slice) return;
#pragma unroll
                    for (int r = 0; r < WN; ++r)
#pragma unroll
                        for (int b = 0; b < WM; ++b) to[r][b] = load16_shared(sums, at + (r * WM + b) * 1024, z * Shape::kSums);
                };
                auto add = [&](const f32x4(&from)[WN][WM]) {
#pragma unroll
                    for (int r = 0; r < WN; ++r)
#pragma unroll
                        for (int b = 0; b < WM; ++b) sum[r][b] += from[r][b];
                };
                auto take = [&](int z, f32x4(&from)[WN][WM]) {
                    if (z >= p.slices) return;
                    if (z == it.slice) add(acc);
                    else add(from);
                    ask(z + 2, from);
                };
                ask(0, even);
                ask(1, odd);
                for (int z = 0; z < p.slices; z += 2) {
                    take(z, even);
                    take(z + 1, odd);
                }
#pragma unroll
                for (int r = 0; r < WN; ++r)
#pragma unroll
                    for (int b = 0; b < WM; ++b) acc[r][b] = sum[r][b];
            }
        }
        // (kStores stores by every wavefront, which the next item's first step need not wait for; 8192 rows, 8192 x 2048, 77 us either way)
        if (finished) {
#pragma unroll
            for (int b = 0; b < WM; ++b) {
                const int m = it.m0 + 16 * (wm * WM + b), rb = it.rb0 + wn * WN;
                store_rows<WN>([&](int r) { return acc[r][b]; }, p.y + ((int64_t)m * p.N + 16 * rb) * 2, it.m1 - m, p.NB - rb, p.N, p.bf16);
            }
        }
        stored = finished;
        if (mine >= total) break;
        it = number == mine ? ahead : item(mine);      // (the copies may be further ahead where items have fewer steps than there is room for)
    }
    arrive<0>();                                       // (no copy into this workgroup's LDS outlives it)
}

namespace {

constexpr size_t kCounterBytes = 64 * 1024;
constexpr int64_t kCounters = kCounterBytes / 4;
constexpr size_t kPartialBytes = 32 * 1024 * 1024;

int64_t most_pieces(const ProductParams& p, int rows) { return product::most_pieces(p.M, p.offsets ? p.experts : 0, rows); }

template <int SRC, int R, int ROWS>
hipError_t launch_stream(ProductParams p, int waves, hipStream_t s) {
    const int nx = (p.NB + R - 1) / R;
    const size_t lds = (size_t)waves * kStreamPlace;
    // (a launch has fewer than 2^16 workgroups along y and 2^32 threads)
    int64_t most = (int64_t(1) << 31) / (int64_t(nx) * waves * 64);
    most = most > 65535 ? 65535 : most;
    const int64_t each = R == 4 ? waves : 1, pieces = most_pieces(p, 16), slots = (pieces + each - 1) / each;
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < slots && e == hipSuccess; at += most) {
        p.slot0 = (int)(at * each);
        const dim3 grid(nx, (unsigned)(slots - at < most ? slots - at : most));
        e = p.offsets ? launch<stream_kernel<SRC, R, ROWS, true>>(grid, waves * 64, lds, p, s)
                      : launch<stream_kernel<SRC, R, ROWS, false>>(grid, waves * 64, lds, p, s);
    }
    return e;
}

// Output channels and rows of a tile, wavefronts, and steps of room, by shape.
struct TileSize { int channels, rows, waves, room; };
constexpr TileSize kTiles[] = {{256, 256, 8, 2}, {128, 128, 4, 2}, {128, 128, 8, 4}, {128, 64, 8, 4}, {64, 64, 4, 4}};

template <int SHAPE, int WN, int WM, int GN, int GM, int DEPTH>
hipError_t launch_tiles(ProductParams p, int cus, hipStream_t s) {
    using Shape = TileShape<WN, WM, GN, GM, DEPTH>;
    static_assert(kTiles[SHAPE].channels == 16 * Shape::kRB && kTiles[SHAPE].rows == 16 * Shape::kMB && kTiles[SHAPE].waves == Shape::kWaves &&
                  kTiles[SHAPE].room == DEPTH, "as the choice knows it");
    constexpr int kAtOnce = 160 * 1024 / Shape::kLds < 8 / Shape::kWaves ? 160 * 1024 / Shape::kLds : 8 / Shape::kWaves;   // per compute unit
    const int64_t nx = (p.NB + Shape::kRB - 1) / Shape::kRB, pieces = most_pieces(p, 16 * Shape::kMB);
    const int64_t most = (int64_t(1) << 30) / (nx * p.slices);                 // pieces of rows per launch: tiles are counted in 32 bits
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < pieces && e == hipSuccess; at += most) {
        p.slot0 = (int)at;
        p.slots = (int)(pieces - at < most ? pieces - at : most);
        const int64_t items = nx * p.slots * p.slices, grid = items < (int64_t)cus * kAtOnce ? items : (int64_t)cus * kAtOnce;
        auto run = [&](auto once) {
            constexpr bool ONCE = decltype(once)::value;
            const dim3 g((unsigned)grid);
            return p.offsets ? launch<tile_kernel<WN, WM, GN, GM, DEPTH, true, ONCE>>(g, Shape::kThreads, Shape::kLds, p, s)
                             : launch<tile_kernel<WN, WM, GN, GM, DEPTH, false, ONCE>>(g, Shape::kThreads, Shape::kLds, p, s);
        };
        if constexpr (Shape::kMB <= 8) e = p.once ? run(std::true_type()) : run(std::false_type());
        else e = run(std::false_type());
    }
    return e;
}

// Whether the weights are streamed past sixteen rows at a time, or which tile shape, and for the smaller ones how many slices of K: the least
// of times estimated from the bytes of weights over the pieces of rows (B), or from the number of tiles on the busiest compute unit (n) and of
// steps (S).  Microseconds, fitted to some 300 products of 17 to 16384 rows, N 256 to 32768, K 512 to 16384.  On 130 other ones the least
// of all shapes and slices was 2 % less on average, on 130 by expert 4 %, and most where many experts have a short K: 1764 rows
// through 87 of 1344 x 768 take 28.2, the 128 x 128 tiles of two workgroups per unit 17.9.
//   streamed        2.3 + B / 6.6 TB/s
//   256 x 256       6.0 + n (1.75 S + 4.5)                one workgroup per compute unit; the 4.5 are its stores
//   128 x 128       1.5 + 1.25 S + 2.6 per two, 0.95 S + 1.3 for one; two workgroups per unit, two steps of room each
//   128 x 128 deep  3.2 + n (0.72 S + 1), 0.63 S for one  one of eight wavefronts, four steps of room; in z slices of K 2.5 + 1.6 z more
//   128 x 64 deep   3.2 + n (0.50 S + 0.7)                the same; in z slices 3 + 0.8 z more
//   64 x 64 deep    3.0 + 0.62 S + 0.9 per two, 0.37 S + 0.9 for one; two of four wavefronts; in z slices 1.8 + z more
// Examples (us, shapes in this order, weights from memory): 17 rows, 6144 x 4096 6.2, and tiles at best 9.2; 28672 x 4096 21.9, and 15.9; 512
// rows, 4096 x 4096 18.6, 30.3, 18.2, 15.8, 12.4, 14.7; 8192 rows, 8192 x 8192 -, 249, 322, 379, 512, 563; 200 rows, 28672 x 4096 112, 33.5, 26.6,
// 29.2, 36.6, 33.4; 200 rows, 5120 x 13824 39.6, 86, 51.5, 37.7, 28.1, 31.1, and 23.0 with 128 x 128 in three slices; 64 rows, 4096 x 14336 17.1, 84,
// 52.9, 38.0, 33.8, 24.5, and 13.2 with 64 x 64 in four.  80 rows through 2 experts of 4096 x 14336: 26.8, in slices 21.7.
// By expert the number of pieces is not known here: every expert is taken to have the mean number of rows and half a piece that is not full.
// Few rows on average stay with the streaming kernel also where one expert has most of them and its weights are read again for every sixteen
// (64 experts of 2816 x 2048, 500 rows, 454 of them one expert's: 29.2, tiles at best 28.2; 16 of 4096 x 4096, 250 rows, 228: 29.6 and 25.9).
struct TileChoice { int shape, slices; };             // shape -1: streamed

TileChoice choose_tiles(int64_t M, int64_t NB, int64_t KT, int64_t experts, int64_t record, int cus) {
    const double S = (double)((KT + 1) / 2);
    const int64_t KQ = (KT + 3) / 4;
    TileChoice best{-1, 1};
    auto tiles = [&](int64_t rb, int64_t rows) {
        const int64_t nx = (NB + rb - 1) / rb;
        if (!experts) return (double)nx * (double)((M + rows - 1) / rows);
        const double some = (double)(M < experts ? M : experts), filled = (double)M / (double)rows + 0.5 * some;
        return (double)nx * (filled > some ? filled : some);
    };
    if (M <= 16 * (experts ? experts : 1) || KT < 4) return best;              // (tiles begin with a whole quad)
    double least = 2.3 + tiles(1, 16) * (double)record / 6.6e6;
    auto consider = [&](int shape, int slices, double us) {
        if (us < least) { least = us; best = {shape, slices}; }
    };
    auto rounds = [&](double t) { return (double)(int64_t)((t + cus - 1) / cus); };
    auto pairs = [&](double n, double one, double two) { return two * (double)(int64_t)(n / 2) + ((int64_t)n % 2 ? one : 0.0); };
    const double t0 = tiles(16, 256), t1 = tiles(8, 128), t3 = tiles(8, 64), t4 = tiles(4, 64);
    const double n0 = rounds(t0), n1 = rounds(t1);
    consider(0, 1, 6.0 + n0 * (1.75 * S + 4.5 * (t0 < cus ? t0 / cus : 1.0)));
    consider(1, 1, 1.5 + pairs(n1, 0.95, 1.25) * S + 1.3 * n1);
    for (int z = 1; z <= 8; ++z) {
        const double steps = (double)((int64_t)(S + z - 1) / z);
        if (z > KQ) break;
        if (z == 1 || t1 * z <= cus) consider(2, z, 3.2 + rounds(t1 * z) * ((t1 > cus ? 0.72 : 0.63) * steps + 1.0) + (z > 1 ? 2.5 + 1.6 * z : 0.0));
        if (z == 1 || t3 * z <= cus) consider(3, z, 3.2 + rounds(t3 * z) * (0.50 * steps + 0.7) + (z > 1 ? 3.0 + 0.8 * z : 0.0));
        if (z == 1 || t4 * z <= 2 * cus) consider(4, z, 3.0 + pairs(rounds(t4 * z), 0.37 * steps + 0.9, 0.62 * steps + 0.9) + (z > 1 ? 1.8 + 1.0 * z : 0.0));
    }
    if (best.slices > 1) {                             // as many as the workspace has room for
        const TileSize t = kTiles[best.shape];
        const int64_t most = (NB * 16 + t.channels - 1) / t.channels * product::most_pieces(M, experts, t.rows);
        while (best.slices > 1 && (most > kCounters || most * best.slices * t.channels * t.rows * 4 > (int64_t)kPartialBytes)) --best.slices;
    }
    return best;
}

// How a product is launched.
struct Choice {
    TileChoice tiles;
    bool apart;                // X of 16 bits is quantised by a launch of its own
    bool once;                 // weights past the caches
    // streamed:
    int wide;                  // row blocks per workgroup
    int rows;                  // of X that are quantised at a time, 0: X is codes
    int waves;                 // per workgroup
};

// `experts`: 0 without.
Choice choose(int64_t M, int64_t NB, int64_t KT, int64_t experts, int64_t record, bool codes, int cus) {
    Choice c{};
    const int KQ = (int)((KT + 3) / 4);
    c.tiles = choose_tiles(M, NB, KT, experts, record, cus);
    // (Figures: us, weights from memory.)  Where the streaming workgroups quantise X on the way in, every one of them does it for all its rows.  Up to
    // four rows, beyond some 160 rows and quads per compute unit that takes longer than a launch which does it once (so and with that launch:
    // 4096 x 14336, 1 row (28) 8.5 and 10.7; 28672 x 4096, 4 rows (128) 15.2 and 15.5; 512 x 16384, 4 rows (128) 8.6 and 8.7; 4096 x 14336, 6 rows
    // (168) 14.1 and 10.9).  More rows cost the same however many they are, like twenty (16 rows, 4096 x 4096 (8 quads) 6.7 and 7.2,
    // 6144 x 4096 (8) 7.1 and 8.4; 6 rows, 1024 x 8192 (16) 8.7 and 7.4, 13824 x 5120 (20) 14.4 and 12.2; 211 rows through 41 experts of 288 x 640 (4)
    // 6.1 and 6.8).
    // Two row blocks per workgroup halve it, and leave fewer wavefronts to hide the reads (one and two: 28672 x 4096, 1 row 13.9 and 13.3;
    // 128256 x 4096, 1 row 47.2 and 45.1; 128 experts of 1536 x 4096, 64 rows 26.7 and 23.1; but 28672 x 4096, 2 rows 13.3 and 14.3, 4 rows 14.3 and
    // 15.2).  Codes gain by two where workgroups are many and share their weights (64 experts of 2816 x 2048, 500 rows 39.3 and 37.0;
    // 128256 x 4096, 13 rows 53.2 and 47.9); with a row or two each it is much the same (60 rows 22.9 and 22.2; 1 row 44.6 and 45.5).  A single quad
    // of K leaves nothing to hide: 8192 rows, 8192 x 384, 101 with one row block, 82 with two, 55 with four.
    const int64_t pieces = experts ? (M < experts ? M : experts) : (M + 15) / 16, groups = NB * pieces, mean = (M + pieces - 1) / pieces;
    int wide = !codes && (groups > 1024 || mean > 4) ? 2 : 1;
    const int64_t rounds = (groups / wide + cus - 1) / cus;                    // of workgroups
    const bool apart = rounds * KQ * (mean > 4 ? 20 : mean) > 160;
    c.apart = !codes && (c.tiles.shape >= 0 || apart);
    if (c.apart) {
        codes = true;
        wide = 1;
    }
    if (codes && groups > (experts ? 2048 : 4096)) wide = KQ == 1 ? 4 : mean > 2 ? 2 : 1;
    // Weights that are read once and take more than half of the 256 MB cache are read past it (kept and past: 57344 x 8192, 250 MB, 1 row
    // 45.4 and 42.9; 128256 x 4096 52.2 and 45.5; 64 experts of 2816 x 2048, 250 rows 35.1 and 31.8; of 1536 x 4096, 1100 rows 49.8 and 47.0).  Smaller
    // ones may still be there at the next call: 28672 x 4096, 13 rows, three matrices in turn 11.4 and 12.5.  Where they are not, because
    // the program reads a cache full of others in between, they lose what past the cache would save, 3 to 9 % from 24 MB on (the same
    // from memory: 14.3 and 13.2).  Nor where several workgroups read the same ones (8 experts of 4096 x 4096, 64 rows, in
    // turn 14.9 and 16.8; 1024 rows, 5120 x 5120 28.9 and 33.0).
    const int64_t shared = c.tiles.shape >= 0 ? (c.tiles.shape == 3 || c.tiles.shape == 4 ? 64 : 128) : experts ? 4 : 16;
    c.once = (experts ? mean : M) <= shared && NB * (experts ? pieces : 1) * record > (int64_t(128) << 20);
    // Wavefronts of a workgroup, up to one per quad: sixteen with one row block (values, 1 row, 4096 x 14336: 12.3 with four, 9.6 with eight, 8.5 with
    // sixteen); eight with two (their registers) or where they quantise and workgroups are many (1 row, with eight and sixteen: 8192 x 8192, 512
    // workgroups, 9.4 and 9.0; 10240 x 8192, 640, 11.1 and 11.4); four where they are so many that their beginnings count (128256 x 4096, 8016 groups: 13
    // rows of codes 47.9 and with eight 48.9; 57344 x 4096, 3584, 1 row 24.6 and 23.4).  By expert, where X is codes, four from fewer workgroups
    // on, and fewer with two quads each where there are very many, as some find that there is nothing for them, and the others lie all
    // over the weights (16 experts of 2048 x 4096, 64 rows: 15.1 with four, 16.2 with eight; 32 of 480 x 4096, 30 rows, 900: 6.7 and 6.8; 65 of
    // 720 x 6272, 100 rows: 24.7 with four, 32.9 with thirteen; 128 of 1536 x 3584, 128 rows: 39.4 with three, 57.0 with seven; 50 of 3376 x 2688, 28
    // rows: 18.8 with three, 19.7 with four; 41 of 480 x 1408, 40 rows, 1200: 4.8 with three, 5.4 with two).
    const int many = groups > 2048 ? (KQ < 4 ? 2 : KQ < 8 ? KQ / 2 : 4) : 4;
    const int most = experts && codes && groups > 900 ? many : groups > 4096 ? 4 : wide > 1 || (!codes && groups > 512) ? 8 : 16;
    c.waves = wide == 4 ? (pieces < 4 ? (int)pieces : 4) : KQ < most ? KQ : most;
    c.wide = wide;
    c.rows = codes ? 0 : mean > 4 ? 16 : mean > 1 ? 4 : 1;
    return c;
}

template <int R, int ROWS> hipError_t launch_stream_of(int src, const ProductParams& p, int waves, hipStream_t s) {
    return src == kF16 ? launch_stream<kF16, R, ROWS>(p, waves, s) : launch_stream<kBF16, R, ROWS>(p, waves, s);
}

lutq_status product_on(const void* X, const void* xe, const void* packed, const int32_t* offsets, int64_t experts, int64_t M,
                       int64_t N, int64_t K, lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, hipStream_t s) {
    if (lutq_mx4_workspace_bytes(M, N, K, experts) == 0) return LUTQ_ERR_SHAPE;
    if (dtype != LUTQ_F16 && dtype != LUTQ_BF16) return LUTQ_ERR_DTYPE;
    if (M == 0) return LUTQ_OK;
    if (!X || !packed || !Y) return LUTQ_ERR_NULL;
    if (!aligned(X, 16) || !aligned(xe, 16) || !aligned(packed, 16) || !aligned(Y, 16) || !aligned(workspace, 16) || !aligned(offsets, 4))
        return LUTQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < lutq_mx4_workspace_bytes(M, N, K, experts)) return LUTQ_ERR_WORKSPACE;

    ProductParams p{};
    p.x = static_cast<const char*>(X); p.xe = static_cast<const char*>(xe);
    p.w = static_cast<const char*>(packed); p.y = static_cast<char*>(Y);
    p.offsets = offsets; p.experts = (int)experts;
    p.record = record_bytes(K); p.expert = N / 16 * p.record;
    p.M = (int)M; p.N = (int)N; p.K = (int)K; p.KT = (int)k_tiles(K); p.KQ = (int)k_quads(K); p.NB = (int)(N / 16);
    p.bf16 = dtype == LUTQ_BF16;
    p.counters = static_cast<uint32_t*>(workspace);
    p.partial = static_cast<char*>(workspace) + kCounterBytes;
    int src = xe ? kF32 : dtype == LUTQ_F16 ? kF16 : kBF16;
    const int cus = compute_units();
    if (cus < 1) return LUTQ_ERR_DEVICE;
    const Choice c = choose(M, p.NB, p.KT, offsets ? experts : 0, p.record, xe != nullptr, cus);
    if (c.apart) {
        char *codes = p.partial + kPartialBytes, *exponents = codes + up256((size_t)M * (K / 2));
        const lutq_status st = quantize_rows_on(X, src, M, nullptr, M, K, codes, exponents, s);
        if (st != LUTQ_OK) return st;
        p.x = codes; p.xe = exponents;
        src = kF32;
    }
    p.once = c.once;
    p.slices = c.tiles.slices;
    hipError_t e;
    switch (c.tiles.shape) {
        case 0: e = launch_tiles<0, 8, 4, 2, 4, 2>(p, cus, s); break;
        case 1: e = launch_tiles<1, 4, 4, 2, 2, 2>(p, cus, s); break;
        case 2: e = launch_tiles<2, 4, 2, 2, 4, 4>(p, cus, s); break;
        case 3: e = launch_tiles<3, 2, 2, 4, 2, 4>(p, cus, s); break;
        case 4: e = launch_tiles<4, 2, 2, 2, 2, 4>(p, cus, s); break;
        default:
            if (c.rows == 0) e = c.wide == 1   ? launch_stream<kF32, 1, 16>(p, c.waves, s)
                                 : c.wide == 2 ? launch_stream<kF32, 2, 16>(p, c.waves, s)
                                               : launch_stream<kF32, 4, 16>(p, c.waves, s);
            else if (c.rows == 16) e = launch_stream_of<2, 16>(src, p, c.waves, s);
            else if (c.rows == 4) e = c.wide == 2 ? launch_stream_of<2, 4>(src, p, c.waves, s) : launch_stream_of<1, 4>(src, p, c.waves, s);
            else e = c.wide == 2 ? launch_stream_of<2, 1>(src, p, c.waves, s) : launch_stream_of<1, 1>(src, p, c.waves, s);
    }
    return e == hipSuccess ? LUTQ_OK : LUTQ_ERR_DEVICE;
}

}  // namespace

}  // namespace mx4
}  // namespace lutq

using namespace lutq::mx4;

extern "C" size_t lutq_mx4_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts) {
    if (!shape_ok(N, K) || !rows_ok(M, K) || experts < 1 || experts > 65536) return 0;
    return kCounterBytes + kPartialBytes + up256((size_t)M * (size_t)(K / 2)) + up256((size_t)M * (size_t)(K / 32));
}

extern "C" lutq_status lutq_mx4_matmul(const void* X, const void* x_exponents, const void* packed, int64_t M, int64_t N, int64_t K,
                                       lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, void* stream) {
    return product_on(X, x_exponents, packed, nullptr, 1, M, N, K, dtype, Y, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_mx4_matmul_grouped(const void* X, const void* x_exponents, const void* packed, const int32_t* offsets,
                                               int64_t experts, int64_t M, int64_t N, int64_t K, lutq_dtype dtype, void* Y,
                                               void* workspace, size_t workspace_bytes, void* stream) {
    if (M > 0 && !offsets) return LUTQ_ERR_NULL;
    return product_on(X, x_exponents, packed, offsets, experts, M, N, K, dtype, Y, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int lutq_calib_mx4_launch(int64_t M, int64_t N, int64_t K, int64_t experts, int x_is_codes, int compute_units, int* launch) {
    if (!launch) return LUTQ_ERR_NULL;
    if (experts < 0 || lutq_mx4_workspace_bytes(M, N, K, experts ? experts : 1) == 0 || M < 1 || compute_units < 1 || compute_units > 4096)
        return LUTQ_ERR_SHAPE;
    const Choice c = choose(M, N / 16, k_tiles(K), experts, record_bytes(K), x_is_codes != 0, compute_units);
    const bool streamed = c.tiles.shape < 0;
    const TileSize t = streamed ? TileSize{16 * c.wide, 16, c.waves, 0} : kTiles[c.tiles.shape];
    const int out[8] = {c.apart, t.channels, t.rows, t.waves, t.room, c.tiles.slices, streamed ? c.rows : 0, c.once && c.tiles.shape != 0};
    for (int i = 0; i < 8; ++i) launch[i] = out[i];
    return LUTQ_OK;
}
