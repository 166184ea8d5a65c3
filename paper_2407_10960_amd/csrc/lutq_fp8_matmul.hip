// Products of the 8-bit form (include/lutq.h): Y = X W^T, the same by expert, the gated block's two projections with its activation and
// product, and the gradient of weights, on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// One instruction sums the products of 128 columns of sixteen rows of either factor, which is one block of the scales: what it returns is multiplied
// with the two blocks' scales in 32 bits and added to the sums.  The scales of the gradient's factors are powers of two, which the
// instruction applies itself.
// Its first operand is the weights, so a lane's four sums are neighbours in a row of Y.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lutq.h"
#include "lutq_calib.h"
#include "lutq_fp8_device.hpp"
#include "lutq_layout.hpp"
#include "lutq_product.hpp"

namespace lutq {
namespace fp8 {

using namespace product;

lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, const int32_t* offsets, int64_t experts,
                             int64_t M, int64_t K, void* codes, float* scales, hipStream_t stream);

// kGated: a workgroup's row blocks are half of the gate's weights, half of the others', the same columns of H.  kPowers: both factors'
// scales are powers of two, one per row and block of 128 columns.
enum Mode { kPlain = 0, kGated = 1, kPowers = 2 };

struct ProductParams {
    const char* x;             // codes [M, K]; or 16-bit values
    const float* xs;           // scales [KT, M]
    const char* w;             // codes [N, K] (kGated: [2 N, K])
    const float* ws;           // scales [ceil(N / 128), KT] (kPowers: [KT, N])
    char* y;                   // [M, N]
    char* saved;               // kGated: [M, 2 N] or null
    const int32_t* offsets;    // by expert: experts + 1; else null
    uint32_t* counters;        // K in slices: how many of a tile's are done, and
    char* partial;             // their sums
    int64_t expert, expert_scales;             // bytes of an expert's weights, numbers of its scales
    int M, N, K, KT, NB;       // blocks of 128 columns, of sixteen columns of Y
    int experts;
    int slot0, slots;          // first piece of rows of this launch, and how many
    int slices;                // of K
    int bf16;                  // type of Y
    int act;
    int once;                  // weights that are read once and do not stay in the caches: past them
    int place_rows;            // streamed: rows of X that a wavefront's place in LDS holds
};

// H from sums of the gate's and the other projection.
__device__ __forceinline__ f32x4 gated(const f32x4& g, const f32x4& u, int act) {
    f32x4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = activated(g[j], act) * u[j];
    return h;
}

// Where something in LDS lies, as its instructions take it.
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Quotient of a lane's numbers.
__device__ __forceinline__ int quotient_of_lane(int a, int b) { return b == 1 ? a : (int)((uint32_t)a / (uint32_t)b); }

// Four neighbouring sums of a row, as 16-bit values.
__device__ __forceinline__ void store_four(char* to, const f32x4& sum, int bf16) {
    *reinterpret_cast<u32x2*>(to) = u32x2{round_pair(sum[0], sum[1], bf16), round_pair(sum[2], sum[3], bf16)};
}

// Few rows: a workgroup has up to sixteen rows of X and a run of row blocks of weights (kGated: of both projections), one after the other over all of K;
// its wavefronts have a part of K each, and their sums are added in LDS in the order of the wavefronts.  Bound by the reads of the weights: they
// are copied from memory to LDS in whole cache lines, DEPTH blocks of 128 columns ahead, without passing through registers, and
// from one row block to the next without a pause.
// X of 16 bits (SRC 1, 2) is quantised into LDS by all wavefronts before the first product, sixteen lanes per block; codes come block by block with the
// weights, XP pieces of eight rows.
// The sums of the codes are exact (Wide): the 16-bit instruction's half rate is far above what the reads leave to do.
// Measured (weights as a program finds them, partly in the caches): one row, 6144 x 4096, 6.0 us; gated 28672 x 4096 16.4 (7.2 TB/s); 250 rows of 64 experts, 2816 x
// 2048, 59 (5.8 TB/s).  A first form with the weights loaded into operand registers took 14 and 28 us a call from Python for the first two, this one 6.9 and 19.4.
constexpr int kStreamWaves = 8;                        // per workgroup at most; registers for two such workgroups a compute unit
constexpr int kAhead = 8;                              // blocks of X per sixteen lanes that are asked for at a time

// Waits until at most BLOCKS times N of this wavefront's global loads are under way.
template <int N> __device__ __forceinline__ void wait_blocks(int blocks) {
    if (blocks >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * N) : "memory");
    else if (blocks == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * N) : "memory");
    else if (blocks == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

constexpr int stream_depth(int mode) { return mode == kGated ? 2 : 4; }
// Bytes of LDS of a wavefront's places, and of its sums, two sets of them in turn.
constexpr int stream_place(int mode, int xp) { return stream_depth(mode) * ((mode == kGated ? 2 : 1) * 2048 + xp * 1024 + (xp ? 256 : 0)); }
constexpr int stream_sums(int mode) { return 2 * (mode == kGated ? 2 : 1) * 1024; }

// A number that every lane has, and that nothing in the launch writes.
__device__ __forceinline__ float scalar_at(const float* p) { return *(const __attribute__((address_space(4))) float*)(uintptr_t)p; }

template <int SRC, int XP, int MODE, bool GROUPED, bool ONCE>
__global__ __launch_bounds__(64 * kStreamWaves, 4) void stream_kernel(const ProductParams p) {
    constexpr int R = MODE == kGated ? 2 : 1, DEPTH = stream_depth(MODE);
    static_assert(DEPTH <= 4, "as wait_blocks knows");
    static_assert((SRC == kF32) == (XP > 0), "codes come in pieces");
    constexpr int kSlot = R * 2048 + XP * 1024 + (XP ? 256 : 0), kCopies = 2 * R + (XP ? XP + 1 : 0);
    extern __shared__ __align__(1024) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, i = lane & 15, o = lane >> 4;
    const int slot = p.slot0 + (int)blockIdx.y;
    int expert = 0, m0 = slot * 16, m1 = min(p.M, m0 + 16);
    if constexpr (GROUPED) {
        Pieces<16> pieces{p.offsets, p.experts, p.M};
        if (slot >= pieces.count()) return;
        const auto in = pieces.find(slot);
        expert = in.expert;
        m0 = in.first + (slot - in.begin) * 16;
        m1 = min(in.end, m0 + 16);
    }
    const int rows = m1 - m0;
    // This workgroup's row blocks and this wavefront's part of K (up to 2^15 blocks over eight wavefronts: the products fit).
    const int run = (int)blockIdx.x, each = quotient(p.NB, (int)gridDim.x), more = p.NB - each * (int)gridDim.x;
    const int rb0 = run * each + min(run, more), rb1 = rb0 + each + (run < more ? 1 : 0);
    const int kb0 = quotient(wave * p.KT, waves), kb1 = quotient((wave + 1) * p.KT, waves);
    const char* const w = p.w + expert * p.expert;
    const float* const ws = p.ws + expert * p.expert_scales;
    char* const place = smem + wave * (DEPTH * kSlot);
    f32x4* const sums = reinterpret_cast<f32x4*>(smem + waves * (DEPTH * kSlot));      // [in turn][wave][row block][lane]
    char* const staged = smem + waves * (DEPTH * kSlot + stream_sums(MODE));
    const int pitch = p.K + 16;                        // (rows sixteen bytes apart: no two in the same banks)
    float* const staged_scales = reinterpret_cast<float*>(staged + p.place_rows * pitch);              // [block][row]

    // Unit u of what is quantised is block u / rows of row u % rows.
    const int units = XP ? 0 : rows * p.KT, teams = (int)blockDim.x >> 4, team = (int)threadIdx.x >> 4;
    Eight<XP ? kF16 : SRC> ahead[XP ? 1 : kAhead];
    auto ask = [&](int u, int t) {
        if (u >= units) return;
        const int kb = quotient_of_lane(u, rows), row = m0 + u - kb * rows;
        ahead[t].v[0] = *reinterpret_cast<const u32x4*>(p.x + ((int64_t)row * p.K + kb * 128 + 8 * i) * 2);
    };
    auto stage = [&](int u, int t) {
        if (u >= units) return;
        const int kb = quotient_of_lane(u, rows), row = u - kb * rows;
        float v[8];
        to_floats<XP ? kF16 : SRC>(ahead[t], v);
        const Scale s = scale_of(largest_of_sixteen(largest(v)));
        const u32x2 codes = to_codes(v, s);
        // (written so, as the compiler would have every copy to LDS that is under way arrive before it lets anything else write there)
        const uint32_t to = lds_offset(staged + row * pitch + kb * 128 + 8 * i), scale_to = lds_offset(staged_scales + kb * rows + row);
        asm volatile("ds_write_b64 %0, %1" ::"v"(to), "v"(codes) : "memory");
        if (i == 0) asm volatile("ds_write_b32 %0, %1" ::"v"(scale_to), "v"(s.scale) : "memory");
    };
    if constexpr (XP == 0) {
#pragma unroll
        for (int t = 0; t < kAhead; ++t) ask(team + t * teams, t);
    }

    const int block = (lane & 7) ^ (lane >> 4);        // of the row that this lane copies, as in the tiles
    uint32_t from[2], xfrom[XP ? XP : 1];
#pragma unroll
    for (int c = 0; c < 2; ++c) from[c] = (uint32_t)(8 * c + (lane >> 3)) * (uint32_t)p.K + (block ^ (4 * c)) * 16;
#pragma unroll
    for (int c = 0; c < XP; ++c) xfrom[c] = (uint32_t)min(8 * c + (lane >> 3), rows - 1) * (uint32_t)p.K + (block ^ (4 * c)) * 16;
    int rb_ahead = rb0, kb_ahead = kb0, d_ahead = 0;   // of the next copies
    auto issue = [&]() {                               // (at the end the last block stays next)
        char* to = place + d_ahead * kSlot;
        const int kb = kb_ahead;
        if constexpr (XP > 0) {
#pragma unroll
            for (int c = 0; c < XP; ++c) copy16(unbounded(p.x + (int64_t)m0 * p.K), xfrom[c], kb * 128, to + R * 2048 + c * 1024);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(unbounded(reinterpret_cast<const char*>(p.xs + (int64_t)kb * p.M + m0)),
                (__attribute__((address_space(3))) void*)(to + R * 2048 + XP * 1024), 4, min(i, rows - 1) * 4, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                copy16<ONCE ? kNonTemporal : 0>(unbounded(w + ((int64_t)r * p.N + rb_ahead * 16) * p.K), from[c], kb * 128, to + r * 2048 + c * 1024);
        d_ahead = d_ahead == DEPTH - 1 ? 0 : d_ahead + 1;
        if (kb_ahead + 1 < kb1) ++kb_ahead;
        else if (rb_ahead + 1 < rb1) {
            kb_ahead = kb0;
            ++rb_ahead;
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) issue();           // (fewer blocks than there is room for: the last again)
    if constexpr (XP == 0) {
#pragma unroll
        for (int t = 0; t < kAhead; ++t) stage(team + t * teams, t);
        for (int u = team + kAhead * teams; u < units; u += kAhead * teams) {
#pragma unroll
            for (int t = 0; t < kAhead; ++t) ask(u + t * teams, t);
#pragma unroll
            for (int t = 0; t < kAhead; ++t) stage(u + t * teams, t);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    const int first_half = (o ^ (i >> 1)) * 16, second_half = ((4 + o) ^ (i >> 1)) * 16, xrow = min(i, rows - 1);
    int d = 0, turn = 0, left = (rb1 - rb0) * (kb1 - kb0);                     // blocks that are still to be multiplied
    for (int rb = rb0; rb < rb1; ++rb) {
        const float* const scales = ws + (int64_t)(rb >> 3) * p.KT;
        f32x4 acc[R] = {};
        for (int kb = kb0; kb < kb1; ++kb, --left) {
            float sw[R];
#pragma unroll
            for (int r = 0; r < R; ++r) sw[r] = scalar_at(scales + (int64_t)r * (p.N >> 7) * p.KT + kb);
            const char* at = place + d * kSlot;
            wait_blocks<kCopies>(min(left, DEPTH) - 1);
            i32x8 wv[R], xv;
            float xs;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const char* a = at + r * 2048 + i * 128;
                wv[r] = operand(*reinterpret_cast<const u32x4*>(a + first_half), *reinterpret_cast<const u32x4*>(a + second_half));
            }
            if constexpr (XP > 0) {
                const int row = XP == 1 ? i & 7 : i;
                const char* a = at + R * 2048 + row * 128;
                xv = operand(*reinterpret_cast<const u32x4*>(a + ((o ^ (row >> 1)) * 16)), *reinterpret_cast<const u32x4*>(a + (((4 + o) ^ (row >> 1)) * 16)));
                xs = *reinterpret_cast<const float*>(at + R * 2048 + XP * 1024 + i * 4);
            } else {
                const char* a = staged + xrow * pitch + kb * 128 + o * 16;
                xv = operand(*reinterpret_cast<const u32x4*>(a), *reinterpret_cast<const u32x4*>(a + 64));
                xs = staged_scales[kb * rows + xrow];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                 // (the place is free)
            if (left > DEPTH) issue();
            d = d == DEPTH - 1 ? 0 : d + 1;
            const Wide x = widen(xv);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float s = xs * sw[r];
                const f32x4 codes = product(widen(wv[r]), x, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][j] = __builtin_fmaf(codes[j], s, acc[r][j]);
            }
        }

        // The wavefronts add up and store in turn.  (A set of sums is written again two row blocks later: behind a barrier that whoever reads
        // it now reaches after that.)
        f32x4* const set = sums + (rb & 1) * (waves * R * 64);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t to = lds_offset(set + (wave * R + r) * 64 + lane);
            asm volatile("ds_write_b128 %0, %1" ::"v"(to), "v"(acc[r]) : "memory");
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const bool my_turn = turn == wave;
        turn = turn == waves - 1 ? 0 : turn + 1;
        if (!my_turn) continue;
        f32x4 sum[R] = {};
        for (int v = 0; v < waves; ++v)
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] += set[(v * R + r) * 64 + lane];
        if (i >= rows) continue;
        const int64_t row = m0 + i;
        const int column = 16 * rb + 4 * o;
        if constexpr (MODE == kGated) {
            store_four(p.y + (row * p.N + column) * 2, gated(sum[0], sum[1], p.act), p.bf16);
            if (p.saved) {
                store_four(p.saved + (row * 2 * p.N + column) * 2, sum[0], p.bf16);
                store_four(p.saved + (row * 2 * p.N + p.N + column) * 2, sum[1], p.bf16);
            }
        } else {
            store_four(p.y + (row * p.N + column) * 2, sum[0], p.bf16);
        }
    }
}

// Many rows: a workgroup of GN x GM wavefronts makes tiles of Y, 16 WN GN rows of weights times 16 WM GM rows of X, each wavefront WN x WM
// blocks of sixteen by sixteen.  K goes by in steps of 128 columns, which are copied from memory into LDS without passing
// through registers; there is room for DEPTH steps, so DEPTH - 1 are under way while one is multiplied.  A step's scales come the same way.
//
// There are at most as many workgroups as run at once, and each takes one tile of Y after the other.  The copies run ahead across the
// tiles' borders: while one is finished and stored, the first steps of the next are under way.
//
// In LDS a piece is sixteen rows of 128 bytes, whole cache lines as they are read; sixteen bytes b of row i lie at 16 (b ^ (i >> 1)), so that the
// sixteen lanes that are served together hit all banks.  A lane's operand is the sixteens o and o + 4 of its row: both factors' columns are in
// the same order, which is all that the products need.
//
// Bound by the issue of instructions and by power: 8192 x 8192 x 8192 takes 435 us on a rested card and 515 in a row of calls (2.1 .. 2.5 PFLOP/s), the matrix instructions
// busy for 69 % of the cycles; exact, 4096 x 28672 x 4096, 820 .. 930 (1.0 .. 1.2), busy for 57 %.
//
// Where Y has too few tiles for the device, K is cut into slices as well.  Each slice leaves its sums in the
// workspace, and the last workgroup of a tile to finish adds them in the order of the slices.  No workgroup waits for another: the sums are
// stored past the caches that the dies do not share (sc1), complete before the workgroup counts itself, and read the same way.
template <int WN, int WM, int GN, int GM, int DEPTH, int MODE> struct TileShape {
    static constexpr int kWaves = GN * GM, kThreads = 64 * kWaves;
    static constexpr int kRB = WN * GN, kMB = WM * GM;                         // pieces of sixteen rows of either factor
    static constexpr int kBlocks = MODE == kGated ? kRB / 2 : kRB;             // row blocks of Y
    static constexpr int kStep = (kRB + kMB) * 2048;
    // Scales of a step, in pieces of 64: of the rows of X, then of the weights (kPowers: of their rows, else of their blocks).
    static constexpr int kXPieces = kMB / 4, kScalePieces = kXPieces + (MODE == kPowers ? kRB / 4 : 1);
    static constexpr int kScales = kScalePieces * 256;
    static constexpr int kLds = DEPTH * (kStep + kScales) + 16;
    static constexpr bool kSlices = WN * WM <= 8;      // (the join of slices holds four times a tile's sums)
    static constexpr int kSums = kWaves * WN * WM * 1024;                      // bytes of a tile's sums
};

template <int WN, int WM, int GN, int GM, int DEPTH, int MODE, bool GROUPED, bool EXACT>
__global__ __launch_bounds__(GN * GM * 64, 2) void tile_kernel(const ProductParams p) {
    using Shape = TileShape<WN, WM, GN, GM, DEPTH, MODE>;
    constexpr int kWaves = Shape::kWaves, kRB = Shape::kRB, kMB = Shape::kMB, kStep = Shape::kStep, kBlocks = Shape::kBlocks;
    // Copies per wavefront and step, eight rows each, and one of scales.
    constexpr int kWLoads = 2 * kRB / kWaves, kXLoads = 2 * kMB / kWaves, kScaleLoads = (Shape::kScalePieces + kWaves - 1) / kWaves;
    constexpr int kLoads = kWLoads + kXLoads + kScaleLoads;
    constexpr int kRing = WN < 4 ? WN : 4;             // row blocks of weights in registers
    constexpr int kTurn = WN - kRing + 1;              // the row block at which the next step is looked at
    // Row blocks of the next step between whose products the last copies are asked for.  With all copies asked for before that, closer together,
    // they keep the reads of LDS waiting: 4096 x 4096 x 28672 takes 436 us instead of 395, 8192 x 8192 x 8192 522 instead of 510.  (Weight
    // gradients, whose steps are shorter, take 400 instead of 411 so.)
    constexpr int kLate = WN == 8 && MODE != kPowers ? 2 : WN == 4 && WM == 4 ? 1 : 0;
    static_assert(kLate <= kTurn, "asked for before the next turn");
    constexpr int kXRing = EXACT && WM > 2 ? 2 : WM;   // of X (EXACT: until it is widened)
    constexpr bool kSpread = EXACT && kRing == 4 && WM == 4;                   // widened between the instructions: 900 us instead of 935 (4096 x 28672 x 4096)
    constexpr int kDelay = EXACT ? 1 : kWaves * WN * WM >= 256 ? 1 : 2;
    static_assert(kWLoads * kWaves == 2 * kRB && kXLoads * kWaves == 2 * kMB && kMB % 4 == 0 && kRB % 4 == 0, "whole loads per wavefront");
    static_assert(MODE != kGated || kWLoads % 2 == 0, "as many of either projection");
    extern __shared__ __align__(1024) char lds[];      // DEPTH steps, then their scales, then a word
    char* const scale_places = lds + DEPTH * kStep;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, o = lane >> 4;

    const int nx = (p.NB + kBlocks - 1) / kBlocks;
    Pieces<16 * kMB> pieces{p.offsets, p.experts, p.M};
    int slots = p.slots;
    if constexpr (GROUPED) slots = min(slots, pieces.count() - p.slot0);
    const int total = slots * nx * p.slices;           // tiles of Y, each `slices` times

    struct Item { int expert, m0, m1, rb0, tile, slice, step, steps; };        // step .. steps - 1 of the whole of K
    // The tiles of an expert (without experts: all) are ordered in bands of at most kBand pieces of rows of X, so that what a die's cache holds
    // of either factor is used several times; higher ones by expert, whose weights come from memory.
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
        it.rb0 = nt * kBlocks;
        it.step = 0;
        it.steps = p.KT;
        if (p.slices > 1) {                            // (up to 2^15 steps and eight slices: the product fits)
            it.step = quotient(it.slice * p.KT, p.slices);
            it.steps = quotient((it.slice + 1) * p.KT, p.slices);
        }
        return it;
    };

    // Where the copies are: an item, its next step, the place they go to, and this lane's byte offsets in what the wavefront copies.  Rows
    // past the end repeat the last.
    const int block = (lane & 7) ^ (lane >> 4);        // of the row that this lane copies (i >> 1 of row i = 8 c + lane / 8 is 4 (c & 1) + lane / 16)
    int number = (int)blockIdx.x, step = 0, steps = 0, place = 0;
    __amdgpu_buffer_rsrc_t wsrc, usrc, xsrc;
    const char* ssrc[kScaleLoads];                     // scales of step 0, and
    int64_t sstep[kScaleLoads];                        // bytes from one step to the next
    uint32_t wfrom[kWLoads], xfrom[kXLoads], sfrom[kScaleLoads];
    // Eight rows `c` of the weights' list, gate before others: where they lie in LDS (in pieces of eight rows).
    auto w_place = [&](int c) {
        if constexpr (MODE != kGated) return c;
        const int other = c >= kRB, b = (c - other * kRB) >> 1;                // row block of the tile, of either projection
        return 2 * (b / (WN / 2) * WN + other * (WN / 2) + b % (WN / 2)) + (c & 1);
    };
    auto aim = [&](const Item& it) {
        step = it.step;
        steps = it.steps;
        const int last_row = (p.NB - it.rb0) * 16 - 1, rows = it.m1 - it.m0;
        const char* w = p.w + it.expert * p.expert + (int64_t)it.rb0 * 16 * p.K;
        wsrc = unbounded(w);
        if constexpr (MODE == kGated) usrc = unbounded(w + (int64_t)p.N * p.K);
        xsrc = unbounded(p.x + (int64_t)it.m0 * p.K);
#pragma unroll
        for (int j = 0; j < kWLoads; ++j) {
            int c = wave + kWaves * j;
            if (MODE == kGated && j >= kWLoads / 2) c -= kRB;
            wfrom[j] = (uint32_t)min(8 * c + (lane >> 3), last_row) * (uint32_t)p.K + (block ^ (4 * (c & 1))) * 16;
        }
#pragma unroll
        for (int j = 0; j < kXLoads; ++j) {
            const int c = wave + kWaves * j;
            xfrom[j] = (uint32_t)min(8 * c + (lane >> 3), rows - 1) * (uint32_t)p.K + (block ^ (4 * (c & 1))) * 16;
        }
#pragma unroll
        for (int j = 0; j < kScaleLoads; ++j) {
            const int c = (wave + kWaves * j) % Shape::kScalePieces;           // (some are copied twice)
            if (c < Shape::kXPieces) {
                ssrc[j] = reinterpret_cast<const char*>(p.xs + it.m0);
                sstep[j] = (int64_t)p.M * 4;
                sfrom[j] = min(64 * c + lane, rows - 1) * 4;
            } else if constexpr (MODE == kPowers) {
                ssrc[j] = reinterpret_cast<const char*>(p.ws + it.rb0 * 16);
                sstep[j] = (int64_t)p.N * 4;
                sfrom[j] = min(64 * (c - Shape::kXPieces) + lane, last_row) * 4;
            } else {                                   // the first blocks from the tile's on; kGated: one of the gate's and one of the others'
                ssrc[j] = reinterpret_cast<const char*>(p.ws + it.expert * p.expert_scales + (int64_t)(it.rb0 >> 3) * p.KT);
                sstep[j] = 4;
                const int here = MODE == kGated ? min(lane, 1) * (p.N >> 7) : min(lane, min(1, (last_row >> 7)));
                sfrom[j] = (uint32_t)here * (uint32_t)p.KT * 4;
            }
        }
    };
    // Copy `j` of this wavefront's kLoads of a step.
    auto load_part = [&](int j) {
        char* to = lds + place * kStep;
        if (j < kWLoads) {
            const int c = wave + kWaves * j;
            copy16(MODE == kGated && j >= kWLoads / 2 ? usrc : wsrc, wfrom[j], step * 128, to + w_place(c) * 1024);
        } else if (j < kWLoads + kXLoads) {
            const int c = wave + kWaves * (j - kWLoads);
            copy16(xsrc, xfrom[j - kWLoads], step * 128, to + kRB * 2048 + c * 1024);
        } else {
            const int s = j - kWLoads - kXLoads, c = (wave + kWaves * s) % Shape::kScalePieces;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(unbounded(ssrc[s] + step * sstep[s]),
                (__attribute__((address_space(3))) void*)(scale_places + place * Shape::kScales + c * 256), 4, sfrom[s], 0, 0, 0);
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
    i32x8 w[kRing], x[kXRing];
    float xs[WM], ws[MODE == kGated ? 2 : 1];          // scales of the step in the registers
    uint32_t we[kRing];
    f32x4 acc[WN][WM];
    int here = 0;                                      // the place of the step being multiplied
    const char* const wplace = lds + i * 128 + wn * WN * 2048;
    const char* const xplace = lds + kRB * 2048 + i * 128 + wm * WM * 2048;
    const int first_half = (o ^ (i >> 1)) * 16, second_half = ((4 + o) ^ (i >> 1)) * 16;
    auto read = [&](const char* at) {
        return operand(*reinterpret_cast<const u32x4*>(at + first_half), *reinterpret_cast<const u32x4*>(at + second_half));
    };
    auto scale_at = [&](int from, int n) { return *reinterpret_cast<const float*>(scale_places + from * Shape::kScales + n * 4); };
    auto read_w = [&](int from, int r) {
        w[r % kRing] = read(wplace + from * kStep + r * 2048);
        if constexpr (MODE == kPowers) we[r % kRing] = __builtin_bit_cast(uint32_t, scale_at(from, Shape::kXPieces * 64 + 16 * (wn * WN + r) + i)) >> 23;
    };
    auto read_x = [&](int from, int b) { x[b % kXRing] = read(xplace + from * kStep + b * 2048); };
    auto read_scales = [&](int from) {
#pragma unroll
        for (int b = 0; b < WM; ++b) xs[b] = scale_at(from, 16 * (wm * WM + b) + i);
        if constexpr (MODE == kPlain) ws[0] = scale_at(from, Shape::kXPieces * 64 + wn * WN / 8);
        if constexpr (MODE == kGated) {
            ws[0] = scale_at(from, Shape::kXPieces * 64);
            ws[1] = scale_at(from, Shape::kXPieces * 64 + 1);
        }
    };

    // A step: row block by row block of the weights.  Its X and its first kRing - 1 row blocks are in the registers; the others, and at the end
    // the next step's, are read kRing - 1 row blocks ahead, X as soon as its last product has been started.  What an instruction
    // returns is added after kDelay more have been started.  Copies of a later step are asked for one at a time between the products.
    // (The empty statements keep the compiler from moving products and additions past each other and past what is read.)
    constexpr int kProducts = WN * WM;
    static_assert(kProducts % kDelay == 0, "a product's place is the same in every step");
    f32x4 pending[kDelay] = {};
    float pending_scale[kDelay] = {};
    auto retire = [&](int n) {                         // product n of this step, or, below 0, of the one before
        f32x4& sum = acc[(n + kProducts) % kProducts / WM][(n + kProducts) % WM];
        const int at = (n + kProducts) % kDelay;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = __builtin_fmaf(pending[at][j], pending_scale[at], sum[j]);
        asm volatile("" : "+v"(sum)::"memory");
    };
    Wide wide[EXACT ? WM : 1], wide_w[kSpread ? 2 : 1];
    // kSpread: one product, and between its four instructions the additions of the one before, a quarter of the next row block, and in turn the next
    // step's X.
    auto spread_product = [&](int r, int b) {
        f32x4 sums = {0.f, 0.f, 0.f, 0.f};
        f32x4& before = acc[(r * WM + b + kProducts - 1) % kProducts / WM][(r * WM + b + kProducts - 1) % WM];
        const int wide_x = r == WN - 1 && b > 0 ? b - 1 : r == 0 && b == 0 ? WM - 1 : -1;       // of X, widened here
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            sums = product(wide_w[r & 1], wide[b], sums, q);
            asm volatile("" : "+v"(sums)::"memory");
            float sum = __builtin_fmaf(pending[0][q], pending_scale[0], before[q]);
            asm volatile("" : "+v"(sum)::"memory");
            before[q] = sum;
            widen_pair(wide_w[(r + 1) & 1], w[(r + 1) % kRing], 4 * b + q);
            asm volatile("" : "+v"(wide_w[(r + 1) & 1].v[b])::"memory");
            if (wide_x >= 0) {
#pragma unroll
                for (int n = 0; n < 4; ++n) widen_pair(wide[wide_x], x[wide_x % kXRing], 4 * q + n);
                asm volatile("" : "+v"(wide[wide_x].v[q])::"memory");
            }
        }
        return sums;
    };
    auto one_step = [&](bool stored) {
        float s[MODE == kGated ? 2 : 1][WM];
        uint32_t xe[WM];
#pragma unroll
        for (int b = 0; b < WM; ++b) {
            if constexpr (MODE == kPowers) xe[b] = __builtin_bit_cast(uint32_t, xs[b]) >> 23;
            else {
#pragma unroll
                for (int h = 0; h < (MODE == kGated ? 2 : 1); ++h) s[h][b] = xs[b] * ws[h];
            }
        }
        const int from = here;
#pragma unroll
        for (int r = 0; r < WN; ++r) {
            if (r == kTurn) {
                next();
                here = (here + 1) % DEPTH;
                // The next step is there, and nobody needs this one's place any more.
                // (A tile's stores may be under way as well, where the copies that are waited for were asked for before them.)
                constexpr int kStores = MODE == kGated || (DEPTH == 2 && kLate > 0) ? 0 : WN / 2 * WM;
                if (stored) arrive<(DEPTH - 2) * kLoads + kStores>();
                else arrive<(DEPTH - 2) * kLoads>();
                __builtin_amdgcn_sched_barrier(0);
            }
            if (r + kRing - 1 < WN) read_w(from, r + kRing - 1);
            else read_w(here, r + kRing - 1 - WN);
            if (r == WN - 1) read_scales(here);
            auto copies = [&](int at, int places) {    // of the places after the turn's, those of one
#pragma unroll
                for (int j = at * kLoads / places; j < (at + 1) * kLoads / places; ++j) load_part(j);
            };
            if constexpr (EXACT && !kSpread) wide_w[0] = widen(w[r % kRing]);
            if constexpr (kSpread) {
                if (r == WN - 2) {
                    read_x(here, 0);
                    read_x(here, 1);
                }
            }
#pragma unroll
            for (int b = 0; b < WM; ++b) {
                const int n = r * WM + b;
                if constexpr (MODE == kPowers) {
                    acc[r][b] = scaled_product(w[r % kRing], x[b], acc[r][b], we[r % kRing], xe[b]);
                    asm volatile("" : "+v"(acc[r][b])::"memory");
                } else if constexpr (kSpread) {
                    const f32x4 sums = spread_product(r, b);
                    pending[0] = sums;
                    pending_scale[0] = s[MODE == kGated && r >= WN / 2][b];
                } else {
                    f32x4 sums = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (EXACT) sums = product(wide_w[0], wide[b], sums);
                    else sums = product(w[r % kRing], x[b], sums);
                    asm volatile("" : "+v"(sums)::"memory");
                    retire(n - kDelay);
                    pending[n % kDelay] = sums;
                    pending_scale[n % kDelay] = s[MODE == kGated && r >= WN / 2][b];
                }
                if (kSpread && r == WN - 1 && (b == 1 || b == 2)) read_x(here, b + 1);
                if (!kSpread && r == WN - 1) {
                    read_x(here, b);
                    if constexpr (EXACT) {
                        if (b > 0) wide[b - 1] = widen(x[(b - 1) % kXRing]);
                        if (b == WM - 1) wide[b] = widen(x[b % kXRing]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (r >= kTurn) copies(n - kTurn * WM, (WN - kTurn + kLate) * WM);
                else if (r < kLate) copies((WN - kTurn + r) * WM + b, (WN - kTurn + kLate) * WM);
            }
        }
    };

    // Two wavefronts share a SIMD, and the older one is served first by itself: with the younger ones preferred they drift apart, and one
    // multiplies while the other waits.
    if (kWaves == 8 && wave >= 4) __builtin_amdgcn_s_setprio(1);
    if (number >= total) return;
    Item it = item(number);
    aim(it);
#pragma unroll
    for (int t = 0; t < DEPTH; ++t) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) load_part(j);
        if (t < DEPTH - 1) next();
    }
    arrive<(DEPTH - 1) * kLoads>();
#pragma unroll
    for (int r = 0; r < kRing - 1; ++r) read_w(0, r);
#pragma unroll
    for (int b = 0; b < WM; ++b) {
        read_x(0, b);
        if constexpr (EXACT) wide[b] = widen(x[b % kXRing]);
    }
    if constexpr (kSpread) wide_w[0] = widen(w[0]);
    read_scales(0);

    bool stored = false;
    for (int mine = (int)blockIdx.x;;) {
#pragma unroll
        for (int r = 0; r < WN; ++r)
#pragma unroll
            for (int b = 0; b < WM; ++b) acc[r][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < kDelay; ++d) {
            pending[d] = f32x4{0.f, 0.f, 0.f, 0.f};
            pending_scale[d] = 0.f;
        }
        mine += (int)gridDim.x;
        int s = it.step;
        one_step(stored);
        for (++s; s < it.steps; ++s) one_step(false);
        if constexpr (MODE != kPowers) {
#pragma unroll
            for (int n = kProducts - kDelay; n < kProducts; ++n) retire(n);
        }

        bool finished = true;
        if constexpr (Shape::kSlices) if (p.slices > 1) {                      // the other slices of this tile
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
                // In the order of the slices, this one from its registers, of the others as many at a time as there are registers for.
                constexpr int kAtATime = 24 / (WN * WM);
                f32x4 sum[WN][WM] = {}, other[kAtATime][WN][WM];
                for (int z0 = 0; z0 < p.slices; z0 += kAtATime) {
#pragma unroll
                    for (int z = 0; z < kAtATime; ++z) {
                        if (z0 + z >= p.slices) continue;
#pragma unroll
                        for (int r = 0; r < WN; ++r)
#pragma unroll
                            for (int b = 0; b < WM; ++b) other[z][r][b] = load16_shared(sums, at + (r * WM + b) * 1024, (z0 + z) * Shape::kSums);
                    }
#pragma unroll
                    for (int z = 0; z < kAtATime; ++z) {
                        if (z0 + z >= p.slices) continue;
#pragma unroll
                        for (int r = 0; r < WN; ++r)
#pragma unroll
                            for (int b = 0; b < WM; ++b) sum[r][b] += z0 + z == it.slice ? acc[r][b] : other[z][r][b];
                    }
                }
#pragma unroll
                for (int r = 0; r < WN; ++r)
#pragma unroll
                    for (int b = 0; b < WM; ++b) acc[r][b] = sum[r][b];
            }
        }
        if (finished) {
#pragma unroll
            for (int b = 0; b < WM; ++b) {
                const int m = it.m0 + 16 * (wm * WM + b), rows = it.m1 - m;
                constexpr int kOut = MODE == kGated ? WN / 2 : WN;             // row blocks of Y
                const int rb = it.rb0 + wn * kOut, blocks = p.NB - rb;
                auto store = [&](auto sum, char* y, int width, int column) {
                    char* to = y + ((int64_t)m * width + column + 16 * rb) * 2;
                    if constexpr (kOut > 1) store_rows<kOut>(sum, to, rows, blocks, width, p.bf16);
                    else if (i < rows && blocks > 0) store_four(to + ((int64_t)i * width + 4 * o) * 2, sum(0), p.bf16);
                };
                if constexpr (MODE == kGated) {
                    store([&](int r) { return gated(acc[r][b], acc[r + WN / 2][b], p.act); }, p.y, p.N, 0);
                    if (p.saved) {
                        store([&](int r) { return acc[r][b]; }, p.saved, 2 * p.N, 0);
                        store([&](int r) { return acc[r + WN / 2][b]; }, p.saved, 2 * p.N, p.N);
                    }
                } else {
                    store([&](int r) { return acc[r][b]; }, p.y, p.N, 0);
                }
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

// Bytes of LDS of X that is staged, with its scales.
constexpr int64_t staged_bytes(int64_t rows, int64_t K) { return rows * (K + 16) + rows * (K / 128) * 4; }

int64_t most_pieces(const ProductParams& p, int rows) { return product::most_pieces(p.M, p.offsets ? p.experts : 0, rows); }

template <int SRC, int XP, int MODE>
hipError_t launch_stream(ProductParams p, int waves, int runs, hipStream_t s) {
    p.place_rows = XP ? 0 : p.M < 16 ? p.M : 16;
    const size_t lds = (size_t)waves * (stream_place(MODE, XP) + stream_sums(MODE)) + staged_bytes(p.place_rows, p.K);
    // (a launch has fewer than 2^16 workgroups along y and 2^32 threads)
    int64_t most = (int64_t(1) << 31) / (int64_t(runs) * waves * 64);
    most = most > 65535 ? 65535 : most;
    const int64_t slots = most_pieces(p, 16);
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < slots && e == hipSuccess; at += most) {
        p.slot0 = (int)at;
        const dim3 grid(runs, (unsigned)(slots - at < most ? slots - at : most));
        auto run = [&](auto once) {
            constexpr bool ONCE = decltype(once)::value;
            return p.offsets ? launch<stream_kernel<SRC, XP, MODE, true, ONCE>>(grid, waves * 64, lds, p, s)
                             : launch<stream_kernel<SRC, XP, MODE, false, ONCE>>(grid, waves * 64, lds, p, s);
        };
        e = p.once ? run(std::true_type()) : run(std::false_type());
    }
    return e;
}

// Output channels (kGated: of both projections) and rows of a tile, wavefronts, and steps of room, by shape.
struct TileSize { int channels, rows, waves, room; };
constexpr TileSize kTiles[] = {{256, 256, 8, 2}, {128, 128, 8, 4}, {128, 64, 8, 4}, {64, 64, 4, 4}, {256, 128, 8, 3}, {256, 192, 8, 2}};

template <int SHAPE, int WN, int WM, int GN, int GM, int DEPTH, int MODE, bool EXACT>
hipError_t launch_tiles(ProductParams p, int cus, hipStream_t s) {
    using Shape = TileShape<WN, WM, GN, GM, DEPTH, MODE>;
    static_assert(kTiles[SHAPE].channels == 16 * Shape::kRB && kTiles[SHAPE].rows == 16 * Shape::kMB && kTiles[SHAPE].waves == Shape::kWaves &&
                  kTiles[SHAPE].room == DEPTH, "as the choice knows it");
    constexpr int kAtOnce = 160 * 1024 / Shape::kLds < 8 / Shape::kWaves ? 160 * 1024 / Shape::kLds : 8 / Shape::kWaves;   // per compute unit
    static_assert(kAtOnce >= 1, "fits a compute unit");
    const int64_t nx = (p.NB + Shape::kBlocks - 1) / Shape::kBlocks, pieces = most_pieces(p, 16 * Shape::kMB);
    const int64_t most = (int64_t(1) << 30) / (nx * p.slices);                 // pieces of rows per launch: tiles are counted in 32 bits
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < pieces && e == hipSuccess; at += most) {
        p.slot0 = (int)at;
        p.slots = (int)(pieces - at < most ? pieces - at : most);
        const int64_t items = nx * p.slots * p.slices, grid = items < (int64_t)cus * kAtOnce ? items : (int64_t)cus * kAtOnce;
        const dim3 g((unsigned)grid);
        if constexpr (MODE == kPowers) e = launch<tile_kernel<WN, WM, GN, GM, DEPTH, MODE, false, EXACT>>(g, Shape::kThreads, Shape::kLds, p, s);
        else e = p.offsets ? launch<tile_kernel<WN, WM, GN, GM, DEPTH, MODE, true, EXACT>>(g, Shape::kThreads, Shape::kLds, p, s)
                           : launch<tile_kernel<WN, WM, GN, GM, DEPTH, MODE, false, EXACT>>(g, Shape::kThreads, Shape::kLds, p, s);
    }
    return e;
}

// Whether the weights are streamed past sixteen rows at a time, or which tile shape, and for the smaller ones how many slices of K: the least
// of times that are estimated, in microseconds, from the bytes of weights over the pieces of rows (B), or from the rounds of tiles (n, for two small tiles
// at once on a unit the number on the busiest) and of steps of 128 columns (S; 1.8 of them for each of the exact sums'):
//   streamed    4.1 + B / 5.8 TB/s (by expert 4, gated 10 from the caches)   256 x 256   4.8 + n (1.52 S + 5.6)         256 x 128   2.8 + n (0.88 S + 2.9)
//   256 x 192   4.8 + n (1.19 S + 4.5)      128 x 128   3.9 + n (0.57 S + 1.4)      128 x 64    3.25 + n (0.428 S + 0.7)       64 x 64     2.25 + n (0.374 S + 0.9), two at once 0.7 S + 0.9
// and for z slices, each of S / z steps, 5.0 + 0.75 z, 3.6 + 0.75 z and 3.0 + 0.45 z more for storing and joining sums.  The constants are least squares
// over 228 drawn calls of every shape, corrected on others; on those the best choice was 1 .. 3 % faster on average, by expert 6 %.  Examples, us (weights from
// memory): 1594 rows, 288 x 13824: 64 x 64 in four slices 21.3, 128 x 128 in six (taken) 24.2, 256 x 128 82; 2048 rows gated, 27648 x 5120: 256 x 256
// (taken) 296, 256 x 128 330; 1751 rows, 5120 x 2944, where tiles of 256 x 256 are 140 for 256 units: 256 x 192 (taken) 32.8, 256 x 256 37.5, 256 x 128 45; 33 rows gated, 2304 x 4224: streamed (taken) 7.2, 64 x 64 in three slices 10.8; 224 rows of 14 experts, 9008 x 1920: streamed 89,
// tiles (taken) 52.
struct TileChoice { int shape, slices; };             // shape -1: streamed

// `NB`: row blocks of weights, kGated: of both projections.
TileChoice choose_tiles(int64_t M, int64_t NB, int64_t KT, int64_t experts, int mode, bool exact, int cus) {
    const double S = (double)KT * (exact ? 1.8 : 1.0);
    TileChoice best{-1, 1};
    auto tiles = [&](int64_t rb, int64_t rows) {
        const int64_t nx = (NB + rb - 1) / rb;
        if (!experts) return (double)nx * (double)((M + rows - 1) / rows);
        const double some = (double)(M < experts ? M : experts), filled = (double)M / (double)rows + 0.5 * some;
        return (double)nx * (filled > some ? filled : some);
    };
    if (mode != kPowers && M <= (experts ? 4 * experts : 16)) return best;
    // (What is read again comes from the second caches where they hold it; of the gated call, whose X goes as far for twice the weights, twice as fast.)
    const double rate = experts ? 4.0e6 : mode == kGated && NB * KT * 2048 <= (int64_t(32) << 20) ? 10.0e6 : 5.8e6;
    double least = mode == kPowers ? 1e30 : 4.1 + tiles(1, 16) * (double)KT * 2048.0 / rate;
    auto consider = [&](int shape, int slices, double us) {
        if (us < least) { least = us; best = {shape, slices}; }
    };
    // Rounds of tiles: by expert, where they may be more or fewer than is estimated, on average; else rounded up, but for a part: the units that have
    // a tile in an uneven last round have more of the memory and of the power to themselves.
    auto rounds = [&](double t) {
        const double exact_rounds = t / cus, up = (double)(int64_t)((t + cus - 1) / cus);
        if (experts) return exact_rounds < 0.6 ? 1.0 : exact_rounds + 0.4;
        return up < 2.0 ? up : 0.8 * up + 0.2 * exact_rounds;
    };
    auto pairs = [&](double n, double one, double two) { return two * (double)(int64_t)(n / 2) + ((int64_t)n % 2 ? one : 0.0); };
    const double t0 = tiles(16, 256), t1 = tiles(8, 128), t2 = tiles(8, 64), t3 = tiles(4, 64), t4 = tiles(16, 128), t5 = tiles(16, 192);
    if (!exact) consider(0, 1, 4.8 + rounds(t0) * (1.52 * S + 5.6 * (t0 < cus ? t0 / cus : 1.0)));
    if (!exact) consider(5, 1, 4.8 + rounds(t5) * (1.19 * S + 4.5 * (t5 < cus ? t5 / cus : 1.0)));
    consider(4, 1, 2.8 + rounds(t4) * (0.88 * S + 2.9));
    const double most = (experts ? 0.7 : 1.0) * cus;   // slices that run at once
    for (int z = 1; z <= 8; ++z) {
        if (z > KT) break;
        const double steps = z > 1 ? (double)((int64_t)((S + z - 1) / z)) : S;
        if (z == 1 || t1 * z <= most) consider(1, z, 3.9 + rounds(t1 * z) * (0.57 * steps + 1.4) + (z > 1 ? 5.0 + 0.75 * z : 0.0));
        if (z == 1 || t2 * z <= most) consider(2, z, 3.25 + rounds(t2 * z) * (0.428 * steps + 0.7) + (z > 1 ? 3.6 + 0.75 * z : 0.0));
        if (z == 1 || t3 * z <= 2 * most) {
            const double n = (double)(int64_t)((t3 * z + cus - 1) / cus);
            consider(3, z, 2.25 + pairs(n, 0.374 * steps + 0.9, 0.7 * steps + 0.9) + (z > 1 ? 3.0 + 0.45 * z : 0.0));
        }
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
    int pieces;                // of eight rows of X that come with them, 0: X is quantised into LDS
    int waves;                 // per workgroup
    int runs;                  // of row blocks, one per workgroup
};

// `experts`: 0 without.
Choice choose(int64_t M, int64_t NB, int64_t KT, int64_t experts, int mode, bool exact, bool codes, int cus) {
    Choice c{};
    c.tiles = choose_tiles(M, NB, KT, experts, mode, exact, cus);
    const int64_t pieces = experts ? (M < experts ? M : experts) : (M + 15) / 16, mean = (M + pieces - 1) / pieces;
    const int64_t blocks = mode == kGated ? NB / 2 : NB, most_rows = M < 16 ? M : 16, staged = staged_bytes(most_rows, KT * 128);
    constexpr int64_t kLds = 160 * 1024, kStagedMost = 72 * 1024, kStagedFew = 20 * 1024;
    // Values of up to four rows, or of up to 20 KiB of codes, are quantised by every workgroup for itself, at the cost of LDS for fewer wavefronts; others
    // once, by a launch of some 2 us.  (7 rows of 640, 336 channels: 0.77 of the time; 13 of 896, 10896 channels 0.92; against 13 of 8960: 1.2 times; by
    // expert with up to four rows on average 0.75 .. 1.2.)  Codes come with the weights: 16 rows of 640, 752 channels 4.3 us, in LDS 5.2.
    const bool into_lds = !codes && c.tiles.shape < 0 && (mean <= 4 || most_rows * KT * 128 <= kStagedFew) && staged <= kStagedMost;
    c.apart = !codes && !into_lds;
    // Past the caches from 40 MiB on, for matrices of which one follows the other: 2 rows, 20224 x 4352, 20.5 us, past them 17.7; below 30 MiB they do
    // not gain (1536 channels of 9856: 12.0 us and 14.1).
    c.once = c.tiles.shape < 0 && (experts ? mean <= 16 : M <= 16) && NB * (experts ? pieces : 1) * KT * 2048 > (int64_t(40) << 20);
    c.pieces = into_lds ? 0 : most_rows > 8 ? 2 : 1;
    const int64_t per_wave = stream_place(mode, c.pieces) + stream_sums(mode), shared = c.pieces ? 0 : staged;
    // A row block's K is shared by as few wavefronts as leave all of them with work: each sum through LDS costs a barrier.  By expert, 14 rows of 18,
    // 3200 x 7808: eight 51.9 us, four 37.9, two 39.0; two of 5, 9984 x 11264: 150, 127, 114; 768 channels of 9856 (48 row blocks): 11.8, 13.6, 20.3.
    // Values of one row, 6144 x 4096: eight 7.5, four 6.9; 640 x 9984: 9.5, 12.0.
    const int64_t all = blocks * pieces, most_waves = into_lds ? (KT <= (experts ? 16 : 32) && all >= cus ? 4 : kStreamWaves) : all < cus ? kStreamWaves : experts && all >= 2 * cus ? 2 : 4;
    int64_t waves = KT < most_waves ? KT : most_waves;
    while (waves > 1 && waves * per_wave + shared > kLds) --waves;
    int64_t at_once = kLds / (waves * per_wave + shared);                      // workgroups per compute unit
    if (at_once > 32 / waves) at_once = 32 / waves;
    const int64_t runs = (cus * at_once + pieces - 1) / pieces;
    c.runs = (int)(runs < blocks ? runs : blocks);
    c.waves = (int)waves;
    return c;
}

template <int MODE> hipError_t launch_stream_of(int src, const Choice& c, const ProductParams& p, hipStream_t s) {
    if (c.pieces == 1) return launch_stream<kF32, 1, MODE>(p, c.waves, c.runs, s);
    if (c.pieces == 2) return launch_stream<kF32, 2, MODE>(p, c.waves, c.runs, s);
    return src == kF16 ? launch_stream<kF16, 0, MODE>(p, c.waves, c.runs, s) : launch_stream<kBF16, 0, MODE>(p, c.waves, c.runs, s);
}

template <int MODE, bool EXACT = false> hipError_t launch_of(const Choice& c, int src, const ProductParams& p, int cus, hipStream_t s) {
    switch (c.tiles.shape) {
        case 0:
            if constexpr (!EXACT) return launch_tiles<0, 8, 4, 2, 4, 2, MODE, EXACT>(p, cus, s);
            return hipErrorInvalidValue;
        case 1: return launch_tiles<1, 4, 2, 2, 4, 4, MODE, EXACT>(p, cus, s);
        case 2: return launch_tiles<2, 2, 2, 4, 2, 4, MODE, EXACT>(p, cus, s);
        case 3: return launch_tiles<3, 2, 2, 2, 2, 4, MODE, EXACT>(p, cus, s);
        case 4: return launch_tiles<4, 4, 4, 4, 2, 3, MODE, EXACT>(p, cus, s);
        case 5:
            if constexpr (!EXACT) return launch_tiles<5, 8, 3, 2, 4, 2, MODE, EXACT>(p, cus, s);
            return hipErrorInvalidValue;
    }
    if constexpr (MODE != kPowers) return launch_stream_of<MODE>(src, c, p, s);
    return hipErrorInvalidValue;
}

// Bytes of the products' scratch before what a gated call adds; 0 if unsupported.
size_t scratch_bytes(int64_t M, int64_t K) { return kCounterBytes + kPartialBytes + up256((size_t)M * (size_t)K) + up256((size_t)M * (size_t)(K / 128) * 4); }

// What the entry points have in common.  N: columns of Y.
struct Call {
    const void* x; const float* xs; const void* w; const float* ws; const int32_t* offsets; int64_t experts;
    int64_t M, N, K; lutq_dtype dtype; void* y; void* saved; void* h_codes; float* h_scales; int mode, act;
    void* workspace; size_t workspace_bytes, needed;
    bool by_expert;
};

lutq_status product_on(const Call& a, hipStream_t s) {
    if (a.needed == 0) return LUTQ_ERR_SHAPE;
    if ((a.dtype != LUTQ_F16 && a.dtype != LUTQ_BF16) || (a.mode == kGated && a.act != LUTQ_SILU && a.act != LUTQ_GELU)) return LUTQ_ERR_DTYPE;
    if (a.M == 0) return LUTQ_OK;
    if (!a.x || !a.w || !a.ws || (!a.y && !a.h_codes) || !a.h_codes != !a.h_scales || (a.by_expert && !a.offsets)) return LUTQ_ERR_NULL;
    if (!aligned(a.x, 16) || !aligned(a.xs, 4) || !aligned(a.w, 16) || !aligned(a.ws, 4) || !aligned(a.y, 16) || !aligned(a.saved, 16) ||
        !aligned(a.h_codes, 16) || !aligned(a.h_scales, 4) || !aligned(a.workspace, 16) || !aligned(a.offsets, 4))
        return LUTQ_ERR_ALIGN;
    if (!a.workspace || a.workspace_bytes < a.needed) return LUTQ_ERR_WORKSPACE;

    ProductParams p{};
    const int64_t w_rows = a.mode == kGated ? 2 * a.N : a.N;
    p.x = static_cast<const char*>(a.x); p.xs = a.xs;
    p.w = static_cast<const char*>(a.w); p.ws = a.ws;
    p.offsets = a.by_expert ? a.offsets : nullptr; p.experts = (int)a.experts;
    p.expert = w_rows * a.K; p.expert_scales = (w_rows + 127) / 128 * (a.K / 128);
    p.M = (int)a.M; p.N = (int)a.N; p.K = (int)a.K; p.KT = (int)(a.K / 128); p.NB = (int)(a.N / 16);
    p.bf16 = a.dtype == LUTQ_BF16; p.act = a.act;
    p.counters = static_cast<uint32_t*>(a.workspace);
    p.partial = static_cast<char*>(a.workspace) + kCounterBytes;
    char* const codes = p.partial + kPartialBytes;
    float* const scales = reinterpret_cast<float*>(codes + up256((size_t)a.M * a.K));
    char* const dense = reinterpret_cast<char*>(scales) + up256((size_t)a.M * (a.K / 128) * 4);
    p.y = a.y ? static_cast<char*>(a.y) : dense; p.saved = static_cast<char*>(a.saved);
    int src = a.xs ? kF32 : a.dtype == LUTQ_F16 ? kF16 : kBF16;
    const int cus = compute_units();
    if (cus < 1) return LUTQ_ERR_DEVICE;
    // What is kept for gradients or quantised is summed exactly: a last bit there becomes a whole step of a code in what is made of it.
    const bool exact = a.saved || a.h_codes;
    const Choice c = choose(a.M, w_rows / 16, p.KT, p.offsets ? a.experts : 0, a.mode, exact, a.xs != nullptr, cus);
    if (c.apart) {
        const lutq_status st = quantize_rows_on(a.x, src, a.M, nullptr, nullptr, 0, a.M, a.K, codes, scales, s);
        if (st != LUTQ_OK) return st;
        p.x = codes; p.xs = scales;
        src = kF32;
    }
    p.once = c.once;
    p.slices = c.tiles.slices;
    const hipError_t e = a.mode == kPowers  ? launch_of<kPowers>(c, src, p, cus, s)
                         : a.mode == kPlain ? launch_of<kPlain>(c, src, p, cus, s)
                         : exact            ? launch_of<kGated, true>(c, src, p, cus, s)
                                            : launch_of<kGated>(c, src, p, cus, s);
    if (e != hipSuccess) return LUTQ_ERR_DEVICE;
    if (!a.h_codes) return LUTQ_OK;
    return quantize_rows_on(p.y, a.dtype == LUTQ_F16 ? kF16 : kBF16, a.M, nullptr, p.offsets, a.experts, a.M, a.N, a.h_codes, a.h_scales, s);
}

bool experts_ok(int64_t experts) { return experts >= 1 && experts <= 65536; }

}  // namespace

}  // namespace fp8
}  // namespace lutq

using namespace lutq::fp8;

extern "C" size_t lutq_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts) {
    if (!shape_ok(N, K) || !rows_ok(M, K) || !experts_ok(experts)) return 0;
    return scratch_bytes(M, K);
}

extern "C" size_t lutq_fp8_gated_workspace_bytes(int64_t M, int64_t F, int64_t K, int64_t experts) {
    if (F < 1 || F % 128 != 0 || F > kMostColumns / 2 || !shape_ok(2 * F, K) || !rows_ok(M, K) || !rows_ok(M, 2 * F) || !experts_ok(experts)) return 0;
    return scratch_bytes(M, K) + lutq::product::up256((size_t)M * (size_t)F * 2);
}

extern "C" lutq_status lutq_fp8_matmul(const void* X, const float* x_scales, const void* W, const float* w_scales, int64_t M, int64_t N, int64_t K,
                                       lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, void* stream) {
    return product_on({X, x_scales, W, w_scales, nullptr, 1, M, N, K, dtype, Y, nullptr, nullptr, nullptr, kPlain, 0, workspace, workspace_bytes,
                       lutq_fp8_workspace_bytes(M, N, K, 1), false}, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_fp8_matmul_grouped(const void* X, const float* x_scales, const void* W, const float* w_scales, const int32_t* offsets,
                                               int64_t experts, int64_t M, int64_t N, int64_t K, lutq_dtype dtype, void* Y, void* workspace,
                                               size_t workspace_bytes, void* stream) {
    return product_on({X, x_scales, W, w_scales, offsets, experts, M, N, K, dtype, Y, nullptr, nullptr, nullptr, kPlain, 0, workspace, workspace_bytes,
                       lutq_fp8_workspace_bytes(M, N, K, experts), true}, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_fp8_gated(const void* X, const float* x_scales, const void* W, const float* w_scales, int64_t M, int64_t F, int64_t K,
                                      lutq_activation activation, lutq_dtype dtype, void* H, void* h_codes, float* h_scales, void* saved,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    return product_on({X, x_scales, W, w_scales, nullptr, 1, M, F, K, dtype, H, saved, h_codes, h_scales, kGated, activation, workspace, workspace_bytes,
                       lutq_fp8_gated_workspace_bytes(M, F, K, 1), false}, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_fp8_gated_grouped(const void* X, const float* x_scales, const void* W, const float* w_scales, const int32_t* offsets,
                                              int64_t experts, int64_t M, int64_t F, int64_t K, lutq_activation activation, lutq_dtype dtype, void* H,
                                              void* h_codes, float* h_scales, void* saved, void* workspace, size_t workspace_bytes, void* stream) {
    return product_on({X, x_scales, W, w_scales, offsets, experts, M, F, K, dtype, H, saved, h_codes, h_scales, kGated, activation, workspace,
                       workspace_bytes, lutq_fp8_gated_workspace_bytes(M, F, K, experts), true}, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_fp8_weight_grad(const void* dY, const float* dy_scales, const void* X, const float* x_scales, int64_t N, int64_t K, int64_t M,
                                            lutq_dtype dtype, void* dW, void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 1 || M % 128 != 0 || N < 1 || N % 16 != 0) return LUTQ_ERR_SHAPE;
    if (!dy_scales) return LUTQ_ERR_NULL;
    return product_on({dY, dy_scales, X, x_scales, nullptr, 1, N, K, M, dtype, dW, nullptr, nullptr, nullptr, kPowers, 0, workspace, workspace_bytes,
                       lutq_fp8_workspace_bytes(N, K, M, 1), false}, static_cast<hipStream_t>(stream));
}

extern "C" int lutq_calib_fp8_launch(int64_t M, int64_t N, int64_t K, int64_t experts, int form, int x_is_codes, int compute_units, int* launch) {
    if (!launch) return LUTQ_ERR_NULL;
    constexpr int kExact = 3;
    const bool gate = form == kGated || form == kExact;
    if (form < 0 || form > 3 || experts < 0 || M < 1 || compute_units < 1 || compute_units > 4096 || (form == kPowers && (experts || !x_is_codes)) ||
        (gate ? lutq_fp8_gated_workspace_bytes(M, N, K, experts ? experts : 1) : lutq_fp8_workspace_bytes(M, N, K, experts ? experts : 1)) == 0)
        return LUTQ_ERR_SHAPE;
    const Choice c = choose(M, N / 16 * (gate ? 2 : 1), K / 128, experts, form == kExact ? kGated : form, form == kExact, x_is_codes != 0, compute_units);
    const bool streamed = c.tiles.shape < 0;
    const TileSize t = streamed ? TileSize{gate ? 32 : 16, 16, c.waves, stream_depth(gate ? kGated : kPlain)} : kTiles[c.tiles.shape];
    const int out[8] = {c.apart, t.channels, t.rows, t.waves, t.room, c.tiles.slices, streamed ? 1 + c.pieces : 0, c.once};
    for (int i = 0; i < 8; ++i) launch[i] = out[i];
    return LUTQ_OK;
}
