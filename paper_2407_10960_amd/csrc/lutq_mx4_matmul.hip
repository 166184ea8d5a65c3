// Products of the microscaled 4-bit form (include/lutq.h): Y = X W^T and the same by expert, on the scaled matrix instruction
// v_mfma_scale_f32_16x16x128_f8f6f4, which takes 128 columns of sixteen rows of either factor and their exponents as they are held.
//
// The instruction's first operand is the weights, so a lane's four sums are neighbours in a row of Y.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lutq.h"
#include "lutq_layout.hpp"
#include "lutq_mx4_device.hpp"

namespace lutq {
namespace mx4 {

lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, int64_t M, int64_t K,
                             void* codes, void* exponents, hipStream_t stream);

// Sixteen bytes per lane from memory to LDS, where lane l's go to `to` + 16 l.
__device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t from, uint32_t lane_at, int at, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_at, at, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t unbounded(const char* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (uint32_t)-1, 0x00020000);
}

struct ProductParams {
    const char* x;             // row form: codes; or 16-bit values
    const char* xe;            // row form: exponents
    const char* w;             // records
    char* y;
    const int32_t* offsets;    // by expert: experts + 1; else null
    int64_t record, expert;    // bytes of a row block's record, of an expert's weights
    int M, N, K, KT, KQ, NB;   // K tiles, quads, row blocks
    int experts;
    int slot0, slots;          // first piece of rows of this launch, and how many
    int bf16;                  // type of Y
};

// Rows [first, end) of X and the expert of the `slot`-th piece of ROWS rows: pieces do not straddle experts and are numbered in order of
// the experts.  False where there are fewer pieces.  Every lane of a wavefront looks at one expert at a time; the whole
// wavefront gets the answer.
template <int ROWS>
__device__ __forceinline__ bool find_piece(const int32_t* offsets, int experts, int M, int slot, int& expert, int& first, int& end) {
    const int lane = threadIdx.x & 63;
    int before = 0;                                    // pieces of the experts looked at so far
    for (int base = 0; base < experts; base += 64) {
        const int g = base + lane;
        int a = 0, b = 0;
        if (g < experts) {
            a = min(max(offsets[g], 0), M);
            b = min(max(offsets[g + 1], 0), M);
        }
        const int mine = b > a ? (b - a + ROWS - 1) / ROWS : 0;
        int sum = mine;                                // inclusive prefix sum over the wavefront
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const uint64_t past = __ballot(before + sum > slot);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int begin = __shfl(before + sum - mine, at);
            expert = __builtin_amdgcn_readfirstlane(base + at);
            first = __builtin_amdgcn_readfirstlane(__shfl(a, at) + (slot - begin) * ROWS);
            end = __builtin_amdgcn_readfirstlane(min(__shfl(b, at), first + ROWS));
            return true;
        }
        before += __builtin_amdgcn_readfirstlane(__shfl(sum, 63));
    }
    return false;
}

// Few rows: a workgroup owns R row blocks of weights and MB blocks of sixteen rows of X over all of K; its wavefronts take the
// quads in turn, and their sums are added in LDS in the order of the wavefronts.  Both factors go from memory into
// the operand registers: the weights as they lie, X by rows (SRC 0), or 16-bit values whose blocks of 32, one per lane, are quantised there.
template <int SRC, int R, int MB, bool GROUPED>
__global__ __launch_bounds__(512) void stream_kernel(const ProductParams p) {
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, i = lane & 15, o = lane >> 4;
    const int slot = p.slot0 + (int)blockIdx.y;
    int expert = 0, m0 = slot * 16 * MB, m1 = min(p.M, m0 + 16 * MB);
    if (GROUPED && !find_piece<16 * MB>(p.offsets, p.experts, p.M, slot, expert, m0, m1)) return;
    const int rb0 = (int)blockIdx.x * R;
    const char* w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = p.w + expert * p.expert + min(rb0 + r, p.NB - 1) * p.record;
    int64_t row[MB];                                   // (rows past the end repeat the last: their sums are not stored)
#pragma unroll
    for (int b = 0; b < MB; ++b) row[b] = min(m0 + 16 * b + i, m1 - 1);

    f32x4 acc[R][MB] = {};
    for (int q = wave; q < p.KQ; q += waves) {
        const int tiles = min(4, p.KT - 4 * q);
        uint32_t we[R];
        u32x4 wv[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            we[r] = *reinterpret_cast<const uint32_t*>(w[r] + (int64_t)p.KT * 1024 + q * 256 + lane * 4);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                wv[r][t] = *reinterpret_cast<const u32x4*>(w[r] + (int64_t)(4 * q + min(t, tiles - 1)) * 1024 + lane * 16);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t >= tiles) break;
            const int64_t block = (int64_t)(4 * q + t) * 4 + o;
            u32x4 xv[MB];
            uint32_t xe[MB];
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                if constexpr (SRC == kF32) {           // (the row form)
                    xv[b] = *reinterpret_cast<const u32x4*>(p.x + row[b] * (p.K / 2) + block * 16);
                    xe[b] = *reinterpret_cast<const uint8_t*>(p.xe + row[b] * (p.K / 32) + block);
                } else {
                    const u32x4* from = reinterpret_cast<const u32x4*>(p.x + (row[b] * p.K + block * 32) * 2);
                    Eight<SRC> v[4];
                    uint32_t a = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j].v[0] = from[j];
#pragma unroll
                    for (int j = 0; j < 16; ++j) max_bits<SRC>(v[j / 4].v[0][j % 4], a);
                    xe[b] = exponent_byte<SRC>(a);     // (255 makes the products NaN whatever the codes)
#pragma unroll
                    for (int j = 0; j < 4; ++j) xv[b][j] = to_codes<SRC>(v[j], power_of(xe[b]));
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    if (t == 0) acc[r][b] = product<0, 0>(wv[r][0], xv[b], acc[r][b], we[r], xe[b]);
                    if (t == 1) acc[r][b] = product<1, 0>(wv[r][1], xv[b], acc[r][b], we[r], xe[b]);
                    if (t == 2) acc[r][b] = product<2, 0>(wv[r][2], xv[b], acc[r][b], we[r], xe[b]);
                    if (t == 3) acc[r][b] = product<3, 0>(wv[r][3], xv[b], acc[r][b], we[r], xe[b]);
                }
        }
    }

    f32x4* sums = reinterpret_cast<f32x4*>(smem);      // [wave][row block, block of X][lane]
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int b = 0; b < MB; ++b) sums[(wave * R * MB + r * MB + b) * 64 + lane] = acc[r][b];
    __syncthreads();
    for (int d = wave; d < R * MB; d += waves) {
        f32x4 s = sums[d * 64 + lane];
        for (int v = 1; v < waves; ++v) s += sums[(v * R * MB + d) * 64 + lane];
        const int m = m0 + 16 * (d % MB) + i, rb = rb0 + d / MB;
        if (m < m1 && rb < p.NB) {
            const u32x2 out = {round_pair(s[0], s[1], p.bf16), round_pair(s[2], s[3], p.bf16)};
            *reinterpret_cast<u32x2*>(p.y + ((int64_t)m * p.N + 16 * rb + 4 * o) * 2) = out;
        }
    }
}

// Waits until at most N of this wavefront's global loads are under way and all its LDS reads are done, then for the workgroup.
template <int N> __device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

// Many rows: a workgroup of GN x GM wavefronts owns 16 WN GN rows of weights times 16 WM GM rows of X, each wavefront WN x WM blocks of
// sixteen by sixteen.  K goes by in steps of two tiles (256 columns), which are copied from memory into LDS without passing through
// registers; two steps fit, so one is under way while the other is multiplied.  The operands of one tile are read from LDS while the matrix
// instructions of the tile before run.  The exponents come the same way, a quad (two steps) at a time.  K >= 512.
//
// In LDS the weights lie as in memory, in operand order.  Of X a piece is sixteen rows of 128 bytes, whole cache lines as they are
// read (a line asked for in halves, a step apart, was fetched twice); block b of row i lies at 16 (b ^ (i >> 1)), so that the
// sixteen lanes that are served together hit all banks.
template <int WN, int WM, int GN, int GM, bool GROUPED>
__global__ __launch_bounds__(GN * GM * 64, 2) void tile_kernel(const ProductParams p) {
    constexpr int kWaves = GN * GM, kRB = WN * GN, kMB = WM * GM;              // pieces of sixteen rows of either factor
    constexpr int kWLoads = kRB / kWaves, kXLoads = 2 * kMB / kWaves;          // per wavefront: pieces of weights, halves of pieces of X
    constexpr int kLoads = 2 * kWLoads + kXLoads;
    constexpr int kExpPieces = (kRB + kMB) / 4, kExpLoads = (kExpPieces + kWaves - 1) / kWaves;
    static_assert(kRB % kWaves == 0 && 2 * kMB % kWaves == 0 && kRB % 4 == 0 && kMB % 4 == 0, "whole loads per wavefront");
    constexpr int kStep = (kRB + kMB) * 2048, kExps = (kRB + kMB) * 256;
    __shared__ __align__(1024) char lds[2 * kStep + kExps];
    using std::integral_constant;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, o = lane >> 4;

    // Workgroups go to the eight dies in turn: each die gets a run of consecutive tiles of Y, ordered in bands of kBand pieces of rows
    // of X, so that what its cache holds of either factor is used several times.
    constexpr int kBand = 4;
    const int nx = (p.NB + kRB - 1) / kRB, per = (int)(gridDim.x >> 3);
    int id = (int)blockIdx.x;
    if (id < per * 8) id = (id & 7) * per + (id >> 3);
    const int band = id / (kBand * nx), inside = id - band * kBand * nx;
    const int high = min(kBand, p.slots - band * kBand);
    const int nt = inside / high, slot = p.slot0 + band * kBand + (inside - nt * high);
    int expert = 0, m0 = slot * 16 * kMB, m1 = min(p.M, m0 + 16 * kMB);
    if (GROUPED && !find_piece<16 * kMB>(p.offsets, p.experts, p.M, slot, expert, m0, m1)) return;
    const int rb0 = nt * kRB, rows = m1 - m0;

    // Byte offsets of this lane in what the wavefront copies.  Rows and row blocks past the end repeat the last.
    const int last_rb = p.NB - 1 - rb0, half = p.K / 2, ebytes = p.K / 32;
    const auto wsrc = unbounded(p.w + expert * p.expert + rb0 * p.record);
    const auto xsrc = unbounded(p.x + (int64_t)m0 * half);
    const auto esrc = unbounded(p.xe + (int64_t)m0 * ebytes);
    const int block = (lane & 7) ^ (lane >> 4);        // of the row that this lane copies (i >> 1 of row i = 8 g + lane / 8 is 4 g + lane / 16)
    uint32_t wfrom[kWLoads], xfrom[kXLoads], efrom[kExpLoads];
#pragma unroll
    for (int j = 0; j < kWLoads; ++j) wfrom[j] = (uint32_t)min(wave + kWaves * j, last_rb) * (uint32_t)p.record + lane * 16;
#pragma unroll
    for (int j = 0; j < kXLoads; ++j) {
        const int c = wave + kWaves * j;               // eight rows
        xfrom[j] = (uint32_t)min(8 * c + (lane >> 3), rows - 1) * (uint32_t)half + (block ^ (4 * (c & 1))) * 16;
    }
#pragma unroll
    for (int j = 0; j < kExpLoads; ++j) {
        const int c = min(wave + kWaves * j, kExpPieces - 1);                  // (the last may be copied twice)
        efrom[j] = c < kRB / 4 ? (uint32_t)min(4 * c + o, last_rb) * (uint32_t)p.record + (uint32_t)p.KT * 1024 + i * 16
                               : (uint32_t)min(64 * (c - kRB / 4) + lane, rows - 1) * (uint32_t)ebytes;
    }
    // Copy `j` of this wavefront's kLoads of a step.
    auto load_part = [&](int step, int buffer, int j) {
        char* to = lds + buffer * kStep;
        // An odd last step has one tile: the second is the first again, so that nothing behind the rows is touched, and
        // has exponents of zero on both sides, 2^-254 for their products, which adds nothing to an fp32 sum.
        const bool whole = 2 * step + 1 < p.KT;
        if (j < 2 * kWLoads) {
            const int c = wave + kWaves * (j >> 1), second = j & 1;
            copy16(wsrc, wfrom[j >> 1], step * 2048 + (second && whole ? 1024 : 0), to + c * 2048 + second * 1024);
        } else {
            const int c = wave + kWaves * (j - 2 * kWLoads);
            const uint32_t at = xfrom[j - 2 * kWLoads], from = whole ? at : at - ((block ^ (4 * (c & 1))) & 4) * 16;
            copy16(xsrc, from, step * 128, to + kRB * 2048 + c * 1024);
        }
    };
    auto load_step = [&](int step, int buffer) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) load_part(step, buffer, j);
    };
    // Exponents of a quad: of a row block of weights its 256 bytes, of a row of X its sixteen.  The row's last quad may be short: the
    // sixteen bytes that end with the row are taken then, so that no byte behind X is touched.
    auto load_exps = [&](int q) {
        char* to = lds + 2 * kStep;
#pragma unroll
        for (int j = 0; j < kExpLoads; ++j) {
            const int c = min(wave + kWaves * j, kExpPieces - 1);
            if (c < kRB / 4) copy16(wsrc, efrom[j], q * 256, to + c * 1024);
            else copy16(esrc, efrom[j], min(q * 16, ebytes - 16), to + c * 1024);
        }
    };

    const int wn = wave % GN, wm = wave / GN;
    u32x4 w[WN], x[2][WM];
    uint32_t we[WN], xe[WM];
    f32x4 acc[WN][WM] = {};
    const char* const wplace = lds + lane * 16 + wn * WN * 2048;
    const char* const xplace = lds + kRB * 2048 + i * 128 + wm * WM * 2048;
    const int xblock[2] = {(o ^ (i >> 1)) * 16, ((4 + o) ^ (i >> 1)) * 16};
    auto read_w = [&](int buffer, int h, int r) { w[r] = *reinterpret_cast<const u32x4*>(wplace + buffer * kStep + h * 1024 + r * 2048); };
    auto read_x = [&](int buffer, int h) {
#pragma unroll
        for (int b = 0; b < WM; ++b) x[h][b] = *reinterpret_cast<const u32x4*>(xplace + xblock[h] + buffer * kStep + b * 2048);
    };
    // A lane's word of exponents has the quad's tiles in its four bytes.  That is how the weights' lie; of X, word t of a row holds the
    // four blocks of tile t, of which this lane needs block o.
    auto read_exps = [&](int q) {
        const char* at = lds + 2 * kStep;
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
    // The tile in the registers, half H of its step; the next one (half 1 - H, in `buffer`) is read meanwhile: of X into registers of
    // their own, of a row block of weights when its last product has been started.  Copies of a later step are asked for one at a
    // time between the products: together, they would keep the wavefronts from issuing anything else for a thousand cycles.
    auto multiply = [&](auto half_of_step, int buffer, auto part) {
        constexpr int H = decltype(half_of_step)::value;
        read_x(buffer, 1 - H);
#pragma unroll
        for (int r = 0; r < WN; ++r) {
#pragma unroll
            for (int b = 0; b < WM; ++b) acc[r][b] = product<H, H>(w[r], x[H][b], acc[r][b], we[r], xe[b]);
            // (without this the compiler moves products behind the branches and barriers that follow)
#pragma unroll
            for (int b = 0; b < WM; ++b) asm volatile("" : "+v"(acc[r][b]));
            __builtin_amdgcn_sched_barrier(0);
            read_w(buffer, 1 - H, r);
            part(r);
        }
    };
    // Step s; its first tile is in the registers.  LOAD: there is a step s + 2.
    auto one_step = [&](int s, auto load) {
        constexpr bool LOAD = decltype(load)::value;
        const int here = s & 1;
        multiply(integral_constant<int, 0>(), here, [](int) {});
        arrive<0>();                                   // the next step is there, and nobody needs this one's place any more
        __builtin_amdgcn_sched_barrier(0);
        if (LOAD && here == 0) load_exps(s / 2 + 1);
        multiply(integral_constant<int, 1>(), 1 - here, [&](int r) {
            if constexpr (LOAD) {
#pragma unroll
                for (int j = r * kLoads / WN; j < (r + 1) * kLoads / WN; ++j) load_part(s + 2, here, j);
            }
        });
        if (here == 0) {
#pragma unroll
            for (int r = 0; r < WN; ++r) we[r] >>= 16;
#pragma unroll
            for (int b = 0; b < WM; ++b) xe[b] >>= 16;
        } else {
            read_exps(s / 2 + 1);
        }
    };
    const int steps = (p.KT + 1) / 2;
    load_exps(0);
    load_step(0, 0);
    load_step(1, 1);
    arrive<2 * kWLoads + kXLoads>();
    read_exps(0);
    read_x(0, 0);
#pragma unroll
    for (int r = 0; r < WN; ++r) read_w(0, 0, r);
    int s = 0;
    for (; s < steps - 2; ++s) one_step(s, std::true_type());
    for (; s < steps; ++s) one_step(s, std::false_type());

    // The lanes of a row of X hold four neighbouring sums each, of either row block of a pair.  The two blocks' words are exchanged
    // between neighbouring rows of lanes, so that every lane stores sixteen bytes: those of even o of the first block, of odd o of the second.
    static_assert(WN % 2 == 0, "row blocks in pairs");
#pragma unroll
    for (int b = 0; b < WM; ++b) {
        const int m = m0 + 16 * (wm * WM + b) + i;
        char* y = p.y + ((int64_t)m * p.N + 16 * (rb0 + wn * WN + (o & 1)) + 8 * (o >> 1)) * 2;
#pragma unroll
        for (int r = 0; r < WN; r += 2) {
            u32x4 out;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto two = __builtin_amdgcn_permlane16_swap(round_pair(acc[r][b][2 * h], acc[r][b][2 * h + 1], p.bf16),
                                                                  round_pair(acc[r + 1][b][2 * h], acc[r + 1][b][2 * h + 1], p.bf16), false, false);
                out[h] = two[0];
                out[2 + h] = two[1];
            }
            if (m < m1 && rb0 + wn * WN + r + (o & 1) < p.NB) *reinterpret_cast<u32x4*>(y + r * 32) = out;
        }
    }
}

namespace {

constexpr size_t kCounterBytes = 64 * 1024;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

// How many pieces of ROWS rows there can be: by expert, at most one short one for each that has rows.
int64_t most_pieces(const ProductParams& p, int rows) {
    return p.offsets ? p.M / rows + (p.M < p.experts ? p.M : p.experts) : (p.M + rows - 1) / rows;
}

template <int SRC, int R, int MB>
void launch_stream(ProductParams p, int waves, hipStream_t s) {
    const int nx = (p.NB + R - 1) / R;
    const size_t lds = (size_t)waves * R * MB * 1024;
    // (a launch has fewer than 2^16 workgroups along y and 2^32 threads)
    int64_t most = (int64_t(1) << 31) / (int64_t(nx) * waves * 64);
    most = most > 65535 ? 65535 : most;
    const int64_t pieces = most_pieces(p, 16 * MB);
    for (int64_t at = 0; at < pieces; at += most) {
        p.slot0 = (int)at;
        const dim3 grid(nx, (unsigned)(pieces - at < most ? pieces - at : most));
        if (p.offsets) stream_kernel<SRC, R, MB, true><<<grid, waves * 64, lds, s>>>(p);
        else stream_kernel<SRC, R, MB, false><<<grid, waves * 64, lds, s>>>(p);
    }
}

template <int WN, int WM, int GN, int GM>
void launch_tiles(ProductParams p, hipStream_t s) {
    const int64_t nx = (p.NB + WN * GN - 1) / (WN * GN), pieces = most_pieces(p, 16 * WM * GM);
    const int64_t most = (int64_t(1) << 31) / (nx * GN * GM * 64);             // (a launch has fewer than 2^32 threads)
    for (int64_t at = 0; at < pieces; at += most) {
        p.slot0 = (int)at;
        p.slots = (int)(pieces - at < most ? pieces - at : most);
        if (p.offsets) tile_kernel<WN, WM, GN, GM, true><<<nx * p.slots, GN * GM * 64, 0, s>>>(p);
        else tile_kernel<WN, WM, GN, GM, false><<<nx * p.slots, GN * GM * 64, 0, s>>>(p);
    }
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
    int src = xe ? kF32 : dtype == LUTQ_F16 ? kF16 : kBF16;
    const int64_t rows = M / experts;                  // rows an expert has on average
    if (src != kF32 && rows > 16) {
        char *codes = static_cast<char*>(workspace) + kCounterBytes, *exponents = codes + up256((size_t)M * (K / 2));
        const lutq_status st = quantize_rows_on(X, src, M, nullptr, M, K, codes, exponents, s);
        if (st != LUTQ_OK) return st;
        p.x = codes; p.xe = exponents;
        src = kF32;
    }
    const int mb = rows > 16 ? 4 : 1;
    const int waves = p.KQ < 8 ? p.KQ : 8;
    if (src == kF16) launch_stream<kF16, 2, 1>(p, waves, s);
    else if (src == kBF16) launch_stream<kBF16, 2, 1>(p, waves, s);
    else if (mb == 1) launch_stream<kF32, 2, 1>(p, waves, s);
    else if (K < 512 || rows <= 128) launch_stream<kF32, 4, 4>(p, waves < 4 ? waves : 4, s);
    else launch_tiles<8, 4, 2, 4>(p, s);
    return hipGetLastError() == hipSuccess ? LUTQ_OK : LUTQ_ERR_DEVICE;
}

}  // namespace

}  // namespace mx4
}  // namespace lutq

using namespace lutq::mx4;

extern "C" size_t lutq_mx4_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts) {
    if (!shape_ok(N, K) || !rows_ok(M, K) || experts < 1 || experts > 65536) return 0;
    return kCounterBytes + up256((size_t)M * (size_t)(K / 2)) + up256((size_t)M * (size_t)(K / 32));
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
