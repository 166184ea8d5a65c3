// Quantisers to the 8-bit form and back, and the gated block's gradient, which ends in them (include/lutq.h).
//
// All are bound by memory traffic.  Sixteen lanes ("team") hold 128 columns, eight values each, so every load is 16 (fp32: 32)
// consecutive bytes per lane and whole cache lines per wavefront.  Where a square of 128 x 128 is looked at as one (weights, columns,
// gradients), a workgroup holds it in registers, a 4 x 8 block per lane: its rows' and columns' codes both leave from there.
// Measured, us and what they read and write a second: rows of 8192 x 8192 bf16 33 (6.1 TB/s), 1003 picked rows of 2176 fp16 3.7; weights 28672 x 4096
// fp32 104 (5.6 TB/s), bf16 with those of the transposed as well 72 (6.5 TB/s); columns of 4096 x 4096 bf16 11; weights back to bf16 50 (7.0 TB/s).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lutq.h"
#include "lutq_fp8_device.hpp"
#include "lutq_layout.hpp"

namespace lutq {
namespace fp8 {

constexpr int kThreads = 256;

struct QuantizeParams {
    const void* x;             // [source_rows, K]
    const int32_t* rows;       // or null
    const int32_t* offsets;    // or null: rows offsets[0] .. offsets[experts] - 1 are written, others stay
    char* codes;
    float* scales;             // [K / 128, M]; weights: [ceil(N / 128), K / 128]
    char* transposed;          // weights: [K, N] or null, and
    float* transposed_scales;  // [K / 128, ceil(N / 128)]
    int64_t source_rows, M, K, padded;
    int experts;
    uint32_t ku, groups;       // K / 128, and workgroups along it
    uint32_t magic, shift;     // u / groups = (u * magic) >> shift for u < 2^31
    uint32_t block0;           // of this launch's workgroups the first
};

// The dense side is read once: non-temporal, as it would drive the codes, which are read soon, out of the caches.
template <int SRC> __device__ __forceinline__ Eight<SRC> load_eight(const void* x, int64_t at) {
    Eight<SRC> r;
    const char* p = static_cast<const char*>(x) + at * (SRC == kF32 ? 4 : 2);
    r.v[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    if constexpr (SRC == kF32) r.v[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16));
    return r;
}
template <int SRC> __device__ __forceinline__ Eight<SRC> no_values() {
    Eight<SRC> r;
    r.v[0] = u32x4{0, 0, 0, 0};
    if constexpr (SRC == kF32) r.v[1] = u32x4{0, 0, 0, 0};
    return r;
}

// Rows.  ROWS 16: a team has a row and UNITS neighbouring blocks of it, a workgroup sixteen rows, whose scales are neighbours; ROWS 1,
// for few rows: a workgroup has one row, a team UNITS blocks that lie sixteen apart.
template <int SRC, int ROWS, int UNITS>
__global__ __launch_bounds__(kThreads) void quantize_rows(const QuantizeParams p) {
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x, group = (uint32_t)(((uint64_t)id * p.magic) >> p.shift);
    const uint32_t k0 = id - group * p.groups;
    const int64_t row = ROWS == 1 ? (int64_t)group : (int64_t)group * 16 + team;
    const uint32_t first = ROWS == 1 ? k0 * (16 * UNITS) + team : k0 * UNITS, step = ROWS == 1 ? 16 : 1;
    if (row >= p.M) return;
    if (p.offsets && (row < p.offsets[0] || row >= p.offsets[p.experts])) return;
    const int64_t from = p.rows ? p.rows[row] : row;
    const bool there = from >= 0 && from < p.source_rows;
    Eight<SRC> x[UNITS];
#pragma unroll
    for (int t = 0; t < UNITS; ++t) {
        const uint32_t u = first + t * step;
        x[t] = there && u < p.ku ? load_eight<SRC>(p.x, from * p.K + (int64_t)u * 128 + 8 * j) : no_values<SRC>();
    }
#pragma unroll
    for (int t = 0; t < UNITS; ++t) {
        const uint32_t u = first + t * step;
        float v[8];
        to_floats<SRC>(x[t], v);
        const Scale s = scale_of(largest_of_sixteen(largest(v)));
        if (u >= p.ku) continue;
        *reinterpret_cast<u32x2*>(p.codes + row * p.K + (int64_t)u * 128 + 8 * j) = to_codes(v, s);
        if (j == 0) p.scales[(int64_t)u * p.M + row] = s.scale;
    }
}

// ---------------------------------------------------------------------------------------------------- squares of 128 x 128
// Lane 16 team + j of a workgroup of 32 teams holds rows 4 team .. 4 team + 3, columns 8 j .. 8 j + 7 of the square.
constexpr int kSquare = 512, kEach = 4;
struct Block { float v[kEach][8]; };

template <int SRC> __device__ __forceinline__ void load_block(const void* x, int64_t row0, int64_t rows, int64_t K, int64_t column, Eight<SRC> (&raw)[kEach]) {
#pragma unroll
    for (int r = 0; r < kEach; ++r) raw[r] = row0 + r < rows ? load_eight<SRC>(x, (row0 + r) * K + column) : no_values<SRC>();
}

// 4 x 4 bytes: word r of `m` is a row, then a column.
__device__ __forceinline__ void transpose_four(uint32_t (&m)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(m[1], m[0], 0x05010400u), b = __builtin_amdgcn_perm(m[1], m[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(m[3], m[2], 0x05010400u), d = __builtin_amdgcn_perm(m[3], m[2], 0x07030602u);
    m[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    m[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    m[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    m[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// The largest over the four teams of a wavefront.
__device__ __forceinline__ uint32_t largest_of_teams(uint32_t a) {
    const auto near = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    a = max(near[0], near[1]);
    const auto far = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    return max(far[0], far[1]);
}

// The codes of the lane's rows to those of its columns, by way of LDS to memory: column c of the square at `to` + c * pitch, 128 bytes, of which those
// of `bytes` rows are written (a multiple of sixteen); `keep` is zero for columns of no codes.  All threads call it; `tile` is 16 KiB, free before and after.
// Sixteen rows q of column c lie at 16 (q ^ ((c >> 3) & 7)): lanes that write, or read, together do not meet in a bank more than twice.
__device__ __forceinline__ void store_columns(const u32x2 (&codes)[kEach], const uint32_t (&keep)[8], char* tile, char* to, int64_t pitch, int bytes) {
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {                      // columns 4 h .. 4 h + 3
        uint32_t m[4] = {codes[0][h], codes[1][h], codes[2][h], codes[3][h]};
        transpose_four(m);
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint32_t*>(tile + (8 * j + 4 * h + c) * 128 + ((team >> 2) ^ (j & 7u)) * 16 + (team & 3u) * 4) = m[c] & keep[4 * h + c];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int c = t * 64 + (int)(threadIdx.x >> 3), q = (int)(threadIdx.x & 7u);
        if (16 * q < bytes) *reinterpret_cast<u32x4*>(to + c * pitch + 16 * q) = *reinterpret_cast<const u32x4*>(tile + c * 128 + ((q ^ (c >> 3)) & 7) * 16);
    }
    __syncthreads();
}

// Codes of the square's rows: a scale per row, as quantize_rows has them.
__device__ __forceinline__ void rows_out(const Block& b, int64_t row0, int64_t rows, char* codes, int64_t pitch, float* scales) {
    const uint32_t j = threadIdx.x & 15u;
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        const Scale s = scale_of(largest_of_sixteen(largest(b.v[r])));
        if (row0 + r >= rows) continue;
        *reinterpret_cast<u32x2*>(codes + (row0 + r) * pitch) = to_codes(b.v[r], s);
        if (j == 0) scales[row0 + r] = s.scale;
    }
}

// Codes of its columns: a power of two per column, and the codes as rows of the transposed matrix.  `most` is 8 * 128 words.
__device__ __forceinline__ void columns_out(const Block& b, char* tile, uint32_t* most, char* to, int64_t pitch, float* scales) {
    const uint32_t j = threadIdx.x & 15u;
    uint32_t a[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        a[c] = 0;
#pragma unroll
        for (int r = 0; r < kEach; ++r) a[c] = max(a[c], magnitude(b.v[r][c]));
        a[c] = largest_of_teams(a[c]);
    }
    if ((threadIdx.x & 48u) == 0) {
        uint32_t* mine = most + (threadIdx.x >> 6) * 128 + 8 * j;
        *reinterpret_cast<u32x4*>(mine) = u32x4{a[0], a[1], a[2], a[3]};
        *reinterpret_cast<u32x4*>(mine + 4) = u32x4{a[4], a[5], a[6], a[7]};
    }
    __syncthreads();
    if (threadIdx.x < 128) {
        uint32_t all = 0;
#pragma unroll
        for (int t = 0; t < kSquare / 64; ++t) all = max(all, most[t * 128 + threadIdx.x]);
        most[threadIdx.x] = all;                       // (this thread alone reads its column)
        scales[threadIdx.x] = power_of_two_scale_of(all).scale;
    }
    __syncthreads();
    float inverse[8];
    uint32_t keep[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const Scale s = power_of_two_scale_of(most[8 * j + c]);
        inverse[c] = s.inverse;
        keep[c] = s.bad ? 0u : 0xffffffffu;
    }
    u32x2 codes[kEach];
#pragma unroll
    for (int r = 0; r < kEach; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float* v = b.v[r] + 4 * h;
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse[4 * h], v[1] * inverse[4 * h + 1], 0, false);
            codes[r][h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse[4 * h + 2], v[3] * inverse[4 * h + 3], w, true);
        }
    store_columns(codes, keep, tile, to, pitch, 128);
}

template <int SRC>
__global__ __launch_bounds__(kSquare) void quantize_weights(const QuantizeParams p) {
    __shared__ __align__(16) char tile[16 * 1024];
    __shared__ uint32_t most[kSquare / 64];
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x, nb = (uint32_t)(((uint64_t)id * p.magic) >> p.shift), kb = id - nb * p.groups;
    const int64_t row0 = (int64_t)nb * 128 + kEach * team, column = (int64_t)kb * 128 + 8 * j;
    Eight<SRC> raw[kEach];
    load_block<SRC>(p.x, row0, p.M, p.K, column, raw);
    uint32_t a = 0;
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        float v[8];
        to_floats<SRC>(raw[r], v);
        a = max(a, largest(v));
    }
    a = largest_of_teams(largest_of_sixteen(a));
    if ((threadIdx.x & 63u) == 0) most[threadIdx.x >> 6] = a;
    __syncthreads();
    a = 0;
#pragma unroll
    for (int t = 0; t < kSquare / 64; ++t) a = max(a, most[t]);
    const Scale s = scale_of(a);
    if (threadIdx.x == 0) {
        p.scales[(int64_t)nb * p.ku + kb] = s.scale;
        if (p.transposed) p.transposed_scales[(int64_t)kb * ((p.M + 127) >> 7) + nb] = s.scale;
    }
    u32x2 codes[kEach];
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        float v[8];
        to_floats<SRC>(raw[r], v);
        codes[r] = to_codes(v, s);
        if (row0 + r < p.M) *reinterpret_cast<u32x2*>(p.codes + (row0 + r) * p.K + column) = codes[r];
    }
    if (p.transposed) {
        const int64_t left = p.M - (int64_t)nb * 128;
        const uint32_t all[8] = {~0u, ~0u, ~0u, ~0u, ~0u, ~0u, ~0u, ~0u};
        store_columns(codes, all, tile, p.transposed + (int64_t)kb * 128 * p.M + (int64_t)nb * 128, p.M, left < 128 ? (int)left : 128);
    }
}

template <int SRC>
__global__ __launch_bounds__(kSquare) void quantize_columns(const QuantizeParams p) {
    __shared__ __align__(16) char tile[16 * 1024];
    __shared__ __align__(16) uint32_t most[8 * 128];
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x, mb = (uint32_t)(((uint64_t)id * p.magic) >> p.shift), kb = id - mb * p.groups;
    Eight<SRC> raw[kEach];
    load_block<SRC>(p.x, (int64_t)mb * 128 + kEach * team, p.M, p.K, (int64_t)kb * 128 + 8 * j, raw);
    Block b;
#pragma unroll
    for (int r = 0; r < kEach; ++r) to_floats<SRC>(raw[r], b.v[r]);
    columns_out(b, tile, most, p.codes + (int64_t)kb * 128 * p.padded + (int64_t)mb * 128, p.padded, p.scales + (int64_t)mb * p.K + (int64_t)kb * 128);
}

// ---------------------------------------------------------------------------------------------------- gradient of the gated block
struct GradParams {
    const char* dh;            // [M, F]
    const char* saved;         // [M, 2 F]: G, U
    char* dense;               // [M, 2 F] or null: dG, dU at 16 bits
    char* codes;               // rows: [M, 2 F] or null, and
    float* scales;             // [2 F / 128, M]
    char* columns;             // [2 F, padded] or null, and
    float* column_scales;      // [padded / 128, 2 F]
    int64_t M, F, padded;
    int act, bf16;
    uint32_t groups, magic, shift, block0;
};

// dU = dH act(G), dG = dH U act'(G), of a square of 128 x 128 of H, in every form that is asked for from the same registers: 6 bytes a value are
// read, 2 written for the codes of rows and 2 for those of columns.  4096 x 14336 bf16: 145 .. 155 us, 3.9 TB/s, vector instructions
// issued for 70 % of the cycles; with registers for one workgroup a unit instead of two (a few values in scratch memory) 177, computed once for either layout 231.
template <int SRC>
__global__ __launch_bounds__(kSquare, 4) void gated_grad(const GradParams p) {
    __shared__ __align__(16) char tile[16 * 1024];
    __shared__ __align__(16) uint32_t most[8 * 128];
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x, mb = (uint32_t)(((uint64_t)id * p.magic) >> p.shift), fb = id - mb * p.groups;
    const int64_t row0 = (int64_t)mb * 128 + kEach * team, column = (int64_t)fb * 128 + 8 * j;
    Eight<SRC> dh[kEach], g[kEach], u[kEach];
    load_block<SRC>(p.dh, row0, p.M, p.F, column, dh);
    load_block<SRC>(p.saved, row0, p.M, 2 * p.F, column, g);
    load_block<SRC>(p.saved, row0, p.M, 2 * p.F, p.F + column, u);
    Block dg, du;
#pragma unroll
    for (int r = 0; r < kEach; ++r) {                  // (rows that do not exist are zeros, and so are their gradients)
        float a[8], x[8], y[8];
        to_floats<SRC>(dh[r], a);
        to_floats<SRC>(g[r], x);
        to_floats<SRC>(u[r], y);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            float f, slope;
            activated(x[c], p.act, f, slope);
            dg.v[r][c] = a[c] * (y[c] * slope);
            du.v[r][c] = a[c] * f;
        }
    }
    auto out = [&](const Block& b, int64_t at) {       // `at`: of the 2 F columns the first of these
        if (p.dense) {
#pragma unroll
            for (int r = 0; r < kEach; ++r) {
                if (row0 + r >= p.M) continue;
                u32x4 w;
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = round_pair(b.v[r][2 * c], b.v[r][2 * c + 1], p.bf16);
                *reinterpret_cast<u32x4*>(p.dense + ((row0 + r) * 2 * p.F + at + column) * 2) = w;
            }
        }
        if (p.codes) rows_out(b, row0, p.M, p.codes + at + column, 2 * p.F, p.scales + (at / 128 + fb) * p.M);
        if (p.columns)
            columns_out(b, tile, most, p.columns + (at + (int64_t)fb * 128) * p.padded + (int64_t)mb * 128, p.padded,
                        p.column_scales + (int64_t)mb * 2 * p.F + at + (int64_t)fb * 128);
    };
    out(dg, 0);
    out(du, p.F);
}

// ---------------------------------------------------------------------------------------------------- back
struct DequantParams {
    const char* codes;
    const float* scales;
    u32x4* out;
    int64_t pieces;            // of eight codes
    uint32_t kp, magic, shift; // pieces of a row
    uint32_t M;                // rows: of the scales' rows; weights: 0
    int bf16;
    uint32_t block0;
};

template <int PIECES>
__global__ __launch_bounds__(kThreads) void dequant(const DequantParams p) {
    const int64_t first = (int64_t)(p.block0 + (uint32_t)blockIdx.x) * (PIECES * kThreads) + threadIdx.x;
    u32x2 c[PIECES];
    float s[PIECES];
#pragma unroll
    for (int t = 0; t < PIECES; ++t) {
        const int64_t w = first + t * kThreads;
        if (w >= p.pieces) continue;
        // (units of sixteen pieces, of which there are fewer than 2^31)
        const uint32_t unit = (uint32_t)(w >> 4), ku = p.kp >> 4, row = (uint32_t)(((uint64_t)unit * p.magic) >> p.shift), kb = unit - row * ku;
        c[t] = *reinterpret_cast<const u32x2*>(p.codes + w * 8);
        s[t] = p.M ? p.scales[(int64_t)kb * p.M + row] : p.scales[(int64_t)(row >> 7) * ku + kb];
    }
#pragma unroll
    for (int t = 0; t < PIECES; ++t) {
        const int64_t w = first + t * kThreads;
        if (w < p.pieces) __builtin_nontemporal_store(from_codes(c[t], s[t], p.bf16), &p.out[w]);
    }
}

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool dtype_ok(lutq_dtype dtype) { return dtype == LUTQ_F16 || dtype == LUTQ_BF16; }

// u / d = (u * magic) >> shift for u < 2^31, 1 <= d < 2^31
void division(uint32_t d, uint32_t* magic, uint32_t* shift) {
    uint32_t s = 0;
    while ((uint64_t(1) << s) < d) ++s;
    *shift = 31 + s;
    *magic = (uint32_t)((uint64_t(1) << (31 + s)) / d + 1);
}

// A launch has fewer than 2^32 threads, which the largest matrices reach.
template <typename P, typename F> void in_launches(P p, int64_t blocks, F launch) {
    constexpr int64_t kMost = (int64_t(1) << 32) / kSquare - 1;
    for (int64_t at = 0; at < blocks; at += kMost) {
        p.block0 = (uint32_t)at;
        launch(p, (uint32_t)(blocks - at < kMost ? blocks - at : kMost));
    }
}

lutq_status launched() { return hipGetLastError() == hipSuccess ? LUTQ_OK : LUTQ_ERR_DEVICE; }

template <int SRC> void launch_rows(QuantizeParams p, hipStream_t s) {
    auto run = [&](auto rows, auto units) {
        constexpr int ROWS = decltype(rows)::value, UNITS = decltype(units)::value;
        const int64_t high = ROWS == 1 ? p.M : (p.M + 15) / 16;
        p.groups = (p.ku + (ROWS == 1 ? 16 : 1) * UNITS - 1) / ((ROWS == 1 ? 16 : 1) * UNITS);
        division(p.groups, &p.magic, &p.shift);
        in_launches(p, high * p.groups, [&](const QuantizeParams& q, uint32_t grid) { quantize_rows<SRC, ROWS, UNITS><<<grid, kThreads, 0, s>>>(q); });
    };
    using std::integral_constant;
    // Four blocks per team where that still leaves work for every compute unit, one where latency is all that counts.
    if (p.M < 16) run(integral_constant<int, 1>(), integral_constant<int, 1>());
    else if (p.M * p.ku >= 4 * 16 * 512) run(integral_constant<int, 16>(), integral_constant<int, 4>());
    else run(integral_constant<int, 16>(), integral_constant<int, 1>());
}

}  // namespace

// Checked arguments; also the products' own call for activations that they do not quantise themselves.
lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, const int32_t* offsets, int64_t experts,
                             int64_t M, int64_t K, void* codes, float* scales, hipStream_t stream) {
    QuantizeParams p{};
    p.x = X; p.rows = rows; p.source_rows = source_rows; p.offsets = offsets; p.experts = (int)experts;
    p.codes = static_cast<char*>(codes); p.scales = scales;
    p.M = M; p.K = K; p.ku = (uint32_t)(K / 128);
    if (source == kF32) launch_rows<kF32>(p, stream);
    else if (source == kF16) launch_rows<kF16>(p, stream);
    else launch_rows<kBF16>(p, stream);
    return launched();
}

}  // namespace fp8
}  // namespace lutq

using namespace lutq::fp8;

static int source_of(int is_f32, lutq_dtype dtype) { return is_f32 ? kF32 : dtype == LUTQ_F16 ? kF16 : kBF16; }

extern "C" lutq_status lutq_fp8_quantize(const void* X, int x_is_f32, lutq_dtype dtype, int64_t source_rows, const int32_t* rows,
                                         int64_t M, int64_t K, void* codes_out, float* scales_out, void* stream) {
    if (!rows_ok(M, K) || source_rows < 0 || source_rows >= (int64_t(1) << 31) || (!rows && M > 0 && source_rows != M))
        return LUTQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return LUTQ_ERR_DTYPE;
    if (M == 0) return LUTQ_OK;
    if ((!X && source_rows > 0) || !codes_out || !scales_out) return LUTQ_ERR_NULL;
    if (!aligned(X, 16) || !aligned(rows, 4) || !aligned(codes_out, 16) || !aligned(scales_out, 4)) return LUTQ_ERR_ALIGN;
    return quantize_rows_on(X, source_of(x_is_f32, dtype), source_rows, rows, nullptr, 0, M, K, codes_out, scales_out, static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_fp8_quantize_weights(const void* W, int w_is_f32, lutq_dtype dtype, int64_t N, int64_t K, void* codes_out,
                                                 float* scales_out, void* transposed_codes_out, float* transposed_scales_out,
                                                 void* stream) {
    if (!W || !codes_out || !scales_out || !transposed_codes_out != !transposed_scales_out) return LUTQ_ERR_NULL;
    if (!shape_ok(N, K) || !rows_ok(N, K)) return LUTQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return LUTQ_ERR_DTYPE;
    if (!aligned(W, 16) || !aligned(codes_out, 16) || !aligned(scales_out, 4) || !aligned(transposed_codes_out, 16) ||
        !aligned(transposed_scales_out, 4))
        return LUTQ_ERR_ALIGN;
    QuantizeParams p{};
    p.x = W; p.codes = static_cast<char*>(codes_out); p.scales = scales_out; p.transposed = static_cast<char*>(transposed_codes_out); p.transposed_scales = transposed_scales_out;
    p.M = N; p.K = K; p.ku = p.groups = (uint32_t)(K / 128);
    division(p.groups, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(p, (N + 127) / 128 * p.groups, [&](const QuantizeParams& q, uint32_t grid) {
        if (w_is_f32) quantize_weights<kF32><<<grid, kSquare, 0, s>>>(q);
        else if (dtype == LUTQ_F16) quantize_weights<kF16><<<grid, kSquare, 0, s>>>(q);
        else quantize_weights<kBF16><<<grid, kSquare, 0, s>>>(q);
    });
    return launched();
}

extern "C" lutq_status lutq_fp8_quantize_columns(const void* X, int x_is_f32, lutq_dtype dtype, int64_t M, int64_t K, void* codes_out,
                                                 float* scales_out, void* stream) {
    if (M < 1 || !rows_ok(M, K)) return LUTQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return LUTQ_ERR_DTYPE;
    if (!X || !codes_out || !scales_out) return LUTQ_ERR_NULL;
    if (!aligned(X, 16) || !aligned(codes_out, 16) || !aligned(scales_out, 4)) return LUTQ_ERR_ALIGN;
    QuantizeParams p{};
    p.x = X; p.codes = static_cast<char*>(codes_out); p.scales = scales_out;
    p.M = M; p.K = K; p.padded = (M + 127) / 128 * 128; p.ku = p.groups = (uint32_t)(K / 128);
    division(p.groups, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(p, p.padded / 128 * p.groups, [&](const QuantizeParams& q, uint32_t grid) {
        if (x_is_f32) quantize_columns<kF32><<<grid, kSquare, 0, s>>>(q);
        else if (dtype == LUTQ_F16) quantize_columns<kF16><<<grid, kSquare, 0, s>>>(q);
        else quantize_columns<kBF16><<<grid, kSquare, 0, s>>>(q);
    });
    return launched();
}

static lutq_status dequant_on(const void* codes, const float* scales, int64_t M, int64_t K, bool weights, lutq_dtype dtype, void* out, void* stream) {
    if (!dtype_ok(dtype)) return LUTQ_ERR_DTYPE;
    if (M == 0) return LUTQ_OK;
    if (!codes || !scales || !out) return LUTQ_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(out, 16)) return LUTQ_ERR_ALIGN;
    DequantParams p{};
    p.codes = static_cast<const char*>(codes); p.scales = scales; p.out = static_cast<u32x4*>(out);
    p.pieces = M * (K / 8); p.kp = (uint32_t)(K / 8); p.M = weights ? 0 : (uint32_t)M; p.bf16 = dtype == LUTQ_BF16;
    division(p.kp / 16, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool many = p.pieces >= int64_t(4) * kThreads * 1024;
    const int64_t per = many ? 4 * kThreads : kThreads;
    in_launches(p, (p.pieces + per - 1) / per, [&](const DequantParams& q, uint32_t grid) {
        if (many) dequant<4><<<grid, kThreads, 0, s>>>(q);
        else dequant<1><<<grid, kThreads, 0, s>>>(q);
    });
    return launched();
}

extern "C" lutq_status lutq_fp8_dequant(const void* codes, const float* scales, int64_t M, int64_t K, lutq_dtype dtype, void* X_out, void* stream) {
    if (!rows_ok(M, K)) return LUTQ_ERR_SHAPE;
    return dequant_on(codes, scales, M, K, false, dtype, X_out, stream);
}

extern "C" lutq_status lutq_fp8_dequant_weights(const void* codes, const float* scales, int64_t N, int64_t K, lutq_dtype dtype, void* W_out, void* stream) {
    if (!shape_ok(N, K) || !rows_ok(N, K)) return LUTQ_ERR_SHAPE;
    return dequant_on(codes, scales, N, K, true, dtype, W_out, stream);
}

extern "C" lutq_status lutq_fp8_gated_grad(const void* dH, const void* saved, int64_t M, int64_t F, lutq_activation activation, lutq_dtype dtype,
                                           void* dense_out, void* codes_out, float* scales_out, void* columns_out, float* column_scales_out,
                                           void* stream) {
    if (F < 1 || F % 128 != 0 || F > kMostColumns / 2 || !rows_ok(M, 2 * F)) return LUTQ_ERR_SHAPE;
    if (!dtype_ok(dtype) || (activation != LUTQ_SILU && activation != LUTQ_GELU)) return LUTQ_ERR_DTYPE;
    if (M == 0) return columns_out ? LUTQ_ERR_SHAPE : LUTQ_OK;
    if (!dH || !saved || (!dense_out && !codes_out && !columns_out) || !codes_out != !scales_out || !columns_out != !column_scales_out)
        return LUTQ_ERR_NULL;
    if (!aligned(dH, 16) || !aligned(saved, 16) || !aligned(dense_out, 16) || !aligned(codes_out, 16) || !aligned(columns_out, 16) ||
        !aligned(scales_out, 4) || !aligned(column_scales_out, 4))
        return LUTQ_ERR_ALIGN;
    GradParams p{};
    p.dh = static_cast<const char*>(dH); p.saved = static_cast<const char*>(saved);
    p.dense = static_cast<char*>(dense_out);
    p.codes = static_cast<char*>(codes_out); p.scales = scales_out;
    p.columns = static_cast<char*>(columns_out); p.column_scales = column_scales_out;
    p.M = M; p.F = F; p.padded = (M + 127) / 128 * 128; p.act = activation; p.bf16 = dtype == LUTQ_BF16;
    p.groups = (uint32_t)(F / 128);
    division(p.groups, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(p, p.padded / 128 * p.groups, [&](const GradParams& q, uint32_t grid) {
        if (dtype == LUTQ_F16) gated_grad<kF16><<<grid, kSquare, 0, s>>>(q);
        else gated_grad<kBF16><<<grid, kSquare, 0, s>>>(q);
    });
    return launched();
}
