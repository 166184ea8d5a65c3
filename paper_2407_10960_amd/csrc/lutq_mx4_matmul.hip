// Products of the microscaled 4-bit form (include/lutq.h): Y = X W^T and the same by expert, on the scaled matrix instruction
// v_mfma_scale_f32_16x16x128_f8f6f4, which takes 128 columns of sixteen rows of either factor and their exponents as they are held.
//
// The instruction's first operand is the weights, so a lane's four sums are neighbours in a row of Y.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "lutq.h"
#include "lutq_layout.hpp"
#include "lutq_mx4_device.hpp"

namespace lutq {
namespace mx4 {

lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, int64_t M, int64_t K,
                             void* codes, void* exponents, hipStream_t stream);

struct ProductParams {
    const char* x;             // row form: codes; or 16-bit values
    const char* xe;            // row form: exponents
    const char* w;             // records
    char* y;
    const int32_t* offsets;    // by expert: experts + 1; else null
    int64_t record, expert;    // bytes of a row block's record, of an expert's weights
    int M, N, K, KT, KQ, NB;   // K tiles, quads, row blocks
    int experts;
    int slot0;                 // first piece of rows of this launch
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
    else launch_stream<kF32, 4, 4>(p, waves < 4 ? waves : 4, s);
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
