// Quantiser and its inverse for the microscaled 4-bit form (include/lutq.h): one exponent byte and 32 codes of 4 bits per block.
//
// Both are bound by memory traffic.  Four neighbouring lanes hold a block, eight values each, so every load is 16 (fp32: 32)
// consecutive bytes per lane and whole cache lines per wavefront; the block's largest magnitude crosses the four lanes with two
// register moves, and one conversion instruction per pair of values scales, rounds and packs.  Sixteen lanes hold 128 columns
// ("unit"); its four exponent bytes are gathered in one lane and stored as one word.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "lutq.h"
#include "lutq_layout.hpp"
#include "lutq_mx4_device.hpp"

namespace lutq {
namespace mx4 {

constexpr int kThreads = 256;

struct QuantizeParams {
    const void* x;             // [source_rows, K]
    const int32_t* rows;       // or null
    uint32_t* codes;           // row form: a word per eight values; packed form: the records
    uint32_t* exponents;       // row form: a word per unit
    int64_t source_rows;
    int64_t record;            // packed form: bytes of a record
    uint32_t units;            // row form: M * K / 128
    uint32_t ku;               // K / 128
    uint32_t magic, shift;     // u / ku = (u * magic) >> shift for u < 2^31
    uint32_t K;
    uint32_t block0;           // of this launch's workgroups the first
};

// The dense side, read or written once, is non-temporal: it would drive the codes, which are read soon, out of the caches, and itself does
// not stay (bf16 8192 x 4096 to codes 18.9 us, so 17.1, and back 18.8, so 14.1; one after the other 38.1 and 30.5).
template <int SRC> __device__ __forceinline__ Eight<SRC> load_eight(const void* x, int64_t at) {
    Eight<SRC> r;
    const char* p = static_cast<const char*>(x) + at * (SRC == kF32 ? 4 : 2);
    r.v[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    if constexpr (SRC == kF32) r.v[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16));
    return r;
}

// Row form: UNITS units per sixteen lanes, all loaded before the first is used.
template <int SRC, int UNITS>
__global__ __launch_bounds__(kThreads) void quantize_rows(const QuantizeParams p) {
    const uint32_t j = threadIdx.x & 15u, team = threadIdx.x >> 4;
    uint32_t u[UNITS];
    Eight<SRC> x[UNITS];
#pragma unroll
    for (int t = 0; t < UNITS; ++t) {
        u[t] = ((p.block0 + (uint32_t)blockIdx.x) * UNITS + t) * (kThreads / 16) + team;
        x[t].v[0] = u32x4{0, 0, 0, 0};
        if constexpr (SRC == kF32) x[t].v[1] = u32x4{0, 0, 0, 0};
        if (u[t] >= p.units) continue;
        int64_t at = (int64_t)u[t] * 128;
        if (p.rows) {
            const uint32_t row = (uint32_t)(((uint64_t)u[t] * p.magic) >> p.shift);
            const int64_t from = p.rows[row];
            if (from < 0 || from >= p.source_rows) continue;
            at = from * p.K + (int64_t)(u[t] - row * p.ku) * 128;
        }
        x[t] = load_eight<SRC>(p.x, at + 8 * j);
    }
#pragma unroll
    for (int t = 0; t < UNITS; ++t) {
        uint32_t e;
        const uint32_t c = quantize_eight<SRC>(x[t], e);
        uint32_t word = e << (8 * (j >> 2));           // byte o of the unit's word is block o: gathered over the sixteen lanes
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x124, 0xf, 0xf, true);   // row_ror 4
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x128, 0xf, 0xf, true);   // row_ror 8
        if (u[t] >= p.units) continue;
        p.codes[(int64_t)u[t] * 16 + j] = c;
        if (j == 0) p.exponents[u[t]] = word;
    }
}

// Packed form: a workgroup writes one quad (16 rows, 512 columns) of a record.  Sixteen lanes take one row of the four tiles one
// after the other, so a lane ends up with the four exponent bytes that are neighbours in the packed form.
template <int SRC>
__global__ __launch_bounds__(kThreads) void quantize_packed(const QuantizeParams p) {
    const uint32_t j = threadIdx.x & 15u, i = threadIdx.x >> 4, o = j >> 2;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x;
    const uint32_t quads = (p.ku + 3) >> 2, rb = (uint32_t)(((uint64_t)id * p.magic) >> p.shift), q = id - rb * quads;
    const int64_t row = (int64_t)rb * 16 + i;
    const uint32_t tiles = min(4u, p.ku - 4 * q);
    Eight<SRC> x[4];
#pragma unroll
    for (uint32_t t = 0; t < 4; ++t)
        if (t < tiles) x[t] = load_eight<SRC>(p.x, row * p.K + (4 * q + t) * 128 + 8 * j);
    char* record = reinterpret_cast<char*>(p.codes) + rb * p.record;
    uint32_t word = 0;
#pragma unroll
    for (uint32_t t = 0; t < 4; ++t) {
        if (t >= tiles) continue;
        uint32_t e;
        const uint32_t c = quantize_eight<SRC>(x[t], e);
        word |= e << (8 * t);
        *reinterpret_cast<uint32_t*>(record + (int64_t)(4 * q + t) * 1024 + (16 * o + i) * 16 + 4 * (j & 3u)) = c;
    }
    if ((j & 3u) == 0) *reinterpret_cast<uint32_t*>(record + (int64_t)p.ku * 1024 + q * 256 + (16 * o + i) * 4) = word;
}

struct DequantParams {
    const uint32_t* codes;
    const uint8_t* exponents;
    u32x4* out;
    int64_t record;
    int64_t words;             // row form: M * K / 8
    uint32_t ku, magic, shift;
    uint32_t K;
    uint32_t block0;           // of this launch's workgroups the first
};

template <bool BF16, int WORDS>
__global__ __launch_bounds__(kThreads) void dequant_rows(const DequantParams p) {
    uint32_t c[WORDS], e[WORDS];
    const int64_t first = (int64_t)(p.block0 + (uint32_t)blockIdx.x) * (WORDS * kThreads) + threadIdx.x;
#pragma unroll
    for (int t = 0; t < WORDS; ++t) {
        const int64_t w = first + t * kThreads;
        if (w < p.words) { c[t] = p.codes[w]; e[t] = p.exponents[w >> 2]; }
    }
#pragma unroll
    for (int t = 0; t < WORDS; ++t) {
        const int64_t w = first + t * kThreads;
        if (w < p.words) __builtin_nontemporal_store(from_codes<BF16>(c[t], power_of(e[t])), &p.out[w]);
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void dequant_packed(const DequantParams p) {
    const uint32_t j = threadIdx.x & 15u, i = threadIdx.x >> 4, o = j >> 2;
    const uint32_t id = p.block0 + (uint32_t)blockIdx.x;
    const uint32_t quads = (p.ku + 3) >> 2, rb = (uint32_t)(((uint64_t)id * p.magic) >> p.shift), q = id - rb * quads;
    const uint32_t tiles = min(4u, p.ku - 4 * q);
    const char* record = reinterpret_cast<const char*>(p.codes) + rb * p.record;
    const uint32_t word = *reinterpret_cast<const uint32_t*>(record + (int64_t)p.ku * 1024 + q * 256 + (16 * o + i) * 4);
    uint32_t c[4];
#pragma unroll
    for (uint32_t t = 0; t < 4; ++t)
        if (t < tiles) c[t] = *reinterpret_cast<const uint32_t*>(record + (int64_t)(4 * q + t) * 1024 + (16 * o + i) * 16 + 4 * (j & 3u));
    u32x4* out = p.out + ((int64_t)rb * 16 + i) * (p.K / 8) + q * 64 + j;
#pragma unroll
    for (uint32_t t = 0; t < 4; ++t)
        if (t < tiles) __builtin_nontemporal_store(from_codes<BF16>(c[t], power_of((word >> (8 * t)) & 255u)), &out[t * 16]);
}

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// u / d = (u * magic) >> shift for u < 2^31, 1 <= d < 2^31
void division(uint32_t d, uint32_t* magic, uint32_t* shift) {
    uint32_t s = 0;
    while ((uint64_t(1) << s) < d) ++s;
    *shift = 31 + s;
    *magic = (uint32_t)((uint64_t(1) << (31 + s)) / d + 1);
}

// A launch has fewer than 2^32 threads, which the largest matrices reach.
template <typename P, typename F> void in_launches(P p, uint32_t blocks, F launch) {
    constexpr uint32_t kMost = (uint32_t)((uint64_t(1) << 32) / kThreads) - 1;
    for (uint32_t at = 0; at < blocks; at += kMost) {
        p.block0 = at;
        launch(p, blocks - at < kMost ? blocks - at : kMost);
    }
}

lutq_status launched() { return hipGetLastError() == hipSuccess ? LUTQ_OK : LUTQ_ERR_DEVICE; }

template <int SRC> void launch_rows(const QuantizeParams& p, hipStream_t s) {
    // Four units per team where that still leaves work for every compute unit, one where latency is all that counts.
    const uint32_t teams = kThreads / 16;
    if (p.units >= 4u * teams * 512u)
        in_launches(p, (p.units + 4 * teams - 1) / (4 * teams), [&](const QuantizeParams& q, uint32_t grid) { quantize_rows<SRC, 4><<<grid, kThreads, 0, s>>>(q); });
    else quantize_rows<SRC, 1><<<(p.units + teams - 1) / teams, kThreads, 0, s>>>(p);
}

}  // namespace

// Checked arguments; also the product's own call for activations that it does not quantise itself.
lutq_status quantize_rows_on(const void* X, int source, int64_t source_rows, const int32_t* rows, int64_t M, int64_t K,
                             void* codes, void* exponents, hipStream_t stream) {
    QuantizeParams p{};
    p.x = X; p.rows = rows; p.source_rows = source_rows;
    p.codes = static_cast<uint32_t*>(codes); p.exponents = static_cast<uint32_t*>(exponents);
    p.ku = (uint32_t)(K / 128); p.K = (uint32_t)K; p.units = (uint32_t)(M * (K / 128));
    division(p.ku, &p.magic, &p.shift);
    if (source == kF32) launch_rows<kF32>(p, stream);
    else if (source == kF16) launch_rows<kF16>(p, stream);
    else launch_rows<kBF16>(p, stream);
    return launched();
}

}  // namespace mx4
}  // namespace lutq

using namespace lutq::mx4;

extern "C" lutq_status lutq_mx4_quantize(const void* X, int x_is_f32, lutq_dtype dtype, int64_t source_rows, const int32_t* rows,
                                         int64_t M, int64_t K, void* codes_out, void* exponents_out, void* stream) {
    if (!rows_ok(M, K) || source_rows < 0 || source_rows >= (int64_t(1) << 31) || (!rows && M > 0 && source_rows != M))
        return LUTQ_ERR_SHAPE;
    if (dtype != LUTQ_F16 && dtype != LUTQ_BF16) return LUTQ_ERR_DTYPE;
    if (M == 0) return LUTQ_OK;
    if ((!X && source_rows > 0) || !codes_out || !exponents_out) return LUTQ_ERR_NULL;
    if (!aligned(X, 16) || !aligned(rows, 4) || !aligned(codes_out, 16) || !aligned(exponents_out, 16)) return LUTQ_ERR_ALIGN;
    return quantize_rows_on(X, x_is_f32 ? kF32 : dtype == LUTQ_F16 ? kF16 : kBF16, source_rows, rows, M, K, codes_out, exponents_out,
                            static_cast<hipStream_t>(stream));
}

extern "C" lutq_status lutq_mx4_quantize_packed(const void* W, int w_is_f32, lutq_dtype dtype, int64_t N, int64_t K,
                                                void* packed_out, void* stream) {
    if (!W || !packed_out) return LUTQ_ERR_NULL;
    if (!shape_ok(N, K) || !rows_ok(N, K)) return LUTQ_ERR_SHAPE;
    if (dtype != LUTQ_F16 && dtype != LUTQ_BF16) return LUTQ_ERR_DTYPE;
    if (!aligned(W, 16) || !aligned(packed_out, 16)) return LUTQ_ERR_ALIGN;
    QuantizeParams p{};
    p.x = W; p.codes = static_cast<uint32_t*>(packed_out); p.record = record_bytes(K);
    p.ku = (uint32_t)(K / 128); p.K = (uint32_t)K;
    const uint32_t quads = (uint32_t)k_quads(K);
    division(quads, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(p, (uint32_t)(N / 16) * quads, [&](const QuantizeParams& q, uint32_t grid) {
        if (w_is_f32) quantize_packed<kF32><<<grid, kThreads, 0, s>>>(q);
        else if (dtype == LUTQ_F16) quantize_packed<kF16><<<grid, kThreads, 0, s>>>(q);
        else quantize_packed<kBF16><<<grid, kThreads, 0, s>>>(q);
    });
    return launched();
}

extern "C" lutq_status lutq_mx4_dequant(const void* codes, const void* exponents, int64_t M, int64_t K, lutq_dtype dtype,
                                        void* X_out, void* stream) {
    if (!rows_ok(M, K)) return LUTQ_ERR_SHAPE;
    if (dtype != LUTQ_F16 && dtype != LUTQ_BF16) return LUTQ_ERR_DTYPE;
    if (M == 0) return LUTQ_OK;
    if (!codes || !exponents || !X_out) return LUTQ_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(exponents, 16) || !aligned(X_out, 16)) return LUTQ_ERR_ALIGN;
    DequantParams p{};
    p.codes = static_cast<const uint32_t*>(codes); p.exponents = static_cast<const uint8_t*>(exponents);
    p.out = static_cast<u32x4*>(X_out); p.words = M * (K / 8);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool many = p.words >= int64_t(4) * kThreads * 1024;
    const uint32_t per = many ? 4 * kThreads : kThreads;
    in_launches(p, (uint32_t)((p.words + per - 1) / per), [&](const DequantParams& q, uint32_t grid) {
        if (dtype == LUTQ_BF16) {
            if (many) dequant_rows<true, 4><<<grid, kThreads, 0, s>>>(q); else dequant_rows<true, 1><<<grid, kThreads, 0, s>>>(q);
        } else {
            if (many) dequant_rows<false, 4><<<grid, kThreads, 0, s>>>(q); else dequant_rows<false, 1><<<grid, kThreads, 0, s>>>(q);
        }
    });
    return launched();
}

extern "C" lutq_status lutq_mx4_dequant_packed(const void* packed, int64_t N, int64_t K, lutq_dtype dtype, void* W_out, void* stream) {
    if (!packed || !W_out) return LUTQ_ERR_NULL;
    if (!shape_ok(N, K) || !rows_ok(N, K)) return LUTQ_ERR_SHAPE;
    if (dtype != LUTQ_F16 && dtype != LUTQ_BF16) return LUTQ_ERR_DTYPE;
    if (!aligned(packed, 16) || !aligned(W_out, 16)) return LUTQ_ERR_ALIGN;
    DequantParams p{};
    p.codes = static_cast<const uint32_t*>(packed); p.out = static_cast<u32x4*>(W_out); p.record = record_bytes(K);
    p.ku = (uint32_t)(K / 128); p.K = (uint32_t)K;
    const uint32_t quads = (uint32_t)k_quads(K);
    division(quads, &p.magic, &p.shift);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(p, (uint32_t)(N / 16) * quads, [&](const DequantParams& q, uint32_t grid) {
        if (dtype == LUTQ_BF16) dequant_packed<true><<<grid, kThreads, 0, s>>>(q);
        else dequant_packed<false><<<grid, kThreads, 0, s>>>(q);
    });
    return launched();
}
