// What the products of quantised factors (lutq_mx4_matmul.hip, lutq_fp8_matmul.hip) have in common: copies from memory to LDS, rows by
// expert, stores of Y, the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "lutq_mx4_device.hpp"

namespace lutq {
namespace product {

using mx4::f32x4;
using mx4::round_pair;
using mx4::u32x4;

constexpr int kSc1 = 16, kNonTemporal = 2;             // past the caches that are a die's own; past the order of all caches

// Sixteen bytes per lane from memory to LDS, where lane l's go to `to` + 16 l.
template <int HOW = 0> __device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t from, uint32_t lane_at, int at, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_at, at, 0, HOW);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t unbounded(const char* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (uint32_t)-1, 0x00020000);
}

// Sixteen bytes per lane that workgroups on other dies read, or wrote, in the same launch.
// Stores of sixteen bytes have their whole offset in the vector register and the instruction, none in a scalar register: the data are read over
// several cycles, and only without a scalar offset does the compiler keep the next instruction from overwriting the first of them (seen to be
// stored overwritten: the address of the next store, in the last lanes of a row).  The additions cost nothing that shows: 28 microscaled calls, listed and drawn
// ones, took 0.986 to 1.012 of the time without them, in turn (8192 x 8192 x 8192 266.9 us and 266.4; 1024 x 4096 x 14336 45.6 and 45.6).
__device__ __forceinline__ void store16_shared(__amdgpu_buffer_rsrc_t to, uint32_t lane_at, int at, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), to, lane_at + at, 0, kSc1);
}
__device__ __forceinline__ f32x4 load16_shared(__amdgpu_buffer_rsrc_t from, uint32_t lane_at, int at) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, lane_at, at, kSc1));
}

// Between what lanes of a wavefront write to LDS and what others of it read there, in either order.  LDS serves a wavefront in order, so this
// is no instruction: it keeps the compiler, to which each lane is a program of its own, from moving the accesses past each other.
__device__ __forceinline__ void between_lanes() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }

// The rows of X in pieces of at most ROWS that do not straddle experts, numbered in order of the experts.  Every lane of a wavefront looks
// at one expert at a time; the whole wavefront gets the answers.
template <int ROWS> struct Pieces {
    const int32_t* offsets;
    int experts, M;
    // More pieces than there can be, unless experts claim the same rows: sums stop there, so that none wraps around, and what comes behind
    // is left out.
    static constexpr int kMost = 1 << 29;
    int a, b, sum;             // of the lane's expert among the 64 last looked at: its rows, its pieces and those of the ones before it

    __device__ __forceinline__ void look(int base) {
        const int lane = threadIdx.x & 63, g = base + lane;
        a = b = 0;
        if (g < experts) {
            a = min(max(offsets[g], 0), M);
            b = min(max(offsets[g + 1], 0), M);
        }
        sum = mine();
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum = min(sum + up, kMost);
        }
    }
    __device__ __forceinline__ int mine() const { return b > a ? (b - a + ROWS - 1) / ROWS : 0; }
    __device__ __forceinline__ int all() const { return __builtin_amdgcn_readlane(sum, 63); }

    __device__ __forceinline__ int count() {
        int n = 0;
        for (int base = 0; base < experts; base += 64) { look(base); n = min(n + all(), kMost); }
        return n;
    }
    // Piece `slot`, which has to exist: its expert, that expert's rows [first, end) and pieces [begin, begin + pieces).  (Up to 64 experts,
    // count() has looked already.)
    struct Found { int expert, first, end, begin, pieces; };
    __device__ __forceinline__ Found find(int slot) {
        int before = 0;
        for (int base = 0; base < experts; base += 64) {
            if (experts > 64) look(base);
            if (before + all() > slot) {
                const int at = __builtin_ctzll(__ballot(before + sum > slot)), n = __builtin_amdgcn_readlane(mine(), at);
                return {base + at, __builtin_amdgcn_readlane(a, at), __builtin_amdgcn_readlane(b, at), before + __builtin_amdgcn_readlane(sum, at) - n, n};
            }
            before = min(before + all(), kMost);
        }
        return {0, 0, 0, 0, 1};
    }
};

// Quotients of scalars, which the compiler computes in vector registers and would leave there.
__device__ __forceinline__ int quotient(int a, int b) { return __builtin_amdgcn_readfirstlane((int)((uint32_t)a / (uint32_t)b)); }

// Workgroups go to the eight dies in turn: the place of workgroup `id` of `n` such that each die gets a run of consecutive places.
__device__ __forceinline__ int by_die(int id, int n) {
    const int per = n >> 3;
    return id < per * 8 ? (id & 7) * per + (id >> 3) : id;
}

// Sixteen rows of Y, WN row blocks wide, from the sums of `row block`, of which `rows` and `blocks` exist.
// The lanes of a row of X hold four neighbouring sums each, of either row block of a pair.  The two blocks' words are exchanged between
// neighbouring rows of lanes, so that every lane has sixteen bytes: those of even o of the first block, of odd o of the second.  With four
// row blocks the lanes of rows i and i + 8 exchange one of their two sixteen bytes as well, and a store writes whole cache lines of
// eight rows, non-temporal ones: Y would drive the factors, which are read again, out of the caches.  (16384 rows, 28672 x 4096:
// 966 us with half lines and kept, 954 with whole ones, 923 non-temporal, 904 with both.  Half lines of the small tiles are kept:
// 512 rows, 4096 x 4096, 12.3 us, non-temporal 12.7.)
// Lanes whose row or row block does not exist store behind what the descriptor covers, which does nothing: always WN / 2 stores.
template <int WN, typename F>
__device__ __forceinline__ void store_rows(F sum, char* y, int rows, int blocks, int N, int bf16) {
    static_assert(WN % 2 == 0, "row blocks in pairs");
    constexpr uint32_t kNowhere = 0x7fffffff;
    const int lane = threadIdx.x & 63, i = lane & 15, o = lane >> 4, at = 16 * (o & 1) + 8 * (o >> 1);
    const int mine = blocks - (o & 1);
    const auto to = __builtin_amdgcn_make_buffer_rsrc(y, 0, 0x40000000, 0x00020000);
    auto pair_of = [&](int r) {
        const f32x4 a = sum(r), b = sum(r + 1);
        u32x4 out;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const auto two = __builtin_amdgcn_permlane16_swap(round_pair(a[2 * h], a[2 * h + 1], bf16), round_pair(b[2 * h], b[2 * h + 1], bf16), false, false);
            out[h] = two[0];
            out[2 + h] = two[1];
        }
        return out;
    };
    if constexpr (WN % 4 == 0) {
        const bool low = i < 8;
        const uint32_t from = (uint32_t)((i & 7) * N + at) * 2 + (low ? 0 : 64);
        const uint32_t to1 = (i & 7) < rows ? from : kNowhere, to2 = 8 + (i & 7) < rows ? from + 16 * N : kNowhere;
#pragma unroll
        for (int r = 0; r < WN; r += 4) {
            const u32x4 first = pair_of(r), second = pair_of(r + 2);
            u32x4 one, two;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint32_t t = low ? second[h] : first[h];
                const uint32_t u = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x128, 0xf, 0xf, true);   // row_ror 8
                one[h] = low ? first[h] : u;
                two[h] = low ? u : second[h];
            }
            const bool there = r + (low ? 0 : 2) < mine;
            __builtin_amdgcn_raw_buffer_store_b128(one, to, (there ? to1 : kNowhere) + r * 32, 0, kNonTemporal);
            __builtin_amdgcn_raw_buffer_store_b128(two, to, (there ? to2 : kNowhere) + r * 32, 0, kNonTemporal);
        }
    } else {
        const uint32_t from = i < rows ? (uint32_t)(i * N + at) * 2 : kNowhere;
#pragma unroll
        for (int r = 0; r < WN; r += 2) __builtin_amdgcn_raw_buffer_store_b128(pair_of(r), to, (r < mine ? from : kNowhere) + r * 32, 0, 0);
    }
}

// Waits until at most N of this wavefront's global loads are under way and all its LDS reads are done, then for the workgroup.
template <int N> __device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

// How many pieces of ROWS rows there can be: by expert, at most one short one for each that has rows.
inline int64_t most_pieces(int64_t M, int64_t experts, int rows) {
    return experts ? M / rows + (M < experts ? M : experts) : (M + rows - 1) / rows;
}

// More than 64 KiB of LDS has to be enabled once per kernel and device.
template <auto KERNEL, typename P> hipError_t launch(dim3 grid, int threads, size_t lds, const P& p, hipStream_t s) {
    if (lds > 64 * 1024) {
        static std::atomic<uint64_t> enabled{0};       // one bit per device
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) return e;
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if (!(enabled.load(std::memory_order_relaxed) & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
            if (e != hipSuccess) return e;
            enabled.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    KERNEL<<<grid, threads, lds, s>>>(p);
    return hipGetLastError();
}

}  // namespace product
}  // namespace lutq
