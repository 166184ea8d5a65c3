/*
 * lutq — fused lookup-table dequantise + small-batch matmul for AMD MI355X (gfx950).
 *
 * C ABI of liblutq.so.  Plain pointers and sizes only; every buffer is owned by
 * the caller.  The library never allocates device memory, never synchronises the
 * device and never aborts: arguments are validated on the host and a status code
 * is returned BEFORE anything is launched, so on error no output is touched.
 *
 * Problem (Section 3 of "Fast Matrix Multiplications for Lookup Table-Quantized
 * LLMs", arXiv 2407.10960): an index matrix Q with entries in {0..2^b-1}, a table
 * T = [v_0 .. v_{2^b-1}] of 16-bit floats, dequantised weights W^ = T[Q], and the
 * product Y = X * W^ with a small number of activation rows.  With the group
 * scales of Section 4.1 ("LUT quantization method") / Section 4.2 the weight is
 *
 *        W^[n, k] = round16( T[Q[n, k]] * S[n, k / group_size] )
 *        Y[m, n]  = sum_k X[m, k] * W^[n, k]          (fp32 accumulation)
 *
 * Orientation: the paper writes Q and W as k-by-n; this library stores their
 * transposes, [N, K] row-major (one row per output channel, as a linear layer
 * does).  A group is `group_size` consecutive elements along K inside one row.
 * round16 is one round-to-nearest-even to the 16-bit type `dtype`.
 *
 * Supported domain: bits in {2,3,4}; group_size in {32,64,128,256}; 1 <= M <= 128
 * (one launch on the caller's stream, the weights streamed once.  Beyond 32 rows that is a kernel of its
 * own with no plan to choose, or at 4 bits up to 64 rows, where that is the faster, a slice of 64 rows; a call with
 * a plan, with a registered plan that slices of 32 rows can run, or
 * with one table per output row is served in slices instead, one launch each: 32 rows, or, at 4 bits where the plan
 * asks for LUTQ_SCHED_ROWS, 64 rows, each such launch preceded by a small one that copies the slice's
 * activations into the workspace in the order the matrix instruction reads them);
 * N a multiple of 16; K a multiple of the K-tile of the bit width (128 for
 * 4-bit, 256 for 2- and 3-bit) and of group_size; device pointers 16-byte aligned.
 *
 * Environment (read once per process, diagnostics only): LUTQ_VERBOSE=1 prints the launch shape
 * of every call and the tuner's finalists to stderr (2: also the tuner's first-pass times);
 * LUTQ_NO_SHARED_X=1 / LUTQ_NO_XM8=1 switch off two activation-load variants for comparisons.
 * They change at most the order of the fp32 summation.
 */
#ifndef LUTQ_H
#define LUTQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LUTQ_OK = 0,
    LUTQ_ERR_NULL = 1,         /* a required pointer is NULL */
    LUTQ_ERR_BITS = 2,         /* bits not in {2,3,4} */
    LUTQ_ERR_GROUP = 3,        /* group_size not in {32,64,128,256} or does not divide K */
    LUTQ_ERR_SHAPE = 4,        /* M, N or K outside the supported domain */
    LUTQ_ERR_ALIGN = 5,        /* a device pointer is not 16-byte aligned */
    LUTQ_ERR_INDEX_RANGE = 6,  /* lutq_pack: an index is >= 2^bits */
    LUTQ_ERR_WORKSPACE = 7,    /* workspace missing or smaller than lutq_workspace_bytes() */
    LUTQ_ERR_DTYPE = 8,        /* dtype not LUTQ_F16 / LUTQ_BF16 */
    LUTQ_ERR_DEVICE = 9,       /* a HIP runtime call failed (launch, device query) */
    LUTQ_ERR_PLAN = 10,        /* lutq_plan fields outside their documented ranges */
    LUTQ_ERR_SCRATCH = 11      /* lutq_matmul_static: the launch needs more than the built-in scratch */
} lutq_status;

typedef enum { LUTQ_F16 = 0, LUTQ_BF16 = 1 } lutq_dtype;

/* Human-readable name of a status code (static storage, never NULL). */
const char* lutq_status_string(lutq_status s);

/* ---------------------------------------------------------------------------
 * Offline restructuring (Section 3.1 "Offline Matrix Restructuring"; first line of
 * Algorithm 1, reorder_and_split).  Host code, run once per weight matrix.
 *
 * The packed form orders indices so that a wavefront's 128-bit loads deliver them
 * already in the operand order of the gfx950 16x16x32 matrix instruction, and
 * splits 3-bit indices into a 2-bit slice and a 1-bit slice so that every load is
 * a power-of-two number of bits.  It does not depend on group_size (the argument is
 * validated and otherwise unused).
 *
 * Packed layout (normative; this library's own -- the paper's is tied to NVIDIA Ampere fragments).
 * Q is [N, K] row-major.  N is cut into row blocks of 16 rows, K into tiles of TK columns (TK = 128
 * for 4-bit, 256 for 2- and 3-bit).  Row blocks are grouped into super-blocks of SB consecutive row
 * blocks: with nb = N / 16, SB = 4 if nb is a multiple of 4, else 2 if nb is even, else 1 -- except
 * SB = 2 for multiples of 4 in 257..512 (a choice tuned for 256 compute units and frozen into the
 * format: it holds on every device; lutq_pack_layout reports SB for a given N, so that it can be
 * recorded next to a packed blob).  Storage order is super-block, then K tile, then row block inside
 * the super-block: tile (rb, kt) starts at byte
 *        (((rb / SB) * (K / TK) + kt) * SB + rb % SB) * TILE_BYTES,
 * so the SB tiles that cover 16*SB rows x TK columns are adjacent.  A tile is what one 64-lane
 * wavefront loads with one 128-bit load per lane (plus one 64-bit load for the 3-bit high slice).
 * v_mfma_f32_16x16x32_{f16,bf16} takes, from lane l = 16*o + i (i = 0..15, o = 0..3), the eight
 * A-matrix elements of row i and columns 8*o .. 8*o+7 of a 16 x 32 block; a tile holds TK/32 such
 * blocks ("steps" t).  Lane l owns, for step t, the indices Q[16*rb + i][TK*kt + 32*t + 8*o + j],
 * j = 0..7, and its bytes sit at offset 16*l of the tile:
 *   4-bit  TILE_BYTES = 1024.  Four little-endian 32-bit words d = 0..3; word d is step d; nibble j
 *          (bits 4j..4j+3) is index j, so byte p of a word is the pair (2p, 2p+1).
 *   2-bit  TILE_BYTES = 1024.  Words d = 0..3; 2-bit field e (bits 2e..2e+1), e = 0..15, of word d is
 *          index j = e % 8 of step t = 2d + e / 8, so byte p holds four consecutive indices.
 *   3-bit  TILE_BYTES = 1536 = 1024 (low slice: index bits 0..1) + 512 (high slice: bit 2).
 *          Low slice, lane l at 16*l, words d = 0..3, byte p = 0..3 of word d:
 *              bits 0..1 low2(index 2p, step 2d)      bits 2..3 low2(index 2p+1, step 2d)
 *              bits 4..5 low2(index 2p, step 2d+1)    bits 6..7 low2(index 2p+1, step 2d+1)
 *          High slice, lane l at 1024 + 8*l, words h = 0..1, byte p of word h, u = 0..3:
 *              bit 2u = bit2(index 2p, step 4h+u)     bit 2u+1 = bit2(index 2p+1, step 4h+u)
 *          so that, for one step, (low word >> 0 or 4) supplies bits 0..3 of each byte and (high word
 *          shifted by 4 - 2u) supplies bits 4..5: four 6-bit pair-table addresses.
 * ------------------------------------------------------------------------- */

/* Geometry of the packed form of an [N, K] matrix at `bits` bits. */
typedef struct {
    int tile_k;                       /* K columns per tile: 128 (4-bit) or 256 */
    int tile_bytes;                   /* 1024, or 1536 at 3 bits */
    int row_blocks_per_super_block;   /* SB: 4, 2 or 1 */
    int64_t row_blocks;               /* N / 16 */
    int64_t k_tiles;                  /* K / tile_k */
} lutq_layout;

/* Fills *out for (N, K, bits).  Errors: NULL, BITS, GROUP, SHAPE. */
lutq_status lutq_pack_layout(int64_t N, int64_t K, int bits, int group_size, lutq_layout* out);

/* Size in bytes of the packed form (N*K*bits/8); 0 if the arguments are unsupported. */
size_t lutq_packed_bytes(int64_t N, int64_t K, int bits, int group_size);

/* indices: host, [N, K] row-major, one index per byte, each < 2^bits.
 * packed_out: host, caller-owned, lutq_packed_bytes() bytes, fully overwritten.
 * Errors: NULL, BITS, GROUP, SHAPE, INDEX_RANGE (packed_out contents then unspecified). */
lutq_status lutq_pack(const uint8_t* indices, int64_t N, int64_t K, int bits, int group_size,
                      void* packed_out);

/* Inverse of lutq_pack (host to host). indices_out: [N, K] row-major, one index per byte. */
lutq_status lutq_unpack(const void* packed, int64_t N, int64_t K, int bits, int group_size,
                        uint8_t* indices_out);

/* ---------------------------------------------------------------------------
 * The fused kernel (Algorithm 1 / Algorithm 2: copy table to on-chip memory, stream
 * packed weights, combine bit-slices, vectorised table lookup + group scale, matrix
 * instruction, Stream-K style partial-sum fix-up through global scratch).
 * ------------------------------------------------------------------------- */

/* Bytes of device scratch lutq_matmul may need for any M with these arguments
 * (the semaphore and partial-sum areas of Algorithm 2).  0 if unsupported. */
size_t lutq_workspace_bytes(int64_t N, int64_t K, int bits, int group_size);

/* Work-decomposition knobs (Section 3.3 Stream-K partitioning; Section 4.1: the kernel instance is
 * chosen per shape).  All fields 0 = let the library choose.  The number of table duplicates, a
 * tuning knob in the paper, is fixed here: one copy per lane (64 copies of a 4-byte entry, 32 of an
 * 8-byte entry), which is conflict-free by construction and makes the entry stride 256 bytes. */
typedef struct {
    int row_blocks_per_wave;  /* R: 16-row blocks each wavefront streams together: 0,1,2,4; must divide N/16 */
    int grid;                 /* number of workgroups: 0 or 1..4096 (grid x row groups per workgroup <= 4096) */
    int waves_per_workgroup;  /* wavefronts that share one table: 0 or 4..16, a multiple of the next-but-one field */
    int tiles_in_flight;      /* K tiles each wavefront keeps in flight (software pipeline depth): 0, 2 or 4 */
    int row_groups_per_workgroup; /* teams: row groups (of R blocks) a workgroup works on side by side, each
                                     by waves_per_workgroup / this many wavefronts that split K: 0 or 1..16;
                                     must divide N / (16 R) */
    int scheduling;           /* how a workgroup's work is dealt to its wavefronts: 0 = library chooses,
                                 LUTQ_SCHED_TEAMS (1) = the static teams described above,
                                 LUTQ_SCHED_QUEUE (2) = a work queue (M <= 4 and K / group_size a multiple of 8
                                 only): a workgroup owns whole row groups over the whole of K, cut into items of
                                 tiles_per_item K tiles that its wavefronts take one after the other from a
                                 counter.  The N / (16 R) row groups are dealt to `grid` workgroups as evenly
                                 as whole row groups allow: row_groups_per_workgroup (1..64) = the whole part of
                                 row groups / grid, the first workgroups one more.  Give grid (then
                                 row_groups_per_workgroup is 0 or that quotient) or row_groups_per_workgroup
                                 (a divisor of the row groups); R is 1 or 2, waves_per_workgroup 4..16 with
                                 no relation to the row groups, tiles_in_flight 2 */
                              /* LUTQ_SCHED_ROWS (3) = activation-stationary (M >= 5): `grid` workgroups own
                                 whole 16-row blocks over the whole of K, dealt as evenly as whole row blocks
                                 allow (row_groups_per_workgroup = the whole part of N / 16 / grid, 0 or that
                                 value; at most 64); the wavefronts (waves_per_workgroup 4..16, as many as the
                                 instance's registers allow) split K, hold a K tile's activations in registers
                                 and stream the weights of row_blocks_per_wave (4 or 8) row blocks past them
                                 side by side, in as many passes as the workgroup's row blocks need;
                                 tiles_in_flight 2.  For M > 32 this scheduling asks for slices of 64 rows
                                 (4 bits; LUTQ_ERR_PLAN where no such
                                 instance exists); that launch has one decomposition (4 row blocks side by
                                 side, one workgroup per compute unit, 8 waves at most), so every other
                                 field is 0 or the value lutq_plan_default reports; any other plan, and
                                 the default where 64-row slices are not faster, means slices of 32 rows.
                                 With tiles_per_item > 0 (launches of up to 32 rows; more rows go in slices
                                 of 32) K is cut into slices of that many K tiles
                                 across workgroups: `grid` (required, a multiple of the number of slices) =
                                 shares x slices, a share being at most row_blocks_per_wave row blocks (one
                                 pass: row_groups_per_workgroup = the whole part of N / 16 / shares), so a
                                 workgroup reads only its slice of the activations; every workgroup leaves
                                 its slice's sums in the scratch and the last of a share to finish adds them
                                 in slice order (shares <= 1024; shares x slices x row_blocks_per_wave x
                                 ceil(M / 16) KiB of scratch) */
    int tiles_per_item;       /* LUTQ_SCHED_QUEUE: K tiles (128 columns at 4 bits, 256 at 2 and 3) per item:
                                 0, or a multiple of tiles_in_flight that divides the K tiles of a row.
                                 LUTQ_SCHED_ROWS: 0 = K is not cut across workgroups, else the K tiles per
                                 slice: the K tiles of a row divided by it, rounded up, is the number of
                                 slices (at least two), which are as even as whole tiles allow */
} lutq_plan;

#define LUTQ_SCHED_TEAMS 1
#define LUTQ_SCHED_QUEUE 2
#define LUTQ_SCHED_ROWS 3

/* Fills *plan with the choice of the library's rules for this problem on the current device.  Passed back, it is what runs.  A
 * call without a plan (NULL, or the all-zero plan) takes that launch, or up to 32 rows another where estimated times say that it is
 * clearly faster.  For M > 32 the plan is the decomposition of the slices, the one a plan can ask for (a call without a plan takes
 * all rows in one launch). */
lutq_status lutq_plan_default(int bits, int group_size, int64_t M, int64_t N, int64_t K,
                              lutq_dtype dtype, lutq_plan* plan);

/* The same choice for a device with `compute_units` compute units (1..4096), without touching any
 * device: host logic only, for planning ahead and for tests.  MI355X has 256. */
lutq_status lutq_plan_default_for(int bits, int group_size, int64_t M, int64_t N, int64_t K,
                                  lutq_dtype dtype, int compute_units, lutq_plan* plan);

/* Whether lutq_matmul_plan would accept `plan` (NULL = the library's choice) for this problem on a device
 * with `compute_units` compute units: LUTQ_OK, or the status lutq_matmul_plan would return for the
 * plan and the problem (BITS, GROUP, SHAPE, DTYPE, PLAN).  Host logic only; no device is touched. */
lutq_status lutq_plan_check(int bits, int group_size, int64_t M, int64_t N, int64_t K, lutq_dtype dtype,
                            int compute_units, const lutq_plan* plan);

/* Plans chosen by measurement (lutq_tune; Section 4.1 picks the kernel configuration per shape offline and
 * dispatches on it): a process-wide table that lutq_matmul and lutq_matmul_static consult, when no plan
 * is passed, before their own choice.  An entry applies to calls with its bits, group_size, dtype, N,
 * K and m_min <= M <= m_max; the first match wins; an entry whose plan the kernels cannot run for a call,
 * or whose plan is all zero, is skipped (the library's own choice is used).  A call of M > 32 goes in slices of
 * 32 rows for the sake of the table where the first match for 32 rows is such that they can run it, and the library's own
 * slices on that shape are not of 64 rows (those have a single decomposition and do not consult the table); the M of each
 * slice counts then. */
typedef struct {
    int bits, group_size;
    lutq_dtype dtype;
    int64_t m_min, m_max, N, K;
    lutq_plan plan;
} lutq_plan_entry;

/* Replaces the table by a copy of entries[0 .. count-1] (count = 0 clears it).  Host memory only; safe to
 * call from any thread, but calls already in flight may still use the old table.  Errors: NULL, SHAPE
 * (count < 0 or > 4096). */
lutq_status lutq_plan_table_set(const lutq_plan_entry* entries, int count);

/* The plan the table holds for this call: LUTQ_OK and *plan, or LUTQ_ERR_PLAN if no entry matches. */
lutq_status lutq_plan_table_lookup(int bits, int group_size, int64_t M, int64_t N, int64_t K, lutq_dtype dtype,
                                   lutq_plan* plan);

/* Y = X * W^T-dequantised, asynchronous on `stream`.
 *   X       device, [M, K] row-major, dtype
 *   packed  device, bytes produced by lutq_pack for (N, K, bits)
 *   scales  device, [N, K / group_size] row-major, dtype
 *   lut     device, 2^bits entries, dtype (any finite values, any order)
 *   Y       device, [M, N] row-major, dtype; fully overwritten
 *   workspace  device, >= lutq_workspace_bytes(); must be zero-filled once before its
 *              first use.  Its first 64 KiB hold the arrival counters, which every successful
 *              call returns to zero; the rest holds partial sums that the next call simply
 *              overwrites.  The same workspace can therefore be reused by any later call on
 *              the same stream without clearing it.  Calls that may run concurrently
 *              (different streams) need separate workspaces.
 *   stream  a hipStream_t (NULL = the default stream)
 * Errors: NULL, BITS, GROUP, SHAPE, ALIGN, WORKSPACE, DTYPE, DEVICE; Y untouched on error. */
lutq_status lutq_matmul(const void* X, const void* packed, const void* scales, const void* lut,
                        int bits, int group_size, int64_t M, int64_t N, int64_t K,
                        lutq_dtype dtype, void* Y,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Same, with an explicit work decomposition (additionally returns LUTQ_ERR_PLAN).
 * The result does not depend on the plan beyond fp32 summation order. */
lutq_status lutq_matmul_plan(const void* X, const void* packed, const void* scales, const void* lut,
                             int bits, int group_size, int64_t M, int64_t N, int64_t K,
                             lutq_dtype dtype, void* Y,
                             void* workspace, size_t workspace_bytes, void* stream,
                             const lutq_plan* plan);

/* lutq_matmul_plan for callers that cannot allocate device memory or hand over a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.  The arrival counters and
 * partial sums live in a device array of the library's own, LUTQ_STATIC_SCRATCH_BYTES large (64 KiB of
 * counters + 16 MiB of partial-sum slots), which every GPU the library runs on holds from the first use
 * of the library on it until the process ends.  The call allocates nothing and calls no allocating
 * routine; the first call on a device looks the array's address up once (make that call outside a
 * graph capture).  Every other argument and the result are those of lutq_matmul_plan, bit for bit under the
 * same plan (NULL, the library's choice, may be another decomposition here: see below).
 * A launch needs partial-sum slots only when its plan cuts output tiles across workgroups: teams
 * grid x row groups per workgroup x 2 slots of R x ceil(M/16) x 1 KiB (M capped at 32), row streaming in K slices
 * grid x R slots of ceil(M/16) x 1 KiB.  If that exceeds the 16 MiB, a call with a plan returns LUTQ_ERR_SCRATCH before anything is launched (Y untouched), and a
 * call without one takes the library's choice among the decompositions that need little scratch (of the
 * LLaMA-3 8B/70B shapes only 70B gate+up in bf16 beyond sixteen rows does not fit with its first choice).
 * All calls on one GPU share the one array: calls that may overlap on a GPU (different streams) race
 * on it and must use lutq_matmul with separate workspaces instead.  The counters are returned to zero by
 * every launch; the slots keep the last call's partial sums and are overwritten before they are read. */
#define LUTQ_STATIC_SCRATCH_BYTES ((size_t)(64 * 1024 + 16 * 1024 * 1024))
lutq_status lutq_matmul_static(const void* X, const void* packed, const void* scales, const void* lut,
                               int bits, int group_size, int64_t M, int64_t N, int64_t K,
                               lutq_dtype dtype, void* Y, void* stream, const lutq_plan* plan);

/* Finer-grained tables: one table per output row (Section 2.3: lookup tables obtained at the
 * output-channel level; Section 5 names flexible tables as what the kernel is for).
 *        W^[n, k] = round16( T[n][Q[n, k]] * S[n, k / group_size] )
 *   luts    device, [N, 2^bits] row-major, dtype, 16-byte aligned
 *   every other argument as in lutq_matmul (scales of 1.0 give tables without group scales).
 * M <= 4 with K / group_size a multiple of 8: the work-queue kernel with the tables of all of a
 * workgroup's row blocks built once and resident (sixteen copies per row block: the four lanes that
 * work on a row share one).  5 <= M <= 32: the row-streaming kernel with the tables of four or eight row blocks side by side, where
 * there are at least two row blocks per compute unit (but for a few classes of five to eight rows); on smaller matrices too from 9 or 17 rows up, if K is long, then with K cut into
 * up to sixteen slices across workgroups, whose partial sums and counters are in the workspace.  Otherwise a workgroup holds the tables
 * of one 16-row block at a time and
 * rebuilds its on-chip copies for every row block it works on (one row block per workgroup, K split
 * over its waves and, for few row blocks, over workgroups, with partial sums in the workspace).  The work decomposition is the library's
 * in all cases.  Errors: those of lutq_matmul. */
lutq_status lutq_matmul_channel(const void* X, const void* packed, const void* scales, const void* luts,
                                int bits, int group_size, int64_t M, int64_t N, int64_t K,
                                lutq_dtype dtype, void* Y,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Vector codebooks (Section 5 names them, beside finer-grained tables, as what a flexible lookup kernel is
 * for): one 8-bit index selects a PAIR of adjacent weights from a codebook of 256 pairs, 4 bits per weight.
 *        W^[n, 2j + c] = round16( C[V[n, j]][c] * S[n, 2j / group_size] ),  c = 0, 1
 *   codebook  device, [256][2] values of dtype (1 KiB), 4-byte aligned
 *   packed    the 4-bit layout of lutq_pack applied to the indices Q[n, 2j] = V[n, j] & 15,
 *             Q[n, 2j + 1] = V[n, j] >> 4 (one byte of the 4-bit layout is one codebook index)
 *   every other argument as in lutq_matmul with bits = 4.
 * The kernels are those of lutq_matmul: their on-chip table at 4 bits already is a table of 256 pairs
 * (built from sixteen scalars there, copied from the codebook here), so the cost is the same.  A codebook
 * with C[e] = (T[e & 15], T[e >> 4]) gives lutq_matmul's result bit for bit.  The work decomposition is the
 * library's.  Errors: those of lutq_matmul; LUTQ_ERR_ALIGN also for a codebook that is not 4-byte aligned.
 *
 * lutq_matmul_quads is the same at 2 bits per weight: one 8-bit index selects FOUR adjacent weights,
 *        W^[n, 4j + c] = round16( C[V[n, j]][c] * S[n, 4j / group_size] ),  c = 0 .. 3
 *   codebook  device, [256][4] values of dtype (2 KiB), 4-byte aligned
 *   packed    the 2-bit layout of lutq_pack applied to Q[n, 4j + c] = (V[n, j] >> 2c) & 3
 * (the 2-bit kernels' on-chip table is a table of 256 quads); a codebook with C[e][c] = T[(e >> 2c) & 3]
 * gives lutq_matmul's 2-bit result bit for bit. */
lutq_status lutq_matmul_pairs(const void* X, const void* packed, const void* scales, const void* codebook,
                              int group_size, int64_t M, int64_t N, int64_t K,
                              lutq_dtype dtype, void* Y,
                              void* workspace, size_t workspace_bytes, void* stream);

lutq_status lutq_matmul_quads(const void* X, const void* packed, const void* scales, const void* codebook,
                              int group_size, int64_t M, int64_t N, int64_t K,
                              lutq_dtype dtype, void* Y,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Instance selection by measurement (Section 4.1: the fastest kernel configuration is picked per
 * shape; Section 3.3: how the K range is cut across workgroups is part of that choice).  Times what a
 * call without a plan launches and the other plans that lutq_tune_candidates lists, first with a few launches
 * each, then the eight fastest and that launch in three rounds of `reps` launches (the minimum per
 * plan counts), with events on `stream`, and
 * writes the fastest to *best and, if best_us is not NULL, its microseconds per launch to *best_us.
 *   packed, scales  host arrays of `ring` >= 1 device pointers each: weight sets of the same shape
 *                   (copies of one matrix will do) that successive launches visit in turn, so that
 *                   with a ring larger than the caches every launch streams from HBM as it would
 *                   inside a model; ring = 1 tunes for weights that stay in cache.
 *   the other arguments are those of lutq_matmul.  Y is overwritten by every candidate.
 * Blocks until the measurements on `stream` are done (it creates and destroys two events, nothing
 * else); must not be called while `stream` is being captured.
 * Errors: those of lutq_matmul; SHAPE also for ring < 1 or reps < 1. */
lutq_status lutq_tune(const void* X, const void* const* packed, const void* const* scales, int ring,
                      const void* lut, int bits, int group_size, int64_t M, int64_t N, int64_t K,
                      lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, void* stream,
                      int reps, lutq_plan* best, float* best_us);

/* The plans lutq_tune tries for this problem on the current device, what a call without a plan launches first: the
 * all-zero plan, followed by lutq_plan_default's, where the two are different launches (M > 32, and up to 32 rows where
 * estimated times choose), else lutq_plan_default's.  (A registered all-zero plan is the library's choice, too.)
 * Writes min(*count, capacity) of them to plans (host) and their number to *count; plans may be
 * NULL when capacity is 0.  Some of them have no kernel instance: lutq_matmul_plan answers those
 * with LUTQ_ERR_PLAN, and lutq_tune skips them. */
lutq_status lutq_tune_candidates(int bits, int group_size, int64_t M, int64_t N, int64_t K,
                                 lutq_dtype dtype, lutq_plan* plans, int capacity, int* count);

/* Quantiser on the GPU (Section 3, first equation: each weight is replaced by the index of the
 * nearest table entry; Section 4.1 "LUT quantization method" / Section 4.2: one absmax scale per
 * group, kept in the 16-bit type), fused with the restructuring of Section 3.1: a dense weight
 * matrix already in device memory becomes scales + packed indices in one pass, ready for lutq_matmul.
 *   scale S[n, g] = round16( max |W[n, k]| over the group )
 *   Q[n, k]       = the lowest c that minimises | W[n, k] / S[n, g] - T[c] |   (u = 0 where S = 0)
 * with the division, the difference and the comparison in IEEE fp64 on the exact input values, so
 * the result depends on the inputs only, not on the launch.
 *   W           device, [N, K] row-major; fp32 if w_is_f32 != 0, else `dtype`; 16-byte aligned; finite
 *   lut         device, 2^bits entries, dtype
 *   scales_out  device, [N, K / group_size] row-major, dtype, fully overwritten
 *   packed_out  device, lutq_packed_bytes() bytes, 16-byte aligned, fully overwritten (the bytes
 *               lutq_pack would produce from Q)
 * Asynchronous on `stream`; allocates nothing.  Errors: NULL, BITS, GROUP, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_quantize(const void* W, int w_is_f32, const void* lut, int bits, int group_size,
                          int64_t N, int64_t K, lutq_dtype dtype, void* scales_out, void* packed_out,
                          void* stream);

/* The separate-kernel path of Section 3 (dequantise to memory): writes
 * W_out[n, k] = round16(T[Q[n,k]] * S[n, k/group_size]), device [N, K] row-major, dtype,
 * using the same on-chip lookup + scale routine as lutq_matmul.  Asynchronous on `stream`. */
lutq_status lutq_dequant(const void* packed, const void* scales, const void* lut,
                         int bits, int group_size, int64_t N, int64_t K, lutq_dtype dtype,
                         void* W_out, void* stream);

/* ---------------------------------------------------------------------------
 * Microscaled 4-bit floating point: both factors of the product at 4 bits, for any number of rows.
 *
 * A row of K values is cut into blocks of 32 consecutive ones.  A block holds one exponent byte e, which stands
 * for 2^(e - 127) (255: not a number, the whole block is), and 32 codes of 4 bits: sign, two bits of exponent, one of
 * mantissa, with the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 in the order of the codes.  The value is code times power of two.
 * (This is the E2M1 / E8M0 pair of the Open Compute microscaling formats, whose products the matrix
 * instruction takes as they are.)
 *
 * Two forms hold it.  ROWS, for activations and for interchange: codes [M, K / 2] bytes, two codes a byte, the even column
 * in the low four bits, and exponents [M, K / 32] bytes, both row-major.  PACKED, for weights (normative): N is cut into
 * row blocks of 16 rows, K into tiles of 128 columns, four tiles to a quad, the last of which may be short.  A row block is a record of
 * (K / 128) * 1024 + ceil(K / 512) * 256 bytes, first its tiles in order of K, then its exponents.  In a tile, lane l = 16 * o + i
 * (i = 0..15, o = 0..3) owns the 16 bytes at offset 16 * l: the codes of row i, columns 32 * o .. 32 * o + 31 of the tile,
 * what v_mfma_scale_f32_16x16x128_f8f6f4 takes from that lane.  In the exponents of a quad, byte t of the 4 bytes at offset
 * 4 * l is the exponent of that lane's block in tile t (zero where the quad has no such tile).
 *
 * Domain: N a multiple of 16, K of 128, both up to 2^24; rows 0 <= M < 2^30 with M * K / 128 < 2^30 (no rows: nothing is
 * done and no pointer is looked at; the quantiser of weights and its inverse take N as M here); device pointers 16-byte aligned (rows and
 * offsets: 4); outputs and workspace overlap neither each other nor an input.  A K of whole blocks that is no multiple of 128, as 2880 is, is padded by the caller, in both factors: columns of
 * zeros, or exponents and codes of 0, behind each row add nothing to the sums; and N with rows of zeros, whose columns of Y are zeros.
 * ------------------------------------------------------------------------- */

/* Bytes of the packed form of an [N, K] matrix; 0 if the arguments are unsupported.  The experts of a grouped product are
 * such records one behind the other. */
size_t lutq_mx4_packed_bytes(int64_t N, int64_t K);

/* From the row form to the packed one and back, host to host (a checkpoint that holds the format already; on the device
 * lutq_mx4_quantize_packed packs what it quantises).  Errors: NULL, SHAPE. */
lutq_status lutq_mx4_pack(const void* codes, const void* exponents, int64_t N, int64_t K, void* packed_out);
lutq_status lutq_mx4_unpack(const void* packed, int64_t N, int64_t K, void* codes_out, void* exponents_out);

/* Quantiser.  For each block, with a = max |x|: e = max(0, 125 + floor(log2 a)), 0 where a = 0; each code is x / 2^(e - 127)
 * rounded to the nearest magnitude, ties to the even code, to 6 beyond it.  A block that holds an infinity or a NaN gets
 * e = 255 and codes 0.
 *   X       device, [source_rows, K] row-major; fp32 if x_is_f32 != 0, else `dtype`
 *   rows    device, M row numbers (int32), or NULL: output row m is row rows[m] of X, a row of zeros where rows[m] is not
 *           in 0 .. source_rows - 1.  NULL: row m (source_rows is then M)
 *   codes_out, exponents_out   device, the row form, fully overwritten
 * lutq_mx4_quantize_packed writes the packed form of W [N, K] instead.
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_mx4_quantize(const void* X, int x_is_f32, lutq_dtype dtype, int64_t source_rows, const int32_t* rows,
                              int64_t M, int64_t K, void* codes_out, void* exponents_out, void* stream);
lutq_status lutq_mx4_quantize_packed(const void* W, int w_is_f32, lutq_dtype dtype, int64_t N, int64_t K,
                                     void* packed_out, void* stream);

/* The values back, rounded once to the 16-bit `dtype` (exact in bf16 but beyond its largest number): [M, K] from the row
 * form, [N, K] from the packed one.  Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_mx4_dequant(const void* codes, const void* exponents, int64_t M, int64_t K, lutq_dtype dtype,
                             void* X_out, void* stream);
lutq_status lutq_mx4_dequant_packed(const void* packed, int64_t N, int64_t K, lutq_dtype dtype, void* W_out, void* stream);

/* Bytes of device scratch of the products below for up to M rows; experts = 1 for lutq_mx4_matmul.  0 if unsupported. */
size_t lutq_mx4_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts);

/* Y[m, n] = sum_k X[m, k] * W[n, k] over the 4-bit values of both, accumulated in fp32 (subnormal sums are kept, sums beyond its
 * largest number are infinite), rounded once to `dtype`.
 *   X, x_exponents   device: the row form of the activations; or, x_exponents NULL, activations [M, K] of `dtype`, which
 *                    are quantised on the way in, to what lutq_mx4_quantize would make of them
 *   packed           device, the packed form of W [N, K]
 *   Y                device, [M, N] row-major, dtype; fully overwritten
 *   workspace        device, >= lutq_mx4_workspace_bytes(M, N, K, 1), zero-filled once before its first use, and then as for
 *                    lutq_matmul: its first 64 KiB are left zero, calls that may run concurrently need one each
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, DEVICE; Y untouched on error. */
lutq_status lutq_mx4_matmul(const void* X, const void* x_exponents, const void* packed, int64_t M, int64_t N, int64_t K,
                            lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, void* stream);

/* The same by expert: rows offsets[g] .. offsets[g + 1] - 1 of X times the weights of expert g.
 *   packed    device, `experts` packed forms of [N, K] one behind the other
 *   offsets   device, experts + 1 row numbers (int32), not decreasing, within 0 .. M: read on the device, so the sizes may
 *             come from a kernel before it on the stream, and a captured call follows them.  (Values outside are taken as the
 *             nearest inside, an expert whose end is before its start has no rows, and each value in rows that
 *             several experts claim is one of theirs, or stays.)
 *   Y         [M, N]; rows before offsets[0] and from offsets[experts] on stay as they were
 *   workspace >= lutq_mx4_workspace_bytes(M, N, K, experts)
 * 1 <= experts <= 65536.  Everything else as for lutq_mx4_matmul. */
lutq_status lutq_mx4_matmul_grouped(const void* X, const void* x_exponents, const void* packed, const int32_t* offsets,
                                    int64_t experts, int64_t M, int64_t N, int64_t K, lutq_dtype dtype, void* Y,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * 8-bit floating point with a scale for each block of 128, and the gated feed-forward block on it.
 *
 * A value is a code of 8 bits times a 32-bit scale.  Codes are E4M3 as the Open Compute formats have it: sign, four bits of exponent,
 * three of mantissa, 448 the largest magnitude, 0x7f and 0xff not a number.  Three forms share it:
 *   ROWS     activations [M, K]: codes [M, K] row-major; scales [K / 128, M]: one for each row and 128 neighbouring columns
 *   WEIGHTS  [N, K]: codes [N, K] row-major; scales [ceil(N / 128), K / 128]: one for each square of 128 x 128 (as checkpoints hold
 *            them; transposed codes and scales are the transposed matrix's, where N is a multiple of 128 too)
 *   COLUMNS  X [M, K] transposed, for sums over its rows: codes [K, M'], M' = M rounded up to a multiple of 128, zeros there; scales
 *            [M' / 128, K], powers of two: one for each column and 128 neighbouring rows
 *
 * Quantiser: with a = max |x| over the block, at least 2^-110, the scale is a / 448 and the codes are x * (448 / a), each of the two quotients and
 * the product one rounding to 32 bits, then to the nearest code, ties to the even one.  By columns the scale is the least power of
 * two that is at least a / 448.  A block that holds an infinity or a NaN has a scale that is not a number, and codes of 0.
 *
 * Products: for each block of 128 columns the sum of the codes' products times the product of the two scales, one fp32 number (it loses precision
 * where it is below 2^-126 and is infinite beyond 2^128), added in fp32.  Anything that is not a number stays in its row or column of the result.
 * Which instruction sums a block, and the order of the additions, go by the launch, which is chosen from the sizes, the number of experts, what is asked
 * for and the device.  A call repeats itself bit for bit, but a row's last bits may be others in a batch of another size.
 *   - Exact, but for roundings of fp32: products of up to 16 rows, those by expert of up to 4 rows for each expert there is (M <= 4 * experts), more rows
 *     where they are streamed too (lutq_calib.h tells), and all gated calls with h_codes or saved.
 *   - All others, lutq_fp8_weight_grad among them: the 8-bit matrix instruction, at twice the rate.  Of eight neighbouring columns' products it cuts what lies
 *     below 2^-13 of the power of two of the largest; products of at least 2^-7 of that power are exact.  A sum is off by 7 2^-13 of the largest of each
 *     eight at most, and by some 2^-18 of the sum of magnitudes on random codes.  These calls take no request for exact sums: a caller who needs them
 *     gives up to 16 rows at a time, or takes the values back (lutq_fp8_dequant) to a 16-bit product.
 *
 * Domain: N a multiple of 16, up to 2^24; K a multiple of 128, up to 2^22; F (columns of H) a multiple of 128, up to 2^21; rows
 * 0 <= M < 2^30 with M * K / 128 < 2^30 (no rows: nothing is done and no pointer is looked at; the quantiser of weights takes N as M here); device
 * pointers 16-byte aligned (rows, offsets and scales: 4); outputs and workspace overlap neither each other nor an input.  A K that
 * is no multiple of 128 is padded by the caller, in both factors: columns of zero codes behind each row add nothing to the sums.
 * ------------------------------------------------------------------------- */

/* Quantiser of rows.
 *   X       device, [source_rows, K] row-major; fp32 if x_is_f32 != 0, else `dtype`
 *   rows    device, M row numbers (int32), or NULL: output row m is row rows[m] of X, a row of zeros where rows[m] is not
 *           in 0 .. source_rows - 1.  NULL: row m (source_rows is then M)
 *   codes_out, scales_out   device, ROWS, fully overwritten
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_fp8_quantize(const void* X, int x_is_f32, lutq_dtype dtype, int64_t source_rows, const int32_t* rows,
                              int64_t M, int64_t K, void* codes_out, float* scales_out, void* stream);

/* Quantiser of weights W [N, K].  transposed_codes_out, transposed_scales_out, or NULL: the codes [K, N] and scales
 * [K / 128, ceil(N / 128)] of W transposed as well.
 * Asynchronous on `stream`.  Errors: NULL (also for one of these two without the other), SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_fp8_quantize_weights(const void* W, int w_is_f32, lutq_dtype dtype, int64_t N, int64_t K, void* codes_out,
                                      float* scales_out, void* transposed_codes_out, float* transposed_scales_out, void* stream);

/* Quantiser of columns: codes_out [K, M'] and scales_out [M' / 128, K] of X [M, K], M >= 1.
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_fp8_quantize_columns(const void* X, int x_is_f32, lutq_dtype dtype, int64_t M, int64_t K, void* codes_out,
                                      float* scales_out, void* stream);

/* The values back, code times scale in fp32, rounded to the 16-bit `dtype`: [M, K] of ROWS, [N, K] of WEIGHTS.
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, DEVICE. */
lutq_status lutq_fp8_dequant(const void* codes, const float* scales, int64_t M, int64_t K, lutq_dtype dtype, void* X_out, void* stream);
lutq_status lutq_fp8_dequant_weights(const void* codes, const float* scales, int64_t N, int64_t K, lutq_dtype dtype, void* W_out, void* stream);

/* Bytes of device scratch of the products below for up to M rows; experts = 1 for those without.  0 if unsupported. */
size_t lutq_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts);
size_t lutq_fp8_gated_workspace_bytes(int64_t M, int64_t F, int64_t K, int64_t experts);

/* Y[m, n] = sum_k X[m, k] * W[n, k], rounded once to `dtype`.
 *   X, x_scales  device: ROWS; or, x_scales NULL, activations [M, K] of `dtype`, which are quantised on the way in, to what
 *                lutq_fp8_quantize would make of them
 *   W, w_scales  device: WEIGHTS [N, K]
 *   Y            device, [M, N] row-major, dtype; fully overwritten
 *   workspace    device, >= lutq_fp8_workspace_bytes(M, N, K, 1), zero-filled once before its first use, and then as for
 *                lutq_matmul: its first 64 KiB are left zero, calls that may run concurrently need one each
 * Asynchronous on `stream`.  Errors: NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, DEVICE; Y untouched on error. */
lutq_status lutq_fp8_matmul(const void* X, const float* x_scales, const void* W, const float* w_scales, int64_t M, int64_t N, int64_t K,
                            lutq_dtype dtype, void* Y, void* workspace, size_t workspace_bytes, void* stream);

/* The same by expert: rows offsets[g] .. offsets[g + 1] - 1 of X times the weights of expert g.
 *   W, w_scales  device: `experts` WEIGHTS [N, K], codes one behind the other and scales one behind the other
 *   offsets      device, experts + 1 row numbers (int32), not decreasing, within 0 .. M: read on the device, as for lutq_mx4_matmul_grouped
 *   Y            [M, N]; rows before offsets[0] and from offsets[experts] on stay as they were
 *   workspace    >= lutq_fp8_workspace_bytes(M, N, K, experts)
 * 1 <= experts <= 65536.  Everything else as for lutq_fp8_matmul. */
lutq_status lutq_fp8_matmul_grouped(const void* X, const float* x_scales, const void* W, const float* w_scales, const int32_t* offsets,
                                    int64_t experts, int64_t M, int64_t N, int64_t K, lutq_dtype dtype, void* Y, void* workspace,
                                    size_t workspace_bytes, void* stream);

typedef enum {
    LUTQ_SILU = 0,             /* g / (1 + exp(-g)) */
    LUTQ_GELU = 1              /* g / 2 (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) */
} lutq_activation;

/* The gated block's projections, activation and product, fused: with G and U the two halves of the rows of X W^T,
 *        H[m, f] = act(G[m, f]) * U[m, f],  G = X W[0 .. F - 1]^T,  U = X W[F .. 2 F - 1]^T
 *   X, x_scales          as for lutq_fp8_matmul;  W, w_scales  WEIGHTS [2 F, K], the gate's rows first
 *   H                    device, [M, F], dtype, or NULL
 *   h_codes, h_scales    device, or NULL: ROWS [M, F], what lutq_fp8_quantize makes of H of `dtype`, ready for the down projection's product.
 *                        H, these, or all of them
 *   saved                device, [M, 2 F], dtype, or NULL: G and U side by side, for lutq_fp8_gated_grad
 *   workspace            >= lutq_fp8_gated_workspace_bytes(M, F, K, 1), as for lutq_fp8_matmul
 * The projections and H are one launch; G and U go through memory only as `saved`, and as partial sums where a small H has K cut into slices.  X of 16 bits
 * and many rows is quantised by a launch before it, and H by one behind it, from H (where H is not asked for, from the workspace).
 * With h_codes or saved the sums are exact at any number of rows (above): a last bit of G or U that differs becomes a whole step of a code where H or the
 * gradients are quantised.  With few rows that costs nothing, with many up to twice the time and a little more (2 F x K, rows: 2816 x 1152, 300: 1.4 times;
 * 27648 x 5120, 2048: 1.75; 28672 x 4096, 512 to 8192: 1.9 to 2.1).  H may differ in its last bits from that of a call without either, and whoever would
 * rather have the codes of that H sooner takes it at 16 bits and gives it to lutq_fp8_quantize.
 * Errors: those of lutq_fp8_matmul; DTYPE also for an activation that there is not.
 * By expert (lutq_fp8_gated_grouped; W: `experts` of them) as for lutq_fp8_matmul_grouped: rows outside stay in every output. */
lutq_status lutq_fp8_gated(const void* X, const float* x_scales, const void* W, const float* w_scales, int64_t M, int64_t F, int64_t K,
                           lutq_activation activation, lutq_dtype dtype, void* H, void* h_codes, float* h_scales, void* saved,
                           void* workspace, size_t workspace_bytes, void* stream);
lutq_status lutq_fp8_gated_grouped(const void* X, const float* x_scales, const void* W, const float* w_scales, const int32_t* offsets,
                                   int64_t experts, int64_t M, int64_t F, int64_t K, lutq_activation activation, lutq_dtype dtype, void* H,
                                   void* h_codes, float* h_scales, void* saved, void* workspace, size_t workspace_bytes, void* stream);

/* Its backward pass, first part: from dH and the saved G, U the gradients of both,
 *        dG = dH * U * act'(G),  dU = dH * act(G),
 * side by side [M, 2 F], in any of three forms (at least one; the others NULL):
 *   dense_out                       device, [M, 2 F], dtype
 *   codes_out, scales_out           device, ROWS [M, 2 F]: lutq_fp8_matmul of them and the transposed weights [K, 2 F] is the gradient of X
 *   columns_out, column_scales_out  device, COLUMNS (codes [2 F, M']): one factor of the gradient of the weights
 * The quantised forms are made of the 32-bit gradients.  saved may come from any program that has G and U (e.g. from H's rows by expert).
 * Asynchronous on `stream`.  Errors: NULL (also for scales without codes), SHAPE (also for columns of no rows), DTYPE, ALIGN, DEVICE. */
lutq_status lutq_fp8_gated_grad(const void* dH, const void* saved, int64_t M, int64_t F, lutq_activation activation, lutq_dtype dtype,
                                void* dense_out, void* codes_out, float* scales_out, void* columns_out, float* column_scales_out,
                                void* stream);

/* Second part, the gradient of any product's weights: dW[n, k] = sum_m dY[m, n] * X[m, k], rounded once to `dtype`.
 *   dY, dy_scales   device, COLUMNS of the gradient of Y: codes [N, M], scales [M / 128, N]
 *   X, x_scales     device, COLUMNS of X: codes [K, M], scales [M / 128, K]
 *   M               rows, with those that fill them up: a multiple of 128, from 128 to 2^22 (they are the product's K; gradients of more are added up by
 *                   the caller)
 *   dW              device, [N, K], dtype; fully overwritten
 *   workspace       >= lutq_fp8_workspace_bytes(N, K, M, 1), as for lutq_fp8_matmul
 * N and K multiples of 16, K up to 2^24, N * M / 128 < 2^30.  The scales have to be powers of two from 2^-126 on (or not a number), as the quantiser of columns makes them: the matrix
 * instruction takes their exponents.  Errors: those of lutq_fp8_matmul; SHAPE for M = 0, too. */
lutq_status lutq_fp8_weight_grad(const void* dY, const float* dy_scales, const void* X, const float* x_scales, int64_t N, int64_t K, int64_t M,
                                 lutq_dtype dtype, void* dW, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LUTQ_H */
