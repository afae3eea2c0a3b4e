// az_block_matmul: out = a b^T for e4m3 operands with a float32 scale for every 128 columns of a row of a and for every
// 128 x 128 block of b.
//
//   out[i][j] = sum_c sa[i][c] sb[j/128][c] D_c[i][j],   D_c[i][j] = sum_{k in block c} a[i][k] b[j][k]
//
// The tensor cores compute D_c, one block of 128 k at a time, into its own columns of TMEM (kind::f8f6f4, fp32); warps of their
// own read it back, multiply it by the block's scales and add it up in registers while the tensor cores are at the next block.
// A thread holds one row of the tile, so a block costs it one scale and one fused multiply-add per column (turned: below).
//
// What the large form waits for is the way of a block's columns around (product, "done", read and add up, "free", next product) and
// the clock under the power limit; how much for each has not been measured apart (the tensor pipe is 50 % active without the limit).
// TMEM holds two blocks of 256 columns; so that the tensor cores wait little, a block is two products of 128 columns, each with its
// own "done" and "free" (a slot), the slot is free as soon as its last columns are in registers, scales are in registers
// before the block is done, and signals are single predicated instructions.
// Measured on the device, a dozen calls in a graph: 8192^3 470 to 550 us (2.0 to 2.3 PFLOP/s, as far as the SM clock falls under
// power: 1.4 to 1.6 GHz; a library product with ONE scale for each operand, which has nothing to add up, takes 362), 77 x 131072 x
// 4096 94 to 98 us (5.7 to 5.9 TB/s, 87 to 90 % of the measured copy bandwidth), 1024 x 1858 x 2048 with float32 results 10.3 us
// (operands from L2: 63 bytes a cycle and SM), 1 x 131072 x 4096 81 to 85 us (6.3 to 6.6 TB/s), 1 x 4096 x 4096 6.3 us (launch, first
// copies and the exchange).  Call after call for seconds, at the power limit: 8192^3 546 us, 77 x 131072 x 4096 114 us (4.9 TB/s).
//
// Operands come by TMA (128-byte swizzle: a tile row is exactly one block of k).  Rows and columns beyond the matrices are
// filled with zeros by the copy.  A tile of a is as many rows as there are (rounded up to sixteen, at most 128): rows of the
// product beyond them are computed from whatever the shared memory holds and read by nobody.
//
// Three forms of one kernel:
//   pairs   clusters of two CTAs on 256 x 256 tiles (tcgen05 .cta_group::2): each CTA brings its own 128 rows of a and half of the
//           tile's rows of b, and holds 128 x 256 of the result.  For many rows, where the tensor cores are the bound.
//   single  128 x 128 tiles.  For some rows, where the stream of b from memory is the bound.
//   turned  the same for at most 64 rows, as out^T = b a^T: the tensor cores take 128 rows of b against the 16 to 64 of a, not against
//           128 of which most are not there.  The stream of b at full rate brings the chip to its power limit, and what is computed
//           for nothing lowers the clock: 1300 MHz against 1860 MHz for 8 x 131072 x 4096.  A thread's sums are rows of a, so every
//           sum has a factor of its own, from shared memory; with more rows that costs more than it saves.
// Where the tiles alone cannot fill the SMs, a cluster shares one tile (single, turned), each CTA summing its own blocks of k; the
// partial sums travel through distributed shared memory, every CTA adding up its share of the columns in the order of the ranks.
#include "common.cuh"
#include "ptx.cuh"

#include <cuda.h>
#include <cuda_fp16.h>
#include <mutex>

#include "az_tokens.h"

namespace az {
namespace {

constexpr int kBlockK = AZ_QUANT_BLOCK;        // codes of a row in a pipeline stage: one scale, 128 bytes
constexpr int kTileM = 128;                     // rows of a, and of b, that a CTA brings
constexpr int kSums = 8;                        // warps that add up the blocks: four lane quarters of TMEM x kParts parts of the columns
constexpr int kParts = kSums / 4;
constexpr int kFirstSum = 4;                    // producer, issuer and two that fetch scales; the sums are whole warpgroups
constexpr int kThreads = 32 * (kFirstSum + kSums);
constexpr int kMaxStages = 12;
constexpr int kSlotCols = 128;                  // of TMEM: a block's products for 128 columns of the result
constexpr int kSlots = (int)(512 / kSlotCols);
constexpr int kScaleBlocks = 8;                 // blocks whose scales are fetched together (32 bytes of a row)
constexpr int kScalePitch = kTileM + 4;         // floats from one block's scales of the tile's rows to the next one's (no bank twice)
constexpr int kScaleFloats = kScaleBlocks * (kScalePitch + 2);     // of the rows; of the tile's two column blocks
constexpr uint32_t kTmemCols = 512;
constexpr int kMaxSplit = 8;
constexpr int kMaxExtent = 0x7fffff00;         // of m, n and k: indices rounded up to a tile stay in 31 bits
constexpr uint32_t kSpinLimit = 1u << 24;

constexpr int kSmemMax = 232448;
constexpr int kBarBytes = 1024;                 // barriers, TMEM address, abort flag; then the tiles, on a 1024-byte boundary; then
enum Form { kPairs, kSingle, kFew };             // of the kernel: see above
constexpr int scale_buffers(Form form) { return form == kFew ? 4 : 2; }       // fetches of scales (the other forms' sums hand theirs back at once)
constexpr int scale_bytes(Form form) { return scale_buffers(form) * kScaleFloats * 4; }       // then the exchange or the staging
constexpr int kExchangePad = 4;
constexpr int kStagingRow = 64;                 // bytes of a row that leave together
constexpr int kStagingBytes = 32 * kStagingRow; // per sums warp
constexpr int kStagingAll = kSums * kStagingBytes;
constexpr int kPiece = 16;                      // turned: rows of a that are read together; a part sums up one or two such pieces
constexpr int kFewRows = kParts * 2 * kPiece;
constexpr int kGroupRows = 8;                   // row tiles that are walked together, so that their operands meet in L2

__device__ uint32_t g_status;

struct Args {
    const float *sa, *sb, *bias;
    void *out;
    long long sa_stride, sb_stride, out_stride;
    int m, n, k_blocks;
    int out_type;
    int tiles_m, tiles_n;
    int tiles;
    int a_rows, stages, split, width_log2;        // width: columns that a CTA of a shared tile adds up
};

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int k, int row, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(k), "r"(row), "r"(bar) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// first row and column of a tile.  Tiles are numbered down groups of kGroupRows row tiles, then along the columns.
template <int kRows, int kCols>
__device__ __forceinline__ void place(const Args &a, int tile, int &m0, int &n0) {
    const int per_group = kGroupRows * a.tiles_n;
    const int group = tile / per_group;
    const int in_group = tile - group * per_group;
    const int height = min(kGroupRows, a.tiles_m - group * kGroupRows);
    const int col = in_group / height;
    m0 = (group * kGroupRows + in_group - col * height) * kRows;
    n0 = col * kCols;
}

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <typename T> struct Out;
template <> struct Out<float> {
    static constexpr int kPerWord = 1;
    __device__ static __forceinline__ uint32_t word(float a, float) { return __float_as_uint(a); }
};
template <> struct Out<__nv_bfloat16> {
    static constexpr int kPerWord = 2;
    __device__ static __forceinline__ uint32_t word(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
};
template <> struct Out<__half> {
    static constexpr int kPerWord = 2;
    __device__ static __forceinline__ uint32_t word(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
};

// Pairs, single: a warp's 32 rows x kCols columns (one row per thread) to global memory, 64 bytes of each row at a time through the
// warp's own 2 KB of shared memory, so that they leave as whole sectors: a thread's four 16-byte pieces go to places exchanged
// by the row's number (no bank twice), and come back four pieces of eight rows per instruction.
template <typename T, int kCols>
__device__ __forceinline__ void store_rows(const Args &a, unsigned char *staging, int row0, int col0, const float2 (&acc)[kCols / 2]) {
    constexpr int kPass = kStagingRow / (int)sizeof(T);    // columns per pass
    const int lane = threadIdx.x & 31;
    T *out = static_cast<T *>(a.out);
    const bool aligned = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(a.out_stride * (long long)sizeof(T))) & 15) == 0;
    const bool in_words = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(a.out_stride * (long long)sizeof(T))) & 3) == 0;
    auto at = [&](int row, int piece) { return staging + row * kStagingRow + ((piece ^ ((row >> 1) & 3)) << 4); };
#pragma unroll
    for (int c = 0; c < kCols; c += kPass) {
        if (col0 + c >= a.n) break;
#pragma unroll
        for (int piece = 0; piece < 4; ++piece) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = c + (piece * 4 + i) * Out<T>::kPerWord;      // column of the word's first element
                const float2 v = acc[j / 2];
                w[i] = sizeof(T) == 4 ? Out<T>::word(j & 1 ? v.y : v.x, 0.0f) : Out<T>::word(v.x, v.y);
            }
            *reinterpret_cast<uint4 *>(at(lane, piece)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
        if (aligned && col0 + c + kPass <= a.n) {
#pragma unroll
            for (int r = 0; r < 32; r += 8) {
                const int row = r + (lane >> 2), piece = lane & 3;
                const uint4 v = *reinterpret_cast<const uint4 *>(at(row, piece));
                if (row0 + row < a.m)
                    *reinterpret_cast<uint4 *>(out + (long long)(row0 + row) * a.out_stride + col0 + c + piece * (16 / (int)sizeof(T))) = v;
            }
        } else if (sizeof(T) == 2 && kCols == 128 && in_words && col0 + c + kPass <= a.n) {
            // rows of an even length that is no multiple of eight: two elements a piece, two rows per instruction (one by one, as below:
            // 121 us instead of 79 for 369 x 130374 x 577)
            uint32_t *dst = reinterpret_cast<uint32_t *>(out + (long long)(row0 + (lane >> 4)) * a.out_stride + col0 + c) + (lane & 15);
            const long long step = a.out_stride;           // words from a row to the one after the next
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 16) {
                uint32_t v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint32_t *>(at(r0 + 2 * i + (lane >> 4), (lane & 15) >> 2) + (lane & 3) * 4);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (row0 + r0 + 2 * i + (lane >> 4) < a.m) dst[(long long)(r0 / 2 + i) * step] = v[i];
            }
        } else {
            // one by one: 32 elements of a row per instruction, or 16 of two rows; eight instructions' loads together
            constexpr int kTogether = 32 / kPass, kBatch = 8;
            const int e = lane % kPass, byte = e * (int)sizeof(T);
            const bool inside = col0 + c + e < a.n;
            T *dst = out + (long long)(row0 + lane / kPass) * a.out_stride + col0 + c + e;
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += kBatch * kTogether) {
                T v[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) v[i] = *reinterpret_cast<const T *>(at(r0 + i * kTogether + lane / kPass, byte >> 4) + (byte & 15));
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (inside && row0 + r0 + i * kTogether + lane / kPass < a.m) dst[(long long)(r0 + i * kTogether) * a.out_stride] = v[i];
            }
        }
        __syncwarp();
    }
}

// Turned: a thread's rows of its column; a warp's elements of a row are neighbours
template <typename T, int kPieces>
__device__ __forceinline__ void store_turned(const Args &a, int row, int col, const float2 (&acc)[kPieces][8]) {
    if (col >= a.n) return;
    T *out = static_cast<T *>(a.out) + (long long)row * a.out_stride + col;
#pragma unroll
    for (int e = 0; e < kPieces * kPiece; ++e) {
        const float2 v = acc[e / kPiece][e % kPiece / 2];
        if (row + e < a.m) *out = from_f32<T>(e & 1 ? v.y : v.x);
        out += a.out_stride;
    }
}

__device__ __forceinline__ void store_out(void *out, int type, long long at, float v) {
    if (type == AZ_TYPE_F32) static_cast<float *>(out)[at] = v;
    else if (type == AZ_TYPE_BF16) static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
    else static_cast<__half *>(out)[at] = __float2half_rn(v);
}

// the barrier (pair: at this offset in both CTAs) arrives once the products issued so far have completed; by the elected lane
template <bool kPair>
__device__ __forceinline__ void commit_elect(uint32_t bar, uint32_t elected) {
    if (kPair)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %0, 0;\n@p tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%1], %2;\n}\n"
                     ::"r"(elected), "r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %0, 0;\n@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n}\n"
                     ::"r"(elected), "r"(bar) : "memory");
}
// an arrival by the lanes whose `yes` is not zero, without a branch
__device__ __forceinline__ void arrive_if(uint32_t yes, uint32_t bar) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %0, 0;\n@p mbarrier.arrive.shared::cta.b64 _, [%1];\n}\n" ::"r"(yes), "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_cluster_if(uint32_t yes, uint32_t cluster_bar) {     // relaxed: it publishes no writes
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %0, 0;\n@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%1];\n}\n" ::"r"(yes), "r"(cluster_bar) : "memory");
}

template <int kN>
__device__ __forceinline__ void add_columns(const uint32_t (&d)[kN], float2 scale, float2 *acc) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) acc[e / 2] = ptx::fma2(make_float2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), scale, acc[e / 2]);
}

template <Form kForm, int kPieces>
__global__ void __launch_bounds__(kThreads, 1)
block_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Args args) {
    constexpr bool kPair = kForm == kPairs, kTurned = kForm == kFew;
    constexpr int kRows = kPair ? 256 : 128, kCols = kPair ? 256 : 128;       // of a tile
    constexpr int kSumCols = kCols / kParts;                                  // pair: of a part
    constexpr int kSlotsPerBlock = kCols / kSlotCols, kBuffers = scale_buffers(kForm);
    extern __shared__ __align__(1024) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = ptx::smem_addr(smem);
    const uint32_t pad = (1024u - (smem_base & 1023u)) & 1023u;            // (the swizzle goes by address)
    const uint32_t bars = smem_base + pad;
    auto bar_full = [&](int s) { return bars + 8u * s; };
    auto bar_empty = [&](int s) { return bars + 8u * (kMaxStages + s); };
    auto bar_peer = [&](int s) { return bars + 8u * (2 * kMaxStages + s); };                      // pair, first CTA's: the second CTA's copies of stage s have landed
    auto bar_done = [&](int s) { return bars + 8u * (3 * kMaxStages + s); };                      // a block's products are in TMEM slot s
    auto bar_free = [&](int s) { return bars + 8u * (3 * kMaxStages + kSlots + s); };          // and have been read (pair: the first CTA's, by both)
    auto bar_scales = [&](int s) { return bars + 8u * (3 * kMaxStages + 2 * kSlots + s); };      // scales are in buffer s
    auto bar_scales_free = [&](int s) { return bars + 8u * (3 * kMaxStages + 2 * kSlots + 4 + s); };
    const uint32_t bar_drain = bars + 8u * (3 * kMaxStages + 2 * kSlots + 8);                  // after a failed wait: no product is in flight
    constexpr int kOffMisc = 8 * (3 * kMaxStages + 2 * kSlots + 9);
    static_assert(kOffMisc + 8 <= kBarBytes, "barriers");
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(smem + pad + kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + pad + kOffMisc + 4);
    const uint32_t tiles_at = bars + kBarBytes;
    // start addresses in matrix descriptors are offsets within THIS CTA's shared memory (inside a cluster a CTA's shared
    // addresses carry its rank in high bits)
    const uint32_t a_bytes = (uint32_t)args.a_rows * kBlockK;
    const uint32_t stage_bytes = a_bytes + kTileM * kBlockK;
    float *scales = reinterpret_cast<float *>(smem + pad + kBarBytes + (size_t)args.stages * stage_bytes);
    unsigned char *behind = reinterpret_cast<unsigned char *>(scales) + scale_bytes(kForm);
    float *exchange = reinterpret_cast<float *>(behind);                   // split: [rank][row][column], rows kExchangePad floats further apart
    const int split = kPair ? 1 : args.split;
    const int rank = kPair || split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const bool leader = !kPair || rank == 0;
    const int part = kPair ? 0 : rank;                                     // this CTA's blocks of k
    const int c_begin = (int)((long long)args.k_blocks * part / split), c_end = (int)((long long)args.k_blocks * (part + 1) / split);
    const int first_tile = (int)blockIdx.x / (kPair ? 2 : split), tile_step = (int)gridDim.x / (kPair ? 2 : split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < args.stages; ++s) { ptx::mbar_init(bar_full(s), 1); ptx::mbar_init(bar_empty(s), 1); ptx::mbar_init(bar_peer(s), 1); }
        for (int s = 0; s < kSlots; ++s) { ptx::mbar_init(bar_done(s), 1); ptx::mbar_init(bar_free(s), kSums); }
        for (int s = 0; s < kBuffers; ++s) { ptx::mbar_init(bar_scales(s), 2); ptx::mbar_init(bar_scales_free(s), kSums); }
        ptx::mbar_init(bar_drain, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 0 && lane == 0) { prefetch_map(&map_a); prefetch_map(&map_b); }
    if (warp == 1) {
        if (kPair) { ptx::tmem_alloc_pair(ptx::smem_addr(tmem_ptr), kTmemCols); ptx::tmem_relinquish_pair(); }
        else { ptx::tmem_alloc(ptx::smem_addr(tmem_ptr), kTmemCols); ptx::tmem_relinquish(); }
    }
    ptx::tc_fence_before();
    __syncthreads();
    // split: this CTA runs, its shared memory may be written after the matching wait.  Pair: nothing may reach into the other CTA
    // before its barriers exist
    if (kPair || split > 1) ptx::cluster_arrive();
    if (kPair) ptx::cluster_wait();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_ptr;
    ptx::grid_dependency_wait();
    ptx::launch_dependents();

    bool ok = true;
    // registers move from the first warpgroup to the others (launched with 3 x 168 for a thread of each; 88 + 2 x 208 asked for)
    if (warp < kFirstSum) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 0) {
            // ---- producer
            int s = 0;
            uint32_t phase = 0;
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step) {
                int row_a, row_b;
                place<kRows, kCols>(args, tile, row_a, row_b);
                if (kPair) { row_a += rank * kTileM; row_b += rank * (kTileM / kSlotsPerBlock); }
#pragma unroll 1
                for (int c = c_begin; c < c_end; ++c) {
                    ok = bounded_wait(bar_empty(s), phase ^ 1u, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (!ok) break;
                    if (lane == 0) {
                        const uint32_t at = tiles_at + (uint32_t)s * stage_bytes;
                        ptx::mbar_arrive_expect_tx(bar_full(s), stage_bytes);
                        tma_load(at, &map_a, c * kBlockK, row_a, bar_full(s));
                        // (pair: this CTA's rows of b are half of each slot's columns, so that a slot is 128 neighbouring columns)
                        for (int h = 0; h < kSlotsPerBlock; ++h)
                            tma_load(at + a_bytes + (uint32_t)(h * (kTileM / kSlotsPerBlock) * kBlockK), &map_b, c * kBlockK, row_b + h * kSlotCols, bar_full(s));
                    }
                    if (++s == args.stages) { s = 0; phase ^= 1u; }
                    __syncwarp();
                }
            }
            // after a failed wait let copies in flight land before the shared memory is released: stages below s were last filled in
            // this turn of the ring, the others in the one before
            for (int i = 0; !ok && i < args.stages; ++i)
                for (uint32_t p = 0; p < (1u << 20); ++p)
                    if (ptx::mbar_try_wait(bar_full(i), i < s ? phase : phase ^ 1u)) break;
        } else if (warp == 1 && !leader) {
            // ---- pair, second CTA: no products are issued here; tell the first CTA when a stage's copies have landed
            // (relaxed: the copies were written by the copy engine and are read by this CTA's own tensor core)
            int s = 0;
            uint32_t phase = 0;
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step)
#pragma unroll 1
                for (int c = c_begin; c < c_end; ++c) {
                    ok = bounded_wait(bar_full(s), phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (!ok) break;
                    if (lane == 0) ptx::mbar_arrive_cluster_relaxed(ptx::map_to_cta(bar_peer(s), 0));
                    if (++s == args.stages) { s = 0; phase ^= 1u; }
                    __syncwarp();
                }
        } else if (warp == 1) {
            // ---- issuer: four K = 32 steps per block, the first of which overwrites the slot
            // (barriers that threads of the pair's other CTA arrive on are waited for with acquire at cluster scope)
            const uint32_t idesc = ptx::idesc_e4m3_f32(kRows, kTurned ? args.a_rows : kSlotCols);
            // 128-byte swizzle (2 at bit 61), 8-row groups 1024 bytes apart, descriptor version 1
            constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t elected = ptx::elect_one();
            int s = 0, t = 0;
            uint32_t phase = 0, t_phase = 0;
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step)
#pragma unroll 1
                for (int c = c_begin; c < c_end; ++c) {
                    ok = bounded_wait(bar_full(s), phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (kPair) ok = ok && bounded_wait<true>(bar_peer(s), phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    const uint32_t at = tiles_at + (uint32_t)s * stage_bytes;
                    const uint32_t a_lo = ((at >> 4) & 0x3fffu) | (1u << 16), b_lo = (((at + a_bytes) >> 4) & 0x3fffu) | (1u << 16);
#pragma unroll
                    for (int h = 0; h < kSlotsPerBlock; ++h) {
                        ok = ok && bounded_wait<kPair>(bar_free(t), t_phase ^ 1u, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        const uint32_t b_half = b_lo + (uint32_t)(h * (kTileM / kSlotsPerBlock) * kBlockK >> 4);
#pragma unroll
                        for (int j = 0; j < kBlockK / 32; ++j) {
                            if (kPair) ptx::mma_e4m3_elect_pair(tmem + (uint32_t)(t * kSlotCols), a_lo + 2u * j, desc_hi, b_half + 2u * j, desc_hi, idesc, j > 0 ? 1u : 0u, elected);
                            else if (!kTurned) ptx::mma_e4m3_elect(tmem + (uint32_t)(t * kSlotCols), a_lo + 2u * j, desc_hi, b_half + 2u * j, desc_hi, idesc, j > 0 ? 1u : 0u, elected);
                            else ptx::mma_e4m3_elect(tmem + (uint32_t)(t * kSlotCols), b_lo + 2u * j, desc_hi, a_lo + 2u * j, desc_hi, idesc, j > 0 ? 1u : 0u, elected);
                        }
                        commit_elect<kPair>(bar_done(t), elected);
                        if (++t == kSlots) { t = 0; t_phase ^= 1u; }
                    }
                    if (!ok) break;
                    commit_elect<kPair>(bar_empty(s), elected);
                    if (++s == args.stages) { s = 0; phase ^= 1u; }
                    __syncwarp();
                }
            if (!ok) {
                if (elected) { if (kPair) ptx::mma_commit_pair(bar_drain); else ptx::mma_commit(bar_drain); }
                __syncwarp();
                for (uint32_t p = 0; p < (1u << 20); ++p)
                    if (ptx::mbar_try_wait(bar_drain, 0)) break;
            }
        } else if (warp >= 2) {
            // ---- scales: eight blocks of a row are one 32-byte sector, four rows a load; transposed on the way into shared memory, so
            // that the sums read consecutive words.  (Read in place by the sums, a warp's 32 rows were 32 accesses per block: 688 us
            // instead of 535 for 8192^3, everything else alike.)
            constexpr int kLoads = 8;
            const int block = lane & 7, at_row = (lane >> 3) + (warp - 2) * (kTileM / 2);
            const int last_block = (args.n - 1) / kBlockK;
            int u = 0;
            uint32_t u_phase = 0;
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step) {
                int m0, n0;
                place<kRows, kCols>(args, tile, m0, n0);
                if (kPair) m0 += rank * kTileM;
                for (int c0 = c_begin; c0 < c_end; c0 += kScaleBlocks) {
                    const int c = min(c0 + block, c_end - 1);
                    ok = bounded_wait(bar_scales_free(u), u_phase ^ 1u, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (!ok) break;
                    float *to = scales + u * kScaleFloats;
                    // (turned: one scale of b for the whole tile, multiplied in here)
                    const float by = !kTurned ? 1.0f : args.sb[(long long)(n0 / kBlockK) * args.sb_stride + c];
                    if (!kTurned && warp == 2 && lane < 16) to[kScaleBlocks * kScalePitch + lane] = args.sb[(long long)min(n0 / kBlockK + (lane >> 3), last_block) * args.sb_stride + c];
#pragma unroll 1
                    for (int i0 = 0; i0 < kTileM / 2; i0 += 4 * kLoads) {
                        if (kTurned && (warp - 2) * (kTileM / 2) + i0 >= args.a_rows) break;
                        float v[kLoads];
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) v[i] = args.sa[(long long)min(m0 + at_row + i0 + 4 * i, args.m - 1) * args.sa_stride + c];
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) to[block * kScalePitch + at_row + i0 + 4 * i] = kTurned ? v[i] * by : v[i];
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar_scales(u));
                    __syncwarp();
                    if (++u == kBuffers) { u = 0; u_phase ^= 1u; }
                }
            }
        }
        __syncwarp();
        if (!kPair && split > 1) {                          // (the sums' barriers, below)
            ptx::cluster_wait();
            ptx::cluster_arrive();
            ptx::cluster_wait();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int quarter = warp & 3, part_n = (warp - kFirstSum) >> 2;
        const uint32_t my_tmem = tmem + ((uint32_t)(quarter * 32) << 16);              // the lanes it may read
        const uint32_t first_lane = lane == 0;
        const int width = 1 << args.width_log2, pitch = width + kExchangePad;
        // partial sums, when they are in the exchange: CTA r adds up columns r * width .. of the tile (one tile per cluster)
        auto add_up = [&] {
            int m0, n0;
            place<kRows, kCols>(args, first_tile, m0, n0);
            const int rows = min(kTileM, args.m - m0);
            __syncwarp();
            ptx::cluster_arrive();
            ptx::cluster_wait();
            n0 += rank * width;
            if (!ok) return;
            for (int e = (warp - kFirstSum) * 32 + lane; e < rows << args.width_log2; e += kSums * 32) {
                const int row = e >> args.width_log2, col = e & (width - 1);
                if (n0 + col >= args.n) continue;
                const float *from = exchange + row * pitch + col;
                float sum = from[0];
#pragma unroll
                for (int r = 1; r < kMaxSplit; ++r)
                    if (r < split) sum += from[r * args.a_rows * pitch];
                store_out(args.out, args.out_type, (long long)(m0 + row) * args.out_stride + n0 + col, sum);
            }
        };
        if constexpr (!kTurned) {
            // ---- sums, pairs and single: this warp's 32 rows (the TMEM lanes it may read), half of the columns
            float2 acc[kSumCols / 2];
            const uint32_t my_columns = my_tmem + (uint32_t)(kPair ? 0 : part_n * kSumCols);
            const uint32_t leader_free = kPair ? ptx::map_to_cta(bar_free(0), 0) : 0;
            static_assert(kSumCols == (kPair ? kSlotCols : kSlotCols / kParts), "pair: a slot per part of the columns");
            int t = kPair ? part_n : 0, u = 0;                 // pair: every other slot is this part's
            uint32_t t_phase = 0, u_phase = 0;
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step) {
                int m0, n0;
                place<kRows, kCols>(args, tile, m0, n0);
                m0 += (kPair ? rank * kTileM : 0) + quarter * 32;
                const bool live = m0 < args.m;                         // of the whole warp
                const int col0 = n0 + part_n * kSumCols;
                if (args.bias && part == 0 && live) {
#pragma unroll
                    for (int j = 0; j < kSumCols / 2; ++j)
                        acc[j] = make_float2(args.bias[min(col0 + 2 * j, args.n - 1)], args.bias[min(col0 + 2 * j + 1, args.n - 1)]);
                } else {
#pragma unroll
                    for (int j = 0; j < kSumCols / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
                }
                for (int c0 = c_begin; c0 < c_end && ok; c0 += kScaleBlocks) {
                    ok = bounded_wait(bar_scales(u), u_phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (!ok) break;
                    float factor[kScaleBlocks];
                    {
                        const float *sa = scales + u * kScaleFloats + quarter * 32 + lane;
                        const float *sb = scales + u * kScaleFloats + kScaleBlocks * kScalePitch + (part_n * kSumCols / kBlockK) * kScaleBlocks;
#pragma unroll
                        for (int i = 0; i < kScaleBlocks; ++i) factor[i] = sa[i * kScalePitch] * sb[i];
                    }
                    __syncwarp();
                    arrive_if(first_lane, bar_scales_free(u));
                    if (++u == kBuffers) { u = 0; u_phase ^= 1u; }
#pragma unroll
                    for (int i = 0; i < kScaleBlocks; ++i) {
                        if (c0 + i >= c_end) break;
                        ok = __all_sync(0xffffffffu, ptx::mbar_try_wait(bar_done(t), t_phase)) ||
                             bounded_wait(bar_done(t), t_phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        const float2 scale = make_float2(factor[i], factor[i]);
                        const uint32_t at = my_columns + (uint32_t)(t * kSlotCols);
                        uint32_t d[2][16];
                        if (live) {
                            ptx::tmem_ld16(at, d[0]);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j + 16 < kSumCols; j += 16) {
                                ptx::tmem_ld16(at + (uint32_t)(j + 16), d[(j / 16 + 1) & 1]);
                                add_columns<16>(d[(j / 16) & 1], scale, acc + j / 2);
                                ptx::tmem_ld_wait();
                            }
                        }
                        // all of the slot is in registers: it is free before the last columns are added up
                        ptx::tc_fence_before();
                        if (kPair) arrive_cluster_if(first_lane, leader_free + 8u * t);
                        else arrive_if(first_lane, bar_free(t));
                        if (live) add_columns<16>(d[(kSumCols / 16 - 1) & 1], scale, acc + (kSumCols - 16) / 2);
                        t += kSlotsPerBlock;
                        if (t >= kSlots) { t -= kSlots; t_phase ^= 1u; }
                    }
                }
                if (ok && split == 1 && live) {
                    unsigned char *staging = behind + (warp - kFirstSum) * kStagingBytes;
                    if (args.out_type == AZ_TYPE_F32) store_rows<float, kSumCols>(args, staging, m0, col0, acc);
                    else if (args.out_type == AZ_TYPE_BF16) store_rows<__nv_bfloat16, kSumCols>(args, staging, m0, col0, acc);
                    else store_rows<__half, kSumCols>(args, staging, m0, col0, acc);
                }
            }
            if (!kPair && split > 1) {
                int m0, n0;
                place<kRows, kCols>(args, first_tile, m0, n0);
                const int rows = min(kTileM, args.m - m0);
                ptx::cluster_wait();                        // every CTA of the cluster runs
                if (quarter * 32 + lane < rows) {
                    const uint32_t here = ptx::smem_addr(exchange) + (uint32_t)((rank * args.a_rows + quarter * 32 + lane) * pitch) * 4u;
#pragma unroll
                    for (int j = 0; j < kSumCols; j += 4) {
                        const int col = part_n * kSumCols + j;
                        ptx::st_cluster_v4(ptx::map_to_cta(here + (uint32_t)(col & (width - 1)) * 4u, (uint32_t)(col >> args.width_log2)),
                                           __float_as_uint(acc[j / 2].x), __float_as_uint(acc[j / 2].y), __float_as_uint(acc[j / 2 + 1].x), __float_as_uint(acc[j / 2 + 1].y));
                    }
                }
                add_up();
            }
        } else {
            // ---- sums, turned: a thread has a column of out (a TMEM lane) and, by part, half of the tile's rows
            float2 acc[kPieces][8];                                     // pairs of rows
            int t = 0, u = 0;
            uint32_t t_phase = 0, u_phase = 0;
            int m0 = 0, col = 0;
            const int row = part_n * kPieces * kPiece;                  // first of the tile
            for (int tile = first_tile; tile < args.tiles && ok; tile += tile_step) {
                int n0;
                place<kRows, kCols>(args, tile, m0, n0);
                col = n0 + quarter * 32 + lane;
                const bool live = n0 + quarter * 32 < args.n && m0 + part_n * kPieces * kPiece < args.m;          // of the whole warp
                const float bias = args.bias && part == 0 ? args.bias[min(col, args.n - 1)] : 0.0f;
#pragma unroll
                for (int p = 0; p < kPieces; ++p)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[p][j] = make_float2(bias, bias);
                for (int c0 = c_begin; c0 < c_end && ok; c0 += kScaleBlocks) {
                    ok = bounded_wait(bar_scales(u), u_phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                    if (!ok) break;
                    const float *factors = scales + u * kScaleFloats + row;
#pragma unroll 1
                    for (int i = 0; i < kScaleBlocks && c0 + i < c_end; ++i, factors += kScalePitch) {
                        float4 f[kPieces][4];
#pragma unroll
                        for (int p = 0; p < kPieces; ++p)
#pragma unroll
                            for (int j = 0; j < 4; ++j) f[p][j] = *reinterpret_cast<const float4 *>(factors + p * kPiece + 4 * j);
                        ok = __all_sync(0xffffffffu, ptx::mbar_try_wait(bar_done(t), t_phase)) ||
                             bounded_wait(bar_done(t), t_phase, abort_flag, &g_status, kStatusWaitTimeout, kSpinLimit);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        const uint32_t at = my_tmem + (uint32_t)(t * kSlotCols + part_n * kPieces * kPiece);
                        uint32_t d[kPieces][kPiece];
                        if (live) {
#pragma unroll
                            for (int p = 0; p < kPieces; ++p) ptx::tmem_ld16(at + (uint32_t)(p * kPiece), d[p]);
                            ptx::tmem_ld_wait();
                        }
                        ptx::tc_fence_before();
                        arrive_if(first_lane, bar_free(t));
                        if (live) {
#pragma unroll
                            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    acc[p][j] = ptx::fma2(make_float2(__uint_as_float(d[p][2 * j]), __uint_as_float(d[p][2 * j + 1])), j & 1 ? make_float2(f[p][j / 2].z, f[p][j / 2].w) : make_float2(f[p][j / 2].x, f[p][j / 2].y), acc[p][j]);
                        }
                        if (++t == kSlots) { t = 0; t_phase ^= 1u; }
                    }
                    __syncwarp();
                    arrive_if(first_lane, bar_scales_free(u));
                    if (++u == kBuffers) { u = 0; u_phase ^= 1u; }
                }
                if (ok && split == 1 && live) {
                    if (args.out_type == AZ_TYPE_F32) store_turned<float>(args, m0 + row, col, acc);
                    else if (args.out_type == AZ_TYPE_BF16) store_turned<__nv_bfloat16>(args, m0 + row, col, acc);
                    else store_turned<__half>(args, m0 + row, col, acc);
                }
                __syncwarp();
            }
            if (split > 1) {
                ptx::cluster_wait();                        // every CTA of the cluster runs
                const int in_tile = quarter * 32 + lane;
                const uint32_t to = ptx::map_to_cta(ptx::smem_addr(exchange) + (uint32_t)((rank * args.a_rows + row) * pitch + (in_tile & (width - 1))) * 4u,
                                                    (uint32_t)(in_tile >> args.width_log2));
#pragma unroll
                for (int e = 0; e < kPieces * kPiece; ++e)
                    if (m0 + row + e < args.m) {
                        const float2 v = acc[e / kPiece][e % kPiece / 2];
                        ptx::st_cluster(to + (uint32_t)(e * pitch) * 4u, __float_as_uint(e & 1 ? v.y : v.x));
                    }
                add_up();
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    // neither CTA of a pair may leave (and release shared memory and TMEM that the pair's products and commits address) before
    // both are through
    if (kPair) { ptx::cluster_arrive(); ptx::cluster_wait(); }
    if (warp == 1) {
        ptx::tc_fence_after();
        if (kPair) ptx::tmem_dealloc_pair(tmem, kTmemCols);
        else ptx::tmem_dealloc(tmem, kTmemCols);
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder of tensor maps (the library is not linked against the driver)
int encoder(EncodeTiled *out) {
    static EncodeTiled found = nullptr;
    static std::mutex lock;
    std::lock_guard<std::mutex> hold(lock);
    if (!found) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult res = cudaDriverEntryPointSymbolNotFound;
        AZ_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &res));
        if (res != cudaDriverEntryPointSuccess || !fn) return AZ_ERR_UNSUPPORTED;
        found = reinterpret_cast<EncodeTiled>(fn);
    }
    *out = found;
    return AZ_OK;
}

// [rows][k] bytes, boxes of box_rows rows x 128 bytes
int make_map(CUtensorMap *map, const void *base, int rows, int k, int64_t stride, int box_rows) {
    EncodeTiled encode = nullptr;
    const int rc = encoder(&encode);
    if (rc != AZ_OK) return rc;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {(cuuint32_t)kBlockK, (cuuint32_t)box_rows};
    const cuuint32_t steps[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled"); return AZ_ERR_CUDA; }
    return AZ_OK;
}

template <Form kForm, int kPieces>
int launch_form(const CUtensorMap &map_a, const CUtensorMap &map_b, const Args &args, unsigned grid, size_t smem, int dev, cudaStream_t s) {
    static bool configured[64] = {};
    static std::mutex lock;
    {
        std::lock_guard<std::mutex> hold(lock);
        if (dev < 0 || dev >= 64 || !configured[dev]) {
            AZ_CUDA(cudaFuncSetAttribute(block_matmul_kernel<kForm, kPieces>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax));
            if (dev >= 0 && dev < 64) configured[dev] = true;
        }
    }
    const unsigned cluster = kForm == kPairs ? 2u : (unsigned)args.split;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    AZ_CUDA(cudaLaunchKernelEx(&cfg, block_matmul_kernel<kForm, kPieces>, map_a, map_b, args));
    return AZ_OK;
}

// how many clusters of 2, 4 or 8 CTAs with all of an SM's shared memory the device holds at a time (asked once)
int clusters_held(int dev, int size, int *held) {
    static int known[64][kMaxSplit + 1] = {};
    static std::mutex lock;
    std::lock_guard<std::mutex> hold(lock);
    int asked = 0;
    int &entry = dev >= 0 && dev < 64 ? known[dev][size] : asked;
    if (entry == 0) {
        auto kernel = block_matmul_kernel<kSingle, 0>;
        AZ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)size); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = kSmemMax;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)size; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        AZ_CUDA(cudaOccupancyMaxActiveClusters(&entry, kernel, &cfg));
        if (entry < 1) entry = 1;
    }
    *held = entry;
    return AZ_OK;
}

int launch(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int k, Args args, cudaStream_t s) {
    int dev = 0, sms = 0;
    AZ_CUDA(cudaGetDevice(&dev));
    AZ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    args.k_blocks = (k + kBlockK - 1) / kBlockK;
    const long long singles = (((int64_t)args.m + 127) / 128) * (((int64_t)args.n + 127) / 128);
    const long long pairs = (((int64_t)args.m + 255) / 256) * (((int64_t)args.n + 255) / 256);
    // pairs where they occupy three quarters of the SMs and b is read for more than three tiles of rows; us, pairs / single:
    //   2048 x 2048 x 2048 12.8 / 14.7, 1024 x 8192 x 2048 22.1 / 26.4, 8192^3 485 / 1445 (its first form);
    //   512 x 4096 x 4096 (32 tiles of pairs) 17.7 / 13.9, 1024 x 1858 x 2048 (32) 13.8 / 10.2;
    //   256 x 20000 x 4096 34.2 / 33.7, 300 x 40000 x 400 24.3 / 21.4, 129 x 20000 x 2048 21.7 / 20.3
    // 16-bit rows of an even length that is no multiple of eight are written two elements at a time by pairs and one by one by single:
    // pairs for them from more than one tile of rows on.  us, pairs / single: 369 x 130374 x 577 80.0 / 98.4, 300 x 40002 x 400
    // 27.7 / 34.4, 129 x 20002 x 2048 22.7 / 25.5, 380 x 50258 x 4096 105.5 / 105.9.  (Two at a time in single as well: 300 x 40002 x 400
    // 23.4, but registers become tight and rows of an odd length, written one by one, go from 34.4 to 41 for 300 x 40001 x 400.)
    const uintptr_t spread = reinterpret_cast<uintptr_t>(args.out) | (uintptr_t)(args.out_stride * 2);
    const bool by_words = args.out_type != AZ_TYPE_F32 && (spread & 15) != 0 && (spread & 3) == 0;
    const bool pair = args.m > (by_words ? 1 : 3) * kTileM && pairs * 8 >= sms * 3;
    // turned up to 64 rows, us for n x k, turned / single (131072 x 4096: held for half a second, the power limit reached):
    //   131072 x 4096   1 row 81.2 / 105.6, 32 rows 87.9 / 109.9, 64 rows 99.9 / 112.6, 77 rows (three pieces a part) 119.0 / 114.9
    //   20001 x 1000    5 rows 6.8 / 10.9, 33 rows 7.9 / 12.4, 64 rows 8.6 / 12.9;   4096 x 4096   1 row 6.7 / 7.4, 64 rows 9.1 / 10.2
    const Form form = pair ? kPairs : args.m <= kFewRows ? kFew : kSingle;
    const int tile = pair ? 256 : 128;
    args.tiles_m = (int)(((int64_t)args.m + tile - 1) / tile);
    args.tiles_n = (int)(((int64_t)args.n + tile - 1) / tile);
    args.tiles = (int)(pair ? pairs : singles);
    args.a_rows = args.m >= kTileM ? kTileM : (args.m + kPiece - 1) / kPiece * kPiece;
    // a cluster per tile, up to eight CTAs, as long as all clusters run at once (of eight CTAs 15 do, not 148 / 8; with
    // eight / four CTAs for 16 tiles, in us: 1 x 2048 x 8192 11.8 / 7.4, 128 x 2048 x 8192 24.4 / 14.1; without a split 1 x 4096 x 4096
    // took 12.2 instead of 7.0, as single), each with a block of k at least; single, where the exchange is larger, with four (128 x 1858
    // x 2048: 9.4, with two 11.8; 300 x 1024 x 1024: 9.4, with two 10.0)
    const int least = form == kSingle ? 4 : 1;
    args.split = 1;
    while (!pair && args.split < kMaxSplit && args.split * 2 * least <= args.k_blocks) {
        int held = 0;
        const int rc = clusters_held(dev, args.split * 2, &held);
        if (rc != AZ_OK) return rc;
        if (args.tiles > held) break;
        args.split *= 2;
    }
    const int stage_bytes = args.a_rows * kBlockK + kTileM * kBlockK;
    args.width_log2 = 7;
    while ((args.split << args.width_log2) > 128) --args.width_log2;
    const int behind = args.split > 1 ? args.split * args.a_rows * ((1 << args.width_log2) + kExchangePad) * 4 : form == kFew ? 0 : kStagingAll;
    const int room = kSmemMax - 1024 - kBarBytes - scale_bytes(form) - behind;
    args.stages = room / stage_bytes < kMaxStages ? room / stage_bytes : kMaxStages;
    const size_t smem = 1024 + kBarBytes + (size_t)args.stages * stage_bytes + scale_bytes(form) + behind;
    const int ctas = args.tiles * (pair ? 2 : args.split);
    const unsigned grid = (unsigned)(ctas < sms ? ctas : pair ? sms & ~1 : sms);
    CUtensorMap map_a, map_b;
    int rc = make_map(&map_a, a, args.m, k, a_stride, args.a_rows);
    if (rc == AZ_OK) rc = make_map(&map_b, b, args.n, k, b_stride, pair ? kTileM / 2 : kTileM);
    if (rc != AZ_OK) return rc;
    return form == kPairs    ? launch_form<kPairs, 0>(map_a, map_b, args, grid, smem, dev, s)
           : form == kSingle ? launch_form<kSingle, 0>(map_a, map_b, args, grid, smem, dev, s)
           : args.a_rows <= kFewRows / 2 ? launch_form<kFew, 1>(map_a, map_b, args, grid, smem, dev, s)
                                         : launch_form<kFew, 2>(map_a, map_b, args, grid, smem, dev, s);
}

// the status words of the calls of az_tokens.h on the current device: the product's, the logit calls'
int status_words(uint32_t *(&words)[2]) {
    AZ_CUDA(cudaGetSymbolAddress(reinterpret_cast<void **>(&words[0]), g_status));
    return logits_status_word(&words[1]);
}

__global__ void clear_bits_kernel(uint32_t *a, uint32_t a_bits, uint32_t *b, uint32_t b_bits) {
    atomicAnd(a, ~a_bits);
    atomicAnd(b, ~b_bits);
}

}  // namespace
}  // namespace az

extern "C" int az_block_matmul(const void *a_dev, int64_t a_stride, const float *a_scales_dev, int64_t a_scales_stride,
                               const void *b_dev, int64_t b_stride, const float *b_scales_dev, int64_t b_scales_stride,
                               const float *bias_dev, int m, int n, int k, void *out_dev, int out_type, int64_t out_stride,
                               void *cuda_stream) {
    if (m < 0 || n < 0 || k <= 0 || out_type < AZ_TYPE_F32 || out_type > AZ_TYPE_F16) return AZ_ERR_BAD_ARG;
    if (m == 0 || n == 0) return AZ_OK;
    if (m > az::kMaxExtent || n > az::kMaxExtent || k > az::kMaxExtent) return AZ_ERR_UNSUPPORTED;
    // (tiles are counted in 32 bits: of 256 x 256 where there are so many, at most 3 x 2^24 of 128 x 128 where there are 384 rows or fewer)
    if ((((int64_t)m + 255) / 256) * (((int64_t)n + 255) / 256) > 0x3fffffff) return AZ_ERR_UNSUPPORTED;
    if (!a_dev || !a_scales_dev || !b_dev || !b_scales_dev || !out_dev) return AZ_ERR_BAD_ARG;
    const uintptr_t element = out_type == AZ_TYPE_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(a_dev) & 15) || (reinterpret_cast<uintptr_t>(b_dev) & 15) ||
        (reinterpret_cast<uintptr_t>(a_scales_dev) & 3) || (reinterpret_cast<uintptr_t>(b_scales_dev) & 3) ||
        (reinterpret_cast<uintptr_t>(bias_dev) & 3) || (reinterpret_cast<uintptr_t>(out_dev) & (element - 1))) return AZ_ERR_BAD_ARG;
    // (a single row has no next one: its stride is not looked at)
    const int64_t k_blocks = ((int64_t)k + AZ_QUANT_BLOCK - 1) / AZ_QUANT_BLOCK, k_up = ((int64_t)k + 15) & ~(int64_t)15;
    const int64_t limit = (int64_t)1 << 39;                       // (a tensor map holds strides below 2^40 bytes)
    if (m == 1) { a_stride = k_up; a_scales_stride = k_blocks; out_stride = n; }
    if (n == 1) b_stride = k_up;
    if (n <= AZ_QUANT_BLOCK) b_scales_stride = k_blocks;
    if (a_stride < k || b_stride < k || (a_stride & 15) || (b_stride & 15) || a_stride > limit || b_stride > limit) return AZ_ERR_BAD_ARG;
    if (a_scales_stride < k_blocks || b_scales_stride < k_blocks || out_stride < n) return AZ_ERR_BAD_ARG;
    az::Args args = {};
    args.sa = a_scales_dev; args.sb = b_scales_dev; args.bias = bias_dev; args.out = out_dev;
    args.sa_stride = a_scales_stride; args.sb_stride = b_scales_stride; args.out_stride = out_stride;
    args.m = m; args.n = n; args.out_type = out_type;
    return az::launch(a_dev, a_stride, b_dev, b_stride, k, args, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int az_tokens_status(void *cuda_stream, uint32_t *status_out) {
    if (!status_out) return AZ_ERR_BAD_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    uint32_t *words[2] = {}, seen[2] = {0, 0};
    const int rc = az::status_words(words);
    if (rc != AZ_OK) return rc;
    for (int i = 0; i < 2; ++i) AZ_CUDA(cudaMemcpyAsync(&seen[i], words[i], sizeof(uint32_t), cudaMemcpyDeviceToHost, s));
    AZ_CUDA(cudaStreamSynchronize(s));
    *status_out = seen[0] | seen[1];
    if (*status_out == 0) return AZ_OK;
    // what this call reports is cleared, bit by bit, and nothing else: kernels on other streams may raise a bit at any time
    az::clear_bits_kernel<<<1, 1, 0, s>>>(words[0], seen[0], words[1], seen[1]);
    AZ_CUDA(cudaGetLastError());
    AZ_CUDA(cudaStreamSynchronize(s));
    return (*status_out & az::kStatusWaitTimeout) ? AZ_ERR_DEVICE_TIMEOUT : AZ_OK;
}

extern "C" int az_selftest_tokens_timeout(int part, void *cuda_stream) {
    if (part < 0 || part > 1) return AZ_ERR_BAD_ARG;
    uint32_t *words[2] = {};
    const int rc = az::status_words(words);
    return rc == AZ_OK ? az::raise_wait_timeout(words[part], static_cast<cudaStream_t>(cuda_stream)) : rc;
}
