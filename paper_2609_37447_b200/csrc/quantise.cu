// az_quantise_blocks: numbers -> e4m3 codes with one float32 scale for each block of 128 columns (of one row, or of
// 128 rows).
//
//   s = max(max |x| / 448, 2^-126),  code = e4m3(x / s) with the REAL quotient rounded once.
//
// A float32 division would round twice (the quotient to 24 bits, then to e4m3's 4) and differ from the definition where
// the quotient lies within half a step of the middle between two codes.
//
// float32 x: about one element in 10^6.  x is multiplied by 1/s shrunk and stretched by 2^-20 and both products are converted: the
// real quotient lies between them, so equal codes are the code.  Where they differ, the sign of |x| - middle * s, exact in
// one fused multiply-add, says which of the two it is.
//
// 16-bit x: one element in a few hundred, but for one reason.  With a the block's largest magnitude and ' the 11-bit integers
// that x and a are up to a power of two, x / (a / 448) equals a middle (5 bits) only if 7 x' = middle' a' 2^i, and misses it by
// 2^-16 of itself or more otherwise.  x / s is that quotient moved by the rounding of s alone: by up to 2^-24, to the same side
// for the whole block.  So a quotient that is right to 2^-22 (and exact where it is a middle: a product with 1/s and one Newton
// correction) is moved by 2^-20 to that side, or not at all where s = a / 448 exactly, and converted.  Four packed operations per
// two elements and no branch (with the float32 method, the second step was taken by nearly every warp: 56.6 us for
// 8192 x 8192 instead of 39.4).
//
// Bound by instruction issue and HBM about alike: a block is read once, held in registers and written once.  8192 x 8192 bf16:
// 39.3 us, 5.2 TB/s (79 % of the measured copy bandwidth); 128 x 128 blocks of 11003 x 4100 float32: 40.7 us, 5.5 TB/s (84 %); on the
// device, in a graph of calls.  Call by call, into outputs allocated each time: 41.7 and 44.9 us.
#include "common.cuh"
#include "ptx.cuh"

#include <cuda_fp16.h>

#include "az_tokens.h"

namespace az {
namespace {

constexpr int kBlock = AZ_QUANT_BLOCK;
constexpr int kPer = 16;                        // elements of a block that one thread holds; eight threads hold a row of it
constexpr int kLanes = kBlock / kPer;
constexpr int kThreads = 256, kTileThreads = 512;
constexpr int kGroups = kThreads / kLanes;      // rows of blocks in flight per step of a CTA

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// Sixteen elements of a row's block, as they are stored.  kVec: consecutive ones from 16- or 32-byte loads; else every eighth,
// one by one.
template <typename T, bool kVec>
struct Slice {
    uint4 raw[sizeof(T) * kPer / 16];

    __device__ static __forceinline__ int column(int lane, int j) { return kVec ? lane * kPer + j : lane + j * kLanes; }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * kPer / 16); ++i) raw[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load(const T *row, int lane, int cols) {
        if (kVec && lane * kPer + kPer <= cols) {
            const uint4 *src = reinterpret_cast<const uint4 *>(row + lane * kPer);
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) * kPer / 16); i += 2) {
                if ((reinterpret_cast<uintptr_t>(src) & 31) == 0) ptx::ld_global_once_v8(src + i, raw[i], raw[i + 1]);
                else { raw[i] = ptx::ld_global_once_v4(src + i); raw[i + 1] = ptx::ld_global_once_v4(src + i + 1); }
            }
        } else {
            T v[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = column(lane, j) < cols ? row[column(lane, j)] : T(0.0f);
            memcpy(raw, v, sizeof raw);
        }
    }
    __device__ __forceinline__ float at(int j) const {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(raw);
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
        const unsigned short h = (unsigned short)(w[j / 2] >> (16 * (j & 1)));
        return to_f32(*reinterpret_cast<const T *>(&h));
    }
    // the largest magnitude as the bits of a float: ordered as integers, NaN above infinity
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(raw);
        if constexpr (sizeof(T) == 4) {
            uint32_t t = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) t = max(t, w[j] & 0x7fffffffu);
            return t;
        } else {
            uint32_t t = 0;                     // two 16-bit magnitudes side by side
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) t = __vmaxu2(t, w[j] & 0x7fff7fffu);
            const unsigned short h = (unsigned short)max(t & 0xffffu, t >> 16);
            return __float_as_uint(to_f32(*reinterpret_cast<const T *>(&h))) & 0x7fffffffu;
        }
    }
};

struct Scale {
    float s, inv;                               // inv: 1 / s to within 2^-23
    float side;                                 // 16-bit inputs: 1 and the block's move
};

__device__ __forceinline__ Scale make_scale(uint32_t top) {
    Scale r;
    const float a = __uint_as_float(top), t = __fdiv_rn(a, 448.0f);
    const bool floor = t < 1.17549435e-38f;                   // (a NaN is not: it stays)
    r.s = floor ? 1.17549435e-38f : t;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.inv) : "f"(r.s));
    const float rest = fmaf(-448.0f, r.s, a);                 // exact; a power of two as the scale divides exactly
    r.side = floor || !(rest != 0.0f) ? 1.0f : rest > 0.0f ? 1.0f + 0x1p-20f : 1.0f - 0x1p-20f;
    return r;
}

// which of two neighbouring codes x / s has (the larger magnitude: high)
__device__ __forceinline__ uint32_t decide(float x, float s, uint32_t low, uint32_t high) {
    float a, b;
    ptx::unpack_e4m3x2((low & 0x7fu) | (high & 0x7fu) << 8, a, b);
    const float by = s < 1.0f ? 0x1p64f : 1.0f;               // (keeps the difference a normal number)
    const float rest = fmaf(-0.5f * (a + b), s * by, fabsf(x) * by);
    return rest < 0.0f || (rest == 0.0f && !(low & 1u)) ? low : high;
}

__device__ __forceinline__ uint32_t pack4(float2 a, float2 b) {
    return ptx::pack_e4m3x2(a.x, a.y) | (ptx::pack_e4m3x2(b.x, b.y) << 16);
}

template <bool kVec>
__device__ __forceinline__ void encode(const Slice<float, kVec> &x, const Scale &sc, uint32_t (&out)[kPer / 4]) {
    const float low = sc.inv * (1.0f - 0x1p-20f), high = sc.inv * (1.0f + 0x1p-20f);
    const float2 low2 = make_float2(low, low), high2 = make_float2(high, high);
#pragma unroll
    for (int w = 0; w < kPer / 4; ++w) {
        const float2 v0 = make_float2(x.at(4 * w), x.at(4 * w + 1)), v1 = make_float2(x.at(4 * w + 2), x.at(4 * w + 3));
        out[w] = pack4(ptx::mul2(v0, low2), ptx::mul2(v1, low2));
        const uint32_t other = pack4(ptx::mul2(v0, high2), ptx::mul2(v1, high2));
        if (out[w] != other) {
            const uint32_t lows = out[w];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = (lows >> (8 * i)) & 0xffu, b = (other >> (8 * i)) & 0xffu;
                if (a != b) out[w] += (decide(x.at(4 * w + i), sc.s, a, b) - a) << (8 * i);
            }
        }
    }
}

template <typename T, bool kVec>
__device__ __forceinline__ void encode(const Slice<T, kVec> &x, const Scale &sc, uint32_t (&out)[kPer / 4]) {
    // a small scale: x and s scaled up, exactly, so that x - q s is no subnormal number
    const bool small = sc.s < 0x1p-60f;
    const float s = small ? sc.s * 0x1p64f : sc.s, inv = small ? sc.inv * 0x1p-64f : sc.inv;
    // (s infinite or NaN: no correction, which would make NaN of the zeros)
    const float back = s < INFINITY ? -s : 0.0f, inv1 = s < INFINITY ? inv : 0.0f;
    const float2 inv2 = make_float2(inv, inv), back2 = make_float2(back, back), inv12 = make_float2(inv1, inv1), side2 = make_float2(sc.side, sc.side);
    auto quotients = [&](int j) {
        float2 v = make_float2(x.at(j), x.at(j + 1));
        if (small) v = ptx::mul2(v, make_float2(0x1p64f, 0x1p64f));
        const float2 q = ptx::mul2(v, inv2);
        return ptx::mul2(ptx::fma2(ptx::fma2(q, back2, v), inv12, q), side2);
    };
#pragma unroll
    for (int w = 0; w < kPer / 4; ++w) out[w] = pack4(quotients(4 * w), quotients(4 * w + 2));
}

template <typename T, bool kVec>
__device__ __forceinline__ void store(unsigned char *row, int lane, int cols, const uint32_t (&code)[kPer / 4]) {
    if (kVec && lane * kPer + kPer <= cols) {
        *reinterpret_cast<uint4 *>(row + lane * kPer) = make_uint4(code[0], code[1], code[2], code[3]);
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = Slice<T, kVec>::column(lane, j);
            if (c < cols) row[c] = (unsigned char)(code[j / 4] >> (8 * (j & 3)));
        }
    }
}

struct Args {
    const void *x;
    unsigned char *codes;
    float *scales;
    long long x_stride, codes_stride, scales_stride;
    int rows, cols, col_blocks;
};

// One row per block.  Blocks are numbered along the rows; a CTA takes kSteps * kGroups consecutive ones and has all of
// their loads in flight before it reduces the first.
constexpr int kSteps = 2;

template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads) quantise_rows_kernel(const Args a) {
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    // the CTA's first block by one division in 64 bits, the others from it in 32
    const long long first = (long long)blockIdx.x * (kSteps * kGroups);
    const long long row0 = first / a.col_blocks;
    const uint32_t col0 = (uint32_t)(first - row0 * a.col_blocks);
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    Slice<T, kVec> x[kSteps];
    long long row[kSteps];
    int block[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const uint32_t c = col0 + (uint32_t)(i * kGroups + group);
        const uint32_t down = c / (uint32_t)a.col_blocks;
        row[i] = row0 + down;
        block[i] = (int)(c - down * (uint32_t)a.col_blocks);
        if (row[i] < a.rows) x[i].load(static_cast<const T *>(a.x) + row[i] * a.x_stride + block[i] * kBlock, lane, a.cols - block[i] * kBlock);
        else x[i].clear();
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        uint32_t top = x[i].top();
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (row[i] >= a.rows) continue;                    // (the eight threads of a block alike)
        const Scale sc = make_scale(top);
        uint32_t code[kPer / 4];
        encode(x[i], sc, code);
        store<T, kVec>(a.codes + row[i] * a.codes_stride + block[i] * kBlock, lane, a.cols - block[i] * kBlock, code);
        if (lane == 0) a.scales[row[i] * a.scales_stride + block[i]] = sc.s;
    }
}

// 128 rows per block: one CTA holds the whole block, two rows of a column slice per thread (with four and half the threads, too few
// loads are in flight: 46.2 us instead of 41.2 for 11003 x 4100 float32).
template <typename T, bool kVec>
__global__ void __launch_bounds__(kTileThreads) quantise_tiles_kernel(const Args a) {
    __shared__ uint32_t tops[kTileThreads / 32];
    constexpr int kGroups = kTileThreads / kLanes, kRows = kBlock / kGroups;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const long long tile = blockIdx.x;
    const long long tile_row = tile / a.col_blocks;
    const int c0 = (int)(tile - tile_row * a.col_blocks) * kBlock;
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    Slice<T, kVec> x[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const long long r = tile_row * kBlock + i * kGroups + group;
        if (r < a.rows) x[i].load(static_cast<const T *>(a.x) + r * a.x_stride + c0, lane, a.cols - c0);
        else x[i].clear();
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) top = max(top, x[i].top());
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileThreads / 32; ++w) top = max(top, tops[w]);
    const Scale sc = make_scale(top);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const long long r = tile_row * kBlock + i * kGroups + group;
        if (r >= a.rows) break;
        uint32_t code[kPer / 4];
        encode(x[i], sc, code);
        store<T, kVec>(a.codes + r * a.codes_stride + c0, lane, a.cols - c0, code);
    }
    if (threadIdx.x == 0) a.scales[tile_row * a.scales_stride + c0 / kBlock] = sc.s;
}

template <typename T>
int launch(const Args &a, int block_rows, cudaStream_t s) {
    // vector loads and stores where every row starts on a 16-byte boundary
    const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.rows == 1 || (a.x_stride * (long long)sizeof(T) & 15) == 0) &&
                     (reinterpret_cast<uintptr_t>(a.codes) & 15) == 0 && (a.rows == 1 || (a.codes_stride & 15) == 0);
    const long long tiles = block_rows == 1 ? ((long long)a.rows * a.col_blocks + kSteps * kGroups - 1) / (kSteps * kGroups)
                                            : (((long long)a.rows + kBlock - 1) / kBlock) * a.col_blocks;
    if (tiles > 0x7fffffffll) return AZ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles), block(kThreads);
    if (block_rows == 1) {
        if (vec) AZ_CUDA(launch_dependent(quantise_rows_kernel<T, true>, grid, block, 0, s, a));
        else AZ_CUDA(launch_dependent(quantise_rows_kernel<T, false>, grid, block, 0, s, a));
    } else {
        if (vec) AZ_CUDA(launch_dependent(quantise_tiles_kernel<T, true>, grid, dim3(kTileThreads), 0, s, a));
        else AZ_CUDA(launch_dependent(quantise_tiles_kernel<T, false>, grid, dim3(kTileThreads), 0, s, a));
    }
    return AZ_OK;
}

}  // namespace
}  // namespace az

extern "C" int az_quantise_blocks(const void *x_dev, int x_type, int rows, int cols, int64_t x_stride, int block_rows,
                                  void *codes_dev, int64_t codes_stride, float *scales_dev, int64_t scales_stride, void *cuda_stream) {
    if (rows < 0 || cols < 0 || x_type < AZ_TYPE_F32 || x_type > AZ_TYPE_F16 || (block_rows != 1 && block_rows != AZ_QUANT_BLOCK)) return AZ_ERR_BAD_ARG;
    if (rows == 0 || cols == 0) return AZ_OK;
    if (!x_dev || !codes_dev || !scales_dev) return AZ_ERR_BAD_ARG;
    const int col_blocks = (int)(((int64_t)cols + az::kBlock - 1) / az::kBlock);
    const int scale_rows = (int)(((int64_t)rows + block_rows - 1) / block_rows);
    // (a single row has no next one: its stride is not looked at)
    if (rows > 1 && (x_stride < cols || codes_stride < cols)) return AZ_ERR_BAD_ARG;
    if (scale_rows > 1 && scales_stride < col_blocks) return AZ_ERR_BAD_ARG;
    const uintptr_t element = x_type == AZ_TYPE_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(x_dev) & (element - 1)) || (reinterpret_cast<uintptr_t>(scales_dev) & 3)) return AZ_ERR_BAD_ARG;
    az::Args a;
    a.x = x_dev; a.codes = static_cast<unsigned char *>(codes_dev); a.scales = scales_dev;
    a.x_stride = x_stride; a.codes_stride = codes_stride; a.scales_stride = scales_stride;
    a.rows = rows; a.cols = cols; a.col_blocks = col_blocks;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (x_type == AZ_TYPE_F32) return az::launch<float>(a, block_rows, s);
    if (x_type == AZ_TYPE_BF16) return az::launch<__nv_bfloat16>(a, block_rows, s);
    return az::launch<__half>(a, block_rows, s);
}
