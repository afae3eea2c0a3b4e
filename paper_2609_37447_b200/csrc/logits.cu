// az_adjust_logits, az_token_probs: penalties for repeated tokens, biases, temperature and masks on rows of logits, and the
// softmax under them.
//
//   t in the history         l = l > 0 ? l / r : l * r          t n > 0 times in the answer   l = (l - f n) - q
//   t in the bias list       l = l + b                          t not allowed                 l = -inf
//   p = exp((l - m) / T) / sum exp((l - m) / T),  m = max l
//
// One pass over the logits.  A cluster of CTAs shares a row, dealt out to them in turn in chunks of 256 elements (neighbouring
// tokens are alike frequent: with contiguous slices the first CTA did most of a history's work and the others waited for it); each CTA
// holds its slice in registers (32-bit floats).  Histories and biases touch few tokens, so they go through shared memory: a word per
// token of the slice and a bitmap of the words in use.
// Each CTA reads the whole history and counts the tokens of its slice (top bit: in the prompt; rest: times in the answer).  Counts
// are integers: the order of the atomics changes nothing.  Then the touched words are turned into the tokens' new logits, biases are
// added to them there, and the threads take them over into their registers.  (With the penalties computed in place in the
// registers, every thread walked through eight elements' worth of branches for one touched token in its warp: 200 us instead of
// 165 for 512 x 131072; with the history shared out and counted in the owner's shared memory across the cluster, frequent tokens
// queued up as remote atomics on one word: 20 us instead of 16 for one row with 30,000 tokens.)
// Each CTA reduces its slice to (max, lowest index, sum) with the sum relative to its OWN max; one exchange through distributed
// shared memory gives the row's max and sum, and a CTA's probabilities are its exponentials times one factor.
//
// Elements are addressed from the 16-byte boundary at or below the row's first one ("virtual index" v = t + head), so rows that
// start anywhere (an odd vocabulary) are still read in 16-byte loads; the first and last group of eight are read one by one.
//
// What bounds it: a row is a chain of latencies (parameters, history, biases, two barriers, the exchange), and two CTAs of an SM are all
// that there is to fill them.  Clusters stay for several rows: a row's logits, its parameters, mask, the first of its history
// and of its biases are copied into shared memory while the one before is worked on, and words and bits are cleared by those who take
// them over.  us on the device, in a graph of calls: 512 x 131072 bf16 162 to 177 with everything on (1.6 TB/s), 83 without rules
// (3.2 TB/s); 256 x 100277 bf16 adjusted 90 (32 without rules); 1 x 131072 with 30,000 tokens of history 16; 1024 x 1858 float32 with
// masks 7.2 (call by call, with three outputs to allocate, 9.0).
#include "common.cuh"
#include "ptx.cuh"

#include <cuda_fp16.h>
#include <mutex>

#include "az_tokens.h"

namespace az {
namespace {

constexpr int kPer = 8;                    // elements of a group: one thread's unit, 16 bytes of 16-bit logits
constexpr uint32_t kInPrompt = 0x80000000u;  // of a token's word; the other bits count
constexpr int kMaxCluster = 16;            // above 8 with the kernels' leave (non-portable cluster sizes)

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
__device__ __forceinline__ void pack8(const float (&x)[kPer], uint4 (&w)[2], float) { memcpy(w, x, sizeof w); }
__device__ __forceinline__ void pack8(const float (&x)[kPer], uint4 (&w)[1], __nv_bfloat16) {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
    memcpy(w, h, sizeof w);
}
__device__ __forceinline__ void pack8(const float (&x)[kPer], uint4 (&w)[1], __half) {
    __half2 h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __floats2half2_rn(x[2 * j], x[2 * j + 1]);
    memcpy(w, h, sizeof w);
}

struct Args {
    const void *logits;
    void *out;                             // adjusted logits or probabilities; null: not wanted
    int32_t *best;
    float *best_logprob;
    long long logits_stride, out_stride;
    int rows;
    uint32_t cluster_magic;                // c * cluster_magic >> 16 = c / cluster for the chunks of a row (at most 1100 of them)
    int vocab, cluster, span;              // span: elements that a row may take with its start moved to a 16-byte boundary
    int out_type;                          // AZ_TYPE_*: the logits' type or float32
    az_logit_rules r;
};

__device__ __forceinline__ float max_nan(float a, float b) {          // a NaN wins
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float warp_max_nan(float v) {
    float d;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(v));
    return d;
}
__device__ __forceinline__ float exp2_approx(float v) {               // off by 2^-22 of itself; results below 2^-126 are 0
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
    return d;
}
__device__ __forceinline__ void copy_async_16(uint32_t dst_smem, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst_smem), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_4(uint32_t dst_smem, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst_smem), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// is v the maximum m (found by max_nan), be it a NaN
__device__ __forceinline__ bool is_max(float v, float m) { return v == m || (m != m && v != v); }

template <typename O>
__device__ __forceinline__ void store_group(O *dst, const float (&x)[kPer]) {
    uint4 words[sizeof(O) * kPer / 16];
    pack8(x, words, O());
#pragma unroll
    for (int i = 0; i < (int)(sizeof(O) * kPer / 16); ++i) __stcs(reinterpret_cast<uint4 *>(dst) + i, words[i]);
}
// the elements of a group that are inside the row, one by one
template <typename O>
__device__ __forceinline__ void store_some(O *row, int v, int head, int end, const float (&x)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (v + j >= head && v + j < end) row[v - head + j] = from_f32<O>(x[j]);
}

__device__ uint32_t g_status;              // of the exchanges (az_tokens_status)

struct Part {                              // what a CTA knows of its row: its max, the max's lowest index, its sum
    float top;
    int index;
    float sum;
    uint32_t pad;
};

// kThreads * kItems groups of eight per CTA; kTabled: there are histories or biases
template <typename T, int kThreads, int kItems, bool kProbs, bool kTabled>
__global__ void __launch_bounds__(kThreads, kItems > 4 ? 1 : 1024 / kThreads) logits_kernel(const Args a) {
    extern __shared__ __align__(16) uint32_t table[];          // kThreads * kItems * 8 words, if there are histories or biases; the next logits
    __shared__ __align__(16) Part parts[2][kMaxCluster];       // (by the parity of the row's turn: a slow CTA may still read the last ones)
    __shared__ __align__(8) unsigned long long arrived[2];     // their bytes are in
    __shared__ uint32_t params[2][8];                          // of the row, by the parity of its turn
    __shared__ Part row_part;
    constexpr int kList = kThreads;
    __shared__ unsigned short list[kTabled ? kList : 1];       // words that the history has touched, in no order
    __shared__ int listed[2];                                  // how many (the list is cut off at kList), by the parity of the row's turn
    __shared__ int abort_flag;
    __shared__ float warp_tops[kThreads / 32], warp_sums[kThreads / 32];
    __shared__ int best_index[2];
    constexpr int kGroups = kThreads * kItems;
    constexpr int kSlice = kGroups * kPer;
    constexpr int kRaw = sizeof(T) * kPer / 16;                // 16-byte words of a group
    constexpr int kAlign = 16 / sizeof(T);
    constexpr int kTokens = 1;                                 // of the history per thread that are copied ahead
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cluster = a.cluster;
    const int rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
    constexpr int kWarps = kThreads / 32, kChunk = 32 * kPer, kChunks = kSlice / kChunk;
    // virtual index of the first element of the CTA's chunk number c, and of this thread's group number i (one of chunk i * kWarps + warp)
    auto chunk_at = [&](int c) { return (c * cluster + rank) * kChunk; };
    auto group_at = [&](int i) { return chunk_at(i * kWarps + warp) + lane * kPer; };
    const bool counting = kTabled && a.r.tokens != nullptr, biased = kTabled && a.r.bias_offsets != nullptr;
    uint32_t *touched = table + kSlice, *claimed = touched + kSlice / 32;                       // bitmaps of the slice
    uint4 *next = reinterpret_cast<uint4 *>(table + (kTabled ? kSlice + kSlice / 16 : 0));       // the row's logits: [item][word][thread]
    int32_t *next_tokens = reinterpret_cast<int32_t *>(next + kItems * kRaw * kThreads);           // [kTokens][thread]
    int32_t *next_bias_tokens = next_tokens + (counting ? kTokens * kThreads : 0);                 // [thread]
    float *next_bias_values = reinterpret_cast<float *>(next_bias_tokens + kThreads);              // [thread]
    uint32_t *masks = reinterpret_cast<uint32_t *>(next_bias_tokens + (biased ? 2 * kThreads : 0));   // [parity][kMaskWords]
    constexpr int kChunkWords = kChunk / 32 + 1, kMaskWords = kChunks * kChunkWords;            // a chunk's bits start anywhere in a word
    const bool shared_inputs = kTabled || a.r.temperature || a.r.allowed;

    if (kTabled) {
        uint4 *t4 = reinterpret_cast<uint4 *>(table);
        for (int i = tid; i < (kSlice + kSlice / 16) / 4; i += kThreads) t4[i] = make_uint4(0, 0, 0, 0);
    }
    if (tid == 0) {
        best_index[0] = 0x7fffffff;
        abort_flag = 0;
        listed[0] = 0;
        for (int i = 0; i < 2; ++i) ptx::mbar_init(ptx::smem_addr(&arrived[i]), 1);
        ptx::fence_barrier_init();
    }
    if (cluster > 1) ptx::cluster_arrive();                   // this CTA runs: its parts may be written after the matching wait
    ptx::grid_dependency_wait();
    ptx::launch_dependents();

    auto head_of = [&](const T *in_row) { return (int)(reinterpret_cast<uintptr_t>(in_row) / sizeof(T)) & (kAlign - 1); };
    // element s of the slice among the row's logits in shared memory
    auto place = [&](int s) -> T * {
        if (kRaw == 1) return reinterpret_cast<T *>(next) + s;
        const int g = s / kPer;
        return reinterpret_cast<T *>(next + (g / kThreads * kRaw + s % kPer / kAlign) * kThreads + g % kThreads) + s % kAlign;
    };
    // does the row fill the groups number i of the whole CTA
    auto inner_item = [&](int i, int head, int end) { return chunk_at(i * kWarps) >= head && chunk_at(i * kWarps + kWarps - 1) + kChunk <= end; };
    // a row on its way into this thread's own places: whole groups by asynchronous copies, the ends one by one
    auto fetch = [&](uint32_t row, int into, int begin, int stop) {
        const T *in_row = static_cast<const T *>(a.logits) + row * a.logits_stride;
        const int head = head_of(in_row), end = a.vocab + head;
        auto copy = [&](int i, int v) {
#pragma unroll
            for (int k = 0; k < kRaw; ++k)
                copy_async_16(ptx::smem_addr(next + (i * kRaw + k) * kThreads + tid), reinterpret_cast<const uint4 *>(in_row + (v - head)) + k);
        };
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int v = group_at(i);
            if (inner_item(i, head, end)) copy(i, v);
            else if (v >= head && v + kPer <= end) copy(i, v);
            else if (v < end && v + kPer > head)
#pragma unroll 1
                for (int j = 0; j < kPer; ++j)
                    if (v + j >= head && v + j < end) *place((tid + i * kThreads) * kPer + j) = in_row[v - head + j];
        }
        if (counting)
#pragma unroll
            for (int k = 0; k < kTokens; ++k)
                if (tid + k * kThreads < a.r.token_room) copy_async_4(ptx::smem_addr(next_tokens + tid + k * kThreads), a.r.tokens + row * a.r.token_stride + tid + k * kThreads);
        if (counting && tid >= kTokens * kThreads / 32 && tid * 32 < a.r.token_room) prefetch_l2(a.r.tokens + row * a.r.token_stride + tid * 32);
        if (tid < stop - begin) {
            copy_async_4(ptx::smem_addr(next_bias_tokens + tid), a.r.bias_tokens + begin + tid);
            copy_async_4(ptx::smem_addr(next_bias_values + tid), a.r.bias_values + begin + tid);
        }
        if (a.r.allowed) {
            const int last = (a.vocab - 1) >> 5;
            for (int i = tid; i < kMaskWords; i += kThreads) {
                const int c = i / kChunkWords, word = ((chunk_at(c) - head) >> 5) + (i - c * kChunkWords);      // (-1: never asked for)
                if (word >= 0 && word <= last) copy_async_4(ptx::smem_addr(masks + into * kMaskWords + i), a.r.allowed + row * a.r.allowed_stride + word);
            }
        }
        if (shared_inputs && tid < 6) {
            const void *from[6] = {a.r.lengths, a.r.prompt_lengths, a.r.repetition, a.r.presence, a.r.frequency, a.r.temperature};
            const void *p = nullptr;
#pragma unroll
            for (int i = 0; i < 6; ++i)
                if (tid == i) p = from[i];
            if (p) copy_async_4(ptx::smem_addr(&params[into][tid]), static_cast<const uint32_t *>(p) + row);
        }
    };
    // a row's part of the bias lists: as the offsets say it, and made fit
    auto biases_of = [&](uint32_t row, int &begin, int &stop) {
        if (biased) { begin = a.r.bias_offsets[row]; stop = a.r.bias_offsets[row + 1]; }
    };
    auto clamp_biases = [&](int &begin, int &stop) {
        if (!biased) return;
        begin = min(max(begin, 0), (int)a.r.bias_count);
        stop = min(max(stop, begin), (int)a.r.bias_count);
    };
    const uint32_t rows = (uint32_t)a.rows, row_step = gridDim.x / (uint32_t)cluster;
    uint32_t row = blockIdx.x / (uint32_t)cluster;             // (unsigned: a step beyond the last of 2^31 - 1 rows leaves 31 bits)
    int turn = 0;
    uint32_t phase = 0;                                       // of arrived[]: of both, it flips after two rows
    int begin = 0, stop = 0, next_begin = 0, next_stop = 0;
    biases_of(row, begin, stop);
    clamp_biases(begin, stop);
    fetch(row, 0, begin, stop);
    __syncwarp();
    if (cluster > 1) ptx::cluster_wait();
    __syncthreads();                                          // words and bits are clear

    for (; row < rows; row += row_step, phase ^= (uint32_t)turn, turn ^= 1, begin = next_begin, stop = next_stop) {
    if (kProbs && cluster > 1 && tid == 0) ptx::mbar_arrive_expect_tx(ptx::smem_addr(&arrived[turn]), (uint32_t)cluster * sizeof(Part));
    // ---- the row's logits, parameters and mask are in shared memory
    copies_wait();
    if (shared_inputs) __syncthreads();
    const T *in_row = static_cast<const T *>(a.logits) + row * a.logits_stride;
    const int head = head_of(in_row);
    const int end = a.vocab + head;                            // virtual indices head .. end
    const int32_t *tokens = counting ? a.r.tokens + row * a.r.token_stride : nullptr;
    const uint32_t *param = params[turn];
    const int said = counting ? min(max((int)param[0], 0), (int)a.r.token_room) : 0;
    const int prompt = counting && a.r.prompt_lengths ? min(max((int)param[1], 0), said) : 0;
    const float temperature = a.r.temperature ? __uint_as_float(param[5]) : 1.0f;
    const uint32_t after = row + row_step;
    if (after < rows) biases_of(after, next_begin, next_stop);
    // what is allowed, where something may not be: a byte per group (bit j: element j is inside the row and its mask)
    bool inner = true;
#pragma unroll
    for (int i = 0; i < kItems; ++i) inner = inner && inner_item(i, head, end);
    const bool closed = !inner || a.r.allowed != nullptr;
    uint32_t open_bits[(kItems + 3) / 4] = {};
    auto open = [&](int i) { return (open_bits[i / 4] >> (8 * (i & 3))) & 0xffu; };
    if (closed)
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int v = group_at(i);
        uint32_t bits = 0;
        if (v < end && v + kPer > head) {
            bits = 0xffu;
            if (v < head) bits &= 0xffu << (head - v);
            if (v + kPer > end) bits &= 0xffu >> (v + kPer - end);
            if (a.r.allowed) {
                const int first = chunk_at(i * kWarps + warp) - head, t = (first & 31) + lane * kPer;     // the mask's bits t .. t + 7 of the chunk's words
                const uint32_t *mask = masks + turn * kMaskWords + (i * kWarps + warp) * kChunkWords + (t >> 5);
                const int shift = t & 31;
                const uint32_t low = mask[0], high = shift > 24 ? mask[1] : 0u;       // (bits beyond the row are cut off above)
                bits &= __funnelshift_r(low, high, shift);
            }
        }
        open_bits[i / 4] |= bits << (8 * (i & 3));
    }

    auto slot = [&](int t) -> int {                            // a token's word in this CTA's table, or -1
        const int v = t + head, c = v / kChunk;
        const int q = (int)((uint32_t)c * a.cluster_magic >> 16);                // c / cluster
        return t >= 0 && t < a.vocab && c - q * cluster == rank ? q * kChunk + v % kChunk : -1;
    };

    auto touch = [&](uint32_t *bits, int s) -> bool {          // was the bit set before
        return *reinterpret_cast<volatile uint32_t *>(bits + (s >> 5)) >> (s & 31) & 1u || atomicOr(bits + (s >> 5), 1u << (s & 31)) >> (s & 31) & 1u;
    };
    // ---- the history: what of it is this slice's
    if (counting) {
        // the words of several tokens at a time, so that shared memory's answers overlap
        auto note = [&](auto const &t, auto in_prompt) {
            constexpr int kN = sizeof(t) / sizeof(t[0]);
            int s[kN];
            uint32_t before[kN];
#pragma unroll
            for (int k = 0; k < kN; ++k) s[k] = slot(t[k]);
            if (in_prompt) {
#pragma unroll
                for (int k = 0; k < kN; ++k) before[k] = s[k] >= 0 ? *reinterpret_cast<volatile uint32_t *>(table + s[k]) : (uint32_t)kInPrompt;
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    if (!(before[k] & kInPrompt)) before[k] = atomicOr(table + s[k], kInPrompt);      // (frequent tokens: once or twice)
            } else {
#pragma unroll
                for (int k = 0; k < kN; ++k) before[k] = s[k] >= 0 ? atomicAdd(table + s[k], 1u) : 1u;
            }
#pragma unroll
            for (int k = 0; k < kN; ++k)
                if (before[k] == 0) {                          // this word's first
                    atomicOr(touched + (s[k] >> 5), 1u << (s[k] & 31));
                    const int n = atomicAdd(&listed[turn], 1);
                    if (n < kList) list[n] = (unsigned short)s[k];
                }
        };
        int own[kTokens];                                      // of the copied ones; -1: none
#pragma unroll
        for (int k = 0; k < kTokens; ++k) own[k] = tid + k * kThreads < prompt ? next_tokens[tid + k * kThreads] : -1;
        note(own, true);
#pragma unroll
        for (int k = 0; k < kTokens; ++k) own[k] = tid + k * kThreads >= prompt && tid + k * kThreads < said ? next_tokens[tid + k * kThreads] : -1;
        note(own, false);
        auto rest = [&](int begin, int stop, bool in_prompt) { // tokens begin .. stop: eight at a time where there are many
            while (stop - begin > 4 * kThreads) {
                int t[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) t[k] = tid + k * kThreads < stop - begin ? tokens[begin + tid + k * kThreads] : -1;
                note(t, in_prompt);
                begin = stop - begin > 8 * kThreads ? begin + 8 * kThreads : stop;         // (no overflow)
            }
            while (begin < stop) {
                int t[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) t[k] = tid + k * kThreads < stop - begin ? tokens[begin + tid + k * kThreads] : -1;
                note(t, in_prompt);
                begin = stop - begin > 2 * kThreads ? begin + 2 * kThreads : stop;
            }
        };
        rest(kTokens * kThreads, prompt, true);
        rest(max(kTokens * kThreads, prompt), said, false);
    }
    // ---- biases: is a token of the slice listed twice
    // (entries are unsigned: a list may end at 2^31 - 1, and the steps beyond its end leave 31 bits)
    int bias_slot = -1;                                        // this thread's first entry
    float bias_value = 0.0f;
    bool twice = false;
    if (tid < stop - begin) {
        bias_slot = slot(next_bias_tokens[tid]);
        bias_value = next_bias_values[tid];
        twice = bias_slot >= 0 && touch(claimed, bias_slot);
        for (uint32_t e = (uint32_t)begin + tid + kThreads; e < (uint32_t)stop; e += kThreads) {
            const int s = slot(a.r.bias_tokens[e]);
            if (s >= 0 && touch(claimed, s)) twice = true;
        }
    }
    // the counts and the claims are complete
    const bool any_twice = kTabled && __syncthreads_or(twice);

    // ---- counts -> logits: a thread per word of the list, or, where it was too short, each thread the bitmap of its groups
    auto hits = [&](int i) -> uint32_t { return reinterpret_cast<const unsigned char *>(touched)[tid + i * kThreads]; };
    if (counting) {
        const float repetition = a.r.repetition ? __uint_as_float(param[2]) : 1.0f;
        const float presence = a.r.presence ? __uint_as_float(param[3]) : 0.0f;
        const float frequency = a.r.frequency ? __uint_as_float(param[4]) : 0.0f;
        auto penalise = [&](int s) {
            const uint32_t count = table[s] & ~kInPrompt;
            float l = to_f32(*place(s));
            l = l > 0.0f ? __fdiv_rn(l, repetition) : __fmul_rn(l, repetition);
            if (count) l = __fsub_rn(__fsub_rn(l, __fmul_rn(frequency, (float)count)), presence);
            table[s] = __float_as_uint(l);
        };
        const int n = listed[turn];
        if (tid == 0) listed[turn ^ 1] = 0;
        if (n <= kList) {
            if (tid < n) penalise(list[tid]);
            if (begin >= stop) __syncthreads();                // (with biases there is a barrier anyway)
        } else {
#pragma unroll 1
            for (int i = 0; i < kItems; ++i)
                for (uint32_t left = hits(i); left; left &= left - 1) penalise((tid + i * kThreads) * kPer + __ffs(left) - 1);
        }
    }
    // ---- biases on top.  Entries of distinct tokens (the rule) are added by one thread each; where a token is listed twice, one
    // warp goes through the list in its order
    if (begin < stop) {                                        // (the same for the whole CTA)
        if (counting) __syncthreads();
        auto now = [&](int s) -> float { return touched[s >> 5] >> (s & 31) & 1u ? __uint_as_float(table[s]) : to_f32(*place(s)); };
        auto add = [&](int s, float b) {                       // a token that one thread sees to
            table[s] = __float_as_uint(__fadd_rn(now(s), b));
            atomicOr(touched + (s >> 5), 1u << (s & 31));
            claimed[s >> 5] = 0;
        };
        if (!any_twice) {
            if (bias_slot >= 0) add(bias_slot, bias_value);
            for (uint32_t e = (uint32_t)begin + tid + kThreads; e < (uint32_t)stop; e += kThreads) {
                const int s = slot(a.r.bias_tokens[e]);
                if (s >= 0) add(s, a.r.bias_values[e]);
            }
        } else if (warp == 0) {
            for (uint32_t e0 = (uint32_t)begin; e0 < (uint32_t)stop; e0 += 32) {
                const uint32_t e = e0 + lane;
                const int s = e < (uint32_t)stop ? slot(a.r.bias_tokens[e]) : -1;
                const float b = s >= 0 ? a.r.bias_values[e] : 0.0f;
                const uint32_t same = __match_any_sync(0xffffffffu, s);
                const bool leader = s >= 0 && lane == __ffs(same) - 1;
                float l = leader ? now(s) : 0.0f;
                for (int from = 0; from < 32; ++from) {        // lanes in order, i.e. the list's order
                    const float next_b = __shfl_sync(0xffffffffu, b, from);
                    if (leader && ((same >> from) & 1u)) l = __fadd_rn(l, next_b);
                }
                __syncwarp();
                if (leader) {
                    table[s] = __float_as_uint(l);
                    atomicOr(touched + (s >> 5), 1u << (s & 31));
                    claimed[s >> 5] = 0;
                }
                __syncwarp();
            }
        }
        __syncthreads();
    }

    // ---- the logits into registers, touched ones from their words
    float x[kItems][kPer];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        uint4 raw[kRaw];
#pragma unroll
        for (int k = 0; k < kRaw; ++k) raw[k] = next[(i * kRaw + k) * kThreads + tid];
        T t[kPer];
        memcpy(t, raw, sizeof t);
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[i][j] = to_f32(t[j]);
        if (kTabled) {
            const uint32_t hit = hits(i);
            if (hit) {
                uint4 *words = reinterpret_cast<uint4 *>(table + (tid + i * kThreads) * kPer);
                const uint4 lo = words[0], hi = words[1];
                const uint32_t w[kPer] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if ((hit >> j) & 1u) x[i][j] = __uint_as_float(w[j]);
                words[0] = words[1] = make_uint4(0, 0, 0, 0);
                reinterpret_cast<unsigned char *>(touched)[tid + i * kThreads] = 0;
            }
        }
    }
    if (after < rows) {
        clamp_biases(next_begin, next_stop);                   // (only now: the offsets are on their way until here)
        fetch(after, turn ^ 1, next_begin, next_stop);
    }
    // ---- what is not allowed (and what a group holds beyond the row)
    if (closed)
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (open(i) != 0xffu) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (!((open(i) >> j) & 1u)) x[i][j] = -INFINITY;
        }

    const float cool = __fdiv_rn(1.0f, temperature);
    // value(i, y) gives the results of the thread's group i
    auto write_row = [&](auto *out_row, auto value) {
        const bool aligned = (reinterpret_cast<uintptr_t>(out_row - head) & 15) == 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int v = group_at(i);
            float y[kPer];
            if (aligned && inner_item(i, head, end)) {
                value(i, y);
                store_group(out_row + (v - head), y);
            } else if (v < end && v + kPer > head) {
                value(i, y);
                if (aligned && v >= head && v + kPer <= end) store_group(out_row + (v - head), y);
                else store_some(out_row, v, head, end, y);
            }
        }
    };
    if constexpr (!kProbs) {
        auto adjusted = [&](int i, float (&y)[kPer]) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) y[j] = x[i][j] * cool;
            if (closed && open(i) != 0xffu) {                  // (a temperature of 0 or less must not touch the mask)
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (!((open(i) >> j) & 1u)) y[j] = -INFINITY;
            }
        };
        write_row(static_cast<T *>(a.out) + row * a.out_stride, adjusted);
    } else {
        // ---- max of the slice
        float own = -INFINITY;
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) own = max_nan(own, x[i][j]);
        const float warp_top = warp_max_nan(own);
        if (lane == 0) warp_tops[warp] = warp_top;
        __syncthreads();
        if (tid == 0) best_index[turn ^ 1] = 0x7fffffff;
        Part mine;
        mine.top = warp_max_nan(lane < kThreads / 32 ? warp_tops[lane] : -INFINITY);
        // ---- its lowest index: only threads that hold it look
        if (is_max(own, mine.top)) {
            int index = 0x7fffffff;
#pragma unroll
            for (int i = kItems - 1; i >= 0; --i)
#pragma unroll
                for (int j = kPer - 1; j >= 0; --j)
                    if (is_max(x[i][j], mine.top) && (!closed || ((open(i) >> j) & 1u))) index = group_at(i) + j - head;
            atomicMin(&best_index[turn], index);
        }
        // ---- exponentials relative to the slice's own max, in base 2, times 2^24 (so that small ones are no subnormal numbers)
        const float scale = 1.44269504f * cool;
        const float base = mine.top == -INFINITY ? 0.0f : mine.top;
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                x[i][j] = exp2_approx(fmaf(x[i][j] - base, scale, 24.0f));
                sums[j & 3] += x[i][j];
            }
        float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) warp_sums[warp] = sum;
        __syncthreads();
        mine.sum = lane < kThreads / 32 ? warp_sums[lane] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine.sum += __shfl_xor_sync(0xffffffffu, mine.sum, o);
        mine.index = best_index[turn];
        // ---- the row's max and sum from all slices; each CTA computes them alike
        Part whole = mine;
        float factor = 1.0f;                                   // exp((slice's max - row's max) / T)
        if (cluster > 1) {
            if (tid < cluster) {
                // asynchronous stores, counted by the receiver's barrier.  (Stores and a barrier of the cluster would also wait for
                // the last row's output to leave: the barrier releases everything written before it.)
                ptx::st_async_cluster_v4(ptx::map_to_cta(ptx::smem_addr(&parts[turn][rank]), (uint32_t)tid), __float_as_uint(mine.top), (uint32_t)mine.index,
                                         __float_as_uint(mine.sum), 0u, ptx::map_to_cta(ptx::smem_addr(&arrived[turn]), (uint32_t)tid));
            }
            // the first warp waits for all of them (acquire at cluster scope: other CTAs wrote them) and tells the others.  (A wait that
            // runs out, which none does short of a fault, leaves the row with what has come in.)
            if (warp == 0) {
                bounded_wait<true>(ptx::smem_addr(&arrived[turn]), phase, &abort_flag, &g_status, kStatusWaitTimeout, 1u << 24);
                Part p = {-INFINITY, 0x7fffffff, 0.0f, 0u};
                if (lane < cluster) p = parts[turn][lane];     // (a lane per CTA)
                whole.top = warp_max_nan(p.top);
                whole.index = __reduce_min_sync(0xffffffffu, is_max(p.top, whole.top) ? p.index : 0x7fffffff);
                whole.sum = p.top != -INFINITY ? p.sum * exp2_approx((p.top - (whole.top == -INFINITY ? 0.0f : whole.top)) * scale) : 0.0f;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) whole.sum += __shfl_xor_sync(0xffffffffu, whole.sum, o);
                if (lane == 0) row_part = whole;
                __syncwarp();
            }
            __syncthreads();
            whole = row_part;
            // (a slice with nothing above -infinity has exponentials of 0 and no max to compare: base is 0 there, far above a low row max)
            const float below = (mine.top == -INFINITY ? -INFINITY : base - whole.top) * scale;
            factor = exp2_approx(below);
            // a slice far below the row's max: its factor over the sum would be a subnormal number, so the exponentials hand their 2^24
            // to the factor (they lose bits below 2^-126 then, where the probability is below 2^-190)
            if (factor < 0x1p-64f) {
                factor = exp2_approx(below + 24.0f);
#pragma unroll
                for (int i = 0; i < kItems; ++i)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) x[i][j] *= 0x1p-24f;
            }
        }
        const bool empty = whole.top == -INFINITY;
        if (rank == 0 && tid == 0) {
            if (a.best) a.best[row] = empty ? -1 : whole.index;
            if (a.best_logprob) a.best_logprob[row] = empty ? -INFINITY : -logf(whole.sum * 0x1p-24f);
        }
        if (a.out) {
            const float inv = empty ? 0.0f : __fdiv_rn(factor, whole.sum);
            auto probabilities = [&](int i, float (&y)[kPer]) {
#pragma unroll
                for (int j = 0; j < kPer; ++j) y[j] = x[i][j] * inv;
                if (closed && inv != inv) {                    // NaN: what is not allowed is 0 all the same
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if (!((open(i) >> j) & 1u)) y[j] = 0.0f;
                }
            };
            if (a.out_type == AZ_TYPE_F32) write_row(static_cast<float *>(a.out) + row * a.out_stride, probabilities);
            else write_row(static_cast<T *>(a.out) + row * a.out_stride, probabilities);
        }
    }
    }
}

template <typename T, int kThreads, int kItems, bool kProbs, bool kTabled>
int launch_form(const Args &args, int rows, cudaStream_t s) {
    Args a = args;
    constexpr int kSlice = kThreads * kItems * kPer;
    a.cluster = (a.span + kSlice - 1) / kSlice;
    a.rows = rows;
    a.cluster_magic = (uint32_t)((65536 + a.cluster - 1) / a.cluster);
    const int table_bytes = (kSlice + kSlice / 16) * 4;           // words and two bitmaps
    const int counting = a.r.tokens != nullptr, biased = a.r.bias_offsets != nullptr, masked = a.r.allowed != nullptr;
    auto smem = [&](int counting, int biased, int masked) {
        return (counting || biased ? table_bytes : 0) + kSlice * (int)sizeof(T) + (counting + 2 * biased) * kThreads * 4 + masked * 2 * (kSlice / 256 * 9) * 4;
    };
    auto kernel = logits_kernel<T, kThreads, kItems, kProbs, kTabled>;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = (size_t)smem(counting, biased, masked); cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    // how many clusters of this size, with so much shared memory, the device holds at a time (asked once)
    int dev = 0, held = 0;
    AZ_CUDA(cudaGetDevice(&dev));
    {
        static int known[64][kMaxCluster + 1][8] = {};
        static std::mutex lock;
        std::lock_guard<std::mutex> hold(lock);
        int asked = 0;
        int &entry = dev >= 0 && dev < 64 ? known[dev][a.cluster][counting + 2 * biased + 4 * masked] : asked;
        if (entry == 0) {
            AZ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem(1, 1, 1)));
            AZ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
            cfg.gridDim = dim3((unsigned)a.cluster);
            cfg.numAttrs = 1;
            AZ_CUDA(cudaOccupancyMaxActiveClusters(&entry, kernel, &cfg));
            cfg.numAttrs = 2;
            if (entry < 1) entry = 1;
        }
        held = entry;
    }
    cfg.gridDim = dim3((unsigned)((rows < held ? rows : held) * a.cluster));
    AZ_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
    return AZ_OK;
}

template <typename T, int kThreads, int kItems, bool kProbs>
int launch_shape(const Args &a, int rows, cudaStream_t s) {
    return a.r.tokens || a.r.bias_offsets ? launch_form<T, kThreads, kItems, kProbs, true>(a, rows, s) : launch_form<T, kThreads, kItems, kProbs, false>(a, rows, s);
}

template <typename T, bool kProbs>
int launch(Args a, int rows, cudaStream_t s) {
    constexpr int kAlign = 16 / (int)sizeof(T);
    const bool alike = rows == 1 || (a.logits_stride & (kAlign - 1)) == 0;      // all rows start at the same place of 16 bytes
    const int span = a.span = a.vocab + (alike ? (int)(reinterpret_cast<uintptr_t>(a.logits) / sizeof(T)) & (kAlign - 1) : kAlign - 1);
    if (span <= 1024) return launch_shape<T, 128, 1, kProbs>(a, rows, s);
    if (span <= 2048) return launch_shape<T, 128, 2, kProbs>(a, rows, s);      // (1024 x 1858 float32: 7.2 us; 256 threads with a group each 8.8, 64 with four 7.6)
    auto fits = [&](int slice, int most = 8) { return (span + slice - 1) / slice <= most; };
    auto fills = [&](int slice) { return (long long)rows * ((span + slice - 1) / slice) >= 120; };
    // The largest slices that still make 120 CTAs, and for few rows the smallest that a cluster holds.  us for slices of
    // 16384 / 8192 / 4096 (histories of 1,000 tokens, bf16):
    //   1 x 131072 7.0 / 5.6 / -, 16 x 131072 9.1 / 10.3 / -, 64 x 131072 19.3 / 27.9 / -
    //   1 x 32000 7.6 / 5.7 / 5.0, 16 x 32000 7.8 / 6.0 / 6.2, 128 x 32000 10.9 / 13.8 / 21.4, 512 x 32000 37.9 / 48.5 / 79.3
    //   64 x 10000 8.5 / 6.1 / 6.8, 600 x 10000 25.1 / 26.4 / 41.8
    if (fits(4096) && !fills(8192)) return launch_shape<T, 512, 1, kProbs>(a, rows, s);
    if (fits(8192, kMaxCluster) && !fills(16384)) return launch_shape<T, 512, 2, kProbs>(a, rows, s);
    if (fits(16384, kMaxCluster)) return launch_shape<T, 512, 4, kProbs>(a, rows, s);
    return launch_shape<T, 512, 5, kProbs>(a, rows, s);
}

bool misaligned(const void *p, uintptr_t element) { return (reinterpret_cast<uintptr_t>(p) & (element - 1)) != 0; }
int type_size(int type) { return type == AZ_TYPE_F32 ? 4 : 2; }

// the rules' own consistency, and their copy (absent: all null)
int check_rules(const az_logit_rules *rules, int rows, int vocab, az_logit_rules *out) {
    *out = az_logit_rules{};
    if (!rules) return AZ_OK;
    const az_logit_rules &r = *rules;
    const void *words[] = {r.tokens, r.lengths, r.prompt_lengths, r.repetition, r.presence, r.frequency, r.bias_offsets,
                           r.bias_tokens, r.bias_values, r.temperature, r.allowed};
    for (const void *p : words)
        if (misaligned(p, 4)) return AZ_ERR_BAD_ARG;
    if (r.tokens) {
        if (!r.lengths || r.token_room < 0 || r.token_room > 0x7fffffffll || (rows > 1 && r.token_stride < r.token_room)) return AZ_ERR_BAD_ARG;
    } else if (r.lengths || r.prompt_lengths || r.repetition || r.presence || r.frequency) return AZ_ERR_BAD_ARG;
    if (r.bias_offsets) {
        if (r.bias_count < 0 || r.bias_count > 0x7fffffffll) return AZ_ERR_BAD_ARG;
        if (r.bias_count > 0 && (!r.bias_tokens || !r.bias_values)) return AZ_ERR_BAD_ARG;
    } else if (r.bias_tokens || r.bias_values) return AZ_ERR_BAD_ARG;
    if (r.allowed && r.allowed_stride != 0 && rows > 1 && r.allowed_stride < (vocab + 31) / 32) return AZ_ERR_BAD_ARG;
    *out = r;
    return AZ_OK;
}

// logits and an output may be the same rows, or share no byte
bool overlap(const void *a, int64_t a_stride, int a_size, const void *b, int64_t b_stride, int b_size, int rows, int vocab) {
    if (a == b && a_size == b_size && (rows == 1 || a_stride == b_stride)) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + ((uintptr_t)(rows - 1) * (uintptr_t)a_stride + (uintptr_t)vocab) * (uintptr_t)a_size;
    const uintptr_t b1 = b0 + ((uintptr_t)(rows - 1) * (uintptr_t)b_stride + (uintptr_t)vocab) * (uintptr_t)b_size;
    if (a0 >= b1 || b0 >= a1) return false;
    // rows side by side in the same wider rows
    const uintptr_t pitch = (uintptr_t)a_stride * (uintptr_t)a_size;
    if (rows == 1 || pitch != (uintptr_t)b_stride * (uintptr_t)b_size) return true;
    const uintptr_t a_row = (uintptr_t)vocab * (uintptr_t)a_size, b_row = (uintptr_t)vocab * (uintptr_t)b_size;
    const uintptr_t ahead = a0 < b0 ? (b0 - a0) % pitch : (pitch - (a0 - b0) % pitch) % pitch;      // from a row of a to the next one of b
    return ahead < a_row || ahead + b_row > pitch;
}

int check_logits(const void *logits, int type, int rows, int vocab, int64_t stride) {
    if (!logits || misaligned(logits, (uintptr_t)type_size(type))) return AZ_ERR_BAD_ARG;
    if (rows > 1 && stride < vocab) return AZ_ERR_BAD_ARG;
    return vocab > AZ_MAX_VOCAB ? AZ_ERR_UNSUPPORTED : AZ_OK;
}

template <bool kProbs>
int launch_type(const Args &a, int type, int rows, cudaStream_t s) {
    if (type == AZ_TYPE_F32) return launch<float, kProbs>(a, rows, s);
    if (type == AZ_TYPE_BF16) return launch<__nv_bfloat16, kProbs>(a, rows, s);
    return launch<__half, kProbs>(a, rows, s);
}

}  // namespace

int logits_status_word(uint32_t **word) {
    AZ_CUDA(cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_status));
    return AZ_OK;
}
}  // namespace az

extern "C" int az_adjust_logits(const void *logits_dev, int type, int rows, int vocab, int64_t logits_stride,
                                const az_logit_rules *rules, void *out_dev, int64_t out_stride, void *cuda_stream) {
    if (rows < 0 || vocab < 0 || type < AZ_TYPE_F32 || type > AZ_TYPE_F16) return AZ_ERR_BAD_ARG;
    if (rows == 0 || vocab == 0) return AZ_OK;
    az::Args a = {};
    int rc = az::check_logits(logits_dev, type, rows, vocab, logits_stride);
    if (rc != AZ_OK) return rc;
    if (!out_dev || az::misaligned(out_dev, (uintptr_t)az::type_size(type)) || (rows > 1 && out_stride < vocab)) return AZ_ERR_BAD_ARG;
    if (az::overlap(logits_dev, logits_stride, az::type_size(type), out_dev, out_stride, az::type_size(type), rows, vocab)) return AZ_ERR_BAD_ARG;
    rc = az::check_rules(rules, rows, vocab, &a.r);
    if (rc != AZ_OK) return rc;
    a.logits = logits_dev; a.out = out_dev; a.logits_stride = logits_stride; a.out_stride = out_stride;
    a.vocab = vocab; a.out_type = type;
    return az::launch_type<false>(a, type, rows, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int az_token_probs(const void *logits_dev, int type, int rows, int vocab, int64_t logits_stride, const az_logit_rules *rules,
                              void *probs_dev, int probs_type, int64_t probs_stride, int32_t *best_dev, float *best_logprob_dev,
                              void *cuda_stream) {
    if (rows < 0 || vocab < 0 || type < AZ_TYPE_F32 || type > AZ_TYPE_F16) return AZ_ERR_BAD_ARG;
    if (rows == 0 || vocab == 0) return AZ_OK;
    az::Args a = {};
    int rc = az::check_logits(logits_dev, type, rows, vocab, logits_stride);
    if (rc != AZ_OK) return rc;
    if (!probs_dev && !best_dev && !best_logprob_dev) return AZ_ERR_BAD_ARG;
    if (az::misaligned(best_dev, 4) || az::misaligned(best_logprob_dev, 4)) return AZ_ERR_BAD_ARG;
    if (probs_dev) {
        if (probs_type != AZ_TYPE_F32 && probs_type != type) return AZ_ERR_BAD_ARG;
        if (az::misaligned(probs_dev, (uintptr_t)az::type_size(probs_type)) || (rows > 1 && probs_stride < vocab)) return AZ_ERR_BAD_ARG;
        if (az::overlap(logits_dev, logits_stride, az::type_size(type), probs_dev, probs_stride, az::type_size(probs_type), rows, vocab)) return AZ_ERR_BAD_ARG;
    }
    rc = az::check_rules(rules, rows, vocab, &a.r);
    if (rc != AZ_OK) return rc;
    a.logits = logits_dev; a.out = probs_dev; a.best = best_dev; a.best_logprob = best_logprob_dev;
    a.logits_stride = logits_stride; a.out_stride = probs_stride;
    a.vocab = vocab; a.out_type = probs_type;
    return az::launch_type<true>(a, type, rows, static_cast<cudaStream_t>(cuda_stream));
}
