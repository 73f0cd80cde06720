// Counts and bitmaps of the tokens that sequences have behind them.
#pragma once

#include "fsd_device.cuh"

namespace fsd {

constexpr int kHistThreads = 1024;
constexpr int kHistSpan = 11264;        // ids a block counts, in shared memory

// A block per sequence and span of the vocabulary.  It looks through all of the sequence's tokens, which the L2 cache has after
// the first block, so that nothing has to be cleared first and each count is written once.  Whole numbers: the order of
// the additions does not matter.  (Places in the lists are counted in 64 bits: an offset may be 2^31 - 1, and a thread's next place
// behind it.)  32 sequences of up to 32768 + 8192 tokens, V = 128256: 10.2 us, of which the longest sequence's
// tokens are most; the counts alone are 2.6 us of memory.
__global__ void __launch_bounds__(kHistThreads) fsd_history_build_kernel(const int32_t* prompt_offsets, const int32_t* prompt_tokens, const int32_t* output_offsets,
                                                                         const int32_t* output_tokens, int V, int W, int spans, int32_t* counts, uint32_t* seen) {
    __shared__ int32_t n[kHistSpan];
    __shared__ uint32_t bits[kHistSpan / 32];
    const int b = blockIdx.x / spans, lo = blockIdx.x % spans * kHistSpan;
    for (int i = threadIdx.x; i < kHistSpan; i += kHistThreads) n[i] = 0;
    for (int i = threadIdx.x; i < kHistSpan / 32; i += kHistThreads) bits[i] = 0u;
    __syncthreads();
#pragma unroll 8
    for (long long i = __ldg(prompt_offsets + b) + static_cast<long long>(threadIdx.x), end = __ldg(prompt_offsets + b + 1); i < end; i += kHistThreads) {
        const int t = __ldg(prompt_tokens + i), k = t - lo;
        if (t >= lo && t < V && k < kHistSpan) atomicOr(&bits[k >> 5], 1u << (k & 31));
    }
    if (output_offsets != nullptr)
#pragma unroll 8
        for (long long i = __ldg(output_offsets + b) + static_cast<long long>(threadIdx.x), end = __ldg(output_offsets + b + 1); i < end; i += kHistThreads) {
            const int t = __ldg(output_tokens + i), k = t - lo;
            if (t >= lo && t < V && k < kHistSpan) {
                atomicAdd(&n[k], 1);
                atomicOr(&bits[k >> 5], 1u << (k & 31));
            }
        }
    __syncthreads();
    FSD_CHECK(&process_debug, lo >= 0 && lo < V && lo % 32 == 0, kChkSlice);
    for (int k = threadIdx.x; k < kHistSpan && lo + k < V; k += kHistThreads) counts[static_cast<size_t>(b) * V + lo + k] = n[k];
    for (int k = threadIdx.x; k < kHistSpan / 32 && lo / 32 + k < W; k += kHistThreads) seen[static_cast<size_t>(b) * W + lo / 32 + k] = bits[k];
}

// A warp per sequence.  path NULL: the first accept_len drafted tokens; else the tokens of the nodes on it.  width: how many there can be.
__global__ void __launch_bounds__(128) fsd_history_append_kernel(const int32_t* tokens, const int32_t* path, const int32_t* accept_len, const int32_t* next_token,
                                                                 int B, int P, int width, int V, int W, int32_t* counts, uint32_t* seen) {
    const int b = blockIdx.x * 4 + static_cast<int>(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= B) return;
    int n = __ldg(accept_len + b);
    n = n < 0 ? 0 : n > width ? width : n;
    for (long long i = lane; i <= n; i += 32) {              // (n may be 2^31 - 1)
        int t;
        if (i == n) {
            t = __ldg(next_token + b);
        } else {
            const int j = path != nullptr ? __ldg(path + static_cast<size_t>(b) * width + i) : static_cast<int>(i);
            t = j >= 0 && j < P ? __ldg(tokens + static_cast<size_t>(b) * P + j) : -1;
        }
        if (t >= 0 && t < V) {
            atomicAdd(counts + static_cast<size_t>(b) * V + t, 1);
            atomicOr(seen + static_cast<size_t>(b) * W + (t >> 5), 1u << (t & 31));
        }
    }
}

}  // namespace fsd
