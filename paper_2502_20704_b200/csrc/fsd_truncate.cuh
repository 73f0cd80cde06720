// Top-k, top-p and min-p on rows of processed logits.
#pragma once

#include "fsd_process.cuh"

namespace fsd {

// ---- order of values as whole numbers ------------------------------------------
// A key rises with the value, -0 and 0 have the same, and all of a type's values have keys of kKeyBits.
template <int DT> constexpr int kKeyBits = DT == FSD_BF16 ? 16 : 32;
template <int DT> constexpr uint32_t kSignBit = DT == FSD_BF16 ? 0x8000u : 0x80000000u;
template <int DT>
__device__ __forceinline__ uint32_t key_of(uint32_t bits) {
    if (bits == kSignBit<DT>) bits = 0u;
    return (bits & kSignBit<DT>) ? (DT == FSD_BF16 ? 0xffffu : 0xffffffffu) ^ bits : bits | kSignBit<DT>;
}
template <int DT>
__device__ __forceinline__ float value_of(uint32_t key) {
    const uint32_t bits = (key & kSignBit<DT>) ? key ^ kSignBit<DT> : (DT == FSD_BF16 ? 0xffffu : 0xffffffffu) ^ key;
    return __uint_as_float(DT == FSD_BF16 ? bits << 16 : bits);
}
template <int DT> __device__ __forceinline__ uint32_t key_of_value(float y) { return key_of<DT>(__float_as_uint(y) >> (DT == FSD_BF16 ? 16 : 0)); }

constexpr int kCutThreads = 1024;

struct CountAndWeight {
    long long n;
    double w;
};
// Sums over the block in a fixed order; all threads have them.
__device__ __forceinline__ CountAndWeight block_total(CountAndWeight v, CountAndWeight* scratch) {
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
        v.n += __shfl_xor_sync(0xffffffffu, v.n, m);
        v.w += shfl_xor_d(v.w, m);
    }
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    CountAndWeight t = {0, 0.0};
    for (int w = 0; w < warps; ++w) { t.n += scratch[w].n; t.w += scratch[w].w; }
    __syncthreads();
    return t;
}

// A block per row, in place.  Thresholds are found a bit at a time: the largest key t for which the tokens at or above it are
// enough of what is asked for.  Every step is a sweep over the row, which is in the L2 cache after the first.
template <int DT>
__global__ void __launch_bounds__(kCutThreads) fsd_truncate_kernel(const ProcArgs a) {
    using elem = typename Logit<DT>::elem;
    using word = typename std::conditional<DT == FSD_BF16, uint16_t, uint32_t>::type;
    __shared__ CountAndWeight scratch[32];
    const int all = a.rows[0] + a.rows[1], b = blockIdx.x / all, q = blockIdx.x % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    const int V = a.V;
    elem* out = static_cast<elem*>(a.out[side]) + (static_cast<size_t>(b) * a.rows[side] + r) * V;
    const word* row = reinterpret_cast<const word*>(out);

    const int top_k = a.top_k != nullptr ? __ldg(a.top_k + b) : 0;
    const float top_p = a.top_p != nullptr ? __ldg(a.top_p + b) : 1.f, min_p = a.min_p != nullptr ? __ldg(a.min_p + b) : 0.f;
    const bool cut_k = top_k > 0 && top_k < V, cut_p = top_p < 1.f, cut_m = min_p > 0.f;
    if (!cut_k && !cut_p && !cut_m) return;

    // the largest value; rows without a distribution are left as they are
    const uint32_t kPosInf = key_of_value<DT>(INFINITY), kNegInf = key_of_value<DT>(-INFINITY);
    uint32_t top = 0u;
    for (int i = threadIdx.x; i < V; i += kCutThreads) {
        const uint32_t bits = row[i];
        const float y = __uint_as_float(DT == FSD_BF16 ? bits << 16 : bits);
        const uint32_t k = y != y ? 0xffffffffu : key_of<DT>(bits);
        top = top > k ? top : k;
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5].n = top;
    __syncthreads();
    for (int w = 0; w < kCutThreads / 32; ++w) top = top > static_cast<uint32_t>(scratch[w].n) ? top : static_cast<uint32_t>(scratch[w].n);
    __syncthreads();
    if (top >= kPosInf || top <= kNegInf) return;
    const double most = value_of<DT>(top);
    const auto weight = [&](uint32_t key) { return exp(static_cast<double>(value_of<DT>(key)) - most); };

    // tokens with keys of at least t: how many, and (with weights) what those above `over` weigh
    const auto at_least = [&](uint32_t t, uint32_t over, bool weights) {
        CountAndWeight v = {0, 0.0};
        for (int i = threadIdx.x; i < V; i += kCutThreads) {
            const uint32_t k = key_of<DT>(row[i]);
            if (k >= t) {
                ++v.n;
                if (weights && k > over) v.w += weight(k);
            }
        }
        return block_total(v, scratch);
    };

    uint32_t cut = 0u;                 // tokens above it are kept, and of those equal to it the first `ties`
    long long ties = V;
    if (cut_k) {
        for (int bit = kKeyBits<DT> - 1; bit >= 0; --bit)
            if (at_least(cut | 1u << bit, 0u, false).n >= top_k) cut |= 1u << bit;
        ties = top_k - at_least(cut + 1u, 0u, false).n;
    }
    if (cut_p) {
        // what the top_k tokens weigh that are at or above t
        const uint32_t over = cut_k ? cut : 0u;
        const double of_ties = cut_k ? static_cast<double>(ties) * weight(cut) : 0.0;
        const auto share = [&](uint32_t t) { return at_least(t, over, true).w + (cut_k && t <= cut ? of_ties : 0.0); };
        const double goal = static_cast<double>(top_p) * share(0u);
        uint32_t t = 0u;
        for (int bit = kKeyBits<DT> - 1; bit >= 0; --bit)
            if (share(t | 1u << bit) >= goal) t |= 1u << bit;
        if (!(goal > 0.0) || t > top) t = top;
        // of the tokens at t: those whose predecessors weigh less than the goal
        const double w = weight(t), above = t < top ? share(t + 1u) : 0.0;
        double j = ceil((goal - above) / w);
        if (j >= 1.0 && above + (j - 1.0) * w >= goal) j -= 1.0;
        if (above + j * w < goal) j += 1.0;
        const long long most_ties = j < 1.0 ? 1 : j > static_cast<double>(V) ? V : static_cast<long long>(j);
        ties = t > cut ? most_ties : ties < most_ties ? ties : most_ties;
        cut = t > cut ? t : cut;
    }
    if (cut_m) {
        // the smallest key whose value is no further below the largest than ln(min_p)
        const double far = log(static_cast<double>(min_p < 1.f ? min_p : 1.f));
        uint32_t lo = kNegInf, hi = top;                    // hi always is, lo never
        while (hi - lo > 1u) {
            const uint32_t mid = lo + (hi - lo) / 2u;
            if (static_cast<double>(value_of<DT>(mid)) - most >= far) hi = mid; else lo = mid;
        }
        if (hi > cut) { cut = hi; ties = V; }
    }

    // Where only some of the tokens at the cut are kept: the id from which on they are not.
    int until = V;
    const long long equal = at_least(cut, 0u, false).n - at_least(cut + 1u, 0u, false).n;
    if (ties < equal) {
        int lo = 0, hi = V;                                 // the smallest id with `ties` of them in front of it
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            CountAndWeight v = {0, 0.0};
            for (int i = threadIdx.x; i < mid; i += kCutThreads) v.n += key_of<DT>(row[i]) == cut;
            if (block_total(v, scratch).n >= ties) hi = mid; else lo = mid + 1;
        }
        until = lo;
    }
    const float none = -INFINITY;
    for (int i = threadIdx.x; i < V; i += kCutThreads) {
        const uint32_t k = key_of<DT>(row[i]);
        if (k < cut || (k == cut && i >= until)) reinterpret_cast<word*>(out)[i] = static_cast<word>(__float_as_uint(none) >> (DT == FSD_BF16 ? 16 : 0));
    }
}

}  // namespace fsd
