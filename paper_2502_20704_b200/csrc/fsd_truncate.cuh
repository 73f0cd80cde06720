// Top-k, top-p and min-p on rows of processed logits.
//
// The tokens that are kept are those above a value, the cut, and the first `ties` by id of those equal to it.  What decides
// about a token near the border of top-p is a sum over the row to within that token's own weight, a millionth of the
// whole in a flat row of 150000: sums are in double precision, and whether two programs agree never hangs on their order.
#pragma once

#include <climits>
#include <cmath>
#include <cstring>
#include <cuda_bf16.h>
#include <type_traits>

#include "fsd_process.cuh"

namespace fsd {

// ---- order of values as whole numbers ------------------------------------------
// A key rises with the value, -0 and 0 have the same, and all of a type's values have keys of kKeyBits.
template <int DT> constexpr int kKeyBits = DT == FSD_BF16 ? 16 : 32;
template <int DT> constexpr uint32_t kSignBit = DT == FSD_BF16 ? 0x8000u : 0x80000000u;
template <int DT> using LogitWord = typename std::conditional<DT == FSD_BF16, uint16_t, uint32_t>::type;
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
template <int DT> __device__ __forceinline__ float float_of(uint32_t word) { return __uint_as_float(DT == FSD_BF16 ? word << 16 : word); }

struct CountAndWeight {
    long long n;
    double w;
};

// What a sequence asks for.
struct CutParams {
    int top_k;
    float top_p, min_p;
    bool k, p, m;
};
__device__ __forceinline__ CutParams cut_params(const uint32_t* settings, int V) {      // top_k, top_p, min_p
    CutParams c;
    c.top_k = static_cast<int>(settings[0]);
    c.top_p = __uint_as_float(settings[1]);
    c.min_p = __uint_as_float(settings[2]);
    c.k = c.top_k > 0 && c.top_k < V;
    c.p = c.top_p < 1.f;
    c.m = c.min_p > 0.f;
    return c;
}

// Of tokens of weight w behind others that weigh `above`: how many have predecessors that weigh less than the goal (at least one).
__device__ __forceinline__ long long ties_below(double above, double w, double goal, int V) {
    double j = ceil((goal - above) / w);
    if (j >= 1.0 && above + (j - 1.0) * w >= goal) j -= 1.0;
    if (above + j * w < goal) j += 1.0;
    return j < 1.0 ? 1 : j > static_cast<double>(V) ? V : static_cast<long long>(j);
}

// (Out of line: the places that need it are many and reached seldom.)
__device__ __noinline__ double exp_d(double x) { return exp(x); }

// exp(x) for x of at most 700, to a few units of the last place: x = n ln 2 + r with |r| <= ln 2 / 2, and e^r by its
// Taylor series up to r^13 / 13! (the next term is below 5e-18).  Sums that say where a border lies need that much of each of
// their terms.  Below -700 it is 0.
__device__ __forceinline__ double exp_of(double x) {
    if (!(x > -700.0)) return 0.0;
    const double shift = 6755399441055744.0;                                      // 1.5 * 2^52: adding it rounds to a whole number
    const double u = __fma_rn(x, kLog2eD, shift);
    const int n = __double2loint(u);
    const double m = u - shift;
    const double r = __fma_rn(m, -2.3190468138462996e-17, __fma_rn(m, -0.69314718055994529, x));      // ln 2 as a double and what it lacks
    double e = 1.0 / 6227020800.0;
    e = __fma_rn(e, r, 1.0 / 479001600.0);
    e = __fma_rn(e, r, 1.0 / 39916800.0);
    e = __fma_rn(e, r, 1.0 / 3628800.0);
    e = __fma_rn(e, r, 1.0 / 362880.0);
    e = __fma_rn(e, r, 1.0 / 40320.0);
    e = __fma_rn(e, r, 1.0 / 5040.0);
    e = __fma_rn(e, r, 1.0 / 720.0);
    e = __fma_rn(e, r, 1.0 / 120.0);
    e = __fma_rn(e, r, 1.0 / 24.0);
    e = __fma_rn(e, r, 1.0 / 6.0);
    e = __fma_rn(e, r, 0.5);
    e = __fma_rn(e, r, 1.0);
    e = __fma_rn(e, r, 1.0);
    return __hiloint2double(__double2hiint(e) + (n << 20), __double2loint(e));     // (|n| is at most 1010: no subnormals)
}

// The smallest key whose value is no further below the largest, `most` with key `top`, than ln(min_p).  It is at the value
// most + ln(min_p) or next to it, unless the difference to `most` does not tell values there apart.
template <int DT>
__device__ __noinline__ uint32_t min_p_key(float min_p, uint32_t top, double most) {
    const double far = log(static_cast<double>(min_p < 1.f ? min_p : 1.f));
    const auto in = [&](uint32_t k) { return static_cast<double>(value_of<DT>(k)) - most >= far; };
    uint32_t lo = key_of_value<DT>(-INFINITY), hi = top;        // hi always is, lo never
    const uint32_t guess = key_of_value<DT>(static_cast<float>(most + far));
    if (guess > lo + 2u && guess + 2u < hi) {
        if (in(guess + 2u)) hi = guess + 2u;
        if (!in(guess - 2u)) lo = guess - 2u;
    }
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (in(mid)) hi = mid; else lo = mid;
    }
    return hi;
}

// ---- a bit at a time: rows of any length and any values -------------------------------
// The cut is the largest key t for which the tokens at or above it are enough of what is asked for, found from its highest
// bit down: a sweep over the row for each.  `row`: n words that this block has of the row, the first of them token first's;
// total / largest: over all blocks that have some of the row.  Where only some of the tokens at the cut are kept, `until` is the id
// from which on they are not.
struct Cut {
    bool any;
    uint32_t key;
    int until;
};
template <int DT, class Total, class Largest>
__device__ __noinline__ Cut find_cut(const LogitWord<DT>* row, int n, int first, int V, const CutParams& c, Total total, Largest largest) {
    const int tid = threadIdx.x, step = blockDim.x;
    uint32_t top = 0u;
    for (int i = tid; i < n; i += step) {
        const uint32_t bits = row[i];
        const float y = float_of<DT>(bits);
        const uint32_t k = y != y ? 0xffffffffu : key_of<DT>(bits);
        top = top > k ? top : k;
    }
    top = largest(top);
    if (top >= key_of_value<DT>(INFINITY) || top <= key_of_value<DT>(-INFINITY)) return {false, 0u, 0};
    const double most = value_of<DT>(top);
    const auto weight = [&](uint32_t key) { return exp_d(static_cast<double>(value_of<DT>(key)) - most); };
    // tokens with keys of at least t: how many, and (with weights) what those above `over` weigh
    const auto at_least = [&](uint32_t t, uint32_t over, bool weights) {
        CountAndWeight v = {0, 0.0};
        for (int i = tid; i < n; i += step) {
            const uint32_t k = key_of<DT>(row[i]);
            if (k >= t) {
                ++v.n;
                if (weights && k > over) v.w += weight(k);
            }
        }
        return total(v);
    };

    uint32_t cut = 0u;                 // tokens above it are kept, and of those equal to it the first `ties`
    long long ties = V;
    if (c.k) {
        for (int bit = kKeyBits<DT> - 1; bit >= 0; --bit)
            if (at_least(cut | 1u << bit, 0u, false).n >= c.top_k) cut |= 1u << bit;
        ties = c.top_k - at_least(cut + 1u, 0u, false).n;
    }
    if (c.p) {
        // what the top_k tokens weigh that are at or above t
        const uint32_t over = c.k ? cut : 0u;
        const double of_ties = c.k ? static_cast<double>(ties) * weight(cut) : 0.0;
        const auto share = [&](uint32_t t) { return at_least(t, over, true).w + (c.k && t <= cut ? of_ties : 0.0); };
        const double goal = static_cast<double>(c.top_p) * share(0u);
        uint32_t t = 0u;
        for (int bit = kKeyBits<DT> - 1; bit >= 0; --bit)
            if (share(t | 1u << bit) >= goal) t |= 1u << bit;
        if (!(goal > 0.0) || t > top) t = top;
        const long long at_t = ties_below(t < top ? share(t + 1u) : 0.0, weight(t), goal, V);
        ties = t > cut ? at_t : ties < at_t ? ties : at_t;
        cut = t > cut ? t : cut;
    }
    if (c.m) {
        const uint32_t t = min_p_key<DT>(c.min_p, top, most);
        if (t > cut) { cut = t; ties = V; }
    }
    int until = V;
    const long long equal = at_least(cut, 0u, false).n - at_least(cut + 1u, 0u, false).n;
    if (ties < equal) {
        int lo = 0, hi = V;                                 // the smallest id with `ties` of them in front of it
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            CountAndWeight v = {0, 0.0};
            for (int i = tid; i < n && first + i < mid; i += step) v.n += key_of<DT>(row[i]) == cut;
            if (total(v).n >= ties) hi = mid; else lo = mid + 1;
        }
        until = lo;
    }
    return {true, cut, until};
}

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
__device__ __forceinline__ uint32_t block_largest(uint32_t k, CountAndWeight* scratch) {
    k = __reduce_max_sync(0xffffffffu, k);
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5].n = k;
    __syncthreads();
    for (int w = 0; w < warps; ++w) k = k > static_cast<uint32_t>(scratch[w].n) ? k : static_cast<uint32_t>(scratch[w].n);
    __syncthreads();
    return k;
}

// A block per row, in place, on rows that are too long for shared memory.
constexpr int kLongThreads = 1024;
template <int DT>
__global__ void __launch_bounds__(kLongThreads) fsd_cut_long_kernel(const ProcArgs a) {
    __shared__ CountAndWeight scratch[32];
    const int all = a.rows[0] + a.rows[1], b = blockIdx.x / all, q = blockIdx.x % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    LogitWord<DT>* row = static_cast<LogitWord<DT>*>(a.out[side]) + (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
    const uint32_t settings[3] = {a.top_k != nullptr ? static_cast<uint32_t>(__ldg(a.top_k + b)) : 0u, __float_as_uint(a.top_p != nullptr ? __ldg(a.top_p + b) : 1.f),
                                  __float_as_uint(a.min_p != nullptr ? __ldg(a.min_p + b) : 0.f)};
    const CutParams c = cut_params(settings, a.V);
    if (!c.k && !c.p && !c.m) return;
    const Cut cut = find_cut<DT>(row, a.V, 0, a.V, c, [&](CountAndWeight v) { return block_total(v, scratch); }, [&](uint32_t k) { return block_largest(k, scratch); });
    if (!cut.any) return;
    for (int i = threadIdx.x; i < a.V; i += kLongThreads) {
        const uint32_t k = key_of<DT>(row[i]);
        if (k < cut.key || (k == cut.key && i >= cut.until)) row[i] = static_cast<LogitWord<DT>>(__float_as_uint(-INFINITY) >> (DT == FSD_BF16 ? 16 : 0));
    }
}

// ---- rows that fit on chip: a cluster of blocks per row ---------------------------
// A block reads its slice of the row once, processes it and keeps it in shared memory.  On the way it counts the values by their
// upper 16 bits: for bf16 a bin is one value, so that the counts alone say where every cut is and what everything weighs, with
// one exponential for a bin instead of one for a token.  For fp32 the bin of the border is split twice more by 8 bits.  The
// first block of the cluster gets all counts (additions into its shared memory, whole numbers, so that their order does
// not matter), finds the cut and tells the others.
// Bins of one value are those of magnitudes from 2^-8 up to 2^7; smaller ones share a bin a sign and are weighed one by one, and where
// a border lies in one of these, or something lies above, the row is cut a bit at a time.
constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kMaxCutCluster = 8;
constexpr uint32_t kMagLo = 0x3b7f, kMagHi = 0x4300;       // upper halves: just below 2^-8, and 2^7
constexpr int kHalfBins = static_cast<int>(kMagHi - kMagLo) + 1;
constexpr int kBins = 2 * kHalfBins;                       // negative magnitudes falling, then positive ones rising
constexpr int kBinUnder = 0, kBinOver = kBins - 1, kBinTinyNeg = kHalfBins - 1, kBinTinyPos = kHalfBins;
constexpr int kBinsEach = ((kBins + kRowThreads - 1) / kRowThreads + 3) / 4 * 4;
constexpr double kFixed = 4398046511104.0;                 // 2^42: weights of a bin's tokens as whole numbers

// The upper 16 bits of the keys of a one-value bin, and back.
__device__ __forceinline__ uint32_t bin_prefix(int bin) {
    return bin >= kHalfBins ? 0x8000u | (kMagLo + static_cast<uint32_t>(bin - kHalfBins)) : 0x7fffu ^ (kMagLo + static_cast<uint32_t>(kHalfBins - 1 - bin));
}
__device__ __forceinline__ bool one_value(int bin) { return bin != kBinUnder && bin != kBinOver && bin != kBinTinyNeg && bin != kBinTinyPos; }
__device__ __forceinline__ int bin_of_value(float y) {      // one of a one-value bin
    const uint32_t bits = __float_as_uint(y), u = (bits >> 16 & 0x7fffu) - kMagLo;
    return static_cast<int>(u ^ static_cast<uint32_t>(static_cast<int>(bits) >> 31)) + kHalfBins;
}
// The value of a bin: bf16 its only one, fp32 the middle of its range.
template <int DT>
__device__ __forceinline__ double bin_value(int bin) {
    if constexpr (DT == FSD_BF16) return value_of<FSD_BF16>(bin_prefix(bin));
    else return value_of<FSD_F32>(bin_prefix(bin) << 16 | 0x8000u);
}

// exp of every bin's value by place, from the highest bin down, and 0 for bins of many values.  The host fills it in front of a
// device's first call; worked out where it is needed it took the first block 2000 cycles a row.
__device__ __align__(16) double bin_weights[kBins];
inline void fill_bin_weights(double* w) {
    for (int k = 0; k < kBins; ++k) w[k] = 0.0;
    for (int u = 1; u < kHalfBins - 1; ++u) {
        const uint32_t bits = (kMagLo + static_cast<uint32_t>(u)) << 16;
        float v;
        memcpy(&v, &bits, 4);
        w[kBins - 1 - (kHalfBins + u)] = ::exp(static_cast<double>(v));
        w[kBins - 1 - (kHalfBins - 1 - u)] = ::exp(-static_cast<double>(v));
    }
}

enum CutKind { kCutNone, kCutDone, kCutByBits, kCutRefineK, kCutRefineP };
struct CutResult {
    int kind;
    uint32_t key;              // of the cut; while it is being refined, its upper bits
    long long ties;
    uint32_t over;             // refining top-k: whether all that are equal to the k-th are kept
    uint32_t equal;            // bf16: how many tokens are equal to the cut
};
struct CutShared {
    double tiny[kMaxCutCluster], above[kMaxCutCluster], rest[kMaxCutCluster];
    uint32_t top[kMaxCutCluster];
    int equal[kMaxCutCluster];
    CountAndWeight slots[2][kMaxCutCluster];
    CountAndWeight scratch[32];
    uint32_t warp_n[kRowWarps];
    double warp_w[kRowWarps];
    uint32_t min_key;
    uint32_t settings[8];
    uint64_t sub_w[256];
    uint32_t sub_n[256];
    CutResult work;            // the first block's
    CutResult told[2];         // what the first block told last, and the time before
    int found[4];
    double goal, above_goal;
    uint16_t list[kRowWarps][256];
};

template <int DT> struct RowSlice {
    uint4* vecs;
    int n;                     // vectors
    int first;                 // id of the first one's first token
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() { cluster_arrive(); cluster_wait(); }

// Exclusive sums over the threads of the block, in thread order.  All threads; ends with a barrier.
struct Run {
    uint32_t n;
    double w;
};
__device__ __forceinline__ Run scan_threads(Run v, CutShared& s, Run& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Run t = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t n = __shfl_up_sync(0xffffffffu, t.n, d);
        const double w = __shfl_up_sync(0xffffffffu, t.w, d);
        if (lane >= d) { t.n += n; t.w += w; }
    }
    if (lane == 31) { s.warp_n[warp] = t.n; s.warp_w[warp] = t.w; }
    Run e;
    e.n = __shfl_up_sync(0xffffffffu, t.n, 1);
    e.w = __shfl_up_sync(0xffffffffu, t.w, 1);
    if (lane == 0) e = {0u, 0.0};
    __syncthreads();
    all = {0u, 0.0};
    Run ahead = {0u, 0.0};
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) {
        if (w == warp) ahead = all;
        all.n += s.warp_n[w];
        all.w += s.warp_w[w];
    }
    e.n += ahead.n;
    e.w += ahead.w;
    __syncthreads();
    return e;
}

// The first block: from the counts of all to the cut (bf16) or to the bins that hold the cuts (fp32).  `place` counts bins from
// the highest one down, a thread has kBinsEach of them.
template <int DT>
__device__ __forceinline__ void solve_bins(const uint32_t* hist, CutShared& s, const CutParams& c, int blocks, int V) {
    const int tid = threadIdx.x;
    if (tid == 0) {
        s.found[0] = -1;                                     // place of the k-th token
        s.found[1] = s.found[2] = kBins;                     // of the highest one, and of the border of top-p
        s.work = {kCutDone, 0u, V, 0u, 0u};
        s.min_key = 0u;
    }
    uint32_t n[kBinsEach];
    double w[kBinsEach];
    Run mine = {0u, 0.0};
    static_assert(kBinsEach % 4 == 0 && kBins % 4 == 0, "whole vectors of bins");
#pragma unroll
    for (int j = 0; j < kBinsEach; j += 4) {
        const int bin = kBins - 4 - (tid * kBinsEach + j);
        const uint4 v = bin >= 0 ? *reinterpret_cast<const uint4*>(hist + bin) : make_uint4(0u, 0u, 0u, 0u);
        n[j] = v.w; n[j + 1] = v.z; n[j + 2] = v.y; n[j + 3] = v.x;
        mine.n += v.x + v.y + v.z + v.w;
    }
    double tiny = 0.0;                                       // the thread of that bin has what those weigh that share it
    if (tid == (kBins - 1 - kBinTinyPos) / kBinsEach) {
#pragma unroll
        for (int k = 0; k < kMaxCutCluster; ++k) tiny += k < blocks ? s.tiny[k] : 0.0;
    }
#pragma unroll
    for (int j = 0; j < kBinsEach; ++j) w[j] = 0.0;
    if (mine.n != 0u) {
        // (fp32: as if all of a bin were at its edge next to zero)
        const double2* table = reinterpret_cast<const double2*>(bin_weights + tid * kBinsEach);
#pragma unroll
        for (int j = 0; j < kBinsEach; j += 2)
            if (tid * kBinsEach + j < kBins) { const double2 t = __ldg(table + j / 2); w[j] = t.x; w[j + 1] = t.y; }
#pragma unroll
        for (int j = 0; j < kBinsEach; ++j) mine.w += n[j] * w[j];
    }
    mine.w += tiny;
    Run all;
    const Run before = scan_threads(mine, s, all);
    const bool cut_k = c.k && all.n > static_cast<uint32_t>(c.top_k);
    if (all.n == 0u) {                                       // nothing finite, and nothing above it either
        if (tid == 0) s.work.kind = kCutNone;
        return;
    }
    if (mine.n != 0u) {
        Run run = before;
#pragma unroll
        for (int j = 0; j < kBinsEach; ++j) {
            const int place = tid * kBinsEach + j, bin = kBins - 1 - place;
            if (n[j] != 0u) {
                if (run.n == 0u) {
                    s.found[1] = place;
                    if (DT == FSD_BF16 && c.m && one_value(bin)) s.min_key = min_p_key<DT>(c.min_p, bin_prefix(bin), bin_value<DT>(bin));
                }
                if (cut_k && run.n < c.top_k && run.n + n[j] >= c.top_k) {
                    s.found[0] = place;
                    s.work.ties = c.top_k - run.n;
                    s.goal = run.w + static_cast<double>(c.top_k - run.n) * w[j];
                }
            }
            run.n += n[j];
            run.w += bin == kBinTinyPos ? tiny : n[j] * w[j];
        }
    }
    __syncthreads();
    const int k_place = s.found[0], k_bin = kBins - 1 - k_place, top_bin = kBins - 1 - s.found[1];
    uint32_t top = bin_prefix(top_bin);
    double most = one_value(top_bin) ? bin_value<DT>(top_bin) : 0.0;
    if constexpr (DT == FSD_F32) {
        top = 0u;
        for (int k = 0; k < blocks; ++k) top = top > s.top[k] ? top : s.top[k];
        most = value_of<FSD_F32>(top);
    }
    // Values off the bins: above them, or a border in a bin of many; below them what is worth nothing beside a highest value of
    // at least -60 (e^-68 of it each) and is nothing but a count.
    const bool off = hist[kBinOver] != 0u || !one_value(top_bin) || (hist[kBinUnder] != 0u && most < -60.0) || (cut_k && !one_value(k_bin));
    const double goal = static_cast<double>(c.top_p) * (cut_k ? s.goal : all.w);
    int p_place = k_place;
    if (c.p && !off) {                                       // the first place at which the tokens so far weigh the goal
        int mine_at = kBins;
        if ((mine.n != 0u || tiny != 0.0) && !(before.w + mine.w < goal * (1.0 - 1e-9)) && before.w < goal) {      // (rounded in another order)
            Run run = before;
#pragma unroll
            for (int j = 0; j < kBinsEach; ++j) {
                const int place = tid * kBinsEach + j, bin = kBins - 1 - place;
                run.w += bin == kBinTinyPos ? tiny : n[j] * w[j];
                if (n[j] != 0u && run.w >= goal && mine_at == kBins) mine_at = place;
            }
        }
        mine_at = __reduce_min_sync(0xffffffffu, mine_at);
        if ((tid & 31) == 0 && mine_at < kBins) atomicMin(&s.found[2], mine_at);
        __syncthreads();
        p_place = s.found[2];
        if (cut_k && p_place > k_place) p_place = k_place;
        if (!(goal > 0.0)) p_place = s.found[1];
        if (p_place >= kBins) {                              // where two threads' sums meet: the first that starts at the goal
            mine_at = __reduce_min_sync(0xffffffffu, mine.n != 0u && before.w >= goal ? tid * kBinsEach : kBins);
            if ((tid & 31) == 0 && mine_at < kBins) atomicMin(&s.found[2], mine_at);
            __syncthreads();
            p_place = s.found[2];
            while (p_place < kBins && hist[kBins - 1 - p_place] == 0u) ++p_place;
            if (cut_k && p_place > k_place) p_place = k_place;
            if (p_place >= kBins) p_place = kBins - 1;       // (not reached: the goal is below the whole)
        }
    }
    const int p_bin = kBins - 1 - p_place;
    if (off || (c.p && !one_value(p_bin))) {
        if (tid == 0) s.work.kind = kCutByBits;
        return;
    }
    if constexpr (DT == FSD_BF16) {
        const bool has = (c.p || cut_k) && p_place / kBinsEach == tid;        // the thread that has the cut's bin
        if (has) {
            Run run = before;
#pragma unroll
            for (int j = 0; j < kBinsEach; ++j) {
                const int bin = kBins - 1 - (tid * kBinsEach + j);
                if (bin == p_bin) {
                    const bool at_k = cut_k && p_place == k_place;
                    long long t = c.p ? ties_below(run.w, w[j], goal, V) : V;
                    if (at_k && s.work.ties < t) t = s.work.ties;
                    s.work.ties = t >= n[j] ? V : t;                          // all of them
                    s.work.equal = n[j];
                    s.work.key = bin_prefix(bin);
                }
                run.w += bin == kBinTinyPos ? tiny : n[j] * w[j];
            }
        }
        if (has || (!c.p && !cut_k && tid == 0)) {
            if (s.min_key > s.work.key) { s.work.key = s.min_key; s.work.ties = V; }
            if (s.work.key == 0u) s.work.kind = kCutNone;
        }
    } else if (tid == 0) {
        s.found[3] = p_bin;
        if (cut_k) {
            s.work.kind = kCutRefineK;
            s.work.key = bin_prefix(k_bin);
        } else if (c.p) {
            s.work.kind = kCutRefineP;
            s.work.key = bin_prefix(p_bin);
        } else if (c.m) {
            s.work.key = min_p_key<DT>(c.min_p, top, most);
        } else {
            s.work.kind = kCutNone;                          // (fewer tokens than top_k)
        }
    }
}

// Counts, by the 8 bits above `shift`, the tokens whose keys have the upper bits `prefix` and are above `over`; with weights also
// what they weigh against the largest value of the bin's range (whole numbers of 1 / kFixed), and what all tokens above and below the
// prefix weigh against `most`.  All into the first block's shared memory.
template <bool WEIGHTS>
__device__ void count_bits(const RowSlice<FSD_F32>& row, CutShared& s, CutShared& first, int rank, uint32_t prefix, int shift, uint32_t over, double most) {
    const int tid = threadIdx.x;
    if (rank != 0) {
        for (int i = tid; i < 256; i += kRowThreads) { s.sub_n[i] = 0u; s.sub_w[i] = 0u; }
        __syncthreads();
    }
    const double edge = value_of<FSD_F32>(prefix << (shift + 8) | ((1u << (shift + 8)) - 1u));
    CountAndWeight above = {0, 0.0}, rest = {0, 0.0};
    for (int i = tid; i < row.n; i += kRowThreads) {
        const uint4 v = row.vecs[i];
        const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t k = key_of<FSD_F32>(bits[e]), high = k >> (shift + 8);
            if (WEIGHTS && bits[e] != 0xff800000u && k > over) {
                if (high != prefix) {
                    const double w = exp_of(static_cast<double>(__uint_as_float(bits[e])) - most);
                    if (high > prefix) above.w += w; else rest.w += w;
                }
            }
            if (high == prefix && k > over) {
                const uint32_t bin = k >> shift & 255u;
                atomicAdd(&s.sub_n[bin], 1u);
                if (WEIGHTS)
                    atomicAdd(reinterpret_cast<unsigned long long*>(&s.sub_w[bin]),
                              __double2ull_rn(exp_of(static_cast<double>(__uint_as_float(bits[e])) - edge) * kFixed));
            }
        }
    }
    if (WEIGHTS) {
        above = block_total(above, s.scratch);
        rest = block_total(rest, s.scratch);
        if (tid == 0) { first.above[rank] = above.w; first.rest[rank] = rest.w; }
    }
    __syncthreads();
    if (rank != 0)
        for (int i = tid; i < 256; i += kRowThreads)
            if (s.sub_n[i] != 0u) {
                atomicAdd(&first.sub_n[i], s.sub_n[i]);
                if (WEIGHTS) atomicAdd(reinterpret_cast<unsigned long long*>(&first.sub_w[i]), static_cast<unsigned long long>(s.sub_w[i]));
            }
}

// The first block tells the others what it found, and clears the counts for the next time.  Two places in turn: a block may still
// be reading what it was told before.
__device__ __forceinline__ CutResult tell_result(CutShared& s, cg::cluster_group& cluster, int rank, int blocks, int& turn, bool clear = true) {
    turn ^= 1;
    if (rank == 0) {
        const int tid = threadIdx.x;
        __syncthreads();
        if (tid < blocks) *cluster.map_shared_rank(&s.told[turn], tid) = s.work;
        if (clear)
            for (int i = tid; i < 256; i += kRowThreads) { s.sub_n[i] = 0u; s.sub_w[i] = 0u; }
    }
    cluster_barrier();
    return s.told[turn];
}

// The next bin in use above (up) or below a bin; -1 if there is none.  All of the first block's threads.
__device__ __forceinline__ int next_bin(const uint32_t* hist, CutShared& s, int bin, bool up) {
    if (threadIdx.x == 0) s.found[0] = up ? kBins : -1;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kRowThreads)
        if (hist[i] != 0u) {
            if (up && i > bin) atomicMin(&s.found[0], i);
            if (!up && i < bin) atomicMax(&s.found[0], i);
        }
    __syncthreads();
    const int found = s.found[0];
    __syncthreads();
    return found == kBins ? -1 : found;
}

__device__ __forceinline__ void at_least_min_p(CutShared& s, const CutParams& c, int V, uint32_t top) {       // one thread
    const uint32_t t = min_p_key<FSD_F32>(c.min_p, top, value_of<FSD_F32>(top));
    if (t > s.work.key) { s.work.key = t; s.work.ties = V; }
}

// fp32: from the bins of the cuts to the cuts.
__device__ CutResult refine(const RowSlice<FSD_F32>& row, const uint32_t* hist, CutShared& s, CutShared& first, cg::cluster_group& cluster, int rank, int blocks,
                            const CutParams& c, int V, uint32_t top, CutResult res, int& turn) {
    const int tid = threadIdx.x;
    const double most = value_of<FSD_F32>(top);
    const bool cut_k = res.kind == kCutRefineK;
    int p_bin = rank == 0 ? s.found[3] : 0;                 // (the first block's) the bin that may have the border of top-p
    if (cut_k) {
        for (int shift = 8; shift >= 0; shift -= 8) {
            count_bits<false>(row, s, first, rank, res.key, shift, 0u, most);
            cluster_barrier();
            if (rank == 0) {
                Run all;
                const int bin = 255 - tid;
                const uint32_t n = tid < 256 ? s.sub_n[bin] : 0u;
                const Run before = scan_threads({n, 0.0}, s, all);
                if (before.n < res.ties && before.n + n >= res.ties) {
                    s.work.key = res.key << 8 | static_cast<uint32_t>(bin);
                    s.work.ties = res.ties - before.n;
                    if (shift == 0) s.work.over = s.work.ties >= n;            // whether all that are equal are kept
                }
                __syncthreads();
                if (tid == 0 && shift == 0 && !c.p) {
                    s.work.kind = kCutDone;
                    if (s.work.over) s.work.ties = V;
                    if (c.m) at_least_min_p(s, c, V, top);
                }
            }
            res = tell_result(s, cluster, rank, blocks, turn);
        }
        if (!c.p) return res;
    }
    // Tokens above `over` are in the top_k, and of those equal to it k_ties.
    const uint32_t over = cut_k ? res.key : 0u;
    const long long k_ties = cut_k ? res.ties : 0;
    const bool all_of_k = cut_k && res.over;
    const double of_ties = cut_k ? static_cast<double>(k_ties) * exp_of(static_cast<double>(value_of<FSD_F32>(over)) - most) : 0.0;
    if (cut_k) {
        if (rank == 0 && tid == 0) s.work = {kCutRefineP, bin_prefix(p_bin), 0, 0u, 0u};
        res = tell_result(s, cluster, rank, blocks, turn);
    }
    // The bin is a guess, made with the middles of the bins; the sums say whether to move to the next one in use.  (Where rounding would
    // send it back and forth, the border is between the two.)
    int last_move = 0;
    while (res.kind == kCutRefineP) {
        const uint32_t prefix = res.key;
        count_bits<true>(row, s, first, rank, prefix, 8, over, most);
        cluster_barrier();
        if (rank == 0) {
            double above = 0.0, rest = 0.0;
            for (int k = 0; k < blocks; ++k) { above += s.above[k]; rest += s.rest[k]; }
            const double unit = exp_of(static_cast<double>(value_of<FSD_F32>(prefix << 16 | 0xffffu)) - most) / kFixed;
            Run all;
            const int bin = 255 - tid;
            const double w = tid < 256 ? static_cast<double>(s.sub_w[bin]) * unit : 0.0;
            const uint32_t n = tid < 256 ? s.sub_n[bin] : 0u;
            const Run before = scan_threads({n, w}, s, all);
            const double goal = static_cast<double>(c.top_p) * (above + all.w + rest + of_ties);
            if (tid == 0) { s.found[1] = -1; s.found[2] = 256; }
            __syncthreads();
            if (n != 0) {
                atomicMax(&s.found[1], tid);                                      // the last sub-bin in use
                if (above + before.w + w >= goal) atomicMin(&s.found[2], tid);
            }
            __syncthreads();
            int place = s.found[2];
            bool up = goal > 0.0 && above >= goal, down = !up && place == 256;
            if (down && s.found[1] >= 0 && last_move > 0) { place = s.found[1]; down = false; }
            if (up && s.found[1] >= 0 && last_move < 0) up = false;               // (place is its first sub-bin in use)
            if (down && cut_k && prefix <= over >> 16) {                          // the border is among the tokens equal to the k-th
                if (tid == 0) {
                    const long long t = ties_below(above + all.w, of_ties / static_cast<double>(k_ties), goal, V);
                    s.work = {kCutDone, over, t < k_ties ? t : all_of_k ? V : k_ties, 0u, 0u};
                }
            } else if (up || down) {
                p_bin = next_bin(hist, s, p_bin, up);
                last_move = up ? 1 : -1;
                if (tid == 0) {
                    if (p_bin < 0 || !one_value(p_bin)) s.work.kind = kCutByBits;
                    else s.work.key = bin_prefix(p_bin);
                }
            } else if (tid == place) {
                s.work.key = prefix << 8 | static_cast<uint32_t>(bin);
                s.work.kind = kCutRefineK;                                        // (the last 8 bits)
                s.goal = goal;
                s.above_goal = above + before.w;
            }
        }
        res = tell_result(s, cluster, rank, blocks, turn);
    }
    if (res.kind == kCutRefineK) {
        const uint32_t prefix = res.key;
        count_bits<false>(row, s, first, rank, prefix, 0, over, most);
        cluster_barrier();
        if (rank == 0) {
            Run all;
            const int bin = 255 - tid;
            const uint32_t key = prefix << 8 | static_cast<uint32_t>(bin);
            const uint32_t n = tid < 256 ? s.sub_n[bin] : 0u;
            const double w = n != 0 ? exp_of(static_cast<double>(value_of<FSD_F32>(key)) - most) : 0.0;
            const Run before = scan_threads({n, static_cast<double>(n) * w}, s, all);
            if (tid == 0) s.found[2] = 256;
            __syncthreads();
            // (where rounding leaves the last of them short of the goal it is the border all the same)
            if (n != 0 && (s.above_goal + before.w + static_cast<double>(n) * w >= s.goal || before.n + n == all.n)) atomicMin(&s.found[2], tid);
            __syncthreads();
            if (tid == s.found[2]) {
                const long long t = ties_below(s.above_goal + before.w, w, s.goal, V);
                s.work = {kCutDone, key, t >= n ? V : t, 0u, 0u};
            }
            __syncthreads();
        }
    }
    if (res.kind != kCutByBits && (res.kind == kCutRefineK || c.m)) {
        if (rank == 0 && tid == 0 && c.m) at_least_min_p(s, c, V, top);
        res = tell_result(s, cluster, rank, blocks, turn);
    }
    return res;
}

template <int DT>
__device__ __forceinline__ void words_of(const uint4& v, uint32_t (&bits)[Logit<DT>::kPerVec]) {      // widened
    if constexpr (DT == FSD_BF16) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) bits[e] = (e & 1) ? w[e / 2] & 0xffff0000u : w[e / 2] << 16;
    } else {
        bits[0] = v.x; bits[1] = v.y; bits[2] = v.z; bits[3] = v.w;
    }
}

// One value into the bins, or (BY -1) out of them; those that share a bin with others of their size are weighed.
template <int BY>
__device__ __noinline__ double count_value(uint32_t bits, uint32_t* hist) {
    if (bits == 0xff800000u) return 0.0;
    const uint32_t mag = bits >> 16 & 0x7fffu, u = (mag < kMagLo ? kMagLo : mag > kMagHi ? kMagHi : mag) - kMagLo;
    int bin = static_cast<int>(u ^ static_cast<uint32_t>(static_cast<int>(bits) >> 31)) + kHalfBins;
    if ((bits & 0x7fffffffu) > 0x7f800000u) bin = kBinOver;
    atomicAdd(&hist[bin], static_cast<uint32_t>(BY));
    if (u != 0u) return 0.0;
    const double y = static_cast<double>(__uint_as_float(bits));                  // below 2^-8: the series up to y^6 / 720 (y^7 / 5040 < 3e-21)
    return 1.0 + y * (1.0 + y * (1.0 / 2.0 + y * (1.0 / 6.0 + y * (1.0 / 24.0 + y * (1.0 / 120.0 + y * (1.0 / 720.0))))));
}
// A vector of values into the bins; returns what is weighed.  bf16: two at a time, in halves of a word.
template <int DT>
__device__ __forceinline__ double count_vec(const uint4& v, uint32_t* hist) {
    double tiny = 0.0;
    if constexpr (DT == FSD_BF16) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t bin[4], lowest = 0xffffffffu, highest = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t m = __vminu2(__vmaxu2(w[k] & 0x7fff7fffu, kMagLo * 0x10001u), kMagHi * 0x10001u);
            lowest = __vminu2(lowest, m);
            highest = __vmaxu2(highest, m);
            uint32_t sign;                                  // each half's sign in all of its bits
            asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(sign) : "r"(w[k]));
            bin[k] = (m - kMagLo * 0x10001u) ^ sign;
        }
        if ((lowest & 0xffffu) == kMagLo || lowest >> 16 == kMagLo || (highest & 0xffffu) == kMagHi || highest >> 16 == kMagHi) {
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                const uint32_t two = k < 2 ? (k < 1 ? v.x : v.y) : (k < 3 ? v.z : v.w);
                tiny += count_value<1>(two << 16, hist) + count_value<1>(two & 0xffff0000u, hist);
            }
        } else {
            uint32_t* mid = hist + kHalfBins;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                atomicAdd(mid + static_cast<int16_t>(bin[k]), 1u);
                atomicAdd(mid + (static_cast<int>(bin[k]) >> 16), 1u);
            }
        }
    } else {
        const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t mag = bits[e] >> 16 & 0x7fffu;
            if (mag <= kMagLo || mag >= kMagHi) tiny += count_value<1>(bits[e], hist);
            else atomicAdd(&hist[static_cast<int>((mag - kMagLo) ^ static_cast<uint32_t>(static_cast<int>(bits[e]) >> 31)) + kHalfBins], 1u);
        }
    }
    return tiny;
}

// How many of a vector's values are equal to one.
template <int DT>
__device__ __forceinline__ int equal_in(const uint4& v, float value) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t n = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DT == FSD_BF16)
            n += __heq2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[k]), __bfloat162bfloat162(__float2bfloat16_rn(value))) & 0x10001u;
        else n += __uint_as_float(w[k]) == value;
    }
    return static_cast<int>(DT == FSD_BF16 ? (n & 0xffffu) + (n >> 16) : n);
}
// A vector with -inf for what is below the cut, and (above) for what is equal to it.
template <int DT>
__device__ __forceinline__ uint4 cut_vec(const uint4& v, float value, bool above) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (DT == FSD_BF16) {
        const __nv_bfloat162 cut = __bfloat162bfloat162(__float2bfloat16_rn(value));      // (it is a value of bf16)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162*>(&w[k]);
            const uint32_t keep = above ? __hgt2_mask(y, cut) : __hge2_mask(y, cut);
            w[k] = (w[k] & keep) | (0xff80ff80u & ~keep);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float y = __uint_as_float(w[k]);
            w[k] = (above ? y > value : y >= value) ? w[k] : 0xff800000u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// A vector of which at most `left` of those equal to the cut are kept, and none from its id number `end` on.
template <int DT>
__device__ __noinline__ uint4 cut_some(uint4 v, float value, int left, int end) {
    constexpr int N = Logit<DT>::kPerVec;
    uint32_t bits[N];
    words_of<DT>(v, bits);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = __uint_as_float(bits[e]);
        const bool at = y == value, keep = y > value || (at && left > 0 && e < end);
        left -= at;
        if (!keep) bits[e] = 0xff800000u;
    }
    if constexpr (DT == FSD_BF16)
        return make_uint4(bits[0] >> 16 | bits[1], bits[2] >> 16 | bits[3], bits[4] >> 16 | bits[5], bits[6] >> 16 | bits[7]);
    else return make_uint4(bits[0], bits[1], bits[2], bits[3]);
}

// raw: the rows are processed already.
template <int DT>
__global__ void __launch_bounds__(kRowThreads, 2) fsd_cut_kernel(const ProcArgs a, int slice, bool raw) {
    constexpr int N = Logit<DT>::kPerVec;
    using elem = typename Logit<DT>::elem;
    extern __shared__ uint4 on_chip[];
    __shared__ CutShared s;
    uint32_t* hist = reinterpret_cast<uint32_t*>(on_chip + slice);
    uint32_t* drafted_ids = hist + kBins;                   // a bit for each of the slice's ids, from a multiple of 32 on; where tokens are drafted
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int blocks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int all = a.rows[0] + a.rows[1], line = blockIdx.x / blocks, b = line / all, q = line % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    const size_t at = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
    const elem* in = static_cast<const elem*>(raw ? a.out[side] : a.in[side]) + at;
    elem* out = static_cast<elem*>(a.out[side]) + at;
    const int lies = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16 / sizeof(elem));
    const bool alike = (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const int row_vecs = (a.V + lies + N - 1) / N, v0 = rank * slice;
    RowSlice<DT> row = {on_chip, row_vecs - v0 < slice ? (row_vecs > v0 ? row_vecs - v0 : 0) : slice, v0 * N - lies};

    constexpr int kAtOnce = 4;
    uint4 got[kAtOnce];
    const auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = i0 + u * kRowThreads, t0 = row.first + i * N;
            if (i < row.n) got[u] = load_ids<DT>(in, t0, a.V, t0 >= 0 && t0 + N <= a.V);
        }
    };
    uint32_t setting = 0u;
    if (tid < 8) {                                          // the sequence's settings, all read at once
        const void* const at_b[8] = {a.top_k, a.top_p, a.min_p, a.repetition, a.frequency, a.presence, a.temperature, nullptr};
        const void* from = nullptr;
#pragma unroll
        for (int k = 0; k < 8; ++k) from = k == tid ? at_b[k] : from;
        setting = from != nullptr ? __ldg(static_cast<const uint32_t*>(from) + b) : tid == 1 || tid == 3 ? 0x3f800000u : 0u;
    }
    fetch(tid);
    const int ctx = context_row(a, b, side, r);
    const int drafts = !raw && a.penalties && a.tokens != nullptr ? a.P : 0;
    const bool history = !raw && a.penalties && a.seen != nullptr;
    const uint32_t* seen = history ? a.seen + static_cast<size_t>(b) * a.W : nullptr;
    const uint32_t* allowed = !raw && a.allowed != nullptr ? a.allowed + (static_cast<size_t>(b) * (a.P + 1) + ctx) * a.W : nullptr;
    const int ids_lo = row.first > 0 ? row.first : 0, ids_hi = row.first + row.n * N < a.V ? row.first + row.n * N : a.V;   // of the slice
    const int word0 = ids_lo >> 5, n_words = ids_hi > ids_lo ? ((ids_hi + 31) >> 5) - word0 : 0;
    for (int i = tid; i < kBins / 4; i += kRowThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (drafts > 0)
        for (int i = tid; i < n_words; i += kRowThreads) drafted_ids[i] = 0u;
    if (DT == FSD_F32)
        for (int i = tid; i < 256; i += kRowThreads) { s.sub_n[i] = 0u; s.sub_w[i] = 0u; }
    if (tid < 8) s.settings[tid] = setting;
    __syncthreads();
    cluster_arrive();                                       // from here on others may add to the first block's counts
    for (int j = tid; j < drafts; j += kRowThreads) {
        const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j);
        if (t >= ids_lo && t < ids_hi) atomicOr(&drafted_ids[(t >> 5) - word0], 1u << (t & 31));
    }
    const CutParams c = cut_params(s.settings, a.V);
    const bool cutting = c.k || c.p || c.m;
    const SeqParams p = seq_params(s.settings + 3);

    // the slice: read, processed, counted, kept
    double tiny = 0.0;
    uint32_t top = 0u;
    for (int i0 = tid; i0 < row.n; i0 += kAtOnce * kRowThreads) {
        if (i0 != tid) fetch(i0);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = i0 + u * kRowThreads, t0 = row.first + i * N;
            if (i >= row.n) break;
            uint4 v = got[u];
            if (!raw) {
                uint32_t may = allowed != nullptr ? bits8(allowed, t0, 4 * a.W) : 0xffu;
                if (t0 < 0 || t0 + N > a.V) may &= ids_of<N>(t0, a.V);        // (what is not in the row counts as masked)
                v = process_vec<DT>(v, may, p.inv_temp);
            }
            row.vecs[i] = v;
            if (!cutting) continue;
            tiny += count_vec<DT>(v, hist);
            if constexpr (DT == FSD_F32) {
                const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
                const uint32_t sparse = (history ? bits8(seen, t0, 4 * a.W) : 0u) | (drafts > 0 ? bits8(drafted_ids, t0 - word0 * 32, 4 * n_words) : 0u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t k = key_of<DT>(bits[e]);
                    if (!(sparse >> e & 1u)) top = top > k ? top : k;
                }
            }
        }
    }
    // Then the ids that are used or drafted, one a thread: what was counted for them without a penalty is taken back.  A warp takes
    // 32 words of the bitmaps at a time, each kRowWarps from the last (low ids are used far more often), and lists their bits,
    // so that its threads have as many each.
    if (history || drafts > 0) {
        __syncthreads();
        LogitWord<DT>* words = reinterpret_cast<LogitWord<DT>*>(row.vecs) - row.first;      // by id
        for (int w0 = warp; w0 < n_words; w0 += kRowWarps * 32) {
            const int w = w0 + lane * kRowWarps;
            uint32_t used = 0u, draft = 0u;
            if (w < n_words) {
                uint32_t may = allowed != nullptr ? allowed[word0 + w] : 0xffffffffu;
                const int t = (word0 + w) * 32;
                if (t < ids_lo) may &= 0xffffffffu << (ids_lo - t);
                if (t + 32 > ids_hi) may &= 0xffffffffu >> (t + 32 - ids_hi);
                used = history ? __ldg(seen + word0 + w) & may : 0u;
                draft = drafts > 0 ? drafted_ids[w] & may : 0u;
            }
            uint32_t todo = used | draft;
            int at = __popc(todo);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, at, d);
                if (lane >= d) at += o;
            }
            const int total = __shfl_sync(0xffffffffu, at, 31);
            at -= __popc(todo);
            for (int base = 0; base < total; base += 256) {
                while (todo != 0u && at < base + 256) {
                    s.list[warp][at - base] = static_cast<uint16_t>(lane * 32 + __ffs(static_cast<int>(todo)) - 1);
                    todo &= todo - 1u;
                    ++at;
                }
                __syncwarp();
                const int n = total - base < 256 ? total - base : 256;
#pragma unroll 4
                for (int k0 = 0; k0 < n; k0 += 32) {
                    const int k = k0 + lane, l = k < n ? s.list[warp][k] : 0;
                    const uint32_t is_used = __shfl_sync(0xffffffffu, used, l >> 5) >> (l & 31) & 1u;
                    const uint32_t is_draft = __shfl_sync(0xffffffffu, draft, l >> 5) >> (l & 31) & 1u;
                    if (k >= n) continue;
                    const int t = (word0 + w0 + (l >> 5) * kRowWarps) * 32 + (l & 31);
                    const int count = is_used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1;
                    const float x = read_id<DT>(in, t);
                    const int d = is_draft ? drafted(a, b, ctx, t) : 0;
                    const uint32_t before = words[t];
                    write_id<DT>(words, t, process_id(x, count, d, 0.f, false, p));
                    if (!cutting) continue;
                    const uint32_t now = words[t];
                    tiny += count_value<1>(__float_as_uint(float_of<DT>(now)), hist) - count_value<-1>(__float_as_uint(float_of<DT>(before)), hist);
                    if constexpr (DT == FSD_F32) { const uint32_t key = key_of<DT>(now); top = top > key ? top : key; }
                }
                __syncwarp();
            }
        }
    }
    if (!cutting) {                                         // (the whole cluster: it is the sequence that asks)
        __syncthreads();
        for (int i = tid; i < row.n; i += kRowThreads) {
            const int t0 = row.first + i * N;
            store_ids<DT>(out, t0, a.V, t0 >= 0 && t0 + N <= a.V && alike, row.vecs[i]);
        }
        cluster_wait();
        return;
    }

    CutShared& first = *cluster.map_shared_rank(&s, 0);
    if (__any_sync(0xffffffffu, tiny != 0.0)) tiny = warp_sum(tiny);
    if constexpr (DT == FSD_F32) top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) { s.warp_w[warp] = tiny; s.warp_n[warp] = top; }
    __syncthreads();
    cluster_wait();
    if (tid == 0) {
        tiny = 0.0;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) { tiny += s.warp_w[w]; top = top > s.warp_n[w] ? top : s.warp_n[w]; }
        first.tiny[rank] = tiny;
        first.top[rank] = top;
    }
    if (rank != 0) {
        uint32_t* sums = cluster.map_shared_rank(hist, 0);
        for (int i = tid; i < kBins / 4; i += kRowThreads) {
            const uint4 v = reinterpret_cast<const uint4*>(hist)[i];
            if (v.x != 0u) atomicAdd(sums + 4 * i, v.x);
            if (v.y != 0u) atomicAdd(sums + 4 * i + 1, v.y);
            if (v.z != 0u) atomicAdd(sums + 4 * i + 2, v.z);
            if (v.w != 0u) atomicAdd(sums + 4 * i + 3, v.w);
        }
    }
    cluster_barrier();
    if (rank == 0) {
        solve_bins<DT>(hist, s, c, blocks, a.V);
        if (DT == FSD_F32 && tid > 0 && tid < blocks)
            for (int k = 0; k < blocks; ++k) cluster.map_shared_rank(&s, tid)->top[k] = s.top[k];
    }
    int turn = 0;
    CutResult res = tell_result(s, cluster, rank, blocks, turn, DT == FSD_F32);
    if constexpr (DT == FSD_F32) {
        if (res.kind == kCutRefineK || res.kind == kCutRefineP) {
            top = 0u;
            for (int k = 0; k < blocks; ++k) top = top > s.top[k] ? top : s.top[k];
            res = refine(row, hist, s, first, cluster, rank, blocks, c, a.V, top, res, turn);
        }
    }

    uint32_t key = res.key;
    int until = a.V;                                        // of the tokens at the cut, those from this id on are not kept
    bool keep_all = res.kind == kCutNone;
    if (res.kind == kCutByBits) {
        const auto total = [&](CountAndWeight v) {
            v = block_total(v, s.scratch);
            turn ^= 1;
            if (tid < blocks) cluster.map_shared_rank(&s, tid)->slots[turn][rank] = v;
            cluster_barrier();
            CountAndWeight t = {0, 0.0};
            for (int k = 0; k < blocks; ++k) { t.n += s.slots[turn][k].n; t.w += s.slots[turn][k].w; }
            return t;
        };
        const auto largest = [&](uint32_t k) {
            k = block_largest(k, s.scratch);
            turn ^= 1;
            if (tid < blocks) cluster.map_shared_rank(&s, tid)->slots[turn][rank].n = k;
            cluster_barrier();
            for (int j = 0; j < blocks; ++j) k = k > static_cast<uint32_t>(s.slots[turn][j].n) ? k : static_cast<uint32_t>(s.slots[turn][j].n);
            return k;
        };
        const Cut cut = find_cut<DT>(reinterpret_cast<const LogitWord<DT>*>(row.vecs), row.n * N, row.first, a.V, c, total, largest);
        key = cut.key;
        keep_all = !cut.any;
        if (cut.any) until = cut.until;
    }
    const long long ties = res.kind == kCutDone ? res.ties : a.V;
    const float value = value_of<DT>(key);
    // Where only the first `ties` of the tokens at the cut are kept: how many of them are in front of this block's.  bf16: the other
    // blocks' counts say it, the first block's own being what is missing from the sum, which it has.
    long long before = 0;
    bool count = ties < a.V;
    if (DT == FSD_BF16 && count) {
        const int bin = bin_of_value(value);
        uint32_t mine = 0u, behind = 0u;
        uint32_t theirs[kMaxCutCluster];
#pragma unroll
        for (int k = 1; k < kMaxCutCluster; ++k) theirs[k] = k < blocks && k >= rank ? *cluster.map_shared_rank(hist + bin, k) : 0u;
#pragma unroll
        for (int k = 1; k < kMaxCutCluster; ++k) {
            behind += theirs[k];
            if (k == rank) mine = theirs[k];
        }
        if (rank == 0) mine = res.equal - behind;
        else before = static_cast<long long>(res.equal) - behind;
        if (before >= ties || before + mine <= ties) count = false;
        cluster_arrive();                                   // (none leaves before the others have read its counts)
    }
    // Each warp has a run of the slice, and counts those in it.
    const int run = (row.n + kRowWarps - 1) / kRowWarps, w0 = warp * run < row.n ? warp * run : row.n, w1 = w0 + run < row.n ? w0 + run : row.n;
    int left = ties < a.V && before >= ties ? 0 : INT_MAX, mine = 0;      // how many of those in the warp's run are kept, and how many there are
    if (count) {
        for (int i = w0 + lane; i < w1; i += 32) mine += equal_in<DT>(row.vecs[i], value);
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) s.warp_n[warp] = static_cast<uint32_t>(mine);
        __syncthreads();
        int sum = 0, ahead = 0;
        for (int w = 0; w < kRowWarps; ++w) { if (w == warp) ahead = sum; sum += static_cast<int>(s.warp_n[w]); }
        if constexpr (DT == FSD_F32) {
            if (tid < blocks) cluster.map_shared_rank(&s, tid)->equal[rank] = sum;
            cluster_barrier();
            for (int k = 0; k < rank; ++k) before += s.equal[k];
        }
        before += ahead;
        left = ties <= before ? 0 : ties - before < mine ? static_cast<int>(ties - before) : INT_MAX;
    }
    const bool some = left > 0 && left != INT_MAX;          // the one run that the last of them is in
    const bool above = left == 0;                           // none in this run: what is kept is above the cut
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane;
        const bool in_run = i < w1;
        uint4 v = in_run ? row.vecs[i] : make_uint4(0u, 0u, 0u, 0u);
        const int t0 = row.first + i * N;
        if (some || until < a.V) {
            if (some) {
                const int equal = in_run ? equal_in<DT>(v, value) : 0;
                int sum = equal;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, sum, d);
                    if (lane >= d) sum += o;
                }
                const int rank_of = sum - equal;            // of the run's tokens at the cut, how many are before this vector's
                const int all_of_them = __shfl_sync(0xffffffffu, sum, 31);
                v = cut_some<DT>(v, value, left - rank_of, N);
                left -= all_of_them;
            } else {
                v = cut_some<DT>(v, value, INT_MAX, until - t0);
            }
        } else if (!keep_all) {
            v = cut_vec<DT>(v, value, above);
        }
        if (in_run) store_ids<DT>(out, t0, a.V, t0 >= 0 && t0 + N <= a.V && alike, v);
    }
    if (DT == FSD_BF16 && ties < a.V) cluster_wait();
}

// ---- bf16: a block per row ---------------------------------------------------------------
// The block reads the row twice and keeps none of it: once to count its values, and again, from the L2 cache for the most part
// (two blocks an SM have 90 MB of rows of 152064 on the way), to write it.  No block waits for another, which is what most of
// a cluster's time went into: 64 x 17 x 152064 took 660 us that way.
// Sparse ids, whose penalties the count leaves out at first, are listed in front: a bitmap of the row's, the sum of its bits up to each word, and for
// each id what becomes of it, worked out once, one a thread, when what was counted for it is taken back.
struct RowsShape {             // of the dynamic shared memory; the last two are in words and ids
    int words, cap;
};
struct RowsShared {
    CutShared cut;
    uint32_t equal[2][kRowWarps];
    int n_sparse;
};

__device__ __forceinline__ float value_at(const uint4& v, int e) {
    const uint32_t w = e < 4 ? (e < 2 ? v.x : v.y) : (e < 6 ? v.z : v.w);
    return (e & 1) ? bf16_hi(w) : bf16_lo(w);
}
__device__ __forceinline__ void put_at(uint4& v, int e, uint32_t half) {
    const uint32_t sel = (e & 1) ? 0x5410u : 0x3254u;
    const int w = e >> 1;
    v.x = w == 0 ? __byte_perm(v.x, half, sel) : v.x;
    v.y = w == 1 ? __byte_perm(v.y, half, sel) : v.y;
    v.z = w == 2 ? __byte_perm(v.z, half, sel) : v.z;
    v.w = w == 3 ? __byte_perm(v.w, half, sel) : v.w;
}

__global__ void __launch_bounds__(kRowThreads, 2) fsd_cut_rows_kernel(const ProcArgs a, const RowsShape shape, bool raw) {
    constexpr int DT = FSD_BF16, N = 8, kAtOnce = 4, kTile = kAtOnce * kRowThreads;
    extern __shared__ uint4 on_chip[];
    __shared__ RowsShared s;
    uint32_t* hist = reinterpret_cast<uint32_t*>(on_chip);
    uint32_t* bitmap = hist + kBins;                        // of the sparse ids
    uint32_t* list = bitmap + shape.words;                  // them
    uint16_t* becomes = reinterpret_cast<uint16_t*>(list + shape.cap);
    uint16_t* ahead = becomes + shape.cap;                  // how many of them are in front of a word
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int all = a.rows[0] + a.rows[1], b = blockIdx.x / all, q = blockIdx.x % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    const size_t at = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
    const uint16_t* in = static_cast<const uint16_t*>(raw ? a.out[side] : a.in[side]) + at;
    uint16_t* out = static_cast<uint16_t*>(a.out[side]) + at;
    const int lies = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16 / 2);
    const bool alike = (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const int n_vecs = (a.V + lies + N - 1) / N;
    // a warp has kAtOnce runs of 32 vectors of a tile, one behind the other
    const auto vec_of = [&](int tile, int u) { return tile + (warp * kAtOnce + u) * 32 + lane; };
    uint4 got[kAtOnce];
    const auto fetch = [&](int tile) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = vec_of(tile, u), t0 = i * N - lies;
            if (i < n_vecs) got[u] = load_ids<DT>(in, t0, a.V, t0 >= 0 && t0 + N <= a.V);
        }
    };
    uint32_t setting = 0u;
    if (tid < 8) {                                          // the sequence's settings, all read at once
        const void* const at_b[8] = {a.top_k, a.top_p, a.min_p, raw ? nullptr : a.repetition, raw ? nullptr : a.frequency, raw ? nullptr : a.presence,
                                     raw ? nullptr : a.temperature, nullptr};
        const void* from = nullptr;
#pragma unroll
        for (int k = 0; k < 8; ++k) from = k == tid ? at_b[k] : from;
        setting = from != nullptr ? __ldg(static_cast<const uint32_t*>(from) + b) : tid == 1 || tid == 3 ? 0x3f800000u : 0u;
    }
    fetch(0);
    const int ctx = context_row(a, b, side, r);
    const int drafts = !raw && a.penalties && a.tokens != nullptr && ctx > 0 ? a.P : 0;
    const bool history = !raw && a.penalties && a.seen != nullptr, sparse = history || drafts > 0;
    const uint32_t* seen = history ? a.seen + static_cast<size_t>(b) * a.W : nullptr;
    const uint32_t* allowed = !raw && a.allowed != nullptr ? a.allowed + (static_cast<size_t>(b) * (a.P + 1) + ctx) * a.W : nullptr;
    for (int i = tid; i < kBins / 4; i += kRowThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < 8) s.cut.settings[tid] = setting;
    if (sparse) {
        for (int w = tid; w < a.W; w += kRowThreads) {
            uint32_t bits = history ? __ldg(seen + w) : 0u;
            if (allowed != nullptr) bits &= __ldg(allowed + w);
            if (w == a.W - 1 && (a.V & 31)) bits &= (1u << (a.V & 31)) - 1u;
            bitmap[w] = bits;
        }
    }
    __syncthreads();
    const CutParams c = cut_params(s.cut.settings, a.V);
    const SeqParams p = seq_params(s.cut.settings + 3);
    const bool cutting = c.k || c.p || c.m;
    const auto process = [&](const uint4& v, int t0) {
        uint32_t may = allowed != nullptr ? bits8(allowed, t0, 4 * a.W) : 0xffu;
        if (t0 < 0 || t0 + N > a.V) may &= ids_of<N>(t0, a.V);                // (what is not in the row counts as masked)
        return process_vec<DT>(v, may, p.inv_temp);
    };
    // what becomes of a sparse id
    const auto value_of_id = [&](int t, float x, int count) {
        return process_id(x, count, drafts > 0 ? drafted(a, b, ctx, t) : 0, 0.f, false, p);
    };
    bool listed = false;
    if (sparse) {
        if (drafts > 0) {
            for (int j = ctx - 1 - tid; j >= 0 && a.parent == nullptr; j -= kRowThreads) {
                const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j);
                if (t >= 0 && t < a.V && (allowed == nullptr || (__ldg(allowed + (t >> 5)) >> (t & 31) & 1u))) atomicOr(&bitmap[t >> 5], 1u << (t & 31));
            }
            if (a.parent != nullptr && tid == 0)
                for (int j = ctx - 1; j >= 0; j = node_before(a, b, j)) {
                    const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j);
                    if (t >= 0 && t < a.V && (allowed == nullptr || (__ldg(allowed + (t >> 5)) >> (t & 31) & 1u))) atomicOr(&bitmap[t >> 5], 1u << (t & 31));
                }
            __syncthreads();
        }
        const int each = (a.W + kRowThreads - 1) / kRowThreads, w0 = tid * each, w1 = w0 + each < a.W ? w0 + each : a.W;
        Run mine = {0u, 0.0}, total;
        for (int w = w0; w < w1; ++w) mine.n += __popc(bitmap[w]);
        uint32_t n = scan_threads(mine, s.cut, total).n;
        listed = total.n <= static_cast<uint32_t>(shape.cap);                 // (else each vector works its own out)
        if (tid == 0) s.n_sparse = static_cast<int>(total.n);
        if (listed)
            for (int w = w0; w < w1; ++w) {
                ahead[w] = static_cast<uint16_t>(n);
                for (uint32_t todo = bitmap[w]; todo != 0u; todo &= todo - 1u) list[n++] = w * 32 + __ffs(static_cast<int>(todo)) - 1;
            }
    }
    __syncthreads();
    const int n_sparse = sparse ? s.n_sparse : 0;
    // a vector with its sparse ids as they become
    const auto patch = [&](uint4 v, const uint4& was, int t0) {
        uint32_t todo = bits8(bitmap, t0, 4 * a.W);
        while (todo != 0u) {
            const int e = __ffs(static_cast<int>(todo)) - 1, t = t0 + e;
            todo &= todo - 1u;
            uint32_t half;
            if (listed) {
                half = becomes[ahead[t >> 5] + __popc(bitmap[t >> 5] & ((1u << (t & 31)) - 1u))];
            } else {
                const bool used = history && (__ldg(seen + (t >> 5)) >> (t & 31) & 1u);
                half = pack_bf16(value_of_id(t, value_at(was, e), used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1), 0.f);
            }
            put_at(v, e, half);
        }
        return v;
    };

    CutResult res = {kCutNone, 0u, a.V, 0u, 0u};
    if (cutting) {
        double tiny = 0.0;
        for (int tile = 0; tile < n_vecs; tile += kTile) {
            if (tile > 0) fetch(tile);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int i = vec_of(tile, u), t0 = i * N - lies;
                if (i >= n_vecs) break;
                uint4 v = process(got[u], t0);
                if (n_sparse > 0 && !listed) v = patch(v, got[u], t0);
                tiny += count_vec<DT>(v, hist);
            }
        }
        if (listed) {
            const uint16_t* row = in;
#pragma unroll 4
            for (int k = tid; k < n_sparse; k += kRowThreads) {
                const int t = list[k];
                const bool used = history && (__ldg(seen + (t >> 5)) >> (t & 31) & 1u);
                const int count = used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1;
                const float x = read_id<DT>(row, t);
                const uint32_t was = pack_bf16(__fmul_rn(x, p.inv_temp), 0.f) & 0xffffu, now = pack_bf16(value_of_id(t, x, count), 0.f) & 0xffffu;
                becomes[k] = static_cast<uint16_t>(now);
                tiny += count_value<1>(now << 16, hist) - count_value<-1>(was << 16, hist);
            }
        }
        if (__any_sync(0xffffffffu, tiny != 0.0)) tiny = warp_sum(tiny);
        if (lane == 0) s.cut.warp_w[warp] = tiny;
        __syncthreads();
        if (tid == 0) {
            tiny = 0.0;
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) tiny += s.cut.warp_w[w];
            s.cut.tiny[0] = tiny;
        }
        __syncthreads();
        solve_bins<DT>(hist, s.cut, c, 1, a.V);
        __syncthreads();
        res = s.cut.work;
    } else if (listed) {
        for (int k = tid; k < n_sparse; k += kRowThreads) {
            const int t = list[k];
            const bool used = history && (__ldg(seen + (t >> 5)) >> (t & 31) & 1u);
            becomes[k] = static_cast<uint16_t>(pack_bf16(value_of_id(t, read_id<DT>(in, t), used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1), 0.f));
        }
        __syncthreads();
    }

    // the row again, cut off
    const bool cut = res.kind == kCutDone;
    const float value = value_of<DT>(res.key);
    long long left = cut && res.ties < a.V ? res.ties : LLONG_MAX;             // how many of the tokens equal to the cut are still kept
    int turn = 0;
    for (int tile = 0; tile < n_vecs; tile += kTile) {
        if (tile > 0 || n_vecs > kTile || !cutting) fetch(tile);
        int equal = 0;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = vec_of(tile, u), t0 = i * N - lies;
            if (i >= n_vecs) break;
            uint4 v = process(got[u], t0);
            if (n_sparse > 0) v = patch(v, got[u], t0);
            got[u] = v;
            if (left > 0 && left != LLONG_MAX) equal += equal_in<DT>(v, value);
        }
        int mine = INT_MAX;                                 // what of them is left for the warp's vectors
        if (left > 0 && left != LLONG_MAX) {
            equal = __reduce_add_sync(0xffffffffu, equal);
            turn ^= 1;
            if (lane == 0) s.equal[turn][warp] = static_cast<uint32_t>(equal);
            __syncthreads();
            int before = 0, sum = 0;
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) {
                if (w == warp) before = sum;
                sum += static_cast<int>(s.equal[turn][w]);
            }
            mine = left <= before ? 0 : left - before < equal ? static_cast<int>(left - before) : INT_MAX;
            left = left > sum ? left - sum : 0;
        } else if (left == 0) {
            mine = 0;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = vec_of(tile, u), t0 = i * N - lies;
            uint4 v = got[u];
            if (cut) {
                if (mine > 0 && mine != INT_MAX) {          // the one warp that the last of them is in
                    const int n = i < n_vecs ? equal_in<DT>(v, value) : 0;
                    int sum = n;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int o = __shfl_up_sync(0xffffffffu, sum, d);
                        if (lane >= d) sum += o;
                    }
                    v = cut_some<DT>(v, value, mine - (sum - n), N);
                    mine -= __shfl_sync(0xffffffffu, sum, 31);
                    mine = mine > 0 ? mine : 0;
                } else {
                    v = cut_vec<DT>(v, value, mine == 0);
                }
            }
            if (i < n_vecs) store_ids<DT>(out, t0, a.V, t0 >= 0 && t0 + N <= a.V && alike, v);
        }
    }
    if (res.kind != kCutByBits) return;
    __syncthreads();                                        // (what the block stored is seen by all of it)
    const Cut by_bits = find_cut<DT>(out, a.V, 0, a.V, c, [&](CountAndWeight v) { return block_total(v, s.cut.scratch); },
                                     [&](uint32_t k) { return block_largest(k, s.cut.scratch); });
    if (!by_bits.any) return;
    for (int i = tid; i < a.V; i += kRowThreads) {
        const uint32_t k = key_of<DT>(out[i]);
        if (k < by_bits.key || (k == by_bits.key && i >= by_bits.until)) out[i] = 0xff80u;
    }
}

}  // namespace fsd
