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

// exp(x) for x of at most 700, to 2^-52 of itself (0.61 of that at most over 750000 values): x = n ln 2 + r with |r| <= ln 2 / 2, and e^r by its
// Taylor series up to r^13 / 13! (the next term is below 5e-18).  Sums that say where a border lies need that much of each of
// their terms.  Below -700 it is 0.
__device__ __forceinline__ double exp_of(double x) {
    if (!(x >= -700.0)) return 0.0;
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
#pragma unroll 8
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
#pragma unroll 8
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
#pragma unroll 8
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

// ---- cuts by the counts of bins -----------------------------------------------------
// Values are counted by the upper 16 bits of their single-precision form.  For bf16 a bin is one value, so that the counts alone say
// where every cut is and what everything weighs, with one exponential for a bin, from a table, instead of one for a token; for
// fp32 they say which bins to look into.  The bins are those of magnitudes from 2^-23 up to 2^8, one for what is smaller
// (zeros; anything else there has the weight of 0 but for 2^-23), one for what is below, as long as it is one value (a mask's
// lowest number), and one for what is above.  Where a cut falls on a bin of several values, where it would be another one with the smaller
// values' weights each off by 2^-23, or where something is above, the row is cut a bit at a time.
constexpr int kRowThreads = 512;
constexpr int kRowWarps = kRowThreads / 32;
constexpr uint32_t kMagLo = 0x33ff, kMagHi = 0x4380;       // upper halves: just below 2^-23, and 2^8
constexpr int kHalfBins = static_cast<int>(kMagHi - kMagLo) + 1;
constexpr int kBins = 2 * kHalfBins;                       // negative magnitudes falling, then positive ones rising
constexpr int kBinUnder = 0, kBinOver = kBins - 1, kBinMid = kHalfBins, kBinNone = kHalfBins - 1;
constexpr int kBinsEach = ((kBins + kRowThreads - 1) / kRowThreads + 3) / 4 * 4;
static_assert(kBins % 4 == 0, "whole vectors of bins");

// exp of every bin's value by place, from the highest bin down, 0 for the first and the last.  The host fills it in front of a
// device's first call; worked out where it is needed it took a block 2000 cycles a row.
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
    w[kBins - 1 - kBinMid] = 1.0;
}

enum CutKind { kCutNone, kCutDone, kCutByBits, kCutRefineK, kCutRefineP };
struct CutResult {
    int kind;
    uint32_t key;              // of the cut; while it is being refined, its upper bits
    long long ties;
    uint32_t over;             // refining top-k: whether all that are equal to the k-th are kept
};
struct Run {
    uint32_t n;
    double w;
};
struct BinsShared {
    uint32_t mixed;            // how many of the middle bin's are no zeros
    uint32_t under_lo, under_hi;       // keys of the lowest bin's values
    CountAndWeight scratch[32];
    uint32_t warp_n[kRowWarps];
    double warp_w[kRowWarps];
    uint32_t min_key;
    uint32_t settings[8];
    CutResult work;
    int found[4], group[3];
    Run before[3];
    uint32_t place_n;
    double goal, above_goal;
};
__device__ __forceinline__ void clear_bins(uint32_t* hist, BinsShared& s) {
    for (int i = threadIdx.x; i < kBins / 4; i += kRowThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (threadIdx.x == 0) { s.mixed = 0u; s.under_lo = 0xffffffffu; s.under_hi = 0u; }
}
__device__ __forceinline__ bool one_value(const BinsShared& s, int bin) {
    return bin == kBinMid ? s.mixed == 0u : bin == kBinUnder ? s.under_lo >= s.under_hi : bin != kBinOver;
}
// The upper 16 bits of the keys of a one-value bin.
template <int DT>
__device__ __forceinline__ uint32_t bin_prefix(const BinsShared& s, int bin) {
    if (bin == kBinMid) return 0x8000u;
    if (bin == kBinUnder) return DT == FSD_BF16 ? s.under_lo : s.under_lo >> 16;
    return bin > kHalfBins ? 0x8000u | (kMagLo + static_cast<uint32_t>(bin - kHalfBins)) : 0x7fffu ^ (kMagLo + static_cast<uint32_t>(kHalfBins - 1 - bin));
}

// One value into the bins, or (BY -1) out of them.
template <int DT, int BY>
__device__ __noinline__ void count_value(uint32_t bits, uint32_t* hist, BinsShared* s) {
    if (bits == 0xff800000u) return;
    const uint32_t mag = bits >> 16 & 0x7fffu, u = (mag < kMagLo ? kMagLo : mag > kMagHi ? kMagHi : mag) - kMagLo;
    int bin = static_cast<int>(u ^ static_cast<uint32_t>(static_cast<int>(bits) >> 31)) + kHalfBins;
    if (u == 0u) {
        bin = kBinMid;
        if (BY > 0 && (bits & 0x7fffffffu) != 0u) atomicAdd(&s->mixed, 1u);
    }
    if ((bits & 0x7fffffffu) > 0x7f800000u) bin = kBinOver;
    if (BY > 0 && bin == kBinUnder) {
        const uint32_t key = key_of<DT>(DT == FSD_BF16 ? bits >> 16 : bits);
        if (key < *reinterpret_cast<volatile uint32_t*>(&s->under_lo)) atomicMin(&s->under_lo, key);
        if (key > *reinterpret_cast<volatile uint32_t*>(&s->under_hi)) atomicMax(&s->under_hi, key);
    }
    FSD_CHECK(&process_debug, bin >= 0 && bin < kBins, kChkBin);
    atomicAdd(&hist[bin], static_cast<uint32_t>(BY));
}
__device__ __forceinline__ uint32_t min_halves(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("min.u16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.u16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}
// A vector of values into the bins.  bf16: two at a time, in halves of a word.
// SKIP: but not those that `skip` has all bits set for; they go to a bin of no value, kBinNone, whose count means nothing.
template <int DT, bool SKIP = false>
__device__ __forceinline__ void count_vec(const uint4& v, uint32_t* hist, BinsShared* s, const uint4& skip = make_uint4(0u, 0u, 0u, 0u)) {
    if constexpr (DT == FSD_BF16) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w}, not_these[4] = {skip.x, skip.y, skip.z, skip.w};
        uint32_t bin[4], lowest = 0xffffffffu, highest = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t m = min_halves(max_halves(w[k] & 0x7fff7fffu, kMagLo * 0x10001u), kMagHi * 0x10001u);
            if (SKIP) m = (m & ~not_these[k]) | (((kMagLo + 1u) * 0x10001u) & not_these[k]);
            lowest = min_halves(lowest, m);
            highest = max_halves(highest, m);
            uint32_t sign;                                  // each half's sign in all of its bits
            asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(sign) : "r"(w[k]));
            bin[k] = (m - kMagLo * 0x10001u) ^ sign;
            if (SKIP) bin[k] |= not_these[k];               // -1: kBinNone
        }
        if ((lowest & 0xffffu) == kMagLo || lowest >> 16 == kMagLo || (highest & 0xffffu) == kMagHi || highest >> 16 == kMagHi) {
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                uint32_t two = k < 2 ? (k < 1 ? v.x : v.y) : (k < 3 ? v.z : v.w);
                if (SKIP) {
                    const uint32_t no = k < 2 ? (k < 1 ? skip.x : skip.y) : (k < 3 ? skip.z : skip.w);
                    two = (two & ~no) | (0xff80ff80u & no);
                }
                if (two == 0xff80ff80u) continue;
                count_value<DT, 1>(two << 16, hist, s);
                count_value<DT, 1>(two & 0xffff0000u, hist, s);
            }
        } else {
            uint32_t* mid = hist + kHalfBins;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                FSD_CHECK(&process_debug, static_cast<int16_t>(bin[k]) >= -kHalfBins && static_cast<int16_t>(bin[k]) < kHalfBins && (static_cast<int>(bin[k]) >> 16) >= -kHalfBins &&
                                              (static_cast<int>(bin[k]) >> 16) < kHalfBins, kChkBin);
                atomicAdd(mid + static_cast<int16_t>(bin[k]), 1u);
                atomicAdd(mid + (static_cast<int>(bin[k]) >> 16), 1u);
            }
        }
    } else {
        const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t mag = bits[e] >> 16 & 0x7fffu;
            if (mag <= kMagLo || mag >= kMagHi) count_value<DT, 1>(bits[e], hist, s);
            else {
                const int bin = static_cast<int>((mag - kMagLo) ^ static_cast<uint32_t>(static_cast<int>(bits[e]) >> 31)) + kHalfBins;
                FSD_CHECK(&process_debug, bin >= 0 && bin < kBins, kChkBin);
                atomicAdd(&hist[bin], 1u);
            }
        }
    }
}

// Exclusive sums over the threads of the block, in thread order.  All threads; ends with a barrier.
__device__ __forceinline__ Run scan_threads(Run v, BinsShared& s, Run& all) {
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

// What takes the weight of a bin's edge next to zero to that of its middle, fp32's: e^(half its width), or one over that.
template <int DT>
__device__ __forceinline__ double to_middle(int bin) {
    if constexpr (DT == FSD_BF16) return 1.0;
    const int u = bin >= kHalfBins ? bin - kHalfBins : kHalfBins - 1 - bin;
    const float half = __uint_as_float((kMagLo + static_cast<uint32_t>(u)) << 16 & 0x7f800000u) * (1.f / 256.f);
    return bin == kBinMid ? 1.0 : static_cast<double>(ex2(bin >= kHalfBins ? half * kLog2e : -half * kLog2e));
}

// The bin in a thread's group of places at which a running sum gets to a goal, found by a warp, a place a lane.  `count`: the
// sum is the number of tokens, else their weight.  Lanes without tokens are passed over; -1: it does not get there, and `above` is then what
// it gets to.
struct PlaceFound {
    int place;
    uint32_t n;                // tokens in the bin
    Run above;                 // what is above it
    double w;                  // weight of each of its tokens
};
template <int DT>
__device__ __forceinline__ PlaceFound find_place(const uint32_t* hist, int group, Run before, bool count, uint32_t n_goal, double w_goal) {
    static_assert(kBinsEach <= 32, "a lane each");
    const int lane = threadIdx.x & 31, place = group * kBinsEach + lane;
    const bool is = lane < kBinsEach && place < kBins;
    const uint32_t n = is ? hist[kBins - 1 - place] : 0u;
    const double w = n != 0u ? __ldg(bin_weights + place) * to_middle<DT>(kBins - 1 - place) : 0.0;
    Run run = {n, n * w};
#pragma unroll
    for (int d = 1; d < kBinsEach; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, run.n, d);
        const double p = __shfl_up_sync(0xffffffffu, run.w, d);
        if (lane >= d) { run.n += o; run.w += p; }
    }
    const bool there = n != 0u && (count ? before.n + run.n >= n_goal : before.w + run.w >= w_goal);
    const uint32_t ballot = __ballot_sync(0xffffffffu, there);
    if (ballot == 0u)
        return {-1, 0u, {before.n + __shfl_sync(0xffffffffu, run.n, kBinsEach - 1), before.w + __shfl_sync(0xffffffffu, run.w, kBinsEach - 1)}, 0.0};
    const int at = __ffs(static_cast<int>(ballot)) - 1;
    PlaceFound f;
    f.place = group * kBinsEach + at;
    f.n = __shfl_sync(0xffffffffu, n, at);
    f.w = __shfl_sync(0xffffffffu, w, at);
    f.above.n = before.n + __shfl_sync(0xffffffffu, run.n - n, at);
    const double up_to = __shfl_sync(0xffffffffu, run.w, at > 0 ? at - 1 : 0);
    f.above.w = at > 0 ? before.w + up_to : before.w;
    return f;
}

// From the counts to the cut (bf16) or to the bins that hold the cuts (fp32).  `place` counts bins from the highest one down, a thread
// has kBinsEach of them.  top: fp32, the largest key.  All of a block's threads; s.work has it behind the next barrier.
template <int DT>
__device__ __forceinline__ void solve_bins(const uint32_t* hist, BinsShared& s, const CutParams& c, int V, uint32_t top) {
    const int tid = threadIdx.x, warp = tid >> 5, p0 = tid * kBinsEach;
    if (tid == 0) {
        s.group[0] = s.group[1] = s.group[2] = kRowThreads;
        s.found[0] = -1;                                     // place of the k-th token
        s.found[1] = s.found[2] = kBins;                     // of the highest one, and of the border of top-p
        s.work = {kCutDone, 0u, V, 0u};
        s.min_key = 0u;
    }
    Run mine = {0u, 0.0};
#pragma unroll
    for (int j = 0; j < kBinsEach; j += 4) {
        const int bin = kBins - 4 - (p0 + j);
        if (bin < 0) break;
        const uint4 v = *reinterpret_cast<const uint4*>(hist + bin);
        if ((v.x | v.y | v.z | v.w) != 0u) {                 // (fp32: as if all of a bin were in its middle)
            const double2* w = reinterpret_cast<const double2*>(bin_weights + p0 + j);
            const double2 w0 = __ldg(w), w1 = __ldg(w + 1);
            mine.n += v.x + v.y + v.z + v.w;
            mine.w += (v.w * w0.x * to_middle<DT>(bin + 3) + v.z * w0.y * to_middle<DT>(bin + 2)) +
                      (v.y * w1.x * to_middle<DT>(bin + 1) + v.x * w1.y * to_middle<DT>(bin));
        }
    }
    Run all;
    const Run before = scan_threads(mine, s, all);
    const uint32_t k = c.k ? static_cast<uint32_t>(c.top_k) : 0xffffffffu;
    const bool cut_k = c.k && all.n > k;
    if (all.n == 0u) {                                       // nothing finite, and nothing above it either
        if (tid == 0) s.work.kind = kCutNone;
        return;
    }
    // the threads that have the highest bin, the k-th token and the border of top-p; a warp each looks for the bin
    const auto tell_goal = [&](double goal) {                // the first whose tokens and those before weigh the goal
        const uint32_t ballot = __ballot_sync(0xffffffffu, mine.n != 0u && before.w + mine.w >= goal);
        if (ballot != 0u && (tid & 31) == 0) atomicMin(&s.group[2], tid + __ffs(static_cast<int>(ballot)) - 1);
    };
    const auto tell = [&](int what) { s.group[what] = tid; s.before[what] = before; };
    if (mine.n != 0u && before.n == 0u) tell(0);
    if (cut_k && before.n < k && before.n + mine.n >= k) tell(1);
    double goal = static_cast<double>(c.top_p) * all.w;
    if (c.p && !cut_k) tell_goal(goal);
    __syncthreads();
    if (warp == 0) {
        const PlaceFound f = find_place<DT>(hist, s.group[0], s.before[0], true, 1u, 0.0);
        if (tid == 0) {
            s.found[1] = f.place;
            const int bin = kBins - 1 - f.place;
            if (DT == FSD_BF16 && c.m && one_value(s, bin)) {
                const uint32_t key = bin_prefix<DT>(s, bin);
                s.min_key = min_p_key<DT>(c.min_p, key, value_of<DT>(key));
            }
        }
    } else if (warp == 1 && cut_k) {
        const PlaceFound f = find_place<DT>(hist, s.group[1], s.before[1], true, k, 0.0);
        if ((tid & 31) == 0) {
            s.found[0] = f.place;
            s.work.ties = k - f.above.n;
            s.goal = f.above.w + static_cast<double>(k - f.above.n) * f.w;
            s.place_n = f.n;
        }
    }
    __syncthreads();
    const int k_place = s.found[0], k_bin = kBins - 1 - k_place, top_bin = kBins - 1 - s.found[1];
    // What is below the bins is worth nothing beside a highest value of at least -180 (e^-76 of it each) and is nothing but a count.
    const float most = DT == FSD_F32 ? value_of<FSD_F32>(top) : value_of<DT>(bin_prefix<DT>(s, top_bin));
    const bool off = hist[kBinOver] != 0u || !one_value(s, top_bin) || ((hist[kBinUnder] != 0u || top_bin == kBinUnder) && !(most >= -180.f)) ||
                     (cut_k && !one_value(s, k_bin));
    if (off) {
        if (tid == 0) s.work.kind = kCutByBits;
        return;
    }
    int p_place = k_place;
    uint32_t n_cut = cut_k ? s.place_n : 0u;                 // tokens in the bin of the cut
    long long ties = s.work.ties;
    bool sure = true;                                        // whether the border is there whatever the values next to zero weigh
    if (c.p) {                                               // the first place at which the tokens so far weigh the goal
        if (cut_k) {
            goal = static_cast<double>(c.top_p) * s.goal;
            tell_goal(goal);
            __syncthreads();
        }
        const int first = s.group[2];
        if (first < kRowThreads && tid / 32 == first / 32) { // (its own warp: s.before has one thread's)
            const Run from = {__shfl_sync(0xffffffffu, before.n, first & 31), __shfl_sync(0xffffffffu, before.w, first & 31)};
            PlaceFound f = find_place<DT>(hist, first, from, false, 0u, goal);
            // (A bin's sum is rounded in another order here than the thread's, so that the goal may be in a later group.)
            for (int g = first + 1; f.place < 0 && g < kRowThreads; ++g) f = find_place<DT>(hist, g, f.above, false, 0u, goal);
            if ((tid & 31) == 0) {
                if (f.place >= 0) s.found[2] = f.place;
                s.before[2] = {f.n, f.above.w};
                s.above_goal = f.w;
            }
        }
        __syncthreads();
        p_place = s.found[2];
        if (!(goal > 0.0)) p_place = s.found[1];
        if (cut_k && p_place > k_place) p_place = k_place;
        const bool at_k = cut_k && p_place == k_place;
        if (p_place == s.found[2]) {
            n_cut = s.before[2].n;
            // Where one value has all of the weight its tokens are counted, for a share may end on one of them exactly (of a thousand
            // equal ones three quarters are 750), which 750 times a rounded weight does not.
            const double equal = cut_k && at_k ? static_cast<double>(k) : static_cast<double>(n_cut);
            const bool alone = DT == FSD_BF16 && goal > 0.0 && s.before[2].w == 0.0 && (cut_k ? s.goal : all.w) == equal * s.above_goal;
            const long long t = alone ? ties_below(0.0, 1.0, static_cast<double>(c.top_p) * equal, V) : ties_below(s.before[2].w, s.above_goal, goal, V);
            const bool all_of_k = at_k && ties <= t;
            ties = all_of_k ? ties : t;
            if (DT == FSD_BF16 && s.mixed != 0u && goal > 0.0) {              // (fp32's sums are of what each token weighs)
                const double off = static_cast<double>(s.mixed) * 0x1p-23;
                sure = (s.before[2].w == 0.0 && ties == 1) || s.before[2].w + static_cast<double>(ties - 1) * s.above_goal < goal - off;
                sure = sure && (all_of_k || s.before[2].w + static_cast<double>(ties) * s.above_goal >= goal + off);
            }
        } else if (!(goal > 0.0)) {
            n_cut = hist[kBins - 1 - p_place];
            ties = 1;
        }
    }
    const int p_bin = kBins - 1 - p_place;
    FSD_CHECK(&process_debug, !(cut_k || c.p) || (p_place >= 0 && p_place <= kBins && k_place >= -1 && k_place < kBins && top_bin >= 0), kChkBin);
    if (c.p && (p_bin < 0 || !one_value(s, p_bin) || !sure)) {
        __syncthreads();
        if (tid == 0) s.work.kind = kCutByBits;
        return;
    }
    __syncthreads();                                         // (s.work.ties has been read)
    if (tid != 0) return;
    if constexpr (DT == FSD_BF16) {
        if (c.p || cut_k) {
            s.work.ties = ties >= n_cut ? V : ties;          // all of them
            s.work.key = bin_prefix<DT>(s, p_bin);
        }
        if (s.min_key > s.work.key) { s.work.key = s.min_key; s.work.ties = V; }
        if (s.work.key == 0u) s.work.kind = kCutNone;
    } else {
        s.found[3] = p_bin;
        if (cut_k) {
            s.work.kind = kCutRefineK;
            s.work.key = bin_prefix<DT>(s, k_bin);
        } else if (c.p) {
            s.work.kind = kCutRefineP;
            s.work.key = bin_prefix<DT>(s, p_bin);
        } else if (c.m) {
            s.work.key = min_p_key<DT>(c.min_p, top, most);
        } else {
            s.work.kind = kCutNone;                          // (fewer tokens than top_k)
        }
    }
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

}  // namespace fsd
