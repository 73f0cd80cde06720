// Logit processing: penalties for used tokens, biases, a grammar's mask and a temperature, a row at a time.
// The mathematics stands in include/fsd_verify.h; each operation below is one of its, rounded by itself, so that the plain
// form of the same operations has the same bits.
#pragma once

#include <climits>

#include "fsd_device.cuh"

namespace fsd {

constexpr int kProcThreads = 256;

struct ProcArgs {
    const void* in[2];         // target and draft logits
    void* out[2];
    int rows[2];               // rows a sequence has of each: P + 1, and P or 0
    const int32_t* tokens;     // [B, P] drafted tokens, NULL: they do not count as used
    const int32_t* parent;     // [B, P] of a tree, NULL: a chain
    int B, P, V, W;
    bool penalties;            // any of the next three
    const float *repetition, *frequency, *presence;
    const int32_t* counts;
    const uint32_t* seen;
    const int32_t *bias_offsets, *bias_tokens;
    const float* bias_values;
    const uint32_t* allowed;
    const float* temperature;
    const int32_t* top_k;
    const float *top_p, *min_p;
};

// What the steps need to know of a sequence.
struct SeqParams {
    float rep, inv_rep, freq, pres, inv_temp;
};
__device__ __forceinline__ SeqParams seq_params(const ProcArgs& a, int b) {
    SeqParams p = {1.f, 1.f, 0.f, 0.f, 1.f};
    if (a.repetition != nullptr) { p.rep = __ldg(a.repetition + b); p.inv_rep = __frcp_rn(p.rep); }
    if (a.frequency != nullptr) p.freq = __ldg(a.frequency + b);
    if (a.presence != nullptr) p.pres = __ldg(a.presence + b);
    if (a.temperature != nullptr) {
        const float t = __ldg(a.temperature + b);
        if (t > 0.f) p.inv_temp = __frcp_rn(t);
    }
    return p;
}

__device__ __forceinline__ float penalised(float x, float n, const SeqParams& p) {
    x = x > 0.f ? __fmul_rn(x, p.inv_rep) : __fmul_rn(x, p.rep);
    x = __fsub_rn(x, __fmul_rn(p.freq, n));
    return n > 0.f ? __fsub_rn(x, p.pres) : x;
}

// The node that stands before node j of the drafted context (a chain's nodes stand in a row).  Always below j, so that a walk ends.
__device__ __forceinline__ int node_before(const ProcArgs& a, int b, int j) {
    if (a.parent == nullptr) return j - 1;
    const int p = __ldg(a.parent + static_cast<size_t>(b) * a.P + j);
    return p >= -1 && p < j ? p : -1;
}
// The target row that has the context of row r of a side: its mask is this row's, and the last node before it is the row's number less one.
__device__ __forceinline__ int context_row(const ProcArgs& a, int b, int side, int r) {
    return side == 0 ? r : node_before(a, b, r) + 1;
}
// How often token t is among the nodes drafted before a context row.
__device__ __forceinline__ int drafted(const ProcArgs& a, int b, int ctx, int t) {
    int n = 0;
    if (a.tokens != nullptr)
        for (int j = ctx - 1; j >= 0; j = node_before(a, b, j)) n += __ldg(a.tokens + static_cast<size_t>(b) * a.P + j) == t;
    return n;
}

// Bits t0 .. t0 + 7 of a row of words; those outside [0, 8 * bytes) are 0.
__device__ __forceinline__ uint32_t bits8(const void* words, int t0, int bytes) {
    const uint8_t* p = static_cast<const uint8_t*>(words);
    const int k = t0 >> 3, s = t0 & 7;
    uint32_t w = k >= 0 && k < bytes ? p[k] : 0u;
    if (s != 0) {
        if (k + 1 >= 0 && k + 1 < bytes) w |= static_cast<uint32_t>(p[k + 1]) << 8;
        w >>= s;
    }
    return w & 0xffu;
}

// Vocabulary ids that need more than the sequence's counts in a block's span: a bitmap of the ids with a bias or among the
// drafted tokens, and for each id the last entry of the list of biases that names it (counted from 1; 0: none).
template <int SPAN> struct Special {
    uint32_t bits[(SPAN + 31) / 32 + 1];
    int bias[SPAN];
    int any;
};
// All of the block's threads.  lo: the span's first id, a multiple of 32 (it may be negative).  Ends with a barrier.
template <int SPAN>
__device__ void find_special(const ProcArgs& a, int b, int lo, Special<SPAN>& s) {
    const int b0 = a.bias_offsets != nullptr ? __ldg(a.bias_offsets + b) : 0, b1 = a.bias_offsets != nullptr ? __ldg(a.bias_offsets + b + 1) : 0;
    const int drafts = a.penalties && a.tokens != nullptr ? a.P : 0;
    if (threadIdx.x == 0) s.any = 0;
    for (int i = threadIdx.x; i < (SPAN + 31) / 32 + 1; i += blockDim.x) s.bits[i] = 0u;
    if (a.bias_offsets != nullptr)
        for (int i = threadIdx.x; i < SPAN; i += blockDim.x) s.bias[i] = 0;
    __syncthreads();
    for (int i = b0 + static_cast<int>(threadIdx.x); i < b1; i += blockDim.x) {
        const int t = __ldg(a.bias_tokens + i), k = t - lo;
        if (t >= 0 && t < a.V && k >= 0 && k < SPAN) {
            atomicMax(&s.bias[k], i - b0 + 1);
            atomicOr(&s.bits[k >> 5], 1u << (k & 31));
            s.any = 1;
        }
    }
    for (int j = threadIdx.x; j < drafts; j += blockDim.x) {
        const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j), k = t - lo;
        if (t >= 0 && t < a.V && k >= 0 && k < SPAN) {
            atomicOr(&s.bits[k >> 5], 1u << (k & 31));
            s.any = 1;
        }
    }
    __syncthreads();
}

// The vector of logits that covers ids t0 .. t0 + N - 1 of a row; ids outside [0, V) are -inf.
template <int DT>
__device__ __forceinline__ uint4 load_ids(const void* row, int t0, int V, bool whole) {
    constexpr int N = Logit<DT>::kPerVec;
    if (whole) return *reinterpret_cast<const uint4*>(static_cast<const typename Logit<DT>::elem*>(row) + t0);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = DT == FSD_BF16 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (t0 + e >= 0 && t0 + e < V) {
            if constexpr (DT == FSD_BF16) w[e / 2] = __byte_perm(w[e / 2], static_cast<const uint16_t*>(row)[t0 + e], (e & 1) ? 0x5410u : 0x3254u);
            else w[e] = static_cast<const uint32_t*>(row)[t0 + e];
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Which of a vector's ids there are.
template <int N>
__device__ __forceinline__ uint32_t ids_of(int t0, int V) {
    uint32_t m = (1u << N) - 1u;
    if (t0 < 0) m &= m << -t0;
    if (t0 + N > V) m &= (1u << (V - t0)) - 1u;
    return m;
}

// Two values rounded to bf16 (nearest, ties to even), the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
template <int DT>
__device__ __forceinline__ uint4 pack_vec(const float (&x)[Logit<DT>::kPerVec]) {
    if constexpr (DT == FSD_BF16)
        return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    else
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <int DT>
__device__ __forceinline__ void store_ids(void* row, int t0, int V, bool whole, const uint4& v) {
    if (whole) {
        *reinterpret_cast<uint4*>(static_cast<typename Logit<DT>::elem*>(row) + t0) = v;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < Logit<DT>::kPerVec; ++e)
            if (t0 + e >= 0 && t0 + e < V) {
                if constexpr (DT == FSD_BF16) static_cast<uint16_t*>(row)[t0 + e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                else static_cast<uint32_t*>(row)[t0 + e] = w[e];
            }
    }
}

// One id of a packed vector, widened, and put back.
template <int DT>
__device__ __forceinline__ float id_of(const uint4& v, int e) {
    if constexpr (DT == FSD_BF16) {
        const uint32_t w = e < 4 ? (e < 2 ? v.x : v.y) : (e < 6 ? v.z : v.w);
        return (e & 1) ? bf16_hi(w) : bf16_lo(w);
    } else {
        return __uint_as_float(e < 2 ? (e < 1 ? v.x : v.y) : (e < 3 ? v.z : v.w));
    }
}
template <int DT>
__device__ __forceinline__ void set_id(uint4& v, int e, float x) {
    if constexpr (DT == FSD_BF16) {
        const uint32_t h = pack_bf16(x, 0.f), sel = (e & 1) ? 0x5410u : 0x3254u;        // h's low half over the word's upper or lower one
        const int w = e >> 1;
        v.x = w == 0 ? __byte_perm(v.x, h, sel) : v.x;
        v.y = w == 1 ? __byte_perm(v.y, h, sel) : v.y;
        v.z = w == 2 ? __byte_perm(v.z, h, sel) : v.z;
        v.w = w == 3 ? __byte_perm(v.w, h, sel) : v.w;
    } else {
        const uint32_t u = __float_as_uint(x);
        v.x = e == 0 ? u : v.x;
        v.y = e == 1 ? u : v.y;
        v.z = e == 2 ? u : v.z;
        v.w = e == 3 ? u : v.w;
    }
}

// The steps on one vector of a row, as it was read.  used: which of its ids the sequence has behind it, special: which of them
// may be drafted or have a bias; may: the row's mask.  count_of: how often an id that is used was generated; bias_of: the entry of the
// list of biases that names an id, counted from 1 (0: none).  The mask and the temperature go over the whole vector, the
// rest over the ids that have it, one after another: there are few, and a step that goes over all eight because one of the
// warp's ids has it made 115 instructions of 20 for each logit.
template <int DT, class CountOf, class BiasOf>
__device__ __forceinline__ uint4 process_vec(const ProcArgs& a, const SeqParams& p, int b, int ctx, int t0, uint4 v, uint32_t used, uint32_t special, uint32_t may,
                                             CountOf count_of, BiasOf bias_of) {
    constexpr int N = Logit<DT>::kPerVec;
    constexpr uint32_t kAll = (1u << N) - 1u;
    const uint4 raw = v;
    if (p.inv_temp != 1.f || (may & kAll) != kAll) {
        float x[N];
        unpack_vec<DT>(v, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __fmul_rn(x[e], p.inv_temp);
        if ((may & kAll) != kAll) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = (may >> e & 1u) ? x[e] : -INFINITY;
        }
        v = pack_vec<DT>(x);
    }
    for (uint32_t todo = (used | special) & may; todo != 0u; todo &= todo - 1u) {
        const int e = __ffs(static_cast<int>(todo)) - 1, t = t0 + e;
        int n = (used >> e & 1u) ? count_of(t) : 0;
        const int d = (special >> e & 1u) && a.penalties ? drafted(a, b, ctx, t) : 0;
        float x = id_of<DT>(raw, e);
        if ((used >> e & 1u) || d > 0) x = penalised(x, static_cast<float>(n + d), p);
        if (special >> e & 1u) {
            const int k = bias_of(t);
            if (k > 0) x = __fadd_rn(x, __ldg(a.bias_values + __ldg(a.bias_offsets + b) + k - 1));
        }
        set_id<DT>(v, e, __fmul_rn(x, p.inv_temp));
    }
    return v;
}

// A block takes a span of the vocabulary, a vector a thread, for some rows of one sequence: the counts are read once for all
// of them.  Vectors are aligned in memory and not in the vocabulary: where a row starts s ids behind a 16-byte boundary, vector v
// covers ids N v - s and on, and a row whose output lies differently is stored an id at a time.
template <int DT>
__global__ void __launch_bounds__(kProcThreads) fsd_process_kernel(const ProcArgs a, int spans, int groups, int group_rows) {
    constexpr int N = Logit<DT>::kPerVec, kSpan = kProcThreads * N + 32;
    using elem = typename Logit<DT>::elem;
    __shared__ Special<kSpan> special;
    __shared__ int counts[kSpan];
    const int span = blockIdx.x % spans, group = blockIdx.x / spans % groups, b = blockIdx.x / spans / groups;
    const int lo = span * kProcThreads * N - 32;
    const bool history = a.penalties && a.seen != nullptr;
    if (history) {
        const int first = lo < 0 ? 0 : lo;
        for (int t = first + static_cast<int>(threadIdx.x) * 8; t < lo + kSpan && t < a.V; t += kProcThreads * 8)
            for (uint32_t todo = bits8(a.seen + static_cast<size_t>(b) * a.W, t, 4 * a.W); todo != 0u; todo &= todo - 1u) {
                const int u = t + __ffs(static_cast<int>(todo)) - 1;
                if (u < a.V && u < lo + kSpan) counts[u - lo] = __ldg(a.counts + static_cast<size_t>(b) * a.V + u);
            }
    }
    find_special<kSpan>(a, b, lo, special);
    const SeqParams p = seq_params(a, b);
    const int all = a.rows[0] + a.rows[1], first = group * group_rows, last = first + group_rows < all ? first + group_rows : all;

    struct Row {                                            // a row's vector on the way
        uint4 v;
        uint32_t may;
        int t0, ctx;
        elem* out;
        bool whole, alike;
    };
    const auto fetch = [&](int q) {
        Row f;
        const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
        const size_t at = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
        const elem* in = static_cast<const elem*>(a.in[side]) + at;
        f.out = static_cast<elem*>(a.out[side]) + at;
        const int s = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16 / sizeof(elem));
        f.alike = (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(f.out)) % 16 == 0;
        f.t0 = (span * kProcThreads + static_cast<int>(threadIdx.x)) * N - s;
        f.whole = f.t0 >= 0 && f.t0 + N <= a.V;
        f.ctx = context_row(a, b, side, r);
        f.may = 0xffu;
        f.v = make_uint4(0u, 0u, 0u, 0u);
        if (f.t0 < a.V) {
            f.v = load_ids<DT>(in, f.t0, a.V, f.whole);
            if (!f.whole) f.may = ids_of<N>(f.t0, a.V);
            if (a.allowed != nullptr) f.may &= bits8(a.allowed + (static_cast<size_t>(b) * (a.P + 1) + f.ctx) * a.W, f.t0, 4 * a.W);
        }
        return f;
    };
    uint32_t used = 0u;
    int used_at = INT_MIN;                                  // the id that `used` starts at
    Row next = fetch(first);
    for (int q = first; q < last; ++q) {
        const Row f = next;
        if (q + 1 < last) next = fetch(q + 1);
        if (f.t0 >= a.V) continue;
        if (history && f.t0 != used_at) { used = bits8(a.seen + static_cast<size_t>(b) * a.W, f.t0, 4 * a.W) & ((1u << N) - 1u); used_at = f.t0; }
        const uint32_t sp = special.any ? bits8(special.bits, f.t0 - lo, sizeof(special.bits)) & ((1u << N) - 1u) : 0u;
        const uint4 y = process_vec<DT>(a, p, b, f.ctx, f.t0, f.v, used, sp, f.may, [&](int t) { return counts[t - lo]; },
                                        [&](int t) { return a.bias_offsets != nullptr ? special.bias[t - lo] : 0; });
        store_ids<DT>(f.out, f.t0, a.V, f.whole && f.alike, y);
    }
}

}  // namespace fsd
