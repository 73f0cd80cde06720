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
__device__ __forceinline__ SeqParams seq_params(const uint32_t* settings) {      // repetition, frequency, presence, temperature
    SeqParams p;
    p.rep = __uint_as_float(settings[0]);
    p.inv_rep = __frcp_rn(p.rep);
    p.freq = __uint_as_float(settings[1]);
    p.pres = __uint_as_float(settings[2]);
    const float t = __uint_as_float(settings[3]);
    p.inv_temp = t > 0.f ? __frcp_rn(t) : 1.f;
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

// The ids of a block's span that need more than the mask and the temperature: used ones, drafted ones and those with a
// bias.  A bitmap of them and a list in no order, how often each was generated, and for each the last entry of the list of
// biases that names it (counted from 1; 0: none).
template <int SPAN> struct Sparse {
    uint32_t drafted[(SPAN + 31) / 32 + 1];                // drafted or biased: to be looked at again in each row
    uint32_t bits[(SPAN + 31) / 32 + 1];
    int bias[SPAN];
    uint16_t list[SPAN];
    int counts[SPAN];                                      // by place in the list; 0 for what is only in the prompt, -1: not used
    int n;
};
// All of the block's threads.  lo: the span's first id, a multiple of 32 (it may be negative).  Ends with a barrier.
// Each block reads all of the sequence's list of biases, which is for lists of a few thousand: 64 x 17 x 152064 takes 124 us with 16 a sequence, 142 with
// 300, 176 with 3000 and 1099 with one for every token; 1 x 152064 6.9, 6.8, 8.8 and 59.
template <int SPAN>
__device__ __forceinline__ void find_sparse(const ProcArgs& a, int b, int lo, Sparse<SPAN>& s) {
    static_assert(SPAN % 32 == 0, "whole words");
    const int b0 = a.bias_offsets != nullptr ? __ldg(a.bias_offsets + b) : 0, b1 = a.bias_offsets != nullptr ? __ldg(a.bias_offsets + b + 1) : 0;
    const int drafts = a.penalties && a.tokens != nullptr ? a.P : 0;
    const bool history = a.penalties && a.seen != nullptr;
    if (threadIdx.x == 0) s.n = 0;
    for (int i = threadIdx.x; i < SPAN / 32 + 1; i += blockDim.x) { s.drafted[i] = 0u; s.bits[i] = 0u; }
    if (a.bias_offsets != nullptr)
        for (int i = threadIdx.x; i < SPAN; i += blockDim.x) s.bias[i] = 0;
    __syncthreads();
    const int biases = b1 > b0 ? b1 - b0 : 0;
    for (int left = biases - static_cast<int>(threadIdx.x); left > 0; left -= static_cast<int>(blockDim.x)) {      // (counted down: an offset may be 2^31 - 1)
        const int t = __ldg(a.bias_tokens + b0 + (biases - left)), k = t - lo;
        if (t >= 0 && t < a.V && k >= 0 && k < SPAN) {
            atomicMax(&s.bias[k], biases - left + 1);
            atomicOr(&s.drafted[k >> 5], 1u << (k & 31));
        }
    }
    for (int j = threadIdx.x; j < drafts; j += blockDim.x) {
        const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j), k = t - lo;
        if (t >= 0 && t < a.V && k >= 0 && k < SPAN) atomicOr(&s.drafted[k >> 5], 1u << (k & 31));
    }
    if (drafts > 0 || b1 > b0) __syncthreads();
    // eight ids a thread
    for (int k = static_cast<int>(threadIdx.x) * 8; k < SPAN; k += static_cast<int>(blockDim.x) * 8) {
        const int t = lo + k;
        if (t < 0 || t >= a.V) continue;
        uint32_t used = history ? bits8(a.seen + static_cast<size_t>(b) * a.W, t, 4 * a.W) : 0u;
        if (t + 8 > a.V) used &= (1u << (a.V - t)) - 1u;
        const uint32_t any = used | (s.drafted[k >> 5] >> (k & 31) & 0xffu);
        if (any == 0u) continue;
        reinterpret_cast<uint8_t*>(s.bits)[k >> 3] = static_cast<uint8_t>(any);
        int at = atomicAdd(&s.n, __popc(any));
        for (uint32_t todo = any; todo != 0u; todo &= todo - 1u) {
            const int e = __ffs(static_cast<int>(todo)) - 1;
            FSD_CHECK(&process_debug, at >= 0 && at < SPAN && t + e < a.V, kChkList);
            s.counts[at] = (used >> e & 1u) ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t + e) : -1;
            s.list[at++] = static_cast<uint16_t>(k + e);
        }
    }
    __syncthreads();
}

// The vector of logits that covers ids t0 .. t0 + N - 1 of a row; ids outside [0, V) are -inf.
template <int DT>
__device__ __forceinline__ uint4 load_ids(const void* row, int t0, int V, bool whole) {
    constexpr int N = Logit<DT>::kPerVec;
    FSD_CHECK(&process_debug, !whole || (t0 >= 0 && t0 + N <= V && reinterpret_cast<uintptr_t>(static_cast<const typename Logit<DT>::elem*>(row) + t0) % 16 == 0), kChkVector);
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
    FSD_CHECK(&process_debug, !whole || (t0 >= 0 && t0 + Logit<DT>::kPerVec <= V && reinterpret_cast<uintptr_t>(static_cast<typename Logit<DT>::elem*>(row) + t0) % 16 == 0), kChkVector);
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

// One id of a row, widened, and put back.
template <int DT>
__device__ __forceinline__ float read_id(const void* row, int t) {
    if constexpr (DT == FSD_BF16) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[t]) << 16);
    else return static_cast<const float*>(row)[t];
}
template <int DT>
__device__ __forceinline__ void write_id(void* row, int t, float x) {
    if constexpr (DT == FSD_BF16) static_cast<uint16_t*>(row)[t] = static_cast<uint16_t>(pack_bf16(x, 0.f));
    else static_cast<float*>(row)[t] = x;
}

// The mask and the temperature on one vector of a row.
template <int DT>
__device__ __forceinline__ uint4 process_vec(uint4 v, uint32_t may, float inv_temp) {
    constexpr int N = Logit<DT>::kPerVec;
    constexpr uint32_t kAll = (1u << N) - 1u;
    if (inv_temp == 1.f && (may & kAll) == kAll) return v;
    float x[N];
    unpack_vec<DT>(v, x);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = __fmul_rn(x[e], inv_temp);
    if ((may & kAll) != kAll) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (may >> e & 1u) ? x[e] : -INFINITY;
    }
    return pack_vec<DT>(x);
}
// All steps but the mask on one logit.  n: how often its token was generated, -1: it is not behind the sequence; d: how often it is drafted.
__device__ __forceinline__ float process_id(float x, int n, int d, float bias, bool biased, const SeqParams& p) {
    if (n >= 0 || d > 0) x = penalised(x, static_cast<float>((n > 0 ? n : 0) + d), p);
    if (biased) x = __fadd_rn(x, bias);
    return __fmul_rn(x, p.inv_temp);
}

// Bits as masks of a vector's halves or words.
template <int DT>
__device__ __forceinline__ uint4 spread_bits(uint32_t bits) {
    if constexpr (DT == FSD_BF16) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (bits >> (2 * k) & 1u) * 0xffffu | (bits >> (2 * k + 1) & 1u) * 0xffff0000u;
        return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        return make_uint4((bits & 1u) * 0xffffffffu, (bits >> 1 & 1u) * 0xffffffffu, (bits >> 2 & 1u) * 0xffffffffu, (bits >> 3 & 1u) * 0xffffffffu);
    }
}
__device__ __forceinline__ uint4 merge(const uint4& a, const uint4& b, const uint4& of_b) {
    return make_uint4((a.x & ~of_b.x) | (b.x & of_b.x), (a.y & ~of_b.y) | (b.y & of_b.y), (a.z & ~of_b.z) | (b.z & of_b.z), (a.w & ~of_b.w) | (b.w & of_b.w));
}

// A block takes a span of the vocabulary, a vector a thread, for some rows of one sequence, so that counts and biases are looked up once
// for all of them.  First the mask and the temperature, a vector at a time, which leave the sparse ids as they were read; then these, one
// id a thread: few of a vector's ids are sparse, but of a warp's 256 some always are, and a loop over a vector's own took 50
// instructions a logit.  Without sparse ids the kernel is bound by memory (64 x 17 x 152064 bf16: 115 us, 90% of the rate of a copy);
// with them by their stores of two bytes each, which the L2 cache takes one by one (250 us with some 11000 used ids a sequence).
// In a tile of four rows in shared memory instead these took 247 us, but 16 x 11 x 32000 26 where it is 19.
// Vectors are aligned in memory and not in the vocabulary: where a row starts s ids behind a 16-byte boundary, vector v
// covers ids N v - s and on, and a row whose output lies differently is stored an id at a time.
// REGULAR: every row's input and output starts on such a boundary and is a whole number of vectors, so that none of this has to be looked
// after (32 x 13 x 128256 with masks 79 -> 71 us).
template <int DT, bool REGULAR>
__global__ void __launch_bounds__(kProcThreads) fsd_process_kernel(const ProcArgs a, int spans, int groups, int group_rows) {
    constexpr int N = Logit<DT>::kPerVec, kIds = kProcThreads * N, kSpan = kIds + 32;
    using elem = typename Logit<DT>::elem;
    __shared__ Sparse<kSpan> sparse;
    const int span = blockIdx.x % spans, group = blockIdx.x / spans % groups, b = blockIdx.x / spans / groups;
    const int lo = span * kIds - 32;
    const bool some = a.penalties || a.bias_offsets != nullptr;
    if (some) find_sparse<kSpan>(a, b, lo, sparse);
    const int n_sparse = some ? sparse.n : 0;
    const uint32_t settings[4] = {__float_as_uint(a.repetition != nullptr ? __ldg(a.repetition + b) : 1.f), __float_as_uint(a.frequency != nullptr ? __ldg(a.frequency + b) : 0.f),
                                  __float_as_uint(a.presence != nullptr ? __ldg(a.presence + b) : 0.f), __float_as_uint(a.temperature != nullptr ? __ldg(a.temperature + b) : 0.f)};
    const SeqParams p = seq_params(settings);
    FSD_CHECK(&process_debug, b < a.B && n_sparse <= kSpan, kChkItem);
    const int all = a.rows[0] + a.rows[1], first = group * group_rows, last = first + group_rows < all ? first + group_rows : all;

    const uint32_t* allowed = a.allowed != nullptr ? a.allowed + static_cast<size_t>(b) * (a.P + 1) * a.W : nullptr;
    uint4 keep = make_uint4(0u, 0u, 0u, 0u);
    int keep_at = INT_MIN;                                  // the id that `keep` starts at
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const int r0 = side == 0 ? first : (first > a.rows[0] ? first - a.rows[0] : 0);
        const int r1 = side == 0 ? (last < a.rows[0] ? last : a.rows[0]) : last - a.rows[0];
        if (r0 >= r1) continue;
        const size_t at = (static_cast<size_t>(b) * a.rows[side] + r0) * a.V;
        const elem* in = static_cast<const elem*>(a.in[side]) + at;
        elem* out = static_cast<elem*>(a.out[side]) + at;
        const bool alike = REGULAR || (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) % 16 == 0;
        const int base = (span * kProcThreads + static_cast<int>(threadIdx.x)) * N;
        struct Row {                                        // a row's vector on the way
            uint4 v;
            uint32_t may;
        };
        const auto first_id = [&](const elem* row) { return REGULAR ? base : base - static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(elem)); };
        const auto fetch = [&](const elem* row, int r) {
            Row f = {make_uint4(0u, 0u, 0u, 0u), 0xffu};
            const int t0 = first_id(row);
            if (t0 < a.V) {
                if (allowed != nullptr) f.may = bits8(allowed + static_cast<size_t>(context_row(a, b, side, r)) * a.W, t0, 4 * a.W);
                f.v = load_ids<DT>(row, t0, a.V, REGULAR || (t0 >= 0 && t0 + N <= a.V));
            }
            return f;
        };
        Row next = fetch(in, r0);
#pragma unroll 2
        for (int r = r0; r < r1; ++r) {
            const Row f = next;
            const int t0 = first_id(in);
            in += a.V;
            if (r + 1 < r1) next = fetch(in, r + 1);
            if (t0 < a.V) {
                uint4 y = process_vec<DT>(f.v, f.may, p.inv_temp);
                if (n_sparse > 0) {
                    if (t0 != keep_at) { keep = spread_bits<DT>(bits8(sparse.bits, t0 - lo, sizeof(sparse.bits))); keep_at = t0; }
                    y = merge(y, f.v, keep);
                }
                store_ids<DT>(out, t0, a.V, REGULAR || (t0 >= 0 && t0 + N <= a.V && alike), y);
            }
            out += a.V;
        }
    }
    if (n_sparse == 0) return;
    __syncthreads();                                        // (what the block's threads stored is seen by all of them)
    // `wide` threads a row, each with the same id in all rows it does
    int wide = 32;
    while (wide < kProcThreads && wide < n_sparse) wide <<= 1;
    const int stride = kProcThreads / wide;
    for (int k = static_cast<int>(threadIdx.x) % wide; k < n_sparse; k += wide) {
        const int at = sparse.list[k], t = lo + at, count = sparse.counts[k];
        FSD_CHECK(&process_debug, at < kSpan && t >= 0 && t < a.V, kChkToken);
        const bool again = sparse.drafted[at >> 5] >> (at & 31) & 1u;
        const int entry = again && a.bias_offsets != nullptr ? sparse.bias[at] : 0;
        const float bias = entry > 0 ? __ldg(a.bias_values + __ldg(a.bias_offsets + b) + entry - 1) : 0.f;
#pragma unroll 4
        for (int q = first + static_cast<int>(threadIdx.x) / wide; q < last; q += stride) {
            const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
            const size_t line = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
            const int s = REGULAR ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(static_cast<const elem*>(a.in[side]) + line) % 16 / sizeof(elem));
            if (static_cast<unsigned>(t + s - span * kIds) >= static_cast<unsigned>(kIds)) continue;      // (another block's, in this row)
            elem* row = static_cast<elem*>(a.out[side]) + line;
            int ctx = 0, d = 0;
            if (again || allowed != nullptr) ctx = context_row(a, b, side, r);
            if (again && a.penalties) d = drafted(a, b, ctx, t);
            const bool may = allowed == nullptr || (__ldg(allowed + static_cast<size_t>(ctx) * a.W + (t >> 5)) >> (t & 31) & 1u);
            // (as it was read: where the row is done in place the vectors left these as they were)
            const float y = process_id(read_id<DT>(static_cast<const elem*>(a.in[side]) + line, t), count, d, bias, entry > 0, p);
            write_id<DT>(row, t, may ? y : -INFINITY);
        }
    }
}

}  // namespace fsd
