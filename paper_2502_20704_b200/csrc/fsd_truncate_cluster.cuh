// Top-k, top-p and min-p on rows of fp32 logits that fit on chip: a cluster of blocks per row.
#pragma once

#include "fsd_truncate.cuh"

namespace fsd {

// A block reads its slice of the row once, processes it, keeps it in shared memory and counts it.  The first block of the cluster gets all
// counts (additions into its shared memory, whole numbers, so that their order does not matter), finds the bin of the cut and tells
// the others; that bin is split twice more, by 8 bits and 8 for top-k, by 7 and 9 for top-p.
// 64 x 17 x 152064 takes 1.9 ms (top-p alone 2.07), 1 x 32000 18 to 31 us by the settings: a dozen steps a row that each wait for the slowest block, with two blocks an SM.
constexpr int kMaxCutCluster = 8;
constexpr int kListed = 96;
constexpr int kDraftedWords = 768;     // of a slice's bitmap of drafted ids in the space that is there for other things later; longer ones have their own
constexpr double kFixed = 18014398509481984.0;             // 2^54: weights of a bin's tokens as whole numbers

struct CutShared : BinsShared {
    double above[kMaxCutCluster], rest[kMaxCutCluster];
    uint32_t top[kMaxCutCluster];
    int equal[kMaxCutCluster];
    CountAndWeight slots[2][kMaxCutCluster];
    CutResult told[2];         // what the first block told last, and the time before
    union {
        struct {                                           // in front of everything else
            uint16_t list[kRowWarps][kListed];             // sparse ids
            uint32_t drafted[kDraftedWords];
        };
        struct {
            uint32_t sub_n[512];                           // of a bin's parts: tokens
            uint32_t digits[4 * 128];                      // and, of 128 parts, their weights' digits
            uint64_t sub_w[2 * 128];                       // the first block's: weights, of all blocks, their lower 32 bits and the rest
        };
    };
};

struct RowSlice {
    uint4* vecs;
    int n;                     // vectors
    int first;                 // id of the first one's first token
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() { cluster_arrive(); cluster_wait(); }

// Counts, by the BITS bits above `shift`, the tokens whose keys have the upper bits `prefix` and are above `over`.  All into the first
// block's shared memory.
template <int BITS>
__device__ void count_bits(const RowSlice& row, CutShared& s, CutShared& first, int rank, uint32_t prefix, int shift, uint32_t over) {
    const int tid = threadIdx.x;
    if (rank != 0) {
        for (int i = tid; i < 1 << BITS; i += kRowThreads) s.sub_n[i] = 0u;
        __syncthreads();
    }
    for (int i = tid; i < row.n; i += kRowThreads) {
        const uint4 v = row.vecs[i];
        const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t k = key_of<FSD_F32>(bits[e]);
            if (k > over && bits[e] != 0xff800000u && k >> (shift + BITS) == prefix) atomicAdd(&s.sub_n[k >> shift & ((1u << BITS) - 1u)], 1u);
        }
    }
    __syncthreads();
    if (rank != 0)
        for (int i = tid; i < 1 << BITS; i += kRowThreads)
            if (s.sub_n[i] != 0u) atomicAdd(&first.sub_n[i], s.sub_n[i]);
}
// What a bin's weights are of: nothing in the bin is above it.  In the bin of the largest value that value, so that it weighs 1 without rounding
// and shares of equal tokens end where they should.
__device__ __forceinline__ double edge_of(uint32_t prefix, double most) {
    const double edge = value_of<FSD_F32>(prefix << 16 | 0xffffu);
    return edge < most ? edge : most;
}
// The same by the 7 bits above 9, and what the tokens weigh against the bin's edge, in whole numbers of 1 / kFixed (which a double from 1/4 to 1
// is: a bin's values are at most 1 apart, but for those below -256, which weigh nothing); and what all tokens above and below the prefix weigh against `most`.
// (Weights are added by their digits to the base 2^16: an addition of 64 bits in shared memory is a loop.  A slice has
// fewer than 2^16 tokens, so that none of the four sums overflows.)
__device__ void weigh_bits(const RowSlice& row, CutShared& s, CutShared& first, int rank, uint32_t prefix, uint32_t over, double most) {
    const int tid = threadIdx.x;
    if (rank != 0) {
        for (int i = tid; i < 512; i += kRowThreads) { s.sub_n[i] = 0u; s.digits[i] = 0u; }
        __syncthreads();
    }
    const double edge = edge_of(prefix, most);
    CountAndWeight above = {0, 0.0}, rest = {0, 0.0};
    for (int i = tid; i < row.n; i += kRowThreads) {
        const uint4 v = row.vecs[i];
        const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t k = key_of<FSD_F32>(bits[e]), high = k >> 16;
            if (k <= over || bits[e] == 0xff800000u) continue;
            const double w = exp_of(static_cast<double>(__uint_as_float(bits[e])) - (high == prefix ? edge : most));
            if (high > prefix) above.w += w;
            if (high < prefix) rest.w += w;
            if (high == prefix) {
                const uint32_t bin = k >> 9 & 127u;
                const unsigned long long fixed = __double2ull_rn(w * kFixed);
                atomicAdd(&s.sub_n[bin], 1u);
                atomicAdd(&s.digits[bin], static_cast<uint32_t>(fixed) & 0xffffu);
                atomicAdd(&s.digits[1 * 128 + bin], static_cast<uint32_t>(fixed) >> 16);
                atomicAdd(&s.digits[2 * 128 + bin], static_cast<uint32_t>(fixed >> 32) & 0xffffu);
                atomicAdd(&s.digits[3 * 128 + bin], static_cast<uint32_t>(fixed >> 48));
            }
        }
    }
    above = block_total(above, s.scratch);
    rest = block_total(rest, s.scratch);
    if (tid == 0) { first.above[rank] = above.w; first.rest[rank] = rest.w; }
    __syncthreads();
    for (int i = tid; i < 128; i += kRowThreads) {
        if (s.sub_n[i] == 0u) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            atomicAdd(reinterpret_cast<unsigned long long*>(&first.sub_w[h * 128 + i]), s.digits[h * 256 + i] + (static_cast<unsigned long long>(s.digits[h * 256 + 128 + i]) << 16));
        if (rank != 0) atomicAdd(&first.sub_n[i], s.sub_n[i]);
    }
}

// The first block tells the others what it found, and clears the counts for the next time.  Two places in turn: a block may still
// be reading what it was told before.
__device__ __forceinline__ CutResult tell_result(CutShared& s, cg::cluster_group& cluster, int rank, int blocks, int& turn) {
    turn ^= 1;
    if (rank == 0) {
        const int tid = threadIdx.x;
        __syncthreads();
        if (tid < blocks) *cluster.map_shared_rank(&s.told[turn], tid) = s.work;
        for (int i = tid; i < 512; i += kRowThreads) { s.sub_n[i] = 0u; s.digits[i] = 0u; }
        for (int i = tid; i < 256; i += kRowThreads) s.sub_w[i] = 0u;
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
__device__ CutResult refine(const RowSlice& row, const uint32_t* hist, CutShared& s, CutShared& first, cg::cluster_group& cluster, int rank, int blocks,
                            const CutParams& c, int V, uint32_t top, CutResult res, int& turn) {
    const int tid = threadIdx.x;
    const double most = value_of<FSD_F32>(top);
    const bool cut_k = res.kind == kCutRefineK;
    int p_bin = rank == 0 ? s.found[3] : 0;                 // (the first block's) the bin that may have the border of top-p
    if (cut_k) {
        for (int shift = 8; shift >= 0; shift -= 8) {
            count_bits<8>(row, s, first, rank, res.key, shift, 0u);
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
        if (rank == 0 && tid == 0) s.work = {kCutRefineP, bin_prefix<FSD_F32>(s, p_bin), 0, 0u};
        res = tell_result(s, cluster, rank, blocks, turn);
    }
    // The bin is a guess, made with the middles of the bins; the sums say whether to move to the next one in use.  (Where rounding would
    // send it back and forth, the border is between the two.)
    int last_move = 0;
    while (res.kind == kCutRefineP) {
        const uint32_t prefix = res.key;
        weigh_bits(row, s, first, rank, prefix, over, most);
        cluster_barrier();
        if (rank == 0) {
            double above = 0.0, rest = 0.0;
            for (int k = 0; k < blocks; ++k) { above += s.above[k]; rest += s.rest[k]; }
            const double unit = exp_of(edge_of(prefix, most) - most) / kFixed;
            Run all;
            const int bin = 127 - tid;
            const double w = tid < 128 ? __fma_rn(static_cast<double>(s.sub_w[128 + bin]), 4294967296.0, static_cast<double>(s.sub_w[bin])) * unit : 0.0;
            const uint32_t n = tid < 128 ? s.sub_n[bin] : 0u;
            const Run before = scan_threads({n, w}, s, all);
            const double goal = static_cast<double>(c.top_p) * (above + all.w + rest + of_ties);
            if (tid == 0) { s.found[1] = -1; s.found[2] = 128; }
            __syncthreads();
            if (n != 0) {
                atomicMax(&s.found[1], tid);                                      // the last sub-bin in use
                if (above + before.w + w >= goal) atomicMin(&s.found[2], tid);
            }
            __syncthreads();
            int place = s.found[2];
            bool up = goal > 0.0 && above >= goal, down = !up && place == 128;
            if (down && s.found[1] >= 0 && last_move > 0) { place = s.found[1]; down = false; }
            if (up && s.found[1] >= 0 && last_move < 0) up = false;               // (place is its first sub-bin in use)
            if (down && cut_k && prefix <= over >> 16) {                          // the border is among the tokens equal to the k-th
                if (tid == 0) {
                    const long long t = ties_below(above + all.w, of_ties / static_cast<double>(k_ties), goal, V);
                    s.work = {kCutDone, over, t < k_ties ? t : all_of_k ? V : k_ties, 0u};
                }
            } else if (up || down) {
                p_bin = next_bin(hist, s, p_bin, up);
                last_move = up ? 1 : -1;
                if (tid == 0) {
                    if (p_bin < 0 || !one_value(s, p_bin)) s.work.kind = kCutByBits;
                    else s.work.key = bin_prefix<FSD_F32>(s, p_bin);
                }
            } else if (tid == place) {
                s.work.key = prefix << 7 | static_cast<uint32_t>(bin);
                s.work.kind = kCutRefineK;                                        // (the last 9 bits)
                s.goal = goal;
                s.above_goal = above + before.w;
            }
        }
        res = tell_result(s, cluster, rank, blocks, turn);
    }
    if (res.kind == kCutRefineK) {
        const uint32_t prefix = res.key;
        count_bits<9>(row, s, first, rank, prefix, 0, over);
        cluster_barrier();
        if (rank == 0) {
            Run all;
            const int bin = 511 - tid;                                            // (a thread each)
            const uint32_t key = prefix << 9 | static_cast<uint32_t>(bin);
            const uint32_t n = s.sub_n[bin];
            const double w = n != 0 ? exp_of(static_cast<double>(value_of<FSD_F32>(key)) - most) : 0.0;
            const Run before = scan_threads({n, static_cast<double>(n) * w}, s, all);
            if (tid == 0) s.found[2] = 512;
            __syncthreads();
            // (where rounding leaves the last of them short of the goal it is the border all the same)
            if (n != 0 && (s.above_goal + before.w + static_cast<double>(n) * w >= s.goal || before.n + n == all.n)) atomicMin(&s.found[2], tid);
            __syncthreads();
            if (tid == s.found[2]) {
                const long long t = ties_below(s.above_goal + before.w, w, s.goal, V);
                s.work = {kCutDone, key, t >= n ? V : t, 0u};
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

// raw: the rows are processed already.
__global__ void __launch_bounds__(kRowThreads, 2) fsd_cut_cluster_kernel(const ProcArgs a, int slice, bool raw) {
    constexpr int DT = FSD_F32, N = Logit<DT>::kPerVec;
    using elem = Logit<DT>::elem;
    extern __shared__ uint4 on_chip[];
    __shared__ CutShared s;
    uint32_t* hist = reinterpret_cast<uint32_t*>(on_chip + slice);
    uint32_t* drafted_ids = slice * N / 32 + 2 <= kDraftedWords ? s.drafted : hist + kBins;      // a bit for each of the slice's ids, from a multiple of 32 on; where tokens are drafted
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int blocks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int all = a.rows[0] + a.rows[1], line = blockIdx.x / blocks, b = line / all, q = line % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    FSD_CHECK(&process_debug, b < a.B && r < a.rows[side] && blocks <= kMaxCutCluster && slice * N <= 65536, kChkItem);
    const size_t at = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
    const elem* in = static_cast<const elem*>(raw ? a.out[side] : a.in[side]) + at;
    elem* out = static_cast<elem*>(a.out[side]) + at;
    const int lies = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16 / sizeof(elem));
    const bool alike = (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const int row_vecs = (a.V + lies + N - 1) / N, v0 = rank * slice;
    RowSlice row = {on_chip, row_vecs - v0 < slice ? (row_vecs > v0 ? row_vecs - v0 : 0) : slice, v0 * N - lies};

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
    FSD_CHECK(&process_debug, row.n <= slice && n_words <= slice * N / 32 + 2, kChkSlice);
    clear_bins(hist, s);
    if (drafts > 0)
        for (int i = tid; i < n_words; i += kRowThreads) drafted_ids[i] = 0u;
    if (tid < 8) s.settings[tid] = setting;
    __syncthreads();
    cluster_arrive();                                       // from here on others may add to the first block's counts
    for (int j = tid; j < drafts; j += kRowThreads) {
        const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j);
        FSD_CHECK(&process_debug, t < ids_lo || t >= ids_hi || ((t >> 5) - word0 >= 0 && (t >> 5) - word0 < n_words), kChkList);
        if (t >= ids_lo && t < ids_hi) atomicOr(&drafted_ids[(t >> 5) - word0], 1u << (t & 31));
    }
    const CutParams c = cut_params(s.settings, a.V);
    const bool cutting = c.k || c.p || c.m;
    const SeqParams p = seq_params(s.settings + 3);

    // the slice: read, processed, counted, kept
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
            count_vec<DT>(v, hist, &s);
            const uint32_t bits[4] = {v.x, v.y, v.z, v.w};
            const uint32_t sparse = (history ? bits8(seen, t0, 4 * a.W) : 0u) | (drafts > 0 ? bits8(drafted_ids, t0 - word0 * 32, 4 * n_words) : 0u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t k = key_of<DT>(bits[e]);
                if (!(sparse >> e & 1u)) top = top > k ? top : k;
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
            for (int base = 0; base < total; base += kListed) {
                while (todo != 0u && at < base + kListed) {
                    FSD_CHECK(&process_debug, at >= base && lane * 32 + 31 < 65536, kChkList);
                    s.list[warp][at - base] = static_cast<uint16_t>(lane * 32 + __ffs(static_cast<int>(todo)) - 1);
                    todo &= todo - 1u;
                    ++at;
                }
                __syncwarp();
                const int n = total - base < kListed ? total - base : kListed;
#pragma unroll 4
                for (int k0 = 0; k0 < n; k0 += 32) {
                    const int k = k0 + lane, l = k < n ? s.list[warp][k] : 0;
                    const uint32_t is_used = __shfl_sync(0xffffffffu, used, l >> 5) >> (l & 31) & 1u;
                    const uint32_t is_draft = __shfl_sync(0xffffffffu, draft, l >> 5) >> (l & 31) & 1u;
                    if (k >= n) continue;
                    const int t = (word0 + w0 + (l >> 5) * kRowWarps) * 32 + (l & 31);
                    FSD_CHECK(&process_debug, t >= ids_lo && t < ids_hi && t - row.first >= 0 && t - row.first < row.n * N, kChkToken);
                    const int count = is_used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1;
                    const float x = read_id<DT>(in, t);
                    const int d = is_draft ? drafted(a, b, ctx, t) : 0;
                    const uint32_t before = words[t];
                    write_id<DT>(words, t, process_id(x, count, d, 0.f, false, p));
                    if (!cutting) continue;
                    const uint32_t now = words[t];
                    count_value<DT, 1>(now, hist, &s);
                    count_value<DT, -1>(before, hist, &s);
                    const uint32_t key = key_of<DT>(now);
                    top = top > key ? top : key;
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
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s.warp_n[warp] = top;
    __syncthreads();
    cluster_wait();
    if (tid == 0) {
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) top = top > s.warp_n[w] ? top : s.warp_n[w];
        first.top[rank] = top;
        if (rank != 0) {
            if (s.mixed != 0u) atomicAdd(&first.mixed, s.mixed);
            if (s.under_lo <= s.under_hi) { atomicMin(&first.under_lo, s.under_lo); atomicMax(&first.under_hi, s.under_hi); }
        }
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
        top = 0u;
        for (int k = 0; k < blocks; ++k) top = top > s.top[k] ? top : s.top[k];
        solve_bins<DT>(hist, s, c, a.V, top);
        if (tid > 0 && tid < blocks) cluster.map_shared_rank(&s, tid)->top[0] = top;
    }
    int turn = 0;
    CutResult res = tell_result(s, cluster, rank, blocks, turn);
    if (res.kind == kCutRefineK || res.kind == kCutRefineP) {
        if (rank != 0) top = s.top[0];
        res = refine(row, hist, s, first, cluster, rank, blocks, c, a.V, top, res, turn);
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
    // Where only the first `ties` of the tokens at the cut are kept, each warp has a run of the slice and counts those before it.
    const int run = (row.n + kRowWarps - 1) / kRowWarps, w0 = warp * run < row.n ? warp * run : row.n, w1 = w0 + run < row.n ? w0 + run : row.n;
    int left = INT_MAX, mine = 0;                           // how many of those in the warp's run are kept, and how many there are
    if (ties < a.V) {
        for (int i = w0 + lane; i < w1; i += 32) mine += equal_in<DT>(row.vecs[i], value);
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) s.warp_n[warp] = static_cast<uint32_t>(mine);
        __syncthreads();
        int sum = 0;
        long long before = 0;
        for (int w = 0; w < kRowWarps; ++w) { if (w == warp) before = sum; sum += static_cast<int>(s.warp_n[w]); }
        if (tid < blocks) cluster.map_shared_rank(&s, tid)->equal[rank] = sum;
        cluster_barrier();
        for (int k = 0; k < rank; ++k) before += s.equal[k];
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
}

}  // namespace fsd
