// Top-k, top-p and min-p on rows of bf16 logits: a block per row.
#pragma once

#include "fsd_truncate.cuh"

namespace fsd {

// The block reads the row twice and keeps none of it: once to count its values, and again, from the L2 cache for the most part
// (two blocks an SM have 90 MB of rows of 152064 on the way), to write it.  No block waits for another, which is what most of
// a cluster's time went into: 64 x 17 x 152064 took 660 us that way and takes 268 (top_p; 347 to 360 with penalties and mixed settings).
// What bounds it now is its instructions, some 300 for 8 logits: 8 additions to the bins and their addresses, the mask, the temperature
// and the border once or twice.
// Sparse ids, which the count of the others leaves out, are listed in front: a bitmap of the row's, the sum of its bits up to each word, and for
// each id what becomes of it, worked out once, one a thread, and counted then.
struct RowsShape {             // of the dynamic shared memory; the last two are in words and ids
    int words, cap;
};
struct RowsShared {
    BinsShared cut;
    uint32_t equal[2][kRowWarps];
    int n_sparse;
    uint32_t from;             // key of the smallest value read that comes to the cut
    int raised;                // whether a sparse id became more than it would be without
    uint32_t some[8];          // the drafted ids' lowest 8 bits
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

// Whether any of a vector's values is at least `from`, or none (NaN: a row that holds one is to be found out).
__device__ __forceinline__ bool some_from(const uint4& v, const __nv_bfloat162& from) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t below = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < 4; ++k) below &= __hlt2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[k]), from);
    return below != 0xffffffffu;
}

// REGULAR: rows start on 16-byte boundaries and are whole numbers of vectors.
template <bool REGULAR>
__global__ void __launch_bounds__(kRowThreads, 2) fsd_cut_rows_kernel(const ProcArgs a, const RowsShape shape, bool raw) {
    constexpr int DT = FSD_BF16, N = 8, kAtOnce = 2, kTile = kAtOnce * kRowThreads;
    extern __shared__ uint4 on_chip[];
    __shared__ RowsShared s;
    uint32_t* hist = reinterpret_cast<uint32_t*>(on_chip);
    uint32_t* bitmap = hist + kBins;                        // of the sparse ids
    uint32_t* list = bitmap + shape.words;                  // them, and then what becomes of them
    uint16_t* ahead = reinterpret_cast<uint16_t*>(list + shape.cap);          // where in the list a word's are
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int all = a.rows[0] + a.rows[1], b = blockIdx.x / all, q = blockIdx.x % all;
    const int side = q >= a.rows[0], r = q - (side ? a.rows[0] : 0);
    FSD_CHECK(&process_debug, b < a.B && r < a.rows[side], kChkItem);
    const size_t at = (static_cast<size_t>(b) * a.rows[side] + r) * a.V;
    const uint16_t* in = static_cast<const uint16_t*>(raw ? a.out[side] : a.in[side]) + at;
    uint16_t* out = static_cast<uint16_t*>(a.out[side]) + at;
    const int lies = REGULAR ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16 / 2);
    const bool alike = REGULAR || (reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const int n_vecs = (a.V + lies + N - 1) / N;
    // a warp has kAtOnce runs of 32 vectors of a tile, one behind the other
    const auto vec_of = [&](int tile, int u) { return tile + (warp * kAtOnce + u) * 32 + lane; };
    uint4 got[kAtOnce];
    const auto fetch = [&](int tile) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = vec_of(tile, u), t0 = i * N - lies;
            if (i < n_vecs) got[u] = load_ids<DT>(in, t0, a.V, REGULAR || (t0 >= 0 && t0 + N <= a.V));
        }
    };
    uint4 now[kAtOnce];                                     // (while a tile is done the next one is on its way)
    const auto take = [&]() {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) now[u] = got[u];
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
    clear_bins(hist, s.cut);
    if (tid == 0) s.raised = 0;
    if (tid < 8) { s.cut.settings[tid] = setting; s.some[tid] = 0u; }
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
    const auto may_of = [&](int t0) {
        uint32_t may = allowed != nullptr ? bits8(allowed, t0, 4 * a.W) : 0xffu;
        if (!REGULAR && (t0 < 0 || t0 + N > a.V)) may &= ids_of<N>(t0, a.V);                // (what is not in the row counts as masked)
        return may;
    };
    // what becomes of a sparse id
    const auto value_of_id = [&](int t, float x, int count) {
        const bool maybe = drafts > 0 && (s.some[t >> 5 & 7] >> (t & 31) & 1u);
        return process_id(x, count, maybe ? drafted(a, b, ctx, t) : 0, 0.f, false, p);
    };
    bool listed = false;
    if (sparse) {
        if (drafts > 0) {
            const auto add = [&](int j) {
                const int t = __ldg(a.tokens + static_cast<size_t>(b) * a.P + j);
                if (t < 0 || t >= a.V || !(allowed == nullptr || (__ldg(allowed + (t >> 5)) >> (t & 31) & 1u))) return;
                FSD_CHECK(&process_debug, t >> 5 < shape.words, kChkList);
                atomicOr(&bitmap[t >> 5], 1u << (t & 31));
                atomicOr(&s.some[t >> 5 & 7], 1u << (t & 31));
            };
            if (a.parent == nullptr) {
                for (int j = tid; j < ctx; j += kRowThreads) add(j);
            } else if (tid == 0) {
                for (int j = ctx - 1; j >= 0; j = node_before(a, b, j)) add(j);
            }
            __syncthreads();
        }
        // (a thread's words are kRowThreads apart: low ids are used far more often)
        Run mine = {0u, 0.0}, total;
        for (int w = tid; w < a.W; w += kRowThreads) mine.n += __popc(bitmap[w]);
        uint32_t n = scan_threads(mine, s.cut, total).n;
        listed = total.n <= static_cast<uint32_t>(shape.cap);                 // (else each vector works its own out)
        if (tid == 0) s.n_sparse = static_cast<int>(total.n);
        if (listed)
            for (int w = tid; w < a.W; w += kRowThreads) {
                ahead[w] = static_cast<uint16_t>(n);
                const uint32_t used = history ? __ldg(seen + w) : 0u;
                for (uint32_t todo = bitmap[w]; todo != 0u; todo &= todo - 1u) {
                    const int e = __ffs(static_cast<int>(todo)) - 1;
                    FSD_CHECK(&process_debug, n < static_cast<uint32_t>(shape.cap) && w * 32 + e < a.V, kChkList);
                    list[n++] = static_cast<uint32_t>(w * 32 + e) | (used >> e & 1u) << 31;
                }
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
            FSD_CHECK(&process_debug, t >= 0 && t < a.V, kChkToken);
            if (listed) {
                FSD_CHECK(&process_debug, ahead[t >> 5] + __popc(bitmap[t >> 5] & ((1u << (t & 31)) - 1u)) < n_sparse, kChkList);
                half = list[ahead[t >> 5] + __popc(bitmap[t >> 5] & ((1u << (t & 31)) - 1u))];
            } else {
                const bool used = history && (__ldg(seen + (t >> 5)) >> (t & 31) & 1u);
                half = pack_bf16(value_of_id(t, value_at(was, e), used ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1), 0.f);
            }
            put_at(v, e, half);
        }
        return v;
    };

    if (listed) {
#pragma unroll 4
        for (int k = tid; k < n_sparse; k += kRowThreads) {
            const uint32_t entry = list[k];                 // (its highest bit: the id is used)
            const int t = static_cast<int>(entry & 0x7fffffffu), count = (entry >> 31) != 0u ? __ldg(a.counts + static_cast<size_t>(b) * a.V + t) : -1;
            FSD_CHECK(&process_debug, t < a.V, kChkToken);
            const float x = read_id<DT>(in, t);
            const uint32_t is = pack_bf16(value_of_id(t, x, count), 0.f) & 0xffffu;
            list[k] = is;
            if (!(__uint_as_float(is << 16) <= __uint_as_float(pack_bf16(__fmul_rn(x, p.inv_temp), 0.f) << 16))) s.raised = 1;
            if (cutting) count_value<DT, 1>(is << 16, hist, &s.cut);
        }
    }
    // The smallest value that was read and is processed to `value` or more: processed values rise with what was read.  A warp; into s.from.
    const auto find_from = [&](float value) {
        const auto comes = [&](uint32_t key) { return __uint_as_float(pack_bf16(__fmul_rn(value_of<DT>(key), p.inv_temp), 0.f) << 16) >= value; };
        uint32_t lo = key_of_value<DT>(-INFINITY), hi = key_of_value<DT>(INFINITY);        // hi does, lo does not
        while (hi - lo > 1u) {
            const uint32_t step = (hi - lo) / 33u + 1u, to = lo + step * (lane + 1u);
            const uint32_t ballot = __ballot_sync(0xffffffffu, to >= hi || comes(to));
            const uint32_t first = ballot != 0u ? __ffs(static_cast<int>(ballot)) - 1 : 32u;
            const uint32_t old = lo;
            if (first > 0u) lo = old + step * first;
            if (old + step * (first + 1u) < hi) hi = old + step * (first + 1u);
        }
        if (lane == 0) s.from = hi;
    };

    CutResult res = {kCutNone, 0u, a.V, 0u};
    if (cutting) {
        // Of a row that keeps few tokens, two tiles say what is below the last of them: vectors of such values alone are passed over.
        // (Not where sparse ids are not listed: they may become more than they were.)  A row of V = 8 n_vecs tokens gains while what the two
        // tiles say leaves few vectors to look at, us without / with it for 1088 rows:
        //   V = 152064: top_k 1 224 / 195, 20 231 / 212, 50 236 / 230, 64 237 / 237, 100 241 / 247, 1000 258 / 275
        //   V = 98304: 20 152 / 142, 32 155 / 151, 50 157 / 157      V = 65536: 10 109 / 103, 20 110 / 108, 32 111 / 113
        //   V = 49152: 20 90.7 / 91.7    V = 32768: 20 68 / 75
        const bool few = c.k && c.top_k <= n_vecs / 320 && n_vecs >= 8 * kTile && (n_sparse == 0 || listed);
        const bool leaving_out = listed || allowed != nullptr;
        bool passing = false;
        __nv_bfloat162 from = __bfloat162bfloat162(__float2bfloat16_rn(0.f));
        for (int tile = 0; tile < n_vecs; tile += kTile) {
            take();
            if (tile + kTile < n_vecs) fetch(tile + kTile);
            else fetch(0);                                  // (for the second time through)
            if (few && tile == 2 * kTile) {
                if (tid == 0) s.from = 0xffffffffu;
                __syncthreads();
                if (tid == 0) hist[kBinNone] = 0u;
                __syncthreads();
                Run mine = {0u, 0.0}, total;
                for (int j = tid * kBinsEach; j < (tid + 1) * kBinsEach && j < kBins; ++j) mine.n += hist[kBins - 1 - j];
                const uint32_t ahead_n = scan_threads(mine, s.cut, total).n, k = static_cast<uint32_t>(c.top_k);
                if (tid == 0) s.cut.found[0] = -1;
                __syncthreads();
                if (total.n > k && ahead_n < k && ahead_n + mine.n >= k) {
                    uint32_t run = ahead_n;
                    int place = tid * kBinsEach;
                    while ((run += hist[kBins - 1 - place]) < k) ++place;
                    s.cut.found[0] = place;
                }
                __syncthreads();
                const int bin = kBins - 1 - s.cut.found[0];
                if (bin < kBins && bin != kBinOver && bin != kBinMid && bin != kBinUnder) {
                    passing = true;
                    if (warp == 0) find_from(value_of<DT>(bin_prefix<DT>(s.cut, bin)));
                    __syncthreads();
                    from = __bfloat162bfloat162(__float2bfloat16_rn(value_of<DT>(s.from)));
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int i = vec_of(tile, u), t0 = i * N - lies;
                if (i >= n_vecs) break;
                if (passing && !some_from(now[u], from)) continue;
                uint32_t may = may_of(t0);
                uint4 v = process_vec<DT>(now[u], may, p.inv_temp);
                if (n_sparse > 0) {
                    const uint32_t bits = bits8(bitmap, t0, 4 * a.W);
                    if (listed) may &= ~bits;
                    else if (bits != 0u) v = patch(v, now[u], t0);
                }
                // (not by vector: some of a warp's nearly always have a bit, and it would do both)
                if (!leaving_out && may == 0xffu) count_vec<DT>(v, hist, &s.cut);
                else if (may != 0u) count_vec<DT, true>(v, hist, &s.cut, spread_bits<DT>(~may));
            }
        }
        __syncthreads();
        if (tid == 0) hist[kBinNone] = 0u;
        __syncthreads();
        solve_bins<DT>(hist, s.cut, c, a.V, 0u);
        __syncthreads();
        res = s.cut.work;
    }
    __syncthreads();

    // Of processed values only those at or above the cut matter, and they rise with what was read: the smallest value that was read
    // and comes to the cut says of most vectors that nothing in them is kept, without processing them.
    if (res.kind == kCutDone && warp == 0) find_from(value_of<DT>(res.key));
    __syncthreads();
    const __nv_bfloat162 from = __bfloat162bfloat162(__float2bfloat16_rn(value_of<DT>(s.from)));

    // the row again, cut off
    const bool cut = res.kind == kCutDone, look_at = !listed || s.raised != 0;
    const float value = value_of<DT>(res.key);
    long long left = cut && res.ties < a.V ? res.ties : LLONG_MAX;             // how many of the tokens equal to the cut are still kept
    int turn = 0;
    for (int tile = 0; tile < n_vecs; tile += kTile) {
        take();
        if (tile + kTile < n_vecs) fetch(tile + kTile);
        int equal = 0;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = vec_of(tile, u), t0 = i * N - lies;
            if (i >= n_vecs) break;
            uint4 v = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
            const bool look = n_sparse > 0 && bits8(bitmap, t0, 4 * a.W) != 0u;
            if (!cut || (look && look_at) || some_from(now[u], from)) {
                v = process_vec<DT>(now[u], may_of(t0), p.inv_temp);
                if (look) v = patch(v, now[u], t0);
            }
            now[u] = v;
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
            uint4 v = now[u];
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
            if (i < n_vecs) store_ids<DT>(out, t0, a.V, REGULAR || (t0 >= 0 && t0 + N <= a.V && alike), v);
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
