// C ABI of the logit processing calls and of the token counts they read: argument checks and launches.
// See include/fsd_verify.h for the contract of every entry point.
#include <climits>
#include <cstdint>
#include <cuda_runtime.h>
#include <mutex>

#include "fsd_verify.h"
#include "fsd_device.cuh"
#ifdef FSD_DEBUG_CHECKS
namespace fsd {
static __device__ int process_debug;       // what range checks of this file's kernels have failed
}
#endif
#include "fsd_history.cuh"
#include "fsd_process.cuh"
#include "fsd_truncate.cuh"
#include "fsd_truncate_cluster.cuh"
#include "fsd_truncate_rows.cuh"

namespace {

using namespace fsd;

constexpr int kMaxV = 1 << 30;
constexpr int kMaxNodes = 1024;        // as in the tree verification
constexpr int kSMs = 148;
constexpr size_t kCutSmem = 200 * 1024;    // dynamic shared memory of a block of the cut kernel at most; it has 13 KB of its own

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na != 0 && nb != 0 && x < y + nb && y < x + na;
}
// The launch's own status: cudaGetLastError() may give what some earlier call of the process left there.
template <typename... KArgs, typename... Args>
int put(void (*kernel)(KArgs...), long long blocks, int threads, size_t smem, cudaStream_t s, int cluster, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks), 1, 1);
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...) == cudaSuccess ? FSD_OK : FSD_ERR_CUDA;
}
inline int words(int V) { return (V + 31) / 32; }

int check(const fsd_process_opts* o) {
    if (o == nullptr) return FSD_ERR_NULL;
    if (o->struct_size != sizeof(fsd_process_opts)) return FSD_ERR_ENUM;
    if (o->logit_dtype < FSD_F32 || o->logit_dtype > FSD_BF16) return FSD_ERR_ENUM;
    if ((o->counts == nullptr) != (o->seen == nullptr)) return FSD_ERR_NULL;
    const int biases = (o->bias_offsets != nullptr) + (o->bias_tokens != nullptr) + (o->bias_values != nullptr);
    if (biases != 0 && biases != 3) return FSD_ERR_NULL;
    for (const void* p : {static_cast<const void*>(o->counts), static_cast<const void*>(o->seen), static_cast<const void*>(o->repetition),
                          static_cast<const void*>(o->frequency), static_cast<const void*>(o->presence), static_cast<const void*>(o->bias_offsets),
                          static_cast<const void*>(o->bias_tokens), static_cast<const void*>(o->bias_values), static_cast<const void*>(o->allowed),
                          static_cast<const void*>(o->temperature), static_cast<const void*>(o->top_k), static_cast<const void*>(o->top_p),
                          static_cast<const void*>(o->min_p)})
        if (!aligned(p, 4)) return FSD_ERR_ALIGN;
    return FSD_OK;
}

// Whether every row starts on a 16-byte boundary and is a whole number of 16-byte vectors.
bool regular(const ProcArgs& a, size_t es) {
    bool is = a.V * es % 16 == 0;
    for (int k = 0; k < 2; ++k) is = is && (a.rows[k] == 0 || (aligned(a.in[k], 16) && aligned(a.out[k], 16)));
    return is;
}

// fp32: how a row lies in the shared memory of a cluster's blocks: at most 4096 vectors a block, and 2048 where there are fewer blocks than two
// an SM.  us with top-p 0.9 by clusters of 1 / 2 / 4 / 8 blocks (- does not fit), what the rule takes in brackets:
//   1 x 8192: 25.6 / [23.4] / 21.6 / 19.5         1 x 32000: 50 / 36 / [25.6] / 22.6      1 x 128256: - / - / 50 / [35.6]
//   32 x 8192: 25.3 / [23.3] / 22.3 / 23.8        32 x 32000: 71 / 48 / [35.6] / 33.7     32 x 128256: - / - / 52 / [52]
//   148 x 8192: 33.6 / [35.8] / 69 / 102          148 x 32000: 71 / [56] / 83 / 118       148 x 128256: - / - / 253 / [229]
//   1088 x 8192: [126] / 194 / 349 / 652          1088 x 16384: 200 / [257] / 407 / 747   1088 x 32000: 394 / [349] / 485 / 796
// It is not always the fastest: a row or two go faster in more blocks (1 x 32000 in eight, by 3 us), and many rows of 16384 in one.
struct CutShape {
    int blocks, slice;         // slice: vectors a block has
    size_t smem;
    bool fits;
};
CutShape cut_shape(const ProcArgs& a, bool raw) {
    constexpr int N = Logit<FSD_F32>::kPerVec;
    CutShape c;
    const long long rows = static_cast<long long>(a.B) * (a.rows[0] + a.rows[1]);
    const int vecs = (a.V + 2 * (N - 1)) / N;             // a row's, wherever it starts
    c.blocks = 1;
    while (c.blocks < kMaxCutCluster && (vecs > c.blocks * 4096ll || (rows * c.blocks < 2 * kSMs && vecs > c.blocks * 2048ll))) c.blocks <<= 1;
    c.slice = (vecs + c.blocks - 1) / c.blocks;
    const bool drafts = !raw && a.penalties && a.tokens != nullptr && c.slice * N / 32 + 2 > kDraftedWords;
    c.smem = static_cast<size_t>(c.slice) * 16 + kBins * sizeof(uint32_t) + (drafts ? (static_cast<size_t>(c.slice) * N / 32 + 2) * sizeof(uint32_t) : 0);
    c.fits = c.smem <= kCutSmem;
    return c;
}

// bf16: the shared memory of a block that does a row: the bins, and where there are sparse ids their bitmap and list, of as many as two blocks
// an SM have room for (16384 at most).  False where the vocabulary is too long for that.
bool rows_shape(const ProcArgs& a, bool raw, RowsShape* shape, size_t* smem) {
    constexpr long long kTwo = 110 * 1024;                // what two blocks an SM may have each
    const bool sparse = !raw && a.penalties && (a.seen != nullptr || a.tokens != nullptr);
    shape->words = sparse ? (a.W + 3) / 4 * 4 : 0;
    shape->cap = 0;
    const long long fixed = static_cast<long long>(kBins) * 4 + static_cast<long long>(shape->words) * 6;      // (a word and where its ids are in the list)
    if (sparse) {
        const long long room = (fixed + 4 * 4096 <= kTwo ? kTwo : static_cast<long long>(kCutSmem)) - fixed;
        if (room < 4 * 256) return false;
        shape->cap = static_cast<int>(room / 4 < 16384 ? room / 16 * 4 : 16384);
    }
    *smem = static_cast<size_t>(fixed) + static_cast<size_t>(shape->cap) * 4;
    return true;
}

// The table that the kernels read, by a stream of its own: one that waits for nothing else, and that is waited for, so that the table is there
// for whatever stream comes next.  (A copy without a stream waits for all blocking streams, and from pageable memory it may return
// before it is done.)  Another thread's capture, or one of this thread's, goes on undisturbed.
bool copy_weights(const double (&weights)[kBins]) {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) return false;
    cudaStream_t own = nullptr;
    bool ok = cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking) == cudaSuccess;
    if (ok) {
        ok = cudaMemcpyToSymbolAsync(bin_weights, weights, sizeof weights, 0, cudaMemcpyHostToDevice, own) == cudaSuccess;
        ok = cudaStreamSynchronize(own) == cudaSuccess && ok;
        ok = cudaStreamDestroy(own) == cudaSuccess && ok;
    }
    return cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess && ok;
}

// Once a device: the kernels' attributes, and the table they read.
int prepare_cut() {
    constexpr int kDevices = 64;
    static bool ready[kDevices] = {};
    static double weights[kBins];
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return FSD_ERR_CUDA;
    std::lock_guard<std::mutex> lock(mu);
    if (ready[dev]) return FSD_OK;
    if (cudaFuncSetAttribute(fsd_cut_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kCutSmem)) != cudaSuccess ||
        cudaFuncSetAttribute(fsd_cut_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kCutSmem)) != cudaSuccess ||
        cudaFuncSetAttribute(fsd_cut_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kCutSmem)) != cudaSuccess)
        return FSD_ERR_CUDA;
    fill_bin_weights(weights);
    if (!copy_weights(weights)) return FSD_ERR_CUDA;
    ready[dev] = true;
    return FSD_OK;
}

// What a launch of the cut needs and could be refused for: in front of a call's first launch, so that a refused call has done nothing.
template <int DT>
int check_cut(const ProcArgs& a, bool raw) {
    const long long rows = static_cast<long long>(a.B) * (a.rows[0] + a.rows[1]);
    if constexpr (DT == FSD_BF16) {
        RowsShape shape;
        size_t smem;
        if (!rows_shape(a, raw, &shape, &smem)) return FSD_ERR_SHAPE;
    } else if (const CutShape c = cut_shape(a, raw); c.fits && rows * c.blocks > INT_MAX) {
        return FSD_ERR_SHAPE;
    }
    return prepare_cut();
}
// Rows that are cut off.  fp32: a cluster of blocks holds a row in shared memory where it fits, else a block sweeps over it in memory.
template <int DT>
int launch_cut(const ProcArgs& a, bool raw, cudaStream_t s) {
    const long long rows = static_cast<long long>(a.B) * (a.rows[0] + a.rows[1]);
    if constexpr (DT == FSD_BF16) {
        RowsShape shape;
        size_t smem;
        rows_shape(a, raw, &shape, &smem);
        return put(regular(a, 2) ? fsd_cut_rows_kernel<true> : fsd_cut_rows_kernel<false>, rows, kRowThreads, smem, s, 0, a, shape, raw);
    } else {
        const CutShape c = cut_shape(a, raw);
        if (!c.fits) return put(fsd_cut_long_kernel<DT>, rows, kLongThreads, 0, s, 0, a);
        return put(fsd_cut_cluster_kernel, rows * c.blocks, kRowThreads, c.smem, s, c.blocks, a, c.slice, raw);
    }
}

template <int DT>
int launch(const ProcArgs& a, bool cut, cudaStream_t s) {
    const int all = a.rows[0] + a.rows[1];
    // The cut kernel does the rest too where it has room for it and there are no biases (whose lookup wants room there).
    RowsShape shape;
    size_t smem;
    const bool room = DT == FSD_BF16 ? rows_shape(a, false, &shape, &smem) : cut_shape(a, false).fits;
    const bool one = cut && a.bias_offsets == nullptr && room;
    // a row's vectors, wherever it starts, by blocks
    const long long spans = (a.V + 2 * (Logit<DT>::kPerVec - 1)) / Logit<DT>::kPerVec / kProcThreads + 1;
    // as many rows a block as leave eight blocks an SM, and four at least: what a block sets up is for all of them
    long long group = spans * a.B * all / (8 * kSMs);
    group = group < 4 ? 4 : group;
    group = group > all ? all : group;
    const long long groups = (all + group - 1) / group;
    if (!one && spans * groups * a.B > INT_MAX) return FSD_ERR_SHAPE;
    if (cut) {
        const int rc = check_cut<DT>(a, !one);
        if (rc != FSD_OK) return rc;
        if (one) return launch_cut<DT>(a, false, s);
    }
    const int rc = put(regular(a, sizeof(typename Logit<DT>::elem)) ? fsd_process_kernel<DT, true> : fsd_process_kernel<DT, false>, spans * groups * a.B, kProcThreads, 0, s, 0,
                       a, static_cast<int>(spans), static_cast<int>(groups), static_cast<int>(group));
    if (rc != FSD_OK) return rc;
    return cut ? launch_cut<DT>(a, true, s) : FSD_OK;
}

int process(const void* target_in, const void* draft_in, const int32_t* parent, const int32_t* tokens, int B, int P, int V,
            const fsd_process_opts* o, void* target_out, void* draft_out, void* stream) {
    if (target_in == nullptr || target_out == nullptr || (draft_in == nullptr) != (draft_out == nullptr)) return FSD_ERR_NULL;
    if (B < 1 || V < 1 || V > kMaxV || static_cast<long long>(B) * (2ll * P + 1) > INT_MAX) return FSD_ERR_SHAPE;
    const size_t es = o->logit_dtype == FSD_BF16 ? 2 : 4;
    if (!aligned(target_in, es) || !aligned(target_out, es) || !aligned(draft_in, es) || !aligned(draft_out, es) || !aligned(parent, 4) || !aligned(tokens, 4))
        return FSD_ERR_ALIGN;
    const size_t W4 = static_cast<size_t>(words(V)) * 4, nB = static_cast<size_t>(B) * 4;
    const size_t nt = static_cast<size_t>(B) * (P + 1) * V * es, nd = draft_in != nullptr ? static_cast<size_t>(B) * P * V * es : 0;
    const struct { const void* p; size_t n; } ins[] = {
        {target_in, nt}, {draft_in, nd}, {parent, nB * P}, {tokens, nB * P}, {o->counts, nB * V}, {o->seen, B * W4}, {o->repetition, nB}, {o->frequency, nB},
        {o->presence, nB}, {o->bias_offsets, nB + 4}, {o->allowed, static_cast<size_t>(B) * (P + 1) * W4}, {o->temperature, nB}, {o->top_k, nB}, {o->top_p, nB},
        {o->min_p, nB}};
    // (a side's own input may be its output, and nothing else that happens to start there)
    for (const auto& in : ins) {
        if (in.p == nullptr) continue;
        if (overlap(in.p, in.n, target_out, nt) && !(&in == &ins[0] && target_in == target_out)) return FSD_ERR_UNSUPPORTED;
        if (nd != 0 && overlap(in.p, in.n, draft_out, nd) && !(&in == &ins[1] && draft_in == draft_out)) return FSD_ERR_UNSUPPORTED;
    }
    if (overlap(target_out, nt, draft_out, nd)) return FSD_ERR_UNSUPPORTED;
    ProcArgs a = {};
    a.in[0] = target_in; a.in[1] = draft_in;
    a.out[0] = target_out; a.out[1] = draft_out;
    a.rows[0] = P + 1; a.rows[1] = draft_in != nullptr ? P : 0;
    a.tokens = P > 0 ? tokens : nullptr;
    a.parent = parent;
    a.B = B; a.P = P; a.V = V; a.W = words(V);
    a.penalties = o->repetition != nullptr || o->frequency != nullptr || o->presence != nullptr;
    a.repetition = o->repetition; a.frequency = o->frequency; a.presence = o->presence;
    a.counts = o->counts; a.seen = o->seen;
    a.bias_offsets = o->bias_offsets; a.bias_tokens = o->bias_tokens; a.bias_values = o->bias_values;
    a.allowed = o->allowed; a.temperature = o->temperature;
    a.top_k = o->top_k; a.top_p = o->top_p; a.min_p = o->min_p;
    const bool cut = o->top_k != nullptr || o->top_p != nullptr || o->min_p != nullptr;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return o->logit_dtype == FSD_BF16 ? launch<FSD_BF16>(a, cut, s) : launch<FSD_F32>(a, cut, s);
}

int append(const int32_t* tokens, const int32_t* path, const int32_t* accept_len, const int32_t* next_token, int B, int P, int width, int V,
           int32_t* counts, uint32_t* seen, void* stream) {
    if (V > kMaxV || static_cast<long long>(B) * (P > width ? P : width) > INT_MAX) return FSD_ERR_SHAPE;
    for (const void* p : {static_cast<const void*>(tokens), static_cast<const void*>(path), static_cast<const void*>(accept_len),
                          static_cast<const void*>(next_token), static_cast<const void*>(counts), static_cast<const void*>(seen)})
        if (!aligned(p, 4)) return FSD_ERR_ALIGN;
    return put(fsd_history_append_kernel, (B + 3ll) / 4, 128, 0, static_cast<cudaStream_t>(stream), 0, tokens, path, accept_len, next_token, B, P, width, V, words(V), counts, seen);
}

}  // namespace

extern "C" {

void fsd_default_process_opts(fsd_process_opts* opts) {
    if (opts == nullptr) return;
    *opts = {};
    opts->struct_size = sizeof(fsd_process_opts);
    opts->logit_dtype = FSD_BF16;
}

int fsd_process_chain(const void* target_in, const void* draft_in, const int32_t* draft_tokens, int B, int gamma, int V,
                      const fsd_process_opts* opts, void* target_out, void* draft_out, void* stream) {
    const int rc = check(opts);
    if (rc != FSD_OK) return rc;
    if (gamma < 0) return FSD_ERR_SHAPE;
    return process(target_in, draft_in, nullptr, draft_tokens, B, gamma, V, opts, target_out, draft_out, stream);
}

int fsd_process_tree(const void* target_in, const void* draft_in, const int32_t* parent, const int32_t* node_tokens, int B, int N, int V,
                     const fsd_process_opts* opts, void* target_out, void* draft_out, void* stream) {
    const int rc = check(opts);
    if (rc != FSD_OK) return rc;
    if (parent == nullptr) return FSD_ERR_NULL;
    if (N < 1 || N > kMaxNodes) return FSD_ERR_SHAPE;
    return process(target_in, draft_in, parent, node_tokens, B, N, V, opts, target_out, draft_out, stream);
}

int fsd_debug_process_word(int* word) {
    if (word == nullptr) return FSD_ERR_NULL;
    *word = 0;
#ifdef FSD_DEBUG_CHECKS
    if (cudaMemcpyFromSymbol(word, process_debug, sizeof *word) != cudaSuccess) return FSD_ERR_CUDA;
#endif
    return FSD_OK;
}

int fsd_history_build(const int32_t* prompt_offsets, const int32_t* prompt_tokens, const int32_t* output_offsets, const int32_t* output_tokens,
                      int B, int V, int32_t* counts, uint32_t* seen, void* stream) {
    if (prompt_offsets == nullptr || prompt_tokens == nullptr || (output_offsets == nullptr) != (output_tokens == nullptr) || counts == nullptr || seen == nullptr)
        return FSD_ERR_NULL;
    const long long spans = (static_cast<long long>(V) + kHistSpan - 1) / kHistSpan;
    if (B < 1 || V < 1 || V > kMaxV || spans * B > INT_MAX) return FSD_ERR_SHAPE;
    for (const void* p : {static_cast<const void*>(prompt_offsets), static_cast<const void*>(prompt_tokens), static_cast<const void*>(output_offsets),
                          static_cast<const void*>(output_tokens), static_cast<const void*>(counts), static_cast<const void*>(seen)})
        if (!aligned(p, 4)) return FSD_ERR_ALIGN;
    return put(fsd_history_build_kernel, spans * B, kHistThreads, 0, static_cast<cudaStream_t>(stream), 0, prompt_offsets, prompt_tokens, output_offsets, output_tokens, V,
               words(V), static_cast<int>(spans), counts, seen);
}

int fsd_history_append_chain(const int32_t* draft_tokens, const int32_t* accept_len, const int32_t* next_token, int B, int gamma, int V,
                             int32_t* counts, uint32_t* seen, void* stream) {
    if (draft_tokens == nullptr || accept_len == nullptr || next_token == nullptr || counts == nullptr || seen == nullptr) return FSD_ERR_NULL;
    if (B < 1 || gamma < 1 || V < 1) return FSD_ERR_SHAPE;
    return append(draft_tokens, nullptr, accept_len, next_token, B, gamma, gamma, V, counts, seen, stream);
}

int fsd_history_append_tree(const int32_t* node_tokens, const int32_t* path, const int32_t* accept_len, const int32_t* next_token, int B, int N,
                            int max_depth, int V, int32_t* counts, uint32_t* seen, void* stream) {
    if (node_tokens == nullptr || path == nullptr || accept_len == nullptr || next_token == nullptr || counts == nullptr || seen == nullptr) return FSD_ERR_NULL;
    if (B < 1 || N < 1 || max_depth < 1 || V < 1) return FSD_ERR_SHAPE;
    return append(node_tokens, path, accept_len, next_token, B, N, max_depth, V, counts, seen, stream);
}

}  // extern "C"
