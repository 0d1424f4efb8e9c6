// Embedding lookup with scaling, and its gradient as sums over sorted tokens.
//
// Forward: out[n] = s * table[id_n].  A copy: bound by the bytes of the rows read and written.
// Backward: dtable[v] = s * sum_{n: id_n = v} dout[n].  What it cannot do without: the rows of dout once,
// the gradient once (all of it, zeros included, in the non-accumulating form: for one micro-batch over
// a full vocabulary that is most of the bytes).  Adding rows with float atomics would make the sum's
// order, and with it the weights, differ from run to run; so the tokens are ordered first by a stable
// radix sort and every sum runs in a fixed order.
#include <cooperative_groups.h>

#include "dte_ops.cuh"

namespace cg = cooperative_groups;

namespace dte {

// ---- forward ----------------------------------------------------------------------------------------
struct LookupParams {
    const void* table;
    const void* ids;
    void* out;
    uint64_t table_ld, out_ld;
    uint32_t ids_dtype, n, rows, hidden, chunks;
    int64_t row_start, vocab;
    float scale;
    uint64_t* flags;
};

constexpr int kLookupThreads = 128;
constexpr int kLookupUnroll = 4;       // accesses in flight per lane

// One warp takes one token's stretch of 32 * V * kLookupUnroll columns.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const LookupParams p) {
    const uint64_t w = (uint64_t)blockIdx.x * (kLookupThreads / 32) + threadIdx.x / 32;
    const uint32_t n = (uint32_t)(w / p.chunks), c = (uint32_t)(w % p.chunks), lane = threadIdx.x & 31;
    if (n >= p.n) return;
    const int64_t id = load_id(p.ids, p.ids_dtype, n);
    const uint64_t row = (uint64_t)id - (uint64_t)p.row_start;
    const bool here = id >= 0 && row < p.rows;
    if (c == 0 && lane == 0 && id >= p.vocab && p.flags)
        atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
    const TI* src = static_cast<const TI*>(p.table) + (here ? row : 0) * p.table_ld;
    TO* dst = static_cast<TO*>(p.out) + (uint64_t)n * p.out_ld;
    const uint32_t col0 = c * (32 * V * kLookupUnroll) + lane * V;
    Vec<TI, V> r[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t col = col0 + u * 32 * V;
        if (here && col < p.hidden) r[u].load(src + col); else r[u].zero();
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t col = col0 + u * 32 * V;
        if (col < p.hidden) {
            float f[V];
            r[u].get(f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = here ? f[j] * p.scale : 0.f;
            Vec<TO, V> o;
            o.set(f);
            o.store(dst + col);
        }
    }
}

template <typename TI, typename TO>
static void lookup_types(const LookupParams& q, bool vec, cudaStream_t st) {
    LookupParams p = q;
    const uint32_t span = 32 * kLookupUnroll * (vec ? 8 : 1);
    p.chunks = (p.hidden + span - 1) / span;
    const uint64_t ctas = ((uint64_t)p.n * p.chunks + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    if (vec) lookup_kernel<TI, TO, 8><<<(unsigned)ctas, kLookupThreads, 0, st>>>(p);
    else lookup_kernel<TI, TO, 1><<<(unsigned)ctas, kLookupThreads, 0, st>>>(p);
}

// ---- stable radix sort of (key, position) -------------------------------------------------------------
// One thread-block cluster sorts: it can synchronise in hardware and read each other's histograms
// through distributed shared memory, so all passes are one launch.  Each warp owns a contiguous stretch of
// the entries, which together with the order of lanes (match mask below the lane) makes the sort stable.
// The kernel that writes the gradient's zeros starts beside it and takes far longer.
constexpr int kSortCtas = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigitBits = 9;
constexpr int kMaxBins = 1 << kMaxDigitBits;
constexpr size_t kSortSmem = ((size_t)kSortWarps * kMaxBins + 2 * kMaxBins + 64) * sizeof(uint32_t);

struct SortParams {
    const void* ids;
    uint32_t ids_dtype, n;
    const uint32_t* n_dev;
    int64_t row_start, vocab;
    uint32_t rows, passes, digit_bits;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint64_t* flags;
};

// Zeros, in small pieces in the order of their addresses: a front of a few MB moving through memory writes
// 7.5 TB/s (2.5 GB in 330 us), while 148 or 296 CTAs that each walk the whole array reach 6.2.
constexpr int kFillThreads = 256;
constexpr uint64_t kFillBytes = kFillThreads * 64;   // of one CTA

struct FillParams {
    uint8_t* data;
    uint64_t rows, row_bytes, ld_bytes, pieces;      // pieces: CTAs per row
};

__global__ void __launch_bounds__(kFillThreads) fill_kernel(const FillParams p) {
    const uint64_t row = blockIdx.x / p.pieces, at = (blockIdx.x % p.pieces) * kFillBytes;
    uint8_t* d = p.data + row * p.ld_bytes + at;
    const uint64_t n = p.row_bytes - at < kFillBytes ? p.row_bytes - at : kFillBytes;
    const uint64_t vecs = (uintptr_t)d & 15u ? 0 : n / 16;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint64_t i = threadIdx.x + u * kFillThreads;
        if (i < vecs) reinterpret_cast<uint4*>(d)[i] = make_uint4(0, 0, 0, 0);
    }
    for (uint64_t i = vecs * 16 + threadIdx.x * 2; i < n; i += kFillThreads * 2) *reinterpret_cast<uint16_t*>(d + i) = 0;
    // the sort runs beside this kernel: whoever follows this kernel must find both complete
    if (blockIdx.x == gridDim.x - 1) wait_for_earlier();
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads, 1) sort_kernel(const SortParams p) {
    extern __shared__ uint32_t sort_smem[];
    let_next_start();
    cg::cluster_group cluster = cg::this_cluster();
    uint32_t* hist = sort_smem;                          // kSortWarps x kMaxBins
    uint32_t* cta_total = hist + kSortWarps * kMaxBins;  // kMaxBins, read by the other CTAs
    uint32_t* base = cta_total + kMaxBins;               // kMaxBins
    uint32_t* scan = base + kMaxBins;                    // 32
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
    const uint32_t rank = blockIdx.x;
    const uint32_t n = p.n_dev ? *p.n_dev : p.n;
    const uint32_t bins = 1u << p.digit_bits, dmask = bins - 1;
    const uint64_t share = ((uint64_t)(n + kSortCtas * kSortWarps - 1) / (kSortCtas * kSortWarps) + 31) / 32 * 32;
    const uint64_t begin = (uint64_t)(rank * kSortWarps + warp) * share;
    const uint64_t end = begin + share < n ? begin + share : n;
    uint32_t* h = hist + warp * kMaxBins;
    bool bad = false;

    for (uint32_t pass = 0; pass < p.passes; ++pass) {
        const uint32_t shift = pass * p.digit_bits;
        const uint32_t* in_key = p.key[(pass & 1) ^ 1];
        const uint32_t* in_pos = p.pos[(pass & 1) ^ 1];
        uint32_t* out_key = p.key[pass & 1];
        uint32_t* out_pos = p.pos[pass & 1];
        auto read_key = [&](uint64_t i) -> uint32_t {
            if (pass) return __ldcg(in_key + i);     // written by other SMs of the cluster: L2
            const int64_t id = load_id(p.ids, p.ids_dtype, i);
            const uint64_t row = (uint64_t)id - (uint64_t)p.row_start;
            bad |= id >= p.vocab;
            return id >= 0 && row < p.rows ? (uint32_t)row : p.rows;
        };
        for (uint32_t d = lane; d < bins; d += 32) h[d] = 0;
        __syncwarp();
        for (uint64_t i0 = begin; i0 < end; i0 += 32) {
            const bool live = i0 + lane < end;
            const uint32_t digit = live ? (read_key(i0 + lane) >> shift) & dmask : kNone;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
            if (live && lane == (uint32_t)(__ffs(same) - 1)) h[digit] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // hist[w][d] := entries of digit d in earlier warps of this CTA
        if (tid < bins) {
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t v = hist[w * kMaxBins + tid];
                hist[w * kMaxBins + tid] = sum;
                sum += v;
            }
            cta_total[tid] = sum;
        }
        cluster.sync();
        // base[d] := entries of smaller digits anywhere + of digit d in earlier CTAs
        uint32_t all = 0, before = 0;
        if (tid < bins) {
            for (uint32_t c = 0; c < kSortCtas; ++c) {
                const uint32_t v = cluster.map_shared_rank(cta_total, c)[tid];
                if (c < rank) before += v;
                all += v;
            }
        }
        uint32_t inc = all;
        if (tid < kMaxBins) {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
                if (lane >= (uint32_t)o) inc += v;
            }
            if (lane == 31) scan[warp] = inc;
        }
        __syncthreads();
        if (tid < bins) {
            uint32_t off = 0;
            for (uint32_t w = 0; w < warp; ++w) off += scan[w];
            base[tid] = off + inc - all + before;
        }
        __syncthreads();
        for (uint32_t d = lane; d < bins; d += 32) h[d] += base[d];
        __syncwarp();
        for (uint64_t i0 = begin; i0 < end; i0 += 32) {
            const bool live = i0 + lane < end;
            const uint32_t key = live ? read_key(i0 + lane) : 0;
            const uint32_t digit = live ? (key >> shift) & dmask : kNone;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
            uint32_t to = 0;
            if (live) to = h[digit] + __popc(same & ((1u << lane) - 1));
            __syncwarp();
            if (live) {
                if (lane == (uint32_t)(__ffs(same) - 1)) h[digit] += __popc(same);
                __stcg(out_key + to, key);
                __stcg(out_pos + to, pass ? __ldcg(in_pos + i0 + lane) : (uint32_t)(i0 + lane));
            }
            __syncwarp();
        }
        __threadfence();
        cluster.sync();      // the pass's output is complete, and cta_total may be reused
    }
    if (bad && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
}

// ---- sums over runs of equal keys ------------------------------------------------------------------------
// The sorted entries are cut into blocks of kSumBlock, whatever the runs are, so a token that makes up
// a tenth of the batch costs no more than rare ones.  A warp sums one block's runs over one stretch of columns;
// a run inside the block is finished there, the ends of runs that cross blocks are left as fp32 partial sums
// (at most two per block: [0] the run that comes in, [1] the run that goes out and began here), which
// the second kernel adds up in order.
constexpr int kSumBlock = 16;          // entries of a warp: two batches of kSumUnroll loads in flight
constexpr int kSumThreads = 128;
constexpr int kSumUnroll = 8;

struct SumParams {
    const uint32_t* key;
    const uint32_t* pos;
    uint32_t n, rows, hidden, chunks;
    const uint32_t* n_dev;
    const void* src;
    uint64_t src_ld;
    const float* weight;
    float scale;
    void* out;
    uint64_t out_ld;
    bool accumulate;
    uint32_t* slot;
    float* partial;      // blocks x 2 x hidden
};

template <typename TO, int V>
__device__ __forceinline__ void write_sum(const SumParams& p, uint32_t key, uint32_t at, uint32_t col, bool active,
                                          float* acc) {
    if (p.slot && col == 0) p.slot[key] = at;
    if (!active) return;
    TO* o = static_cast<TO*>(p.out) + (uint64_t)(p.slot ? at : key) * p.out_ld + col;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] *= p.scale;
    Vec<TO, V> v;
    if (p.accumulate) {
        float old[V];
        v.load(o);
        v.get(old);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += old[j];
    }
    v.set(acc);
    v.store(o);
}

template <typename TS, typename TO, int V, bool WEIGHTED>
__global__ void __launch_bounds__(kSumThreads) sum_runs_kernel(const SumParams p) {
    wait_for_earlier();
    const uint64_t w = (uint64_t)blockIdx.x * (kSumThreads / 32) + threadIdx.x / 32;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t block = w / p.chunks, first = block * kSumBlock;
    const uint32_t n = p.n_dev ? *p.n_dev : p.n;
    if (first >= n) return;
    const uint32_t col = (uint32_t)(w % p.chunks) * (32 * V) + lane * V;
    const bool active = col < p.hidden;
    const bool mine = lane < kSumBlock && first + lane < n;
    const uint32_t key = mine ? p.key[first + lane] : p.rows;
    const uint32_t pos = mine ? p.pos[first + lane] : 0;
    const uint32_t prev = first ? p.key[first - 1] : kNone;
    const uint32_t next = first + kSumBlock < n ? p.key[first + kSumBlock] : kNone;
    const float wt = WEIGHTED && key < p.rows ? p.weight[pos] : 1.f;
    const TS* src = static_cast<const TS*>(p.src) + col;
    float* part = p.partial + block * 2 * p.hidden + col;

    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    uint32_t cur = __shfl_sync(0xFFFFFFFFu, key, 0), start = 0;
    bool incoming = cur == prev;
    for (uint32_t i0 = 0; i0 < kSumBlock && cur < p.rows; i0 += kSumUnroll) {
        Vec<TS, V> r[kSumUnroll];
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, i0 + u), q = __shfl_sync(0xFFFFFFFFu, pos, i0 + u);
            if (k < p.rows && active) r[u].load_cs(src + (uint64_t)q * p.src_ld); else r[u].zero();
        }
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, i0 + u);
            const float f = WEIGHTED ? __shfl_sync(0xFFFFFFFFu, wt, i0 + u) : 1.f;
            if (cur < p.rows && k != cur) {              // uniform over the warp
                if (incoming) {
                    if (active) {
                        Vec<float, V> v;
                        v.set(acc);
                        v.store(part);
                    }
                } else {
                    write_sum<TO, V>(p, cur, (uint32_t)first + start, col, active, acc);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = 0.f;
                cur = k;
                start = i0 + u;
                incoming = false;
            }
            if (k < p.rows) {
                float x[V];
                r[u].get(x);
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = WEIGHTED ? fmaf(f, x[j], acc[j]) : acc[j] + x[j];
            }
        }
    }
    if (cur >= p.rows) return;
    if (incoming || next == cur) {
        if (active) {
            Vec<float, V> v;
            v.set(acc);
            v.store(part + (incoming ? 0 : p.hidden));
        }
    } else {
        write_sum<TO, V>(p, cur, (uint32_t)first + start, col, active, acc);
    }
}

template <typename TO, int V>
__global__ void __launch_bounds__(kSumThreads) sum_crossing_kernel(const SumParams p) {
    wait_for_earlier();
    const uint64_t w = (uint64_t)blockIdx.x * (kSumThreads / 32) + threadIdx.x / 32;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t block = w / p.chunks, first = block * kSumBlock;
    const uint32_t n = p.n_dev ? *p.n_dev : p.n;
    if (first + kSumBlock >= n) return;                       // nothing goes out of the last block
    // lane l: key of entry first - 1 + l, so that one load answers all questions about this block's last run
    const uint32_t at = lane <= kSumBlock + 1 ? lane : kSumBlock + 1;
    const uint32_t key = first + at >= 1 ? p.key[first + at - 1] : kNone;
    const uint32_t last = __shfl_sync(0xFFFFFFFFu, key, kSumBlock);
    if (last >= p.rows || __shfl_sync(0xFFFFFFFFu, key, kSumBlock + 1) != last) return;
    const uint32_t same = __ballot_sync(0xFFFFFFFFu, key == last);
    if ((same & 3u) == 3u) return;                            // an earlier block began this run
    const uint32_t start = __ffs(same & ~1u) - 2;
    // the block in which the run ends: the first behind this one whose last entry is another key
    uint64_t last_block = block + 1;
    while (true) {
        const uint64_t e = (last_block + lane) * kSumBlock + kSumBlock - 1;
        const uint32_t ends = __ballot_sync(0xFFFFFFFFu, e >= n || p.key[e] != last);
        if (ends) {
            last_block += __ffs(ends) - 1;
            // a run that fills its last full block exactly ends there although that block's last key is the same
            if (last_block * kSumBlock >= n || p.key[last_block * kSumBlock] != last) --last_block;
            break;
        }
        last_block += 32;
    }
    const uint32_t col = (uint32_t)(w % p.chunks) * (32 * V) + lane * V;
    const bool active = col < p.hidden;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    if (active) {
        const float* part = p.partial + col;
        Vec<float, V> v;
        v.load(part + (block * 2 + 1) * p.hidden);
        v.get(acc);
#pragma unroll 4
        for (uint64_t b = block + 1; b <= last_block; ++b) {
            float x[V];
            v.load(part + b * 2 * p.hidden);
            v.get(x);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += x[j];
        }
    }
    write_sum<TO, V>(p, last, (uint32_t)first + start, col, active, acc);
}

template <typename TS, typename TO, int V, bool WEIGHTED = false>
static dte_status launch_sums(const SumParams& p, cudaStream_t st) {
    const uint64_t blocks = ((uint64_t)p.n + kSumBlock - 1) / kSumBlock;
    const unsigned ctas = (unsigned)((blocks * p.chunks + kSumThreads / 32 - 1) / (kSumThreads / 32));
    DTE_CUDA(launch_after(sum_runs_kernel<TS, TO, V, WEIGHTED>, dim3(ctas), kSumThreads, 0, st, p));
    if (p.n > kSumBlock) DTE_CUDA(launch_after(sum_crossing_kernel<TO, V>, dim3(ctas), kSumThreads, 0, st, p));
    return DTE_OK;
}

uint64_t sorted_sum_workspace_bytes(uint64_t n, uint64_t hidden) {
    const uint64_t blocks = (n + kSumBlock - 1) / kSumBlock;
    return 4 * align_up(n * 4, kWorkspaceAlign) + align_up(blocks * 2 * hidden * 4, kWorkspaceAlign);
}

dte_status launch_sorted_sum(const SortedSum& q, bool vec, void* workspace, int device, cudaStream_t st) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const uint64_t arr = align_up((uint64_t)q.n * 4, kWorkspaceAlign);
    SortParams s = {};
    s.ids = q.ids;
    s.ids_dtype = q.ids_dtype;
    s.n = q.n;
    s.n_dev = q.n_dev;
    s.row_start = q.row_start;
    s.vocab = (int64_t)q.vocab;
    s.rows = q.rows;
    uint32_t bits = 1;                                   // keys 0 .. rows (rows: dropped entries)
    while (bits < 32 && (q.rows >> bits)) ++bits;
    s.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    s.digit_bits = (bits + s.passes - 1) / s.passes;
    s.key[0] = reinterpret_cast<uint32_t*>(ws);
    s.key[1] = reinterpret_cast<uint32_t*>(ws + arr);
    s.pos[0] = reinterpret_cast<uint32_t*>(ws + 2 * arr);
    s.pos[1] = reinterpret_cast<uint32_t*>(ws + 3 * arr);
    s.flags = q.flags;
    static std::atomic<uint64_t> sort_ready{0};
    dte_status status = allow_smem(sort_kernel, kSortSmem, device, sort_ready);
    if (status != DTE_OK) return status;
    sort_kernel<<<kSortCtas, kSortThreads, kSortSmem, st>>>(s);
    DTE_CUDA(cudaGetLastError());
    if (!q.slot && !q.accumulate) {
        const uint32_t es = elem_size(q.out_dtype);
        FillParams f;
        f.data = static_cast<uint8_t*>(q.out);
        f.rows = q.rows;
        f.row_bytes = (uint64_t)q.hidden * es;
        f.ld_bytes = q.out_ld * es;
        if (q.rows == 1 || f.ld_bytes == f.row_bytes) {      // one row of everything
            f.row_bytes *= f.rows;
            f.rows = 1;
        }
        f.pieces = (f.row_bytes + kFillBytes - 1) / kFillBytes;
        DTE_CUDA(launch_after(fill_kernel, dim3((unsigned)(f.rows * f.pieces)), kFillThreads, 0, st, f));
    }
    if (q.n == 0) return DTE_OK;
    SumParams p = {};
    p.key = s.key[(s.passes & 1) ^ 1];
    p.pos = s.pos[(s.passes & 1) ^ 1];
    p.n = q.n;
    p.n_dev = q.n_dev;
    p.rows = q.rows;
    p.hidden = q.hidden;
    p.chunks = (q.hidden + (vec ? 256 : 32) - 1) / (vec ? 256 : 32);
    p.src = q.src;
    p.src_ld = q.src_ld;
    p.weight = q.weight;
    p.scale = q.scale;
    p.out = q.out;
    p.out_ld = q.out_ld;
    p.accumulate = q.accumulate;
    p.slot = q.slot;
    p.partial = reinterpret_cast<float*>(ws + 4 * arr);
    const bool sb = q.src_dtype == DTE_BF16, ob = q.out_dtype == DTE_BF16;
    if (p.weight) return launch_sums<__nv_bfloat16, float, 8, true>(p, st);      // the head's gradient
    if (vec) {
        if (sb && ob) return launch_sums<__nv_bfloat16, __nv_bfloat16, 8>(p, st);
        if (sb) return launch_sums<__nv_bfloat16, float, 8>(p, st);
        if (ob) return launch_sums<float, __nv_bfloat16, 8>(p, st);
        return launch_sums<float, float, 8>(p, st);
    }
    if (sb && ob) return launch_sums<__nv_bfloat16, __nv_bfloat16, 1>(p, st);
    if (sb) return launch_sums<__nv_bfloat16, float, 1>(p, st);
    if (ob) return launch_sums<float, __nv_bfloat16, 1>(p, st);
    return launch_sums<float, float, 1>(p, st);
}

dte_status device_sms(int device, int* sms) {
    static std::atomic<int> known[kMaxDevices];
    if (device < 0 || device >= kMaxDevices) return op_fail(DTE_ERR_INVALID_ARG, "device ordinal out of range");
    int v = known[device].load(std::memory_order_relaxed);
    if (!v) {
        DTE_CUDA(cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device));
        known[device].store(v, std::memory_order_relaxed);
    }
    *sms = v;
    return DTE_OK;
}

}  // namespace dte

using namespace dte;

extern "C" dte_status dte_embedding_forward(const dte_matrix* table, const dte_ids* ids, uint64_t row_start,
                                            uint64_t vocab, double scale, const dte_matrix* out, uint64_t* flags,
                                            int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_matrix(table, "table is null", false)) != DTE_OK) return s;
    if ((s = check_matrix(out, "out is null", true)) != DTE_OK) return s;
    if ((s = check_ids(ids)) != DTE_OK) return s;
    if ((s = check_range(row_start, table->rows, vocab)) != DTE_OK) return s;
    if (!std::isfinite(scale)) return op_fail(DTE_ERR_INVALID_ARG, "scale is not finite");
    if (table->cols != out->cols || out->rows != ids->count)
        return op_fail(DTE_ERR_INVALID_ARG, "out must be ids.count x table.cols");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if (ids->count == 0) return DTE_OK;
    OpDeviceGuard g(device);
    const bool vec = vec8_ok(table) && vec8_ok(out);
    LookupParams p = {};
    p.table = table->data;
    p.ids = ids->data;
    p.out = out->data;
    p.table_ld = table->ld;
    p.out_ld = out->ld;
    p.ids_dtype = ids->dtype;
    p.n = (uint32_t)ids->count;
    p.rows = (uint32_t)table->rows;
    p.hidden = (uint32_t)table->cols;
    p.row_start = (int64_t)row_start;
    p.vocab = (int64_t)vocab;
    p.scale = (float)scale;
    p.flags = flags;
    const uint64_t span = 32 * kLookupUnroll * (vec ? 8 : 1);
    if (ids->count * ((table->cols + span - 1) / span) >= (1ull << 32))
        return op_fail(DTE_ERR_INVALID_ARG, "ids.count x hidden is too large for one call");
    const bool ib = table->dtype == DTE_BF16, ob = out->dtype == DTE_BF16;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (ib && ob) lookup_types<__nv_bfloat16, __nv_bfloat16>(p, vec, st);
    else if (ib) lookup_types<__nv_bfloat16, float>(p, vec, st);
    else if (ob) lookup_types<float, __nv_bfloat16>(p, vec, st);
    else lookup_types<float, float>(p, vec, st);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

extern "C" uint64_t dte_embedding_backward_workspace_bytes(uint64_t n_ids, uint64_t hidden) {
    if (n_ids >= kMaxDim || hidden >= kMaxDim) return UINT64_MAX;   // refused by the call
    return sorted_sum_workspace_bytes(n_ids, hidden);
}

extern "C" dte_status dte_embedding_backward(const dte_matrix* dout, const dte_ids* ids, uint64_t row_start,
                                             uint64_t vocab, double scale, int accumulate, const dte_matrix* dtable,
                                             void* workspace, uint64_t workspace_bytes, uint64_t* flags, int device,
                                             void* cuda_stream) {
    dte_status s;
    if ((s = check_matrix(dout, "dout is null", false)) != DTE_OK) return s;
    if ((s = check_matrix(dtable, "dtable is null", true)) != DTE_OK) return s;
    if ((s = check_ids(ids)) != DTE_OK) return s;
    if ((s = check_range(row_start, dtable->rows, vocab)) != DTE_OK) return s;
    if (!std::isfinite(scale)) return op_fail(DTE_ERR_INVALID_ARG, "scale is not finite");
    if (dtable->cols != dout->cols || dout->rows != ids->count)
        return op_fail(DTE_ERR_INVALID_ARG, "dout must be ids.count x dtable.cols");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if ((s = check_workspace(workspace, workspace_bytes, sorted_sum_workspace_bytes(ids->count, dout->cols))) != DTE_OK) return s;
    const bool vec = vec8_ok(dout) && vec8_ok(dtable);
    const uint64_t chunks = (dout->cols + (vec ? 255 : 31)) / (vec ? 256 : 32);
    if ((ids->count / kSumBlock + 1) * chunks >= (1ull << 32))
        return op_fail(DTE_ERR_INVALID_ARG, "ids.count x hidden is too large for one call");
    const uint64_t row_bytes = dtable->cols * elem_size(dtable->dtype);
    if (dtable->rows * (row_bytes / kFillBytes + 1) >= (1ull << 31)) return op_fail(DTE_ERR_INVALID_ARG, "dtable is too large for one call");
    if (dtable->rows == 0) return DTE_OK;
    OpDeviceGuard g(device);
    int sms = 0;
    if ((s = device_sms(device, &sms)) != DTE_OK) return s;
    SortedSum q = {};
    q.ids = ids->data;
    q.ids_dtype = ids->dtype;
    q.n = (uint32_t)ids->count;
    q.row_start = (int64_t)row_start;
    q.vocab = vocab;
    q.rows = (uint32_t)dtable->rows;
    q.src = dout->data;
    q.src_dtype = dout->dtype;
    q.src_ld = dout->ld;
    q.hidden = (uint32_t)dout->cols;
    q.scale = (float)scale;
    q.out = dtable->data;
    q.out_dtype = dtable->dtype;
    q.out_ld = dtable->ld;
    q.accumulate = accumulate != 0;
    q.flags = flags;
    return launch_sorted_sum(q, vec, workspace, device, (cudaStream_t)cuda_stream);
}
