// Embedding lookup with scaling, and its gradient as sums over sorted tokens.
//
// Forward: out[n] = s * table[id_n].  A copy: bound by the bytes of the rows read and written.
// Backward: dtable[v] = s * sum_{n: id_n = v} dout[n].  What it cannot do without: the rows of dout once,
// the gradient once (all of it, zeros included, in the non-accumulating form: for one micro-batch over
// a full vocabulary that is most of the bytes).  Adding rows with float atomics would make the sum's
// order, and with it the weights, differ from run to run; so the tokens are grouped by row first, in the
// order of the tokens, and every sum runs in a fixed order.
#include "dte_ops.cuh"

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

// One warp takes one token's stretch of 32 * V * kLookupUnroll columns: small CTAs in the order of the output, which
// the memory takes fastest.  16384 x 4096 bf16: 35 us, 7.6 TB/s of rows in and out (repeated rows come from L2).
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
static void lookup_types(const LookupParams& q, int vec, cudaStream_t st) {
    LookupParams p = q;
    const uint32_t span = 32 * kLookupUnroll * vec;
    p.chunks = (p.hidden + span - 1) / span;
    const uint64_t ctas = ((uint64_t)p.n * p.chunks + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    if (vec == 8) lookup_kernel<TI, TO, 8><<<(unsigned)ctas, kLookupThreads, 0, st>>>(p);
    else if (vec == 2) lookup_kernel<TI, TO, 2><<<(unsigned)ctas, kLookupThreads, 0, st>>>(p);
    else lookup_kernel<TI, TO, 1><<<(unsigned)ctas, kLookupThreads, 0, st>>>(p);
}

// ---- tokens grouped by row ------------------------------------------------------------------------------
// The rows are cut into ranges, one CTA each.  Every CTA reads all ids (they stay in L2: 16384 ids are 128 KB),
// counts those of its range per row and those of smaller rows in all, and so knows where its entries start
// without hearing from any other CTA: one launch, no communication.  Each warp owns a contiguous stretch of the ids
// and a histogram of its own, which together with the order of the lanes makes the grouping stable: entries of
// a row are in the order of the tokens.  (A radix sort in one thread-block cluster took 22 us for 16384
// ids and 152 k rows.)
constexpr int kGroupThreads = 1024;
constexpr int kGroupWarps = kGroupThreads / 32;
constexpr uint32_t kMaxBins = 1536;            // rows of a CTA: 32 histograms of this many words fill 192 KB
constexpr uint32_t kGroupCtas = 148;           // ranges to aim for: one per SM
constexpr int kGroupUnroll = 16;               // ids of a lane in flight: 16384 ids are one round

struct GroupParams {
    const void* ids;
    uint32_t ids_dtype, n;
    int64_t row_start, vocab;
    uint32_t rows, bins, warps;    // warps that have entries
    uint32_t* first;           // rows + 1: where each row's entries start
    uint32_t* key;             // entries: row ...
    uint32_t* pos;             // ... and token
    uint32_t* counters;        // cleared for the kernel behind
    uint32_t n_counters;
    uint64_t* flags;
};

__global__ void __launch_bounds__(kGroupThreads, 1) group_kernel(const GroupParams p) {
    extern __shared__ uint32_t group_hist[];    // warps x bins
    __shared__ uint32_t s_warp[32];
    __shared__ uint32_t s_below;
    // reads what the caller passed and writes what no kernel in front of it in this call uses, so it need not wait for them
    let_next_start();
    const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid & 31, below_lanes = (1u << lane) - 1;
    const uint32_t n = p.n;
    const uint32_t r0 = blockIdx.x * p.bins, count = min(p.bins, p.rows - r0);
    const uint64_t share = ((uint64_t)n + p.warps * 32 - 1) / (p.warps * 32) * 32;
    const uint64_t begin = min(warp * share, (uint64_t)n), end = min(begin + share, (uint64_t)n);
    uint32_t* h = group_hist + warp * p.bins;
    for (uint32_t i = tid; i < p.warps * p.bins; i += kGroupThreads) group_hist[i] = 0;
    for (uint32_t i = blockIdx.x * kGroupThreads + tid; i < p.n_counters; i += gridDim.x * kGroupThreads) p.counters[i] = 0;
    if (tid == 0) s_below = 0;
    __syncthreads();

    // calls f(index, row - r0, mask of lanes with the same row) for the entries of this range, in order
    uint32_t below = 0;
    bool bad = false;
    auto scan = [&](bool first_time, auto&& f) {
        for (uint64_t i0 = begin; i0 < end; i0 += 32 * kGroupUnroll) {
            int64_t id[kGroupUnroll];
#pragma unroll
            for (int u = 0; u < kGroupUnroll; ++u) {
                const uint64_t i = i0 + u * 32 + lane;
                id[u] = i < end ? load_id(p.ids, p.ids_dtype, i) : -1;
            }
#pragma unroll
            for (int u = 0; u < kGroupUnroll; ++u) {
                const uint64_t row = (uint64_t)id[u] - (uint64_t)p.row_start;
                const bool valid = id[u] >= 0 && row < p.rows;
                const bool mine = valid && (uint32_t)row - r0 < count;
                if (first_time) {
                    below += valid && row < r0;
                    bad |= id[u] >= p.vocab;
                }
                if (__any_sync(0xFFFFFFFFu, mine)) {
                    const uint32_t bin = mine ? (uint32_t)row - r0 : kNone;
                    const uint32_t same = __match_any_sync(0xFFFFFFFFu, bin);
                    f(i0 + u * 32 + lane, mine, bin, same);
                    __syncwarp();
                }
            }
        }
    };
    scan(true, [&](uint64_t, bool mine, uint32_t bin, uint32_t same) {
        if (mine && !(same & below_lanes)) h[bin] += __popc(same);
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) below += __shfl_xor_sync(0xFFFFFFFFu, below, o);
    if (lane == 0) atomicAdd(&s_below, below);
    __syncthreads();
    // thread t: bins 2t and 2t + 1
    uint32_t total[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t bin = 2 * tid + j;
        if (bin < count)
            for (uint32_t w = 0; w < p.warps; ++w) {
                const uint32_t v = group_hist[w * p.bins + bin];
                group_hist[w * p.bins + bin] = total[j];
                total[j] += v;
            }
    }
    uint32_t inc = total[0] + total[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= (uint32_t)o) inc += v;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    uint32_t off = lane < warp ? s_warp[lane] : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) off += __shfl_xor_sync(0xFFFFFFFFu, off, o);
    uint32_t at = s_below + off + inc - total[0] - total[1];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t bin = 2 * tid + j;
        if (bin < count) {
            p.first[r0 + bin] = at;
            if (r0 + bin + 1 == p.rows) p.first[p.rows] = at + total[j];
            if (total[j])
                for (uint32_t w = 0; w < p.warps; ++w) group_hist[w * p.bins + bin] += at;
            at += total[j];
        }
    }
    __syncthreads();
    scan(false, [&](uint64_t i, bool mine, uint32_t bin, uint32_t same) {
        uint32_t to = 0;
        if (mine) to = h[bin] + __popc(same & below_lanes);
        __syncwarp();
        if (mine) {
            if (!(same & below_lanes)) h[bin] += __popc(same);
            p.key[to] = r0 + bin;
            p.pos[to] = (uint32_t)i;
        }
    });
    if (bad && blockIdx.x == 0 && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
    if (blockIdx.x == 0) wait_for_earlier();      // whoever waits for this kernel waits for the ones in front of it, too
}

// ---- zeros ---------------------------------------------------------------------------------------------------
// Written beside the grouping, in small pieces in the order of their addresses: such a front of a few MB moving
// through memory writes 7.5 TB/s (2.5 GB in 330 us), while 148 or 296 CTAs that each walk the whole array reach 6.2.
// Rows with entries are written twice; to look up first which rows have none cost each small CTA more
// (2.5 GB in 515 us) than the second write.
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
    // the grouping runs beside this kernel: whoever follows this kernel must find both complete
    if (blockIdx.x == gridDim.x - 1) wait_for_earlier();
}

// ---- sums over the entries of a row -------------------------------------
// The grouped entries are cut into blocks, whatever the rows are, so a token that makes up a tenth of
// the batch costs no more than rare ones.  A warp sums one block's runs of equal rows over one stretch of columns; a
// run inside the block is finished there.  Of a run that crosses blocks each block leaves an fp32 partial sum (at most
// two per block: [0] of the run that comes in, [1] of the run that began here and goes on), and the warp that leaves
// the last of them adds them up, in the order of the blocks whoever it is.
constexpr uint32_t kMaxSumBlock = 16;   // entries of a warp, fewer where there are too few to fill the GPU (see sum_block)
constexpr uint32_t kMinSumBlock = 4;
constexpr int kSumThreads = 128;
constexpr int kSumUnroll = 4;          // entries of a batch: with 8 the registers cost more warps than the loads gain (411 -> 393 us)

struct SumParams {
    const uint32_t* first;
    const uint32_t* key;
    const uint32_t* pos;
    uint32_t rows, hidden, chunks, block;
    const void* src;
    uint64_t src_ld;
    const float* weight;
    float scale;
    void* out;
    uint64_t out_ld;
    bool accumulate, compact;
    float* partial;          // blocks x 2 x hidden
    uint32_t* counters;      // blocks x chunks: partial sums left of the run that begins in the block and goes on
};

template <int V>
__device__ __forceinline__ void load_partial(const float* p, float* f) {       // written by other SMs: from L2
    if constexpr (V == 2) {
        const float2 a = __ldcg(reinterpret_cast<const float2*>(p));
        f[0] = a.x;
        f[1] = a.y;
    } else if constexpr (V == 8) {
        const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
        f[0] = __ldcg(p);
    }
}

template <typename TO, int V>
__device__ __forceinline__ void write_sum(const SumParams& p, uint32_t row, uint32_t col, bool active, float* acc) {
    if (!active) return;
    TO* o = static_cast<TO*>(p.out) + row * p.out_ld + col;
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

// Leaves this block's share of a run that crosses blocks; the last to do so finishes the run.
template <typename TO, int V>
__device__ __forceinline__ void leave_partial(const SumParams& p, uint64_t block, uint32_t chunk, uint32_t key, uint32_t col, bool active,
                                              float* acc) {
    const uint32_t begin = p.first[key], end = p.first[key + 1];
    const uint64_t b0 = begin / p.block, b1 = (end - 1) / p.block;
    if (active) {
        Vec<float, V> v;
        v.set(acc);
        v.store(p.partial + (block * 2 + (block == b0)) * p.hidden + col);
    }
    __threadfence();
    __syncwarp();
    uint32_t last = 0;
    if ((threadIdx.x & 31) == 0) last = atomicAdd(p.counters + b0 * p.chunks + chunk, 1u) == (uint32_t)(b1 - b0);
    if (!__shfl_sync(0xFFFFFFFFu, last, 0)) return;
    __threadfence();
    if (active) {
        const float* part = p.partial + col;
        float sum[V];
        load_partial<V>(part + (b0 * 2 + 1) * p.hidden, sum);
#pragma unroll 2
        for (uint64_t b = b0 + 1; b <= b1; ++b) {
            float x[V];
            load_partial<V>(part + b * 2 * p.hidden, x);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += x[j];
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = sum[j];
    }
    write_sum<TO, V>(p, p.compact ? begin : key, col, active, acc);
}

template <typename TS, typename TO, int V, bool WEIGHTED>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumParams p) {
    wait_for_earlier();
    const uint32_t w = blockIdx.x * (kSumThreads / 32) + threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t block = w / p.chunks, chunk = w % p.chunks, first = block * p.block;
    const uint32_t n = p.first[p.rows];                      // entries of this shard
    if (first >= n) return;
    const uint32_t col = chunk * (32 * V) + lane * V;
    const bool active = col < p.hidden;
    const bool mine = lane < p.block && first + lane < n;
    const uint32_t key = mine ? p.key[first + lane] : kNone;
    const uint32_t pos = mine ? p.pos[first + lane] : 0;
    const uint32_t prev = first ? p.key[first - 1] : kNone;
    const uint32_t next = first + p.block < n ? p.key[first + p.block] : kNone;
    const float wt = WEIGHTED && mine ? p.weight[pos] : 1.f;
    const TS* src = static_cast<const TS*>(p.src) + col;

    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    uint32_t cur = __shfl_sync(0xFFFFFFFFu, key, 0), start = 0;
    bool incoming = cur == prev;
    for (uint32_t i0 = 0; i0 < p.block && first + i0 < n; i0 += kSumUnroll) {
        Vec<TS, V> r[kSumUnroll];
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const uint32_t q = __shfl_sync(0xFFFFFFFFu, pos, i0 + u);
            if (first + i0 + u < n && active) r[u].load_cs(src + q * p.src_ld); else r[u].zero();
        }
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, i0 + u);
            const float f = WEIGHTED ? __shfl_sync(0xFFFFFFFFu, wt, i0 + u) : 1.f;
            if (k == kNone) break;                           // uniform over the warp, like the next one
            if (k != cur) {
                if (incoming) leave_partial<TO, V>(p, block, chunk, cur, col, active, acc);
                else write_sum<TO, V>(p, p.compact ? first + start : cur, col, active, acc);
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = 0.f;
                cur = k;
                start = i0 + u;
                incoming = false;
            }
            float x[V];
            r[u].get(x);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = WEIGHTED ? fmaf(f, x[j], acc[j]) : acc[j] + x[j];
        }
    }
    if (incoming || next == cur) leave_partial<TO, V>(p, block, chunk, cur, col, active, acc);
    else write_sum<TO, V>(p, p.compact ? first + start : cur, col, active, acc);
}

static uint64_t sum_chunks(uint64_t hidden, int vec) { return (hidden + 32 * vec - 1) / (32 * vec); }

struct SumLayout {
    uint64_t first, key, pos, counters, partial, total;
};

// Entries of a block: the most, unless that leaves the GPU short of warps.  921 entries x 2048 (the head's gradient): blocks
// of 16 18.5 us, of 4 10.8 us; 16384 x 4096: blocks of 16 393 us with the zeros, of 8 405 us.
static uint32_t sum_block(uint64_t n, uint64_t chunks) {
    uint32_t block = kMaxSumBlock;
    while (block > kMinSumBlock && n / block * chunks < kGroupCtas * 32) block /= 2;
    return block;
}

static SumLayout sum_layout(uint64_t n, uint64_t rows, uint64_t hidden) {
    const uint64_t most = sum_chunks(hidden, 1);       // element by element
    const uint64_t blocks = (n + kMinSumBlock - 1) / kMinSumBlock;
    // smaller blocks are used only while twice their size gives fewer than kGroupCtas * 32 warps (sum_block)
    const uint64_t by_most = (n + kMaxSumBlock - 1) / kMaxSumBlock;
    const uint64_t few = 2 * kGroupCtas * 32 / sum_chunks(hidden, 8) + 2;
    const uint64_t used = by_most > (blocks < few ? blocks : few) ? by_most : (blocks < few ? blocks : few);
    SumLayout l;
    l.first = 0;
    l.key = l.first + align_up((rows + 1) * 4, kWorkspaceAlign);
    l.pos = l.key + align_up(n * 4, kWorkspaceAlign);
    l.counters = l.pos + align_up(n * 4, kWorkspaceAlign);
    l.partial = l.counters + align_up(used * most * 4, kWorkspaceAlign);
    l.total = l.partial + align_up(used * 2 * hidden * 4, kWorkspaceAlign);
    return l;
}

uint64_t sorted_sum_workspace_bytes(uint64_t n, uint64_t rows, uint64_t hidden) { return sum_layout(n, rows, hidden).total; }

const uint32_t* sorted_sum_first(const void* workspace) { return static_cast<const uint32_t*>(workspace); }

bool sorted_sum_fits(uint64_t n, uint64_t rows, uint64_t hidden, uint32_t out_dtype) {
    const uint64_t sums = (n / kMinSumBlock + 1) * sum_chunks(hidden, 1);
    const uint64_t fills = rows * (hidden * elem_size(out_dtype) / kFillBytes + 1);
    return sums < (1ull << 31) && fills < (1ull << 31) && sums + fills < (1ull << 31);
}

template <typename TS, typename TO, bool WEIGHTED = false>
static dte_status launch_sums(const SumParams& p, int vec, unsigned ctas, cudaStream_t st) {
    if (vec == 8) DTE_CUDA(launch_after(sum_kernel<TS, TO, 8, WEIGHTED>, dim3(ctas), kSumThreads, 0, st, p));
    else if (vec == 2) DTE_CUDA(launch_after(sum_kernel<TS, TO, 2, WEIGHTED>, dim3(ctas), kSumThreads, 0, st, p));
    else DTE_CUDA(launch_after(sum_kernel<TS, TO, 1, WEIGHTED>, dim3(ctas), kSumThreads, 0, st, p));
    return DTE_OK;
}

dte_status launch_sorted_sum(const SortedSum& q, int vec, void* workspace, bool after, int device, cudaStream_t st) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const SumLayout l = sum_layout(q.n, q.rows, q.hidden);
    const uint64_t chunks = sum_chunks(q.hidden, vec);
    const uint32_t block = sum_block(q.n, chunks);
    const uint64_t blocks = ((uint64_t)q.n + block - 1) / block;
    GroupParams g = {};
    g.ids = q.ids;
    g.ids_dtype = q.ids_dtype;
    g.n = q.n;
    g.row_start = q.row_start;
    g.vocab = (int64_t)q.vocab;
    g.rows = q.rows;
    g.bins = (q.rows + kGroupCtas - 1) / kGroupCtas;
    if (g.bins > kMaxBins) g.bins = kMaxBins;
    // a warp takes at least one round of loads: few entries leave fewer histograms to add up
    const uint64_t warps = ((uint64_t)q.n + 32 * kGroupUnroll - 1) / (32 * kGroupUnroll);
    g.warps = (uint32_t)(warps < 1 ? 1 : warps > kGroupWarps ? kGroupWarps : warps);
    g.first = reinterpret_cast<uint32_t*>(ws + l.first);
    g.key = reinterpret_cast<uint32_t*>(ws + l.key);
    g.pos = reinterpret_cast<uint32_t*>(ws + l.pos);
    g.counters = reinterpret_cast<uint32_t*>(ws + l.counters);
    g.n_counters = (uint32_t)(blocks * chunks);
    g.flags = q.flags;
    static std::atomic<uint64_t> ready{0};
    dte_status s = allow_smem(group_kernel, (size_t)kGroupWarps * kMaxBins * 4, device, ready);
    if (s != DTE_OK) return s;
    const unsigned ranges = (q.rows + g.bins - 1) / g.bins;
    const size_t smem = (size_t)g.warps * g.bins * 4;
    if (after) {
        DTE_CUDA(launch_after(group_kernel, dim3(ranges), kGroupThreads, smem, st, g));
    } else {
        group_kernel<<<ranges, kGroupThreads, smem, st>>>(g);
        DTE_CUDA(cudaGetLastError());
    }
    SumParams p = {};
    p.first = g.first;
    p.key = g.key;
    p.pos = g.pos;
    p.rows = q.rows;
    p.hidden = q.hidden;
    p.chunks = (uint32_t)chunks;
    p.block = block;
    p.src = q.src;
    p.src_ld = q.src_ld;
    p.weight = q.weight;
    p.scale = q.scale;
    p.out = q.out;
    p.out_ld = q.out_ld;
    p.accumulate = q.accumulate;
    p.compact = q.compact;
    p.partial = reinterpret_cast<float*>(ws + l.partial);
    p.counters = g.counters;
    if (!q.compact && !q.accumulate) {
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
    const unsigned ctas = (unsigned)((blocks * chunks + kSumThreads / 32 - 1) / (kSumThreads / 32));
    const bool sb = q.src_dtype == DTE_BF16, ob = q.out_dtype == DTE_BF16;
    if (p.weight) return launch_sums<__nv_bfloat16, float, true>(p, vec, ctas, st);       // the head's gradient
    if (sb && ob) return launch_sums<__nv_bfloat16, __nv_bfloat16>(p, vec, ctas, st);
    if (sb) return launch_sums<__nv_bfloat16, float>(p, vec, ctas, st);
    if (ob) return launch_sums<float, __nv_bfloat16>(p, vec, ctas, st);
    return launch_sums<float, float>(p, vec, ctas, st);
}

dte_status device_sms(int device, int* sms) {
    static std::atomic<int> known[kMaxDevices];
    if (device < 0 || device >= kMaxDevices) return op_fail(DTE_ERR_INVALID_ARG, "device ordinal out of range");
    int v = known[device].load(std::memory_order_relaxed);
    if (!v) {
        int count = 0;
        DTE_CUDA(cudaGetDeviceCount(&count));
        if (device >= count) return op_fail(DTE_ERR_INVALID_ARG, "there is no such CUDA device");
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
    if (!std::isfinite((float)scale)) return op_fail(DTE_ERR_INVALID_ARG, "scale is not finite in fp32");
    if (table->cols != out->cols || out->rows != ids->count)
        return op_fail(DTE_ERR_INVALID_ARG, "out must be ids.count x table.cols");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if (ids->count == 0) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    const int vec = vec_of(table, out);
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
    const uint64_t span = 32 * kLookupUnroll * vec;
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

// The workspace helper does not know the table: it leaves room for the row index of the largest one (8 MB).
constexpr uint64_t kMaxTableRows = (1u << 21) - 1;

extern "C" uint64_t dte_embedding_backward_workspace_bytes(uint64_t n_ids, uint64_t hidden) {
    if (n_ids >= kMaxDim || hidden >= kMaxDim) return UINT64_MAX;   // refused by the call
    return sorted_sum_workspace_bytes(n_ids, kMaxTableRows, hidden);
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
    if (!std::isfinite((float)scale)) return op_fail(DTE_ERR_INVALID_ARG, "scale is not finite in fp32");
    if (dtable->cols != dout->cols || dout->rows != ids->count)
        return op_fail(DTE_ERR_INVALID_ARG, "dout must be ids.count x dtable.cols");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if ((s = check_workspace(workspace, workspace_bytes, sorted_sum_workspace_bytes(ids->count, kMaxTableRows, dout->cols))) != DTE_OK) return s;
    const int vec = vec_of(dout, dtable);
    if (dtable->rows > kMaxTableRows) return op_fail(DTE_ERR_INVALID_ARG, "at most 2097151 rows of a table");
    if (!sorted_sum_fits(ids->count, dtable->rows, dout->cols, dtable->dtype))
        return op_fail(DTE_ERR_INVALID_ARG, "ids.count x hidden or dtable is too large for one call");
    if (dtable->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
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
    return launch_sorted_sum(q, vec, workspace, false, device, (cudaStream_t)cuda_stream);
}
