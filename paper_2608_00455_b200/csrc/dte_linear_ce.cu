// Softmax cross entropy of a linear head over a large vocabulary, without storing the logits, and its
// gradient.  z = s x W^T;  lse = log sum_v exp z_v;  with p = exp(z - lse), f = s * dloss:
//   dx = (f p') W + c W[target],   dW = (f p')^T x + (rows of c x, added up by target),
// where p' is p with 0 in the target's column and c = f (p_target - 1) = f expm1(z_target - lse).
//
// Bound by the tensor cores (2 tokens V hidden operations forward, 6 backward: the logits are made
// again rather than kept) for more than a few hundred tokens, by reading W for a few.  One persistent
// tcgen05 kernel serves all four products; what differs is how its operands lie in memory and what its
// epilogue does with a finished tile of accumulators:
//   kLse   logits tile -> per row the maximum and the sum of exponentials of its columns (registers only)
//   kProb  logits tile -> f p' as bf16, for one piece of the vocabulary
//   kDx    piece of f p' times W: adds to fp32 sums over pieces
//   kDw    (f p')^T x: complete for the piece's vocabulary rows, the target term added, rounded and written
// Tokens without a target are dropped before the first product: the rows that count are copied together,
// so prompts cost nothing and what their rows hold (NaN included) reaches no sum.  The target's column stays out
// of the bf16 operand and has its whole coefficient c in fp32.  For p_target near 0, c is the largest entry of
// its row by far and its rounding would be most of the gradient's error; for p_target near 1, c is what is left of two
// nearly equal numbers, so neither of them may be rounded first.  z_target is an fp32 sum for the same
// reason; an error of c beyond fp32's relative one comes from the lse that is passed in: 2^-24 |lse| f at most.
//
// Measured: logits 8192 x 151936 x 4096 7.6 to 7.9 ms = 1.28 to 1.34 PFLOP/s in a loop of seconds at the 1000 W limit (a
// bf16 library product of that shape, which stores its logits: 7.4 ms); the backward pass 24.1 to 24.5 ms = 1.25 to 1.27
// PFLOP/s over its three products; with zero operands, which the power limit does not slow, kProb has its tensor cores
// active 93 % of the time.  8 tokens: kLse reads W at 6.4 TB/s.  64 tokens x 151936 x 4096, gradients: kProb 221, kDx 183, kDw 467
// us, where W and dW are 190 us of memory each: up to 128 tokens there is one piece, so kDx finds nothing of W in L2, and
// kDw's tiles have one or two steps along K, so its epilogue sets the pace.
// The tensor cores truncate: log-sum-exps are good to 5e-7 (8 tokens) and 9e-7 (8192), relative, sums in fp32 to 2e-7 and 6e-7.
#include <atomic>

#include "dte_mma.cuh"
#include "dte_ops.cuh"

namespace dte {

enum CeKind { kLse = 0, kProb = 1, kDx = 2, kDw = 3 };

constexpr uint32_t kTileM = 128;                 // accumulator rows of one CTA: the 128 lanes of tensor memory
constexpr uint32_t kTileK = 64;                  // 128 bytes of bf16: one swizzle row
constexpr uint32_t kMaxTileN = 256;
constexpr uint32_t kEpilogueWarps = 8;           // two for each quarter of tensor memory's lanes, half a tile's columns each
constexpr uint32_t kCeThreads = 64 + 32 * kEpilogueWarps;   // TMA warp, MMA warp, epilogue
constexpr uint32_t kStageBytesA = kTileM * kTileK * 2;
constexpr uint32_t kTmemColumns = 512;           // two accumulator tiles: one is filled while the other is drained
// Up to this many tokens (ignored ones included: the host does not know how many those are) half of a tile's rows are free, and
// so f p' is kept as two bf16 numbers, the rounded value and the rest, as if every token were there twice: of a few tokens,
// whose roundings do not average out, f p' is stored to 2^-16 for nothing.  p itself is as good as the tensor cores'
// logits: 4e-6 of a logit at 4096 products.
constexpr uint32_t kSplitTokens = 64;
constexpr uint64_t kPadRows = 256;               // token rows are padded to this, with zero rows
constexpr double kLog2eD = 1.44269504088896340736;
constexpr float kLog2e = (float)kLog2eD;
constexpr float kLn2 = 0.69314718055994530942f;
// Work is split for this many SMs whatever the device has, so that results do not depend on it.
constexpr uint32_t kSplitSms = 148;

// The two matrices that this file makes itself, the rows that count and f p', are stored in blocks of 64 x 64, row-major
// inside (8 KB, 128 bytes a row: the swizzled operand tile as TMA writes it).  Every load of them is then 8 KB
// in one stretch, whether the tile is wanted along its rows or its columns, and one tensor map serves both.
constexpr uint32_t kBlock = 64;
__device__ __forceinline__ uint64_t blocked(uint32_t row, uint32_t col, uint32_t blocks) {
    return ((uint64_t)(row / kBlock) * blocks + col / kBlock) * (kBlock * kBlock) + (row % kBlock) * kBlock + col % kBlock;
}

template <int CTAS>
struct CeStage {
    static constexpr uint32_t kBytesB = kMaxTileN / CTAS * kTileK * 2;
    static constexpr uint32_t kBytes = kStageBytesA + kBytesB;
    static constexpr uint32_t kStages = 196608 / kBytes;
    static constexpr uint32_t kSmem = kStages * kBytes + 1024 + 256;
};

struct CeParams {
    uint32_t m, n, k;            // extents; the one that counts tokens is replaced by *tokens
    const uint32_t* tokens;      // tokens that count
    uint32_t tile_n, splits;
    uint32_t prob_blocks;        // blocks of 64 columns in a row of the blocked f p'
    bool w_chunks;               // kDx: W is mapped as chunks of 64 columns (hidden a multiple of 64)
    uint32_t w_row;              // first row of W of this piece
    uint32_t wait_limit;         // tries of a wait inside the kernel
    uint64_t* flags;
    // kLse, kProb
    float k2;                    // logit_scale * log2(e): accumulators -> base-2 exponents
    float scale;
    const int32_t* target;       // row of this shard, or -1
    float2* stats;               // kLse: (maximum, sum) per tile of columns and token
    uint64_t stats_ld;
    float* target_logit;         // kLse: the target's logit as the tensor cores added it up
    bool split;                  // kProb: the upper kSplitTokens rows hold what rounding to bf16 took from the lower ones
    const float* f;              // kProb: logit_scale * dloss per token (the target's column gets 0, see `target`)
    const float* neg_lse2;       //        -lse * log2(e)
    __nv_bfloat16* prob;         //        blocked, prob_blocks blocks wide
    // kDx
    float* dx_sum;               // splits x padded tokens x hidden
    uint64_t dx_split;           // elements of one split's part
    bool add;
    // kDw
    void* dweight;
    uint64_t dweight_ld;
    bool dweight_bf16, accumulate;
    bool whole_sectors;          // every group of 32 bytes of a row of dweight starts on a sector
    const uint32_t* first;       // per vocabulary row: where its target term lies, if the next row's lies further on
    const float* target_sum;
};

// Position of a tile in the order in which CTAs take them: groups of `group` rows of tiles, and inside a
// group the row index runs fastest, so that the CTAs at work share few rows and few columns in L2.
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t group, uint32_t* split,
                                        uint32_t* tm, uint32_t* tn) {
    const uint32_t per_split = tiles_m * tiles_n;
    *split = t / per_split;
    t -= *split * per_split;
    const uint32_t g = t / (group * tiles_n);
    t -= g * group * tiles_n;
    const uint32_t rows = min(group, tiles_m - g * group);
    *tm = g * group + t % rows;
    *tn = t / rows;
}

__device__ __forceinline__ void load_tile(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    tmem_load32(addr, r);
    tmem_load_wait(r);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// o += the (up to) four groups of 8 columns at d
template <typename T>
__device__ __forceinline__ void add_old(const T* d, uint32_t groups, float (&o)[32]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (groups <= (uint32_t)j) break;
        Raw8<T> r;
        float old[8];
        r.load(d + 8 * j);
        r.get(old);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[8 * j + i] += old[i];
    }
}

// The 128 columns from c0 (half a tile) of row `row`; lane_row: the row within the CTA's 128.
template <int KIND>
__device__ __forceinline__ void ce_epilogue(const CeParams& p, uint32_t tmem, uint32_t row, uint32_t lane_row, uint32_t half, uint32_t buf,
                                            uint32_t tn, uint32_t split, uint32_t tokens, bool empty, float2 (*s_stat)[kTileM]) {
    const uint32_t n0 = tn * p.tile_n, c0 = half * (kMaxTileN / 2), c1 = min(c0 + kMaxTileN / 2, p.tile_n);
    if (KIND == kLse) {
        const bool valid = row < tokens;
        const int64_t tcol = valid ? (int64_t)p.target[row] - n0 : -1;
        float top = -INFINITY, sum = 0.f;
        for (uint32_t c = c0; c < c1; c += 32) {
            if (n0 + c >= p.n) break;
            float v[32];
            load_tile(tmem + c, v);
            const uint32_t left = min(p.n - (n0 + c), c1 - c);      // a tile is a multiple of 16 columns wide
            const bool mine = tcol >= (int64_t)c && tcol < (int64_t)c + 32 && tcol < (int64_t)(c + left);
            if (__any_sync(0xFFFFFFFFu, mine)) {
                float at = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) at = tcol == (int64_t)(c + j) ? v[j] : at;
                if (mine) p.target_logit[row] = at * p.scale;
            }
            if (left < 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j >= (int)left) v[j] = -INFINITY;
            }
            float peak = fmaxf(v[0], v[1]);
#pragma unroll
            for (int j = 2; j < 32; j += 2) peak = fmaxf(peak, fmaxf(v[j], v[j + 1]));
            const float now = fmaxf(top, peak * p.k2);
            // nothing but -inf so far: keep the exponents at -inf instead of forming inf - inf
            const float from = now == -INFINITY ? 0.f : now;
            float part = 0.f, part2 = 0.f;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                part += exp2_fast(fmaf(v[j], p.k2, -from));
                part2 += exp2_fast(fmaf(v[j + 1], p.k2, -from));
            }
            sum = fmaf(sum, exp2_fast(top - from), part + part2);
            top = now;
        }
        // the two halves of a row meet in shared memory (two buffers: the next tile may begin before this one is read)
        if (half) s_stat[buf][lane_row] = make_float2(top, sum);
        asm volatile("bar.sync %0, 64;" ::"r"(1 + lane_row / 32) : "memory");
        if (!half && valid) {
            const float2 o = s_stat[buf][lane_row];
            const float now = fmaxf(top, o.x), from = now == -INFINITY ? 0.f : now;
            p.stats[(uint64_t)tn * p.stats_ld + row] = make_float2(now, sum * exp2_fast(top - from) + o.y * exp2_fast(o.x - from));
        }
    } else if (KIND == kProb) {
        const float f = p.f[row], nl = p.neg_lse2[row];     // zero for padding rows
        // the target's column, counted from the tile's first one; of no tile's columns where it is another piece's
        const int32_t tcol = row < tokens ? p.target[p.split ? row % kSplitTokens : row] - (int32_t)(p.w_row + n0) : -1;
        for (uint32_t c = c0; c < c1; c += 32) {
            float v[32];
            load_tile(tmem + c, v);
            const uint32_t left = p.n > n0 + c ? p.n - (n0 + c) : 0;
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = f * exp2_fast(fmaf(v[j], p.k2, nl));
            const uint32_t at = (uint32_t)(tcol - (int32_t)c);
            if (__any_sync(0xFFFFFFFFu, at < 32)) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = at == (uint32_t)j ? 0.f : v[j];
            }
            if (left < 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j >= (int)left) v[j] = 0.f;
            }
            if (p.split && row >= kSplitTokens) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
            }
#pragma unroll
            for (int j = 0; j < 32; j += 16) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = row < tokens ? pack_bf16(v[j + 2 * i], v[j + 2 * i + 1]) : 0u;
                store32(p.prob + blocked(row, n0 + c + j, p.prob_blocks), w);
            }
        }
    } else if (KIND == kDx) {
        float* out = p.dx_sum + split * p.dx_split + (uint64_t)row * p.n + n0;
        const bool add = p.add && row < tokens;
        for (uint32_t c = c0; c < c1; c += 32) {
            if (n0 + c >= p.n) break;
            uint32_t old[4][8];
            if (add) {                                      // in flight while the tile is read
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (n0 + c + 8 * j < p.n) load32(out + c + 8 * j, old[j]);
            }
            float v[32];
            load_tile(tmem + c, v);
            if (row < tokens) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (n0 + c + 8 * j >= p.n) break;
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float x = empty ? 0.f : v[8 * j + i];
                        if (add) x += __uint_as_float(old[j][i]);
                        w[i] = __float_as_uint(x);
                    }
                    store32(out + c + 8 * j, w);
                }
            }
        }
    } else {
        const uint64_t vrow = (uint64_t)p.w_row + row;
        const bool valid = row < p.m;
        const uint32_t at = valid ? p.first[vrow] : 0;
        const bool hit = valid && p.first[vrow + 1] > at;   // a token has this row as its target
        const float* term = p.target_sum + (uint64_t)(hit ? at : 0) * p.n + n0;
        // few rows are hit, but most warps hold one: its terms are loaded a step ahead
        uint32_t w[4][8], ahead[4][8];
        auto fetch = [&](uint32_t c, uint32_t (&to)[4][8]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int i = 0; i < 8; ++i) to[j][i] = 0u;
                if (hit && c < c1 && n0 + c + 8 * j < p.n) load32(term + c + 8 * j, to[j]);
            }
        };
        fetch(c0, ahead);
        for (uint32_t c = c0; c < c1; c += 32) {
            if (n0 + c >= p.n) break;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[j][i] = ahead[j][i];
            fetch(c + 32, ahead);
            float v[32];
            load_tile(tmem + c, v);
            if (!valid) continue;
            const uint64_t off = vrow * p.dweight_ld + n0 + c;
            const uint32_t left = (p.n - (n0 + c)) / 8;      // groups of 8 columns
            float o[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = (empty ? 0.f : v[j]) + __uint_as_float(w[j / 8][j % 8]);
            if (p.dweight_bf16) {
                __nv_bfloat16* d = static_cast<__nv_bfloat16*>(p.dweight) + off;
                if (p.accumulate) add_old(d, left, o);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t q[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = pack_bf16(o[16 * j + 2 * i], o[16 * j + 2 * i + 1]);
                    if (p.whole_sectors && left >= 2u * j + 2) {
                        store32(d + 16 * j, q);
                    } else {
                        uint4* e = reinterpret_cast<uint4*>(d + 16 * j);
                        if (left > 2u * j) e[0] = make_uint4(q[0], q[1], q[2], q[3]);
                        if (left > 2u * j + 1) e[1] = make_uint4(q[4], q[5], q[6], q[7]);
                    }
                }
            } else {
                float* d = static_cast<float*>(p.dweight) + off;
                if (p.accumulate) add_old(d, left, o);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (left <= (uint32_t)j) break;
                    uint32_t q[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(o[8 * j + i]);
                    if (p.whole_sectors) {
                        store32(d + 8 * j, q);
                    } else {
                        uint4* e = reinterpret_cast<uint4*>(d + 8 * j);
                        e[0] = make_uint4(q[0], q[1], q[2], q[3]);
                        e[1] = make_uint4(q[4], q[5], q[6], q[7]);
                    }
                }
            }
        }
    }
}

// One CTA (CTAS == 1) or a pair of CTAs on neighbouring SMs (CTAS == 2) per tile of 128 * CTAS rows.  Of a
// pair, each CTA holds its own 128 rows of A and half of B; the leader's MMA reads both halves, so every byte
// of B is loaded and stored once per pair.  Barriers: full (leader: both CTAs' loads), empty (each: the stage
// has been multiplied), done (each: the tile's accumulators are complete), drained (leader: both CTAs'
// epilogues have read them).
template <int KIND, int CTAS>
__global__ void __launch_bounds__(kCeThreads, 1)
    ce_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CeParams p) {
    using S = CeStage<CTAS>;
    constexpr bool kAmn = KIND == kDw, kBmn = KIND == kDx || KIND == kDw;
    extern __shared__ uint8_t ce_smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[2 * S::kStages + 5];
    __shared__ uint32_t s_tmem, s_gave_up, s_issued, s_taken;      // loads asked for; loads that the products have waited for
    __shared__ uint32_t s_peer[2];                                 // the other CTA's s_gave_up and s_issued
    __shared__ uint32_t s_ok[2][2][4];
    __shared__ float2 s_stat[KIND == kLse ? 2 : 1][kTileM];

    const uint32_t stage0 = (smem_addr(ce_smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_addr(s_bar);
    auto full = [&](uint32_t i) { return bar0 + 8 * i; };
    auto empty = [&](uint32_t i) { return bar0 + 8 * (S::kStages + i); };
    auto done = [&](uint32_t i) { return bar0 + 8 * (2 * S::kStages + i); };
    auto drained = [&](uint32_t i) { return bar0 + 8 * (2 * S::kStages + 2 + i); };
    const uint32_t last_bar = bar0 + 8 * (2 * S::kStages + 4);
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t rank = CTAS == 2 ? cluster_rank() : 0;
    const bool leader = rank == 0;

    let_next_start();      // the next kernel sets up its barriers and tensor memory on the SMs that this one leaves first
    if (threadIdx.x == 0) {
        tma_prefetch_map(&map_a);
        tma_prefetch_map(&map_b);
        for (uint32_t i = 0; i < S::kStages; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(done(i), 1);
            mbar_init(drained(i), kEpilogueWarps * CTAS);
        }
        mbar_init(last_bar, 1);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CTAS>(smem_addr(&s_tmem), kTmemColumns);
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();
    tc_fence_after();
    wait_for_earlier();
    const uint32_t tmem = *(volatile uint32_t*)&s_tmem;
    volatile uint32_t* gave_up = &s_gave_up;

    const uint32_t tokens = *p.tokens;
    const uint32_t m = KIND == kDw ? p.m : tokens, k = KIND == kDw ? tokens : p.k;
    const uint32_t tiles_m = (m + kTileM * CTAS - 1) / (kTileM * CTAS), tiles_n = (p.n + p.tile_n - 1) / p.tile_n;
    const uint32_t total = tiles_m * tiles_n * p.splits;
    const uint32_t group = 16 / CTAS;
    const uint32_t blocks_k = (k + kTileK - 1) / kTileK;
    const uint32_t first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
    const uint32_t part_n = p.tile_n / CTAS;             // columns of B in this CTA
    const uint32_t load_bytes = kStageBytesA + part_n * kTileK * 2;      // of this CTA per stage

    if (warp == 0 && lane == 0) {
        // ---- loads ----
        uint32_t stage = 0, phase = 0, issued = 0;
        bool ok = true;
        for (uint32_t t = first; t < total && ok; t += step) {
            uint32_t split, tm, tn;
            tile_at(t, tiles_m, tiles_n, group, &split, &tm, &tn);
            const uint32_t m0 = (tm * CTAS + rank) * kTileM, n0 = tn * p.tile_n + rank * part_n;
            const uint32_t kb0 = (uint32_t)((uint64_t)split * blocks_k / p.splits), kb1 = (uint32_t)((uint64_t)(split + 1) * blocks_k / p.splits);
            for (uint32_t kb = kb0; kb < kb1; ++kb) {
                if (!(ok = mbar_wait(empty(stage), phase ^ 1, p.wait_limit, gave_up))) break;
                const uint32_t a = stage0 + stage * S::kBytes, b = a + kStageBytesA;
                const uint32_t bar = CTAS == 2 ? cluster_map(full(stage), 0) : full(stage);
                if (leader) mbar_expect_tx(full(stage), CTAS * load_bytes);
                const int k0 = (int)(kb * kTileK);
                // One load per operand and stage: with two per operand the loads, not the tensor cores, set the pace of the
                // products along columns (kDw: 74 % of the tensor cores' cycles).  A: blocks of a blocked matrix, two
                // rows of blocks along K, or two neighbours in one row of blocks.
                const int mb = (int)(m0 / kBlock);
                if (kAmn) tma_load_3d<CTAS>(a, &map_a, 0, (int)m0, (int)kb, bar);
                else tma_load_3d<CTAS>(a, &map_a, 0, k0, mb, bar);
                if (KIND == kDw) {
                    tma_load_3d<CTAS>(b, &map_b, 0, (int)n0, (int)kb, bar);
                } else if (KIND == kDx) {
                    if (p.w_chunks) {
                        tma_load_3d<CTAS>(b, &map_b, 0, k0 + (int)p.w_row, (int)(n0 / kBlock), bar);
                    } else {
                        for (uint32_t j = 0; j < part_n; j += 64)
                            tma_load_2d<CTAS>(b + j * kTileK * 2, &map_b, (int)(n0 + j), k0 + (int)p.w_row, bar);
                    }
                } else {
                    tma_load_2d<CTAS>(b, &map_b, k0, (int)(n0 + p.w_row), bar);
                }
                ++issued;
                if (++stage == S::kStages) { stage = 0; phase ^= 1; }
            }
        }
        s_issued = issued;
    } else if (warp == 1 && lane == 0 && leader) {
        // ---- matrix products ----
        const uint32_t desc = mma_desc(kTileM * CTAS, p.tile_n, kAmn, kBmn);
        const uint32_t chunk = kTileK * 128;              // MN-major: 64 columns x 64 k
        uint32_t stage = 0, phase = 0, use = 0, taken = 0;
        bool ok = true;
        for (uint32_t t = first; t < total && ok; t += step, ++use) {
            const uint32_t split = t / (tiles_m * tiles_n);
            const uint32_t kb0 = (uint32_t)((uint64_t)split * blocks_k / p.splits), kb1 = (uint32_t)((uint64_t)(split + 1) * blocks_k / p.splits);
            const uint32_t buf = use & 1, acc = tmem + buf * kMaxTileN;
            if (!(ok = mbar_wait(drained(buf), ((use >> 1) & 1) ^ 1, p.wait_limit, gave_up))) break;
            tc_fence_after();
            for (uint32_t kb = kb0; kb < kb1; ++kb) {
                if (!(ok = mbar_wait(full(stage), phase, p.wait_limit, gave_up))) break;
                ++taken;
                tc_fence_after();
                const uint32_t a = stage0 + stage * S::kBytes, b = a + kStageBytesA;
                uint64_t da = operand_desc(a, kAmn ? chunk : 16), db = operand_desc(b, kBmn ? chunk : 16);
#pragma unroll
                for (uint32_t i = 0; i < kTileK / 16; ++i) {
                    mma_bf16<CTAS>(acc, da, db, desc, kb != kb0 || i != 0);
                    da += kAmn ? 2048 >> 4 : 32 >> 4;      // 16 further along K
                    db += kBmn ? 2048 >> 4 : 32 >> 4;
                }
                mma_commit<CTAS>(empty(stage));
                if (++stage == S::kStages) { stage = 0; phase ^= 1; }
            }
            if (ok) mma_commit<CTAS>(done(buf));
        }
        s_taken = taken;
    } else if (warp >= 2) {
        // ---- epilogue: warp w may read the quarter w % 4 of tensor memory's lanes ----
        const uint32_t quarter = warp & 3, half = (warp - 2) / 4;
        const uint32_t lane_row = quarter * 32 + lane;
        uint32_t use = 0;
        for (uint32_t t = first; t < total; t += step, ++use) {
            uint32_t split, tm, tn;
            tile_at(t, tiles_m, tiles_n, group, &split, &tm, &tn);
            const uint32_t buf = use & 1;
            bool ok = mbar_wait(done(buf), (use >> 1) & 1, p.wait_limit, gave_up);
            ok = !__any_sync(0xFFFFFFFFu, !ok);
            if (KIND == kLse) {
                // the two warps of a quarter go on or stop together: they meet again inside the epilogue
                if (lane == 0) s_ok[buf][half][quarter] = ok;
                asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory");
                ok = s_ok[buf][0][quarter] && s_ok[buf][1][quarter];
            }
            if (!ok) break;
            tc_fence_after();
            const uint32_t kb0 = (uint32_t)((uint64_t)split * blocks_k / p.splits), kb1 = (uint32_t)((uint64_t)(split + 1) * blocks_k / p.splits);
            ce_epilogue<KIND>(p, tmem + buf * kMaxTileN + (quarter * 32 << 16), (tm * CTAS + rank) * kTileM + lane_row, lane_row, half, buf, tn,
                              split, tokens, kb0 == kb1, s_stat);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_map(drained(buf), 0));
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    bool failed = *gave_up;
    if (CTAS == 2) {
        if (threadIdx.x == 0) {
            cluster_store(cluster_map(smem_addr(s_peer), rank ^ 1), *gave_up);
            cluster_store(cluster_map(smem_addr(s_peer + 1), rank ^ 1), s_issued);
        }
        cluster_sync_all();     // the peer may still signal barriers here, or read this CTA's operands
        failed |= *(volatile uint32_t*)s_peer;
    }
    if (failed) {
        // A wait ran out, whichever it was (all threads of the CTA or pair agree).  All roles have stopped; what they left in
        // flight ends here, again with a limit: the products of the thread that issued them, and every load that no product
        // has waited for, before shared and tensor memory go away.
        if (warp == 1 && lane == 0) {
            if (leader) mma_commit<CTAS>(last_bar);
            for (uint32_t i = 0; i < kWaitTries && !mbar_try_wait(last_bar, 0); ++i) {}
        }
        if (threadIdx.x == 0 && leader) {
            const uint32_t peer = CTAS == 2 ? *(volatile uint32_t*)(s_peer + 1) : 0, most = max(s_issued, peer);
            uint32_t left = kWaitTries;
            for (uint32_t i = s_taken; i < most; ++i) {
                if (i >= s_issued) mbar_expect_tx(full(i % S::kStages), load_bytes);      // a load of the peer's alone
                while (left && !mbar_try_wait(full(i % S::kStages), (i / S::kStages) & 1)) --left;
            }
        }
        __syncwarp();
        if (CTAS == 2) cluster_sync_all(); else __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) tmem_free<CTAS>(tmem, kTmemColumns);
    if (threadIdx.x == 0 && failed && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_TIMEOUT);
}

// ---- before and after the products --------------------------------------------------------------------------
struct RowsParams {
    const void* targets;
    uint32_t targets_dtype, n;
    int64_t vocab_start, vocab;
    uint32_t vocab_rows;
    uint32_t* count;         // [0] tokens that count, [1] rows of the backward products
    bool split;              // [1] is twice kSplitTokens, if any token counts
    int32_t* source;         // [i] = token of compact row i
    int32_t* target;         // [i] = its target as a row of this shard, or -1
    int32_t* place;          // [token] = compact row or -1 (NULL: not wanted)
    float *lse, *target_logit, *loss;   // forward: zero for ignored tokens
    uint64_t* flags;
};

constexpr int kRowsThreads = 1024;
constexpr int kRowsPer = 8;      // consecutive tokens of a thread

// One round of a CTA of THREADS threads, each with the kRowsPer tokens from i0 + threadIdx.x * kRowsPer: their targets (-1 past the
// end), how many tokens of the round that count lie in front of this thread's, and (returned) how many there are.
// s_warp may be written again behind the next barrier.
template <int THREADS>
__device__ __forceinline__ uint32_t count_tokens(const RowsParams& p, uint64_t i0, int64_t (&id)[kRowsPer], uint32_t& before, bool& bad,
                                                 uint32_t (&s_warp)[THREADS / 32]) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < kRowsPer; ++j) {
        const uint64_t i = i0 + threadIdx.x * kRowsPer + j;
        id[j] = i < p.n ? load_id(p.targets, p.targets_dtype, i) : -1;
    }
#pragma unroll
    for (int j = 0; j < kRowsPer; ++j) {
        mine += id[j] >= 0;
        bad |= id[j] >= p.vocab;
    }
    uint32_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= (uint32_t)o) inc += v;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    before = inc - mine;
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        before += w < (int)warp ? s_warp[w] : 0;
        all += s_warp[w];
    }
    return all;
}

// A target as a row of this shard, or -1.
__device__ __forceinline__ int32_t shard_row(const RowsParams& p, int64_t id) {
    const uint64_t row = (uint64_t)id - (uint64_t)p.vocab_start;
    return id >= 0 && row < p.vocab_rows ? (int32_t)row : -1;
}

// Leaves what the kernels behind need of token i, the at-th that counts if it does.
__device__ __forceinline__ void leave_token(const RowsParams& p, uint64_t i, int64_t id, uint32_t at) {
    if (p.place) p.place[i] = id >= 0 ? (int32_t)at : -1;
    if (id >= 0) {
        p.source[at] = (int32_t)i;
        p.target[at] = shard_row(p, id);
    } else {
        if (p.lse) p.lse[i] = 0.f;
        if (p.target_logit) p.target_logit[i] = 0.f;
        if (p.loss) p.loss[i] = 0.f;
    }
}

// Numbers the tokens that count, in order.  One CTA: the list is short next to everything else.
__global__ void __launch_bounds__(kRowsThreads) ce_rows_kernel(const RowsParams p) {
    __shared__ uint32_t s_warp[kRowsThreads / 32];
    let_next_start();
    uint32_t base = 0;
    bool bad = false;
    for (uint64_t i0 = 0; i0 < p.n; i0 += kRowsThreads * kRowsPer) {
        int64_t id[kRowsPer];
        uint32_t at;
        const uint32_t all = count_tokens<kRowsThreads>(p, i0, id, at, bad, s_warp);
        at += base;
#pragma unroll
        for (int j = 0; j < kRowsPer; ++j) {
            const uint64_t i = i0 + threadIdx.x * kRowsPer + j;
            if (i >= p.n) break;
            leave_token(p, i, id[j], at);
            at += id[j] >= 0;
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) p.count[0] = p.count[1] = base;
    if (bad && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
}

struct GatherRowsParams {
    uint32_t* count;
    int32_t* source;
    RowsParams rows_of;      // few tokens: every CTA numbers them itself (see kFewTokens)
    bool few;
    const __nv_bfloat16* x;
    uint64_t x_ld;
    uint32_t hidden;
    bool vec;
    __nv_bfloat16* rows;     // blocked: padded tokens x blocks of 64
    uint32_t blocks;
    // the target's logit is added up in fp32 here
    int32_t* target;
    const __nv_bfloat16* weight;
    uint64_t weight_ld;
    // forward (compact order)
    float* exact_logit;      // the target's logit
    float* target_logit;     // the same as the tensor cores add it up later; cleared
    // backward
    float* coef;             // [token] = f (p_target - 1), of tokens whose target is in this shard
    const float* dloss;
    const float* lse;
    float scale;
    float* f;
    float* neg_lse2;
};

// Up to this many tokens every CTA of ce_gather_kernel numbers the tokens for itself, which takes it a microsecond
// and saves the launch of ce_rows_kernel in front of it.
constexpr int kGatherThreads = 256;
constexpr uint32_t kFewTokens = kGatherThreads * kRowsPer;

// Copies the rows that count together and clears the padding rows up to the next multiple of kPadRows.
__global__ void __launch_bounds__(kGatherThreads) ce_gather_kernel(const GatherRowsParams p) {
    __shared__ float s_part[kGatherThreads / 32];
    __shared__ uint32_t s_warp[kGatherThreads / 32];
    __shared__ int32_t s_mine[2];          // token and target of this CTA's row
    wait_for_earlier();
    let_next_start();
    const bool split = p.rows_of.split;               // only with few tokens
    const uint32_t i = blockIdx.x, mine_at = split && i < 2 * kSplitTokens ? i % kSplitTokens : i;
    uint32_t count, src;
    int32_t target;
    if (p.few) {
        const RowsParams& q = p.rows_of;
        int64_t id[kRowsPer];
        uint32_t at;
        bool bad = false;
        if (threadIdx.x < 2) s_mine[threadIdx.x] = threadIdx.x ? -1 : 0;
        count = count_tokens<kGatherThreads>(q, 0, id, at, bad, s_warp);
        const bool writer = i == 0;        // one CTA leaves the numbering for the kernels behind
#pragma unroll
        for (int j = 0; j < kRowsPer; ++j) {
            const uint32_t t = threadIdx.x * kRowsPer + j;
            if (t >= q.n) break;
            if (id[j] >= 0 && at == mine_at) {
                s_mine[0] = (int32_t)t;
                s_mine[1] = shard_row(q, id[j]);
            }
            if (writer) leave_token(q, t, id[j], at);
            at += id[j] >= 0;
        }
        if (writer) {
            if (threadIdx.x == 0) {
                q.count[0] = count;
                q.count[1] = split && count ? 2 * kSplitTokens : count;
            }
            if (bad && q.flags) atomicOr((unsigned long long*)q.flags, (unsigned long long)DTE_DEV_BOUNDS);
        }
        __syncthreads();
        src = (uint32_t)s_mine[0];
        target = s_mine[1];
    } else {
        count = *p.count;
        src = i < count ? (uint32_t)p.source[i] : 0;
        target = i < count ? p.target[i] : -1;
    }
    const uint32_t padded = (uint32_t)((count + kPadRows - 1) / kPadRows * kPadRows);
    if (i >= padded) return;
    const bool live = mine_at < count;
    if (mine_at != i) target = -1;       // the second row of a token that is there twice
    const __nv_bfloat16* in = p.x + (uint64_t)src * p.x_ld;
    float dot = 0.f;
    for (uint32_t c = threadIdx.x * 8; c < p.blocks * kBlock; c += kGatherThreads * 8) {
        Raw8<__nv_bfloat16> r, w;
        if (c >= p.hidden) {             // the last block's columns past the row: zeros, they meet zeros of W
            r.zero();
            r.store(p.rows + blocked(i, c, p.blocks));
            continue;
        }
        if (target >= 0) w.load(p.weight + (uint64_t)target * p.weight_ld + c);
        float f[8];
        if (!live) {
            r.zero();
        } else if (p.vec) {
            r.load(in + c);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = to_f(in[c + j]);
            r.set(f);
        }
        r.store(p.rows + blocked(i, c, p.blocks));
        if (target >= 0) {
            float g[8];
            r.get(f);
            w.get(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = fmaf(f[j], g[j], dot);
        }
    }
    if (target >= 0) {                   // the same for the whole CTA
        dot = warp_sum(dot);
        if ((threadIdx.x & 31) == 0) s_part[threadIdx.x / 32] = dot;
        __syncthreads();
    }
    if (threadIdx.x) return;
    float logit = 0.f;
    if (target >= 0) {
#pragma unroll
        for (int w = 1; w < kGatherThreads / 32; ++w) dot += s_part[w];
        logit = dot * p.scale;
    }
    if (p.exact_logit) {
        p.exact_logit[i] = logit;
        p.target_logit[i] = 0.f;
    } else {
        const float f = live ? p.scale * p.dloss[src] : 0.f, lse = live ? p.lse[src] : 0.f;
        p.f[i] = f;
        p.neg_lse2[i] = -lse * kLog2e;
        if (target >= 0) p.coef[src] = f * expm1f(logit - lse);
    }
}

struct CombineParams {
    const uint32_t* count;
    const int32_t* source;
    const int32_t* target;
    const float2* stats;
    uint64_t stats_ld;
    uint32_t tiles;
    const float* row_target_logit;
    const float* exact_logit;
    float *lse, *target_logit, *loss;
};

constexpr int kCombineRows = 8;      // tokens of a CTA: their statistics of one tile fill two sectors
constexpr int kCombineThreads = 1024;

// log-sum-exp of a token from its tiles' statistics.  The tensor cores add a logit's products up with
// truncation (4e-6 of its size at 4096 products), which matters for one logit, the target's: it is taken from the
// fp32 sum, and lse is moved by what that changes in the sum of exponentials, so that a loss near zero stays exact.
__global__ void __launch_bounds__(kCombineThreads) ce_combine_kernel(const CombineParams p) {
    __shared__ float s_top[kCombineThreads / 32][kCombineRows], s_sum[kCombineThreads / 32][kCombineRows];
    wait_for_earlier();
    const uint32_t count = *p.count, r = threadIdx.x % kCombineRows, part = threadIdx.x / kCombineRows;
    constexpr uint32_t kParts = kCombineThreads / kCombineRows;
    const uint32_t i = blockIdx.x * kCombineRows + r;
    if (blockIdx.x * kCombineRows >= count) return;
    auto join = [](float& top, float& sum, float t2, float s2) {
        const float now = fmaxf(top, t2), from = now == -INFINITY ? 0.f : now;
        sum = sum * exp2_fast(top - from) + s2 * exp2_fast(t2 - from);
        top = now;
    };
    // what the last step needs, asked for before the statistics
    constexpr uint32_t kWarps = kCombineThreads / 32;      // then: kWarps lanes per row
    const uint32_t row = blockIdx.x * kCombineRows + threadIdx.x / kWarps;
    const bool writer = threadIdx.x < kCombineRows * kWarps && threadIdx.x % kWarps == 0 && row < count;
    const float made = writer ? p.row_target_logit[row] : 0.f, exact = writer ? p.exact_logit[row] : 0.f;
    const uint32_t n = writer ? (uint32_t)p.source[row] : 0;
    const bool here = writer && p.target[row] >= 0;
    float top = -INFINITY, sum = 0.f;
    if (i < count) {
#pragma unroll 8
        for (uint32_t t = part; t < p.tiles; t += kParts) {
            const float2 v = p.stats[(uint64_t)t * p.stats_ld + i];
            join(top, sum, v.x, v.y);
        }
    }
#pragma unroll
    for (int o = kCombineRows; o < 32; o <<= 1) {
        const float t2 = __shfl_xor_sync(0xFFFFFFFFu, top, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        join(top, sum, t2, s2);
    }
    if ((threadIdx.x & 31) < kCombineRows) {
        s_top[threadIdx.x / 32][r] = top;
        s_sum[threadIdx.x / 32][r] = sum;
    }
    __syncthreads();
    if (threadIdx.x >= kCombineRows * kWarps) return;
    top = s_top[threadIdx.x % kWarps][threadIdx.x / kWarps];
    sum = s_sum[threadIdx.x % kWarps][threadIdx.x / kWarps];
#pragma unroll
    for (int o = kWarps / 2; o; o /= 2) {
        const float t2 = __shfl_xor_sync(0xFFFFFFFFu, top, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        join(top, sum, t2, s2);
    }
    if (writer) {
        float lse = (top + log2f(sum)) * kLn2;
        if (here && made != exact) {
            const float move = exp2_fast((made - lse) * kLog2e) * expm1f(exact - made);
            if (fabsf(move) < 0.5f) lse += log1pf(move);      // else the logits are not finite or beyond fp32's reach
        }
        p.lse[n] = lse;
        if (p.target_logit) p.target_logit[n] = exact;
        if (p.loss) p.loss[n] = lse - exact;
    }
}

struct DxParams {
    const int32_t* place;
    const int32_t* target;
    const float* coef;       // [token], see GatherRowsParams
    const float* sums;
    uint64_t split_elems;
    uint32_t splits, hidden;
    bool split;              // kProb's: two rows per token
    const __nv_bfloat16* weight;
    uint64_t weight_ld;
    __nv_bfloat16* dx;
    uint64_t dx_ld;
};

// dx of every token: its splits' sums and the target's row; zero for ignored tokens.
__global__ void __launch_bounds__(256) ce_dx_kernel(const DxParams p) {
    wait_for_earlier();
    const int32_t i = p.place[blockIdx.x];
    __nv_bfloat16* out = p.dx + (uint64_t)blockIdx.x * p.dx_ld;
    const int32_t target = i >= 0 ? p.target[i] : -1;
    const float coef = target >= 0 ? p.coef[blockIdx.x] : 0.f;
    for (uint32_t c = threadIdx.x * 8; c < p.hidden; c += 256 * 8) {
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (i >= 0) {
            for (uint32_t s = 0; s < p.splits; ++s) {
                Raw8<float> r;
                float v[8];
                r.load(p.sums + s * p.split_elems + (uint64_t)i * p.hidden + c);
                r.get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += v[j];
                if (p.split) {
                    r.load(p.sums + s * p.split_elems + (uint64_t)(i + kSplitTokens) * p.hidden + c);
                    r.get(v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] += v[j];
                }
            }
            if (target >= 0) {
                Raw8<__nv_bfloat16> r;
                float w[8];
                r.load(p.weight + (uint64_t)target * p.weight_ld + c);
                r.get(w);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = fmaf(coef, w[j], o[j]);
            }
        }
        Raw8<__nv_bfloat16> r;
        r.set(o);
        r.store(out + c);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------
static int pair_of(uint64_t tokens) { return tokens > kTileM ? 2 : 1; }

struct CeShape {
    uint64_t padded, piece, pieces;
    int ctas;
    uint32_t splits;       // of kDx's long axis
};

constexpr uint64_t kProbBytes = 256ull << 20;    // f p' of one piece
constexpr uint64_t kMinPiece = 2048;

static CeShape ce_shape(uint64_t tokens, uint64_t vocab, uint64_t hidden, uint64_t prob_bytes) {
    CeShape s;
    s.padded = align_up(tokens ? tokens : 1, kPadRows);
    s.ctas = pair_of(tokens);
    uint64_t piece = prob_bytes / (2 * s.padded) / kMaxTileN * kMaxTileN;
    if (piece < kMinPiece) piece = kMinPiece;
    const uint64_t all = align_up(vocab ? vocab : 1, kMaxTileN);
    if (piece > all) piece = all;
    s.pieces = (all + piece - 1) / piece;
    s.piece = align_up((all + s.pieces - 1) / s.pieces, kMaxTileN);
    s.pieces = (all + s.piece - 1) / s.piece;
    // few tiles: cut the long axis so that the GPU is full, in parts of at least 4 blocks
    const uint64_t tiles = s.padded / kPadRows * ((hidden + kMaxTileN - 1) / kMaxTileN);
    uint64_t splits = (kSplitSms / s.ctas) / (tiles ? tiles : 1);
    const uint64_t most = s.piece / kTileK / 4;
    if (splits > most) splits = most;
    if (splits > 32) splits = 32;
    s.splits = (uint32_t)(splits ? splits : 1);
    return s;
}

// Offsets of everything in a workspace.
struct CeLayout {
    uint64_t count, source, target, place, rows, scalar0, scalar1, stats, coef, prob, dx_sum, target_sum, sums, total;
};

static uint64_t take(uint64_t& at, uint64_t bytes) {
    const uint64_t here = at;
    at += align_up(bytes, kWorkspaceAlign);
    return here;
}

// Columns of a tile of kLse.  More than 128 tokens: 256, the widest.  Up to 128 tokens there is one row of tiles and
// reading W is all the time there is: the width that gives every SM the same share of W's rows
// (151936 rows: 208, five tiles for each of 148 SMs, 198 us; 256 gives 5 tiles to two of them and 4 to the others, 209 us).
static uint32_t lse_tile_n(uint64_t tokens, uint64_t vocab) {
    if (pair_of(tokens) == 2) return kMaxTileN;
    uint32_t best = kMaxTileN;
    uint64_t best_rows = UINT64_MAX;
    for (uint32_t n = kMaxTileN; n >= 128; n -= 16) {
        const uint64_t tiles = (vocab + n - 1) / n, rows = (tiles + kSplitSms - 1) / kSplitSms * n;
        if (rows < best_rows) {
            best_rows = rows;
            best = n;
        }
    }
    return best;
}

static CeLayout common_layout(uint64_t hidden, uint64_t padded, uint64_t& at) {
    CeLayout l = {};
    l.count = take(at, 8);
    l.source = take(at, padded * 4);
    l.target = take(at, padded * 4);
    l.place = take(at, padded * 4);
    l.rows = take(at, padded * align_up(hidden, kBlock) * 2);
    l.scalar0 = take(at, padded * 4);
    l.scalar1 = take(at, padded * 4);
    return l;
}

static CeLayout forward_layout(uint64_t tokens, uint64_t vocab, uint64_t hidden) {
    const CeShape s = ce_shape(tokens, vocab, hidden, kProbBytes);
    uint64_t at = 0;
    CeLayout l = common_layout(hidden, s.padded, at);
    const uint64_t tn = lse_tile_n(tokens, vocab);
    l.stats = take(at, (vocab + tn - 1) / tn * s.padded * sizeof(float2));
    l.total = at;
    return l;
}

static CeLayout backward_layout(uint64_t tokens, uint64_t vocab, uint64_t hidden, const CeShape& s) {
    uint64_t at = 0;
    CeLayout l = common_layout(hidden, s.padded, at);
    l.coef = take(at, s.padded * 4);
    l.prob = take(at, s.padded * s.piece * 2);
    l.dx_sum = take(at, s.splits * s.padded * hidden * 4);
    l.target_sum = take(at, s.padded * hidden * 4);
    l.sums = take(at, sorted_sum_workspace_bytes(s.padded, vocab, hidden));
    l.total = at;
    return l;
}

// The driver's tensor-map encoder, found through the runtime: no link against libcuda.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static dte_status encoder(EncodeTiled* out) {
    static std::atomic<void*> known{nullptr};
    void* f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult r;
        DTE_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r));
        if (r != cudaDriverEntryPointSuccess || !f) return op_fail(DTE_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
        known.store(f, std::memory_order_relaxed);
    }
    *out = reinterpret_cast<EncodeTiled>(f);
    return DTE_OK;
}

// bf16 matrix rows x cols with row stride ld, read in boxes of 64 columns x box_rows
static dte_status encode(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_rows) {
    EncodeTiled f;
    dte_status s = encoder(&f);
    if (s != DTE_OK) return s;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {(rows > 1 ? ld : align_up(cols, 8)) * 2};     // one row: its stride means nothing
    const cuuint32_t box[2] = {kTileK, box_rows};
    const cuuint32_t unit[2] = {1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, unit,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return op_fail(DTE_ERR_CUDA, "cuTensorMapEncodeTiled refused a matrix");
    return DTE_OK;
}

static dte_status encode_3d(CUtensorMap* map, const void* base, const cuuint64_t (&dims)[3], const cuuint64_t (&strides)[2],
                            const cuuint32_t (&box)[3]) {
    EncodeTiled f;
    dte_status s = encoder(&f);
    if (s != DTE_OK) return s;
    const cuuint32_t unit[3] = {1, 1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, unit,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return op_fail(DTE_ERR_CUDA, "cuTensorMapEncodeTiled refused a matrix");
    return DTE_OK;
}

// A blocked matrix of rows x blocks blocks of 64 columns, as (column in the block, block and row in it, row of blocks); boxes of
// `along` rows within a row of blocks and `down` rows of blocks.
static dte_status encode_blocked(CUtensorMap* map, const void* base, uint64_t rows, uint64_t blocks, uint32_t along, uint32_t down) {
    return encode_3d(map, base, {kBlock, blocks * kBlock, rows / kBlock}, {kBlock * 2, blocks * kBlock * kBlock * 2}, {kBlock, along, down});
}

// rows x cols, cols a multiple of 64, as (column in the chunk, row, chunk of 64 columns); boxes of 64 rows of `chunks` chunks
static dte_status encode_chunks(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t chunks) {
    return encode_3d(map, base, {kBlock, rows, cols / kBlock}, {(rows > 1 ? ld : cols) * 2, kBlock * 2}, {kBlock, kTileK, chunks});
}

template <int KIND, int CTAS>
static dte_status launch_ce_as(const CUtensorMap& a, const CUtensorMap& b, const CeParams& p, uint64_t most_tiles, int device, cudaStream_t st) {
    using S = CeStage<CTAS>;
    static std::atomic<uint64_t> ready{0};
    dte_status s = allow_smem(ce_kernel<KIND, CTAS>, S::kSmem, device, ready);
    if (s != DTE_OK) return s;
    int sms = 0;
    if ((s = device_sms(device, &sms)) != DTE_OK) return s;
    cudaLaunchConfig_t cfg = {};
    const uint64_t teams = (uint64_t)(sms / CTAS);
    cfg.gridDim = dim3((unsigned)((most_tiles < teams ? most_tiles : teams) * CTAS));
    cfg.blockDim = dim3(kCeThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // as launch_after
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CTAS;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    DTE_CUDA(cudaLaunchKernelEx(&cfg, ce_kernel<KIND, CTAS>, a, b, p));
    return DTE_OK;
}

template <int KIND>
static dte_status launch_ce(int ctas, const CUtensorMap& a, const CUtensorMap& b, const CeParams& p, uint64_t rows, int device, cudaStream_t st) {
    const uint64_t tiles = (rows + kTileM * ctas - 1) / (kTileM * ctas) * ((p.n + p.tile_n - 1) / p.tile_n) * p.splits;
    return ctas == 2 ? launch_ce_as<KIND, 2>(a, b, p, tiles, device, st) : launch_ce_as<KIND, 1>(a, b, p, tiles, device, st);
}

static std::atomic<uint32_t> g_wait_limit{kWaitTries};

static dte_status check_head(const dte_matrix* x, const dte_matrix* weight, const dte_ids* targets, uint64_t vocab_start,
                             uint64_t vocab, double logit_scale, const uint64_t* flags) {
    dte_status s;
    if ((s = check_matrix(x, "x is null", false)) != DTE_OK) return s;
    if ((s = check_matrix(weight, "weight is null", false)) != DTE_OK) return s;
    if ((s = check_ids(targets)) != DTE_OK) return s;
    if (x->dtype != DTE_BF16 || weight->dtype != DTE_BF16) return op_fail(DTE_ERR_INVALID_ARG, "x and weight must be BF16");
    if (x->cols != weight->cols || x->rows != targets->count)
        return op_fail(DTE_ERR_INVALID_ARG, "x must be targets.count x weight.cols");
    if (weight->rows == 0) return op_fail(DTE_ERR_INVALID_ARG, "weight has no rows");
    if (x->cols % 8) return op_fail(DTE_ERR_INVALID_ARG, "hidden must be a multiple of 8");
    if (((uintptr_t)weight->data & 15u) || weight->ld % 8 || (weight->rows > 1 && weight->ld < weight->cols))
        return op_fail(DTE_ERR_INVALID_ARG, "weight must be 16-byte aligned with ld >= cols, a multiple of 8");
    if ((s = check_range(vocab_start, weight->rows, vocab)) != DTE_OK) return s;
    if (!(logit_scale > 0) || !std::isfinite((float)(logit_scale * kLog2eD)))
        return op_fail(DTE_ERR_INVALID_ARG, "logit_scale must be > 0 and, times log2(e), finite in fp32");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if (targets->count > (1u << 24) || weight->rows > (1u << 24) || x->cols > (1u << 20))
        return op_fail(DTE_ERR_INVALID_ARG, "at most 2^24 tokens, 2^24 vocabulary rows and 2^20 hidden");
    if (align_up(targets->count, kPadRows) * ((x->cols + kBlock - 1) / kBlock) >= (1ull << 31))
        return op_fail(DTE_ERR_INVALID_ARG, "tokens x hidden is too large for one call");
    if ((targets->count / kTileM + 1) * (weight->rows / 128 + 1) >= (1ull << 31))
        return op_fail(DTE_ERR_INVALID_ARG, "tokens x vocabulary is too large for one call");
    return DTE_OK;
}

static bool ce_sizes_ok(uint64_t tokens, uint64_t vocab, uint64_t hidden) {
    return tokens <= (1u << 24) && vocab <= (1u << 24) && hidden <= (1u << 20);
}

static dte_status prepare_rows(const CeLayout& l, uint8_t* ws, const dte_matrix* x, const dte_matrix* weight, const dte_ids* targets,
                               uint64_t vocab_start, uint64_t vocab, uint64_t padded, float scale, float* lse, float* target_logit,
                               float* loss, const float* lse_in, const float* dloss, uint64_t* flags, cudaStream_t st) {
    RowsParams r = {};
    r.targets = targets->data;
    r.targets_dtype = targets->dtype;
    r.n = (uint32_t)targets->count;
    r.vocab_start = (int64_t)vocab_start;
    r.vocab = (int64_t)vocab;
    r.vocab_rows = (uint32_t)weight->rows;
    r.count = reinterpret_cast<uint32_t*>(ws + l.count);
    r.source = reinterpret_cast<int32_t*>(ws + l.source);
    r.target = reinterpret_cast<int32_t*>(ws + l.target);
    r.split = dloss && targets->count <= kSplitTokens;
    r.place = dloss ? reinterpret_cast<int32_t*>(ws + l.place) : nullptr;
    r.lse = lse;
    r.target_logit = target_logit;
    r.loss = loss;
    r.flags = flags;
    GatherRowsParams g = {};
    g.rows_of = r;
    g.few = targets->count <= kFewTokens;
    g.count = r.count;
    g.source = r.source;
    g.x = static_cast<const __nv_bfloat16*>(x->data);
    g.x_ld = x->ld;
    g.hidden = (uint32_t)x->cols;
    g.vec = vec8_ok(x);
    g.rows = reinterpret_cast<__nv_bfloat16*>(ws + l.rows);
    g.blocks = (uint32_t)((x->cols + kBlock - 1) / kBlock);
    g.scale = scale;
    g.weight = static_cast<const __nv_bfloat16*>(weight->data);
    g.weight_ld = weight->ld;
    if (dloss) {
        g.dloss = dloss;
        g.lse = lse_in;
        g.coef = reinterpret_cast<float*>(ws + l.coef);
        g.f = reinterpret_cast<float*>(ws + l.scalar0);
        g.neg_lse2 = reinterpret_cast<float*>(ws + l.scalar1);
    } else {
        g.target_logit = reinterpret_cast<float*>(ws + l.scalar0);
        g.exact_logit = reinterpret_cast<float*>(ws + l.scalar1);
    }
    g.target = r.target;
    if (g.few) {
        ce_gather_kernel<<<(unsigned)padded, kGatherThreads, 0, st>>>(g);
    } else {
        ce_rows_kernel<<<1, kRowsThreads, 0, st>>>(r);
        DTE_CUDA(cudaGetLastError());
        DTE_CUDA(launch_after(ce_gather_kernel, dim3((unsigned)padded), kGatherThreads, 0, st, g));
    }
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

}  // namespace dte

using namespace dte;

extern "C" void dte_linear_ce_set_wait_limit(uint32_t tries) {
    g_wait_limit.store(tries ? tries : kWaitTries, std::memory_order_relaxed);
}

extern "C" uint64_t dte_linear_ce_forward_workspace_bytes(uint64_t tokens, uint64_t vocab_rows, uint64_t hidden) {
    if (!ce_sizes_ok(tokens, vocab_rows, hidden)) return UINT64_MAX;     // refused by the call
    return forward_layout(tokens, vocab_rows, hidden).total;
}

extern "C" dte_status dte_linear_ce_forward(const dte_matrix* x, const dte_matrix* weight, const dte_ids* targets, uint64_t vocab_start,
                                            uint64_t vocab, double logit_scale, float* lse, float* target_logit, float* loss,
                                            void* workspace, uint64_t workspace_bytes, uint64_t* flags, int device,
                                            void* cuda_stream) {
    dte_status s;
    if ((s = check_head(x, weight, targets, vocab_start, vocab, logit_scale, flags)) != DTE_OK) return s;
    if (targets->count && !lse) return op_fail(DTE_ERR_INVALID_ARG, "lse is null");
    if (((uintptr_t)lse | (uintptr_t)target_logit | (uintptr_t)loss) & 3u)
        return op_fail(DTE_ERR_INVALID_ARG, "lse, target_logit and loss must be 4-byte aligned");
    const uint64_t n = targets->count, V = weight->rows, H = x->cols;
    const CeLayout l = forward_layout(n, V, H);
    if ((s = check_workspace(workspace, workspace_bytes, l.total)) != DTE_OK) return s;
    if (n == 0) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const CeShape sh = ce_shape(n, V, H, kProbBytes);
    if ((s = prepare_rows(l, ws, x, weight, targets, vocab_start, vocab, sh.padded, (float)logit_scale, lse, target_logit, loss, nullptr,
                          nullptr, flags, st)) != DTE_OK)
        return s;
    const uint32_t tn = lse_tile_n(n, V);
    CeParams p = {};
    p.n = (uint32_t)V;
    p.k = (uint32_t)H;
    p.tokens = reinterpret_cast<uint32_t*>(ws + l.count);
    p.tile_n = tn;
    p.splits = 1;
    p.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    p.flags = flags;
    p.scale = (float)logit_scale;
    p.k2 = (float)(logit_scale * kLog2eD);
    p.target = reinterpret_cast<int32_t*>(ws + l.target);
    p.stats = reinterpret_cast<float2*>(ws + l.stats);
    p.stats_ld = sh.padded;
    p.target_logit = reinterpret_cast<float*>(ws + l.scalar0);
    CUtensorMap ma, mb;
    if ((s = encode_blocked(&ma, ws + l.rows, sh.padded, (H + kBlock - 1) / kBlock, kBlock, kTileM / kBlock)) != DTE_OK) return s;
    if ((s = encode(&mb, weight->data, V, H, weight->ld, tn / sh.ctas)) != DTE_OK) return s;
    if ((s = launch_ce<kLse>(sh.ctas, ma, mb, p, n, device, st)) != DTE_OK) return s;
    CombineParams c = {};
    c.count = p.tokens;
    c.source = reinterpret_cast<int32_t*>(ws + l.source);
    c.stats = p.stats;
    c.stats_ld = p.stats_ld;
    c.tiles = (uint32_t)((V + tn - 1) / tn);
    c.target = p.target;
    c.row_target_logit = p.target_logit;
    c.exact_logit = reinterpret_cast<float*>(ws + l.scalar1);
    c.lse = lse;
    c.target_logit = target_logit;
    c.loss = loss;
    DTE_CUDA(launch_after(ce_combine_kernel, dim3((unsigned)((n + kCombineRows - 1) / kCombineRows)), kCombineThreads, 0, st, c));
    return DTE_OK;
}

extern "C" uint64_t dte_linear_ce_backward_workspace_bytes(uint64_t tokens, uint64_t vocab_rows, uint64_t hidden) {
    if (!ce_sizes_ok(tokens, vocab_rows, hidden)) return UINT64_MAX;     // refused by the call
    return backward_layout(tokens, vocab_rows, hidden, ce_shape(tokens, vocab_rows, hidden, kProbBytes)).total;
}

extern "C" uint64_t dte_linear_ce_backward_workspace_min_bytes(uint64_t tokens, uint64_t vocab_rows, uint64_t hidden) {
    if (!ce_sizes_ok(tokens, vocab_rows, hidden)) return UINT64_MAX;
    return backward_layout(tokens, vocab_rows, hidden, ce_shape(tokens, vocab_rows, hidden, 0)).total;
}

extern "C" dte_status dte_linear_ce_backward(const dte_matrix* x, const dte_matrix* weight, const dte_ids* targets, uint64_t vocab_start,
                                             uint64_t vocab, double logit_scale, const float* lse, const float* dloss, int accumulate,
                                             const dte_matrix* dx, const dte_matrix* dweight, void* workspace, uint64_t workspace_bytes,
                                             uint64_t* flags, int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_head(x, weight, targets, vocab_start, vocab, logit_scale, flags)) != DTE_OK) return s;
    const uint64_t n = targets->count, V = weight->rows, H = x->cols;
    if (n && (!lse || !dloss)) return op_fail(DTE_ERR_INVALID_ARG, "lse / dloss is null");
    if (((uintptr_t)lse | (uintptr_t)dloss) & 3u) return op_fail(DTE_ERR_INVALID_ARG, "lse and dloss must be 4-byte aligned");
    if (dx) {
        if ((s = check_matrix(dx, "dx is null", true)) != DTE_OK) return s;
        if (dx->dtype != DTE_BF16 || dx->rows != n || dx->cols != H) return op_fail(DTE_ERR_INVALID_ARG, "dx must have x's shape, BF16");
        if (!vec8_ok(dx)) return op_fail(DTE_ERR_INVALID_ARG, "dx rows must be 16-byte aligned");
    }
    if (dweight) {
        if ((s = check_matrix(dweight, "dweight is null", true)) != DTE_OK) return s;
        if (dweight->rows != V || dweight->cols != H) return op_fail(DTE_ERR_INVALID_ARG, "dweight must have weight's shape");
        if (!vec8_ok(dweight)) return op_fail(DTE_ERR_INVALID_ARG, "dweight rows must be 16-byte aligned");
    }
    // the largest piece this workspace holds
    uint64_t budget = kProbBytes;
    CeShape sh = ce_shape(n, V, H, budget);
    CeLayout l = backward_layout(n, V, H, sh);
    while (l.total > workspace_bytes && budget) {
        budget = budget > (1u << 20) ? budget / 2 : 0;
        sh = ce_shape(n, V, H, budget);
        l = backward_layout(n, V, H, sh);
    }
    if ((s = check_workspace(workspace, workspace_bytes, l.total)) != DTE_OK) return s;
    if (!dx && !dweight) return DTE_OK;
    if (n == 0 && (!dweight || accumulate)) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (n == 0) {
        DTE_CUDA(cudaMemset2DAsync(dweight->data, dweight->ld * elem_size(dweight->dtype), 0, H * elem_size(dweight->dtype), V, st));
        return DTE_OK;
    }
    if ((s = prepare_rows(l, ws, x, weight, targets, vocab_start, vocab, sh.padded, (float)logit_scale, nullptr, nullptr, nullptr, lse, dloss,
                          flags, st)) != DTE_OK)
        return s;
    const uint32_t* count = reinterpret_cast<uint32_t*>(ws + l.count);
    const float* coef = reinterpret_cast<float*>(ws + l.coef);
    const int32_t* target = reinterpret_cast<int32_t*>(ws + l.target);
    float* target_sum = reinterpret_cast<float*>(ws + l.target_sum);
    if (dweight) {
        SortedSum q = {};
        q.ids = targets->data;
        q.ids_dtype = targets->dtype;
        q.n = (uint32_t)n;
        q.row_start = (int64_t)vocab_start;
        q.vocab = vocab;
        q.rows = (uint32_t)V;
        q.src = x->data;
        q.src_dtype = DTE_BF16;
        q.src_ld = x->ld;
        q.weight = coef;
        q.hidden = (uint32_t)H;
        q.scale = 1.f;                    // coef has it already
        q.out = target_sum;
        q.out_dtype = DTE_F32;
        q.out_ld = H;
        q.compact = true;
        if ((s = launch_sorted_sum(q, vec8_ok(x) ? 8 : vec2_ok(x) ? 2 : 1, ws + l.sums, true, device, st)) != DTE_OK) return s;
    }
    CeParams p = {};
    p.tokens = count + 1;
    p.split = n <= kSplitTokens;
    p.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    p.flags = flags;
    p.scale = (float)logit_scale;
    p.k2 = (float)(logit_scale * kLog2eD);
    p.target = target;
    p.f = reinterpret_cast<float*>(ws + l.scalar0);
    p.neg_lse2 = reinterpret_cast<float*>(ws + l.scalar1);
    p.prob = reinterpret_cast<__nv_bfloat16*>(ws + l.prob);
    p.prob_blocks = (uint32_t)(sh.piece / kBlock);
    p.dx_sum = reinterpret_cast<float*>(ws + l.dx_sum);
    p.dx_split = sh.padded * H;
    if (dweight) {
        p.dweight = dweight->data;
        p.dweight_ld = dweight->ld;
        p.dweight_bf16 = dweight->dtype == DTE_BF16;
        p.whole_sectors = !(((uintptr_t)dweight->data | dweight->ld * elem_size(dweight->dtype)) & 31u);
    }
    p.accumulate = accumulate != 0;
    p.first = sorted_sum_first(ws + l.sums);
    p.target_sum = target_sum;
    CUtensorMap rows_k, rows_n, prob_k, prob_m, w_k, w_n;
    const uint32_t bn = kMaxTileN, part = bn / sh.ctas, down = kTileM / kBlock;
    const uint64_t x_blocks = (H + kBlock - 1) / kBlock;
    p.w_chunks = H % kBlock == 0;
    if ((s = encode_blocked(&rows_k, ws + l.rows, sh.padded, x_blocks, kBlock, down)) != DTE_OK) return s;
    if ((s = encode_blocked(&rows_n, ws + l.rows, sh.padded, x_blocks, part, 1)) != DTE_OK) return s;
    if ((s = encode_blocked(&prob_k, ws + l.prob, sh.padded, p.prob_blocks, kBlock, down)) != DTE_OK) return s;
    if ((s = encode_blocked(&prob_m, ws + l.prob, sh.padded, p.prob_blocks, kTileM, 1)) != DTE_OK) return s;
    if ((s = encode(&w_k, weight->data, V, H, weight->ld, part)) != DTE_OK) return s;
    if ((s = p.w_chunks ? encode_chunks(&w_n, weight->data, V, H, weight->ld, part / kBlock)
                        : encode(&w_n, weight->data, V, H, weight->ld, kTileK)) != DTE_OK)
        return s;
    for (uint64_t piece = 0; piece < sh.pieces; ++piece) {
        const uint64_t v0 = piece * sh.piece, vc = V - v0 < sh.piece ? V - v0 : sh.piece;
        p.w_row = (uint32_t)v0;
        p.tile_n = bn;
        p.splits = 1;
        p.n = (uint32_t)vc;
        p.k = (uint32_t)H;
        if ((s = launch_ce<kProb>(sh.ctas, rows_k, w_k, p, n, device, st)) != DTE_OK) return s;
        if (dx) {
            p.n = (uint32_t)H;
            p.k = (uint32_t)vc;
            p.splits = sh.splits;
            p.add = piece > 0;
            if ((s = launch_ce<kDx>(sh.ctas, prob_k, w_n, p, n, device, st)) != DTE_OK) return s;
        }
        if (dweight) {
            p.m = (uint32_t)vc;
            p.n = (uint32_t)H;
            p.splits = 1;
            if ((s = launch_ce<kDw>(sh.ctas, prob_m, rows_n, p, vc, device, st)) != DTE_OK) return s;
        }
    }
    if (dx) {
        DxParams d = {};
        d.place = reinterpret_cast<int32_t*>(ws + l.place);
        d.target = target;
        d.coef = coef;
        d.sums = p.dx_sum;
        d.split_elems = p.dx_split;
        d.splits = sh.splits;
        d.split = p.split;
        d.hidden = (uint32_t)H;
        d.weight = static_cast<const __nv_bfloat16*>(weight->data);
        d.weight_ld = weight->ld;
        d.dx = static_cast<__nv_bfloat16*>(dx->data);
        d.dx_ld = dx->ld;
        DTE_CUDA(launch_after(ce_dx_kernel, dim3((unsigned)n), 256, 0, st, d));
    }
    return DTE_OK;
}
