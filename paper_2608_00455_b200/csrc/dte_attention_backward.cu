// Gradient of causal attention over packed sequences, in two passes over the scores that share nothing but delta, so that
// the order of every sum is fixed (one pass would have to add dq up across CTAs):
//   att_delta_kernel  delta = sum over a head's columns of dout * out
//   att_dkv_kernel    a tile of 128 keys of one key head against the queries of its group that see them:  dk, dv
//   att_dq_kernel     a tile of 128 queries of one head against its keys:  dq
// With p = exp(z - lse), dz = p (dout v^T - delta): dq = scale dz k, dk = scale dz^T q, dv = p^T dout.  The first pass has four products
// per pair of tiles, the second three, where one pass would have five.  Both draw their tiles, the largest first, from a counter,
// and the second one starts on the SMs that the first one leaves: few, unequal key tiles leave most SMs early.
//
// Both: one CTA per SM, a warp that loads, two that issue products, eight that turn scores into operands, each thread half a
// row.  The first pass works on the transposed scores (rows are keys), so that p and dz are, as they come out of the
// registers, the left operands of dv and dk in tensor memory.
//
// p and dz are rounded to bf16, the operand type of the products they enter, and delta is made of out as it was rounded; sums are fp32.  For
// random inputs dq, dk and dv are then 2.7e-3 to 3.0e-3, 2.4e-3 to 2.6e-3 and 2.3e-3 off (relative, rms), of which their own rounding
// to bf16 is 1.7e-3; where sequences have few tokens, dout v^T - delta cancels more, and dq is up to 4.1e-3, dk 3.6e-3 off.  dz as two
// bf16 numbers makes the first two 2.2e-3 and 1.9e-3 and the passes 16 % slower, so it is not kept so.
//
// Measured, heads of 128, all three kernels: 16384 tokens, 32 heads on 8: 6.7 ms in a loop at the power limit (0.82 PFLOP/s of the five
// products that the formulas need, 1.15 of the seven that are made); 8192 tokens in 19 sequences, 32 heads on 4: 299 us; 4001 tokens in 57
// sequences, 16 heads of 64: 72 us.  A step takes 3300 cycles in the first pass, 2048 of them the tensor cores', and 2200 in the second,
// 1536: the chain of p (1500 and 1250 cycles, 1024 of which the special function unit needs) and of the products that wait for it sets the
// pace.  A piece of work costs 4000 to 7000 cycles beside its steps.  Tried and left: sixteen score warps (dk / dv 3.6 to 3.8 ms), p in
// shared memory so that the next S need not wait for dv (7.2 ms against 6.7: operands of products in shared memory cost its bandwidth), p in
// two parts so that dv begins early (equal), a polynomial for a share of the exponentials (slower).
#include <atomic>

#include "dte_attention.cuh"

namespace dte {

constexpr uint32_t kBwdThreads = 3 * 128;         // registers as in the forward kernel
constexpr uint32_t kBwdWarps = 8;                 // that work on scores
constexpr int kFewRegs = 72, kManyRegs = 208;     // 128 * (72 + 2 * 208) = 62464 of the 384 * 168 = 64512 at launch
constexpr uint32_t kRing3 = 3, kRing2 = 2;         // tiles in flight of the two streams, a ring each: every barrier has one reader in order
constexpr uint32_t kBwdSmem = (2 + kRing3 + kRing2) * kTileBytes;
// The score warps count their steps to where places and phases of both rings repeat: a CTA may take more than 2^32 of them.
constexpr uint32_t kSteps = 4 * kRing3;
static_assert(kSteps % (2 * kRing2) == 0, "");
__device__ __forceinline__ uint32_t next_step(uint32_t g) { return g + 1 == kSteps ? 0 : g + 1; }
constexpr uint32_t kHalf = kAttTile / 2;          // columns of a tile that a thread works on
// In tensor memory a tile of scores takes 128 columns.  The bf16 operand made of it lies over it, each half over the
// columns that the same threads have read.

__device__ __forceinline__ void load_half(uint32_t tmem, float (&z)[kHalf]) {
    uint32_t a[32], b[32];
    tmem_load32(tmem, a);
    tmem_load32(tmem + 32, b);
    tmem_load_wait(a);
    tmem_load_wait(b);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        z[j] = __uint_as_float(a[j]);
        z[32 + j] = __uint_as_float(b[j]);
    }
}

__device__ __forceinline__ void store_half(uint32_t tmem, const float (&z)[kHalf]) {
    uint32_t v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = pack_bf16(z[2 * j], z[2 * j + 1]);
    tmem_store32(tmem, v);
    tmem_store_wait();
    tc_fence_before();
    __syncwarp();
}

// Zeros for the columns outside [low, high), which may lie anywhere.
__device__ __forceinline__ void keep_columns(float (&z)[kHalf], int low, int high) {
    auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1; };
    const uint32_t kept[2] = {below(high) & ~below(low), below(high - 32) & ~below(low - 32)};
#pragma unroll
    for (int c = 0; c < (int)kHalf; ++c) z[c] = kept[c / 32] & (1u << (c % 32)) ? z[c] : 0.f;
}

// ---- delta ------------------------------------------------------------------------------------------------------
constexpr uint32_t kDeltaThreads = 256;

// Into how many parts, a power of two whose exponent is given, the first pass cuts the query heads of each key head, so that one key
// tile's work need not run on alone.  A part leaves its sums of dk and dv in the workspace, 128 KB that are written and read again, and
// the last part of a tile to finish adds all of them up.  So groups are halved while that saves more than it costs, in steps of the first pass: the
// longest piece becomes half as long, which is of use down to what every SM has to do on average (in both passes, whose steps take about 3 to 2),
// and every piece on an SM costs about ten steps, and the waiting for the last part two.  Whole backward pass, uncut and cut, from a cold L2, one
// sequence: 300 tokens, 32 heads on 4: 73 and 44 us, 1024: 140 and 67, 2048: 265 and 157, 4096: 515 and 422; 2048, 32 on 1: 960 and 165; 4096,
// 32 on 1 of 64: 1590 and 370.  Uncut by this rule: 2048, 32 on 8, 150 us, cut 157.
__device__ __forceinline__ uint32_t group_cut(const AttParams& p, uint32_t heads) {
    if (p.group == 1 || !plan_ok(p)) return 0;
    const PlanHead* h = reinterpret_cast<const PlanHead*>(p.plan);
    const uint64_t kv_heads = heads / p.group, pieces = h->tiles * kv_heads;
    if (pieces == 0) return 0;
    float longest = (float)((reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader)->tile + 1) * p.group);
    const float average = 5.f / 3.f * (float)h->steps * (float)heads / kSms;
    uint32_t cut = 0;
    for (; (p.group >> cut) % 2 == 0 && pieces << (cut + 1) <= kMostParts; ++cut, longest /= 2)
        if (longest - fmaxf(longest / 2, average) <= 2.f + 10.f * (float)(pieces << (cut + 1)) / kSms) break;
    return cut;
}

// A warp takes eight times LANES' share of 32 rows of a head: LANES lanes a row, 8 columns each.  The first CTA sets up the counters of the
// two passes instead.
template <uint32_t LANES>
__global__ void __launch_bounds__(kDeltaThreads) att_delta_kernel(const AttParams p, uint32_t heads) {
    constexpr uint32_t kRows = 32 / LANES, kTokens = 8 * kRows;
    let_next_start();
    if (blockIdx.x == 0) {
        for (uint64_t i = threadIdx.x; i < min((uint64_t)kMostParts, p.tokens * heads) * 8 && p.group > 1; i += kDeltaThreads) p.parts_done[i] = 0;
        if (threadIdx.x == 0) {
            p.next[0] = p.next[1] = p.next[3] = 0;
            p.next[2] = group_cut(p, heads);
        }
        return;
    }
    const uint64_t unit = (uint64_t)(blockIdx.x - 1) * (kDeltaThreads / 32) + threadIdx.x / 32, first = unit / heads * kTokens;
    const uint32_t lane = threadIdx.x & 31, h = (uint32_t)(unit % heads), row = lane / LANES, col = lane % LANES * 8;
    if (first >= p.tokens) return;
    const bool here = col < p.head_dim;
    Raw8<__nv_bfloat16> o[8], d[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        const uint64_t at = min(first + kRows * j + row, p.tokens - 1);
        o[j].load(p.o + at * p.o_ld + h * p.head_dim + (here ? col : 0));
        d[j].load(p.d_o + at * p.do_ld + h * p.head_dim + (here ? col : 0));
    }
    float mine = 0.f;                  // of token kRows * (lane % LANES) + row, for the first eight of a row's lanes
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        float a[8], b[8], sum = 0.f;
        o[j].get(a);
        d[j].get(b);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum = fmaf(a[c], b[c], sum);
        sum = here ? sum : 0.f;
#pragma unroll
        for (uint32_t c = LANES / 2; c; c >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, c);
        if (lane % LANES == j) mine = sum;
    }
    const uint64_t token = first + kRows * (lane % LANES) + row;
    if (lane % LANES < 8 && token < p.tokens) p.delta[h * p.tokens + token] = mine;
}

// ---- dq -------------------------------------------------------------------------------------------------------
// Tensor memory: S at columns 0 and 128 in turn (dz over it), dP at 256, dq at 384.
__global__ void __launch_bounds__(kBwdThreads, 1)
    att_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_do, const __grid_constant__ AttParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];          // the swizzle's period
    enum { kKFull, kKEmpty = kRing3, kVFull = 2 * kRing3, kVEmpty = kVFull + kRing2, kQFull = kVEmpty + kRing2, kQEmpty, kSFull, kDsFull = kSFull + 2, kDpFull = kDsFull + 2, kDpRead, kDqFull,
           kWorkFull, kWorkEmpty = kWorkFull + 2, kLast = kWorkEmpty + 2, kBars };
    __shared__ __align__(8) uint64_t s_bar[kBars];
    __shared__ uint32_t s_tmem, s_gave_up, s_issued[3], s_taken[3];         // loads of K, V, and Q with dout
    __shared__ bool s_seen;
    __shared__ uint4 s_work[2];            // start, length, tile and head of the next pieces of work; no tile: the end
    const uint32_t q0 = smem_addr(smem), do0 = q0 + kTileBytes, kt0 = q0 + 2 * kTileBytes, vt0 = kt0 + kRing3 * kTileBytes;
    auto bar = [bar0 = smem_addr(s_bar)](uint32_t i) { return bar0 + 8 * i; };
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
        tma_prefetch_map(&map_do);
        for (uint32_t i = 0; i < kBars; ++i)
            mbar_init(bar(i), i == kDsFull || i == kDsFull + 1 || i == kDpRead ? kBwdWarps
                              : i == kWorkEmpty || i == kWorkEmpty + 1         ? 3 + kBwdWarps
                              : i == kQEmpty || i == kLast                     ? 2
                                                                               : 1);
        s_gave_up = 0;
        for (uint32_t i = 0; i < 3; ++i) s_issued[i] = s_taken[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&s_tmem), 512);
    // The first pass runs on; delta, the counters and the inputs are there, as it has seen.
    if (threadIdx.x == 96) s_seen = seen_earlier(p.next + 3, p.wait_limit);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("fence.proxy.async;" ::: "memory");          // for the loads of tiles, too
    const uint32_t tmem = uniform(*(volatile uint32_t*)&s_tmem);
    volatile uint32_t* gave_up = &s_gave_up;
    const bool seen = s_seen;
    if (!seen) *gave_up = 1;
    const uint32_t total = seen && plan_ok(p) ? reinterpret_cast<const PlanHead*>(p.plan)->tiles * p.units : 0;
    const PlanItem* list = reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader);
    const uint32_t chunks = (p.head_dim + 63) / 64, tile_bytes = chunks * kChunkBytes;
    // The next piece of work, by a whole warp; false at the end, or where the wait runs out.
    auto take_work = [&](uint32_t& n, PlanItem& it, uint32_t& h) {
        if (!warp_wait(bar(kWorkFull + (n & 1)), n >> 1 & 1, p.wait_limit, gave_up)) return false;
        const uint4 w = s_work[n & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kWorkEmpty + (n & 1)));
        ++n;
        it = PlanItem{w.x, w.y, w.z, 0};
        h = w.w;
        return w.z != kNone;
    };

    if (warp < 4) {
        regs_down<kFewRegs>();
        if (warp == 0) {
            // ---- loads: one lane ----
            uint32_t tiles = 0, k_issued = 0, q_issued = 0, works = 0;
            RingAt<kRing3> ka;
            RingAt<kRing2> va;
            bool ok = true;
            PlanItem it;
            uint32_t h;
            while (ok && take_work(works, it, h)) {
                if (lane == 0) {
                    const uint32_t kh = h / p.group, row = it.start + it.tile * kAttTile;
                    if ((ok = mbar_wait(bar(kQEmpty), (q_issued & 1) ^ 1, p.wait_limit, gave_up))) {
                        mbar_expect_tx(bar(kQFull), 2 * tile_bytes);
                        load_rows(q0, &map_q, chunks, h, row, bar(kQFull));
                        load_rows(do0, &map_do, chunks, h, row, bar(kQFull));
                        ++q_issued;
                    }
                    for (uint32_t t = 0; t <= it.tile && ok; ++t) {
                        if (!(ok = mbar_wait(bar(kKEmpty + ka.i), ka.phase ^ 1, p.wait_limit, gave_up))) break;
                        mbar_expect_tx(bar(kKFull + ka.i), tile_bytes);
                        load_rows(kt0 + ka.i * kTileBytes, &map_k, chunks, kh, it.start + t * kAttTile, bar(kKFull + ka.i));
                        ka.next();
                        ++k_issued;
                        if (!(ok = mbar_wait(bar(kVEmpty + va.i), va.phase ^ 1, p.wait_limit, gave_up))) break;
                        mbar_expect_tx(bar(kVFull + va.i), tile_bytes);
                        load_rows(vt0 + va.i * kTileBytes, &map_v, chunks, kh, it.start + t * kAttTile, bar(kVFull + va.i));
                        va.next();
                        ++tiles;
                    }
                }
                ok = __all_sync(0xFFFFFFFFu, ok);
            }
            if (lane == 0) {
                s_issued[0] = k_issued;
                s_issued[1] = tiles;
                s_issued[2] = q_issued;
            }
        } else if (warp == 1) {
            // ---- products, S and dq: the whole warp waits, one lane issues.  An issue blocks until the tensor cores are nearly
            // through with it, so dP has a warp of its own ----
            const uint32_t desc_s = mma_desc(kAttTile, kAttTile, false, false), steps = (p.head_dim + 15) / 16;
            const uint32_t desc_d = mma_desc(kAttTile, steps * 16, false, true);
            uint32_t q_taken = 0, works = 0, g = 0, made = 0;       // g, made: steps of dq and of S so far
            RingAt<kRing3> sa, da;
            bool ok = true;
            auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(bar(b), parity, p.wait_limit, gave_up); };
            PlanItem it;
            uint32_t h;
            while (ok && take_work(works, it, h)) {
                const uint32_t n = it.tile + 1;
                if (!wait(kQFull, q_taken & 1)) break;
                ++q_taken;
                auto scores = [&](uint32_t t) {
                    if (!wait(kKFull + sa.i, sa.phase)) return;
                    const uint32_t k = uniform(kt0 + sa.i * kTileBytes), to = uniform(made & 1);
                    if (elect_lane()) {
                        mma_rows(tmem + to * 128, q0, k, steps, desc_s);
                        mma_commit<1>(bar(kSFull + to));
                        if (t + 1 == n) mma_commit<1>(bar(kQEmpty));
                    }
                    sa.next();
                    ++made;
                };
                scores(0);
                if (n > 1) scores(1);
                for (uint32_t t = 0; t < n && ok; ++t, ++g) {
                    const uint32_t k = uniform(kt0 + da.i * kTileBytes), release = uniform(bar(kKEmpty + da.i)), from = uniform(tmem + (g & 1) * 128);
                    if (!wait(kDsFull + (g & 1), g >> 1 & 1)) break;
                    if (elect_lane()) {
                        mma_tile<kHalf>(tmem + 384, from, k, desc_d, t != 0);
                        mma_commit<1>(release);
                        if (t + 1 == n) mma_commit<1>(bar(kDqFull));
                    }
                    da.next();
                    if (t + 2 < n) scores(t + 2);
                }
            }
            if (lane == 0) {
                s_taken[0] = made;
                s_taken[2] = q_taken;
            }
        } else if (warp == 2) {
            // ---- products, dP ----
            const uint32_t desc_s = mma_desc(kAttTile, kAttTile, false, false), steps = (p.head_dim + 15) / 16;
            uint32_t q_taken = 0, works = 0, g = 0;
            RingAt<kRing2> va;
            bool ok = true, begun = false;           // begun: there is a dP in front whose reading has to be waited for
            auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(bar(b), parity, p.wait_limit, gave_up); };
            PlanItem it;
            uint32_t h;
            while (ok && take_work(works, it, h)) {
                const uint32_t n = it.tile + 1;
                if (!wait(kQFull, q_taken++ & 1)) break;
                for (uint32_t t = 0; t < n && ok; ++t) {
                    if (!wait(kVFull + va.i, va.phase)) break;
                    const uint32_t v = uniform(vt0 + va.i * kTileBytes), release = uniform(bar(kVEmpty + va.i));
                    va.next();
                    ++g;
                    if (begun && !wait(kDpRead, g & 1)) break;
                    begun = true;
                    if (elect_lane()) {
                        mma_rows(tmem + 256, do0, v, steps, desc_s);
                        mma_commit<1>(bar(kDpFull));
                        mma_commit<1>(release);
                        if (t + 1 == n) mma_commit<1>(bar(kQEmpty));
                    }
                }
            }
            if (lane == 0) s_taken[1] = g;
        } else if (lane == 0) {
            // ---- work: tiles of queries in falling order of their keys, from the counter that all CTAs share ----
            for (uint32_t n = 0;; ++n) {
                if (!mbar_wait(bar(kWorkEmpty + (n & 1)), (n >> 1 & 1) ^ 1, p.wait_limit, gave_up)) break;
                const uint32_t w = atomicAdd(p.next + 1, 1u);
                const bool more = w < total;
                uint4 v = make_uint4(0, 0, kNone, 0);
                if (more) {
                    const PlanItem it = list[w / p.units];
                    v = make_uint4(it.start, it.len, it.tile, w % p.units);
                }
                s_work[n & 1] = v;
                mbar_arrive(bar(kWorkFull + (n & 1)));
                if (!more) break;
            }
        }
    } else {
        regs_up<kManyRegs>();
        // ---- scores: warp w may read the quarter w % 4 of tensor memory's lanes ----
        const uint32_t half = (warp - 4) / 4, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t mine = tmem + (quarter * 32 << 16);
        uint32_t g = 0, done = 0, works = 0;
        bool ok = true;
        auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(bar(b), parity, p.wait_limit, gave_up); };
        // A finished tile's dq is read from tensor memory only when the next work's first p is made: its last product and the next
        // one's first scores take their time meanwhile.
        __nv_bfloat16* out = nullptr;                   // of the tile that waits, NULL: a row past its sequence
        bool waits = false;
        auto finish = [&]() {
            if (!wait(kDqFull, done++ & 1)) return;
            for (uint32_t c = half * 32; c < p.head_dim; c += 64) store_columns(out, mine + 384, c, p.head_dim, p.scale, out != nullptr, p.sectors);
            tc_fence_before();
            waits = false;
        };
        PlanItem it;
        uint32_t h;
        while (ok && take_work(works, it, h)) {
            const uint32_t n = it.tile + 1, row = it.tile * kAttTile + r;
            const uint64_t stat = h * p.tokens + it.start + min(row, it.len - 1);
            const float lse2 = p.lse_in[stat] * -(float)kLog2eD, delta = p.delta[stat];
            for (uint32_t t = 0; t < n; ++t, g = next_step(g)) {
                const uint32_t s_at = mine + (g & 1) * 128 + half * kHalf;
                if (!wait(kSFull + (g & 1), g >> 1 & 1)) break;
                float z[kHalf];
                load_half(s_at, z);
#pragma unroll
                for (int j = 0; j < (int)kHalf; ++j) z[j] = exp2_fast(fmaf(z[j], p.k2, lse2));
                if (waits) finish();
                if (!wait(kDpFull, g & 1)) break;
                float d[kHalf];
                load_half(mine + 256 + half * kHalf, d);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kDpRead));
#pragma unroll
                for (int j = 0; j < (int)kHalf; ++j) z[j] *= d[j] - delta;
                if (t + 1 == n) keep_columns(z, 0, row == 0 ? 0 : (int)r - (int)(half * kHalf) + 1);      // a query that sees one key has a constant weight
                if ((t + 1) * kAttTile > it.len)              // keys past the sequence
                    clear_rows(smem + (2 + g % kRing3) * kTileBytes, chunks, it.len - t * kAttTile, threadIdx.x - 128, 256);
                store_half(s_at, z);
                if (lane == 0) mbar_arrive(bar(kDsFull + (g & 1)));
            }
            out = row < it.len ? p.dq + ((uint64_t)it.start + row) * p.dq_ld + h * p.head_dim : nullptr;
            waits = true;
        }
        if (ok && waits) finish();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    const bool failed = *gave_up;
    if (failed) {      // as in the forward kernel
        if ((warp == 1 || warp == 2) && elect_lane()) {      // the lanes that issued them
            mma_commit<1>(bar(kLast));
            for (uint32_t i = 0; i < kWaitTries && !mbar_try_wait(bar(kLast), 0); ++i) {}
        }
        if (threadIdx.x == 0) {
            uint32_t left = kWaitTries;
            drain_loads(bar(kKFull), kRing3, s_taken[0], s_issued[0], left);
            drain_loads(bar(kVFull), kRing2, s_taken[1], s_issued[1], left);
            drain_loads(bar(kQFull), 1, s_taken[2], s_issued[2], left);
        }
        __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) tmem_free<1>(tmem, 512);
    wait_for_earlier();        // the first pass may still run; what follows in the stream must find both done
    if (threadIdx.x == 0 && failed && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_TIMEOUT);
}

// ---- dk, dv -----------------------------------------------------------------------------------------------------
// A key tile's work: for each query head of the group, the query tiles from its own to the sequence's last.
struct DkvWork {
    uint32_t start, len, kv_head, tile, tiles, n;     // tiles: of queries per head; n: in all
    uint32_t head, heads;                             // the first query head, and how many
    uint32_t piece;                                   // where the group is cut: which of all pieces
};

// it: an item of the list, which falls in the number of tiles in front: taken from the other end, in the number of tiles behind.  A
// group cut into 1 << cut parts is that many pieces of work, one behind the other.  unit: which part of the tile's work, and, where groups
// are cut, 65536 times which of all pieces.
__device__ __forceinline__ DkvWork dkv_work(const AttParams& p, const PlanItem& it, uint32_t unit, uint32_t cut) {
    DkvWork f;
    f.piece = unit >> 16;
    f.heads = p.group >> cut;
    f.head = (unit & 0xFFFF) * f.heads;
    f.kv_head = (unit & 0xFFFF) >> cut;
    f.start = it.start;
    f.len = it.len;
    f.tiles = it.tile + 1;
    f.tile = (it.len + kAttTile - 1) / kAttTile - f.tiles;
    f.n = f.tiles * f.heads;
    return f;
}

// The end of a piece whose group is cut, by one score warp for its 32 rows and its groups of 32 columns: leaves its sums in the workspace;
// the last part's warp adds up those of all parts, in their order, whichever came last.
__device__ __forceinline__ void add_parts(const AttParams& p, const DkvWork& f, uint32_t cut, uint32_t mine, __nv_bfloat16* dv, __nv_bfloat16* dk,
                                          uint32_t half, bool valid) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32 - 4;
    // four columns of all rows side by side
    auto place = [&](uint32_t piece, uint32_t which, uint32_t c) {
        return p.parts + (uint64_t)piece * kPartFloats + ((warp * 2 + which) * 2 + c / 64) * 1024 + lane * 4;
    };
    for (uint32_t which = 0; which < 2; ++which)
        for (uint32_t c = half * 32; c < p.head_dim; c += 64) {
            uint32_t v[32];
            tmem_load32(mine + (which ? 384 : 256) + c, v);
            tmem_load_wait(v);
            uint4* to = reinterpret_cast<uint4*>(place(f.piece, which, c));
#pragma unroll
            for (int i = 0; i < 8; ++i) to[32 * i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
    __threadfence();
    __syncwarp();
    const uint32_t parts = 1u << cut, first = f.piece >> cut << cut;
    const uint32_t before = __shfl_sync(0xFFFFFFFFu, lane == 0 ? atomicAdd(p.parts_done + (f.piece >> cut) * 8 + warp, 1u) : 0u, 0);
    if (before + 1 != parts) return;
    __threadfence();
    for (uint32_t which = 0; which < 2; ++which)
        for (uint32_t c = half * 32; c < p.head_dim; c += 64) {
            float sum[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[i] = 0.f;
#pragma unroll 2
            for (uint32_t k = 0; k < parts; ++k) {
                const float4* from = reinterpret_cast<const float4*>(place(first + k, which, c));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float4 x = __ldcg(from + 32 * i);
                    sum[4 * i] += x.x;
                    sum[4 * i + 1] += x.y;
                    sum[4 * i + 2] += x.z;
                    sum[4 * i + 3] += x.w;
                }
            }
            if (valid) {
                const float by = which ? p.scale : 1.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (c + 8 * i >= p.head_dim) break;
                    float o[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] = sum[8 * i + k] * by;
                    Raw8<__nv_bfloat16> x;
                    x.set(o);
                    x.store((which ? dk : dv) + c + 8 * i);
                }
            }
        }
}

// Tensor memory: transposed S at column 0 (p over it), transposed dP at 128 (dz over it), dv at 256, dk at 384.  While dz is made
// of one pair of tiles, the tensor cores add its dv up and make the next pair's S; while p is made of that, dk and the next dP.
__global__ void __launch_bounds__(kBwdThreads, 1)
    att_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_do, const __grid_constant__ AttParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];          // the swizzle's period
    enum { kQFull, kQEmpty = kRing3, kDoFull = 2 * kRing3, kDoEmpty = kDoFull + kRing2, kKvFull = kDoEmpty + kRing2, kKvEmpty, kSFull, kPFull, kDpFull, kDsFull,
           kAccFull, kTurn, kStatFull = kTurn + 2, kStatEmpty = kStatFull + 2, kWorkFull = kStatEmpty + 2, kWorkEmpty = kWorkFull + 2, kLast = kWorkEmpty + 2, kBars };
    __shared__ __align__(8) uint64_t s_bar[kBars];
    __shared__ uint32_t s_tmem, s_gave_up, s_issued[3], s_taken[3];         // loads of Q, dout, and K with V
    __shared__ uint4 s_work[2];            // as in att_dq_kernel
    __shared__ __align__(16) float s_stat[2][2][kAttTile];       // -lse log2(e) and -delta of a tile of queries
    const uint32_t k0 = smem_addr(smem), v0 = k0 + kTileBytes, qt0 = k0 + 2 * kTileBytes, dot0 = qt0 + kRing3 * kTileBytes;
    auto bar = [bar0 = smem_addr(s_bar)](uint32_t i) { return bar0 + 8 * i; };
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
        tma_prefetch_map(&map_do);
        for (uint32_t i = 0; i < kBars; ++i) {
            const bool warps = i == kPFull || i == kDsFull || i == kStatEmpty || i == kStatEmpty + 1;
            const bool both = (i >= kQEmpty && i < kDoFull) || (i >= kDoEmpty && i < kKvFull) || i == kKvEmpty || i == kAccFull || i == kLast;
            const bool all = i == kWorkEmpty || i == kWorkEmpty + 1;
            mbar_init(bar(i), warps ? kBwdWarps : all ? 3 + kBwdWarps : both ? 2 : 1);
        }
        s_gave_up = 0;
        for (uint32_t i = 0; i < 3; ++i) s_issued[i] = s_taken[i] = 0;
        mbar_arrive(bar(kTurn));               // the first turn is warp 1's
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&s_tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*(volatile uint32_t*)&s_tmem);
    volatile uint32_t* gave_up = &s_gave_up;
    wait_for_earlier();        // for delta
    if (threadIdx.x == 0) {    // the second pass needs no more than this one has now
        pass_on(p.next + 3);
        let_next_start();
    }
    const uint32_t cut = p.next[2];
    const uint32_t total = plan_ok(p) ? reinterpret_cast<const PlanHead*>(p.plan)->tiles * (p.units << cut) : 0;
    const PlanItem* list = reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader);
    const uint32_t chunks = (p.head_dim + 63) / 64, tile_bytes = chunks * kChunkBytes;
    // The next piece of work, by a whole warp; false at the end, or where the wait runs out.
    auto take_work = [&](uint32_t& n, DkvWork& f) {
        if (!warp_wait(bar(kWorkFull + (n & 1)), n >> 1 & 1, p.wait_limit, gave_up)) return false;
        const uint4 w = s_work[n & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kWorkEmpty + (n & 1)));
        ++n;
        f = dkv_work(p, PlanItem{w.x, w.y, w.z, 0}, w.w, cut);
        return w.z != kNone;
    };

    if (warp < 4) {
        regs_down<kFewRegs>();
        if (warp == 0) {
            // ---- loads: one lane ----
            uint32_t q_issued = 0, do_issued = 0, kv_issued = 0, works = 0;
            RingAt<kRing3> qa;
            RingAt<kRing2> da;
            bool ok = true;
            DkvWork f;
            while (ok && take_work(works, f)) {
                if (lane == 0 && (ok = mbar_wait(bar(kKvEmpty), (kv_issued & 1) ^ 1, p.wait_limit, gave_up))) {
                    mbar_expect_tx(bar(kKvFull), 2 * tile_bytes);
                    load_rows(k0, &map_k, chunks, f.kv_head, f.start + f.tile * kAttTile, bar(kKvFull));
                    load_rows(v0, &map_v, chunks, f.kv_head, f.start + f.tile * kAttTile, bar(kKvFull));
                    ++kv_issued;
                    for (uint32_t h = f.head; h < f.head + f.heads && ok; ++h)
                        for (uint32_t t = f.tile; t < f.tile + f.tiles; ++t) {
                            if (!(ok = mbar_wait(bar(kQEmpty + qa.i), qa.phase ^ 1, p.wait_limit, gave_up))) break;
                            mbar_expect_tx(bar(kQFull + qa.i), tile_bytes);
                            load_rows(qt0 + qa.i * kTileBytes, &map_q, chunks, h, f.start + t * kAttTile, bar(kQFull + qa.i));
                            qa.next();
                            ++q_issued;
                            if (!(ok = mbar_wait(bar(kDoEmpty + da.i), da.phase ^ 1, p.wait_limit, gave_up))) break;
                            mbar_expect_tx(bar(kDoFull + da.i), tile_bytes);
                            load_rows(dot0 + da.i * kTileBytes, &map_do, chunks, h, f.start + t * kAttTile, bar(kDoFull + da.i));
                            da.next();
                            ++do_issued;
                        }
                }
                ok = __all_sync(0xFFFFFFFFu, ok);
            }
            if (lane == 0) {
                s_issued[0] = q_issued;
                s_issued[1] = do_issued;
                s_issued[2] = kv_issued;
            }
        } else if (warp == 1 || warp == 2) {
            // ---- products: the whole warp waits, one lane issues.  Warp 1 has what reads and writes S and p (S of the next step behind dv
            // of this one), warp 2 what reads and writes dP and dz (dk, the next dP).  An issue blocks until the tensor cores are
            // nearly through with it: one waits for barriers while the other one issues, and they take turns ----
            const bool first = warp == 1;
            const uint32_t desc_s = mma_desc(kAttTile, kAttTile, false, false), steps = (p.head_dim + 15) / 16;
            const uint32_t desc_d = mma_desc(kAttTile, steps * 16, false, true);
            const uint32_t scores_at = first ? tmem : tmem + 128, sums_at = first ? tmem + 256 : tmem + 384, own = first ? k0 : v0;
            const uint32_t made_bar = first ? kSFull : kDpFull, ready_bar = first ? kPFull : kDsFull;
            uint32_t kv_taken = 0, g = 0, turns = 0, taken = 0;
            RingAt<kRing3> qa;                  // warp 1: the next tile for S; warp 2: the tile for dk
            RingAt<kRing2> da;                  // warp 1: the tile for dv; warp 2: the next tile for dP
            bool ok = true;
            auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(bar(b), parity, p.wait_limit, gave_up); };
            uint32_t works = 0;
            DkvWork f;
            while (ok && take_work(works, f)) {
                const int n = (int)f.n;
                if (!wait(kKvFull, kv_taken & 1)) break;
                ++kv_taken;
                // step -1 makes the first scores; step j adds step j's product up and makes the scores of the next one
                for (int j = -1; j < n && ok; ++j) {
                    const bool more = j + 1 < n;
                    // made from, and added up with: a tile of q and one of dout, or the other way round
                    uint32_t from = 0, from_release = 0, with = 0, with_release = 0;
                    if (more) {
                        if (!(first ? wait(kQFull + qa.i, qa.phase) : wait(kDoFull + da.i, da.phase))) break;
                        from = uniform(first ? qt0 + qa.i * kTileBytes : dot0 + da.i * kTileBytes);
                        from_release = uniform(first ? bar(kQEmpty + qa.i) : bar(kDoEmpty + da.i));
                        if (first) qa.next(); else da.next();
                        ++taken;
                    }
                    if (j >= 0) {
                        with = uniform(first ? dot0 + da.i * kTileBytes : qt0 + qa.i * kTileBytes);
                        with_release = uniform(first ? bar(kDoEmpty + da.i) : bar(kQEmpty + qa.i));
                        if (first) da.next(); else qa.next();
                    }
                    if (!wait(first ? kTurn : kTurn + 1, turns++ & 1)) break;
                    if (j >= 0 && !wait(ready_bar, g++ & 1)) break;       // last: what is behind it is the tensor cores' time
                    if (elect_lane()) {
                        if (j >= 0) mma_tile<kHalf>(sums_at, scores_at, with, desc_d, j != 0);
                        if (more) {
                            mma_rows(scores_at, own, from, steps, desc_s);
                            mma_commit<1>(bar(made_bar));
                        }
                        mbar_arrive(bar(first ? kTurn + 1 : kTurn));
                        if (j >= 0) mma_commit<1>(with_release);
                        if (more) mma_commit<1>(from_release);
                        if (j + 2 == n) mma_commit<1>(bar(kKvEmpty));
                        if (!more) mma_commit<1>(bar(kAccFull));
                    }
                }
            }
            if (lane == 0) {
                s_taken[first ? 0 : 1] = taken;
                if (first) s_taken[2] = kv_taken;
            }
        } else if (warp == 3) {
            // ---- work, from the counter that all CTAs share, and lse and delta of its tiles of queries ----
            uint32_t g = 0, works = 0;
            bool ok = true;
            auto draw = [&]() {
                const uint32_t w = __shfl_sync(0xFFFFFFFFu, lane == 0 ? atomicAdd(p.next, 1u) : 0u, 0);
                if (w >= total) return make_uint4(0, 0, kNone, 0);
                const PlanItem it = list[w / (p.units << cut)];
                return make_uint4(it.start, it.len, it.tile, w % (p.units << cut) | (cut ? w << 16 : 0));
            };
            auto publish = [&](const uint4& w) {
                if (!(ok = warp_wait(bar(kWorkEmpty + (works & 1)), (works >> 1 & 1) ^ 1, p.wait_limit, gave_up))) return;
                if (lane == 0) {
                    s_work[works & 1] = w;
                    mbar_arrive(bar(kWorkFull + (works & 1)));
                }
                ++works;
            };
            uint4 now = draw();
            publish(now);
            while (ok && now.z != kNone) {
                const DkvWork f = dkv_work(p, PlanItem{now.x, now.y, now.z, 0}, now.w, cut);
                uint32_t left = f.n;
                for (uint32_t h = f.head; h < f.head + f.heads && ok; ++h)
                    for (uint32_t t = f.tile; t < f.tile + f.tiles; ++t, ++g) {
                        const uint32_t row = t * kAttTile + lane * 4;
                        const uint64_t at = h * p.tokens + f.start + row;
                        float l[4], d[4];
                        // The next piece is drawn when this one's last loads are about to be issued: drawn earlier, a large piece would keep
                        // a second one waiting behind it while other CTAs have none.
                        if (left == min(f.n, 3u)) {
                            publish(now = draw());
                            if (!ok) break;
                        }
                        --left;
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) {
                            l[j] = row + j < f.len ? p.lse_in[at + j] * -(float)kLog2eD : 0.f;
                            d[j] = row + j < f.len ? -p.delta[at + j] : 0.f;
                        }
                        if (!(ok = warp_wait(bar(kStatEmpty + (g & 1)), (g >> 1 & 1) ^ 1, p.wait_limit, gave_up))) break;
                        *reinterpret_cast<float4*>(&s_stat[g & 1][0][lane * 4]) = make_float4(l[0], l[1], l[2], l[3]);
                        *reinterpret_cast<float4*>(&s_stat[g & 1][1][lane * 4]) = make_float4(d[0], d[1], d[2], d[3]);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(kStatFull + (g & 1)));
                    }
            }
        }
    } else {
        regs_up<kManyRegs>();
        // ---- scores: warp w may read the quarter w % 4 of tensor memory's lanes ----
        const uint32_t half = (warp - 4) / 4, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t mine = tmem + (quarter * 32 << 16), s_at = mine + half * kHalf, d_at = s_at + 128;
        uint32_t g = 0, done = 0;
        bool ok = true;
        auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(bar(b), parity, p.wait_limit, gave_up); };
        uint32_t works = 0;
        DkvWork f;
        while (ok && take_work(works, f)) {
            uint32_t t = f.tile;
            for (uint32_t j = 0; j < f.n; ++j, g = next_step(g)) {
                const uint32_t first = t * kAttTile + half * kHalf;       // query of this thread's first column
                const bool edge = t == f.tile || (t + 1) * kAttTile > f.len;
                const bool tail = (t + 1) * kAttTile > f.len;
                const float4* lse = reinterpret_cast<const float4*>(&s_stat[g & 1][0][half * kHalf]);
                const float4* delta = reinterpret_cast<const float4*>(&s_stat[g & 1][1][half * kHalf]);
                if (!wait(kStatFull + (g & 1), g >> 1 & 1) || !wait(kSFull, g & 1)) break;
                float z[kHalf];
                load_half(s_at, z);
#pragma unroll
                for (int c = 0; c < (int)kHalf / 4; ++c) {
                    const float4 l = lse[c];
                    z[4 * c] = exp2_fast(fmaf(z[4 * c], p.k2, l.x));
                    z[4 * c + 1] = exp2_fast(fmaf(z[4 * c + 1], p.k2, l.y));
                    z[4 * c + 2] = exp2_fast(fmaf(z[4 * c + 2], p.k2, l.z));
                    z[4 * c + 3] = exp2_fast(fmaf(z[4 * c + 3], p.k2, l.w));
                }
                if (edge) {                   // on the diagonal, or past the sequence: columns [low, high) are seen
                    const int low = (int)(f.tile * kAttTile + r) - (int)first, high = (int)f.len - (int)first;
                    keep_columns(z, low, high);
                }
                if ((t + 1) * kAttTile > f.len) {             // rows past the sequence, of q and of dout
                    if (!wait(kDoFull + g % kRing2, g / kRing2 & 1)) break;
                    clear_rows(smem + (2 + g % kRing3) * kTileBytes, chunks, f.len - t * kAttTile, threadIdx.x - 128, 256);
                    clear_rows(smem + (2 + kRing3 + g % kRing2) * kTileBytes, chunks, f.len - t * kAttTile, threadIdx.x - 128, 256);
                }
                store_half(s_at, z);
                if (lane == 0) mbar_arrive(bar(kPFull));
                if (!wait(kDpFull, g & 1)) break;
                float d[kHalf];
                load_half(d_at, d);
#pragma unroll
                for (int c = 0; c < (int)kHalf / 4; ++c) {
                    const float4 l = delta[c];
                    z[4 * c] *= d[4 * c] + l.x;
                    z[4 * c + 1] *= d[4 * c + 1] + l.y;
                    z[4 * c + 2] *= d[4 * c + 2] + l.z;
                    z[4 * c + 3] *= d[4 * c + 3] + l.w;
                }
                // 0 * what lies past the sequence; a query that sees one key has a constant weight
                if (tail) keep_columns(z, 0, (int)f.len - (int)first);
                if (first == 0) z[0] = 0.f;
                store_half(d_at, z);
                if (lane == 0) {
                    mbar_arrive(bar(kDsFull));
                    mbar_arrive(bar(kStatEmpty + (g & 1)));
                }
                if (++t == f.tile + f.tiles) t = f.tile;
            }
            if (!ok || !wait(kAccFull, done++ & 1)) break;
            const uint32_t row = f.tile * kAttTile + r;
            const uint64_t at = (uint64_t)f.start + row;
            __nv_bfloat16 *dv = p.dv + at * p.dv_ld + f.kv_head * p.head_dim, *dk = p.dk + at * p.dk_ld + f.kv_head * p.head_dim;
            if (cut == 0) {
                for (uint32_t c = half * 32; c < p.head_dim; c += 64) {
                    store_columns(dv, mine + 256, c, p.head_dim, 1.f, row < f.len, p.sectors);
                    store_columns(dk, mine + 384, c, p.head_dim, p.scale, row < f.len, p.sectors);
                }
            } else {
                add_parts(p, f, cut, mine, dv, dk, half, row < f.len);
            }
            tc_fence_before();
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    const bool failed = *gave_up;
    if (failed) {      // as in the forward kernel
        if ((warp == 1 || warp == 2) && elect_lane()) {      // the lanes that issued them
            mma_commit<1>(bar(kLast));
            for (uint32_t i = 0; i < kWaitTries && !mbar_try_wait(bar(kLast), 0); ++i) {}
        }
        if (threadIdx.x == 0) {
            uint32_t left = kWaitTries;
            drain_loads(bar(kQFull), kRing3, s_taken[0], s_issued[0], left);
            drain_loads(bar(kDoFull), kRing2, s_taken[1], s_issued[1], left);
            drain_loads(bar(kKvFull), 1, s_taken[2], s_issued[2], left);
        }
        __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) tmem_free<1>(tmem, 512);
    if (threadIdx.x == 0 && failed && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_TIMEOUT);
}

dte_status launch_attention_backward(const AttParams& params, const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, const dte_matrix* dout,
                                     uint64_t tiles, int device, int sms, cudaStream_t st) {
    dte_status s;
    CUtensorMap mq, mk, mv, md;
    if ((s = encode_heads(&mq, q, params.head_dim)) != DTE_OK) return s;
    if ((s = encode_heads(&mk, k, params.head_dim)) != DTE_OK) return s;
    if ((s = encode_heads(&mv, v, params.head_dim)) != DTE_OK) return s;
    if ((s = encode_heads(&md, dout, params.head_dim)) != DTE_OK) return s;
    static std::atomic<uint64_t> ready_dq{0}, ready_dkv{0};
    if ((s = allow_smem(att_dq_kernel, kBwdSmem, device, ready_dq)) != DTE_OK) return s;
    if ((s = allow_smem(att_dkv_kernel, kBwdSmem, device, ready_dkv)) != DTE_OK) return s;
    AttParams p = params;
    auto sectors = [&](const __nv_bfloat16* x, uint64_t ld) { return !(((uintptr_t)x | ld * 2 | p.head_dim * 2u) & 31u); };
    p.sectors = sectors(p.dq, p.dq_ld) && sectors(p.dk, p.dk_ld) && sectors(p.dv, p.dv_ld);
    const uint32_t heads = (uint32_t)(q->cols / p.head_dim);
    const bool narrow = p.head_dim <= 64;
    const uint64_t tokens_per_warp = narrow ? 32 : 16, warps = (p.tokens + tokens_per_warp - 1) / tokens_per_warp * heads, per_cta = kDeltaThreads / 32;
    const unsigned delta_grid = (unsigned)(1 + (warps + per_cta - 1) / per_cta);
    const unsigned grid = (unsigned)(tiles * heads < (uint64_t)sms ? tiles * heads : sms);      // of the first pass, too, whose groups may be cut
    if (narrow) att_delta_kernel<8><<<delta_grid, kDeltaThreads, 0, st>>>(p, heads);
    else att_delta_kernel<16><<<delta_grid, kDeltaThreads, 0, st>>>(p, heads);
    DTE_CUDA(cudaGetLastError());
    p.units = (uint32_t)(k->cols / p.head_dim);
    DTE_CUDA(launch_after(att_dkv_kernel, dim3(grid), kBwdThreads, kBwdSmem, st, mq, mk, mv, md, p));
    p.units = heads;
    DTE_CUDA(launch_after(att_dq_kernel, dim3(grid), kBwdThreads, kBwdSmem, st, mq, mk, mv, md, p));
    return DTE_OK;
}

}  // namespace dte
