// Causal attention over packed sequences with grouped heads: the plan, the forward pass, and the entry points of both passes.
//   z = scale q k^T over the keys at or before a query in its sequence,  lse = log sum exp z,  out = sum exp(z - lse) v
// in one pass over the keys with the running maximum and sum, scores never stored.
//
// Bound by the tensor cores (4 head_dim operations per head and pair of a query and a key that it sees) for long sequences, by what a
// tile costs beside its products for short ones.  Measured, heads of 128: 32768 tokens, 32 heads on 8: 8.1 ms in a loop, 1.09 PFLOP/s
// at the power limit, and 7.1 to 7.4 ms = 1.2 PFLOP/s over ten calls (a bf16 library product: 1.39 and 1.69); 8192 tokens in 19
// sequences, 32 heads on 4: 81 to 84 us (0.58 PFLOP/s); 77 tokens: 8.3 us; heads of 64, 32 on 8: 32768 tokens 6.0 ms (0.73 PFLOP/s: half the
// products for the same exponentials), 8192 in 19 sequences 69 us.  A step of two slots takes 3600 cycles of which the tensor cores
// work 2048; a slot's own chain is 1750 of softmax, 1024 of products, and 600 of barriers and waiting for its turn.
#include <atomic>

#include "dte_attention.cuh"

namespace dte {

constexpr uint32_t kPlanThreads = 1024;
constexpr uint32_t kPlanLevels = 4096;
// the gradient's groups are cut by the longest tile, the list's first: its place is certain wherever so few tiles are cut
static_assert(kPlanLevels > kMostParts, "");

struct PlanParams {
    const void* starts;
    uint32_t starts_dtype;
    uint32_t n;                // sequences
    uint64_t tokens;
    uint8_t* plan;
    uint64_t pairs_at;
    uint64_t* flags;
};

// Lists the tiles of all sequences, and the pairs of tiles that an odd group of heads takes, the ones with the most keys in front of them
// first: CTAs that take them in turn finish together.  Tiles from kPlanLevels on count as equally long.  One CTA, a warp per sequence,
// bound by the latency of the starts' loads: 6 us for 19 sequences, 53 for 1000, 4.7 ms for 100000.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p) {
    __shared__ uint32_t s_at[2][kPlanLevels];        // tiles of a level, then where the next one of it goes
    __shared__ uint32_t s_warp[2][kPlanThreads / 32];
    __shared__ uint32_t s_bad;
    __shared__ unsigned long long s_steps;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    PlanHead* head = reinterpret_cast<PlanHead*>(p.plan);
    for (uint32_t i = threadIdx.x; i < kPlanLevels; i += kPlanThreads) s_at[0][i] = s_at[1][i] = 0;
    if (threadIdx.x == 0) {
        s_bad = 0;
        s_steps = 0;
    }
    __syncthreads();
    bool bad = false;
    for (uint32_t i = threadIdx.x; i <= p.n; i += kPlanThreads) {
        const int64_t a = load_id(p.starts, p.starts_dtype, i);
        bad |= a < 0 || (uint64_t)a > p.tokens || (i < p.n && load_id(p.starts, p.starts_dtype, i + 1) < a);
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (s_bad) {
        if (threadIdx.x == 0) {
            *head = PlanHead{kPlanMagic, p.tokens, 0, 0, p.pairs_at, 0};
            if (p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
        }
        return;
    }
    for (int round = 0; round < 2; ++round) {
        for (uint32_t i = warp; i < p.n; i += kPlanThreads / 32) {
            const uint32_t start = (uint32_t)load_id(p.starts, p.starts_dtype, i);
            const uint32_t len = (uint32_t)load_id(p.starts, p.starts_dtype, i + 1) - start, tiles = (len + kAttTile - 1) / kAttTile;
            if (round == 0 && lane == 0) atomicAdd(&s_steps, (unsigned long long)tiles * (tiles + 1) / 2);
            for (uint32_t which = 0; which < 2; ++which) {
                const uint32_t rows = kAttTile << which;
                PlanItem* list = reinterpret_cast<PlanItem*>(p.plan + (which ? p.pairs_at : kPlanHeader));
                for (uint32_t t = lane; t * rows < len; t += 32) {
                    const uint32_t at = atomicAdd(&s_at[which][min(t, kPlanLevels - 1)], 1u);
                    if (round) list[at] = PlanItem{start, len, t, 0};
                }
            }
        }
        __syncthreads();
        if (round) break;
        // counts -> first place of each level, the highest level first
        constexpr uint32_t kPer = kPlanLevels / kPlanThreads;
        uint32_t before[2];
        for (uint32_t which = 0; which < 2; ++which) {
            uint32_t mine = 0;
            for (uint32_t j = 0; j < kPer; ++j) mine += s_at[which][kPlanLevels - 1 - (threadIdx.x * kPer + j)];
            uint32_t inc = mine;
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
                if (lane >= (uint32_t)o) inc += v;
            }
            if (lane == 31) s_warp[which][warp] = inc;
            before[which] = inc - mine;
        }
        __syncthreads();
        uint32_t all[2] = {0, 0};
        for (uint32_t which = 0; which < 2; ++which) {
            for (uint32_t w = 0; w < kPlanThreads / 32; ++w) {
                before[which] += w < warp ? s_warp[which][w] : 0;
                all[which] += s_warp[which][w];
            }
            for (uint32_t j = 0; j < kPer; ++j) {
                uint32_t& at = s_at[which][kPlanLevels - 1 - (threadIdx.x * kPer + j)];
                const uint32_t count = at;
                at = before[which];
                before[which] += count;
            }
        }
        if (threadIdx.x == 0) *head = PlanHead{kPlanMagic, p.tokens, all[0], all[1], p.pairs_at, s_steps};
        __syncthreads();
    }
}

// ---- forward ------------------------------------------------------------------------------------------------
// One CTA per SM takes pairs of tiles of 128 queries that share keys and values: two query heads of one key head, or, where the
// group of query heads is odd, two neighbouring tiles of one head.  Each half of the pair ("slot") has its own
// accumulators in tensor memory and its own four softmax warps, so that the tensor cores work for one slot while the other
// one's exponentials are made.  Per tile of 128 keys and slot:
//   product warp   S = Q K^T into tensor memory                               -> kSFull
//   softmax warps  row maximum, P = exp2(S - m) as bf16 over S, sums in fp32  -> kPFull
//   product warp   O += P V, P straight from tensor memory
// A thread holds a whole row of S (tensor memory's lane), so no reduction crosses threads.  P is rounded to bf16, the operand type of the
// second product; the sum is made of what it was before.  Tried and left: a share of the exponentials by a polynomial on the fp32 pipes (7.33 to
// 7.46 ms against 7.27), S read from tensor memory twice instead of held (10.8), O of a finished tile read behind the next one's first
// softmax (92 us against 90 for the packed case).
// A warpgroup of which one warp loads and two issue products, then one per slot.  Registers: 168 each at launch, 384 * 168 = 64512
// in all; the first warpgroup gives up what the others, with whole rows of S in registers, take: 128 * (72 + 2 * 208) = 62464.
constexpr uint32_t kFwdThreads = 3 * 128;
constexpr int kFewRegs = 72, kManyRegs = 208;
constexpr uint32_t kFwdRing = 5;                  // tiles of K and V in flight, in turn
constexpr uint32_t kFwdSmem = (2 + kFwdRing) * kTileBytes;
// O is brought to a new maximum only when that has grown by more than 2^8: until then P is up to 2^8 instead of 1, which costs
// bf16 and fp32 nothing.
constexpr float kRescaleAbove = 8.f;

struct FwdWork {
    uint32_t start, len;
    uint32_t n[2], row0[2], head[2];     // per slot: tiles of keys (0: the slot is empty), first row, query head
    uint32_t kv_head, n_max;
};

__device__ __forceinline__ FwdWork fwd_work(const AttParams& p, Turns& turns) {
    PlanItem it;
    uint32_t unit;
    turns.take(it, unit);
    FwdWork f;
    f.start = it.start;
    f.len = it.len;
    if (p.pair_heads) {
        f.head[0] = 2 * unit;
        f.head[1] = 2 * unit + 1;
        f.row0[0] = f.row0[1] = it.tile * kAttTile;
        f.n[0] = f.n[1] = it.tile + 1;
    } else {
        f.head[0] = f.head[1] = unit;
        f.row0[0] = 2 * it.tile * kAttTile;
        f.row0[1] = f.row0[0] + kAttTile;
        f.n[0] = 2 * it.tile + 1;
        f.n[1] = f.row0[1] < it.len ? 2 * it.tile + 2 : 0;
    }
    f.kv_head = f.head[0] / p.group;
    f.n_max = max(f.n[0], f.n[1]);
    return f;
}

// This thread's row of S; on the diagonal, keys behind the row are hidden.
__device__ __forceinline__ void load_scores(uint32_t (&v)[4][32], uint32_t s_at, bool diagonal, uint32_t row) {
#pragma unroll
    for (int c = 0; c < 4; ++c) tmem_load32(s_at + c * 32, v[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) tmem_load_wait(v[c]);
    if (diagonal) {
#pragma unroll
        for (int j = 0; j < 128; ++j) v[j / 32][j % 32] = (uint32_t)j > row ? __float_as_uint(-INFINITY) : v[j / 32][j % 32];
    }
}

// The largest of a row and `top`, in four chains so that latencies overlap; a NaN spreads to the whole row through it.
__device__ __forceinline__ float row_max(const uint32_t (&v)[4][32], float top) {
    float high[4] = {top, top, top, top};
#pragma unroll
    for (int j = 0; j < 32; j += 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) high[c] = max3_nan(high[c], __uint_as_float(v[c][j]), __uint_as_float(v[c][j + 1]));
    return max3_nan(max3_nan(high[0], high[1], high[2]), high[3], high[3]);
}

// P of a row, as bf16 pairs, and its sum in fp32.
__device__ __forceinline__ float make_weights(const uint32_t (&v)[4][32], float k2, float from, uint32_t (&w)[64]) {
    const F2 by2 = f2(k2, k2), from2 = f2(from, from);
    F2 part[4] = {f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
    for (int j = 0; j < 64; ++j) {
        const uint32_t* x = &v[j / 16][j % 16 * 2];
        const F2 arg = f2_fma(f2(__uint_as_float(x[0]), __uint_as_float(x[1])), by2, from2);
        float lo, hi;
        f2_get(arg, lo, hi);
        const F2 e = f2(exp2_fast(lo), exp2_fast(hi));
        part[j % 4] = f2_add(part[j % 4], e);
        w[j] = pack_bf16(e);
    }
    float even, odd;
    f2_get(f2_add(f2_add(part[0], part[1]), f2_add(part[2], part[3])), even, odd);
    return even + odd;
}

__global__ void __launch_bounds__(kFwdThreads, 1)
    att_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];          // the swizzle's period
    __shared__ __align__(8) uint64_t s_bar[2 * kFwdRing + 12 + 1];
    __shared__ uint32_t s_tmem, s_gave_up, s_issued, s_taken[2], s_q_issued[2], s_q_taken[2];
    const uint32_t q0 = smem_addr(smem), ring0 = q0 + 2 * kTileBytes, bar0 = smem_addr(s_bar);
    auto full = [&](uint32_t i) { return bar0 + 8 * i; };
    auto empty = [&](uint32_t i) { return bar0 + 8 * (kFwdRing + i); };
    auto bar = [&](uint32_t kind, uint32_t s) { return bar0 + 8 * (2 * kFwdRing + 2 * kind + s); };
    enum { kQFull, kQEmpty, kSFull, kPFull, kOFull, kTurn };
    const uint32_t last_bar = bar0 + 8 * (2 * kFwdRing + 12);
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    // asked for before the setup, needed behind it
    const PlanHead* head = reinterpret_cast<const PlanHead*>(p.plan);
    const uint32_t items = plan_ok(p) ? (p.pair_heads ? head->tiles : head->pairs) : 0, total = items * p.units;
    const PlanItem* list = reinterpret_cast<const PlanItem*>(p.plan + (p.pair_heads ? kPlanHeader : items ? head->pairs_at : 0));

    if (threadIdx.x == 0) {
        tma_prefetch_map(&map_q);
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
        for (uint32_t i = 0; i < kFwdRing; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 2);
        }
        for (uint32_t s = 0; s < 2; ++s) {
            mbar_init(bar(kQFull, s), 1);
            mbar_init(bar(kQEmpty, s), 1);
            mbar_init(bar(kSFull, s), 1);
            mbar_init(bar(kPFull, s), 4);
            mbar_init(bar(kOFull, s), 1);
            mbar_init(bar(kTurn, s), 1);
        }
        mbar_init(last_bar, 2);
        s_gave_up = s_issued = s_taken[0] = s_taken[1] = s_q_issued[0] = s_q_issued[1] = s_q_taken[0] = s_q_taken[1] = 0;
        mbar_arrive(bar(kTurn, 0));            // the first turn is slot 0's
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&s_tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*(volatile uint32_t*)&s_tmem);         // S of the slots at columns 0 and 128, O at 256 and 384
    volatile uint32_t* gave_up = &s_gave_up;
    const uint32_t chunks = (p.head_dim + 63) / 64, tile_bytes = chunks * kChunkBytes;

    if (warp < 4) {
        regs_down<kFewRegs>();
        if (warp == 0 && lane == 0) {
            // ---- loads ----
            uint32_t issued = 0, q_issued[2] = {0, 0};
            RingAt<kFwdRing> at;
            bool ok = true;
            auto load = [&](const CUtensorMap* map, uint32_t head_at, uint32_t row) {
                if (!(ok = ok && mbar_wait(empty(at.i), at.phase ^ 1, p.wait_limit, gave_up))) return;
                mbar_expect_tx(full(at.i), tile_bytes);
                load_rows(ring0 + at.i * kTileBytes, map, chunks, head_at, row, full(at.i));
                at.next();
                ++issued;
            };
            for (Turns work(list, total, p.units); work.more() && ok;) {
                const FwdWork f = fwd_work(p, work);
#pragma unroll
                for (uint32_t s = 0; s < 2; ++s) {
                    if (!f.n[s] || !ok) continue;
                    if (!(ok = mbar_wait(bar(kQEmpty, s), (q_issued[s] & 1) ^ 1, p.wait_limit, gave_up))) continue;
                    mbar_expect_tx(bar(kQFull, s), tile_bytes);
                    load_rows(q0 + s * kTileBytes, &map_q, chunks, f.head[s], f.start + f.row0[s], bar(kQFull, s));
                    ++q_issued[s];
                    if (s == 0) load(&map_k, f.kv_head, f.start);
                }
                for (uint32_t t = 0; t < f.n_max && ok; ++t) {
                    load(&map_v, f.kv_head, f.start + t * kAttTile);
                    if (t + 1 < f.n_max) load(&map_k, f.kv_head, f.start + (t + 1) * kAttTile);
                }
            }
            s_issued = issued;
            s_q_issued[0] = q_issued[0];
            s_q_issued[1] = q_issued[1];
        } else if (warp == 1 || warp == 2) {
            // ---- matrix products of one slot: the whole warp waits, one lane issues ----
            // An issue blocks until the tensor cores are nearly through with it, so whatever else the issuing warp does leaves them
            // idle: there is a warp per slot, and one waits for barriers while the other one issues.  They take turns, so that
            // products run as wholes and the slots stay half a step apart (without turns: 9.15 ms; one warp for both: 7.5).
            const uint32_t s = warp - 1, s_at = tmem + s * 128, o_at = tmem + 256 + s * 128, qs = q0 + s * kTileBytes;
            const uint32_t desc_s = mma_desc(kAttTile, kAttTile, false, false);
            const uint32_t desc_o = mma_desc(kAttTile, (p.head_dim + 15) / 16 * 16, false, true), steps = (p.head_dim + 15) / 16;
            uint32_t taken = 0, q_taken = 0, p_taken = 0, turns = 0;
            RingAt<kFwdRing> at;
            bool ok = true;
            auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(b, parity, p.wait_limit, gave_up); };
            // the next tile of the ring: its address, and the barrier that lets it go
            auto take = [&](uint32_t& tile, uint32_t& release) {
                if (!wait(full(at.i), at.phase)) return;
                tile = uniform(ring0 + at.i * kTileBytes);
                release = uniform(empty(at.i));
                at.next();
                ++taken;
            };
            for (Turns work(list, total, p.units); work.more() && ok;) {
                const FwdWork f = fwd_work(p, work);
                const uint32_t n = s ? f.n[1] : f.n[0];
                uint32_t k = 0, k_release = 0, v = 0, v_release = 0;
                // step -1 makes the first scores; step t adds up the values of tile t and makes the scores of the next one.  A slot
                // that is through takes its turns and lets the tiles go, as the other one does.
                for (int t = -1; t < (int)f.n_max && ok; ++t) {
                    const bool more = t + 1 < (int)f.n_max, mine = t >= 0 && t < (int)n, next = t + 1 < (int)n;
                    if (t >= 0) take(v, v_release);
                    if (more) take(k, k_release);
                    if (t < 0 && n && wait(bar(kQFull, s), q_taken & 1)) ++q_taken;
                    if (!wait(bar(kTurn, s), turns++ & 1)) break;
                    if (mine && !wait(bar(kPFull, s), p_taken++ & 1)) break;      // last: what is behind it is the tensor cores' time
                    if (elect_lane()) {
                        if (mine) mma_tile<32>(o_at, s_at, v, desc_o, t != 0);
                        if (next) {
                            mma_rows(s_at, qs, k, steps, desc_s);
                            mma_commit<1>(bar(kSFull, s));
                        }
                        mbar_arrive(bar(kTurn, s ^ 1));
                        if (mine && !next) mma_commit<1>(bar(kOFull, s));
                        if (t + 2 == (int)n) mma_commit<1>(bar(kQEmpty, s));
                        if (t >= 0) mma_commit<1>(v_release);
                        if (more) mma_commit<1>(k_release);
                    }
                }
            }
            if (lane == 0) {
                s_taken[s] = taken;
                s_q_taken[s] = q_taken;
            }
        }
    } else {
        regs_up<kManyRegs>();
        // ---- softmax: warp w may read the quarter w % 4 of tensor memory's lanes ----
        const uint32_t s = (warp - 4) / 4, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lanes = quarter * 32 << 16, s_at = tmem + s * 128 + lanes, o_at = tmem + 256 + s * 128 + lanes;
        const float k2 = p.k2;
        uint32_t tiles = 0, items_done = 0, loads = 0;      // loads: tiles of keys and values of the work so far, modulo the ring's period
        bool ok = true;
        auto wait = [&](uint32_t b, uint32_t parity) { return ok = ok && warp_wait(b, parity, p.wait_limit, gave_up); };
        for (Turns work(list, total, p.units); work.more() && ok;) {
            const FwdWork f = fwd_work(p, work);
            const uint32_t first_load = loads;
            loads = (loads + 2 * f.n_max) % (2 * kFwdRing);
            const uint32_t n = s ? f.n[1] : f.n[0], head_at = s ? f.head[1] : f.head[0];
            if (!n) continue;
            const uint32_t row = (s ? f.row0[1] : f.row0[0]) + r;             // in its sequence
            float top = -INFINITY, sum = 0.f;               // top: what O and sum are relative to
            for (uint32_t t = 0; t < n; ++t) {
                if (!wait(bar(kSFull, s), tiles++ & 1)) break;
                const bool diagonal = t + 1 == n;
                uint32_t v[4][32], w[64];
                load_scores(v, s_at, diagonal, r);
                float peak = row_max(v, top);
                if (t == 0) top = peak;
                // P relative to the maximum of the tiles in front, made beside this tile's maximum; only where that has grown by much
                // (each row decides for itself, so that no row's rounding depends on its neighbours; a NaN counts, once) P is made again
                float part = make_weights(v, k2, top == -INFINITY ? 0.f : -top * k2, w);
                const bool grown = (peak - top) * k2 > kRescaleAbove || (peak != peak && top == top);
                if (__any_sync(0xFFFFFFFFu, grown)) {
                    const float by = grown ? exp2_fast((top - peak) * k2) : 1.f;
                    top = grown ? peak : top;
                    sum *= by;
                    for (uint32_t c = 0; c < p.head_dim; c += 32) {
                        uint32_t o[32];
                        tmem_load32(o_at + c, o);
                        tmem_load_wait(o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * by);
                        tmem_store32(o_at + c, o);
                    }
                    load_scores(v, s_at, diagonal, r);
                    part = make_weights(v, k2, top == -INFINITY ? 0.f : -top * k2, w);
                }
                sum += part;
                tmem_store64(s_at, w);
                if ((t + 1) * kAttTile > f.len) {           // values past the sequence; they lie where the load behind the keys' went
                    const uint32_t at = first_load + 2 * t + 1, i = at % kFwdRing;
                    if (!wait(full(i), at / kFwdRing & 1)) break;
                    clear_rows(smem + (2 + i) * kTileBytes, chunks, f.len - t * kAttTile, r, 128);
                }
                tmem_store_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kPFull, s));
            }
            if (!ok || !wait(bar(kOFull, s), items_done++ & 1)) break;
            const bool valid = row < f.len;
            const uint64_t at = (uint64_t)f.start + row;
            if (valid && p.lse) p.lse[head_at * p.tokens + at] = fmaf(top, p.scale, logf(sum));
            const float by = 1.f / sum;
            __nv_bfloat16* out = p.out + at * p.out_ld + head_at * p.head_dim;
            for (uint32_t c = 0; c < p.head_dim; c += 32) store_columns(out, o_at, c, p.head_dim, by, valid, p.sectors);
            tc_fence_before();
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    const bool failed = *gave_up;
    if (failed) {
        // A wait ran out: all roles have stopped.  What they left in flight ends here, again with a limit: the products, and every
        // load that no product has waited for.
        if ((warp == 1 || warp == 2) && elect_lane()) {      // the lanes that issued them
            mma_commit<1>(last_bar);
            for (uint32_t i = 0; i < kWaitTries && !mbar_try_wait(last_bar, 0); ++i) {}
        }
        if (threadIdx.x == 0) {
            uint32_t left = kWaitTries;
            drain_loads(full(0), kFwdRing, max(s_taken[0], s_taken[1]), s_issued, left);
            for (uint32_t s = 0; s < 2; ++s) drain_loads(bar(kQFull, s), 1, s_q_taken[s], s_q_issued[s], left);
        }
        __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) tmem_free<1>(tmem, 512);
    if (threadIdx.x == 0 && failed && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_TIMEOUT);
}

// ---- host --------------------------------------------------------------------------------------------------
static uint64_t plan_tiles_most(uint64_t tokens, uint64_t n, uint64_t rows) { return tokens / rows + n; }
static uint64_t plan_pairs_at(uint64_t tokens, uint64_t n) { return kPlanHeader + plan_tiles_most(tokens, n, kAttTile) * sizeof(PlanItem); }

// Tiles that a plan of this size can list; one at least, to look at the plan.
static uint64_t tiles_most(uint64_t plan_bytes, uint64_t tokens) {
    const uint64_t room = plan_bytes < kPlanHeader ? 0 : (plan_bytes - kPlanHeader) / sizeof(PlanItem), most = room < tokens ? room : tokens;
    return most ? most : 1;
}

static dte_status check_heads(const dte_matrix* m, const char* null_msg, uint32_t head_dim, uint64_t rows, bool output) {
    dte_status s;
    if ((s = check_matrix(m, null_msg, output)) != DTE_OK) return s;
    if (m->dtype != DTE_BF16) return op_fail(DTE_ERR_INVALID_ARG, "attention takes BF16 matrices");
    if (m->rows != rows) return op_fail(DTE_ERR_INVALID_ARG, "attention's matrices need one row per token");
    if (m->cols % head_dim) return op_fail(DTE_ERR_INVALID_ARG, "columns must be a multiple of head_dim");
    if (((uintptr_t)m->data & 15u) || (m->rows > 1 && (m->ld % 8 || m->ld < m->cols)))
        return op_fail(DTE_ERR_INVALID_ARG, "attention's matrices must be 16-byte aligned with ld >= cols, a multiple of 8");
    return DTE_OK;
}

static dte_status check_attention(const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, uint32_t head_dim, const void* plan,
                                  uint64_t plan_bytes, double scale, const uint64_t* flags) {
    dte_status s;
    if (head_dim == 0 || head_dim > kMaxAttDim || head_dim % 8) return op_fail(DTE_ERR_INVALID_ARG, "head_dim must be a multiple of 8 up to 128");
    if (!q) return op_fail(DTE_ERR_INVALID_ARG, "q is null");
    if ((s = check_heads(q, "q is null", head_dim, q->rows, false)) != DTE_OK) return s;
    if ((s = check_heads(k, "k is null", head_dim, q->rows, false)) != DTE_OK) return s;
    if ((s = check_heads(v, "v is null", head_dim, q->rows, false)) != DTE_OK) return s;
    if (k->cols != v->cols || q->cols % k->cols) return op_fail(DTE_ERR_INVALID_ARG, "query heads must be a multiple of k's heads, v must have k's");
    if (q->rows > kMaxAttTokens) return op_fail(DTE_ERR_INVALID_ARG, "at most 2^24 tokens");
    if (q->cols / head_dim > 65535) return op_fail(DTE_ERR_INVALID_ARG, "at most 65535 heads");
    if (tiles_most(plan_bytes, q->rows) * (q->cols / head_dim) >= (1ull << 31) || (q->rows / kAttTile + 1) * (q->cols / head_dim) >= (1ull << 31))
        return op_fail(DTE_ERR_INVALID_ARG, "tiles x heads are too many for one call");
    // a scale that fp32 holds as zero would make NaN of hidden scores (0 * infinity), a subnormal one has lost bits
    if (!(scale > 0) || !std::isnormal((float)scale) || !std::isfinite((float)(scale * kLog2eD)))
        return op_fail(DTE_ERR_INVALID_ARG, "scale must be > 0, a normal number in fp32 and, times log2(e), finite there");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if (!plan || ((uintptr_t)plan & (kWorkspaceAlign - 1)) || plan_bytes < kPlanHeader)
        return op_fail(DTE_ERR_INVALID_ARG, "plan is null, not 256-byte aligned or too small");
    return DTE_OK;
}

static std::atomic<uint32_t> g_att_wait_limit{kWaitTries};

// A matrix of heads as (column, head, token), read in boxes of 64 columns of one head and kAttTile tokens; columns past the
// head are zeros.
dte_status encode_heads(CUtensorMap* map, const dte_matrix* m, uint32_t head_dim) {
    const uint64_t ld = m->rows > 1 ? m->ld : m->cols;
    return encode_3d(map, m->data, {head_dim, m->cols / head_dim, m->rows}, {head_dim * 2ull, ld * 2}, {64, 1, kAttTile});
}

static AttParams att_params(const dte_matrix* q, const dte_matrix* k, uint32_t head_dim, const void* plan, uint64_t plan_bytes, double scale,
                            uint64_t* flags) {
    AttParams p = {};
    p.plan_bytes = plan_bytes;
    p.plan = static_cast<const uint8_t*>(plan);
    p.tokens = q->rows;
    p.head_dim = head_dim;
    p.group = (uint32_t)(q->cols / k->cols);
    p.scale = (float)scale;
    p.k2 = (float)(scale * kLog2eD);
    p.wait_limit = g_att_wait_limit.load(std::memory_order_relaxed);
    p.flags = flags;
    return p;
}

}  // namespace dte

using namespace dte;

extern "C" void dte_attention_set_wait_limit(uint32_t tries) {
    g_att_wait_limit.store(tries ? tries : kWaitTries, std::memory_order_relaxed);
}

extern "C" uint64_t dte_attention_plan_bytes(uint64_t tokens, uint64_t n_sequences) {
    if (tokens > kMaxAttTokens || n_sequences > kMaxSequences) return UINT64_MAX;       // refused by the call
    return align_up(plan_pairs_at(tokens, n_sequences) + plan_tiles_most(tokens, n_sequences, 2 * kAttTile) * sizeof(PlanItem), kWorkspaceAlign);
}

extern "C" dte_status dte_attention_plan(const dte_ids* starts, uint64_t tokens, void* plan, uint64_t plan_bytes, uint64_t* flags,
                                         int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_ids(starts)) != DTE_OK) return s;
    if (starts->count == 0) return op_fail(DTE_ERR_INVALID_ARG, "starts need one entry more than there are sequences");
    if (tokens > kMaxAttTokens || starts->count - 1 > kMaxSequences) return op_fail(DTE_ERR_INVALID_ARG, "at most 2^24 tokens and 2^20 sequences");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if ((s = check_workspace(plan, plan_bytes, dte_attention_plan_bytes(tokens, starts->count - 1))) != DTE_OK) return s;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    PlanParams p = {};
    p.starts = starts->data;
    p.starts_dtype = starts->dtype;
    p.n = (uint32_t)(starts->count - 1);
    p.tokens = tokens;
    p.plan = static_cast<uint8_t*>(plan);
    p.pairs_at = plan_pairs_at(tokens, p.n);
    p.flags = flags;
    plan_kernel<<<1, kPlanThreads, 0, (cudaStream_t)cuda_stream>>>(p);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

extern "C" dte_status dte_attention_forward(const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, uint32_t head_dim,
                                            const void* plan, uint64_t plan_bytes, double scale, const dte_matrix* out, float* lse,
                                            uint64_t* flags, int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_attention(q, k, v, head_dim, plan, plan_bytes, scale, flags)) != DTE_OK) return s;
    if ((s = check_heads(out, "out is null", head_dim, q->rows, true)) != DTE_OK) return s;
    if (out->cols != q->cols) return op_fail(DTE_ERR_INVALID_ARG, "out must have q's columns");
    if ((uintptr_t)lse & 3u) return op_fail(DTE_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    const uint64_t tiles = tiles_most(plan_bytes, q->rows);
    if (q->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    int sms = 0;
    if ((s = g.enter(device, &sms)) != DTE_OK) return s;
    AttParams p = att_params(q, k, head_dim, plan, plan_bytes, scale, flags);
    p.out = static_cast<__nv_bfloat16*>(out->data);
    p.out_ld = out->ld;
    p.lse = lse;
    p.sectors = !(((uintptr_t)out->data | out->ld * 2 | head_dim * 2u) & 31u);
    p.pair_heads = p.group % 2 == 0;
    p.units = (uint32_t)(q->cols / head_dim / (p.pair_heads ? 2 : 1));
    CUtensorMap mq, mk, mv;
    if ((s = encode_heads(&mq, q, head_dim)) != DTE_OK) return s;
    if ((s = encode_heads(&mk, k, head_dim)) != DTE_OK) return s;
    if ((s = encode_heads(&mv, v, head_dim)) != DTE_OK) return s;
    static std::atomic<uint64_t> ready{0};
    if ((s = allow_smem(att_forward_kernel, kFwdSmem, device, ready)) != DTE_OK) return s;
    const uint64_t work = (uint64_t)tiles * p.units;
    att_forward_kernel<<<(unsigned)(work < (uint64_t)sms ? work : sms), kFwdThreads, kFwdSmem, (cudaStream_t)cuda_stream>>>(mq, mk, mv, p);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

// Where everything lies in the backward pass's workspace: delta, the counters, and what cut groups need.
struct BackwardLayout {
    uint64_t next, parts_done, parts, total;
};

static BackwardLayout backward_layout(uint64_t tokens, uint64_t heads) {
    BackwardLayout l;
    const uint64_t most = tokens * heads < kMostParts ? tokens * heads : kMostParts;
    l.next = align_up(tokens * heads * sizeof(float), kWorkspaceAlign);
    l.parts_done = l.next + kWorkspaceAlign;
    l.parts = l.parts_done + align_up(most * 8 * sizeof(uint32_t), kWorkspaceAlign);
    l.total = l.parts + most * kPartFloats * sizeof(float);
    return l;
}

extern "C" uint64_t dte_attention_backward_workspace_bytes(uint64_t tokens, uint64_t heads) {
    if (tokens > kMaxAttTokens || heads > 65535) return UINT64_MAX;
    return backward_layout(tokens, heads).total;
}

extern "C" dte_status dte_attention_backward(const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, uint32_t head_dim,
                                             const dte_matrix* out, const float* lse, const dte_matrix* dout, const void* plan,
                                             uint64_t plan_bytes, double scale, const dte_matrix* dq, const dte_matrix* dk,
                                             const dte_matrix* dv, void* workspace, uint64_t workspace_bytes, uint64_t* flags,
                                             int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_attention(q, k, v, head_dim, plan, plan_bytes, scale, flags)) != DTE_OK) return s;
    if ((s = check_heads(out, "out is null", head_dim, q->rows, false)) != DTE_OK) return s;
    if ((s = check_heads(dout, "dout is null", head_dim, q->rows, false)) != DTE_OK) return s;
    if ((s = check_heads(dq, "dq is null", head_dim, q->rows, true)) != DTE_OK) return s;
    if ((s = check_heads(dk, "dk is null", head_dim, q->rows, true)) != DTE_OK) return s;
    if ((s = check_heads(dv, "dv is null", head_dim, q->rows, true)) != DTE_OK) return s;
    if (out->cols != q->cols || dout->cols != q->cols || dq->cols != q->cols || dk->cols != k->cols || dv->cols != k->cols)
        return op_fail(DTE_ERR_INVALID_ARG, "out, dout and dq must have q's columns, dk and dv k's");
    if (q->rows && (!lse || ((uintptr_t)lse & 3u))) return op_fail(DTE_ERR_INVALID_ARG, "lse is null or not 4-byte aligned");
    const uint64_t heads = q->cols / head_dim;
    if ((s = check_workspace(workspace, workspace_bytes, dte_attention_backward_workspace_bytes(q->rows, heads))) != DTE_OK) return s;
    const uint64_t tiles = tiles_most(plan_bytes, q->rows);
    if (q->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    int sms = 0;
    if ((s = g.enter(device, &sms)) != DTE_OK) return s;
    AttParams p = att_params(q, k, head_dim, plan, plan_bytes, scale, flags);
    p.o = static_cast<const __nv_bfloat16*>(out->data);
    p.d_o = static_cast<const __nv_bfloat16*>(dout->data);
    p.o_ld = out->ld;
    p.do_ld = dout->ld;
    p.dq = static_cast<__nv_bfloat16*>(dq->data);
    p.dk = static_cast<__nv_bfloat16*>(dk->data);
    p.dv = static_cast<__nv_bfloat16*>(dv->data);
    p.dq_ld = dq->ld;
    p.dk_ld = dk->ld;
    p.dv_ld = dv->ld;
    p.lse_in = lse;
    p.delta = static_cast<float*>(workspace);
    const BackwardLayout l = backward_layout(q->rows, heads);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.next = reinterpret_cast<uint32_t*>(ws + l.next);
    p.parts_done = reinterpret_cast<uint32_t*>(ws + l.parts_done);
    p.parts = reinterpret_cast<float*>(ws + l.parts);
    return launch_attention_backward(p, q, k, v, dout, tiles, device, sms, (cudaStream_t)cuda_stream);
}
