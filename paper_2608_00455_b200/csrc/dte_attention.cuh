// What the kernels of causal attention over packed sequences share: the plan, tiles of a head's rows and the products of two
// of them.
#pragma once

#include "dte_mma.cuh"
#include "dte_ops.cuh"

namespace dte {

constexpr uint32_t kAttTile = 128;               // rows of a tile of queries or keys
constexpr uint32_t kMaxAttDim = 128;
constexpr uint64_t kPlanMagic = 0x6474652d61747431ull;
constexpr uint64_t kMaxAttTokens = 1ull << 24, kMaxSequences = 1ull << 20;
constexpr uint64_t kPlanHeader = 256;
constexpr uint32_t kSms = 148;                   // for rules that choose an order of sums, which is the same on every device
constexpr uint32_t kMostParts = 4 * kSms;        // pieces that the gradient's first pass may cut its work into
constexpr uint32_t kPartFloats = 8 * 2 * 2 * 32 * 32;      // of a piece: score warps, dv and dk, groups of 32 columns, columns, rows
constexpr double kLog2eD = 1.44269504088896340736;

// One tile of one sequence.
struct PlanItem {
    uint32_t start, len;       // the sequence's rows
    uint32_t tile;             // tile of the sequence
    uint32_t pad;
};

struct PlanHead {
    uint64_t magic, tokens;
    uint32_t tiles, pairs;     // tiles of kAttTile rows, tiles of twice as many
    uint64_t pairs_at;         // where in the plan the second list starts; the first follows the header
    uint64_t steps;            // pairs of a tile of queries and one of keys that it sees
};
static_assert(sizeof(PlanItem) == 16 && sizeof(PlanHead) <= kPlanHeader, "");

constexpr uint32_t kChunkBytes = kAttTile * 128; // a tile's 64 columns: one swizzled operand of 16 KB
constexpr uint32_t kTileBytes = 2 * kChunkBytes; // up to 128 columns

struct AttParams {
    const uint8_t* plan;
    uint64_t plan_bytes, tokens;
    uint32_t head_dim, group;
    uint32_t units;            // of work per tile: pairs of query heads, or query heads
    bool pair_heads;
    uint32_t wait_limit;       // tries of a wait inside the kernel
    float scale, k2;           // k2: scale * log2(e)
    const __nv_bfloat16 *o, *d_o;          // q, k, v and d_o as operands of products come through tensor maps
    uint64_t o_ld, do_ld;
    __nv_bfloat16 *out, *dq, *dk, *dv;
    uint64_t out_ld, dq_ld, dk_ld, dv_ld;
    float *lse, *delta;
    // backwards
    uint32_t* next;            // the next piece of work of the two passes; then the exponent of how many parts the first one cuts a key head's group into;
                               // then the counter that hands memory on to the second one
    uint32_t* parts_done;      // per key tile and score warp, where groups are cut
    float* parts;              // what a part's score warps leave
    const float* lse_in;
    uint64_t* flags;
    bool sectors;              // every 16 columns of the outputs are a whole sector of 32 bytes
};

// The two passes over the scores of the backward pass.
dte_status launch_attention_backward(const AttParams& p, const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, const dte_matrix* dout,
                                     uint64_t tiles, int device, int sms, cudaStream_t st);
dte_status encode_heads(CUtensorMap* map, const dte_matrix* m, uint32_t head_dim);

#ifdef __CUDACC__
// Whether a plan was made for this many tokens and lies in its buffer; another one is flagged.
__device__ __forceinline__ bool plan_ok(const AttParams& p) {
    const PlanHead* h = reinterpret_cast<const PlanHead*>(p.plan);
    if (h->magic == kPlanMagic && h->tokens == p.tokens && h->pairs_at + (uint64_t)h->pairs * sizeof(PlanItem) <= p.plan_bytes) return true;
    if (threadIdx.x + blockIdx.x + blockIdx.y == 0 && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
    return false;
}

// Both chunks of a tile of 128 rows of a head.
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, uint32_t chunks, uint32_t head, uint32_t row, uint32_t bar) {
    for (uint32_t c = 0; c < chunks; ++c) tma_load_3d<1>(dst + c * kChunkBytes, map, (int)(c * 64), (int)head, (int)row, bar);
}

// Rows from `from` on of a tile in shared memory become zeros: rows of another sequence, or of none, would otherwise meet zeros of
// the other operand, and 0 * NaN is NaN.  By the `threads` threads that write that operand, before they say that it is there.
__device__ __forceinline__ void clear_rows(uint8_t* tile, uint32_t chunks, uint32_t from, uint32_t thread, uint32_t threads) {
    for (uint32_t c = 0; c < chunks; ++c)
        for (uint32_t i = from * 8 + thread; i < kAttTile * 8; i += threads)
            *reinterpret_cast<uint4*>(tile + c * kChunkBytes + i * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// A wait of a whole warp; all lanes go on or stop together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t limit, volatile uint32_t* gave_up) {
    bool ok = mbar_test_wait(bar, parity);
    if (!__all_sync(0xFFFFFFFFu, ok)) {
        ok = mbar_wait(bar, parity, limit, gave_up);
        ok = __all_sync(0xFFFFFFFFu, ok);
    }
    tc_fence_after();
    return ok;
}

// Place in a ring of N tiles.
template <uint32_t N>
struct RingAt {
    uint32_t i = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++i == N) {
            i = 0;
            phase ^= 1;
        }
    }
};

// Products are issued by one lane that the warp elects: the compiler then knows the branch, and with `uniform` the operands'
// addresses, to be the same for the whole warp, and keeps descriptors in uniform registers.  (An issue by `lane == 0`, descriptors made
// anew for each: 147 cycles per instruction that takes the tensor cores 64.)
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }

// D (+)= A B^T over head_dim: both operands rows of a head, along their columns.
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t steps, uint32_t desc) {
    const uint64_t da = operand_desc(a, 16), db = operand_desc(b, 16);
#pragma unroll
    for (uint32_t i = 0; i < kMaxAttDim / 16; ++i) {
        const uint32_t at = ((i / 4) * kChunkBytes + (i % 4) * 32) >> 4;
        if (i < steps) mma_bf16<1>(d, da + at, db + at, desc, i != 0);
    }
}

// D (+)= A B: A 128 x 128 in tensor memory, B 128 rows of a head.  HALF: columns of tensor memory from A's first 64 bf16 to the
// other 64.
template <uint32_t HALF>
__device__ __forceinline__ void mma_tile(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool add) {
    const uint64_t db = operand_desc(b, kChunkBytes);
#pragma unroll
    for (uint32_t i = 0; i < kAttTile / 16; ++i) mma_bf16_tmem(d, a + (i / 4) * HALF + (i % 4) * 8, db + (i * 2048 >> 4), desc, add || i != 0);
}

// Columns c .. c + 31 of this thread's row in tensor memory, times by, as bf16.  Every lane writes to another row: whole sectors where
// the rows allow it.
__device__ __forceinline__ void store_columns(__nv_bfloat16* out, uint32_t tmem, uint32_t c, uint32_t head_dim, float by, bool valid, bool sectors) {
    uint32_t v[32];
    tmem_load32(tmem + c, v);
    tmem_load_wait(v);
    if (!valid) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(__uint_as_float(v[16 * j + 2 * i]) * by, __uint_as_float(v[16 * j + 2 * i + 1]) * by);
        const uint32_t at = c + 16 * j;
        if (sectors && at < head_dim) {
            store32(out + at, w);
        } else {
            uint4* to = reinterpret_cast<uint4*>(out + at);
            if (at < head_dim) to[0] = make_uint4(w[0], w[1], w[2], w[3]);
            if (at + 8 < head_dim) to[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

// The pieces of work of this CTA: item w / units of the list and unit w % units of it, for the w of each of its rounds.  The list is in
// falling order of work, and every other round runs backwards, so that the shares come out even.  The next item is read while the
// one in front is worked on.
struct Turns {
    const PlanItem* list;
    uint32_t total, units, round, w;
    PlanItem ahead;            // item of w, if w < total
    __device__ __forceinline__ Turns(const PlanItem* list_, uint32_t total_, uint32_t units_) : list(list_), total(total_), units(units_), round(0) { look(); }
    __device__ __forceinline__ void look() {
        w = round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        if (w < total) ahead = list[w / units];
    }
    __device__ __forceinline__ bool more() const { return w < total; }      // past the end, no later round has work either
    __device__ __forceinline__ uint32_t unit() const { return w % units; }
    __device__ __forceinline__ void take(PlanItem& it, uint32_t& unit_) {
        it = ahead;
        unit_ = unit();
        ++round;
        look();
    }
};

// Waits for the loads that no product has waited for, after a wait that ran out: load i signals the barrier at
// bars + 8 * (i % n) for the (i / n)-th time.
__device__ __forceinline__ void drain_loads(uint32_t bars, uint32_t n, uint32_t taken, uint32_t issued, uint32_t& left) {
    for (uint32_t i = taken; i < issued; ++i)
        while (left && !mbar_try_wait(bars + 8 * (i % n), i / n & 1)) --left;
}
#endif  // __CUDACC__

}  // namespace dte
