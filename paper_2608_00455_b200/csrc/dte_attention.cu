// Causal attention over packed sequences with grouped heads, and its gradient.
#include "dte_ops.cuh"

namespace dte {

constexpr uint32_t kAttTile = 128;               // rows of a tile of queries or keys
constexpr uint32_t kMaxAttDim = 128;
constexpr uint32_t kPlanThreads = 1024;
constexpr uint32_t kPlanLevels = 4096;
constexpr uint64_t kPlanMagic = 0x6474652d61747431ull;
constexpr uint64_t kMaxAttTokens = 1ull << 24, kMaxSequences = 1ull << 20;
constexpr uint64_t kPlanHeader = 256;

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
};
static_assert(sizeof(PlanItem) == 16 && sizeof(PlanHead) <= kPlanHeader, "");

struct PlanParams {
    const void* starts;
    uint32_t starts_dtype;
    uint32_t n;                // sequences
    uint64_t tokens;
    uint8_t* plan;
    uint64_t pairs_at;
    uint64_t* flags;
};

// Lists the tiles of all sequences, the ones with the most keys in front of them first: CTAs that take them in turn
// finish together.  Tiles from kPlanLevels on count as equally long.  One CTA.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p) {
    __shared__ uint32_t s_at[2][kPlanLevels];        // tiles of a level, then where the next one of it goes
    __shared__ uint32_t s_warp[2][kPlanThreads / 32];
    __shared__ uint32_t s_bad;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    PlanHead* head = reinterpret_cast<PlanHead*>(p.plan);
    for (uint32_t i = threadIdx.x; i < kPlanLevels; i += kPlanThreads) s_at[0][i] = s_at[1][i] = 0;
    if (threadIdx.x == 0) s_bad = 0;
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
            *head = PlanHead{kPlanMagic, p.tokens, 0, 0, p.pairs_at};
            if (p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
        }
        return;
    }
    for (int round = 0; round < 2; ++round) {
        for (uint32_t i = warp; i < p.n; i += kPlanThreads / 32) {
            const uint32_t start = (uint32_t)load_id(p.starts, p.starts_dtype, i);
            const uint32_t len = (uint32_t)load_id(p.starts, p.starts_dtype, i + 1) - start;
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
        if (threadIdx.x == 0) *head = PlanHead{kPlanMagic, p.tokens, all[0], all[1], p.pairs_at};
        __syncthreads();
    }
}

struct AttParams {
    const uint8_t* plan;
    uint64_t plan_bytes, tokens;
    uint32_t head_dim, group;
    float scale;
    const __nv_bfloat16 *q, *k, *v, *o, *d_o;
    uint64_t q_ld, k_ld, v_ld, o_ld, do_ld;
    __nv_bfloat16 *out, *dq, *dk, *dv;
    uint64_t out_ld, dq_ld, dk_ld, dv_ld;
    float *lse, *delta;
    const float* lse_in;
    uint64_t* flags;
};

// Tiles of a plan that was made for this many tokens and lies in its buffer; another one's are none, and flagged.
__device__ __forceinline__ uint32_t plan_tiles(const AttParams& p) {
    const PlanHead* h = reinterpret_cast<const PlanHead*>(p.plan);
    if (h->magic == kPlanMagic && h->tokens == p.tokens && h->pairs_at + (uint64_t)h->pairs * sizeof(PlanItem) <= p.plan_bytes) return h->tiles;
    if (threadIdx.x + blockIdx.x + blockIdx.y == 0 && p.flags) atomicOr((unsigned long long*)p.flags, (unsigned long long)DTE_DEV_BOUNDS);
    return 0;
}

struct Row {
    float f[4];
    __device__ void load(const __nv_bfloat16* p, uint32_t lane, uint32_t d) {
        for (int j = 0; j < 4; ++j) f[j] = lane * 4 + j < d ? to_f(p[lane * 4 + j]) : 0.f;
    }
    __device__ void store(__nv_bfloat16* p, uint32_t lane, uint32_t d, float s) const {
        for (int j = 0; j < 4; ++j)
            if (lane * 4 + j < d) p[lane * 4 + j] = from_f<__nv_bfloat16>(f[j] * s);
    }
    __device__ float dot(const Row& o) const {
        float s = 0;
        for (int j = 0; j < 4; ++j) s = fmaf(f[j], o.f[j], s);
        return warp_sum(s);
    }
    __device__ void add(float a, const Row& o) { for (int j = 0; j < 4; ++j) f[j] = fmaf(a, o.f[j], f[j]); }
    __device__ void mul(float a) { for (int j = 0; j < 4; ++j) f[j] *= a; }
    __device__ void zero() { for (int j = 0; j < 4; ++j) f[j] = 0; }
};

__global__ void __launch_bounds__(256) att_forward_kernel(const AttParams p) {
    if (blockIdx.x >= plan_tiles(p)) return;
    const PlanItem it = reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader)[blockIdx.x];
    const uint32_t lane = threadIdx.x & 31, d = p.head_dim, h = blockIdx.y, kh = h / p.group;
    for (uint32_t r = it.tile * kAttTile + threadIdx.x / 32; r < min(it.len, (it.tile + 1) * kAttTile); r += 8) {
        const uint64_t row = it.start + r;
        Row q, k, o;
        q.load(p.q + row * p.q_ld + h * d, lane, d);
        o.zero();
        float top = -INFINITY, sum = 0;
        for (uint32_t j = 0; j <= r; ++j) {
            k.load(p.k + (uint64_t)(it.start + j) * p.k_ld + kh * d, lane, d);
            const float z = q.dot(k) * p.scale, now = fmaxf(top, z), from = now == -INFINITY ? 0.f : now;
            const float w = expf(z - from), keep = expf(top - from);
            k.load(p.v + (uint64_t)(it.start + j) * p.v_ld + kh * d, lane, d);
            o.mul(keep);
            o.add(w, k);
            sum = sum * keep + w;
            top = now;
        }
        o.store(p.out + row * p.out_ld + h * d, lane, d, 1.f / sum);
        if (p.lse && lane == 0) p.lse[h * p.tokens + row] = top + logf(sum);
    }
}

__global__ void __launch_bounds__(256) att_dq_kernel(const AttParams p) {
    if (blockIdx.x >= plan_tiles(p)) return;
    const PlanItem it = reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader)[blockIdx.x];
    const uint32_t lane = threadIdx.x & 31, d = p.head_dim, h = blockIdx.y, kh = h / p.group;
    for (uint32_t r = it.tile * kAttTile + threadIdx.x / 32; r < min(it.len, (it.tile + 1) * kAttTile); r += 8) {
        const uint64_t row = it.start + r;
        Row q, k, o, g;
        q.load(p.q + row * p.q_ld + h * d, lane, d);
        g.load(p.d_o + row * p.do_ld + h * d, lane, d);
        o.load(p.o + row * p.o_ld + h * d, lane, d);
        const float delta = g.dot(o), lse = p.lse_in[h * p.tokens + row];
        if (lane == 0) p.delta[h * p.tokens + row] = delta;
        o.zero();
        for (uint32_t j = 0; j <= r && r; ++j) {           // a query that sees one key: its weight is constant
            Row v;
            k.load(p.k + (uint64_t)(it.start + j) * p.k_ld + kh * d, lane, d);
            v.load(p.v + (uint64_t)(it.start + j) * p.v_ld + kh * d, lane, d);
            o.add(expf(q.dot(k) * p.scale - lse) * (g.dot(v) - delta), k);
        }
        if (p.dq) o.store(p.dq + row * p.dq_ld + h * d, lane, d, p.scale);
    }
}

__global__ void __launch_bounds__(256) att_dkv_kernel(const AttParams p) {
    if (blockIdx.x >= plan_tiles(p)) return;
    const PlanItem it = reinterpret_cast<const PlanItem*>(p.plan + kPlanHeader)[blockIdx.x];
    const uint32_t lane = threadIdx.x & 31, d = p.head_dim, kh = blockIdx.y;
    for (uint32_t j = it.tile * kAttTile + threadIdx.x / 32; j < min(it.len, (it.tile + 1) * kAttTile); j += 8) {
        const uint64_t row = it.start + j;
        Row k, v, dk, dv;
        k.load(p.k + row * p.k_ld + kh * d, lane, d);
        v.load(p.v + row * p.v_ld + kh * d, lane, d);
        dk.zero();
        dv.zero();
        for (uint32_t h = kh * p.group; h < (kh + 1) * p.group; ++h)
            for (uint32_t r = j; r < it.len; ++r) {
                Row q, g;
                const uint64_t at = it.start + r;
                q.load(p.q + at * p.q_ld + h * d, lane, d);
                g.load(p.d_o + at * p.do_ld + h * d, lane, d);
                const float w = expf(q.dot(k) * p.scale - p.lse_in[h * p.tokens + at]);
                dv.add(w, g);
                if (r) dk.add(w * (g.dot(v) - p.delta[h * p.tokens + at]), q);
            }
        dk.store(p.dk + row * p.dk_ld + kh * d, lane, d, p.scale);
        dv.store(p.dv + row * p.dv_ld + kh * d, lane, d, 1.f);
    }
}

// ---- host --------------------------------------------------------------------------------------------------
static uint64_t plan_tiles_most(uint64_t tokens, uint64_t n, uint64_t rows) { return tokens / rows + n; }
static uint64_t plan_pairs_at(uint64_t tokens, uint64_t n) { return kPlanHeader + plan_tiles_most(tokens, n, kAttTile) * sizeof(PlanItem); }

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
    if (!(scale > 0) || !std::isfinite((float)(scale * 1.44269504088896340736)))
        return op_fail(DTE_ERR_INVALID_ARG, "scale must be > 0 and, times log2(e), finite in fp32");
    if ((uintptr_t)flags & 7u) return op_fail(DTE_ERR_INVALID_ARG, "flags must be 8-byte aligned");
    if (!plan || ((uintptr_t)plan & (kWorkspaceAlign - 1)) || plan_bytes < kPlanHeader)
        return op_fail(DTE_ERR_INVALID_ARG, "plan is null, not 256-byte aligned or too small");
    return DTE_OK;
}

static AttParams att_params(const dte_matrix* q, const dte_matrix* k, const dte_matrix* v, uint32_t head_dim, const void* plan, uint64_t plan_bytes,
                            double scale, uint64_t* flags) {
    AttParams p = {};
    p.plan_bytes = plan_bytes;
    p.plan = static_cast<const uint8_t*>(plan);
    p.tokens = q->rows;
    p.head_dim = head_dim;
    p.group = (uint32_t)(q->cols / k->cols);
    p.scale = (float)scale;
    p.q = static_cast<const __nv_bfloat16*>(q->data);
    p.k = static_cast<const __nv_bfloat16*>(k->data);
    p.v = static_cast<const __nv_bfloat16*>(v->data);
    p.q_ld = q->ld;
    p.k_ld = k->ld;
    p.v_ld = v->ld;
    p.flags = flags;
    return p;
}

// Tiles that a plan of this size can list; one at least, to look at the plan.
static unsigned tiles_most(uint64_t plan_bytes, uint64_t tokens) {
    const uint64_t room = (plan_bytes - kPlanHeader) / sizeof(PlanItem), most = room < tokens ? room : tokens;
    return (unsigned)(most ? most : 1);
}

}  // namespace dte

using namespace dte;

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
    const unsigned tiles = tiles_most(plan_bytes, q->rows);
    if (q->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    AttParams p = att_params(q, k, v, head_dim, plan, plan_bytes, scale, flags);
    p.out = static_cast<__nv_bfloat16*>(out->data);
    p.out_ld = out->ld;
    p.lse = lse;
    att_forward_kernel<<<dim3(tiles, (unsigned)(q->cols / head_dim)), 256, 0, (cudaStream_t)cuda_stream>>>(p);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

extern "C" uint64_t dte_attention_backward_workspace_bytes(uint64_t tokens, uint64_t heads) {
    if (tokens > kMaxAttTokens || heads > 65535) return UINT64_MAX;
    return align_up(tokens * heads * sizeof(float), kWorkspaceAlign);
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
    const unsigned tiles = tiles_most(plan_bytes, q->rows);
    if (q->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    AttParams p = att_params(q, k, v, head_dim, plan, plan_bytes, scale, flags);
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
    cudaStream_t st = (cudaStream_t)cuda_stream;
    att_dq_kernel<<<dim3(tiles, (unsigned)heads), 256, 0, st>>>(p);
    DTE_CUDA(cudaGetLastError());
    att_dkv_kernel<<<dim3(tiles, (unsigned)(k->cols / head_dim)), 256, 0, st>>>(p);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}
