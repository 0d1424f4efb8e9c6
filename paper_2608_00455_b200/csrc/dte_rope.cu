// Rotary positions: pairs of a head's columns turned by position * frequency, queries and keys in one launch.
//
// Bound by memory: every element is read once and written once.  Angles cost two 64-bit multiplications and one sine and
// cosine per token and pair, shared by all heads of the token through shared memory.  Measured: 16384 tokens, 32 + 8 heads of 128 in bf16:
// 60 us = 5.6 TB/s; 8191 tokens, 32 + 4 heads of 128 in fp32, half of each turned, interleaved: 48 us = 6.2 TB/s (a copy: 6.46); 8 tokens: 2.5 us.
// Halves that are no multiple of 8 columns take 4-byte accesses: 16384 tokens, 32 + 8 heads of 72 in bf16: 60 us = 3.2 TB/s, 36 of 96 columns 116 us.
#include "dte_ops.cuh"

namespace dte {

constexpr uint32_t kRopeThreads = 128;
constexpr uint32_t kMaxHeadDim = 1024;
constexpr uint32_t kMaxRopeHeads = 4095;     // of queries and keys together; see RopeParams::by_pieces
// Tokens of a CTA: two, so that every thread has one angle and several vectors of heads of 128 (16384 tokens of 40 heads: 60 us; 69
// with one, 63 with four and 256 threads), where that leaves each multiprocessor some CTAs; one for few tokens.
constexpr uint32_t kRopeTokens = 2;
constexpr int kAhead = 2;                    // pieces that a thread loads before it uses the first one

struct RopeSide {
    const void* x;
    void* y;
    uint64_t x_ld, y_ld;
};

struct RopeParams {
    RopeSide side[2];            // queries, keys
    uint32_t q_heads, heads;     // heads: of both
    const void* positions;
    uint32_t positions_dtype;
    uint32_t tokens, head_dim, rot;
    const double* frequencies;
    float amplitude;
    bool inverse;
    uint32_t pieces, turned;     // vectors of work per head, and how many of them are pairs
    uint32_t per_cta;            // tokens
    bool few;                    // tokens: fewer than multiprocessors
    uint32_t by_pieces, by_heads;  // ceil(2^32 / n): the quotient by multiplication is exact below 2^32 / n
};

// cos and sin of position * frequency.  In turns, so that whole ones drop out exactly: what is left of the product after
// its nearest quarter is at most an eighth of a turn, and rounding that to fp32 costs 2^-28 of a turn.
__device__ __forceinline__ float2 rope_turn(int64_t position, double frequency, bool inverse) {
    const double turns = (double)position * (frequency * 0.15915494309189533577);
    const double quarters = rint(4.0 * turns);
    const float rest = (float)fma(-0.25, quarters, turns);
    float s, c;
    sincospif(2.f * rest, &s, &c);
    const int quadrant = (int)((long long)quarters & 3);
    const float cs = quadrant & 1 ? -s : c, sn = quadrant & 1 ? c : s;
    const float sign = quadrant & 2 ? -1.f : 1.f;
    return make_float2(sign * cs, inverse ? -sign * sn : sign * sn);
}

__device__ __forceinline__ void rope_pair(float2 t, float a, float b, float& lo, float& hi) {
    lo = fmaf(a, t.x, -(b * t.y));
    hi = fmaf(b, t.x, a * t.y);
}

__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t d, uint32_t by) { return d == 1 ? n : __umulhi(n, by); }

// A piece is V pairs (half layout: V columns of each half), V / 2 pairs (interleaved; V = 1: a pair) or V columns that are
// copied.
template <typename T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
    extern __shared__ float2 s_turn[];               // per token: rot / 2 cosines and sines
    __shared__ bool s_padding[kRopeTokens];
    constexpr int W = INTERLEAVED && V == 1 ? 2 : V;     // columns of a piece of interleaved pairs
    const uint32_t first = blockIdx.x * p.per_cta, tokens = min(p.per_cta, p.tokens - first), half = p.rot / 2;
    const uint32_t work = tokens * p.heads * p.pieces;
    struct Piece {
        const T* x;
        T* y;
        uint32_t turn, kind;                         // turn: in s_turn, token in the upper 8 bits; kind 0: pairs, 1: copied, 2: nothing to do
        Vec<T, V> a, b;
    };
    auto load = [&](uint32_t i, Piece& c) {
        c.kind = 2;
        if (i >= work) return;
        const uint32_t row = quotient(i, p.pieces, p.by_pieces), piece = i - row * p.pieces;
        const uint32_t token = quotient(row, p.heads, p.by_heads), head = row - token * p.heads;
        const RopeSide& side = p.side[head >= p.q_heads];
        const bool pairs = piece < p.turned;
        const uint32_t col = (head - (head >= p.q_heads ? p.q_heads : 0)) * p.head_dim +
                             (!pairs ? p.rot + (piece - p.turned) * V : INTERLEAVED ? piece * W : piece * V);
        c.x = static_cast<const T*>(side.x) + (uint64_t)(first + token) * side.x_ld + col;
        c.y = static_cast<T*>(side.y) + (uint64_t)(first + token) * side.y_ld + col;
        c.turn = (token * half + (INTERLEAVED ? piece * W / 2 : piece * V)) | token << 24;
        c.kind = pairs ? 0 : c.x == c.y ? 2 : 1;
        if (c.kind == 2) return;
        c.a.load(c.x);
        if (pairs && !INTERLEAVED) c.b.load(c.x + half);
        if (pairs && INTERLEAVED && V == 1) c.b.load(c.x + 1);
    };
    auto finish = [&](Piece& c) {
        if (c.kind == 2) return;
        if (c.kind == 1) {
            c.a.store(c.y);
            return;
        }
        const bool padding = s_padding[c.turn >> 24];
        const float2* turn = s_turn + (c.turn & 0xFFFFFFu);
        float a[V], b[V];
        c.a.get(a);
        if (INTERLEAVED && V > 1) {
            if (!padding) {
#pragma unroll
                for (int j = 0; j + 1 < V; j += 2) rope_pair(turn[j / 2], a[j], a[j + 1], a[j], a[j + 1]);
            }
            c.a.set(a);
            c.a.store(c.y);
        } else {
            c.b.get(b);
            if (!padding) {
#pragma unroll
                for (int j = 0; j < V; ++j) rope_pair(turn[j], a[j], b[j], a[j], b[j]);
            }
            c.a.set(a);
            c.b.set(b);
            c.a.store(c.y);
            c.b.store(c.y + (INTERLEAVED ? 1 : half));
        }
    };
    // few tokens: their heads are shared by the CTAs of a column of the grid
    const uint32_t start = blockIdx.y * kAhead * kRopeThreads + threadIdx.x;
    Piece c[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(start + u * kRopeThreads, c[u]);      // on the way while the angles are made
    for (uint32_t i = threadIdx.x; i < tokens * half; i += kRopeThreads) {
        const uint32_t token = i / half, pair = i - token * half;
        const int64_t position = load_id(p.positions, p.positions_dtype, first + token);
        if (pair == 0) s_padding[token] = position < 0;
        const float2 t = rope_turn(position, p.frequencies[pair], p.inverse);
        s_turn[i] = make_float2(t.x * p.amplitude, t.y * p.amplitude);
    }
    __syncthreads();
    for (uint32_t i = start; i < work; i += gridDim.y * kAhead * kRopeThreads) {
        if (i != start) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load(i + u * kRopeThreads, c[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) finish(c[u]);
    }
}

template <typename T, int V>
static void launch_rope(const RopeParams& p, bool interleaved, cudaStream_t st) {
    const uint32_t work = p.per_cta * p.heads * p.pieces, round = kAhead * kRopeThreads;
    const dim3 grid((p.tokens + p.per_cta - 1) / p.per_cta, p.few ? (work + round - 1) / round : 1);
    const size_t smem = p.per_cta * (p.rot / 2) * sizeof(float2);        // 8 KB at most
    if (interleaved) rope_kernel<T, V, true><<<grid, kRopeThreads, smem, st>>>(p);
    else rope_kernel<T, V, false><<<grid, kRopeThreads, smem, st>>>(p);
}

template <typename T>
static void launch_rope_vec(const RopeParams& p, int vec, bool interleaved, cudaStream_t st) {
    if (vec == 8) launch_rope<T, 8>(p, interleaved, st);
    else if (vec == 2) launch_rope<T, 2>(p, interleaved, st);
    else launch_rope<T, 1>(p, interleaved, st);
}

// Elements per access that a matrix of heads allows: rows, heads and both halves of what is turned start on that boundary.
static int rope_vec(const dte_matrix* x, const dte_matrix* y, uint32_t head_dim, uint32_t rot, bool interleaved) {
    const uint32_t unit = interleaved ? rot : rot / 2;
    const int fits = unit % 8 == 0 && head_dim % 8 == 0 ? 8 : unit % 2 == 0 && head_dim % 2 == 0 ? 2 : 1;
    const int may = vec_of(x, y);
    return may < fits ? may : fits;
}

}  // namespace dte

using namespace dte;

extern "C" dte_status dte_rope_frequencies(uint32_t rot, double base, uint32_t scaling, double factor, double original_positions,
                                           double fast_turns, double slow_turns, double* frequencies, double* amplitude) {
    if (rot < 2 || rot % 2 || rot > kMaxHeadDim) return op_fail(DTE_ERR_INVALID_ARG, "rot must be even, 2 to 1024");
    if (!(base > 1) || !std::isfinite(base)) return op_fail(DTE_ERR_INVALID_ARG, "base must be > 1 and finite");
    if (scaling > DTE_ROPE_RAMP) return op_fail(DTE_ERR_INVALID_ARG, "unknown scaling of the frequencies");
    if (scaling != DTE_ROPE_PLAIN && (!(factor >= 1) || !std::isfinite(factor)))
        return op_fail(DTE_ERR_INVALID_ARG, "factor must be >= 1 and finite");
    if (scaling == DTE_ROPE_BASE && rot == 2) return op_fail(DTE_ERR_INVALID_ARG, "a changed base needs more than one pair");
    if (scaling == DTE_ROPE_RAMP && (!(original_positions > 0) || !std::isfinite(original_positions) || !(slow_turns > 0) ||
                                     !(fast_turns >= slow_turns) || !std::isfinite(fast_turns)))
        return op_fail(DTE_ERR_INVALID_ARG, "the ramp needs original_positions > 0 and fast_turns >= slow_turns > 0");
    if (!frequencies || !amplitude) return op_fail(DTE_ERR_INVALID_ARG, "frequencies or amplitude is null");
    if (scaling == DTE_ROPE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    if (!std::isfinite(base)) return op_fail(DTE_ERR_INVALID_ARG, "base times the factor's power is beyond fp64");
    double lo = 0, hi = 0;
    bool slow = false;         // even the first pair turns fewer than slow_turns times
    if (scaling == DTE_ROPE_RAMP) {
        // index of the pair that turns n times over the original positions: base^(-2 i / rot) * positions = 2 pi n
        const double two_pi = 6.28318530717958647693;
        auto index = [&](double n) { return rot * std::log(original_positions / (n * two_pi)) / (2 * std::log(base)); };
        lo = std::fmax(0.0, std::floor(index(fast_turns)));
        hi = std::fmin(rot - 1.0, std::ceil(index(slow_turns)));
        slow = index(slow_turns) < 0;
    }
    for (uint32_t i = 0; i < rot / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot);
        if (scaling == DTE_ROPE_LINEAR) {
            frequencies[i] = f / factor;
        } else if (scaling == DTE_ROPE_RAMP) {
            const double ramp = slow ? 1.0 : std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 1e-3)));
            frequencies[i] = f * (1.0 - ramp) + f / factor * ramp;
        } else {
            frequencies[i] = f;
        }
    }
    *amplitude = scaling == DTE_ROPE_RAMP ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return DTE_OK;
}

extern "C" dte_status dte_rope(const dte_matrix* q, const dte_matrix* k, uint32_t head_dim, const dte_ids* positions,
                               const double* frequencies, uint32_t rot, uint32_t layout, double amplitude, int inverse,
                               const dte_matrix* q_out, const dte_matrix* k_out, int device, void* cuda_stream) {
    dte_status s;
    const dte_matrix* in[2] = {q, k};
    const dte_matrix* out[2] = {q_out, k_out};
    if ((s = check_ids(positions)) != DTE_OK) return s;
    if (head_dim == 0 || head_dim > kMaxHeadDim || rot < 2 || rot % 2 || rot > head_dim)
        return op_fail(DTE_ERR_INVALID_ARG, "rot must be even and 2 <= rot <= head_dim <= 1024");
    if (layout > DTE_ROPE_INTERLEAVED) return op_fail(DTE_ERR_INVALID_ARG, "unknown layout of the pairs");
    if (!std::isfinite((float)amplitude)) return op_fail(DTE_ERR_INVALID_ARG, "amplitude is not finite in fp32");
    if (!frequencies || ((uintptr_t)frequencies & 7u)) return op_fail(DTE_ERR_INVALID_ARG, "frequencies are null or not 8-byte aligned");
    const bool interleaved = layout == DTE_ROPE_INTERLEAVED;
    RopeParams p = {};
    int vec = 8;
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && !k && !k_out) break;
        if ((s = check_matrix(in[i], i ? "k is null" : "q is null", false)) != DTE_OK) return s;
        if ((s = check_matrix(out[i], i ? "k_out is null" : "q_out is null", true)) != DTE_OK) return s;
        if (in[i]->cols % head_dim) return op_fail(DTE_ERR_INVALID_ARG, "columns must be a multiple of head_dim");
        if (in[i]->rows != positions->count || out[i]->rows != in[i]->rows || out[i]->cols != in[i]->cols)
            return op_fail(DTE_ERR_INVALID_ARG, "inputs and outputs need one row per position and the same columns");
        if (in[i]->dtype != q->dtype || out[i]->dtype != q->dtype)
            return op_fail(DTE_ERR_INVALID_ARG, "q, k and their outputs must have one type");
        if (in[i]->data == out[i]->data && in[i]->rows > 1 && in[i]->ld != out[i]->ld)
            return op_fail(DTE_ERR_INVALID_ARG, "in place needs the input's ld");
        RopeSide& side = p.side[i];
        side.x = in[i]->data;
        side.y = out[i]->data;
        side.x_ld = in[i]->ld;
        side.y_ld = out[i]->ld;
        const uint64_t heads = in[i]->cols / head_dim;
        if (p.heads + heads > kMaxRopeHeads) return op_fail(DTE_ERR_INVALID_ARG, "at most 4095 heads");
        if (i == 0) p.q_heads = (uint32_t)heads;
        p.heads += (uint32_t)heads;
        const int v = rope_vec(in[i], out[i], head_dim, rot, interleaved);
        vec = v < vec ? v : vec;
    }
    p.positions = positions->data;
    p.positions_dtype = positions->dtype;
    p.tokens = (uint32_t)positions->count;
    p.head_dim = head_dim;
    p.rot = rot;
    p.frequencies = frequencies;
    p.amplitude = (float)amplitude;
    p.inverse = inverse != 0;
    p.turned = interleaved && vec > 1 ? rot / vec : rot / 2 / (interleaved ? 1 : vec);
    p.pieces = p.turned + (head_dim - rot) / vec;
    p.by_pieces = (uint32_t)(((1ull << 32) + p.pieces - 1) / p.pieces);
    p.by_heads = (uint32_t)(((1ull << 32) + p.heads - 1) / p.heads);
    if (p.tokens == 0) return DTE_OK;
    OpDeviceGuard g;
    int sms = 0;
    if ((s = g.enter(device, &sms)) != DTE_OK) return s;
    const uint64_t reach = (uint64_t)kRopeTokens * p.heads * p.pieces * (p.pieces > p.heads ? p.pieces : p.heads);
    p.per_cta = p.tokens >= (uint32_t)sms * 4 * kRopeTokens && reach < (1ull << 32) ? kRopeTokens : 1;
    p.few = p.tokens < (uint32_t)sms;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (q->dtype == DTE_BF16) launch_rope_vec<__nv_bfloat16>(p, vec, interleaved, st);
    else launch_rope_vec<float>(p, vec, interleaved, st);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}
