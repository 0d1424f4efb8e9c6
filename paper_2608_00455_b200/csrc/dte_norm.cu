// Layer norm and RMS norm, forward and backward.
//
// Both directions are bound by the bytes of the row matrices: a row is read once into registers,
// its statistics are reduced there (the variance from the centred values, not as E[x^2] - E[x]^2) and
// the result is written.  CTAs are persistent over rows: the weights, and in the backward pass the
// running sums of the weight's gradient, belong to columns and so stay in the same thread's
// registers for all its rows, and the next row is loaded before the current row's reduction, which
// hides the reduction's latency behind the loads.
//
// A row is held by a team: 8, 16 or 32 lanes of a warp for up to 256 columns (a head's norm: several
// rows per warp, reductions by shuffles alone), else one CTA of ceil(columns / 8) threads, eight columns
// per thread, up to 8192 columns.  Longer rows take the kernels that pass over the row from memory again.
#include "dte_ops.cuh"

namespace dte {

constexpr int kPer = 8;                  // columns per thread
constexpr int kTeamThreads = 256;        // CTA size when teams are parts of a warp
constexpr uint32_t kMaxRegCols = 1024 * kPer;
constexpr int kLongThreads = 512;

struct NormParams {
    const void* x;
    const void* dout;
    void* out;                // forward: y, backward: dx (or NULL)
    const void* weight;
    const void* bias;
    uint64_t x_ld, dout_ld, out_ld;
    uint32_t rows, cols, param_dtype;
    float eps, inv_cols;
    float* mean;
    float* rstd;
    bool want_bias;           // backward: dbias is wanted
    float* partial;           // backward: teams' sums, grid x 2 x cols (NULL: no weight gradient wanted)
};

__device__ __forceinline__ float load_param(const void* p, uint32_t dtype, uint32_t i, float none) {
    if (!p) return none;
    return dtype == DTE_BF16 ? to_f(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}

__device__ __forceinline__ float f2_sum(F2 a) {
    float lo, hi;
    f2_get(a, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ float f2_at(const F2* a, int j) {
    float lo, hi;
    f2_get(a[j / 2], lo, hi);
    return j & 1 ? hi : lo;
}

// The eight columns of thread t of a team of n threads.  VEC: 16-byte accesses (8 consecutive bf16, or
// two groups of 4 consecutive floats n threads apart); else element by element, n columns apart.
template <typename T, bool VEC>
struct RowPart;

template <>
struct RowPart<__nv_bfloat16, true> {
    uint4 a;
    static __device__ __forceinline__ uint32_t col(uint32_t t, uint32_t, int j) { return t * 8 + j; }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, uint32_t t, uint32_t, uint32_t cols) {
        a = t * 8 < cols ? __ldcs(reinterpret_cast<const uint4*>(p + t * 8)) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void get(F2* f) const {
        f[0] = f2(bf16_lo(a.x), bf16_hi(a.x));
        f[1] = f2(bf16_lo(a.y), bf16_hi(a.y));
        f[2] = f2(bf16_lo(a.z), bf16_hi(a.z));
        f[3] = f2(bf16_lo(a.w), bf16_hi(a.w));
    }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, uint32_t t, uint32_t, uint32_t cols, const float* f) {
        if (t * 8 < cols)
            *reinterpret_cast<uint4*>(p + t * 8) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]),
                                                              pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
};
template <>
struct RowPart<float, true> {
    float4 a, b;
    static __device__ __forceinline__ uint32_t col(uint32_t t, uint32_t n, int j) { return (j / 4) * 4 * n + t * 4 + j % 4; }
    __device__ __forceinline__ void load(const float* p, uint32_t t, uint32_t n, uint32_t cols) {
        const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
        a = t * 4 < cols ? __ldcs(reinterpret_cast<const float4*>(p + t * 4)) : z;
        b = (n + t) * 4 < cols ? __ldcs(reinterpret_cast<const float4*>(p + (n + t) * 4)) : z;
    }
    __device__ __forceinline__ void get(F2* f) const {
        f[0] = f2(a.x, a.y);
        f[1] = f2(a.z, a.w);
        f[2] = f2(b.x, b.y);
        f[3] = f2(b.z, b.w);
    }
    static __device__ __forceinline__ void put(float* p, uint32_t t, uint32_t n, uint32_t cols, const float* f) {
        if (t * 4 < cols) *reinterpret_cast<float4*>(p + t * 4) = make_float4(f[0], f[1], f[2], f[3]);
        if ((n + t) * 4 < cols) *reinterpret_cast<float4*>(p + (n + t) * 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
};
template <typename T>
struct RowPart<T, false> {
    T a[kPer];
    static __device__ __forceinline__ uint32_t col(uint32_t t, uint32_t n, int j) { return t + j * n; }
    __device__ __forceinline__ void load(const T* p, uint32_t t, uint32_t n, uint32_t cols) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) a[j] = t + j * n < cols ? p[t + j * n] : from_f<T>(0.f);
    }
    __device__ __forceinline__ void get(F2* f) const {
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) f[j] = f2(to_f<T>(a[2 * j]), to_f<T>(a[2 * j + 1]));
    }
    static __device__ __forceinline__ void put(T* p, uint32_t t, uint32_t n, uint32_t cols, const float* f) {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (t + j * n < cols) p[t + j * n] = from_f<T>(f[j]);
    }
};

// Sum of v[0..N) over the team; every member gets the result.  TEAM > 32: the whole CTA, of at most TEAM
// threads (buf: N x 32 floats, not reused before the CTA has passed another barrier).
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* buf) {
#pragma unroll
    for (int o = (TEAM < 32 ? TEAM : 32) / 2; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if (TEAM > 32) {
        const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, warps = blockDim.x / 32;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[i * 32 + warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lane < warps ? buf[i * 32 + lane] : 0.f;
#pragma unroll
            for (int o = 16; o; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
        }
    }
}

template <typename T, bool VEC, int TEAM, uint32_t KIND>
__global__ void __launch_bounds__(TEAM <= 32 ? kTeamThreads : TEAM) norm_forward_kernel(const NormParams p) {
    __shared__ float buf[2][32];
    const uint32_t n = TEAM <= 32 ? TEAM : blockDim.x;
    const uint32_t t = TEAM <= 32 ? threadIdx.x % n : threadIdx.x;
    const uint32_t teams = TEAM <= 32 ? gridDim.x * (kTeamThreads / n) : gridDim.x;
    const uint32_t me = TEAM <= 32 ? blockIdx.x * (kTeamThreads / n) + threadIdx.x / n : blockIdx.x;
    const T* x = static_cast<const T*>(p.x);
    T* y = static_cast<T*>(p.out);
    F2 w[kPer / 2], b[kPer / 2], in[kPer / 2];            // in: 1 for columns of the row, 0 past its end
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) {
        float u[2], v[2], q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = RowPart<T, VEC>::col(t, n, 2 * j + i);
            q[i] = c < p.cols ? 1.f : 0.f;
            u[i] = c < p.cols ? load_param(p.weight, p.param_dtype, c, 1.f) : 0.f;
            v[i] = c < p.cols ? load_param(p.bias, p.param_dtype, c, 0.f) : 0.f;
        }
        w[j] = f2(u[0], u[1]);
        b[j] = f2(v[0], v[1]);
        in[j] = f2(q[0], q[1]);
    }
    RowPart<T, VEC> next;
    if (me < p.rows) next.load(x + (uint64_t)me * p.x_ld, t, n, p.cols);
    // all lanes of a warp go round together, so that shuffles stay full; a team past the end idles
    const uint32_t rounds = (p.rows + teams - 1) / teams;
    for (uint32_t k = 0; k < rounds; ++k) {
        const uint64_t row = (uint64_t)k * teams + me;
        if (TEAM > 32 && row >= p.rows) break;
        F2 f[kPer / 2];
        next.get(f);
        if (row + teams < p.rows) next.load(x + (row + teams) * p.x_ld, t, n, p.cols);
        float mean = 0.f;
        if (KIND == DTE_NORM_LAYER) {
            float s[1] = {f2_sum(f2_add(f2_add(f[0], f[1]), f2_add(f[2], f[3])))};
            team_sum<TEAM, 1>(s, buf[0]);
            mean = s[0] * p.inv_cols;
            const F2 m = f2(-mean, -mean);
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) f[j] = f2_fma(in[j], m, f[j]);
        }
        F2 q2 = f2_mul(f[0], f[0]);
#pragma unroll
        for (int j = 1; j < kPer / 2; ++j) q2 = f2_fma(f[j], f[j], q2);
        float q[1] = {f2_sum(q2)};
        team_sum<TEAM, 1>(q, KIND == DTE_NORM_LAYER ? buf[1] : buf[k & 1]);
        const float rstd = 1.f / sqrtf(q[0] * p.inv_cols + p.eps);
        if (row < p.rows) {
            const F2 r = f2(rstd, rstd);
            float o[kPer];
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) f2_get(f2_fma(f2_mul(f[j], r), w[j], b[j]), o[2 * j], o[2 * j + 1]);
            RowPart<T, VEC>::put(y + row * p.out_ld, t, n, p.cols, o);
            if (t == 0) {
                if (KIND == DTE_NORM_LAYER && p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
        }
    }
}

template <typename T, bool VEC, int TEAM, uint32_t KIND>
__global__ void __launch_bounds__(TEAM <= 32 ? kTeamThreads : TEAM) norm_backward_kernel(const NormParams p) {
    __shared__ float buf[2][64];
    const uint32_t n = TEAM <= 32 ? TEAM : blockDim.x;
    const uint32_t t = TEAM <= 32 ? threadIdx.x % n : threadIdx.x;
    const uint32_t teams = TEAM <= 32 ? gridDim.x * (kTeamThreads / n) : gridDim.x;
    const uint32_t me = TEAM <= 32 ? blockIdx.x * (kTeamThreads / n) + threadIdx.x / n : blockIdx.x;
    const T* x = static_cast<const T*>(p.x);
    const T* dy = static_cast<const T*>(p.dout);
    T* dx = static_cast<T*>(p.out);
    F2 w[kPer / 2], dw[kPer / 2], db[kPer / 2];
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) {
        float u[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = RowPart<T, VEC>::col(t, n, 2 * j + i);
            u[i] = c < p.cols ? load_param(p.weight, p.param_dtype, c, 1.f) : 0.f;
        }
        w[j] = f2(u[0], u[1]);
        dw[j] = db[j] = f2(0.f, 0.f);
    }
    RowPart<T, VEC> nx, ny;
    float nmean = 0.f, nrstd = 0.f;
    auto fetch = [&](uint64_t row) {
        nx.load(x + row * p.x_ld, t, n, p.cols);
        ny.load(dy + row * p.dout_ld, t, n, p.cols);
        if (KIND == DTE_NORM_LAYER) nmean = p.mean[row];
        nrstd = p.rstd[row];
    };
    if (me < p.rows) fetch(me);
    const uint32_t rounds = (p.rows + teams - 1) / teams;
    for (uint32_t k = 0; k < rounds; ++k) {
        const uint64_t row = (uint64_t)k * teams + me;
        if (TEAM > 32 && row >= p.rows) break;
        F2 xh[kPer / 2], g[kPer / 2];
        nx.get(xh);
        ny.get(g);
        const float mean = nmean, rstd = nrstd;
        if (row + teams < p.rows) fetch(row + teams);
        const bool live = row < p.rows;
        const F2 r = f2(rstd, rstd), m = f2(-mean * rstd, -mean * rstd);
        F2 s2 = f2(0.f, 0.f), s1 = f2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
            // columns past the end hold zero in g and w, so they add nothing: xh is finite there
            xh[j] = KIND == DTE_NORM_LAYER ? f2_fma(xh[j], r, m) : f2_mul(xh[j], r);
            if (live) {
                dw[j] = f2_fma(g[j], xh[j], dw[j]);
                if (KIND == DTE_NORM_LAYER || p.want_bias) db[j] = f2_add(db[j], g[j]);
            }
            g[j] = f2_mul(g[j], w[j]);
            s2 = f2_fma(g[j], xh[j], s2);
            if (KIND == DTE_NORM_LAYER) s1 = f2_add(s1, g[j]);
        }
        float c1 = 0.f, c2;
        if (KIND == DTE_NORM_LAYER) {
            float s[2] = {f2_sum(s2), f2_sum(s1)};
            team_sum<TEAM, 2>(s, buf[k & 1]);
            c2 = s[0];
            c1 = s[1];
        } else {
            float s[1] = {f2_sum(s2)};
            team_sum<TEAM, 1>(s, buf[k & 1]);
            c2 = s[0];
        }
        if (live && dx) {
            // rstd * (g - c1 - xh * c2)
            c2 *= -p.inv_cols * rstd;
            c1 *= -p.inv_cols * rstd;
            const F2 a = f2(c2, c2), b = f2(c1, c1);
            float o[kPer];
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j)
                f2_get(f2_fma(xh[j], a, KIND == DTE_NORM_LAYER ? f2_fma(g[j], r, b) : f2_mul(g[j], r)), o[2 * j], o[2 * j + 1]);
            RowPart<T, VEC>::put(dx + row * p.out_ld, t, n, p.cols, o);
        }
    }
    if (!p.partial) return;
    if (TEAM <= 32) {
        // the CTA's teams hold sums of the same columns: add them up in order of the teams
        __shared__ float sums[2][kTeamThreads * kPer];
        constexpr uint32_t kTeams = TEAM <= 32 ? kTeamThreads / TEAM : 1;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t c = RowPart<T, VEC>::col(t, n, j);
            sums[0][(threadIdx.x / n) * (n * kPer) + c] = f2_at(dw, j);
            sums[1][(threadIdx.x / n) * (n * kPer) + c] = f2_at(db, j);
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * p.cols; i += kTeamThreads) {
            const uint32_t which = i >= p.cols, c = which ? i - p.cols : i;
            float v = 0.f;
            for (uint32_t m = 0; m < kTeams; ++m) v += sums[which][m * (n * kPer) + c];
            p.partial[((uint64_t)blockIdx.x * 2 + which) * p.cols + c] = v;
        }
    } else {
        float* o = p.partial + (uint64_t)blockIdx.x * 2 * p.cols;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t c = RowPart<T, VEC>::col(t, n, j);
            if (c < p.cols) {
                o[c] = f2_at(dw, j);
                o[p.cols + c] = f2_at(db, j);
            }
        }
    }
}

// Adds up the CTAs' sums: 32 columns per CTA, 32 threads per column, each a stretch of the partial rows.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const float* partial, uint32_t parts, uint32_t cols, bool accumulate,
                                                         float* dweight, float* dbias) {
    __shared__ float sums[32][33];
    wait_for_earlier();
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const uint32_t lane = threadIdx.x & 31, part = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < cols) {
        const float* src = partial + (uint64_t)blockIdx.y * cols + c;
#pragma unroll 4
        for (uint32_t i = part; i < parts; i += 32) v += src[(uint64_t)i * 2 * cols];
    }
    sums[part][lane] = v;
    __syncthreads();
    // warp w sums column w of this CTA
    v = warp_sum(sums[lane][part]);
    const uint32_t col = blockIdx.x * 32 + part;
    if (lane == 0 && col < cols) out[col] = accumulate ? out[col] + v : v;
}

// ---- rows longer than a CTA's registers: the row is read from memory (from L2, mostly) once per pass ----------
template <int N>
__device__ __forceinline__ void cta_sum(float (&v)[N], float* buf) {
    __syncthreads();
    team_sum<kLongThreads, N>(v, buf);
}

template <typename T, uint32_t KIND>
__global__ void __launch_bounds__(kLongThreads) norm_forward_long_kernel(const NormParams p) {
    __shared__ float buf[32];
    for (uint64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_ld;
        T* y = static_cast<T*>(p.out) + row * p.out_ld;
        float mean = 0.f, s[1] = {0.f};
        if (KIND == DTE_NORM_LAYER) {
            for (uint32_t c = threadIdx.x; c < p.cols; c += kLongThreads) s[0] += to_f<T>(x[c]);
            cta_sum<1>(s, buf);
            mean = s[0] * p.inv_cols;
        }
        s[0] = 0.f;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kLongThreads) {
            const float d = to_f<T>(x[c]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        cta_sum<1>(s, buf);
        const float rstd = 1.f / sqrtf(s[0] * p.inv_cols + p.eps);
        for (uint32_t c = threadIdx.x; c < p.cols; c += kLongThreads)
            y[c] = from_f<T>(fmaf((to_f<T>(x[c]) - mean) * rstd, load_param(p.weight, p.param_dtype, c, 1.f),
                                  load_param(p.bias, p.param_dtype, c, 0.f)));
        if (threadIdx.x == 0) {
            if (KIND == DTE_NORM_LAYER && p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <typename T, uint32_t KIND>
__global__ void __launch_bounds__(kLongThreads) norm_backward_long_kernel(const NormParams p) {
    __shared__ float buf[64];
    for (uint64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_ld;
        const T* dy = static_cast<const T*>(p.dout) + row * p.dout_ld;
        T* dx = static_cast<T*>(p.out) + row * p.out_ld;
        const float mean = KIND == DTE_NORM_LAYER ? p.mean[row] : 0.f, rstd = p.rstd[row];
        float s[2] = {0.f, 0.f};
        for (uint32_t c = threadIdx.x; c < p.cols; c += kLongThreads) {
            const float g = to_f<T>(dy[c]) * load_param(p.weight, p.param_dtype, c, 1.f);
            s[0] = fmaf(g, (to_f<T>(x[c]) - mean) * rstd, s[0]);
            s[1] += g;
        }
        cta_sum<2>(s, buf);
        const float c2 = s[0] * p.inv_cols, c1 = KIND == DTE_NORM_LAYER ? s[1] * p.inv_cols : 0.f;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kLongThreads) {
            const float g = to_f<T>(dy[c]) * load_param(p.weight, p.param_dtype, c, 1.f);
            const float xh = (to_f<T>(x[c]) - mean) * rstd;
            dx[c] = from_f<T>(rstd * (fmaf(-xh, c2, g) - c1));
        }
    }
}

// Column sums of a slab of rows: blockIdx.y takes every gridDim.y-th row.
template <typename T, uint32_t KIND>
__global__ void __launch_bounds__(256) norm_columns_long_kernel(const NormParams p) {
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.cols) return;
    float dw = 0.f, db = 0.f;
    for (uint64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const float g = to_f<T>(static_cast<const T*>(p.dout)[row * p.dout_ld + c]);
        const float xv = to_f<T>(static_cast<const T*>(p.x)[row * p.x_ld + c]);
        dw = fmaf(g, (KIND == DTE_NORM_LAYER ? xv - p.mean[row] : xv) * p.rstd[row], dw);
        db += g;
    }
    float* o = p.partial + (uint64_t)blockIdx.y * 2 * p.cols;
    o[c] = dw;
    o[p.cols + c] = db;
}

// ---- launches ------------------------------------------------------------------------------------------
// Team of a row length, threads of a CTA and CTAs of a launch.
struct NormShape {
    int team;             // 8, 16, 32 lanes; 512, 1024: one CTA of up to that many threads per row; 0: long rows
    unsigned threads, ctas;
};

constexpr unsigned kCtasPerSm = 8;       // upper bound of the backward grid per SM, for the workspace

static NormShape norm_shape(uint64_t rows, uint64_t cols, int sms, unsigned threads_per_sm) {
    NormShape s;
    uint64_t need;
    if (cols > kMaxRegCols) {
        s.team = 0;
        s.threads = kLongThreads;
        need = rows;
    } else if (cols <= 32 * kPer) {
        s.team = cols <= 8 * kPer ? 8 : cols <= 16 * kPer ? 16 : 32;
        s.threads = kTeamThreads;
        need = (rows + kTeamThreads / s.team - 1) / (kTeamThreads / s.team);
    } else {
        s.threads = (unsigned)((cols + kPer * 32 - 1) / (kPer * 32) * 32);
        s.team = s.threads <= 512 ? 512 : 1024;
        need = rows;
    }
    unsigned per_sm = threads_per_sm / s.threads;
    if (per_sm < 1) per_sm = 1;
    if (per_sm > kCtasPerSm) per_sm = kCtasPerSm;
    const uint64_t most = (uint64_t)sms * per_sm;
    s.ctas = (unsigned)(need < most ? need : most);
    return s;
}

template <typename T, bool VEC, uint32_t KIND>
static void forward_team(const NormParams& p, const NormShape& s, cudaStream_t st) {
    if (s.team == 8) norm_forward_kernel<T, VEC, 8, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 16) norm_forward_kernel<T, VEC, 16, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 32) norm_forward_kernel<T, VEC, 32, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 512) norm_forward_kernel<T, VEC, 512, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 1024) norm_forward_kernel<T, VEC, 1024, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else norm_forward_long_kernel<T, KIND><<<s.ctas, s.threads, 0, st>>>(p);
}

template <typename T, bool VEC, uint32_t KIND>
static void backward_team(const NormParams& p, const NormShape& s, cudaStream_t st) {
    if (s.team == 8) norm_backward_kernel<T, VEC, 8, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 16) norm_backward_kernel<T, VEC, 16, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 32) norm_backward_kernel<T, VEC, 32, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 512) norm_backward_kernel<T, VEC, 512, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else if (s.team == 1024) norm_backward_kernel<T, VEC, 1024, KIND><<<s.ctas, s.threads, 0, st>>>(p);
    else {
        if (p.out) norm_backward_long_kernel<T, KIND><<<s.ctas, s.threads, 0, st>>>(p);
        if (p.partial) norm_columns_long_kernel<T, KIND><<<dim3((p.cols + 255) / 256, s.ctas), 256, 0, st>>>(p);
    }
}

template <bool BACK>
static void norm_launch(const NormParams& p, const NormShape& s, bool bf16, bool vec, uint32_t kind, cudaStream_t st) {
#define DTE_NORM_CASE(T, V, K) \
    if (BACK) backward_team<T, V, K>(p, s, st); else forward_team<T, V, K>(p, s, st)
    if (kind == DTE_NORM_LAYER) {
        if (bf16 && vec) { DTE_NORM_CASE(__nv_bfloat16, true, DTE_NORM_LAYER); }
        else if (bf16) { DTE_NORM_CASE(__nv_bfloat16, false, DTE_NORM_LAYER); }
        else if (vec) { DTE_NORM_CASE(float, true, DTE_NORM_LAYER); }
        else { DTE_NORM_CASE(float, false, DTE_NORM_LAYER); }
    } else {
        if (bf16 && vec) { DTE_NORM_CASE(__nv_bfloat16, true, DTE_NORM_RMS); }
        else if (bf16) { DTE_NORM_CASE(__nv_bfloat16, false, DTE_NORM_RMS); }
        else if (vec) { DTE_NORM_CASE(float, true, DTE_NORM_RMS); }
        else { DTE_NORM_CASE(float, false, DTE_NORM_RMS); }
    }
#undef DTE_NORM_CASE
}

static dte_status check_params(const void* w, const void* b, uint32_t dtype) {
    if (dtype != DTE_F32 && dtype != DTE_BF16) return op_fail(DTE_ERR_INVALID_ARG, "param_dtype must be DTE_F32 or DTE_BF16");
    if (((uintptr_t)w | (uintptr_t)b) & (elem_size(dtype) - 1))
        return op_fail(DTE_ERR_INVALID_ARG, "weight / bias are not aligned to their type");
    return DTE_OK;
}

constexpr int kMostSms = 256;            // the workspace helper does not know the device

}  // namespace dte

using namespace dte;

extern "C" dte_status dte_norm_forward(const dte_matrix* x, const void* weight, const void* bias, uint32_t param_dtype,
                                       uint32_t kind, double eps, const dte_matrix* out, float* mean, float* rstd,
                                       int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_matrix(x, "x is null", false)) != DTE_OK) return s;
    if ((s = check_matrix(out, "out is null", true)) != DTE_OK) return s;
    if ((s = check_params(weight, bias, param_dtype)) != DTE_OK) return s;
    if (kind != DTE_NORM_LAYER && kind != DTE_NORM_RMS) return op_fail(DTE_ERR_INVALID_ARG, "unknown norm kind");
    if (!(eps >= 0) || !std::isfinite(eps)) return op_fail(DTE_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (x->rows != out->rows || x->cols != out->cols || x->dtype != out->dtype)
        return op_fail(DTE_ERR_INVALID_ARG, "out must have x's shape and type");
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3u) return op_fail(DTE_ERR_INVALID_ARG, "mean / rstd must be 4-byte aligned");
    if (x->rows == 0) return DTE_OK;
    OpDeviceGuard g(device);
    int sms = 0;
    if ((s = device_sms(device, &sms)) != DTE_OK) return s;
    NormParams p = {};
    p.x = x->data;
    p.out = out->data;
    p.weight = weight;
    p.bias = bias;
    p.x_ld = x->ld;
    p.out_ld = out->ld;
    p.rows = (uint32_t)x->rows;
    p.cols = (uint32_t)x->cols;
    p.param_dtype = param_dtype;
    p.eps = (float)eps;
    p.inv_cols = (float)(1.0 / (double)x->cols);
    p.mean = mean;
    p.rstd = rstd;
    norm_launch<false>(p, norm_shape(x->rows, x->cols, sms, 1024), x->dtype == DTE_BF16, vec8_ok(x) && vec8_ok(out), kind,
                       (cudaStream_t)cuda_stream);
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

extern "C" uint64_t dte_norm_backward_workspace_bytes(uint64_t rows, uint64_t hidden) {
    if (rows >= kMaxDim || hidden >= kMaxDim) return UINT64_MAX;    // refused by the call
    const uint64_t most = (uint64_t)kMostSms * kCtasPerSm;
    return align_up((rows < most ? rows : most) * 2 * hidden * sizeof(float), kWorkspaceAlign);
}

extern "C" dte_status dte_norm_backward(const dte_matrix* dout, const dte_matrix* x, const void* weight,
                                        uint32_t param_dtype, uint32_t kind, const float* mean, const float* rstd,
                                        int accumulate, const dte_matrix* dx, float* dweight, float* dbias,
                                        void* workspace, uint64_t workspace_bytes, int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_matrix(dout, "dout is null", false)) != DTE_OK) return s;
    if ((s = check_matrix(x, "x is null", false)) != DTE_OK) return s;
    if (dx && (s = check_matrix(dx, "dx is null", true)) != DTE_OK) return s;
    if ((s = check_params(weight, nullptr, param_dtype)) != DTE_OK) return s;
    if (kind != DTE_NORM_LAYER && kind != DTE_NORM_RMS) return op_fail(DTE_ERR_INVALID_ARG, "unknown norm kind");
    if (dout->rows != x->rows || dout->cols != x->cols || dout->dtype != x->dtype ||
        (dx && (dx->rows != x->rows || dx->cols != x->cols || dx->dtype != x->dtype)))
        return op_fail(DTE_ERR_INVALID_ARG, "dout and dx must have x's shape and type");
    if (x->rows && (!rstd || (kind == DTE_NORM_LAYER && !mean))) return op_fail(DTE_ERR_INVALID_ARG, "mean / rstd is null");
    if (((uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dweight | (uintptr_t)dbias) & 3u)
        return op_fail(DTE_ERR_INVALID_ARG, "mean, rstd, dweight and dbias must be 4-byte aligned");
    const bool want = dweight || dbias;
    if (want && (s = check_workspace(workspace, workspace_bytes, dte_norm_backward_workspace_bytes(x->rows, x->cols))) != DTE_OK)
        return s;
    if (!dx && !want) return DTE_OK;
    OpDeviceGuard g(device);
    int sms = 0;
    if ((s = device_sms(device, &sms)) != DTE_OK) return s;
    if (sms > kMostSms) sms = kMostSms;
    NormParams p = {};
    p.x = x->data;
    p.dout = dout->data;
    p.out = dx ? dx->data : nullptr;
    p.weight = weight;
    p.x_ld = x->ld;
    p.dout_ld = dout->ld;
    p.out_ld = dx ? dx->ld : 0;
    p.rows = (uint32_t)x->rows;
    p.cols = (uint32_t)x->cols;
    p.param_dtype = param_dtype;
    p.inv_cols = (float)(1.0 / (double)x->cols);
    p.mean = const_cast<float*>(mean);
    p.rstd = const_cast<float*>(rstd);
    p.want_bias = dbias != nullptr;
    p.partial = want ? static_cast<float*>(workspace) : nullptr;
    const NormShape sh = norm_shape(x->rows, x->cols, sms, 1024);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (x->rows) {
        norm_launch<true>(p, sh, x->dtype == DTE_BF16, vec8_ok(x) && vec8_ok(dout) && (!dx || vec8_ok(dx)), kind, st);
        DTE_CUDA(cudaGetLastError());
    }
    if (want) {
        DTE_CUDA(launch_after(norm_sums_kernel, dim3((p.cols + 31) / 32, 2), 1024, 0, st, p.partial, x->rows ? sh.ctas : 0, p.cols,
                              accumulate != 0, dweight, dbias));
    }
    return DTE_OK;
}
