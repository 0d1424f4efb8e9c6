// Layer norm and RMS norm, forward and backward.
//
// Both directions are bound by the bytes of the row matrices: a row is read from memory once,
// its statistics are reduced in registers (the variance from the centred values, not as E[x^2] - E[x]^2) and
// the result is written.  CTAs are persistent over rows: the weights, and in the backward pass the
// running sums of the weight's gradient, belong to columns and so stay in the same thread's
// registers for all its rows.  The rows to come are on their way into shared memory meanwhile: every thread copies
// its own columns of the next rows (asynchronous 16-byte copies) and reads back what it copied, so the
// ring needs no barrier.  (One row ahead in registers keeps 32 KB per SM in flight: 4.1 TB/s.)  The forward pass reaches
// 5.9 TB/s (8191 x 4096 fp32, 45 us; a plain copy of the same size 43 us), the backward pass 4.6 TB/s
// (16384 x 4096 bf16, 88 us, of which centring each row before it is scaled takes 2.4): 16 warps per SM, all that the sums'
// registers leave room for, do not quite hide a row's reduction.
//
// A row is held by a team: 8, 16 or 32 lanes of a warp for up to 512 columns (a head's norm: several
// rows per warp, reductions by shuffles alone), else one CTA of ceil(columns / 16) threads, sixteen columns
// per thread, up to 16384 columns.  Sixteen, because what a warp spends on a row beside its columns (reduction,
// addresses, statistics) was half of its instructions at eight.  Longer rows take the kernels that pass over the
// row from memory again.
//
// The shape was chosen at 4096 and 128 columns.  Elsewhere (2^26 bf16 elements, forward / backward in TB/s): 2048 5.2 / 4.9,
// 4096 5.1 / 4.8, 6144 4.3 / 4.6, 8192 4.7 / 4.5; just above 4096 an SM holds one CTA of 288 threads instead of 512 threads: 4104
// 3.0 / 3.6, 5120 3.7 / 4.3.  From 8193 columns a CTA has more than 512 threads, so 64 registers each, and a row spills to
// local memory: 16384 2.6 / 3.1.  Columns or strides that allow no 16-byte accesses go element by element, one row ahead:
// 2001 and 2002 2.3 / 2.3.  20000 (several passes) 0.9 / 0.9.
#include "dte_ops.cuh"

namespace dte {

constexpr int kPer = 16;                 // columns per thread
constexpr int kTeamThreads = 256;        // CTA size when teams are parts of a warp
constexpr uint32_t kMaxRegCols = 1024 * kPer;
constexpr int kLongThreads = 512;
// Shared memory of a thread's rows in flight and threads per SM, measured together (us, layer norm 8191 x 4096 fp32 / its
// gradient 16384 x 4096 bf16, then without centring): these 45 / 84; half the ring 53 / 99; 1024 threads 46 forward.  More rows in flight
// than 64 KB per SM make the forward pass slower, not faster.
constexpr int kRingForward = 128, kRingBackward = 256;
constexpr unsigned kSmThreadsForward = 512, kSmThreadsBackward = 512;

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

// 16 bytes into shared memory, asynchronously; zeros where `live` is false (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int AHEAD>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory"); }
__device__ __forceinline__ uint4 shared16(uint32_t from) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from));
    return v;
}

// The columns of thread t of a team of n threads.  VEC: 16-byte pieces, n pieces apart; else element by element,
// n columns apart.
template <typename T, bool VEC>
struct RowPart;

template <typename T>
struct RowPart<T, true> {
    static constexpr int kPiece = 16 / sizeof(T), kPieces = kPer / kPiece;
    static __device__ __forceinline__ uint32_t col(uint32_t t, uint32_t n, int j) { return ((j / kPiece) * n + t) * kPiece + j % kPiece; }
    // shared memory: piece i of the thread lies i * step bytes behind `at`
    static __device__ __forceinline__ void copy(uint32_t at, uint32_t step, const T* p, uint32_t t, uint32_t n, uint32_t cols) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) copy16(at + i * step, p + col(t, n, i * kPiece), col(t, n, i * kPiece) < cols);
    }
    static __device__ __forceinline__ void get(uint32_t at, uint32_t step, F2* f) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint4 a = shared16(at + i * step);
            if (sizeof(T) == 2) {
                f[4 * i] = f2(bf16_lo(a.x), bf16_hi(a.x));
                f[4 * i + 1] = f2(bf16_lo(a.y), bf16_hi(a.y));
                f[4 * i + 2] = f2(bf16_lo(a.z), bf16_hi(a.z));
                f[4 * i + 3] = f2(bf16_lo(a.w), bf16_hi(a.w));
            } else {
                f[2 * i] = f2(__uint_as_float(a.x), __uint_as_float(a.y));
                f[2 * i + 1] = f2(__uint_as_float(a.z), __uint_as_float(a.w));
            }
        }
    }
    static __device__ __forceinline__ void put(T* p, uint32_t t, uint32_t n, uint32_t cols, const F2* f) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if (col(t, n, i * kPiece) >= cols) break;
            uint4 a;
            if (sizeof(T) == 2)
                a = make_uint4(pack_bf16(f[4 * i]), pack_bf16(f[4 * i + 1]), pack_bf16(f[4 * i + 2]), pack_bf16(f[4 * i + 3]));
            else
                a = make_uint4((uint32_t)f[2 * i].v, (uint32_t)(f[2 * i].v >> 32), (uint32_t)f[2 * i + 1].v, (uint32_t)(f[2 * i + 1].v >> 32));
            *reinterpret_cast<uint4*>(p + col(t, n, i * kPiece)) = a;
        }
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
    static __device__ __forceinline__ void put(T* p, uint32_t t, uint32_t n, uint32_t cols, const F2* f) {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (t + j * n < cols) p[t + j * n] = from_f<T>(f2_at(f, j));
    }
};

// How many rows a team works on at once, so that their reductions share shuffles and barriers, and how many are on
// their way or at work, in shared memory.
template <typename T, bool VEC, int INPUTS, int TEAM>
struct Rows {
    // an SM has 227 KB: of fp32 rows of more than 8192 columns the backward ring holds just the one at work
    static constexpr int kMost = INPUTS == 1 ? kRingForward : TEAM > 512 ? 128 : kRingBackward;
    static constexpr int kRowBytes = kPer * sizeof(T) * INPUTS;      // of a thread
    static constexpr int kBatch = VEC && sizeof(T) * INPUTS <= 4 && kMost >= 2 * kRowBytes ? 2 : 1;
    static constexpr int kRing = VEC ? kMost / kRowBytes : kBatch;
    static constexpr int kBytes = VEC ? kRing * kRowBytes : 0;
    static_assert(kRing % kBatch == 0 && kRing >= kBatch, "batches must not wrap around the ring");
};

// A thread's columns of row after row of INPUTS matrices: round k is row me + k * apart.
template <typename T, bool VEC, int INPUTS, int TEAM>
struct Feed {
    using R = Rows<T, VEC, INPUTS, TEAM>;
    static constexpr uint32_t kPieces = VEC ? kPer * sizeof(T) / 16 : 1;
    RowPart<T, VEC> next[INPUTS];                 // !VEC: one row ahead, in registers
    const T* from[INPUTS];                        // of the round to ask for next
    uint64_t step[INPUTS];
    uint32_t asked, rounds;                       // rounds asked for, rounds that have a row
    uint32_t t, n, cols, begin, end, at;          // shared memory of the ring; the oldest round
    __device__ __forceinline__ Feed(const NormParams& p, uint32_t smem, uint32_t me, uint32_t apart, uint32_t rounds_, uint32_t t_, uint32_t n_)
        : asked(0), rounds(rounds_), t(t_), n(n_), cols(p.cols), begin(smem + threadIdx.x * 16) {
        end = begin + R::kRing * INPUTS * kPieces * blockDim.x * 16;
        at = begin;
        from[0] = static_cast<const T*>(p.x) + me * p.x_ld;
        step[0] = apart * p.x_ld;
        if constexpr (INPUTS == 2) {
            from[1] = static_cast<const T*>(p.dout) + me * p.dout_ld;
            step[1] = apart * p.dout_ld;
        }
#pragma unroll
        for (int k = 0; k < R::kRing; ++k) ask();
    }
    // asks for the next round's row; a round without a row asks for nothing
    __device__ __forceinline__ void ask() {
        const bool live = asked < rounds;
        if constexpr (VEC) {
            if (live)
#pragma unroll
                for (int i = 0; i < INPUTS; ++i)
                    RowPart<T, true>::copy(at + i * kPieces * blockDim.x * 16, blockDim.x * 16, from[i], t, n, cols);
            copy_commit();
            at += INPUTS * kPieces * blockDim.x * 16;
            if (at == end) at = begin;
        } else if (live) {
#pragma unroll
            for (int i = 0; i < INPUTS; ++i) next[i].load(from[i], t, n, cols);
        }
        ++asked;
#pragma unroll
        for (int i = 0; i < INPUTS; ++i) from[i] += step[i];
    }
    // waits for the oldest kBatch rounds asked for and not done
    __device__ __forceinline__ void wait() {
        if constexpr (VEC) copy_wait<R::kRing - R::kBatch>();
    }
    // row j of those, matrix i
    __device__ __forceinline__ void get(int j, int i, F2 (&f)[kPer / 2]) const {
        if constexpr (VEC) RowPart<T, true>::get(at + (j * INPUTS + i) * kPieces * blockDim.x * 16, blockDim.x * 16, f);
        else next[i].get(f);
    }
};

// Sums of v[0..N) over the team, N a power of two; every member gets them.  Lanes first trade values, so that
// each goes on with half of them (4 sums take 6 shuffles, not 20).  TEAM > 32: the whole CTA, of at most TEAM threads
// (buf: N x 32 floats, not reused before the CTA has passed another barrier).
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* buf) {
    constexpr int kLanes = TEAM < 32 ? TEAM : 32;
    const uint32_t lane = threadIdx.x & 31;
    int o = kLanes / 2;
#pragma unroll
    for (int half = N / 2; half; half /= 2, o /= 2) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float give = upper ? v[i] : v[half + i], keep = upper ? v[half + i] : v[i];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, o);
        }
    }
    // now every group of kLanes / N lanes holds a share of one sum: sum i in the i-th group
    float s = v[0];
#pragma unroll
    for (; o; o /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (TEAM > 32) {
        const uint32_t warp = threadIdx.x / 32, warps = blockDim.x / 32;
        if (lane % (32 / N) == 0) buf[warp * N + lane / (32 / N)] = s;
        __syncthreads();
        s = 0.f;
        for (uint32_t w = lane / N; w < warps; w += 32 / N) s += buf[w * N + lane % N];
#pragma unroll
        for (int q = 16; q >= N; q /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, q);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = N == 1 ? s : __shfl_sync(0xFFFFFFFFu, s, i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = N == 1 ? s : __shfl_sync(0xFFFFFFFFu, s, i * (kLanes / N), kLanes);
    }
}

template <typename T, bool VEC, int TEAM, uint32_t KIND>
__global__ void __launch_bounds__(TEAM <= 32 ? kTeamThreads : TEAM) norm_forward_kernel(const NormParams p) {
    __shared__ float buf[2][64];
    const uint32_t n = TEAM <= 32 ? TEAM : blockDim.x;
    const uint32_t t = TEAM <= 32 ? threadIdx.x % n : threadIdx.x;
    const uint32_t teams = TEAM <= 32 ? gridDim.x * (kTeamThreads / n) : gridDim.x;
    const uint32_t me = TEAM <= 32 ? blockIdx.x * (kTeamThreads / n) + threadIdx.x / n : blockIdx.x;
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
    extern __shared__ __align__(16) uint8_t norm_smem[];
    Feed<T, VEC, 1, TEAM> feed(p, (uint32_t)__cvta_generic_to_shared(norm_smem), me, teams, me < p.rows ? (p.rows - me + teams - 1) / teams : 0, t, n);
    constexpr int B = Rows<T, VEC, 1, TEAM>::kBatch;
    // all lanes of a warp go round together, so that shuffles stay full; a team past the end idles
    const uint32_t rounds = (p.rows + teams * B - 1) / (teams * B);
    uint32_t row = me;
    for (uint32_t k = 0; k < rounds; ++k, row += teams * B) {
        if (TEAM > 32 && row >= p.rows) break;
        F2 f[B][kPer / 2];
        float mean[B], q[B];
        feed.wait();
#pragma unroll
        for (int j = 0; j < B; ++j) feed.get(j, 0, f[j]);
        if (KIND == DTE_NORM_LAYER) {
#pragma unroll
            for (int j = 0; j < B; ++j) {
                F2 a = f2_add(f[j][0], f[j][1]);
#pragma unroll
                for (int i = 2; i < kPer / 2; i += 2) a = f2_add(a, f2_add(f[j][i], f[j][i + 1]));
                mean[j] = f2_sum(a);
            }
            team_sum<TEAM, B>(mean, buf[0]);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                mean[j] *= p.inv_cols;
                const F2 m = f2(-mean[j], -mean[j]);
#pragma unroll
                for (int i = 0; i < kPer / 2; ++i) f[j][i] = f2_fma(in[i], m, f[j][i]);
            }
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            F2 q2 = f2_mul(f[j][0], f[j][0]);
#pragma unroll
            for (int i = 1; i < kPer / 2; ++i) q2 = f2_fma(f[j][i], f[j][i], q2);
            q[j] = f2_sum(q2);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) feed.ask();              // into the places that these rows have left
        team_sum<TEAM, B>(q, KIND == DTE_NORM_LAYER ? buf[1] : buf[k & 1]);
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t r = row + j * teams;
            if (r >= p.rows) break;
            const float rstd = 1.f / sqrtf(q[j] * p.inv_cols + p.eps);
            const F2 s = f2(rstd, rstd);
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) f[j][i] = f2_fma(f2_mul(f[j][i], s), w[i], b[i]);
            RowPart<T, VEC>::put(y + r * p.out_ld, t, n, p.cols, f[j]);
            if (t == 0) {
                if (KIND == DTE_NORM_LAYER && p.mean) p.mean[r] = mean[j];
                if (p.rstd) p.rstd[r] = rstd;
            }
        }
    }
}

template <typename T, bool VEC, int TEAM, uint32_t KIND>
__global__ void __launch_bounds__(TEAM <= 32 ? kTeamThreads : TEAM, TEAM <= 32 ? 2 : 1) norm_backward_kernel(const NormParams p) {
    __shared__ float buf[2][128];
    const uint32_t n = TEAM <= 32 ? TEAM : blockDim.x;
    const uint32_t t = TEAM <= 32 ? threadIdx.x % n : threadIdx.x;
    const uint32_t teams = TEAM <= 32 ? gridDim.x * (kTeamThreads / n) : gridDim.x;
    const uint32_t team = TEAM <= 32 ? blockIdx.x * (kTeamThreads / n) + threadIdx.x / n : blockIdx.x;
    constexpr int B = Rows<T, VEC, 2, TEAM>::kBatch, S = KIND == DTE_NORM_LAYER ? 2 : 1;
    const uint32_t rounds = (p.rows + teams * B - 1) / (teams * B);
    // a CTA's rows follow one another (every 296th row: 3 us more of 84, without centring); teams of a CTA share out its stretch row by row
    const uint32_t apart = TEAM > 32 ? 1 : teams, me = TEAM > 32 ? team * rounds * B : team;
    const uint32_t end = TEAM > 32 ? min(me + rounds * B, p.rows) : p.rows;
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
    extern __shared__ __align__(16) uint8_t norm_smem[];
    Feed<T, VEC, 2, TEAM> feed(p, (uint32_t)__cvta_generic_to_shared(norm_smem), me, apart, me < end ? (end - me + apart - 1) / apart : 0, t, n);
    float nmean[B], nrstd[B];                               // statistics of the next rounds
    auto fetch = [&](uint32_t row) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t r = row + j * apart;
            nmean[j] = KIND == DTE_NORM_LAYER && r < end ? p.mean[r] : 0.f;
            nrstd[j] = r < end ? p.rstd[r] : 0.f;
        }
    };
    fetch(me);
    uint32_t row = me;
    for (uint32_t k = 0; k < rounds; ++k, row += apart * B) {
        if (TEAM > 32 && row >= end) break;
        float sums[B * S];
        F2 r[B], m[B];                                      // xhat = (x + m) * r: centred first, so that an offset of the row costs no digits
#pragma unroll
        for (int j = 0; j < B; ++j) {
            r[j] = f2(nrstd[j], nrstd[j]);
            m[j] = f2(-nmean[j], -nmean[j]);
        }
        fetch(row + apart * B);
        feed.wait();
#pragma unroll
        for (int j = 0; j < B; ++j) {
            F2 xh[kPer / 2], g[kPer / 2];
            feed.get(j, 0, xh);
            feed.get(j, 1, g);
            const bool live = row + j * apart < end;
            F2 s2 = f2(0.f, 0.f), s1 = f2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) {
                // columns past the end hold zero in g and w, so they add nothing: xh is finite there
                xh[i] = f2_mul(KIND == DTE_NORM_LAYER ? f2_add(xh[i], m[j]) : xh[i], r[j]);
                if (live) {
                    dw[i] = f2_fma(g[i], xh[i], dw[i]);
                    if (KIND == DTE_NORM_LAYER || p.want_bias) db[i] = f2_add(db[i], g[i]);
                }
                g[i] = f2_mul(g[i], w[i]);
                s2 = f2_fma(g[i], xh[i], s2);
                if (KIND == DTE_NORM_LAYER) s1 = f2_add(s1, g[i]);
            }
            sums[j * S] = f2_sum(s2);
            if (S == 2) sums[j * S + 1] = f2_sum(s1);
        }
        team_sum<TEAM, B * S>(sums, buf[k & 1]);
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t at = row + j * apart;
            if (at < end && dx) {
                // rstd * (g - c1 - xh * c2); the row is read from shared memory again: cheaper than its registers
                float rstd, unused;
                f2_get(r[j], rstd, unused);
                const float c2 = -sums[j * S] * p.inv_cols * rstd, c1 = S == 2 ? -sums[j * S + S - 1] * p.inv_cols * rstd : 0.f;
                const F2 a = f2(c2, c2), b = f2(c1, c1);
                F2 xh[kPer / 2], g[kPer / 2];
                feed.get(j, 0, xh);
                feed.get(j, 1, g);
#pragma unroll
                for (int i = 0; i < kPer / 2; ++i) {
                    xh[i] = f2_mul(KIND == DTE_NORM_LAYER ? f2_add(xh[i], m[j]) : xh[i], r[j]);
                    g[i] = f2_mul(g[i], w[i]);
                    g[i] = f2_fma(xh[i], a, KIND == DTE_NORM_LAYER ? f2_fma(g[i], r[j], b) : f2_mul(g[i], r[j]));
                }
                RowPart<T, VEC>::put(dx + at * p.out_ld, t, n, p.cols, g);
            }
        }
#pragma unroll
        for (int j = 0; j < B; ++j) feed.ask();              // into the places that these rows have left
    }
    if (!p.partial) return;
    if (TEAM <= 32) {
        // the CTA's teams hold sums of the same columns: add them up in order of the teams
        __shared__ float sums[kTeamThreads * kPer];
        constexpr uint32_t kTeams = TEAM <= 32 ? kTeamThreads / TEAM : 1;
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                sums[(threadIdx.x / n) * (n * kPer) + RowPart<T, VEC>::col(t, n, j)] = f2_at(which ? db : dw, j);
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < p.cols; c += kTeamThreads) {
                float v = 0.f;
                for (uint32_t m = 0; m < kTeams; ++m) v += sums[m * (n * kPer) + c];
                p.partial[((uint64_t)blockIdx.x * 2 + which) * p.cols + c] = v;
            }
            __syncthreads();
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
#pragma unroll 10
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

constexpr unsigned kCtasPerSm = 8;       // at most

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

template <typename T, bool VEC, int TEAM, uint32_t KIND>
static dte_status forward_as(const NormParams& p, const NormShape& s, int device, cudaStream_t st) {
    constexpr size_t kPerThread = Rows<T, VEC, 1, TEAM>::kBytes;
    static std::atomic<uint64_t> ready{0};
    dte_status r = allow_smem(norm_forward_kernel<T, VEC, TEAM, KIND>, kPerThread * (TEAM <= 32 ? kTeamThreads : TEAM), device, ready);
    if (r != DTE_OK) return r;
    norm_forward_kernel<T, VEC, TEAM, KIND><<<s.ctas, s.threads, kPerThread * s.threads, st>>>(p);
    return DTE_OK;
}

template <typename T, bool VEC, uint32_t KIND>
static dte_status forward_team(const NormParams& p, const NormShape& s, int device, cudaStream_t st) {
    if (s.team == 0) {
        norm_forward_long_kernel<T, KIND><<<s.ctas, s.threads, 0, st>>>(p);
        return DTE_OK;
    }
    if (s.team == 8) return forward_as<T, VEC, 8, KIND>(p, s, device, st);
    if (s.team == 16) return forward_as<T, VEC, 16, KIND>(p, s, device, st);
    if (s.team == 32) return forward_as<T, VEC, 32, KIND>(p, s, device, st);
    if (s.team == 512) return forward_as<T, VEC, 512, KIND>(p, s, device, st);
    return forward_as<T, VEC, 1024, KIND>(p, s, device, st);
}

template <typename T, bool VEC, int TEAM, uint32_t KIND>
static dte_status backward_as(const NormParams& p, const NormShape& s, int device, cudaStream_t st) {
    constexpr size_t kPerThread = Rows<T, VEC, 2, TEAM>::kBytes;
    static std::atomic<uint64_t> ready{0};
    dte_status r = allow_smem(norm_backward_kernel<T, VEC, TEAM, KIND>, kPerThread * (TEAM <= 32 ? kTeamThreads : TEAM), device, ready);
    if (r != DTE_OK) return r;
    norm_backward_kernel<T, VEC, TEAM, KIND><<<s.ctas, s.threads, kPerThread * s.threads, st>>>(p);
    return DTE_OK;
}

template <typename T, bool VEC, uint32_t KIND>
static dte_status backward_team(const NormParams& p, const NormShape& s, int device, cudaStream_t st) {
    if (s.team == 0) {
        if (p.out) norm_backward_long_kernel<T, KIND><<<s.ctas, s.threads, 0, st>>>(p);
        if (p.partial) norm_columns_long_kernel<T, KIND><<<dim3((p.cols + 255) / 256, s.ctas), 256, 0, st>>>(p);
        return DTE_OK;
    }
    if (s.team == 8) return backward_as<T, VEC, 8, KIND>(p, s, device, st);
    if (s.team == 16) return backward_as<T, VEC, 16, KIND>(p, s, device, st);
    if (s.team == 32) return backward_as<T, VEC, 32, KIND>(p, s, device, st);
    if (s.team == 512) return backward_as<T, VEC, 512, KIND>(p, s, device, st);
    return backward_as<T, VEC, 1024, KIND>(p, s, device, st);
}

template <bool BACK, typename T, bool VEC, uint32_t KIND>
static dte_status norm_direction(const NormParams& p, const NormShape& s, int device, cudaStream_t st) {
    if constexpr (BACK) return backward_team<T, VEC, KIND>(p, s, device, st);
    else return forward_team<T, VEC, KIND>(p, s, device, st);
}

template <bool BACK, uint32_t KIND>
static dte_status norm_launch(const NormParams& p, const NormShape& s, bool bf16, bool vec, int device, cudaStream_t st) {
    if (bf16 && vec) return norm_direction<BACK, __nv_bfloat16, true, KIND>(p, s, device, st);
    if (bf16) return norm_direction<BACK, __nv_bfloat16, false, KIND>(p, s, device, st);
    if (vec) return norm_direction<BACK, float, true, KIND>(p, s, device, st);
    return norm_direction<BACK, float, false, KIND>(p, s, device, st);
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
    if (!(eps >= 0) || !std::isfinite((float)eps)) return op_fail(DTE_ERR_INVALID_ARG, "eps must be finite in fp32 and >= 0");
    if (x->rows != out->rows || x->cols != out->cols || x->dtype != out->dtype)
        return op_fail(DTE_ERR_INVALID_ARG, "out must have x's shape and type");
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3u) return op_fail(DTE_ERR_INVALID_ARG, "mean / rstd must be 4-byte aligned");
    if (x->rows == 0) return DTE_OK;
    OpDeviceGuard g;
    int sms = 0;
    if ((s = g.enter(device, &sms)) != DTE_OK) return s;
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
    const NormShape sh = norm_shape(x->rows, x->cols, sms, kSmThreadsForward);
    const bool bf16 = x->dtype == DTE_BF16, vec = vec8_ok(x) && vec8_ok(out);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    s = kind == DTE_NORM_LAYER ? norm_launch<false, DTE_NORM_LAYER>(p, sh, bf16, vec, device, st)
                               : norm_launch<false, DTE_NORM_RMS>(p, sh, bf16, vec, device, st);
    if (s != DTE_OK) return s;
    DTE_CUDA(cudaGetLastError());
    return DTE_OK;
}

extern "C" uint64_t dte_norm_backward_workspace_bytes(uint64_t rows, uint64_t hidden) {
    if (rows >= kMaxDim || hidden >= kMaxDim) return UINT64_MAX;    // refused by the call
    const NormShape s = norm_shape(rows, hidden, kMostSms, kSmThreadsBackward);
    return align_up((uint64_t)s.ctas * 2 * hidden * sizeof(float), kWorkspaceAlign);
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
    OpDeviceGuard g;
    int sms = 0;
    if ((s = g.enter(device, &sms)) != DTE_OK) return s;
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
    const NormShape sh = norm_shape(x->rows, x->cols, sms, kSmThreadsBackward);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (x->rows) {
        const bool bf16 = x->dtype == DTE_BF16, vec = vec8_ok(x) && vec8_ok(dout) && (!dx || vec8_ok(dx));
        s = kind == DTE_NORM_LAYER ? norm_launch<true, DTE_NORM_LAYER>(p, sh, bf16, vec, device, st)
                                   : norm_launch<true, DTE_NORM_RMS>(p, sh, bf16, vec, device, st);
        if (s != DTE_OK) return s;
        DTE_CUDA(cudaGetLastError());
    }
    if (want) {
        DTE_CUDA(launch_after(norm_sums_kernel, dim3((p.cols + 31) / 32, 2), 1024, 0, st, p.partial, x->rows ? sh.ctas : 0, p.cols,
                              accumulate != 0, dweight, dbias));
    }
    return DTE_OK;
}
