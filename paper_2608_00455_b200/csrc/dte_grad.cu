// Global gradient norm and clipping over many tensors.
//
// Both kernels are streams bound by memory: the norm reads every element once, clipping reads and writes every
// element once.  Measured: sum of 965 M bf16 300 us = 6.4 TB/s, of 75 M fp32 51 us; clipping them into fp32 985 us = 5.9 TB/s and 97 us =
// 6.2 TB/s (a copy: 6.46), in place 614 us = 6.3 TB/s and 108 us = 5.5 TB/s; six tensors of 2 M elements 3 + 2 + 4.5 us.  The list of
// tensors travels in the launch's parameters, so a call needs no copy to the device and can be captured; a CTA finds the tensor of its next chunk by bisection.
#include "dte_ops.cuh"

namespace dte {

// Tensors in a launch's parameters: 28 bytes each of the 32764 that it may carry; few tensors take the short list, because
// parameters cost the host time.
constexpr uint32_t kListTensors = 1024, kShortList = 64;
constexpr uint32_t kGradThreads = 256;
constexpr uint32_t kGradChunk = 16384;              // elements of a chunk, the unit of work of a CTA
constexpr uint32_t kGradGrid = 148 * 8;             // CTAs at most, whatever the device has: the order of the sums
constexpr uint64_t kMaxElements = 1ull << 44;       // of all tensors together: chunks are numbered in 32 bits
constexpr uint64_t kInBf16 = 1ull << 63, kOutBf16 = 1ull << 62;      // in GradList::numel

template <uint32_t N>
struct GradList {
    static constexpr uint32_t kMost = N;
    const void* in[N];
    void* out[N];
    uint64_t numel[N];
    uint32_t first[N + 1];                          // first chunk of each tensor, then the number of chunks
    uint32_t n;
};

template <uint32_t N>
struct SumParams {
    GradList<N> list;
    double* part;                                   // one per CTA
};

template <uint32_t N>
struct ClipParams {
    GradList<N> list;
    const double* sum_squares;
    float* norm;
    double max_norm;
};
static_assert(sizeof(SumParams<kListTensors>) <= 32764 && sizeof(ClipParams<kListTensors>) <= 32764, "a launch carries at most 32764 bytes");

template <uint32_t N>
__device__ __forceinline__ uint32_t tensor_of(const GradList<N>& l, uint32_t chunk) {
    uint32_t lo = 0, hi = l.n;                      // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (l.first[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}

// Sum of the squares of the n values in f.  In fp32 where none of them can have been lost there: a sum
// above 2^100 may have overflowed, one below 2^-80 may lack squares below fp32's range.
template <int N>
__device__ __forceinline__ double sum_squares_of(const float (&f)[N]) {
    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j) a[j % 4] = fmaf(f[j], f[j], a[j % 4]);
    const float s = (a[0] + a[1]) + (a[2] + a[3]);
    if (s < 0x1p100f && s > 0x1p-80f) return s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < N; ++j) d = fma((double)f[j], (double)f[j], d);
    return d;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// The CTA's sum, in thread 0.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_warp[kGradThreads / 32];
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x / 32] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (uint32_t w = 1; w < kGradThreads / 32; ++w) v += s_warp[w];
    return v;
}

template <typename T>
__device__ double chunk_squares(const T* x, uint32_t n) {
    double sum = 0.0;
    uint32_t at = 0;
    if (!((uintptr_t)x & 15u)) {
        constexpr uint32_t kPer = 32, kStep = kGradThreads * kPer;
        for (; at + kStep <= n; at += kStep) {
            Raw8<T> r[kPer / 8];
            float f[kPer];
#pragma unroll
            for (uint32_t j = 0; j < kPer / 8; ++j) r[j].load_cs(x + at + (j * kGradThreads + threadIdx.x) * 8);
#pragma unroll
            for (uint32_t j = 0; j < kPer / 8; ++j) r[j].get(f + 8 * j);
            sum += sum_squares_of(f);
        }
        for (uint32_t i = at + threadIdx.x * 8; i + 8 <= n; i += kGradThreads * 8) {
            Raw8<T> r;
            float f[8];
            r.load_cs(x + i);
            r.get(f);
            sum += sum_squares_of(f);
        }
        at = n / 8 * 8;
    }
    for (uint32_t i = at + threadIdx.x; i < n; i += kGradThreads) {
        const float f[1] = {to_f(x[i])};
        sum += sum_squares_of(f);
    }
    return sum;
}

template <uint32_t N>
__global__ void __launch_bounds__(kGradThreads) sum_squares_kernel(const __grid_constant__ SumParams<N> p) {
    const GradList<N>& l = p.list;
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < l.first[l.n]; c += gridDim.x) {
        const uint32_t t = tensor_of(l, c);
        const uint64_t numel = l.numel[t] & ~(kInBf16 | kOutBf16), at = (uint64_t)(c - l.first[t]) * kGradChunk;
        const uint32_t n = (uint32_t)(numel - at < kGradChunk ? numel - at : kGradChunk);
        if (l.numel[t] & kInBf16) sum += chunk_squares(static_cast<const __nv_bfloat16*>(l.in[t]) + at, n);
        else sum += chunk_squares(static_cast<const float*>(l.in[t]) + at, n);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) p.part[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kGradThreads) join_squares_kernel(const double* part, uint32_t n, double* out, bool accumulate) {
    wait_for_earlier();
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += kGradThreads) sum += part[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) *out = accumulate ? *out + sum : sum;
}

constexpr float kTinyUnit = 0x1p-126f;
// y = x * factor; TINY: times kTinyUnit, for factors that fp32 would hold as subnormal numbers (see clip_kernel).
template <bool TINY, typename In, typename Out>
__device__ void chunk_scale(const In* x, Out* y, uint32_t n, float factor) {
    uint32_t at = 0;
    if (!(((uintptr_t)x | (uintptr_t)y) & 15u)) {
        auto finish = [&](const Raw8<In>& r, uint32_t i) {
            Raw8<Out> o;
            float f[8];
            r.get(f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = TINY ? f[j] * factor * kTinyUnit : f[j] * factor;
            o.set(f);
            o.store(y + i);
        };
        constexpr uint32_t kAhead = 4, kStep = kGradThreads * 8;
        uint32_t i = threadIdx.x * 8;
        for (; at + kAhead * kStep <= n; at += kAhead * kStep, i += kAhead * kStep) {
            Raw8<In> r[kAhead];
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) r[j].load_cs(x + i + j * kStep);
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) finish(r[j], i + j * kStep);
        }
        for (; i + 8 <= n; i += kStep) {
            Raw8<In> r;
            r.load_cs(x + i);
            finish(r, i);
        }
        at = n / 8 * 8;
    }
    for (uint32_t i = at + threadIdx.x; i < n; i += kGradThreads) y[i] = from_f<Out>(TINY ? to_f(x[i]) * factor * kTinyUnit : to_f(x[i]) * factor);
}

// This CTA's chunks of all tensors.
template <bool TINY, uint32_t N>
__device__ __forceinline__ void scale_chunks(const GradList<N>& l, float factor) {
    for (uint32_t c = blockIdx.x; c < l.first[l.n]; c += gridDim.x) {
        const uint32_t t = tensor_of(l, c);
        const bool in16 = l.numel[t] & kInBf16, out16 = l.numel[t] & kOutBf16;
        if (!TINY && factor == 1.f && l.in[t] == l.out[t]) continue;
        const uint64_t numel = l.numel[t] & ~(kInBf16 | kOutBf16), at = (uint64_t)(c - l.first[t]) * kGradChunk;
        const uint32_t n = (uint32_t)(numel - at < kGradChunk ? numel - at : kGradChunk);
        const __nv_bfloat16* x16 = static_cast<const __nv_bfloat16*>(l.in[t]) + at;
        const float* x32 = static_cast<const float*>(l.in[t]) + at;
        __nv_bfloat16* y16 = static_cast<__nv_bfloat16*>(l.out[t]) + at;
        float* y32 = static_cast<float*>(l.out[t]) + at;
        if (in16 && out16) chunk_scale<TINY>(x16, y16, n, factor);
        else if (in16) chunk_scale<TINY>(x16, y32, n, factor);
        else if (out16) chunk_scale<TINY>(x32, y16, n, factor);
        else chunk_scale<TINY>(x32, y32, n, factor);
    }
}

template <uint32_t N>
__global__ void __launch_bounds__(kGradThreads) clip_kernel(const __grid_constant__ ClipParams<N> p) {
    const double norm = sqrt(*p.sum_squares);
    const float shown = (float)norm;
    if (p.norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = shown;
    // a norm that is not finite, as the caller sees it, leaves everything as it is
    const double quotient = norm > p.max_norm && shown <= 0x1.fffffep127f ? p.max_norm / norm : 1.0;
    // Below fp32's normal numbers the quotient would lose bits that a large element's product can hold: it is brought up by 2^126,
    // and the product down again, which is exact unless the product is itself subnormal.
    if (quotient < (double)kTinyUnit) scale_chunks<true>(p.list, (float)(quotient / (double)kTinyUnit));
    else scale_chunks<false>(p.list, (float)quotient);
}

static dte_status check_tensors(const dte_tensor* t, uint64_t n) {
    if (n && !t) return op_fail(DTE_ERR_INVALID_ARG, "tensors are null");
    if (n > (1u << 20)) return op_fail(DTE_ERR_INVALID_ARG, "at most 2^20 tensors");
    uint64_t all = 0;
    for (uint64_t i = 0; i < n; ++i) {
        if (t[i].dtype != DTE_F32 && t[i].dtype != DTE_BF16) return op_fail(DTE_ERR_INVALID_ARG, "tensors must be DTE_F32 or DTE_BF16");
        if (t[i].numel > kMaxElements || (all += t[i].numel) > kMaxElements)
            return op_fail(DTE_ERR_INVALID_ARG, "at most 2^44 elements in one call");
        if (t[i].numel && !t[i].data) return op_fail(DTE_ERR_INVALID_ARG, "a tensor's data is null");
        if ((uintptr_t)t[i].data & (elem_size(t[i].dtype) - 1)) return op_fail(DTE_ERR_INVALID_ARG, "a tensor is not aligned to its type");
    }
    return DTE_OK;
}

// The next launch's share of the tensors from `from` on, empty ones left out.  Returns where the one after it starts.
template <uint32_t N>
static uint64_t fill(GradList<N>& l, const dte_tensor* t, const dte_tensor* outs, uint64_t from, uint64_t n) {
    uint64_t chunks = 0;
    l.n = 0;
    for (; from < n && l.n < N; ++from) {
        const dte_tensor& a = t[from];
        const dte_tensor& b = outs ? outs[from] : a;
        if (a.numel == 0) continue;
        l.in[l.n] = a.data;
        l.out[l.n] = b.data;
        l.numel[l.n] = a.numel | (a.dtype == DTE_BF16 ? kInBf16 : 0) | (b.dtype == DTE_BF16 ? kOutBf16 : 0);
        l.first[l.n++] = (uint32_t)chunks;
        chunks += (a.numel + kGradChunk - 1) / kGradChunk;
    }
    l.first[l.n] = (uint32_t)chunks;
    return from;
}

template <uint32_t N>
static uint32_t grid_of(const GradList<N>& l) { return l.first[l.n] < kGradGrid ? l.first[l.n] : kGradGrid; }

static uint64_t launches_of(uint64_t n) { return (n + kListTensors - 1) / kListTensors; }

template <uint32_t N>
static dte_status launch_sums(const dte_tensor* tensors, uint64_t n, double* part, uint32_t& parts, cudaStream_t st) {
    SumParams<N> p;
    for (uint64_t at = 0; at < n;) {
        at = fill(p.list, tensors, nullptr, at, n);
        if (p.list.n == 0) break;
        p.part = part + parts;
        const uint32_t grid = grid_of(p.list);
        sum_squares_kernel<N><<<grid, kGradThreads, 0, st>>>(p);
        DTE_CUDA(cudaGetLastError());
        parts += grid;
    }
    return DTE_OK;
}

template <uint32_t N>
static dte_status launch_clip(const dte_tensor* tensors, uint64_t n, const double* sum_squares, double max_norm, const dte_tensor* outs,
                              float* norm, cudaStream_t st) {
    ClipParams<N> p;
    p.sum_squares = sum_squares;
    p.norm = norm;
    p.max_norm = max_norm;
    for (uint64_t at = 0; at < n || p.norm;) {
        at = fill(p.list, tensors, outs, at, n);
        if (p.list.n == 0 && !p.norm) break;
        // A CTA per chunk, in the order of addresses, writes fastest (965 M bf16 into fp32: 985 us, a fixed grid 1200); in place the CTAs are
        // few, because where nothing is clipped starting them is all the work there is (75 M fp32: 6 us, 965 M bf16: 58).
        const uint32_t grid = outs ? p.list.first[p.list.n] : grid_of(p.list);
        clip_kernel<N><<<grid ? grid : 1, kGradThreads, 0, st>>>(p);
        DTE_CUDA(cudaGetLastError());
        p.norm = nullptr;              // written by the first launch
    }
    return DTE_OK;
}

}  // namespace dte

using namespace dte;

extern "C" uint64_t dte_grad_sum_squares_workspace_bytes(uint64_t n_tensors) {
    if (n_tensors > (1u << 20)) return UINT64_MAX;      // refused by the call
    return align_up((launches_of(n_tensors) + 1) * kGradGrid * sizeof(double), kWorkspaceAlign);
}

extern "C" dte_status dte_grad_sum_squares(const dte_tensor* tensors, uint64_t n_tensors, int accumulate, double* sum_squares,
                                           void* workspace, uint64_t workspace_bytes, int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_tensors(tensors, n_tensors)) != DTE_OK) return s;
    if (!sum_squares || ((uintptr_t)sum_squares & 7u)) return op_fail(DTE_ERR_INVALID_ARG, "sum_squares is null or not 8-byte aligned");
    if ((s = check_workspace(workspace, workspace_bytes, dte_grad_sum_squares_workspace_bytes(n_tensors))) != DTE_OK) return s;
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    double* part = static_cast<double*>(workspace);
    uint32_t parts = 0;
    s = n_tensors <= kShortList ? launch_sums<kShortList>(tensors, n_tensors, part, parts, st) : launch_sums<kListTensors>(tensors, n_tensors, part, parts, st);
    if (s != DTE_OK) return s;
    DTE_CUDA(launch_after(join_squares_kernel, dim3(1), kGradThreads, 0, st, part, parts, sum_squares, accumulate != 0));
    return DTE_OK;
}

extern "C" dte_status dte_grad_clip(const dte_tensor* tensors, uint64_t n_tensors, const double* sum_squares, double max_norm,
                                    const dte_tensor* outs, float* norm, int device, void* cuda_stream) {
    dte_status s;
    if ((s = check_tensors(tensors, n_tensors)) != DTE_OK) return s;
    if (outs && (s = check_tensors(outs, n_tensors)) != DTE_OK) return s;
    for (uint64_t i = 0; outs && i < n_tensors; ++i) {
        if (outs[i].numel != tensors[i].numel) return op_fail(DTE_ERR_INVALID_ARG, "outs must have the tensors' sizes");
        if (outs[i].numel && outs[i].data == tensors[i].data && outs[i].dtype != tensors[i].dtype)
            return op_fail(DTE_ERR_INVALID_ARG, "a tensor clipped in place keeps its type");
    }
    if (!sum_squares || ((uintptr_t)sum_squares & 7u)) return op_fail(DTE_ERR_INVALID_ARG, "sum_squares is null or not 8-byte aligned");
    if (!(max_norm > 0) || !std::isfinite(max_norm)) return op_fail(DTE_ERR_INVALID_ARG, "max_norm must be > 0 and finite");
    if ((uintptr_t)norm & 3u) return op_fail(DTE_ERR_INVALID_ARG, "norm must be 4-byte aligned");
    OpDeviceGuard g;
    if ((s = g.enter(device)) != DTE_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    return n_tensors <= kShortList ? launch_clip<kShortList>(tensors, n_tensors, sum_squares, max_norm, outs, norm, st)
                                   : launch_clip<kListTensors>(tensors, n_tensors, sum_squares, max_norm, outs, norm, st);
}
