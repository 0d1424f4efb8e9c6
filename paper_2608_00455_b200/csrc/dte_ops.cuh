// Shared by the operators at the two ends of the model (embedding, norm, linear cross entropy):
// argument checks on the host, typed vector access and reductions on the device, and the sorted-token
// sum that the embedding gradient and the head's gradient both need.
#pragma once

#include <cuda_bf16.h>

#include <atomic>
#include <cmath>

#include "dte_internal.cuh"

namespace dte {

constexpr uint64_t kWorkspaceAlign = 256;

inline uint64_t align_up(uint64_t n, uint64_t a) { return (n + a - 1) / a * a; }

// ---- host: argument checks ------------------------------------------------------------------------
inline dte_status op_fail(dte_status s, const char* msg) {
    set_error(msg);
    return s;
}

dte_status device_sms(int device, int* sms);   // checks the ordinal; multiprocessor count, cached per device

// Makes `device` current for a call.  The ordinal is checked first: nothing runs on another device instead, and a refused
// one leaves no CUDA error behind for a later call to find.
struct OpDeviceGuard {
    int prev = -1;
    dte_status enter(int dev, int* sms = nullptr) {
        int known = 0;
        const dte_status s = device_sms(dev, sms ? sms : &known);
        if (s != DTE_OK) return s;
        DTE_CUDA(cudaGetDevice(&prev));
        if (prev == dev) {
            prev = -1;
            return DTE_OK;
        }
        const cudaError_t e = cudaSetDevice(dev);
        if (e != cudaSuccess) {
            prev = -1;
            return cuda_fail(e, "cudaSetDevice");
        }
        return DTE_OK;
    }
    ~OpDeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

inline uint32_t elem_size(uint32_t dtype) { return dtype == DTE_BF16 ? 2u : dtype == DTE_I64 ? 8u : 4u; }

// Multiplications and the vector kernels' index arithmetic stay far below 2^63 with these limits.
constexpr uint64_t kMaxDim = 1ull << 31;

inline dte_status check_matrix(const dte_matrix* m, const char* null_msg, bool output) {
    if (!m) return op_fail(DTE_ERR_INVALID_ARG, null_msg);
    if (m->dtype != DTE_F32 && m->dtype != DTE_BF16) return op_fail(DTE_ERR_INVALID_ARG, "matrix dtype must be DTE_F32 or DTE_BF16");
    if (m->cols == 0 || m->cols >= kMaxDim || m->rows >= kMaxDim || m->ld >= (1ull << 40))
        return op_fail(DTE_ERR_INVALID_ARG, "matrix needs 1 <= cols < 2^31, rows < 2^31 and ld < 2^40");
    if (m->rows && !m->data) return op_fail(DTE_ERR_INVALID_ARG, null_msg);
    if ((uintptr_t)m->data & (elem_size(m->dtype) - 1)) return op_fail(DTE_ERR_INVALID_ARG, "matrix data is not aligned to its element type");
    if (output && m->rows > 1 && m->ld < m->cols) return op_fail(DTE_ERR_INVALID_ARG, "output rows overlap: ld < cols");
    return DTE_OK;
}

inline dte_status check_ids(const dte_ids* t) {
    if (!t || (t->count && !t->data)) return op_fail(DTE_ERR_INVALID_ARG, "ids are null");
    if (t->dtype != DTE_I32 && t->dtype != DTE_I64) return op_fail(DTE_ERR_INVALID_ARG, "ids must be DTE_I32 or DTE_I64");
    if ((uintptr_t)t->data & (elem_size(t->dtype) - 1)) return op_fail(DTE_ERR_INVALID_ARG, "ids are not aligned to their type");
    if (t->count >= kMaxDim) return op_fail(DTE_ERR_INVALID_ARG, "ids.count must be < 2^31");
    return DTE_OK;
}

inline dte_status check_range(uint64_t start, uint64_t rows, uint64_t vocab) {
    if (vocab >= (1ull << 62) || start > vocab || rows > vocab - start)
        return op_fail(DTE_ERR_INVALID_ARG, "the shard's rows do not lie inside the vocabulary");
    return DTE_OK;
}

inline dte_status check_workspace(const void* ws, uint64_t have, uint64_t need) {
    if ((uintptr_t)ws & (kWorkspaceAlign - 1)) return op_fail(DTE_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (have < need) return op_fail(DTE_ERR_CAPACITY, "workspace is too small; see the operator's workspace_bytes");
    if (need && !ws) return op_fail(DTE_ERR_INVALID_ARG, "workspace is null");
    return DTE_OK;
}

// 16-byte accesses of whole rows: data and every row start aligned, columns a multiple of 8 elements.
inline bool vec8_ok(const dte_matrix* m) {
    const uint64_t unit = 16 / elem_size(m->dtype);
    return !((uintptr_t)m->data & 15u) && (m->cols % 8 == 0) && (m->rows <= 1 || m->ld % unit == 0);
}

// Pairs of elements: data, every row start and the number of columns a multiple of two.
inline bool vec2_ok(const dte_matrix* m) {
    return !((uintptr_t)m->data & (2 * elem_size(m->dtype) - 1)) && m->cols % 2 == 0 && (m->rows <= 1 || m->ld % 2 == 0);
}

inline int vec_of(const dte_matrix* a, const dte_matrix* b) {
    return vec8_ok(a) && vec8_ok(b) ? 8 : vec2_ok(a) && vec2_ok(b) ? 2 : 1;
}

// Raises a kernel's dynamic shared memory limit, once per device.
template <typename Kernel>
inline dte_status allow_smem(Kernel* kernel, size_t bytes, int device, std::atomic<uint64_t>& done) {
    const uint64_t bit = 1ull << device;                 // device < kMaxDevices = 64: checked by device_sms
    if (done.load(std::memory_order_relaxed) & bit) return DTE_OK;
    DTE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done.fetch_or(bit, std::memory_order_relaxed);
    return DTE_OK;
}

// ---- sums over the tokens of a row -----------------------------------------------------------------
// out[row] = scale * sum over the entries with that row of weight[entry] * src[entry], in the order of the entries
struct SortedSum {
    // row of an entry: id - row_start where that lies in [0, rows), else the entry is dropped
    const void* ids;
    uint32_t ids_dtype;
    uint32_t n;               // entries
    int64_t row_start;
    uint64_t vocab;
    uint32_t rows;
    const void* src;          // n x hidden
    uint32_t src_dtype;
    uint64_t src_ld;
    const float* weight;      // per entry, or NULL; with weights: src bf16, out fp32 compact
    uint32_t hidden;
    float scale;
    // compact: out is fp32, n x hidden, and the sum of a row lies at position first[row] (see
    // sorted_sum_first) if first[row + 1] > first[row]; else out is rows x hidden of out_dtype, added to or written whole
    void* out;
    uint32_t out_dtype;
    uint64_t out_ld;
    bool accumulate, compact;
    uint64_t* flags;
};
uint64_t sorted_sum_workspace_bytes(uint64_t n, uint64_t rows, uint64_t hidden);
const uint32_t* sorted_sum_first(const void* workspace);     // rows + 1 positions, valid behind launch_sorted_sum
bool sorted_sum_fits(uint64_t n, uint64_t rows, uint64_t hidden, uint32_t out_dtype);
// after: an earlier kernel of the same call is in front (see launch_after)
// vec: elements per access that the matrices allow, 8, 2 or 1
dte_status launch_sorted_sum(const SortedSum& p, int vec, void* workspace, bool after, int device, cudaStream_t st);

#ifdef __CUDACC__
// ---- dependent launches ------------------------------------------------------------------------------
// A kernel launched with launch_after may start while the one before it in the stream still runs (its launch
// costs nothing then); it calls wait_for_earlier before it touches memory, which returns when all earlier
// work is complete and visible.  Used only inside a call, between its own kernels.
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets the kernel behind this one start now, as far as there is room.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... KernelArgs, typename... Args>
inline cudaError_t launch_after(void (*kernel)(KernelArgs...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KernelArgs(args)...);
}

// ---- device: typed access --------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight consecutive elements as they lie in memory (16 or 32 bytes), loaded now, converted later.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_cs(const __nv_bfloat16* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float* f) const {
        f[0] = bf16_lo(a.x); f[1] = bf16_hi(a.x); f[2] = bf16_lo(a.y); f[3] = bf16_hi(a.y);
        f[4] = bf16_lo(a.z); f[5] = bf16_hi(a.z); f[6] = bf16_lo(a.w); f[7] = bf16_hi(a.w);
    }
    __device__ __forceinline__ void set(const float* f) {
        a = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = a; }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void load_cs(const float* p) {
        a = __ldcs(reinterpret_cast<const float4*>(p));
        b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float* f) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float* f) {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void store(float* p) const {
        reinterpret_cast<float4*>(p)[0] = a;
        reinterpret_cast<float4*>(p)[1] = b;
    }
};

// V consecutive elements: V == 8 through Raw8, V == 2 a pair on a boundary of its size, V == 1 one element of any alignment.
template <typename T, int V>
struct Vec;
template <typename T>
struct Vec<T, 8> : Raw8<T> {};
template <>
struct Vec<__nv_bfloat16, 2> {
    uint32_t a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint32_t*>(p); }
    __device__ __forceinline__ void load_cs(const __nv_bfloat16* p) { a = __ldcs(reinterpret_cast<const uint32_t*>(p)); }
    __device__ __forceinline__ void zero() { a = 0; }
    __device__ __forceinline__ void get(float* f) const { f[0] = bf16_lo(a); f[1] = bf16_hi(a); }
    __device__ __forceinline__ void set(const float* f) { a = pack_bf16(f[0], f[1]); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint32_t*>(p) = a; }
};
template <>
struct Vec<float, 2> {
    float2 a;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float2*>(p); }
    __device__ __forceinline__ void load_cs(const float* p) { a = __ldcs(reinterpret_cast<const float2*>(p)); }
    __device__ __forceinline__ void zero() { a = make_float2(0.f, 0.f); }
    __device__ __forceinline__ void get(float* f) const { f[0] = a.x; f[1] = a.y; }
    __device__ __forceinline__ void set(const float* f) { a = make_float2(f[0], f[1]); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float2*>(p) = a; }
};
template <typename T>
struct Vec<T, 1> {
    T a;
    __device__ __forceinline__ void load(const T* p) { a = *p; }
    __device__ __forceinline__ void load_cs(const T* p) { a = *p; }
    __device__ __forceinline__ void zero() { a = from_f<T>(0.f); }
    __device__ __forceinline__ void get(float* f) const { f[0] = to_f<T>(a); }
    __device__ __forceinline__ void set(const float* f) { a = from_f<T>(f[0]); }
    __device__ __forceinline__ void store(T* p) const { *p = a; }
};

__device__ __forceinline__ int64_t load_id(const void* ids, uint32_t dtype, uint64_t i) {
    return dtype == DTE_I64 ? (int64_t) static_cast<const long long*>(ids)[i] : (int64_t) static_cast<const int*>(ids)[i];
}

// Two floats in one 64-bit register pair: the packed instructions do two operations per issue slot.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f2_get(F2 a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ uint32_t pack_bf16(F2 a) {
    float lo, hi;
    f2_get(a, lo, hi);
    return pack_bf16(lo, hi);
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
#endif  // __CUDACC__

}  // namespace dte
