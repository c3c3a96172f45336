// Shared by the training operators (layer norm, expert router, orthogonalisation): element types, reductions, host checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "trv_dev.cuh"

namespace trv {

constexpr int kSMs = 148;               // B200

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Two binary32 operations in one instruction (sm_100 packed FP32), each rounded to nearest
__device__ __forceinline__ unsigned long long f2_bits(float2 v) { return *reinterpret_cast<unsigned long long*>(&v); }
__device__ __forceinline__ float2 f2_of(unsigned long long u) { return *reinterpret_cast<float2*>(&u); }
__device__ __forceinline__ float2 f2_splat(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 f2_add(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_of(r);
}
__device__ __forceinline__ float2 f2_mul(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_of(r);
}
__device__ __forceinline__ float2 f2_fma(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)), "l"(f2_bits(c)));
    return f2_of(r);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// ---- host side
// allow_big_smem, once per device: `done` has a bit for each and belongs to one kernel and one size
template <typename K>
inline bool allow_big_smem_once(K kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_acquire) & bit)) return true;
    if (!allow_big_smem(kernel, bytes)) return false;
    done.fetch_or(bit, std::memory_order_release);
    return true;
}
inline size_t dtype_bytes(trv_dtype_t t) { return t == TRV_BFLOAT16 || t == TRV_FLOAT16 ? 2 : 4; }
inline bool float_dtype(trv_dtype_t t) { return t == TRV_FLOAT32 || t == TRV_BFLOAT16 || t == TRV_FLOAT16; }
// bytes from the first to behind the last element of a strided matrix
inline size_t matrix_bytes(size_t rows, size_t cols, size_t stride, size_t es) { return rows ? ((rows - 1) * stride + cols) * es : 0; }
// Memory of an operand: `bytes` from p on; a matrix also says which of them are its own, `row` of every `stride` bytes
struct Span {
    const void* p;
    size_t bytes, row, stride;
};
inline Span matrix_span(const void* p, size_t rows, size_t cols, size_t stride, size_t es) {
    return {p, matrix_bytes(rows, cols, stride, es), cols * es, stride * es};
}
inline bool meet(const Span& a, const Span& b) {
    if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    if (x >= y + b.bytes || y >= x + a.bytes) return false;
    // column slices of one buffer: equal strides, and b's columns behind a's and before a's next row
    if (a.stride && a.stride == b.stride) {
        const size_t off = y >= x ? (y - x) % a.stride : (a.stride - (x - y) % a.stride) % a.stride;
        return off < a.row || off + b.row > a.stride;
    }
    return true;
}
// no output may touch an input or another output
template <int NI, int NO>
inline bool disjoint(const Span (&in)[NI], const Span (&out)[NO]) {
    for (int o = 0; o < NO; ++o) {
        for (int i = 0; i < NI; ++i)
            if (meet(out[o], in[i])) return false;
        for (int q = o + 1; q < NO; ++q)
            if (meet(out[o], out[q])) return false;
    }
    return true;
}
inline bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

}  // namespace trv
