// Loads and stores of float32, bf16 and fp16 elements as float32 values, for the kernels whose tensors may begin at any
// element: eight in a row through 16-byte accesses that need no more alignment than an element's.
#pragma once
#include "dp_common.h"

namespace dpk {

// 16 bytes at the alignment of an element (one global_load_dwordx4 / global_store_dwordx4: gfx950 takes any address)
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));

// Addresses out of a descriptor are generic to the compiler, and generic accesses count as LDS accesses too: the tensors are in
// global memory.
template <class T> using Global = __attribute__((address_space(1))) T;
template <class T> __device__ __forceinline__ const Global<T>* global_in(const void* p) { return (const Global<T>*)(uintptr_t)p; }
template <class T> __device__ __forceinline__ Global<T>* global_out(void* p) { return (Global<T>*)(uintptr_t)p; }

// DT: 0 = float32, 1 = bf16, 2 = fp16
template <int DT> __device__ __forceinline__ float load_one(const void* p, int64_t k) {
    if constexpr (DT == 0) return global_in<float>(p)[k];
    else return In16<DT == 2>::lo(global_in<uint16_t>(p)[k]);
}
template <int DT> __device__ __forceinline__ void store_one(void* p, int64_t k, float v) {
    if constexpr (DT == 0) global_out<float>(p)[k] = v;
    else global_out<uint16_t>(p)[k] = (uint16_t)In16<DT == 2>::pack(v, 0.f);
}

// eight elements, as they are in memory
template <int DT> struct Raw8;
template <> struct Raw8<0> { u32x4_any4 a, b; };
template <> struct Raw8<1> { u32x4_any2 a; };
template <> struct Raw8<2> { u32x4_any2 a; };
template <int DT> __device__ __forceinline__ Raw8<DT> load_raw8(const void* p, int64_t k) {
    Raw8<DT> r;
    if constexpr (DT == 0) {
        const Global<u32x4_any4>* q = global_in<u32x4_any4>(static_cast<const float*>(p) + k);
        r.a = q[0];
        r.b = q[1];
    } else {
        r.a = *global_in<u32x4_any2>(static_cast<const uint16_t*>(p) + k);
    }
    return r;
}
template <int DT> __device__ __forceinline__ void widen8(const Raw8<DT>& r, float (&v)[8]) {
    if constexpr (DT == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[j] = __uint_as_float(r.a[j]); v[4 + j] = __uint_as_float(r.b[j]); }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[2 * j] = In16<DT == 2>::lo(r.a[j]); v[2 * j + 1] = In16<DT == 2>::hi(r.a[j]); }
    }
}
template <int DT> __device__ __forceinline__ void load8(const void* p, int64_t k, float (&v)[8]) { widen8<DT>(load_raw8<DT>(p, k), v); }
// rounded to nearest, ties to even
template <int DT> __device__ __forceinline__ void store8(void* p, int64_t k, const float (&v)[8]) {
    if constexpr (DT == 0) {
        Global<u32x4_any4>* q = global_out<u32x4_any4>(static_cast<float*>(p) + k);
        u32x4_any4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) { a[j] = __float_as_uint(v[j]); b[j] = __float_as_uint(v[4 + j]); }
        q[0] = a;
        q[1] = b;
    } else {
        u32x4_any2 a;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = In16<DT == 2>::pack(v[2 * j], v[2 * j + 1]);
        *global_out<u32x4_any2>(static_cast<uint16_t*>(p) + k) = a;
    }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}
// Sum over the 256 threads of a workgroup in a fixed order, valid in every thread.  `red` is 4 doubles of LDS that the
// caller does not touch again before a barrier.
__device__ __forceinline__ double block_sum_256_f64(double v, double* red) {
    v = wave_sum_f64(v);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

}  // namespace dpk
