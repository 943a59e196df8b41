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
// rounded to nearest, ties to even; PAST: past the caches, for outputs that do not fit them
template <bool PAST, class T> __device__ __forceinline__ void store_raw(const T& v, Global<T>* p) {
    if constexpr (PAST) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <int DT, bool PAST = false> __device__ __forceinline__ void store8(void* p, int64_t k, const float (&v)[8]) {
    if constexpr (DT == 0) {
        Global<u32x4_any4>* q = global_out<u32x4_any4>(static_cast<float*>(p) + k);
        u32x4_any4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) { a[j] = __float_as_uint(v[j]); b[j] = __float_as_uint(v[4 + j]); }
        store_raw<PAST>(a, q);
        store_raw<PAST>(b, q + 1);
    } else {
        u32x4_any2 a;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = In16<DT == 2>::pack(v[2 * j], v[2 * j + 1]);
        store_raw<PAST>(a, global_out<u32x4_any2>(static_cast<uint16_t*>(p) + k));
    }
}

// 1, 2, 4 or 8 elements
template <int DT, int N> __device__ __forceinline__ void load_piece(const void* p, int64_t k, float (&v)[N]) {
    if constexpr (N == 8) {
        load8<DT>(p, k, v);
    } else if constexpr (N == 1) {
        v[0] = load_one<DT>(p, k);
    } else if constexpr (DT == 0) {
        typedef uint32_t piece __attribute__((ext_vector_type(N), aligned(4)));
        const piece r = *global_in<piece>(static_cast<const float*>(p) + k);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = __uint_as_float(r[j]);
    } else if constexpr (N == 2) {
        typedef uint32_t piece __attribute__((aligned(2)));
        const uint32_t r = *global_in<piece>(static_cast<const uint16_t*>(p) + k);
        v[0] = In16<DT == 2>::lo(r);
        v[1] = In16<DT == 2>::hi(r);
    } else {
        typedef uint32_t piece __attribute__((ext_vector_type(N / 2), aligned(2)));
        const piece r = *global_in<piece>(static_cast<const uint16_t*>(p) + k);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) { v[2 * j] = In16<DT == 2>::lo(r[j]); v[2 * j + 1] = In16<DT == 2>::hi(r[j]); }
    }
}
template <int DT, bool PAST = false, int N> __device__ __forceinline__ void store_piece(void* p, int64_t k, const float (&v)[N]) {
    static_assert(!PAST || N >= 4);
    if constexpr (N == 8) {
        store8<DT, PAST>(p, k, v);
    } else if constexpr (N == 1) {
        store_one<DT>(p, k, v[0]);
    } else if constexpr (DT == 0) {
        typedef uint32_t piece __attribute__((ext_vector_type(N), aligned(4)));
        piece r;
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = __float_as_uint(v[j]);
        store_raw<PAST>(r, global_out<piece>(static_cast<float*>(p) + k));
    } else if constexpr (N == 2) {
        typedef uint32_t piece __attribute__((aligned(2)));
        *global_out<piece>(static_cast<uint16_t*>(p) + k) = In16<DT == 2>::pack(v[0], v[1]);
    } else {
        typedef uint32_t piece __attribute__((ext_vector_type(N / 2), aligned(2)));
        piece r;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) r[j] = In16<DT == 2>::pack(v[2 * j], v[2 * j + 1]);
        store_raw<PAST>(r, global_out<piece>(static_cast<uint16_t*>(p) + k));
    }
}
// The first n of eight elements, 0 < n < 8, in pieces of 4, 2 and 1: zeros behind them, and nothing behind them is touched.
template <int DT> __device__ __forceinline__ void load_first(const void* p, int64_t k, int n, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (n & 4) { float f[4]; load_piece<DT>(p, k, f); v[0] = f[0]; v[1] = f[1]; v[2] = f[2]; v[3] = f[3]; }
    if (n & 2) {
        float f[2];
        load_piece<DT>(p, k + (n & 4), f);
        const bool up = n & 4;
        v[4] = up ? f[0] : 0.f; v[5] = up ? f[1] : 0.f;
        v[0] = up ? v[0] : f[0]; v[1] = up ? v[1] : f[1];
    }
    if (n & 1) {
        float f[1];
        load_piece<DT>(p, k + (n & 6), f);
#pragma unroll
        for (int j = 0; j < 8; j += 2)
            if ((n & 6) == j) v[j] = f[0];
    }
}
// (The elements go by value: with an array behind a reference the compiler joins the branches' stores into one of an element by
// index, and gives the array a place in scratch memory or in LDS.  For LDS it reads the workgroup's size from the dispatch packet,
// in host memory: 13 us for a launch.)
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <int DT> __device__ __forceinline__ void store_first(void* p, int64_t k, int n, f32x8 v) {
    if (n & 4) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        store_piece<DT>(p, k, f);
        v = __builtin_shufflevector(v, v, 4, 5, 6, 7, 4, 5, 6, 7);
        k += 4;
    }
    if (n & 2) {
        const float f[2] = {v[0], v[1]};
        store_piece<DT>(p, k, f);
        v = __builtin_shufflevector(v, v, 2, 3, 2, 3, 2, 3, 2, 3);
        k += 2;
    }
    if (n & 1) store_one<DT>(p, k, v[0]);
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
