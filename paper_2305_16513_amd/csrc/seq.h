// What the operators of token sequences (norms.hip, short_conv.hip, delta_*.hip) share: elements of three storage types widened to fp32,
// eight at a time, and the functions of their arithmetic.
#pragma once
#include <initializer_list>
#include <type_traits>

#include "sws_internal.h"

namespace sws {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef float v8f __attribute__((ext_vector_type(8)));

typedef v8f v8f_m __attribute__((aligned(16)));       // eight floats in memory

template <class E> struct Vec;                        // eight / four elements of a type
template <> struct Vec<float> { typedef v8f_m v8; typedef v4f v4; };
template <> struct Vec<__bf16> { typedef v8bf v8; typedef v4bf v4; };
template <> struct Vec<_Float16> { typedef v8h v8; typedef v4h v4; };

// Eight elements from p on as fp32.  FULL: all eight are there and p is a multiple of 16 bytes.  Otherwise the first n (any
// number, also none) one by one, and zeros: nothing beyond them is read.
template <bool FULL, class E>
__device__ __forceinline__ void load8(const E *p, int n, float (&f)[8])
{
    if constexpr (FULL) {
        const typename Vec<E>::v8 v = *(const typename Vec<E>::v8 *)p;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = e < n ? (float)p[e] : 0.0f;
    }
}

// The same, widened when they are needed: half the registers of a load in flight (16-bit types)
template <bool FULL, class E>
__device__ __forceinline__ typename Vec<E>::v8 fetch8(const E *p, int n)
{
    if constexpr (FULL) return *(const typename Vec<E>::v8 *)p;
    else {
        typename Vec<E>::v8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : (E)0.0f;
        return v;
    }
}

template <bool FULL, class E>
__device__ __forceinline__ void store8(E *p, int n, const float (&f)[8])
{
    if constexpr (FULL) {
        typename Vec<E>::v8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (E)f[e];
        *(typename Vec<E>::v8 *)p = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (E)f[e];
    }
}

// 1 / (1 + exp(-x)).  fp32 storage: to the last bits; 16-bit storage: v_exp_f32 and v_rcp_f32, whose errors (a few 2^-23, and |x| times
// 2^-24 of the exponent's own rounding) are far below the storage's.
template <class E>
__device__ __forceinline__ float sigmoid(float x)
{
    if constexpr (sizeof(E) == 4) return 1.0f / (1.0f + expf(-x));
    else return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
}

// The sum over 2^k neighbouring lanes (n of them, uniform in the kernel), in all of them: within sixteen by DPP (neighbours, pairs of them, fours and
// eights the other way round), beyond by shuffles.
__device__ __forceinline__ float sum_lanes(float v, int n)
{
#define SWS_ADD(CTRL) v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true))
    if (n >= 2) SWS_ADD(0xb1);
    if (n >= 4) SWS_ADD(0x4e);
    if (n >= 8) SWS_ADD(0x141);
    if (n >= 16) SWS_ADD(0x140);
#undef SWS_ADD
    if (n >= 32) v += __shfl_xor(v, 16);
    if (n >= 64) v += __shfl_xor(v, 32);
    return v;
}
__device__ __forceinline__ float sum16(float v) { return sum_lanes(v, 16); }

// Whether all of some pointers are multiples of 16 bytes (an absent one is)
inline bool sixteen(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if ((uintptr_t)p & 15) return false;
    return true;
}

// n workgroups of so many threads as a grid, `across` in y: a launch has fewer than 2^32 threads in x, so that more go on in z, the last of which may
// reach beyond n.  False: more than 31 bits.
inline bool spread(int64_t n, int threads, dim3 &grid, unsigned across = 1)
{
    const int64_t most = 0xffffffffll / threads, z = (n + most - 1) / most;
    if (n > 0x7fffffff) return false;
    grid = dim3((unsigned)(z > 1 ? (n + z - 1) / z : n), across, (unsigned)(z > 1 ? z : 1));
    return true;
}
// Which of them this one is
__device__ __forceinline__ unsigned group_of() { return blockIdx.z * gridDim.x + blockIdx.x; }

// f with a null pointer of the storage type
template <class F>
hipError_t by_type(int dtype, F &&f)
{
    if (dtype == SWS_DTYPE_BF16) return f((__bf16 *)nullptr);
    if (dtype == SWS_DTYPE_F16) return f((_Float16 *)nullptr);
    return f((float *)nullptr);
}

// out[c] = sum over g of part[g * stride + c] in a fixed order, for `columns` columns; from column `split` on it goes to more[c - split] (nullptr: nowhere)
hipError_t launch_column_sums(const float *part, float *out, float *more, int64_t split, int parts, int64_t stride, int64_t columns, hipStream_t s);

}  // namespace sws
