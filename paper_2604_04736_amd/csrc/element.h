// Tensors of float32, bfloat16 and float16 in sixteen-byte pieces that lie on any element: what norm.hip and head.hip read and write.
#ifndef HOT_ELEMENT_H
#define HOT_ELEMENT_H

#include <hip/hip_runtime.h>

#include "hot.h"

namespace {

// N elements of T are sixteen bytes.  Loads and stores ask for the alignment of one element only: the hardware takes 16-byte accesses
// on any address, so rows of odd pitch need no kernel of their own.
template <class T>
struct Piece {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(N)));
    typedef V Loose __attribute__((aligned(sizeof(T))));
    typedef float F __attribute__((ext_vector_type(N)));

    // elements at .. at + N - 1 of a row of n; zeros behind its end
    static __device__ __forceinline__ V take(const T *row, long at, long n)
    {
        if (at + N <= n) return *reinterpret_cast<const Loose *>(row + at);
        V v;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = at + j < n ? row[at + j] : (T)0.0f;
        return v;
    }
    static __device__ __forceinline__ F load(const T *row, long at, long n) { return __builtin_convertvector(take(row, at, n), F); }
    static __device__ __forceinline__ void store(T *row, long at, long n, F v)
    {
        const V o = __builtin_convertvector(v, V);
        if (at + N <= n) {
            *reinterpret_cast<Loose *>(row + at) = o;
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (at + j < n) row[at + j] = o[j];
    }
};

// N floats of an array of the type `type` names (uniform over the launch), for small operands whose type is not the kernel's own
template <int N, class F>
__device__ __forceinline__ F load_as(const void *p, int type, long at, long n)
{
    F v;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        v[j] = 0.0f;
        if (at + j < n)
            v[j] = type == HOT_F32 ? static_cast<const float *>(p)[at + j]
                                   : (type == HOT_BF16 ? (float)static_cast<const __bf16 *>(p)[at + j] : (float)static_cast<const _Float16 *>(p)[at + j]);
    }
    return v;
}

__device__ __forceinline__ void store_as(void *p, int type, long at, float v)
{
    if (type == HOT_F32) static_cast<float *>(p)[at] = v;
    else if (type == HOT_BF16) static_cast<__bf16 *>(p)[at] = (__bf16)v;
    else static_cast<_Float16 *>(p)[at] = (_Float16)v;
}

inline bool known_type(int t) { return t == HOT_F32 || t == HOT_BF16 || t == HOT_F16; }
inline int type_bytes(int t) { return t == HOT_F32 ? 4 : 2; }
inline bool on_element(const void *p, int type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }

}  // namespace

#endif  // HOT_ELEMENT_H
