// Element types of the training operators, sixteen-byte accesses to rows of them, and sums over groups of lanes.
//
// Every operator reads and writes 32-bit floats, bfloat16 or half precision and computes in 32-bit floats; a result of a
// 16-bit type is rounded once, to nearest even, where it is stored.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace chicle_train {

typedef __bf16 bf16;
typedef _Float16 f16;

template <typename T> struct Elem { static constexpr int VEC = 16 / (int)sizeof(T); };   // values of one access

// A row may begin at any multiple of its element's size (a slice of a wider buffer): the accesses assume no more.
template <typename T> struct Vec { T v[Elem<T>::VEC]; };

template <typename T>
__device__ __forceinline__ void load_vec(const T *row, int64_t c, int64_t d, float *out)
{
    constexpr int V = Elem<T>::VEC;
    if (c + V <= d) {
        Vec<T> x;
        __builtin_memcpy(&x, row + c, 16);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = (float)x.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = c + i < d ? (float)row[c + i] : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store_vec(T *row, int64_t c, int64_t d, const float *in)
{
    constexpr int V = Elem<T>::VEC;
    if (c + V <= d) {
        Vec<T> x;
#pragma unroll
        for (int i = 0; i < V; ++i) x.v[i] = (T)in[i];
        __builtin_memcpy(row + c, &x, 16);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i < d) row[c + i] = (T)in[i];
    }
}

// Sum over `lanes` neighbouring lanes (a power of two up to 64), in all of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Index arrays come in 32 or 64 bits.
__device__ __forceinline__ int64_t index_at(const void *p, int wide, int64_t i)
{
    return wide ? ((const int64_t *)p)[i] : (int64_t)((const int32_t *)p)[i];
}

constexpr int FLAG_LABEL_RANGE = 1, FLAG_ID_RANGE = 2;

}  // namespace chicle_train
