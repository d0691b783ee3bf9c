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

// A row may begin at any multiple of its element's size (a slice of a wider buffer): the accesses assume no more.  Sixteen bytes
// stay what they are until they are used: taking them apart where they are asked for would wait for them there.
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_at_2 __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
__device__ __forceinline__ void unpack(u32x4 x, float *out)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = __uint_as_float(x[i]);
    } else if constexpr (__is_same(T, bf16)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { out[2 * i] = __uint_as_float(x[i] << 16); out[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
    } else {
        T v[8];
        __builtin_memcpy(v, &x, 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (float)v[i];
    }
}

template <typename T>
__device__ __forceinline__ u32x4 pack(const float *in)
{
    T v[Elem<T>::VEC];
#pragma unroll
    for (int i = 0; i < Elem<T>::VEC; ++i) v[i] = (T)in[i];
    u32x4 x;
    __builtin_memcpy(&x, v, 16);
    return x;
}

// A vector of a row of d values, zeros past its end, in two steps.  `ask_raw` asks for sixteen bytes that lie in the row, the last of the row
// where the vector ends behind it; `settle` moves those to their place, when they are used.  So a load never waits for
// itself, whatever d is.  (Rows shorter than a vector are put together value by value.)  ONCE: data that is read once, or written and not
// read soon, is not kept in the caches, which is faster for what does not fit there (reads of 2 GiB: 7.1 instead of 6.4 TB/s).
template <typename T, bool ONCE = false>
__device__ __forceinline__ u32x4 ask_raw(const T *row, int64_t c, int64_t d)
{
    constexpr int V = Elem<T>::VEC;
    if (d >= V) {
        const T *p = row + (c < d - V ? c : d - V);
        if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4_at_2 *)p);
        else return *(const u32x4_at_2 *)p;
    }
    u32x4 x = {0u, 0u, 0u, 0u};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (c + i < d) x[i] = ((const unsigned *)row)[c + i];
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (c + i < d) x[i / 2] |= (unsigned)((const uint16_t *)row)[c + i] << (i % 2 * 16);
    }
    return x;
}

template <typename T>
__device__ __forceinline__ u32x4 settle(u32x4 x, int64_t c, int64_t d)
{
    constexpr int V = Elem<T>::VEC;
    if (__builtin_expect(c + V > d && d >= V, 0)) {
        const int64_t past = c + V - d;                  // values that are not the vector's, at the front
        const int bits = past < V ? (int)past * 8 * (int)sizeof(T) : 128;
        const unsigned long long lo = (unsigned long long)x[1] << 32 | x[0], hi = (unsigned long long)x[3] << 32 | x[2];
        const unsigned long long a = bits >= 128 ? 0ull : bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits), b = bits >= 64 ? 0ull : hi >> bits;
        x = u32x4{(unsigned)a, (unsigned)(a >> 32), (unsigned)b, (unsigned)(b >> 32)};
    }
    return x;
}

template <typename T, bool ONCE = false>
__device__ __forceinline__ u32x4 load_raw(const T *row, int64_t c, int64_t d)
{
    return settle<T>(ask_raw<T, ONCE>(row, c, d), c, d);
}

template <typename T, bool ONCE = false>
__device__ __forceinline__ void load_vec(const T *row, int64_t c, int64_t d, float *out)
{
    unpack<T>(load_raw<T, ONCE>(row, c, d), out);
}

template <typename T, bool ONCE = false>
__device__ __forceinline__ void store_vec(T *row, int64_t c, int64_t d, const float *in)
{
    constexpr int V = Elem<T>::VEC;
    const u32x4 x = pack<T>(in);
    if (__builtin_expect(c + V <= d, 1)) {
        if constexpr (ONCE) __builtin_nontemporal_store((u32x4_at_2)x, (u32x4_at_2 *)(row + c));
        else *(u32x4_at_2 *)(row + c) = x;
    } else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
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

__global__ void take_flags(int *flags, int *out) { *out = atomicExch(flags, 0); }

}  // namespace chicle_train
