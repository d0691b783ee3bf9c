// Rows kept in 8 bits: whole numbers from -127 to 127 with one scale for 32 neighbouring columns, a power of two.
//
//   m = max |x| of a group's columns;  e = the least integer >= -126 with m <= 127 2^e;  q = rint(x 2^-e), the byte of the scale e + 127
//
// A value is off by at most half a step 2^e, a 127th of m (or 2^-127).  Where the type's largest values would round to a power of two
// that it does not have, q stops at 63, off by less than a whole step.  A group that holds an infinity or NaN has the byte 255 and zeros:
// it unpacks to NaN.  The byte 0 stands for zeros.  Powers of two because they cost no rounding of their own, neither here nor in the
// product that takes a value out again: what 8 bits hold is a number of every type.  Rows lie `ld` bytes apart, a multiple of 32 that has room for
// whole groups, zeros behind the last column; their scales ld / 32 apart.
//
// The bound is the memory.  A lane packs sixteen bytes of a row, a group's maximum goes over its four or eight lanes by DPP.  65,536 x 4096 in bfloat16:
// packed in 130 us (6.2 TB/s), unpacked in 116 (7.0); 9001 x 1537 in float32, 1540 apart: 17.8 (3.9), and 8.5 into bfloat16; rows begin inside of lines there.
#pragma once
#include "elements.hpp"

namespace chicle_train {

constexpr int PACK_GROUP = 32;
constexpr int PACK_THREADS = 256;

struct Packed {
    int8_t *q;
    uint8_t *scales;
    int64_t ld;
};

// Factor of a scale's byte (255: infinity, which makes NaN of the group's zeros), and one over it (of 1 to 249).
__device__ __forceinline__ float pack_step(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float pack_inverse(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// The byte for a largest magnitude, given as its bits: as whole numbers NaN stands above infinity, and that above all others.
__device__ __forceinline__ unsigned pack_byte(unsigned top)
{
    const int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7e0000u);        // (127 = 1.984375 * 2^6)
    return top >= 0x7f800000u ? 255u : e > 1 ? (unsigned)e : 1u;
}

// The largest q: where values of T up to its largest would round to a power of two that T does not have, one less.
template <typename T> __device__ __forceinline__ float pack_most(unsigned byte, unsigned top)
{
    if constexpr (__is_same(T, f16)) return byte == 137 && top <= 0x477fe000u ? 63.f : 127.f;              // (65504)
    else return byte == 249 ? 63.f : 127.f;
}

// The maximum over the lanes of a group, 4 or 8 neighbouring ones, in all of them.
template <int LANES> __device__ __forceinline__ unsigned group_max(unsigned x)
{
    auto with = [](unsigned a, int b) { return a > (unsigned)b ? a : (unsigned)b; };
    x = with(x, __builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));              // lane ^ 1
    x = with(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));              // lane ^ 2
    if constexpr (LANES == 8) x = with(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));   // 7 - lane of eight: the other four
    return x;
}

// Packs a lane's values of columns c on (zeros behind the row's end); the lanes of a group take part together, c below the whole groups' end.
template <typename T>
__device__ __forceinline__ void pack_vec(const float *v, int8_t *q, uint8_t *scales, int64_t c)
{
    constexpr int V = Elem<T>::VEC;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const unsigned a = __float_as_uint(v[i]) & 0x7fffffffu;
        top = a > top ? a : top;
    }
    top = group_max<PACK_GROUP / V>(top);
    const unsigned byte = pack_byte(top);
    const float inverse = byte == 255 ? 0.f : pack_inverse(byte), most = pack_most<T>(byte, top);
    unsigned w[V / 4];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        // (an infinity or NaN times 0 is no number, of which the maximum below makes -127; the group becomes zeros)
        const float r = fminf(fmaxf(rintf(v[i] * inverse), -most), most);
        const unsigned b = byte == 255 ? 0u : (unsigned)(int)r & 0xffu;
        if (i % 4 == 0) w[i / 4] = b;
        else w[i / 4] |= b << (i % 4 * 8);
    }
    if constexpr (V == 8) *(uint2 *)(q + c) = make_uint2(w[0], w[1]);
    else *(unsigned *)(q + c) = w[0];
    if (c % PACK_GROUP == 0) scales[c / PACK_GROUP] = (uint8_t)byte;
}

// A vector of a packed row as it was asked for, and its values.
template <typename T> struct RawPacked {
    unsigned w[Elem<T>::VEC / 4], byte;
};

template <typename T, bool ONCE = false>
__device__ __forceinline__ RawPacked<T> ask_packed(const int8_t *q, const uint8_t *scales, int64_t c)
{
    RawPacked<T> x;
    if constexpr (Elem<T>::VEC == 8) {
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 v = ONCE ? __builtin_nontemporal_load((const u32x2 *)(q + c)) : *(const u32x2 *)(q + c);
        x.w[0] = v[0];
        x.w[1] = v[1];
    } else {
        x.w[0] = ONCE ? __builtin_nontemporal_load((const unsigned *)(q + c)) : *(const unsigned *)(q + c);
    }
    x.byte = scales[c / PACK_GROUP];
    return x;
}

template <typename T>
__device__ __forceinline__ void unpack8(const RawPacked<T> &x, float *out)
{
    const float step = pack_step(x.byte);
#pragma unroll
    for (int i = 0; i < Elem<T>::VEC; ++i) out[i] = (float)(int8_t)(x.w[i / 4] >> (i % 4 * 8)) * step;
}

// Vectors of all rows one after the other, PACK_EACH to a thread, which are asked for together.
constexpr int PACK_EACH = 4;

// Row and first column of the it-th vector of this thread; `per_row` vectors to a row.
template <int V> struct PackPlace {
    int64_t row, c;
    __device__ __forceinline__ PackPlace(int64_t first_row, int first_vec, int per_row, int it)
    {
        const unsigned at = (unsigned)first_vec + it * PACK_THREADS + threadIdx.x;
        const unsigned over = at / (unsigned)per_row;
        row = first_row + over;
        c = (int64_t)(at - over * (unsigned)per_row) * V;
    }
};

template <typename T>
__global__ __launch_bounds__(PACK_THREADS) void pack_rows(const T *__restrict__ x, int64_t ldx, int64_t n, int64_t d, int per_row, Packed p)
{
    constexpr int V = Elem<T>::VEC;
    const int64_t first = (int64_t)blockIdx.x * (PACK_THREADS * PACK_EACH), row0 = first / per_row;
    const int vec0 = (int)(first - row0 * per_row);
    u32x4 raw[PACK_EACH];
#pragma unroll
    for (int it = 0; it < PACK_EACH; ++it) {
        const PackPlace<V> at(row0, vec0, per_row, it);
        raw[it] = ask_raw<T, true>(x + (at.row < n ? at.row : n - 1) * ldx, at.c, d);
    }
#pragma unroll
    for (int it = 0; it < PACK_EACH; ++it) {
        const PackPlace<V> at(row0, vec0, per_row, it);
        if (at.row >= n) return;                         // (a row has whole groups of lanes)
        float v[V];
        unpack<T>(settle<T>(raw[it], at.c, d), v);
        pack_vec<T>(v, p.q + at.row * p.ld, p.scales + at.row * (p.ld / PACK_GROUP), at.c);
    }
}

template <typename T>
__global__ __launch_bounds__(PACK_THREADS) void unpack_rows(Packed p, int64_t n, int64_t d, int per_row, T *__restrict__ out, int64_t ldo)
{
    constexpr int V = Elem<T>::VEC;
    const int64_t first = (int64_t)blockIdx.x * (PACK_THREADS * PACK_EACH), row0 = first / per_row;
    const int vec0 = (int)(first - row0 * per_row);
    RawPacked<T> raw[PACK_EACH];
#pragma unroll
    for (int it = 0; it < PACK_EACH; ++it) {
        const PackPlace<V> at(row0, vec0, per_row, it);
        const int64_t row = at.row < n ? at.row : n - 1;
        raw[it] = ask_packed<T, true>(p.q + row * p.ld, p.scales + row * (p.ld / PACK_GROUP), at.c);
    }
#pragma unroll
    for (int it = 0; it < PACK_EACH; ++it) {
        const PackPlace<V> at(row0, vec0, per_row, it);
        if (at.row >= n) return;
        float v[V];
        unpack8<T>(raw[it], v);
        if (at.c < d) store_vec<T, true>(out + at.row * ldo, at.c, d, v);
    }
}

}  // namespace chicle_train
