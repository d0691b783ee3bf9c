// The norm of many tensors together, and the tensors times min(1, max_norm / (norm + 1e-6)).
//
// Every workgroup of the first launch leaves the sum of squares of its pieces.  Where there are few pieces, every workgroup of the
// second launch adds all of these up by itself, in one order, before it scales its piece; where there are many, a launch between
// the two does it once.  Sums are held in double: the squares of any finite 32-bit floats add up without overflow.
// The bound is the memory: one read and one write, and a second read that comes from the caches as far as the tensors fit there.
// 1.28e9 values in bfloat16: 1230 us (squares 420 us, 6.1 TB/s; scaling 825, 6.2 TB/s); 5 million in 32 bits: 8 + 11 us and as much again
// for gathering 49 tensors' addresses on the host.
#pragma once
#include "elements.hpp"

namespace chicle_train {

constexpr int CLIP_TENSORS = 112;            // tensors of one launch: their table is part of the kernel's arguments
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_MOST_PARTS = 2048;        // workgroups of all launches of a call that add up squares

struct ClipTable {
    const void *in[CLIP_TENSORS];
    void *out[CLIP_TENSORS];
    int64_t count[CLIP_TENSORS];
    int32_t first_piece[CLIP_TENSORS + 1];   // pieces of a launch are numbered through its tensors
    int32_t tensors;
    int32_t first_part;                      // where the launch's workgroups leave their sums
};

__device__ __forceinline__ double block_sum(double x)
{
    __shared__ double s[CLIP_THREADS / 64];
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
    for (int i = 1; i < CLIP_THREADS / 64; ++i) x += s[i];
    return x;
}

// Calls f(tensor, first value, end) for this workgroup's pieces of `piece` values: blockIdx.x, gridDim.x further on, and so on.
template <typename F>
__device__ __forceinline__ void clip_pieces(const ClipTable &t, int64_t piece, F f)
{
    int k = 0;
    for (int p = blockIdx.x; p < t.first_piece[t.tensors]; p += gridDim.x) {
        int hi = t.tensors - 1;                          // the last tensor that begins at this piece or before
        while (k < hi) {
            const int mid = (k + hi + 1) / 2;
            if (t.first_piece[mid] <= p) k = mid;
            else hi = mid - 1;
        }
        const int64_t a = (int64_t)(p - t.first_piece[k]) * piece;
        f(k, a, min(t.count[k], a + piece));
    }
}

// CLIP_AHEAD vectors of a thread are on their way together.
constexpr int CLIP_AHEAD = 4;

template <typename T>
__device__ __forceinline__ void clip_ask(const T *p, int64_t c, int64_t end, u32x4 (&u)[CLIP_AHEAD])
{
    constexpr int STEP = CLIP_THREADS * Elem<T>::VEC;
#pragma unroll
    for (int q = 0; q < CLIP_AHEAD; ++q) u[q] = ask_raw<T, true>(p, c + q * STEP, end);
}

template <typename T>
__global__ __launch_bounds__(CLIP_THREADS) void squares(ClipTable t, int64_t piece, double *__restrict__ part)
{
    constexpr int V = Elem<T>::VEC, ALL = CLIP_THREADS * V * CLIP_AHEAD;
    double sums[CLIP_AHEAD] = {};                        // (sums of their own do not wait for each other)
    auto add = [&](int64_t c, int64_t end, const u32x4 (&u)[CLIP_AHEAD]) {
#pragma unroll
        for (int q = 0; q < CLIP_AHEAD; ++q) {
            float w[V];
            unpack<T>(settle<T>(u[q], c + q * CLIP_THREADS * V, end), w);
#pragma unroll
            for (int i = 0; i < V; ++i) sums[q] += (double)w[i] * (double)w[i];
        }
    };
    clip_pieces(t, piece, [&](int k, int64_t a, int64_t end) {
        const T *p = (const T *)t.in[k];
        u32x4 u[CLIP_AHEAD];
        for (int64_t c = a + (int64_t)threadIdx.x * V; c < end; c += ALL) { clip_ask(p, c, end, u); add(c, end, u); }
    });
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < CLIP_AHEAD; ++q) sum += sums[q];
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[t.first_part + blockIdx.x] = sum;
}

__device__ __forceinline__ float norm_of_parts(const double *part, int parts)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += CLIP_THREADS) s += part[i];
    return (float)sqrt(block_sum(s));
}

__global__ __launch_bounds__(CLIP_THREADS) void norm_only(const double *__restrict__ part, int parts, float *__restrict__ norm_out)
{
    const float norm = norm_of_parts(part, parts);
    if (threadIdx.x == 0) *norm_out = norm;
}

// parts 0: the norm is there already
template <typename T>
__global__ __launch_bounds__(CLIP_THREADS) void clip_scale(ClipTable t, int64_t piece, const double *__restrict__ part, int parts,
                                                           float max_norm, float *__restrict__ norm_out)
{
    constexpr int V = Elem<T>::VEC, ALL = CLIP_THREADS * V * CLIP_AHEAD;
    float norm;
    if (parts) {
        norm = norm_of_parts(part, parts);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    } else norm = *norm_out;
    const float ratio = max_norm / (norm + 1e-6f);
    const float factor = ratio > 1.f ? 1.f : ratio;      // (a norm that is no number makes the factor none)
    clip_pieces(t, piece, [&](int k, int64_t a, int64_t end) {
        const T *p = (const T *)t.in[k];
        T *q = (T *)t.out[k];
        if (factor == 1.f && p == q) return;             // nothing changes
        auto scale = [&](int64_t c, const u32x4 (&u)[CLIP_AHEAD]) {
#pragma unroll
            for (int h = 0; h < CLIP_AHEAD; ++h) {
                float w[V];
                unpack<T>(settle<T>(u[h], c + h * CLIP_THREADS * V, end), w);
#pragma unroll
                for (int i = 0; i < V; ++i) w[i] *= factor;
                store_vec<T, true>(q, c + h * CLIP_THREADS * V, end, w);
            }
        };
        u32x4 u[CLIP_AHEAD];
        for (int64_t c = a + (int64_t)threadIdx.x * V; c < end; c += ALL) { clip_ask(p, c, end, u); scale(c, u); }
    });
}

}  // namespace chicle_train
