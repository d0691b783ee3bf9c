// The norm of many tensors together, and the tensors times min(1, max_norm / (norm + 1e-6)).
//
// Two launches: every workgroup leaves the sum of squares of its piece, and every workgroup of the second launch adds all of
// these up by itself, in one order, before it scales its piece.  Sums are held in double: the squares of any finite 32-bit floats
// add up without overflow.  The bound is the memory: one read and one write, and a second read that comes from the caches as
// far as the tensors fit there.
#pragma once
#include "elements.hpp"

namespace chicle_train {

constexpr int CLIP_TENSORS = 112;            // tensors of one launch: their table is part of the kernel's arguments
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_MOST_PARTS = 2048;        // workgroups of all launches of a call

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
        while (p >= t.first_piece[k + 1]) ++k;
        const int64_t a = (int64_t)(p - t.first_piece[k]) * piece;
        f(k, a, min(t.count[k], a + piece));
    }
}

template <typename T>
__global__ __launch_bounds__(CLIP_THREADS) void squares(ClipTable t, int64_t piece, double *__restrict__ part)
{
    constexpr int V = Elem<T>::VEC;
    double sum = 0.0;
    clip_pieces(t, piece, [&](int k, int64_t a, int64_t end) {
        const T *p = (const T *)t.in[k];
        for (int64_t c = a + (int64_t)threadIdx.x * V; c < end; c += CLIP_THREADS * V) {
            float u[V];
            load_vec(p, c, end, u);
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < V; ++i) s += (double)u[i] * (double)u[i];
            sum += s;
        }
    });
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

template <typename T>
__global__ __launch_bounds__(CLIP_THREADS) void clip_scale(ClipTable t, int64_t piece, const double *__restrict__ part, int parts,
                                                           float max_norm, float *__restrict__ norm_out)
{
    constexpr int V = Elem<T>::VEC;
    const float norm = norm_of_parts(part, parts);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    const float ratio = max_norm / (norm + 1e-6f);
    const float factor = ratio > 1.f ? 1.f : ratio;      // (a norm that is no number makes the factor none)
    clip_pieces(t, piece, [&](int k, int64_t a, int64_t end) {
        const T *p = (const T *)t.in[k];
        T *q = (T *)t.out[k];
        if (factor == 1.f && p == q) return;             // nothing changes
        for (int64_t c = a + (int64_t)threadIdx.x * V; c < end; c += CLIP_THREADS * V) {
            float u[V];
            load_vec(p, c, end, u);
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] *= factor;
            store_vec(q, c, end, u);
        }
    });
}

}  // namespace chicle_train
