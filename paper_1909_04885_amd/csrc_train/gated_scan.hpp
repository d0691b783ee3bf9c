// A gated linear recurrence over the rows of sequences, its gradients, and its form for one row of every sequence.
//
//   a_t = 1 / (1 + exp(-f_t)),  h_t = a_t h_{t-1} + (1 - a_t) u_t,  y_t = h_t, from the sequence's first state or from 0
//   G_t = dy_t + a_{t+1} G_{t+1}, the last row's with the gradient of the last state:
//   du_t = (1 - a_t) G_t,  df_t = G_t (h_{t-1} - u_t) a_t (1 - a_t),  dh0 = a_first G_first
//
// Of a gate, s = min(a, 1 - a) = e / (1 + e) with e = exp(-|f|) is what is held, with the sign of f: both a and 1 - a come from it without
// losing what is small, h_t = (1 - s) x + s z with x the one of h_{t-1} and u_t that keeps more.  Gates beyond +-87 are closed: s = 0, and what they
// keep out counts nowhere, whatever it holds.
//
// States are 32-bit floats.  The forward pass leaves the state that enters every SCAN_KEPT-th row; the gradient works out those between again.
#pragma once
#include "elements.hpp"
#include "packed.hpp"

namespace chicle_train {

constexpr int SCAN_KEPT = 32;

// s with the sign of f.
__device__ __forceinline__ float gate_of(float f)
{
    constexpr float LOG2E = 1.44269502162933349609375f, LOG2E_REST = 1.92596299e-8f, LN2 = 0.693147182f;
    const float x = fabsf(f), p = -x * LOG2E;
    const float rest = fmaf(-x, LOG2E_REST, fmaf(-x, LOG2E, -p));         // what rounding took from the power of two
    float e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, rest * LN2, e);
    const float s = e * __builtin_amdgcn_rcpf(1.f + e);
    return copysignf(x > 87.f ? 0.f : s, f);
}

// (1 - s) x, and s x; nothing of x where its share is none.
__device__ __forceinline__ float gate_more(float s, float x) { return s == 0.f ? x : fmaf(-s, x, x); }
__device__ __forceinline__ float gate_less(float s, float x) { return s == 0.f ? 0.f : s * x; }

__device__ __forceinline__ float gate_step(float g, float h, float u)
{
    const bool keep = !signbit(g);
    const float s = fabsf(g), x = keep ? h : u, z = keep ? u : h;
    return s == 0.f ? x : fmaf(s, z, fmaf(-s, x, x));
}
__device__ __forceinline__ float gate_through(float g, float x) { return signbit(g) ? gate_less(fabsf(g), x) : gate_more(fabsf(g), x); }     // a x
__device__ __forceinline__ float gate_into(float g, float x) { return signbit(g) ? gate_more(fabsf(g), x) : gate_less(fabsf(g), x); }        // (1 - a) x
__device__ __forceinline__ float gate_slope(float g, float x)             // a (1 - a) x
{
    const float s = fabsf(g);
    return s == 0.f ? 0.f : fmaf(-s, s, s) * x;
}

// Rows of T, or packed ones.
template <typename T, bool PACKED> struct ScanInput;
template <typename T> struct ScanInput<T, false> {
    const T *p;
    int64_t ld;
    __device__ __forceinline__ float at(int64_t row, int64_t c) const { return (float)p[row * ld + c]; }
};
template <typename T> struct ScanInput<T, true> {
    const int8_t *q;
    const uint8_t *scales;
    int64_t ld;
    __device__ __forceinline__ float at(int64_t row, int64_t c) const
    {
        return (float)q[row * ld + c] * pack_step(scales[row * (ld / PACK_GROUP) + c / PACK_GROUP]);
    }
};

// Where sequences begin: sequence j has the rows from at(j) to at(j + 1).
struct ScanOrder {
    const void *offsets;                     // null: one sequence of all rows
    int wide;
    int64_t count, n;
    __device__ __forceinline__ int64_t at(int64_t j) const { return offsets ? index_at(offsets, wide, j) : j == 0 ? 0 : n; }
};

template <typename T, bool PACKED> struct Scan {
    ScanInput<T, PACKED> u;
    ScanOrder order;
    const T *f, *dy;
    const float *h0, *dlast;                 // or null
    float *states;                           // written by the forward pass (or null), read by the gradient
    float *last, *dh0;                       // or null
    T *y, *df, *du;
    int64_t ldf, lddy, ldy, lddf, lddu, d;
    int *flags;
};

// The rows of sequence j; none, and a report, where they are no rows of the call.
__device__ __forceinline__ void scan_rows(const ScanOrder &o, int64_t j, int *flags, int64_t &lo, int64_t &hi)
{
    lo = o.at(j);
    hi = o.at(j + 1);
    if (lo < 0 || hi < lo || hi > o.n) {
        if (flags) atomicOr(flags, FLAG_OFFSETS);
        lo = hi = 0;
    }
}

// One thread to a column, which goes through the rows of a sequence.
template <typename T, bool PACKED>
__global__ __launch_bounds__(64) void scan_forward(const Scan<T, PACKED> a)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x, d = a.d, n = a.order.n;
    if (c >= d) return;
    auto none = [&](int64_t from, int64_t to) {
        for (int64_t t = from < 0 ? 0 : from; t < to && t < n; ++t) {
            a.y[t * a.ldy + c] = (T)0.f;
            if (a.states && t % SCAN_KEPT == 0) a.states[t / SCAN_KEPT * d + c] = 0.f;
        }
    };
    if (blockIdx.y == 0) {
        none(0, a.order.at(0));
        none(a.order.at(a.order.count), n);
    }
    for (int64_t j = blockIdx.y; j < a.order.count; j += gridDim.y) {
        int64_t lo, hi;
        scan_rows(a.order, j, a.flags, lo, hi);
        float h = a.h0 ? a.h0[j * d + c] : 0.f;
        for (int64_t t = lo; t < hi; ++t) {
            if (a.states && t % SCAN_KEPT == 0) a.states[t / SCAN_KEPT * d + c] = h;
            h = gate_step(gate_of((float)a.f[t * a.ldf + c]), h, a.u.at(t, c));
            a.y[t * a.ldy + c] = (T)h;
        }
        if (a.last) a.last[j * d + c] = h;
    }
}

template <typename T, bool PACKED>
__global__ __launch_bounds__(64) void scan_backward(const Scan<T, PACKED> a)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x, d = a.d, n = a.order.n;
    if (c >= d) return;
    auto none = [&](int64_t from, int64_t to) {
        for (int64_t t = from < 0 ? 0 : from; t < to && t < n; ++t) a.df[t * a.lddf + c] = a.du[t * a.lddu + c] = (T)0.f;
    };
    if (blockIdx.y == 0) {
        none(0, a.order.at(0));
        none(a.order.at(a.order.count), n);
    }
    for (int64_t j = blockIdx.y; j < a.order.count; j += gridDim.y) {
        int64_t lo, hi;
        scan_rows(a.order, j, a.flags, lo, hi);
        float g = a.dlast ? a.dlast[j * d + c] : 0.f;
        for (int64_t end = hi; end > lo;) {
            const int64_t block = (end - 1) / SCAN_KEPT * SCAN_KEPT, begin = block > lo ? block : lo;
            float h[SCAN_KEPT];                          // the state that enters row block + r
            float x = block >= lo ? a.states[block / SCAN_KEPT * d + c] : a.h0 ? a.h0[j * d + c] : 0.f;
#pragma unroll
            for (int r = 0; r < SCAN_KEPT; ++r) {
                const int64_t t = block + r;
                h[r] = x;
                if (t >= begin && t < end) x = gate_step(gate_of((float)a.f[t * a.ldf + c]), x, a.u.at(t, c));
            }
#pragma unroll
            for (int r = SCAN_KEPT - 1; r >= 0; --r) {
                const int64_t t = block + r;
                if (t < begin || t >= end) continue;
                const float gate = gate_of((float)a.f[t * a.ldf + c]);
                g += (float)a.dy[t * a.lddy + c];
                a.df[t * a.lddf + c] = (T)gate_slope(gate, g * (h[r] - a.u.at(t, c)));
                a.du[t * a.lddu + c] = (T)gate_into(gate, g);
                g = gate_through(gate, g);
            }
            end = begin;
        }
        if (a.dh0) a.dh0[j * d + c] = g;
    }
}

// state = a state + (1 - a) u, y = state, one row of every sequence.  A thread has one vector of a row.
constexpr int STEP_THREADS = 256;

template <typename T>
__global__ __launch_bounds__(STEP_THREADS) void scan_step(const T *__restrict__ f, int64_t ldf, const T *__restrict__ u, int64_t ldu, float *__restrict__ state,
                                                          int64_t lds, T *__restrict__ y, int64_t ldy, int64_t n, int64_t d, int lanes)
{
    constexpr int V = Elem<T>::VEC;
    const int64_t row = (int64_t)blockIdx.x * (STEP_THREADS / lanes) + threadIdx.x / lanes;
    if (row >= n) return;
    for (int64_t c = (int64_t)(threadIdx.x % lanes) * V; c < d; c += (int64_t)lanes * V) {
        const u32x4 fs = ask_raw<T, true>(f + row * ldf, c, d), us = ask_raw<T, true>(u + row * ldu, c, d);
        float hs[V], fv[V], uv[V];
#pragma unroll
        for (int k = 0; k < V; k += 4) load_vec(state + row * lds, c + k, d, hs + k);
        unpack<T>(settle<T>(fs, c, d), fv);
        unpack<T>(settle<T>(us, c, d), uv);
#pragma unroll
        for (int i = 0; i < V; ++i) hs[i] = gate_step(gate_of(fv[i]), hs[i], uv[i]);
#pragma unroll
        for (int k = 0; k < V; k += 4)
            if (c + k < d) store_vec(state + row * lds, c + k, d, hs + k);
        store_vec<T, true>(y + row * ldy, c, d, hs);
    }
}

}  // namespace chicle_train
