// Layer norm over rows and its gradients.
//
//   mean = sum_c x_c / d,  rstd = 1 / sqrt(sum_c (x_c - mean)^2 / d + eps),  y_c = (x_c - mean) rstd gamma_c + beta_c
//   with xhat_c = (x_c - mean) rstd and g_c = dy_c gamma_c:
//   dx_c = rstd (g_c - mean(g) - xhat_c mean(g xhat)),  dgamma_c = sum_rows dy_c xhat_c,  dbeta_c = sum_rows dy_c
//
// A row is held in registers by `lanes` neighbouring threads, NV vectors of sixteen bytes each, and read once: the variance
// is that of the centred values, not a difference of sums.  Rows that no workgroup holds (NV = 0) are read again for every sum.
// The bound is the memory: one read and one write (gradients: two reads and one write).  65,536 x 4096 in bfloat16: forward 231 us
// (4.7 TB/s), gradients 293 us (5.5 TB/s; a large copy on the same card runs at 4.9); 9001 x 1537 in 32 bits, gradients 48 us (3.5 TB/s,
// 7 of them the sums over the workgroups).  One row: 4.5 us, a launch.
#pragma once
#include "elements.hpp"

namespace chicle_train {

constexpr int LN_MOST_THREADS = 1024;

// Sums of two values over the `lanes` threads of a row (all threads of the workgroup where lanes > 64); every thread of the
// workgroup takes part in the same calls.
__device__ __forceinline__ float2 row_sum2(float2 s, int lanes)
{
    s.x = lanes_sum(s.x, lanes < 64 ? lanes : 64);
    s.y = lanes_sum(s.y, lanes < 64 ? lanes : 64);
    if (lanes <= 64) return s;
    __shared__ float2 part[LN_MOST_THREADS / 64];
    const int wave = threadIdx.x >> 6, waves = lanes >> 6;
    __syncthreads();                                     // (the sums before these have been read)
    if ((threadIdx.x & 63) == 0) part[wave] = s;
    __syncthreads();
    const int first = wave / waves * waves;              // (waves is a power of two: the row's own)
    s = part[first];
    for (int i = 1; i < waves; ++i) { s.x += part[first + i].x; s.y += part[first + i].y; }
    return s;
}

// blockDim.x is a multiple of lanes; a workgroup takes blockDim.x / lanes rows.
template <typename T, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void layer_norm_rows(const T *__restrict__ x, int64_t ldx, const T *__restrict__ gamma,
                                                      const T *__restrict__ beta, T *__restrict__ y, int64_t ldy,
                                                      float *__restrict__ mean_out, float *__restrict__ rstd_out, int64_t n, int64_t d, int lanes, float eps)
{
    constexpr int V = Elem<T>::VEC;
    const int lane = threadIdx.x % lanes;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
    const bool live = row < n;
    const T *xr = x + (live ? row : n - 1) * ldx;        // (threads without a row go through the sums with the others)
    T *yr = y + (live ? row : n - 1) * ldy;
    const int64_t first = (int64_t)lane * V, step = (int64_t)lanes * V;
    float v[NV ? NV : 1][V];
    float2 s = {0.f, 0.f};
    if constexpr (NV > 0) {
        constexpr int RAW = NV * V <= 16 || THREADS <= 256 ? NV : 1;       // vectors that are asked for together, as registers allow
        u32x4 raw[RAW];
#pragma unroll
        for (int k = 0; k < RAW; ++k) raw[k] = ask_raw<T, true>(xr, first + k * step, d);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (RAW == 1 && k > 0) raw[0] = ask_raw<T, true>(xr, first + k * step, d);
            unpack<T>(settle<T>(raw[RAW == 1 ? 0 : k], first + k * step, d), v[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s.x += v[k][i];
        }
    } else {
        for (int64_t c = first; c < d; c += step) {
            load_vec(xr, c, d, v[0]);
#pragma unroll
            for (int i = 0; i < V; ++i) s.x += v[0][i];
        }
    }
    const float mean = row_sum2(s, lanes).x / (float)d;
    s = {0.f, 0.f};
    auto square = [&](int64_t c, const float *u) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = c + i < d ? u[i] - mean : 0.f;
            s.x += t * t;
        }
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) square(first + k * step, v[k]);
    } else {
        for (int64_t c = first; c < d; c += step) { load_vec(xr, c, d, v[0]); square(c, v[0]); }
    }
    const float rstd = 1.f / sqrtf(row_sum2(s, lanes).x / (float)d + eps);
    if (!live) return;
    if (lane == 0) { mean_out[row] = mean; rstd_out[row] = rstd; }
    auto write = [&](int64_t c, float *u) {
        if (c >= d) return;
        float g[V], b[V];
        load_vec(gamma, c, d, g);
        load_vec(beta, c, d, b);
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = (u[i] - mean) * rstd * g[i] + b[i];
        store_vec<T, true>(yr, c, d, u);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) write(first + k * step, v[k]);
    } else {
        for (int64_t c = first; c < d; c += step) { load_vec(xr, c, d, v[0]); write(c, v[0]); }
    }
}

// The same pointer, of which the compiler does not know that it is: what is loaded from it is not kept from an earlier load.
template <typename T>
__device__ __forceinline__ const T *fresh(const T *p)
{
    asm volatile("" : "+s"(p));
    return p;
}

// Gradients.  Workgroup b takes rows b * groups + group, then gridDim.x * groups further on, and leaves its sums of dy xhat and
// of dy by column in part[b][0 .. d) and part[b][d .. 2 d): the sums over rows have one order whatever the timing.
template <typename T, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void layer_norm_grad_rows(const T *__restrict__ dy, int64_t lddy, const T *__restrict__ x, int64_t ldx,
                                                           const T *__restrict__ gamma, const float *__restrict__ mean_in,
                                                           const float *__restrict__ rstd_in, T *__restrict__ dx, int64_t lddx,
                                                           float *__restrict__ part, int64_t n, int64_t d, int lanes)
{
    constexpr int V = Elem<T>::VEC, N = NV ? NV : 1;
    extern __shared__ __align__(16) float group_sums[];
    const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, groups = blockDim.x / lanes;
    int64_t first = (int64_t)lane * V;
    const int64_t step = (int64_t)lanes * V;
    float *mine = part + (int64_t)blockIdx.x * 2 * d;
    constexpr bool HELD = NV == 1 || (NV > 1 && THREADS <= 256);           // gamma in registers, where there are enough
    float sg[N][V] = {}, sb[N][V] = {}, ga[HELD ? N : 1][V];
    if constexpr (NV > 0) {
        if constexpr (HELD)
#pragma unroll
            for (int k = 0; k < NV; ++k) load_vec(gamma, first + k * step, d, ga[k]);
    } else {
        for (int64_t c = first; c < d; c += step)
            for (int i = 0; i < V && c + i < d; ++i) mine[c + i] = mine[d + c + i] = 0.f;
    }
    // The next row is on its way while this one is added up, where there are registers for it.
    constexpr bool AHEAD = HELD;
    u32x4 next_x[AHEAD ? N : 1], next_dy[AHEAD ? N : 1];
    float next_mean, next_rstd;
    auto ask = [&](int64_t row) {
        row = min(row, n - 1);
        next_mean = mean_in[row];
        next_rstd = rstd_in[row];
        if constexpr (AHEAD)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                next_x[k] = ask_raw<T, true>(x + row * ldx, first + k * step, d);
                next_dy[k] = ask_raw<T, true>(dy + row * lddy, first + k * step, d);
            }
    };
    ask((int64_t)blockIdx.x * groups + group);
    for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < n; row0 += (int64_t)gridDim.x * groups) {
        const int64_t row = row0 + group;
        const bool live = row < n;
        const T *xr = x + (live ? row : n - 1) * ldx, *dyr = dy + (live ? row : n - 1) * lddy;
        T *dxr = dx + (live ? row : n - 1) * lddx;
        const float mean = next_mean, rstd = next_rstd;
        float h[N][V], g[N][V];                          // xhat and dy
        float2 s = {0.f, 0.f};
        if constexpr (AHEAD) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                unpack<T>(settle<T>(next_x[k], first + k * step, d), h[k]);
                unpack<T>(settle<T>(next_dy[k], first + k * step, d), g[k]);
            }
        }
        ask(row + (int64_t)gridDim.x * groups);
        if constexpr (NV > 1 && !HELD) asm volatile("" : "+v"(first));     // (nor addresses from the row before: the registers are full)
        // Past the end of the row dy is zero, so what xhat has there counts nowhere.
        auto take = [&](int64_t c, float *hk, float *gk, const float *gak) {
            if constexpr (!AHEAD) {
                load_vec(xr, c, d, hk);
                load_vec(dyr, c, d, gk);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                hk[i] = (hk[i] - mean) * rstd;
                s.x += gk[i] * gak[i];
                s.y += gk[i] * gak[i] * hk[i];
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if constexpr (!HELD) load_vec(fresh(gamma), first + k * step, d, ga[0]);
                take(first + k * step, h[k], g[k], ga[HELD ? k : 0]);
            }
        } else {
            for (int64_t c = first; c < d; c += step) { load_vec(gamma, c, d, ga[0]); take(c, h[0], g[0], ga[0]); }
        }
        s = row_sum2(s, lanes);
        const float mg = s.x / (float)d, mh = s.y / (float)d;
        if (!live) continue;
        auto give = [&](int64_t c, const float *hk, float *gk, const float *gak) {
#pragma unroll
            for (int i = 0; i < V; ++i) gk[i] = rstd * (gk[i] * gak[i] - mg - hk[i] * mh);
            if (c < d) store_vec<T, true>(dxr, c, d, gk);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
#pragma unroll
                for (int i = 0; i < V; ++i) { sg[k][i] += g[k][i] * h[k][i]; sb[k][i] += g[k][i]; }
                if constexpr (!HELD) load_vec(fresh(gamma), first + k * step, d, ga[0]);
                give(first + k * step, h[k], g[k], ga[HELD ? k : 0]);
            }
        } else {
            for (int64_t c = first; c < d; c += step) {
                load_vec(gamma, c, d, ga[0]);
                take(c, h[0], g[0], ga[0]);
                for (int i = 0; i < V && c + i < d; ++i) { mine[c + i] += g[0][i] * h[0][i]; mine[d + c + i] += g[0][i]; }
                give(c, h[0], g[0], ga[0]);
            }
        }
    }
    if constexpr (NV > 0) {
        // the groups of a workgroup by halves
        for (int k = 0; k < NV; ++k)
            for (int which = 0; which < 2; ++which) {
                float *u = which ? sb[k] : sg[k];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < V; ++i) group_sums[threadIdx.x * V + i] = u[i];
                __syncthreads();
                for (int half = groups / 2; half > 0; half /= 2) {
                    if (group < half)
#pragma unroll
                        for (int i = 0; i < V; ++i) group_sums[threadIdx.x * V + i] += group_sums[(threadIdx.x + half * lanes) * V + i];
                    __syncthreads();
                }
                if (group == 0)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int64_t c = first + k * step + i;
                        if (c < d) mine[which * d + c] = group_sums[threadIdx.x * V + i];
                    }
            }
    }
}

// Sums of the workgroups' parts: LN_SUM_COLUMNS columns of [dgamma | dbeta] to a workgroup, from `first` on, 64 threads to a column.
constexpr int LN_SUM_COLUMNS = 16;

template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_grad_sums(const float *__restrict__ part, int parts, int64_t d, int64_t first, T *__restrict__ dgamma,
                                                             T *__restrict__ dbeta)
{
    constexpr int SLICES = 1024 / LN_SUM_COLUMNS;
    __shared__ float s[SLICES][LN_SUM_COLUMNS + 1];
    const int col = threadIdx.x % LN_SUM_COLUMNS, slice = threadIdx.x / LN_SUM_COLUMNS;
    const int64_t c = first + (int64_t)blockIdx.x * LN_SUM_COLUMNS + col;
    float t = 0.f;
    if (c < 2 * d) {
#pragma unroll 8
        for (int p = slice; p < parts; p += SLICES) t += part[(int64_t)p * 2 * d + c];
    }
    s[slice][col] = t;
    __syncthreads();
    for (int half = SLICES / 2; half > 0; half /= 2) {
        if (slice < half) s[slice][col] += s[slice + half][col];
        __syncthreads();
    }
    if (slice || c >= 2 * d) return;
    t = s[0][col];
    if (c < d) dgamma[c] = (T)t;
    else dbeta[c - d] = (T)t;
}

}  // namespace chicle_train
