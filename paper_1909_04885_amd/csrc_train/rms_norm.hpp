// Root-mean-square norm on a residual stream, and its gradients.
//
//   r = x + residual, rounded to the type,  rstd = 1 / sqrt(sum_c r_c^2 / d + eps),  y_c = r_c rstd gamma_c
//   with h_c = r_c rstd and g_c = dy_c gamma_c:
//   dx_c = rstd (g_c - h_c mean(g h)) + dr_c,  dgamma_c = sum_rows dy_c h_c
//
// dx is the gradient of x and of the residual; dr is what reaches r on the other way.  y can be given in 8 bits instead of the type
// (from its 32-bit values), and r a second time in 8 bits, which is what the gradient then takes.
//
// A row is held in registers by `lanes` neighbouring threads, NV vectors of sixteen bytes each, and read once: NV is two for rows of up to 4096 columns
// of 16 bits, where a workgroup of 256 threads has one, and short rows share a workgroup.  Rows that no workgroup holds (NV = 0) are read again.
// The bound is the memory (a large copy: 4.95 TB/s).  Forward, 32,768 x 4096 in bfloat16 with a residual, y and r in 8 bits: 181 us, 6.0 TB/s; one row of
// 4096: 4.0 us, a launch.  Gradients, 65,536 x 4096 in bfloat16 from r in 8 bits with dr: 330 us, 5.7 TB/s, and 6 for the sums over workgroups;
// 9001 x 1537 in float32, 1540 apart: 46 and 5, 4.9 TB/s.  Gradients of rows that no workgroup holds read twice: 3000 x 20,000 in bfloat16 369 us, 1.3 TB/s.
#pragma once
#include "elements.hpp"
#include "layer_norm.hpp"
#include "packed.hpp"

namespace chicle_train {

// The sum over the `lanes` threads of a row (all threads of the workgroup where lanes > 64); every thread of the workgroup takes part in
// the same calls.  beside: gets that of the row beside it where a workgroup of 256 threads has two such rows, else the row's own.
__device__ __forceinline__ float row_sum(float s, int lanes, float *beside = nullptr)
{
    s = lanes_sum(s, lanes < 64 ? lanes : 64);
    if (beside) *beside = s;
    if (lanes <= 64) return s;
    __shared__ float part[LN_MOST_THREADS / 64];
    const int wave = threadIdx.x >> 6, waves = lanes >> 6;
    __syncthreads();                                     // (the sums before these have been read)
    if ((threadIdx.x & 63) == 0) part[wave] = s;
    __syncthreads();
    const int first = wave / waves * waves;              // (waves is a power of two: the row's own)
    s = part[first];
    for (int i = 1; i < waves; ++i) s += part[first + i];
    if (beside) *beside = lanes == 128 ? part[first ^ 2] + part[first ^ 3] : s;
    return s;
}

template <typename T> struct RmsRows {
    const T *x, *residual, *gamma;                       // residual: or null
    T *sum, *y;                                          // each or null
    float *rstd;
    Packed y8, sum8;                                     // q null: not asked for
    int64_t ldx, ldres, ldsum, ldy, n, d;
    int lanes;
    float eps;
};

// blockDim.x is a multiple of lanes, and lanes hold whole groups of columns.
template <typename T, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void rms_norm_rows(const RmsRows<T> a)
{
    constexpr int V = Elem<T>::VEC;
    const int lane = threadIdx.x % a.lanes;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / a.lanes) + threadIdx.x / a.lanes;
    const bool live = row < a.n;
    const int64_t at = live ? row : a.n - 1, d = a.d;    // (threads without a row go through the sums with the others)
    const T *xr = a.x + at * a.ldx, *resr = a.residual ? a.residual + at * a.ldres : nullptr;
    const int64_t first = (int64_t)lane * V, step = (int64_t)a.lanes * V, whole = (d + PACK_GROUP - 1) / PACK_GROUP * PACK_GROUP;
    float v[NV ? NV : 1][V];
    float s = 0.f;
    auto add = [&](u32x4 xs, u32x4 rs, int64_t c, float *u) {
        unpack<T>(settle<T>(xs, c, d), u);
        if (resr) {
            float w[V];
            unpack<T>(settle<T>(rs, c, d), w);
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = (float)(T)(u[i] + w[i]);
        }
    };
    auto square = [&](const float *u) {
#pragma unroll
        for (int i = 0; i < V; ++i) s += u[i] * u[i];
    };
    if constexpr (NV > 0) {
        u32x4 xs[NV], rs[NV] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            xs[k] = ask_raw<T, true>(xr, first + k * step, d);
            if (resr) rs[k] = ask_raw<T, true>(resr, first + k * step, d);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            add(xs[k], rs[k], first + k * step, v[k]);
            square(v[k]);
        }
    } else {
        for (int64_t c = first; c < d; c += step) {
            add(ask_raw<T>(xr, c, d), resr ? ask_raw<T>(resr, c, d) : u32x4{0u, 0u, 0u, 0u}, c, v[0]);
            square(v[0]);
        }
    }
    float beside, mean = row_sum(s, a.lanes, &beside) / (float)d + a.eps, scale = 1.f;
    // Squares of values beyond 2^64 are no 32-bit numbers, and, where eps is none, those below 2^-64 lose theirs: such a row is summed once more, its values times
    // 2^-96 or 2^96.  (Half precision has neither.)  Two rows whose sums have barriers go the same way; with a barrier of its own for that, 200,000 x 1000 in
    // bfloat16 took 284 us instead of 275.
    if constexpr (!__is_same(T, f16)) {
        auto outside = [](float x) { return x < 0x1p-100f || x == __builtin_huge_valf(); };
        const bool out = outside(mean), again = out || outside(beside / (float)d + a.eps);
        if (__builtin_expect(again, 0)) {
            const float by = mean > 1.f ? 0x1p-96f : 0x1p96f;
            s = 0.f;
            auto square_again = [&](const float *u) {
#pragma unroll
                for (int i = 0; i < V; ++i) s += (u[i] * by) * (u[i] * by);
            };
            if constexpr (NV > 0) {
#pragma unroll
                for (int k = 0; k < NV; ++k) square_again(v[k]);
            } else {
                for (int64_t c = first; c < d; c += step) {
                    add(ask_raw<T>(xr, c, d), resr ? ask_raw<T>(resr, c, d) : u32x4{0u, 0u, 0u, 0u}, c, v[0]);
                    square_again(v[0]);
                }
            }
            const float other = row_sum(s, a.lanes) / (float)d + a.eps * by * by;
            if (out) {
                mean = other;
                scale = by;
            }
        }
    }
    const float rstd = scale / sqrtf(mean);
    if (!live) return;
    if (lane == 0) a.rstd[row] = rstd;
    auto write = [&](int64_t c, float *u) {
        if (c >= whole) return;
        if (a.sum && c < d) store_vec<T, true>(a.sum + row * a.ldsum, c, d, u);
        if (a.sum8.q) pack_vec<T>(u, a.sum8.q + row * a.sum8.ld, a.sum8.scales + row * (a.sum8.ld / PACK_GROUP), c);
        float g[V];
        load_vec(a.gamma, c, d, g);
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = u[i] * rstd * g[i];
        if (a.y && c < d) store_vec<T, true>(a.y + row * a.ldy, c, d, u);
        if (a.y8.q) pack_vec<T>(u, a.y8.q + row * a.y8.ld, a.y8.scales + row * (a.y8.ld / PACK_GROUP), c);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) write(first + k * step, v[k]);
    } else {
        for (int64_t c = first; c < whole; c += step) {
            add(ask_raw<T>(xr, c, d), resr ? ask_raw<T>(resr, c, d) : u32x4{0u, 0u, 0u, 0u}, c, v[0]);
            write(c, v[0]);
        }
    }
}

// Rows of T, or packed ones.
template <typename T, bool PACKED> struct RmsKept;
template <typename T> struct RmsKept<T, false> {
    typedef u32x4 raw;
    const T *p;
    int64_t ld;
    __device__ __forceinline__ raw ask(int64_t row, int64_t c, int64_t d) const { return ask_raw<T, true>(p + row * ld, c, d); }
    static __device__ __forceinline__ void values(const raw &x, int64_t c, int64_t d, float *out) { unpack<T>(settle<T>(x, c, d), out); }
};
template <typename T> struct RmsKept<T, true> {
    typedef RawPacked<T> raw;
    const int8_t *q;
    const uint8_t *scales;
    int64_t ld;
    __device__ __forceinline__ raw ask(int64_t row, int64_t c, int64_t d) const
    {
        // (past the last column dy is zero and counts; what is asked for there is some group that is there)
        const int64_t most = (d + PACK_GROUP - 1) / PACK_GROUP * PACK_GROUP - Elem<T>::VEC;
        return ask_packed<T, true>(q + row * ld, scales + row * (ld / PACK_GROUP), c < most ? c : most);
    }
    static __device__ __forceinline__ void values(const raw &x, int64_t, int64_t, float *out) { unpack8<T>(x, out); }
};

template <typename T, bool PACKED> struct RmsGrad {
    RmsKept<T, PACKED> r;
    const T *dy, *dr, *gamma;                            // dr: or null
    const float *rstd;
    T *dx;
    float *part;
    int64_t lddy, lddr, lddx, n, d;
    int lanes;
};

// Workgroup b takes rows b * groups + group, then gridDim.x * groups further on, and leaves its sums of dy h by column in part[b][0 .. d):
// the sums over rows have one order whatever the timing.
template <typename T, int NV, int THREADS, bool PACKED>
__global__ __launch_bounds__(THREADS) void rms_norm_grad_rows(const RmsGrad<T, PACKED> a)
{
    constexpr int V = Elem<T>::VEC, N = NV ? NV : 1;
    typedef RmsKept<T, PACKED> Kept;
    extern __shared__ __align__(16) float group_sums[];
    const int64_t d = a.d;
    const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = blockDim.x / a.lanes;
    const int64_t first = (int64_t)lane * V, step = (int64_t)a.lanes * V;
    float *mine = a.part + (int64_t)blockIdx.x * d;
    // gamma, and the next row, in registers, where there are enough; else a thread's vectors of gamma lie in LDS, where they do not wait behind the next
    // row (read from memory twice a row: 10,143 x 10,061 in bfloat16 280 us instead of 245)
    constexpr bool HELD = NV > 0 && (NV * V <= 8 || THREADS <= 256), AHEAD = HELD || (NV > 0 && sizeof(T) == 2);
    float sg[N][V] = {}, ga[HELD ? N : 1][V];
    u32x4 *own_gamma = (u32x4 *)group_sums + threadIdx.x;
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (HELD) load_vec(a.gamma, first + k * step, d, ga[k]);
            else own_gamma[k * blockDim.x] = load_raw(a.gamma, first + k * step, d);
        }
    } else {
        for (int64_t c = first; c < d; c += step)
            for (int i = 0; i < V && c + i < d; ++i) mine[c + i] = 0.f;
    }
    typename Kept::raw next_r[AHEAD ? N : 1];
    u32x4 next_dy[AHEAD ? N : 1];
    float next_rstd;
    auto ask = [&](int64_t row) {
        row = min(row, a.n - 1);
        next_rstd = a.rstd[row];
        if constexpr (AHEAD)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                next_r[k] = a.r.ask(row, first + k * step, d);
                next_dy[k] = ask_raw<T, true>(a.dy + row * a.lddy, first + k * step, d);
            }
    };
    ask((int64_t)blockIdx.x * groups + group);
    for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < a.n; row0 += (int64_t)gridDim.x * groups) {
        const int64_t row = row0 + group;
        const bool live = row < a.n;
        const int64_t at = live ? row : a.n - 1;
        const T *dyr = a.dy + at * a.lddy, *drr = a.dr ? a.dr + at * a.lddr : nullptr;
        const float rstd = next_rstd;
        float h[N][V], g[N][V];                          // h and dy
        u32x4 drs[N] = {};
        float s = 0.f;
        if constexpr (AHEAD) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                Kept::values(next_r[k], first + k * step, d, h[k]);
                unpack<T>(settle<T>(next_dy[k], first + k * step, d), g[k]);
                if (drr) drs[k] = ask_raw<T, true>(drr, first + k * step, d);
            }
        }
        ask(row + (int64_t)gridDim.x * groups);
        // Past the end of the row dy is zero, so what h has there counts nowhere.
        auto take = [&](int64_t c, float *hk, float *gk, const float *gak) {
            if constexpr (!AHEAD) {
                Kept::values(a.r.ask(at, c, d), c, d, hk);
                load_vec(dyr, c, d, gk);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                hk[i] *= rstd;
                s += gk[i] * gak[i] * hk[i];
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if constexpr (!HELD) unpack<T>(own_gamma[k * blockDim.x], ga[0]);
                take(first + k * step, h[k], g[k], ga[HELD ? k : 0]);
            }
        } else {
            for (int64_t c = first; c < d; c += step) { load_vec(a.gamma, c, d, ga[0]); take(c, h[0], g[0], ga[0]); }
        }
        const float mh = row_sum(s, a.lanes) / (float)d;
        if (!live) continue;
        auto give = [&](int64_t c, const float *hk, float *gk, const float *gak, u32x4 more) {
            float o[V] = {};
            if (drr) unpack<T>(settle<T>(more, c, d), o);
#pragma unroll
            for (int i = 0; i < V; ++i) gk[i] = rstd * (gk[i] * gak[i] - hk[i] * mh) + o[i];
            if (c < d) store_vec<T, true>(a.dx + row * a.lddx, c, d, gk);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
#pragma unroll
                for (int i = 0; i < V; ++i) sg[k][i] += g[k][i] * h[k][i];
                if constexpr (!HELD) unpack<T>(own_gamma[k * blockDim.x], ga[0]);
                if constexpr (!AHEAD)
                    if (drr) drs[k] = ask_raw<T, true>(drr, first + k * step, d);
                give(first + k * step, h[k], g[k], ga[HELD ? k : 0], drs[k]);
            }
        } else {
            for (int64_t c = first; c < d; c += step) {
                load_vec(a.gamma, c, d, ga[0]);
                if (drr) drs[0] = ask_raw<T>(drr, c, d);
                take(c, h[0], g[0], ga[0]);
                for (int i = 0; i < V && c + i < d; ++i) mine[c + i] += g[0][i] * h[0][i];
                give(c, h[0], g[0], ga[0], drs[0]);
            }
        }
    }
    if constexpr (NV > 0) {
        // the groups of a workgroup by halves
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) group_sums[threadIdx.x * V + i] = sg[k][i];
            __syncthreads();
            for (int half = groups / 2; half > 0; half /= 2) {
                if (group < half)
#pragma unroll
                    for (int i = 0; i < V; ++i) group_sums[threadIdx.x * V + i] += group_sums[(threadIdx.x + half * a.lanes) * V + i];
                __syncthreads();
            }
            if (group == 0)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int64_t c = first + k * step + i;
                    if (c < d) mine[c] = group_sums[threadIdx.x * V + i];
                }
        }
    }
}

// Sums of the workgroups' parts: LN_SUM_COLUMNS columns to a workgroup, from `first` on, 64 threads to a column.
template <typename T>
__global__ __launch_bounds__(1024) void rms_norm_grad_sums(const float *__restrict__ part, int parts, int64_t d, int64_t first, T *__restrict__ dgamma)
{
    constexpr int SLICES = 1024 / LN_SUM_COLUMNS;
    __shared__ float s[SLICES][LN_SUM_COLUMNS + 1];
    const int col = threadIdx.x % LN_SUM_COLUMNS, slice = threadIdx.x / LN_SUM_COLUMNS;
    const int64_t c = first + (int64_t)blockIdx.x * LN_SUM_COLUMNS + col;
    float t = 0.f;
    if (c < d) {
#pragma unroll 8
        for (int p = slice; p < parts; p += SLICES) t += part[(int64_t)p * d + c];
    }
    s[slice][col] = t;
    __syncthreads();
    for (int half = SLICES / 2; half > 0; half /= 2) {
        if (slice < half) s[slice][col] += s[slice + half][col];
        __syncthreads();
    }
    if (slice == 0 && c < d) dgamma[c] = (T)s[0][col];
}

}  // namespace chicle_train
