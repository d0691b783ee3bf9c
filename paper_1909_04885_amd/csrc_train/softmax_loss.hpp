// Softmax cross entropy over many classes and its gradients, without keeping the logits.
//
//   z_iv = x_i . w_v,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i,label(i)
//   G_iv = weight_i (exp(z_iv - lse_i) - [v = label(i)]),  dx_i = sum_v G_iv w_v,  dw_v = sum_i G_iv x_i
//   A row whose label is negative has the loss 0 and G = 0; its x counts nowhere, whatever it holds.
//
// The loss: logits exist only as tiles of a product in registers.  `loss_tiles` leaves of a wavefront's part of a tile, for every row, the
// largest logit and the sum of exponentials below it, and `loss_rows` joins these.
//
// The gradient in 16 bits forms the logits again, a piece of the classes at a time, and turns them in registers into G, which is stored for
// the two products that read it.  Rows of G add up to zero, so what all classes (or those that a row's softmax lies on) have in
// common drops out of dx; 8 or 11 bits of G do not add up to zero, and leave that common part times their errors: with classes around a common mean
// the relative error of dx was 0.033 in bfloat16, where the rounding of dx itself is 0.0017.  G is held in two planes that add up to it,
// the second what the first's rounding leaves, 16 bits or 22 together, and each goes through the products.  Half precision would
// lose small G: there it comes 2^14 times as large, divided by the largest weight, and the products times it.  In 32 bits a
// product costs eight times as much, and the logits of a piece of the rows are kept until they are G; so are those of few rows and of
// few classes, which are few bytes.
//
// The bound is the matrix cores: 2 n d classes operations for the loss, and twice that again for the gradients (five times in 16 bits).
// With gradients, 8192 rows of 2048 and 128,000 classes in bfloat16: 22.7 ms, 1135 TFLOP/s of the six products; 4096 rows of 1024 and
// 50,021 classes: 2.46 ms, 1020; 333 rows of 250 and 20,000 classes in 32 bits: 160 us, 62 TFLOP/s of 154, three products of 8 to 11
// slices each, most of whose time is their beginning and end.  Few rows are bound by reading w: one row against 32,000 classes of
// 1024 in bfloat16 16 us, 13.5 of them the product at 4.8 TB/s.
#pragma once
#include "matmul.hpp"

namespace chicle_train {

// ---- operands laid out for the products -----------------------------------------------------------------------------

// out[r][c] = in[r][c], zeros in columns [cols, ld) and in rows [rows, rows_out): whole slices of aligned chunks.  With labels, rows that
// have none are zeros too.
template <typename T>
__global__ __launch_bounds__(256) void lay_rows(const T *__restrict__ in, int64_t ldi, T *__restrict__ out, int64_t ld, int64_t rows, int64_t rows_out,
                                                int64_t cols, const void *labels, int wide, int64_t classes)
{
    const int64_t per_row = ld / MM_CHUNK<T>;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < rows_out * per_row; e += (int64_t)gridDim.x * 256) {
        const int64_t r = e / per_row, c = (e - r * per_row) * MM_CHUNK<T>;
        bool has = r < rows;
        if (has && labels) {
            const int64_t label = index_at(labels, wide, r);
            has = label >= 0 && label < classes;
        }
        *(u32x4 *)(out + r * ld + c) = has ? load_raw(in + r * ldi, c, cols) : u32x4{0u, 0u, 0u, 0u};
    }
}

// ---- the loss -------------------------------------------------------------------------------------------------------

struct LossRows {
    const void *labels;
    int wide, n, classes;
    const float *lse;            // gradient
    const float *weight;
    const float *power;          // half precision: G comes times this; else null
    float2 *part;                // [row][wavefront's part of a tile of classes]: largest logit, sum of exponentials below it
    float *picked;               // [row]: the label's logit
};

// The row's class, or -1
__device__ __forceinline__ int label_at(const LossRows &l, int j)
{
    const int64_t label = j < l.n ? index_at(l.labels, l.wide, j) : -1;
    return label >= 0 && label < l.classes ? (int)label : -1;
}

constexpr float MINUS_INF = -__builtin_inff();

// exp(a - b), 0 where a is minus infinity
template <bool EXACT> __device__ __forceinline__ float exp_diff(float a, float b)
{
    return a == MINUS_INF ? 0.f : EXACT ? expf(a - b) : __expf(a - b);
}

constexpr float LOG2E = 1.44269504088896340736f;

// exp(z - m).  EXACT: the library's exponential; else the instruction's, whose error of 2^-22 and |z - m| 2^-24 is far below what
// 16-bit gradients show.  The difference comes first: of two numbers of the type's lowest value it is zero.
template <bool EXACT> __device__ __forceinline__ float exp_of(float z, float m)
{
    return EXACT ? expf(z - m) : __builtin_amdgcn_exp2f((z - m) * LOG2E);
}

// i: classes, j: rows.  logits: null, or [row][ldz], where they are kept (KEEP: they may be).
template <typename T, typename C, bool KEEP>
__global__ __launch_bounds__(C::THREADS, C::PER_SIMD) void loss_tiles(MmShape s, LossRows l, float *__restrict__ logits, int64_t ldz)
{
    constexpr bool EXACT = sizeof(T) == 4;
    mm_tiles<T, C, false, false>(s, [&](const MmTile &t, f32x4 (&acc)[C::MI][C::NJ]) __attribute__((always_inline)) {
        const MmPlace<C, false> at(t);
        if ((t.i + 1) * C::TILE_I > l.classes) {         // the last tile: what lies past the classes counts nowhere
#pragma unroll
            for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at.i0 + at.place(mi) + r >= l.classes)
#pragma unroll
                        for (int nj = 0; nj < C::NJ; ++nj) acc[mi][nj][r] = MINUS_INF;
        }
#pragma unroll
        for (int nj = 0; nj < C::NJ; ++nj) {
            const int j = at.j0 + nj * 16, rel = label_at(l, j) - at.i0;
            if (rel >= 0 && rel < C::MI * 16 && (rel & 31) < 8) {          // the label's logit is this lane's
                float z = 0.f;
#pragma unroll
                for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z = rel == at.place(mi) + r ? acc[mi][nj][r] : z;
                l.picked[j] = z;
            }
            if constexpr (KEEP)
                if (logits && j < l.n)                   // (rows of logits are whole tiles long)
#pragma unroll
                    for (int mi = 0; mi < C::MI; ++mi) *(f32x4 *)(logits + (int64_t)j * ldz + at.i0 + at.place(mi)) = acc[mi][nj];
            float m = MINUS_INF;
#pragma unroll
            for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[mi][nj][r]);
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const float shift = m == MINUS_INF ? 0.f : m;
            float e = 0.f;
#pragma unroll
            for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
                for (int r = 0; r < 4; ++r) e += exp_of<EXACT>(acc[mi][nj][r], shift);
            e += __shfl_xor(e, 16);
            e += __shfl_xor(e, 32);
            if (at.lane < 16 && j < l.n) l.part[(int64_t)j * s.tiles_i * C::W_I + t.i * C::W_I + at.wi] = make_float2(m, e);
        }
    });
}

// A wavefront to a row, ROW_PARTS parts of a lane at a time.
constexpr int ROW_PARTS = 8;

__global__ __launch_bounds__(256) void loss_rows(LossRows l, int tiles, float *__restrict__ loss, float *__restrict__ lse_out, int *flags)
{
    const int j = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (j >= l.n) return;
    const int64_t label = index_at(l.labels, l.wide, j);
    const float2 *p = l.part + (int64_t)j * tiles;
    float m = MINUS_INF, e = 0.f;
    for (int i = lane; i < tiles; i += 64 * ROW_PARTS) {
        float2 u[ROW_PARTS];                             // (on their way together)
#pragma unroll
        for (int q = 0; q < ROW_PARTS; ++q) u[q] = i + q * 64 < tiles ? p[i + q * 64] : make_float2(MINUS_INF, 0.f);
        float top = m;
#pragma unroll
        for (int q = 0; q < ROW_PARTS; ++q) top = fmaxf(top, u[q].x);
        e *= exp_diff<true>(m, top);
        m = top;
#pragma unroll
        for (int q = 0; q < ROW_PARTS; ++q) e += u[q].y * exp_diff<true>(u[q].x, m);
    }
    float top = m;
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    e = lanes_sum(e * exp_diff<true>(m, top), 64);
    if (lane) return;
    const float lse = top + logf(e);
    if (label >= l.classes && flags) atomicOr(flags, FLAG_LABEL_RANGE);
    lse_out[j] = lse;
    loss[j] = label >= 0 && label < l.classes ? lse - l.picked[j] : 0.f;
}

// The same of logits that come in several parts, where there are few tiles and each is a long sum: a workgroup to a row.  The first part is
// left as their sum.
__global__ __launch_bounds__(256) void loss_join(LossRows l, float *parts, int64_t ldz, int64_t copy, int copies, float *__restrict__ loss,
                                                 float *__restrict__ lse_out, int *flags)
{
    __shared__ float s[8], picked;
    const int j = blockIdx.x, label = label_at(l, j), wave = threadIdx.x >> 6;
    float *z = parts + j * ldz;
    float m = MINUS_INF;
    for (int c = threadIdx.x; c < l.classes; c += 256) {
        float t = 0.f;
#pragma unroll 4
        for (int k = 0; k < copies; ++k) t += z[k * copy + c];
        z[c] = t;
        if (c == label) picked = t;
        m = fmaxf(m, t);
    }
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if ((threadIdx.x & 63) == 0) s[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    const float shift = m == MINUS_INF ? 0.f : m;
    float e = 0.f;
    for (int c = threadIdx.x; c < l.classes; c += 256) e += exp_of<true>(z[c], shift);
    e = lanes_sum(e, 64);
    if ((threadIdx.x & 63) == 0) s[4 + wave] = e;
    __syncthreads();
    if (threadIdx.x) return;
    const float lse = m + logf((s[4] + s[5]) + (s[6] + s[7]));
    if (index_at(l.labels, l.wide, j) >= l.classes && flags) atomicOr(flags, FLAG_LABEL_RANGE);
    lse_out[j] = lse;
    loss[j] = label >= 0 ? lse - picked : 0.f;
}

// power[0]: what takes the largest weight of a row with a label to `top`, power[1] its inverse.  One workgroup.
__global__ __launch_bounds__(1024) void loss_power(LossRows l, float top, float *power)
{
    __shared__ float s[16];
    float m = 0.f;
    for (int i = threadIdx.x; i < l.n; i += 1024) {
        const float w = label_at(l, i) >= 0 ? fabsf(l.weight[i]) : 0.f;
        if (!__builtin_isinf(w)) m = fmaxf(m, w);        // (NaN neither)
    }
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
    const bool plain = m < 1e-30f;                       // (no weight, or one whose inverse is out of range)
    power[0] = plain ? 1.f : top / m;
    power[1] = plain ? 1.f : m / top;
}

// ---- the gradients --------------------------------------------------------------------------------------------------

// The two planes of x: what is rounded, and what that leaves (nothing of an infinity).
template <typename T> __device__ __forceinline__ void two_planes(float x, T &high, T &low)
{
    high = (T)x;
    const float rest = x - (float)high;
    low = (T)(__builtin_isinf(x) || __builtin_isinf((float)high) ? 0.f : rest);
}

// G of a piece of the classes, 16 bits: s.a is the piece's rows of w, `first` the piece's first class.  g[row][class of the piece], with
// zeros up to ldg and in rows [n, rows_out), the second plane `plane` values further on.
template <typename T, typename C>
__global__ __launch_bounds__(C::THREADS, C::PER_SIMD) void loss_grad_tiles(MmShape s, LossRows l, int first, int piece, T *__restrict__ g, int64_t ldg,
                                                                           int64_t plane, int rows_out)
{
    const float power = l.power ? l.power[0] : 1.f;
    mm_tiles<T, C, false, false>(s, [&](const MmTile &t, f32x4 (&acc)[C::MI][C::NJ]) __attribute__((always_inline)) {
        const MmPlace<C, false> at(t);
#pragma unroll
        for (int nj = 0; nj < C::NJ; ++nj) {
            const int j = at.j0 + nj * 16, label = label_at(l, j), rel = label - first - at.i0;
            const float weight = label >= 0 ? l.weight[j] * power : 0.f, lse = label >= 0 ? l.lse[j] : 0.f;
            T *row = g + (int64_t)j * ldg;
#pragma unroll
            for (int mp = 0; mp < C::MI / 2; ++mp) {     // eight neighbouring classes
                T v[8], low[8];
                const int i = at.i0 + mp * 32;
#pragma unroll
                for (int h = 0; h < 8; ++h) {
                    float p = exp_of<false>(acc[2 * mp + h / 4][nj][h % 4], lse);
                    if (rel == mp * 32 + h) p -= 1.f;
                    two_planes(weight != 0.f && i + h < piece ? p * weight : 0.f, v[h], low[h]);
                }
                if (j < rows_out && i < ldg) {
                    __builtin_memcpy(row + i, v, 16);
                    __builtin_memcpy(row + plane + i, low, 16);
                }
            }
        }
    });
}

// G of logits that were kept: g[row][class] of all classes, zeros up to ldg and in rows [n, rows_out).  In 32 bits g may be the logits
// themselves; in 16 the second plane lies `plane` values further on.  Grid: (rows, columns).
template <typename T>
__global__ __launch_bounds__(256) void loss_grad_kept(const float *logits, int64_t ldz, LossRows l, T *g, int64_t ldg, int64_t plane)
{
    const int j = blockIdx.x, label = label_at(l, j);
    const float power = l.power ? l.power[0] : 1.f;
    const float weight = label >= 0 ? l.weight[j] * power : 0.f, lse = label >= 0 ? l.lse[j] : 0.f;
    for (int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4; c < ldg; c += (int64_t)gridDim.y * 1024) {
        T v[4], low[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float p = 0.f;
            if (weight != 0.f && c + h < l.classes) {
                p = expf(logits[j * ldz + c + h] - lse);
                if (c + h == label) p -= 1.f;
                p *= weight;
            }
            if constexpr (sizeof(T) == 4) v[h] = p;
            else two_planes(p, v[h], low[h]);
        }
        __builtin_memcpy(g + j * ldg + c, v, sizeof v);
        if constexpr (sizeof(T) == 2) __builtin_memcpy(g + plane + j * ldg + c, low, sizeof low);
    }
}

// A product as it is: out[j][i] in 32 bits, split `split` of the sum in its own copy of `out`; or added to what is there.
template <typename T, typename C, bool A_BY_K, bool B_BY_K, bool ADD = false>
__global__ __launch_bounds__(C::THREADS, C::PER_SIMD) void product_parts(MmShape s, float *__restrict__ out, int64_t ld, int64_t copy)
{
    mm_tiles<T, C, A_BY_K, B_BY_K>(s, [&](const MmTile &t, f32x4 (&acc)[C::MI][C::NJ]) __attribute__((always_inline)) {
        const MmPlace<C, A_BY_K> at(t);
        float *mine = out + t.split * copy;
#pragma unroll
        for (int nj = 0; nj < C::NJ; ++nj)
#pragma unroll
            for (int mi = 0; mi < C::MI; ++mi) {
                const int i = at.i0 + at.place(mi), j = at.j0 + nj * 16;
                if (j >= s.b.rows || i >= s.a.rows) continue;
                f32x4 *dst = (f32x4 *)(mine + (int64_t)j * ld + i);
                if constexpr (ADD) *dst += acc[mi][nj];
                else *dst = acc[mi][nj];
            }
    });
}

// x by G, both of which lie by k: out[j][i] = scale * sum, rounded; or added to what out holds.
template <typename T, typename C, bool ADD>
__global__ __launch_bounds__(C::THREADS, C::PER_SIMD) void product_out(MmShape s, T *__restrict__ out, int64_t ld, const float *__restrict__ scale)
{
    const float f = scale ? *scale : 1.f;
    mm_tiles<T, C, true, true>(s, [&](const MmTile &t, f32x4 (&acc)[C::MI][C::NJ]) __attribute__((always_inline)) {
        const MmPlace<C, true> at(t);
#pragma unroll
        for (int nj = 0; nj < C::NJ; ++nj)
#pragma unroll
            for (int mi = 0; mi < C::MI; ++mi) {
                const int i = at.i0 + at.place(mi), j = at.j0 + nj * 16;
                if (j >= s.b.rows) continue;
                T *dst = out + (int64_t)j * ld + i;
                if constexpr (ADD)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i + r < s.a.rows) acc[mi][nj][r] += (float)dst[r];
                T v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = (T)(acc[mi][nj][r] * f);
                if (i + 4 <= s.a.rows) __builtin_memcpy(dst, v, sizeof v);
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i + r < s.a.rows) dst[r] = v[r];
            }
    });
}

// out = scale * the sum of the copies, in their order: SLICES threads to four columns, each of which adds up a run of the copies.  ld of a copy
// is a multiple of four.  l.labels: null, or the rows are those of x, and one without a label is zero, whatever w holds.
template <typename O, int SLICES>
__global__ __launch_bounds__(256) void sum_parts(const float *__restrict__ part, int64_t ld, int64_t copy, int copies, O *__restrict__ out, int64_t ldo,
                                                 int64_t rows, int64_t cols, const float *__restrict__ scale, LossRows l)
{
    constexpr int EACH = 256 / SLICES;
    __shared__ f32x4 s[SLICES][EACH];
    const int64_t per_row = ld / 4, all = rows * per_row;
    const float f = scale ? *scale : 1.f;
    const int slice = threadIdx.x / EACH, mine = threadIdx.x % EACH;
    const int first = (int)((int64_t)copies * slice / SLICES), end = (int)((int64_t)copies * (slice + 1) / SLICES);
    for (int64_t e0 = (int64_t)blockIdx.x * EACH; e0 < all; e0 += (int64_t)gridDim.x * EACH) {
        const int64_t e = min(e0 + mine, all - 1), r = e / per_row, c = (e - r * per_row) * 4;
        const float *src = part + r * ld + c;
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = first; k < end; ++k) t += *(const f32x4 *)(src + k * copy);
        if constexpr (SLICES > 1) {
            __syncthreads();
            s[slice][mine] = t;
            __syncthreads();
            for (int q = 1; q < SLICES; ++q) t += slice == 0 ? s[q][mine] : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (slice || e0 + mine >= all) continue;
        if (l.labels && label_at(l, (int)r) < 0) t = f32x4{0.f, 0.f, 0.f, 0.f};
        O v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (O)(t[i] * f);
        O *dst = out + r * ldo + c;
        if (c + 4 <= cols) __builtin_memcpy(dst, v, sizeof v);
        else
            for (int i = 0; i < 3; ++i)
                if (c + i < cols) dst[i] = v[i];
    }
}

// ---- few rows -------------------------------------------------------------------------------------------------------
//
// Few rows are bound by reading w, and laying it out would read and write it once more.  `loss_few` reads it as it lies, whatever its distance and alignment: a wavefront takes sixteen classes at a
// time, its lanes' sixteen bytes being the matrix instruction's operand as they come, and x lies in LDS.  For the gradient it leaves
// the logits.  `loss_grad_few`, for the fewest rows, reads w once more: a thread owns a vector of columns and forms dw's rows and its
// part of dx in 32 bits.

constexpr int FEW_ROWS = 32, FEW_GRAD_ROWS = 8, FEW_AHEAD = 8, FEW_THREADS = 512;
template <typename T> constexpr int FEW_BATCH = MM_K<T> / 2 * FEW_AHEAD;   // k of a batch of accesses

// Rows 16 q + l % 16 of x in LDS, `chunk` columns at a time where not all of them fit: x[row][chunk + one chunk], zeros past d; then (largest,
// sum) of every wavefront and row.  part[row][workgroup]; logits[row][ldz], may be null.  chunk is a multiple of a batch.
template <typename T, int NR>
__global__ __launch_bounds__(FEW_THREADS) void loss_few(const T *__restrict__ x, int64_t ldx, const T *__restrict__ w, int64_t ldw, int64_t d, LossRows l,
                                                        int chunk, int passes, float *__restrict__ logits, int64_t ldz)
{
    typedef typename Mfma<T>::frag frag;
    constexpr int U = FEW_AHEAD, K = MM_K<T> / 2, V = MM_CHUNK<T>;         // K of an access
    constexpr bool EXACT = sizeof(T) == 4;
    extern __shared__ __align__(16) char lds[];
    T *xs = (T *)lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, l16 = lane & 15, quarter = lane >> 4, ld = chunk + V;
    const int k_end = (int)((d + K - 1) / K * K);
    int at[NR], label[NR];
    float m[NR], sum[NR];
#pragma unroll
    for (int q = 0; q < NR; ++q) {
        at[q] = min(16 * q + l16, l.n - 1) * ld + quarter * V;
        label[q] = label_at(l, 16 * q + l16);
        m[q] = MINUS_INF;
        sum[q] = 0.f;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int64_t v0 = (((int64_t)pass * gridDim.x + blockIdx.x) * waves + wave) * 16;
        const T *row = w + min(v0 + l16, (int64_t)l.classes - 1) * ldw;
        f32x4 acc[NR];
#pragma unroll
        for (int q = 0; q < NR; ++q) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto ask = [&](u32x4 (&raw)[U], int k0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = load_raw<T, true>(row, k0 + u * K + quarter * V, d);
        };
        auto use = [&](const u32x4 (&raw)[U], int k0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                frag b[NR];
#pragma unroll
                for (int q = 0; q < NR; ++q) b[q] = *(const frag *)(xs + at[q] + k0 + u * K);
#pragma unroll
                for (int e = 0; e < Mfma<T>::STEPS; ++e)
#pragma unroll
                    for (int q = 0; q < NR; ++q) acc[q] = Mfma<T>::step(__builtin_bit_cast(frag, raw[u]), b[q], e, acc[q]);
            }
        };
        for (int kc = 0; kc < k_end; kc += chunk) {
            const int end = min(chunk, k_end - kc);
            u32x4 raw0[U], raw1[U];
            ask(raw0, kc);                               // (on its way while x goes to LDS)
            if (pass == 0 || chunk < k_end) {
                __syncthreads();
                for (int e = threadIdx.x; e < l.n * (chunk / V); e += blockDim.x) {
                    const int r = e / (chunk / V), c = (e - r * (chunk / V)) * V;
                    *(u32x4 *)(xs + r * ld + c) = load_raw<T>(x + r * ldx, kc + c, d);
                }
                __syncthreads();
            }
            constexpr int BATCH = FEW_BATCH<T>;
            for (int k0 = 0; k0 < end; k0 += 2 * BATCH) {
                if (k0 + BATCH < end) ask(raw1, kc + k0 + BATCH);
                use(raw0, k0);
                if (k0 + 2 * BATCH < end) ask(raw0, kc + k0 + 2 * BATCH);
                if (k0 + BATCH < end) use(raw1, k0 + BATCH);
            }
        }
        // this lane: classes v0 + 4 quarter + r of rows 16 q + l16
        const int64_t first = v0 + 4 * quarter;
#pragma unroll
        for (int q = 0; q < NR; ++q) {
            const int j = 16 * q + l16;
            float top = m[q];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (first + r >= l.classes) acc[q][r] = MINUS_INF;
                else {
                    if (first + r == label[q]) l.picked[j] = acc[q][r];
                    if (logits && j < l.n) logits[j * ldz + first + r] = acc[q][r];
                }
                top = fmaxf(top, acc[q][r]);
            }
            const float shift = top == MINUS_INF ? 0.f : top;
            sum[q] *= exp_diff<EXACT>(m[q], shift);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[q] += exp_of<EXACT>(acc[q][r], shift);
            m[q] = top;
        }
    }
    // lanes of one row, then wavefronts
    __syncthreads();
    float2 *parts = (float2 *)lds;
#pragma unroll
    for (int q = 0; q < NR; ++q) {
        for (int o = 16; o <= 32; o <<= 1) {
            const float m2 = __shfl_xor(m[q], o), s2 = __shfl_xor(sum[q], o), top = fmaxf(m[q], m2);
            sum[q] = sum[q] * exp_diff<EXACT>(m[q], top) + s2 * exp_diff<EXACT>(m2, top);
            m[q] = top;
        }
        if (lane < 16) parts[wave * 16 * NR + 16 * q + lane] = make_float2(m[q], sum[q]);
    }
    __syncthreads();
    const int j = threadIdx.x;
    if (j >= l.n) return;
    float2 t = parts[j];
    for (int v = 1; v < waves; ++v) {
        const float2 y = parts[v * 16 * NR + j];
        const float top = fmaxf(t.x, y.x);
        t = make_float2(top, t.y * exp_diff<EXACT>(t.x, top) + y.y * exp_diff<EXACT>(y.x, top));
    }
    l.part[(int64_t)j * gridDim.x + blockIdx.x] = t;
}

// Workgroup (b, y): classes [b * each, ..), columns from y * 256 * VEC on.  part[b][row][ldp] is its share of dx.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void loss_grad_few(const T *__restrict__ x, int64_t ldx, const T *__restrict__ w, int64_t ldw, int64_t d, LossRows l, int each,
                                                     const float *__restrict__ logits, int64_t ldz, T *__restrict__ dw, int64_t lddw,
                                                     float *__restrict__ part, int64_t ldp)
{
    constexpr int V = Elem<T>::VEC, CHUNK = 64, AHEAD = 4;
    __shared__ float g[CHUNK][ROWS];
    __shared__ int labels[ROWS];
    const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * V;
    if (threadIdx.x < ROWS) labels[threadIdx.x] = label_at(l, threadIdx.x);
    __syncthreads();
    float xv[ROWS][V], sum[ROWS][V] = {};
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (labels[j] >= 0) load_vec(x + j * ldx, c, d, xv[j]);
        else
#pragma unroll
            for (int k = 0; k < V; ++k) xv[j][k] = 0.f;  // (such a row counts nowhere, whatever it holds)
    }
    const int64_t v0 = (int64_t)blockIdx.x * each, v1 = min((int64_t)l.classes, v0 + each);
    for (int64_t v = v0; v < v1; v += CHUNK) {
        __syncthreads();
        for (int e = threadIdx.x; e < CHUNK * ROWS; e += 256) {
            const int j = e / CHUNK, q = e % CHUNK;
            float p = 0.f;
            if (labels[j] >= 0 && v + q < v1) {
                const float weight = l.weight[j];
                p = expf(logits[j * ldz + v + q] - l.lse[j]) - (v + q == labels[j] ? 1.f : 0.f);
                p = weight != 0.f ? p * weight : 0.f;
            }
            g[q][j] = p;
        }
        __syncthreads();
        const int many = (int)min((int64_t)CHUNK, v1 - v);
        if (c < d)
            for (int q0 = 0; q0 < many; q0 += AHEAD) {
                u32x4 raw[AHEAD];
#pragma unroll
                for (int h = 0; h < AHEAD; ++h) raw[h] = load_raw<T, true>(w + (v + min(q0 + h, many - 1)) * ldw, c, d);
#pragma unroll
                for (int h = 0; h < AHEAD; ++h) {
                    if (q0 + h >= many) break;
                    float wv[V], out[V] = {};
                    unpack<T>(raw[h], wv);
#pragma unroll
                    for (int j = 0; j < ROWS; ++j) {
                        const float p = g[q0 + h][j];
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            sum[j][k] += p * wv[k];
                            out[k] += p * xv[j][k];
                        }
                    }
                    store_vec<T, true>(dw + (v + q0 + h) * lddw, c, d, out);
                }
            }
    }
    if (c >= d) return;
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (j < l.n)
#pragma unroll
            for (int k = 0; k < V; k += 4)
                *(f32x4 *)(part + ((int64_t)blockIdx.x * l.n + j) * ldp + c + k) = f32x4{sum[j][k], sum[j][k + 1], sum[j][k + 2], sum[j][k + 3]};
}

}  // namespace chicle_train
