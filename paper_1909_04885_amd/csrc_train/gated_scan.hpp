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
#include <type_traits>
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

constexpr int SCAN_ROWS = SCAN_KEPT, SCAN_WAVES = 4, SCAN_THREADS = 64 * SCAN_WAVES;
constexpr int SCAN_TILE = SCAN_ROWS * SCAN_WAVES;        // rows of a workgroup's tile
constexpr int SCAN_RUN = 16;                             // tiles of one column block whose products are added up before a state is handed on
template <typename T> constexpr int SCAN_V = 4 / (int)sizeof(T);          // columns of a lane
template <typename T> constexpr int SCAN_COLS = 64 * SCAN_V<T>;           // columns of a tile

typedef unsigned u32_at_2 __attribute__((aligned(2)));

// A lane's columns of a tile, counted from the tile's first: rows are given by uniform pointers to that one.  Lanes past the last column read
// some column that is there and store nothing.
template <typename T> struct ScanLane {
    int64_t first;                           // the tile's first column
    int e, left;                             // the lane's first column; columns from the tile's first to the last one, or the tile's
    bool full, odd;                          // all columns are there; the last one has no neighbour (16 bits)
    __device__ __forceinline__ ScanLane(int64_t block, int64_t d) : first(block * SCAN_COLS<T>), e((threadIdx.x & 63) * SCAN_V<T>)
    {
        left = d - first < SCAN_COLS<T> ? (int)(d - first) : SCAN_COLS<T>;
        full = left == SCAN_COLS<T>;
        odd = SCAN_V<T> == 2 && (left & 1);
    }
    // The lane's values of SCAN_ROWS rows: the last of `many` again in place of those that are not there.
    template <typename L> static __device__ __forceinline__ void each_row(int many, L load)
    {
        if (many == SCAN_ROWS) {
#pragma unroll
            for (int r = 0; r < SCAN_ROWS; ++r) load(r, 1);
        } else {
#pragma unroll
            for (int r = 0; r < SCAN_ROWS; ++r) load(r, r + 1 < many);
        }
    }
    __device__ __forceinline__ void load(const T *row, int64_t ld, int many, unsigned (&out)[SCAN_ROWS]) const
    {
        const T *p = row + first;
        if constexpr (SCAN_V<T> == 1) {
            const unsigned off = e < left ? e : left - 1;
            each_row(many, [&](int r, bool further) {
                out[r] = __builtin_nontemporal_load((const unsigned *)p + off);
                p += further ? ld : 0;
            });
        } else if (odd) {
            const unsigned off = e < left ? e : left - 1, next = e + 1 < left ? e + 1 : left - 1;
            each_row(many, [&](int r, bool further) {
                out[r] = ((const uint16_t *)p)[off] | (unsigned)((const uint16_t *)p)[next] << 16;
                p += further ? ld : 0;
            });
        } else {
            const unsigned off = e < left ? e : left - 2;
            each_row(many, [&](int r, bool further) {
                out[r] = __builtin_nontemporal_load((const u32_at_2 *)(p + off));
                p += further ? ld : 0;
            });
        }
    }
    static __device__ __forceinline__ void values(unsigned x, float *out)
    {
        if constexpr (sizeof(T) == 4) out[0] = __uint_as_float(x);
        else if constexpr (__is_same(T, bf16)) { out[0] = __uint_as_float(x << 16); out[1] = __uint_as_float(x & 0xffff0000u); }
        else {
            f16 v[2];
            __builtin_memcpy(v, &x, 4);
            out[0] = (float)v[0];
            out[1] = (float)v[1];
        }
    }
    // `row`: the tile's first column
    template <bool FULL> __device__ __forceinline__ void store(T *row, const float *in) const
    {
        if constexpr (SCAN_V<T> == 1) {
            if (FULL || e < left) __builtin_nontemporal_store((float)in[0], (float *)row + (unsigned)e);
        } else {
            T v[2] = {(T)in[0], (T)in[1]};
            unsigned x;
            __builtin_memcpy(&x, v, 4);
            if (FULL || e + 1 < left) __builtin_nontemporal_store(x, (u32_at_2 *)(row + (unsigned)e));
            else if (e < left) row[e] = v[0];
        }
    }
    // Row j of floats (of a null pointer: zeros).
    __device__ __forceinline__ void load_floats(const float *p, int64_t j, int64_t d, float *out) const
    {
        const float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < SCAN_V<T>; ++v) out[v] = p ? row[(unsigned)(e + v < left ? e + v : left - 1)] : 0.f;
    }
    __device__ __forceinline__ void store_floats(float *p, int64_t j, int64_t d, const float *in) const
    {
        float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < SCAN_V<T>; ++v)
            if (e + v < left) row[(unsigned)(e + v)] = in[v];
    }
};

// Rows of T, or packed ones: what is asked for of a row, in one register, and its values.
template <typename T, bool PACKED> struct ScanInput;
template <typename T> struct ScanInput<T, false> {
    const T *p;
    int64_t ld;
    __device__ __forceinline__ void load(int64_t row, int64_t, int many, const ScanLane<T> &at, unsigned (&out)[SCAN_ROWS]) const
    {
        at.load(p + row * ld, ld, many, out);
    }
    static __device__ __forceinline__ void values(unsigned x, float *out) { ScanLane<T>::values(x, out); }
};
template <typename T> struct ScanInput<T, true> {
    const int8_t *q;
    const uint8_t *scales;
    int64_t ld;
    __device__ __forceinline__ void load(int64_t row, int64_t d, int many, const ScanLane<T> &at, unsigned (&out)[SCAN_ROWS]) const
    {
        constexpr int V = SCAN_V<T>;
        const int64_t whole = (d + PACK_GROUP - 1) / PACK_GROUP * PACK_GROUP - at.first;
        const int left = whole < SCAN_COLS<T> ? (int)whole : SCAN_COLS<T>;
        const unsigned off = at.e < left ? at.e : left - V;
        const int8_t *p = q + row * ld + at.first;
        const uint8_t *scale = scales + row * (ld / PACK_GROUP) + at.first / PACK_GROUP;
        at.each_row(many, [&](int r, bool further) {
            if constexpr (V == 1) out[r] = ((const uint8_t *)p)[off];
            else out[r] = *(const uint16_t *)(p + off);
            out[r] |= (unsigned)scale[off / PACK_GROUP] << 16;
            p += further ? ld : 0;
            scale += further ? ld / PACK_GROUP : 0;
        });
    }
    static __device__ __forceinline__ void values(unsigned x, float *out)
    {
        const float step = pack_step(x >> 16);
#pragma unroll
        for (int v = 0; v < SCAN_V<T>; ++v) out[v] = (float)(int8_t)(x >> (8 * v)) * step;
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
    // what workgroups hand on; null where there is one tile in a column block
    unsigned *ticket;
    unsigned long long *products, *handed;
    unsigned tiles, blocks;                  // tiles of a column block, column blocks
};

constexpr unsigned long long SCAN_NOTHING = ~0ull;       // what no product is: its lower half is no NaN of these bits

__global__ __launch_bounds__(256) static void scan_begin(unsigned *ticket, unsigned long long *words, int64_t count)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) words[i] = SCAN_NOTHING;
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
}

// What rows do to what comes into them: x becomes a x + b; a = 0 where it does not get through, whatever it is.
struct ScanProduct {
    float a, b;
    __device__ __forceinline__ float of(float x) const { return a == 0.f ? b : fmaf(a, x, b); }
    __device__ __forceinline__ unsigned long long word() const
    {
        const unsigned lo = a == a ? __float_as_uint(a) : 0x7fc00000u;
        return (unsigned long long)__float_as_uint(b) << 32 | lo;
    }
    static __device__ __forceinline__ ScanProduct from(unsigned long long w) { return {__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32))}; }
};

__device__ __forceinline__ unsigned long long scan_look(const unsigned long long *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void scan_tell(unsigned long long *p, unsigned long long w) { __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ unsigned long long scan_wait(const unsigned long long *p, unsigned long long w)
{
    while (w == SCAN_NOTHING) {
        __builtin_amdgcn_s_sleep(1);
        w = scan_look(p);
    }
    return w;
}

// What the workgroup knows of its rows: where sequences begin and end among them (a sequence's number, or -1), which rows belong to none, and the
// tile that the sequence of the first row (backwards: of the last one) begins (ends) in.
struct ScanMarks {
    int start[SCAN_TILE], end[SCAN_TILE];
    unsigned from, to;
};

// How many of the offsets are at most t, by the whole wavefront.
__device__ __forceinline__ int64_t scan_count(const ScanOrder &o, int64_t t)
{
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = o.count + 1;
    while (lo < hi) {                                    // (the distance shrinks, whatever the offsets are)
        const int64_t step = (hi - lo + 63) >> 6, j = lo + (lane + 1) * step - 1;
        const int many = __popcll(__ballot(j < hi && o.at(j < hi ? j : lo) <= t));
        const int64_t next = lo + (many + 1) * step - 1;
        lo += many * step;
        hi = next < hi ? next : hi;
        lo = lo < hi ? lo : hi;
    }
    return lo;
}

// Marks the tile's rows.  `empty(j)` is called by whole wavefronts for the sequences without rows that lie in the tile.
template <typename F>
__device__ __forceinline__ void scan_mark(const ScanOrder &o, ScanMarks &m, unsigned tile, unsigned tiles, unsigned block, int *flags, F empty)
{
    const int64_t t0 = (int64_t)tile * SCAN_TILE, t1 = t0 + SCAN_TILE;
    const bool last = tile + 1 == tiles;
    for (int i = threadIdx.x; i < SCAN_TILE; i += SCAN_THREADS) m.start[i] = m.end[i] = -1;
    if (threadIdx.x == 0) m.from = m.to = tile;
    const int64_t first = scan_count(o, t0 - 1);         // offsets below the tile's first row
    __syncthreads();
    bool wrong = false, more = true;
    for (int64_t j0 = first > 0 ? first - 1 : 0; more && j0 < o.count; j0 += SCAN_THREADS) {
        const int64_t j = j0 + threadIdx.x;
        bool none = false;
        more = false;
        if (j < o.count) {
            const int64_t lo = o.at(j), hi = o.at(j + 1);
            more = lo < t1 || last;
            if (lo < 0 || hi < lo || hi > o.n) wrong = true;
            else if (lo == hi) none = lo >= t0 && more;
            else {
                if (lo >= t0 && lo < t1) m.start[lo - t0] = (int)j;
                if (hi > t0 && hi <= t1) m.end[hi - 1 - t0] = (int)j;
                if (lo < t0 && hi > t0) m.from = (unsigned)(lo / SCAN_TILE);
                if (lo < t1 && hi > t1) m.to = (unsigned)((hi - 1) / SCAN_TILE);
            }
        }
        more = __any(more);                              // (offsets ascend: the lanes in front decide)
        for (unsigned long long left = __ballot(none); left; left &= left - 1) empty(j0 + (threadIdx.x & ~63) + __builtin_ctzll(left));
    }
    if (block == 0)                                      // every offset is looked at by some tile
        for (int64_t j = (int64_t)tile * SCAN_THREADS + threadIdx.x; j < o.count; j += (int64_t)tiles * SCAN_THREADS) {
            const int64_t lo = o.at(j), hi = o.at(j + 1);
            wrong |= lo < 0 || hi < lo || hi > o.n;
        }
    if (wrong && flags) atomicOr(flags, FLAG_OFFSETS);
}

// The wavefront's 32 rows in three masks.
struct ScanRows {
    unsigned starts, ends, none;
    __device__ __forceinline__ ScanRows(const ScanOrder &o, const ScanMarks &m, int64_t t, int row0)
    {
        const int lane = threadIdx.x & 63, r = row0 + (lane & 31);
        const int64_t lo = o.at(0), hi = o.at(o.count), row = t + (lane & 31);
        starts = (unsigned)__ballot(m.start[r] >= 0);
        ends = (unsigned)__ballot(m.end[r] >= 0);
        none = (unsigned)__ballot(row < lo || row >= hi || row >= o.n);
    }
};

// What comes into the q-th tile of a column block, in the order in which tiles are taken, from tile `from` on, whose product lets nothing through; hands
// on what comes out.  By one wavefront.
//
// Tiles are taken in the order of tickets, those of all column blocks in turn: whoever waits does so for tiles with earlier tickets, whose
// workgroups have begun and, first of all, tell their products without waiting.  So every wait ends.  What is added up, and in which order, follows
// from the offsets alone.  A word is told whole, and says by itself whether it has been.
template <typename T, bool PACKED>
__device__ __forceinline__ void scan_hand(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned from, const ScanProduct (&own)[SCAN_V<T>], float (&x)[SCAN_V<T>])
{
    constexpr int V = SCAN_V<T>, AHEAD = 8;
    const int lane = threadIdx.x & 63;
    const int64_t line = (int64_t)a.blocks * SCAN_COLS<T>, at = (int64_t)block * SCAN_COLS<T> + lane;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        scan_tell(a.products + q * line + at + v * 64, own[v].word());
        x[v] = 0.f;
    }
    const unsigned run = q / SCAN_RUN;
    if (from < q) {
        if (from < run * SCAN_RUN) {
            from = run * SCAN_RUN;
            const unsigned long long *p = a.handed + (int64_t)(run - 1) * line + at;
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = __uint_as_float((unsigned)scan_wait(p + v * 64, scan_look(p + v * 64)));
        }
        for (unsigned i = from; i < q; i += AHEAD) {
            const unsigned long long *p = a.products + i * line + at;
            unsigned long long w[AHEAD][V];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) w[k][v] = i + k < q ? scan_look(p + k * line + v * 64) : 0;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k < q)
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = ScanProduct::from(scan_wait(p + k * line + v * 64, w[k][v])).of(x[v]);
        }
    }
    if (q % SCAN_RUN == SCAN_RUN - 1)
#pragma unroll
        for (int v = 0; v < V; ++v) scan_tell(a.handed + (int64_t)run * line + at + v * 64, __float_as_uint(own[v].of(x[v])));
}

// A sequence's number, the same in all lanes.
__device__ __forceinline__ int64_t scan_number(int j) { return __builtin_amdgcn_readfirstlane(j); }

// What the workgroup's tile is: tickets give tiles in the order in which workgroups begin.
template <typename T, bool PACKED>
__device__ __forceinline__ void scan_unit(const Scan<T, PACKED> &a, unsigned &q, unsigned &block)
{
    __shared__ unsigned unit;
    if (a.ticket) {
        if (threadIdx.x == 0) unit = atomicAdd(a.ticket, 1u);
        __syncthreads();
        q = __builtin_amdgcn_readfirstlane(unit) / a.blocks;
        block = __builtin_amdgcn_readfirstlane(unit) - q * a.blocks;
    } else {
        q = 0;
        block = blockIdx.x;
    }
}

// Rows are worked on four at a time: without an end to it the compiler begins all of them, more than there are registers for.
__device__ __forceinline__ void scan_four(int r)
{
    if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
}

// The same value, of which the compiler does not know that it is: what an earlier pass worked out of it is worked out again instead of being kept.
template <typename X> __device__ __forceinline__ void scan_anew(X &x) { asm volatile("" : "+v"(x)); }

// f(whether sequences begin or end among the rows, or rows belong to none)
template <typename F>
__device__ __forceinline__ void scan_rows(unsigned special, F f)
{
    if (special) f(std::true_type());
    else f(std::false_type());
}

template <typename T, bool PACKED>
__global__ __launch_bounds__(SCAN_THREADS, 2) void scan_forward(const Scan<T, PACKED> a)
{
    constexpr int V = SCAN_V<T>;
    __shared__ ScanMarks marks;
    __shared__ ScanProduct products[SCAN_WAVES][V][64];
    __shared__ float into[V][64];
    unsigned q, block;
    scan_unit(a, q, block);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const ScanLane<T> at(block, a.d);
    const int64_t n = a.order.n, t0 = (int64_t)q * SCAN_TILE + wave * SCAN_ROWS;
    const int many = (int)(n - t0 < SCAN_ROWS ? n - t0 < 0 ? 0 : n - t0 : SCAN_ROWS);
    unsigned fs[SCAN_ROWS], us[SCAN_ROWS];
    if (many > 0) {
        at.load(a.f + t0 * a.ldf, a.ldf, many, fs);
        a.u.load(t0, a.d, many, at, us);
    }
    scan_mark(a.order, marks, q, a.tiles, block, a.flags, [&](int64_t j) {
        float h[V];
        if (!a.last) return;
        at.load_floats(a.h0, j, a.d, h);
        at.store_floats(a.last, j, a.d, h);
    });
    __syncthreads();
    const ScanRows rows(a.order, marks, t0, wave * SCAN_ROWS);
    auto first_state = [&](int r, float *h) {
        at.load_floats(a.h0, scan_number(marks.start[wave * SCAN_ROWS + r]), a.d, h);
    };
    float g[SCAN_ROWS][V];
    if (many > 0)
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r) {
            float f[V];
            at.values(fs[r], f);
#pragma unroll
            for (int v = 0; v < V; ++v) g[r][v] = gate_of(f[v]);
            scan_four(r);
        }
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    if (many > 0)
        scan_rows(rows.starts | rows.none, [&](auto special) {
#pragma unroll
            for (int r = 0; r < SCAN_ROWS; ++r) {
                if constexpr (decltype(special)::value) {
                    if (rows.none >> r & 1) {
#pragma unroll
                        for (int v = 0; v < V; ++v) p[v] = {0.f, 0.f};
                        continue;
                    }
                    if (rows.starts >> r & 1) {
                        float h[V];
                        first_state(r, h);
#pragma unroll
                        for (int v = 0; v < V; ++v) p[v] = {0.f, h[v]};
                    }
                }
                float u[V];
                a.u.values(us[r], u);
#pragma unroll
                for (int v = 0; v < V; ++v) p[v] = {gate_through(g[r][v], p[v].a), gate_step(g[r][v], p[v].b, u[v])};
            }
        });
#pragma unroll
    for (int v = 0; v < V; ++v) products[wave][v][lane] = p[v];
    __syncthreads();
    if (wave == 0) {
        float x[V] = {};
        if (a.ticket) {
            ScanProduct own[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                own[v] = p[v];
#pragma unroll
                for (int w = 1; w < SCAN_WAVES; ++w) {
                    const ScanProduct next = products[w][v][lane];
                    own[v] = {next.a == 0.f ? 0.f : own[v].a * next.a, next.of(own[v].b)};
                }
            }
            scan_hand(a, q, block, marks.from, own, x);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) into[v][lane] = x[v];
    }
    __syncthreads();
    if (many == 0) return;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {
        scan_anew(us[r]);
#pragma unroll
        for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    }
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = into[v][lane];
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = products[w][v][lane].of(h[v]);
    T *y = a.y + t0 * a.ldy + at.first;
    scan_rows(rows.starts | rows.ends | rows.none | !at.full, [&](auto special) {
        constexpr bool SPECIAL = decltype(special)::value;
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r) {
            const bool none = SPECIAL && (rows.none >> r & 1);
            if (SPECIAL && r >= many) break;
            if (SPECIAL && none) {
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = 0.f;
            }
            if (SPECIAL && (rows.starts >> r & 1)) first_state(r, h);
            if (r == 0 && a.states) at.store_floats(a.states, t0 / SCAN_KEPT, a.d, h);
            if (!none) {
                float u[V];
                a.u.values(us[r], u);
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = gate_step(g[r][v], h[v], u[v]);
            }
            at.template store<!SPECIAL>(y, h);
            y += a.ldy;
            if (SPECIAL && (rows.ends >> r & 1) && a.last) at.store_floats(a.last, scan_number(marks.end[wave * SCAN_ROWS + r]), a.d, h);
        }
    });
}

template <typename T, bool PACKED>
__global__ __launch_bounds__(SCAN_THREADS, 2) void scan_backward(const Scan<T, PACKED> a)
{
    constexpr int V = SCAN_V<T>;
    __shared__ ScanMarks marks;
    __shared__ ScanProduct products[SCAN_WAVES][V][64];
    __shared__ float into[V][64];
    unsigned q, block;
    scan_unit(a, q, block);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const ScanLane<T> at(block, a.d);
    const unsigned tile = a.tiles - 1 - q;
    const int64_t n = a.order.n, t0 = (int64_t)tile * SCAN_TILE + wave * SCAN_ROWS;
    const int many = (int)(n - t0 < SCAN_ROWS ? n - t0 < 0 ? 0 : n - t0 : SCAN_ROWS);
    unsigned fs[SCAN_ROWS], us[SCAN_ROWS], dys[SCAN_ROWS];
    float h[V] = {};
    if (many > 0) {
        at.load(a.f + t0 * a.ldf, a.ldf, many, fs);
        a.u.load(t0, a.d, many, at, us);
        at.load_floats(a.states, t0 / SCAN_KEPT, a.d, h);
        at.load(a.dy + t0 * a.lddy, a.lddy, many, dys);
    }
    scan_mark(a.order, marks, tile, a.tiles, block, a.flags, [&](int64_t j) {
        float x[V];
        if (!a.dh0) return;
        at.load_floats(a.dlast, j, a.d, x);
        at.store_floats(a.dh0, j, a.d, x);
    });
    __syncthreads();
    const ScanRows rows(a.order, marks, t0, wave * SCAN_ROWS);
    auto last_gradient = [&](int r, float *x) {
        at.load_floats(a.dlast, scan_number(marks.end[wave * SCAN_ROWS + r]), a.d, x);
    };
    float g[SCAN_ROWS][V], wide[SCAN_ROWS][V];           // gates, and h_{t-1} - u_t
    if (many > 0)
        scan_rows(rows.starts, [&](auto special) {
#pragma unroll
            for (int r = 0; r < SCAN_ROWS; ++r) {
                float f[V], u[V];
                if constexpr (decltype(special)::value)
                    if (rows.starts >> r & 1) at.load_floats(a.h0, scan_number(marks.start[wave * SCAN_ROWS + r]), a.d, h);
                at.values(fs[r], f);
                a.u.values(us[r], u);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    g[r][v] = gate_of(f[v]);
                    wide[r][v] = h[v] - u[v];
                    h[v] = gate_step(g[r][v], h[v], u[v]);
                }
                scan_four(r);
            }
        });
    if (many > 0)
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    // x: what goes from a row to the one before, a G
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    if (many > 0)
        scan_rows(rows.ends | rows.none, [&](auto special) {
#pragma unroll
            for (int r = SCAN_ROWS - 1; r >= 0; --r) {
                if constexpr (decltype(special)::value) {
                    if (rows.none >> r & 1) {
#pragma unroll
                        for (int v = 0; v < V; ++v) p[v] = {0.f, 0.f};
                        continue;
                    }
                    if (rows.ends >> r & 1) {
                        float x[V];
                        last_gradient(r, x);
#pragma unroll
                        for (int v = 0; v < V; ++v) p[v] = {0.f, x[v]};
                    }
                }
                float dy[V];
                at.values(dys[r], dy);
#pragma unroll
                for (int v = 0; v < V; ++v) p[v] = {gate_through(g[r][v], p[v].a), gate_through(g[r][v], p[v].b + dy[v])};
                scan_four(r + 3);
            }
        });
#pragma unroll
    for (int v = 0; v < V; ++v) products[wave][v][lane] = p[v];
    __syncthreads();
    if (wave == SCAN_WAVES - 1) {
        float x[V] = {};
        if (a.ticket) {
            ScanProduct own[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                own[v] = p[v];
#pragma unroll
                for (int w = SCAN_WAVES - 2; w >= 0; --w) {
                    const ScanProduct next = products[w][v][lane];
                    own[v] = {next.a == 0.f ? 0.f : own[v].a * next.a, next.of(own[v].b)};
                }
            }
            scan_hand(a, q, block, a.tiles - 1 - marks.to, own, x);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) into[v][lane] = x[v];
    }
    __syncthreads();
    if (many == 0) return;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {
        scan_anew(dys[r]);
#pragma unroll
        for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    }
    float x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = into[v][lane];
    for (int w = SCAN_WAVES - 1; w > wave; --w)
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = products[w][v][lane].of(x[v]);
    T *df_row = a.df + (t0 + many - 1) * a.lddf + at.first, *du_row = a.du + (t0 + many - 1) * a.lddu + at.first;
    scan_rows(rows.starts | rows.ends | rows.none | !at.full, [&](auto special) {
        constexpr bool SPECIAL = decltype(special)::value;
#pragma unroll
        for (int r = SCAN_ROWS - 1; r >= 0; --r) {
            if (SPECIAL && r >= many) continue;
            float df[V] = {}, du[V] = {};
            if (SPECIAL && (rows.none >> r & 1)) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = 0.f;
            } else {
                if (SPECIAL && (rows.ends >> r & 1)) last_gradient(r, x);
                float dy[V];
                at.values(dys[r], dy);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float y = x[v] + dy[v];
                    df[v] = gate_slope(g[r][v], y * wide[r][v]);
                    du[v] = gate_into(g[r][v], y);
                    x[v] = gate_through(g[r][v], y);
                }
            }
            at.template store<!SPECIAL>(df_row, df);
            at.template store<!SPECIAL>(du_row, du);
            df_row -= a.lddf;
            du_row -= a.lddu;
            scan_four(r + 3);
            if (SPECIAL && (rows.starts >> r & 1) && a.dh0) at.store_floats(a.dh0, scan_number(marks.start[wave * SCAN_ROWS + r]), a.d, x);
        }
    });
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
