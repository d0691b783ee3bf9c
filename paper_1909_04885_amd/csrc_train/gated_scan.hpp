// A gated linear recurrence over the rows of sequences, its gradients, and its form for one row of every sequence.
//
//   a_t = 1 / (1 + exp(-f_t)),  c_t = 1 - a_t,  h_t = a_t h_{t-1} + c_t u_t,  y_t = h_t, from the sequence's first state or from 0
//   G_t = dy_t + a_{t+1} G_{t+1}, the last row's with the gradient of the last state:
//   du_t = c_t G_t,  df_t = G_t (h_{t-1} - u_t) a_t c_t,  dh0 = a_first G_first
//
// Of a gate, the smaller share is worked out, s = e / (1 + e) with e = exp(-|f|), the other one is 1 - s: neither loses what is small.  Where
// e is no 32-bit number (beyond +-104) a gate is closed, s = 0, and what it keeps out counts nowhere, whatever it holds.
//
// States are 32-bit floats.  A workgroup has a tile of SCAN_TILE rows, a wavefront SCAN_ROWS of them, a lane SCAN_V columns, held in registers and
// read once.  What the rows of a wavefront do to the state that comes into them is a product and a sum; those of the tile are joined in LDS, and tiles
// hand on what comes out of them (scan_hand).  The forward pass leaves the state that enters every SCAN_KEPT-th row; the gradient works out those
// between again from the tile's first, and goes through the tiles from the last one.
#pragma once
#include <type_traits>
#include "elements.hpp"
#include "packed.hpp"

namespace chicle_train {

constexpr int SCAN_KEPT = 32;

// s with the sign of f.
__device__ __forceinline__ float gate_of(float f)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(f));
    return copysignf(e * __builtin_amdgcn_rcpf(1.f + e), f);
}

struct GateShares { float a, c; };
__device__ __forceinline__ GateShares gate_shares(float g)
{
    const float s = fabsf(g), more = 1.f - s;
    return signbit(g) ? GateShares{s, more} : GateShares{more, s};
}

// A share of x.  CLOSED: none of it where the share is none, whatever x is.
template <bool CLOSED> __device__ __forceinline__ float share_of(float share, float x) { return CLOSED && share == 0.f ? 0.f : share * x; }
// a h + b
template <bool CLOSED> __device__ __forceinline__ float gate_step(float a, float h, float b) { return CLOSED && a == 0.f ? b : fmaf(a, h, b); }

constexpr int SCAN_ROWS = SCAN_KEPT, SCAN_WAVES = 4, SCAN_THREADS = 64 * SCAN_WAVES;
constexpr int SCAN_TILE = SCAN_ROWS * SCAN_WAVES;        // rows of a workgroup's tile
constexpr int SCAN_FORWARD_HELD = 4, SCAN_BACKWARD_HELD = 3;            // workgroups of a compute unit, as registers allow
constexpr int SCAN_GROUP = 8, SCAN_RUN = 64;             // tiles whose products are joined, and tiles from one state that is handed on to the next
// Columns of a lane: forward two of 16 bits; backward, where a row takes four registers a column, one.
template <typename T, bool BACKWARD> constexpr int SCAN_V = 1;

constexpr int SCAN_TICKET = 32;                          // places from one column block's ticket to the next: lines of their own

typedef unsigned u32_at_2 __attribute__((aligned(2)));

// A lane's columns of a tile, counted from the tile's first: rows are given by uniform pointers to that one.  Lanes past the last column read
// some column that is there and store nothing.
template <typename T, int V> struct ScanLane {
    static constexpr int COLS = 64 * V;
    typedef typename std::conditional<V * sizeof(T) == 4, unsigned, uint16_t>::type word;
    int64_t first;                           // the tile's first column
    int e, left;                             // the lane's first column; columns from the tile's first to the last one, or the tile's
    bool full, odd;                          // all columns are there; the last one has no neighbour (16 bits)
    __device__ __forceinline__ ScanLane(int64_t block, int64_t d) : first(block * COLS), e((threadIdx.x & 63) * V)
    {
        left = d - first < COLS ? (int)(d - first) : COLS;
        full = left == COLS;
        odd = V == 2 && (left & 1);
    }
    // The lane's values of SCAN_ROWS rows: the last of `many` again in place of those that are not there.
    template <typename L> static __device__ __forceinline__ void each_row(int many, L load)
    {
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r) {
            asm volatile("" : "+s"(many));               // (one row's pointer after the other: all of them at once are too many scalars)
            load(r, r + 1 < many);
        }
    }
    __device__ __forceinline__ void load(const T *row, int64_t ld, int many, unsigned (&out)[SCAN_ROWS]) const
    {
        const T *p = row + first;
        if constexpr (V == 1) {
            const unsigned off = e < left ? e : left - 1;
            each_row(many, [&](int r, bool further) {
                out[r] = __builtin_nontemporal_load((const word *)p + off);
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
        else if constexpr (__is_same(T, bf16)) {
            out[0] = __uint_as_float(x << 16);
            if constexpr (V == 2) out[1] = __uint_as_float(x & 0xffff0000u);
        } else {
            f16 v[2];
            __builtin_memcpy(v, &x, 4);
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = (float)v[i];
        }
    }
    __device__ __forceinline__ bool here() const { return e < left; }
    // `row`: the tile's first column; only lanes that have one
    __device__ __forceinline__ void store(T *row, const float *in) const { __builtin_nontemporal_store((T)in[0], row + (unsigned)e); }
    // Row j of floats (of a null pointer: zeros).
    __device__ __forceinline__ void load_floats(const float *p, int64_t j, int64_t d, float *out) const
    {
        const float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < V; ++v) out[v] = p ? row[(unsigned)(e + v < left ? e + v : left - 1)] : 0.f;
    }
    __device__ __forceinline__ void store_floats(float *p, int64_t j, int64_t d, const float *in) const
    {
        float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (e + v < left) row[(unsigned)(e + v)] = in[v];
    }
};

// The second input's rows, of T or packed: what a lane asks for of SCAN_ROWS of them, and its values.
template <typename T, bool PACKED> struct ScanInput;
template <typename T> struct ScanInput<T, false> {
    struct Raw { unsigned x[SCAN_ROWS]; };
    const T *p;
    int64_t ld;
    template <int V> __device__ __forceinline__ void load(int64_t row, int64_t, int many, const ScanLane<T, V> &at, Raw &out) const
    {
        at.load(p + row * ld, ld, many, out.x);
    }
    template <int V> static __device__ __forceinline__ void values(const Raw &raw, int r, float (&out)[V]) { ScanLane<T, V>::values(raw.x[r], out); }
};
template <typename T> struct ScanInput<T, true> {
    struct Raw { unsigned x[SCAN_ROWS], step; };         // step: of row lane / 2 and, of the tile's two groups, lane % 2
    const int8_t *q;
    const uint8_t *scales;
    int64_t ld;
    template <int V> __device__ __forceinline__ void load(int64_t row, int64_t d, int many, const ScanLane<T, V> &at, Raw &out) const
    {
        static_assert(V == 1 && SCAN_ROWS == 32 && PACK_GROUP == 32, "a lane for every scale");
        const int64_t whole = (d + PACK_GROUP - 1) / PACK_GROUP * PACK_GROUP - at.first;
        const int left = whole < at.COLS ? (int)whole : at.COLS, lane = threadIdx.x & 63;
        const unsigned off = at.e < left ? at.e : left - 1;
        const int which = lane >> 1 < many ? lane >> 1 : many > 0 ? many - 1 : 0;
        out.step = scales[(row + which) * (ld / PACK_GROUP) + at.first / PACK_GROUP + ((lane & 1) * PACK_GROUP < left ? lane & 1 : 0)];
        const uint8_t *p = (const uint8_t *)q + row * ld + at.first;
        at.each_row(many, [&](int r, bool further) {
            out.x[r] = __builtin_nontemporal_load(p + off);
            p += further ? ld : 0;
        });
    }
    template <int V> static __device__ __forceinline__ void values(const Raw &raw, int r, float (&out)[V])
    {
        const int from = 2 * r + ((threadIdx.x & 63) >> 5);
        out[0] = (float)(int8_t)raw.x[r] * pack_step((unsigned)__builtin_amdgcn_ds_bpermute(from * 4, (int)raw.step));
    }
};

// Where sequences begin: sequence j has the rows from at(j) to at(j + 1).
struct ScanOrder {
    const void *offsets;                     // null: one sequence of all rows
    int wide;
    int64_t count, n;
    __device__ __forceinline__ int64_t at(int64_t j) const { return offsets ? index_at(offsets, wide, j) : j == 0 ? 0 : n; }
    // The same for a j that all lanes have in common: scalar loads, which do not wait behind the rows' loads.
    __device__ __forceinline__ int64_t common(int64_t j) const
    {
        if (!offsets) return j == 0 ? 0 : n;
        if (wide) return ((const __attribute__((address_space(4))) int64_t *)offsets)[j];
        return ((const __attribute__((address_space(4))) int32_t *)offsets)[j];
    }
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
    unsigned *tickets;
    unsigned long long *products, *groups, *handed;
    unsigned tiles, blocks;                  // tiles of a column block, column blocks
};

constexpr unsigned long long SCAN_NOTHING = ~0ull;       // what no product is: its lower half is no NaN of these bits

__global__ __launch_bounds__(256) static void scan_begin(unsigned *tickets, unsigned blocks, unsigned long long *words, int64_t count)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        words[i] = SCAN_NOTHING;
        if (i < blocks) tickets[i * SCAN_TICKET] = 0;    // (there are more words than column blocks)
    }
}

// What rows do to what comes into them: x becomes a x + b; where a = 0 it does not get through, whatever it is.
struct ScanProduct {
    float a, b;
    __device__ __forceinline__ float of(float x) const { return gate_step<true>(a, x, b); }
    // What the rows do after `before`.
    __device__ __forceinline__ ScanProduct after(const ScanProduct &before) const { return {share_of<true>(a, before.a), of(before.b)}; }
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

// How many of the offsets are at most t.  (In 32 bits, which is enough: hipcc 7.2 has been seen to take the condition of one choice between uniform
// 64-bit numbers for that of the next.)
__device__ __forceinline__ unsigned scan_count(const ScanOrder &o, int64_t t)
{
    unsigned lo = 0, hi = (unsigned)o.count + 1;
    while (lo < hi) {                                    // (the distance shrinks, whatever the offsets are)
        const unsigned step = (hi - lo + 3) >> 2;
        unsigned many = 0;
#pragma unroll
        for (int k = 1; k <= 4; ++k) {
            const unsigned j = lo + k * step - 1;
            if (j < hi && o.common(j) <= t) ++many;
        }
        const unsigned next = lo + (many + 1) * step - 1;
        lo = min(lo + many * step, hi);
        hi = min(next, hi);
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
    const unsigned first = scan_count(o, t0 - 1);        // offsets below the tile's first row
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
        const int64_t lo = o.common(0), hi = o.common(o.count), row = t + (lane & 31);
        starts = (unsigned)__ballot(m.start[r] >= 0);
        ends = (unsigned)__ballot(m.end[r] >= 0);
        none = (unsigned)__ballot(row < lo || row >= hi || row >= o.n);
    }
};

// What comes into the q-th tile of a column block, in the order in which tiles are taken, from tile `from` on, whose product lets nothing through
// (from = q: nothing comes in, the tile's own lets nothing through); tells what others need.  By one wavefront.
//
// A tile tells its product; the last one of SCAN_GROUP tiles tells theirs, joined; the last one of SCAN_RUN tiles hands on the state that comes out.  So a
// tile reads at most SCAN_GROUP - 1 products, those of as many groups and a state, and a state goes through a long sequence in steps of SCAN_RUN
// tiles, everything else of which has been joined by then.
//
// Tiles are taken in the order of their column block's tickets: whoever waits does so for tiles with earlier tickets, whose workgroups have begun.  These tell their products without waiting, groups once the products of the group are told, and states after all that is before them.
// So every wait ends.  What is joined, and in which order, follows from the offsets alone.  A word is told whole, and says by itself whether it
// has been.
template <int V>
__device__ __forceinline__ void scan_join(const unsigned long long *words, int64_t line, unsigned from, unsigned to, ScanProduct (&x)[V])
{
    constexpr int AHEAD = SCAN_GROUP - 1;
    for (unsigned i = from; i < to; i += AHEAD) {
        const unsigned long long *p = words + i * line;
        unsigned long long w[AHEAD][V];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) w[k][v] = i + k < to ? scan_look(p + k * line + v * 64) : 0;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i + k < to)
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = ScanProduct::from(scan_wait(p + k * line + v * 64, w[k][v])).after(x[v]);
    }
}

template <typename T, bool PACKED, int V>
__device__ __forceinline__ void scan_hand(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned from, const ScanProduct (&own)[V], float (&x)[V])
{
    const int64_t line = (int64_t)a.blocks * 64 * V, at = (int64_t)block * 64 * V + (threadIdx.x & 63);
    const unsigned group = q / SCAN_GROUP, run = q / SCAN_RUN;
    ScanProduct near[V], far[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        scan_tell(a.products + q * line + at + v * 64, own[v].word());
        near[v] = far[v] = {1.f, 0.f};
        x[v] = 0.f;
    }
    scan_join<V>(a.products + at, line, from > group * SCAN_GROUP ? from : group * SCAN_GROUP, q, near);
    if (q % SCAN_GROUP == SCAN_GROUP - 1)
#pragma unroll
        for (int v = 0; v < V; ++v) scan_tell(a.groups + group * line + at + v * 64, own[v].after(near[v]).word());
    if (from < group * SCAN_GROUP) {
        const unsigned first = run * (SCAN_RUN / SCAN_GROUP);
        scan_join<V>(a.groups + at, line, from / SCAN_GROUP > first ? from / SCAN_GROUP : first, group, far);
        if (from < run * SCAN_RUN) {
            const unsigned long long *p = a.handed + (int64_t)(run - 1) * line + at;
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = __uint_as_float((unsigned)scan_wait(p + v * 64, scan_look(p + v * 64)));
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        x[v] = near[v].after(far[v]).of(x[v]);
        if (q % SCAN_RUN == SCAN_RUN - 1) scan_tell(a.handed + (int64_t)run * line + at + v * 64, __float_as_uint(own[v].of(x[v])));
    }
}

// A sequence's number, the same in all lanes.
__device__ __forceinline__ int64_t scan_number(int j) { return __builtin_amdgcn_readfirstlane(j); }

// What the workgroup's tile is: tickets, those of each column block for themselves, give tiles in the order in which workgroups begin.
template <typename S> __device__ __forceinline__ unsigned scan_tile(const S &a, unsigned block)
{
    __shared__ unsigned tile;
    if (!a.tickets) return 0;
    if (threadIdx.x == 0) tile = atomicAdd(a.tickets + block * SCAN_TICKET, 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(tile);
}

// What the wavefronts of a workgroup tell one another.
template <int V> struct ScanShared {
    ScanMarks marks;
    ScanProduct products[SCAN_WAVES][V][64];
    float into[V][64];
};

// States or gradients of sequences that begin or end among the wavefront's rows, each in the place of its row: a lane's own, read and written by no other.
template <int V> struct ScanEdges {
    float place[SCAN_ROWS][V][64];
    __device__ __forceinline__ void get(int r, float (&x)[V]) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = place[r][v][threadIdx.x & 63];
    }
    __device__ __forceinline__ void put(int r, const float (&x)[V])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) place[r][v][threadIdx.x & 63] = x[v];
    }
    // Fetches them for the rows of `which`, whose sequences `numbers` has; zeros of a null pointer.
    template <typename L> __device__ __forceinline__ void fetch(unsigned which, const int *numbers, const float *from, int64_t d, const L &at)
    {
        constexpr int AHEAD = 4;
        while (which) {
            float x[AHEAD][V];
            unsigned left = which;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int r = left ? __builtin_ctz(left) : 0;
                if (left) at.load_floats(from, scan_number(numbers[r]), d, x[k]);
                left &= left - 1;
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (which) put(__builtin_ctz(which), x[k]);
                which &= which - 1;
            }
        }
    }
    template <typename L> __device__ __forceinline__ void store(unsigned which, const int *numbers, float *to, int64_t d, const L &at) const
    {
        for (; which; which &= which - 1) {
            const int r = __builtin_ctz(which);
            float x[V];
            get(r, x);
            at.store_floats(to, scan_number(numbers[r]), d, x);
        }
    }
};

// The same value, of which the compiler does not know that it is: what an earlier pass worked out of it is worked out again instead of being kept.
template <typename X> __device__ __forceinline__ void scan_anew(X &x) { asm volatile("" : "+v"(x)); }

// f(whether there is something that makes rows special)
template <typename F>
__device__ __forceinline__ void scan_rows(bool special, F f)
{
    if (special) f(std::true_type());
    else f(std::false_type());
}

// The gates of the wavefront's rows, and whether one of them is closed.
template <typename T, int V>
__device__ __forceinline__ bool scan_gates(const unsigned (&fs)[SCAN_ROWS], float (&g)[SCAN_ROWS][V])
{
    float least = 1.f;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {
        float f[V];
        ScanLane<T, V>::values(fs[r], f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            g[r][v] = gate_of(f[v]);
            least = fminf(least, fabsf(g[r][v]));
        }
        if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);               // (not all rows at once: there are no registers for that)
    }
    return __any(least == 0.f);
}

// Where there are no rows: what goes into the sequences comes out.
static __global__ __launch_bounds__(256) void scan_nothing(const ScanOrder o, const float *in, float *out, int64_t d, int *flags)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < o.count * d; i += (int64_t)gridDim.x * 256) {
        if (out) out[i] = in ? in[i] : 0.f;
        if (flags && i % d == 0 && (o.at(i / d) != 0 || o.at(i / d + 1) != 0)) atomicOr(flags, FLAG_OFFSETS);
    }
}

template <typename T, bool PACKED>
__global__ __launch_bounds__(SCAN_THREADS, SCAN_FORWARD_HELD) void scan_forward(const Scan<T, PACKED> a)
{
    constexpr int V = SCAN_V<T, false>;
    __shared__ ScanShared<V> told;
    __shared__ ScanEdges<V> all_edges[SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ScanEdges<V> &edges = all_edges[wave];
    const unsigned block = blockIdx.x % a.blocks, q = scan_tile(a, block);
    const ScanLane<T, V> at(block, a.d);
    const int64_t n = a.order.n, t0 = (int64_t)q * SCAN_TILE + wave * SCAN_ROWS;
    // (wavefronts behind the last row have that one, as rows of no sequence, and store nothing)
    const int many = (int)(n - t0 < SCAN_ROWS ? n - t0 < 0 ? 0 : n - t0 : SCAN_ROWS);
    const int64_t from = many > 0 ? t0 : n - 1;
    unsigned fs[SCAN_ROWS];
    typename ScanInput<T, PACKED>::Raw us;
    at.load(a.f + from * a.ldf, a.ldf, many, fs);
    a.u.load(from, a.d, many, at, us);
    scan_mark(a.order, told.marks, q, a.tiles, block, a.flags, [&](int64_t j) {
        float h[V];
        if (!a.last) return;
        at.load_floats(a.h0, j, a.d, h);
        at.store_floats(a.last, j, a.d, h);
    });
    __syncthreads();
    const ScanRows rows(a.order, told.marks, t0, wave * SCAN_ROWS);
    edges.fetch(rows.starts, told.marks.start + wave * SCAN_ROWS, a.h0, a.d, at);
    // every row as h = A h + B, the first one of a sequence with A = 0, and with it those of none
    float A[SCAN_ROWS][V], B[SCAN_ROWS][V];
    const bool closed = scan_gates<T, V>(fs, A) || rows.none;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {
        float u[V];
        a.u.values(us, r, u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const GateShares g = gate_shares(A[r][v]);
            A[r][v] = g.a;
            B[r][v] = share_of<true>(g.c, u[v]);
        }
        if (rows.starts >> r & 1) {
            float h[V];
            edges.get(r, h);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                B[r][v] = gate_step<true>(A[r][v], h[v], B[r][v]);
                A[r][v] = 0.f;
            }
        }
    }
    if (rows.none)
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r)
            if (rows.none >> r & 1)
#pragma unroll
                for (int v = 0; v < V; ++v) A[r][v] = B[r][v] = 0.f;
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    scan_rows(closed, [&](auto special) {
#pragma unroll
        for (int r = 0; r < SCAN_ROWS; ++r) {
            if (rows.starts >> r & 1)
#pragma unroll
                for (int v = 0; v < V; ++v) p[v] = {0.f, 0.f};
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] = {p[v].a * A[r][v], gate_step<decltype(special)::value>(A[r][v], p[v].b, B[r][v])};
        }
    });
#pragma unroll
    for (int v = 0; v < V; ++v) told.products[wave][v][lane] = p[v];
    __syncthreads();
    if (wave == 0) {
        float x[V] = {};
        if (a.tickets) {
            ScanProduct own[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                own[v] = p[v];
#pragma unroll
                for (int w = 1; w < SCAN_WAVES; ++w) own[v] = told.products[w][v][lane].after(own[v]);
            }
            scan_hand<T, PACKED, V>(a, q, block, told.marks.from, own, x);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) told.into[v][lane] = x[v];
    }
    __syncthreads();
    if (many == 0) return;
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = told.into[v][lane];
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = told.products[w][v][lane].of(h[v]);
    if (a.states) {
        float enters[V];
#pragma unroll
        for (int v = 0; v < V; ++v) enters[v] = rows.none & 1 ? 0.f : h[v];
        if (rows.starts & 1) edges.get(0, enters);
        at.store_floats(a.states, t0 / SCAN_KEPT, a.d, enters);
    }
    const unsigned ends = a.last ? rows.ends : 0;
    T *y = a.y + t0 * a.ldy + at.first;
    if (at.here())
        scan_rows(closed || many < SCAN_ROWS, [&](auto special) {
            constexpr bool SPECIAL = decltype(special)::value;
#pragma unroll
            for (int r = 0; r < SCAN_ROWS; ++r) {
                if (SPECIAL && r >= many) break;
                if (rows.starts >> r & 1)
#pragma unroll
                    for (int v = 0; v < V; ++v) h[v] = 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = gate_step<SPECIAL>(A[r][v], h[v], B[r][v]);
                at.store(y, h);
                y += a.ldy;
                if (ends >> r & 1) edges.put(r, h);
            }
        });
    edges.store(ends, told.marks.end + wave * SCAN_ROWS, a.last, a.d, at);
}

template <typename T, bool PACKED>
__global__ __launch_bounds__(SCAN_THREADS, SCAN_BACKWARD_HELD) void scan_backward(const Scan<T, PACKED> a)
{
    constexpr int V = SCAN_V<T, true>;
    __shared__ ScanShared<V> told;
    __shared__ ScanEdges<V> all_edges[SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ScanEdges<V> &edges = all_edges[wave];
    const unsigned block = blockIdx.x % a.blocks, q = scan_tile(a, block), tile = a.tiles - 1 - q;
    const ScanLane<T, V> at(block, a.d);
    const int64_t n = a.order.n, t0 = (int64_t)tile * SCAN_TILE + wave * SCAN_ROWS;
    const int many = (int)(n - t0 < SCAN_ROWS ? n - t0 < 0 ? 0 : n - t0 : SCAN_ROWS);
    const int64_t from = many > 0 ? t0 : n - 1;
    unsigned fs[SCAN_ROWS], dys[SCAN_ROWS];
    typename ScanInput<T, PACKED>::Raw us;
    float h[V];
    at.load(a.f + from * a.ldf, a.ldf, many, fs);
    a.u.load(from, a.d, many, at, us);
    at.load_floats(a.states, from / SCAN_KEPT, a.d, h);
    at.load(a.dy + from * a.lddy, a.lddy, many, dys);
    scan_mark(a.order, told.marks, tile, a.tiles, block, a.flags, [&](int64_t j) {
        float x[V];
        if (!a.dh0) return;
        at.load_floats(a.dlast, j, a.d, x);
        at.store_floats(a.dh0, j, a.d, x);
    });
    __syncthreads();
    const ScanRows rows(a.order, told.marks, t0, wave * SCAN_ROWS);
    edges.fetch(rows.starts, told.marks.start + wave * SCAN_ROWS, a.h0, a.d, at);
    float g[SCAN_ROWS][V], wide[SCAN_ROWS][V];       // gates, and h_{t-1} - u_t
    const bool closed = scan_gates<T, V>(fs, g) || rows.none;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {
        float u[V];
        if (rows.starts >> r & 1) edges.get(r, h);
        a.u.values(us, r, u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const GateShares shares = gate_shares(g[r][v]);
            wide[r][v] = h[v] - u[v];
            h[v] = gate_step<true>(shares.a, h[v], share_of<true>(shares.c, u[v]));
        }
    }
    edges.fetch(rows.ends, told.marks.end + wave * SCAN_ROWS, a.dlast, a.d, at);
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    // x: what goes from a row to the one before, a G
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    scan_rows(closed, [&](auto special) {
        constexpr bool SPECIAL = decltype(special)::value;
#pragma unroll
        for (int r = SCAN_ROWS - 1; r >= 0; --r) {
            float dy[V];
            if (rows.ends >> r & 1) {
                float x[V];
                edges.get(r, x);
#pragma unroll
                for (int v = 0; v < V; ++v) p[v] = {0.f, x[v]};
            }
            at.values(dys[r], dy);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float share = gate_shares(g[r][v]).a;
                p[v] = {p[v].a * share, share_of<SPECIAL>(share, p[v].b + dy[v])};
                if (SPECIAL && (rows.none >> r & 1)) p[v] = {0.f, 0.f};
            }
        }
    });
#pragma unroll
    for (int v = 0; v < V; ++v) told.products[wave][v][lane] = p[v];
    __syncthreads();
    if (wave == SCAN_WAVES - 1) {
        float x[V] = {};
        if (a.tickets) {
            ScanProduct own[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                own[v] = p[v];
#pragma unroll
                for (int w = SCAN_WAVES - 2; w >= 0; --w) own[v] = told.products[w][v][lane].after(own[v]);
            }
            scan_hand<T, PACKED, V>(a, q, block, a.tiles - 1 - told.marks.to, own, x);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) told.into[v][lane] = x[v];
    }
    __syncthreads();
    if (many == 0) return;
#pragma unroll
    for (int r = 0; r < SCAN_ROWS; ++r) {            // (not kept from the pass above)
        scan_anew(dys[r]);
#pragma unroll
        for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    }
    float x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = told.into[v][lane];
    for (int w = SCAN_WAVES - 1; w > wave; --w)
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = told.products[w][v][lane].of(x[v]);
    const unsigned starts = a.dh0 ? rows.starts : 0;
    T *df_row = a.df + (t0 + many - 1) * a.lddf + at.first, *du_row = a.du + (t0 + many - 1) * a.lddu + at.first;
    if (at.here())
        scan_rows(closed || many < SCAN_ROWS, [&](auto special) {
            constexpr bool SPECIAL = decltype(special)::value;
#pragma unroll
            for (int r = SCAN_ROWS - 1; r >= 0; --r) {
                if (SPECIAL && r >= many) continue;
                if (rows.ends >> r & 1) edges.get(r, x);
                float dy[V], df[V], du[V];
                at.values(dys[r], dy);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float G = x[v] + dy[v];
                    const GateShares shares = gate_shares(g[r][v]);
                    df[v] = share_of<SPECIAL>(shares.a * shares.c, G * wide[r][v]);
                    du[v] = share_of<SPECIAL>(shares.c, G);
                    x[v] = share_of<SPECIAL>(shares.a, G);
                    if (SPECIAL && (rows.none >> r & 1)) df[v] = du[v] = x[v] = 0.f;
                }
                at.store(df_row, df);
                at.store(du_row, du);
                df_row -= a.lddf;
                du_row -= a.lddu;
                if (starts >> r & 1) edges.put(r, x);
            }
        });
    edges.store(starts, told.marks.start + wave * SCAN_ROWS, a.dh0, a.d, at);
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
        for (int i = 0; i < V; ++i) {
            const GateShares g = gate_shares(gate_of(fv[i]));
            hs[i] = gate_step<true>(g.a, hs[i], share_of<true>(g.c, uv[i]));
        }
#pragma unroll
        for (int k = 0; k < V; k += 4)
            if (c + k < d) store_vec(state + row * lds, c + k, d, hs + k);
        store_vec<T, true>(y + row * ldy, c, d, hs);
    }
}

}  // namespace chicle_train
