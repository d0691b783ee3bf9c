// A gated linear recurrence over the rows of sequences, its gradients, and its form for one row of every sequence.
//
//   a_t = 1 / (1 + exp(-f_t)),  c_t = 1 - a_t,  h_t = a_t h_{t-1} + c_t u_t,  y_t = h_t, from the sequence's first state or from 0
//   G_t = dy_t + a_{t+1} G_{t+1}, the last row's with the gradient of the last state:
//   du_t = c_t G_t,  df_t = G_t (h_{t-1} - u_t) a_t c_t,  dh0 = a_first G_first
//
// Of a gate, the smaller share is worked out, s = e / (1 + e) with e = exp(-|f|), the other one is 1 - s: neither loses what is small, down to the last 32-bit
// number, 2^-149.  Where e is rounded to nothing, from 150 ln 2 = 103.97 on, a gate is closed, s = 0, and what it keeps out counts nowhere, whatever it holds.
//
// States are 32-bit floats.  A workgroup has a tile of rows and columns (ScanShape), a wavefront some of its rows, a lane one or two columns of them, held in
// registers and read once.  What the rows of a wavefront do to the state that comes into them is a product and a sum (ScanProduct); those of the tile are
// joined in LDS, and tiles tell one another theirs (ScanShared::join), so that one long sequence fills the chip as well as many short ones.  The forward
// pass leaves the state that enters every SCAN_KEPT-th row; the gradient works out those between again, and goes through the tiles from the last one.
//
// What bounds it is memory: every value is read and written once, a large copy goes at 4.95 TB/s.  65,536 rows of 2048 columns in bfloat16, forward
// and its gradients: sequences of 128 rows 176 and 270 us (4.7 and 5.0 TB/s), one sequence 210 and 303 us (3.9 and 4.5): there tiles wait for what comes
// into them; rows of 1024 in float32 140 and 241 us (5.8 and 5.6), one sequence 159 and 252 (5.1 and 5.4).  A thread that goes through its column alone takes
// 29,950 us for 65,536 rows in one sequence.  Small calls are launches: 333 x 250 in float32 9.2 and 12.0 us, of which 4 are a state's way through the three tiles.
#pragma once
#include <type_traits>
#include "elements.hpp"
#include "packed.hpp"

namespace chicle_train {

constexpr int SCAN_KEPT = 32;

// s with the sign of f.  The exponential of the hardware gives no numbers below 2^-126: there it is that of 64 more, which the quotient brings down by
// 2^64 (where 1 + e is 1), with its one rounding.  (65,536 x 2048 in bfloat16, sequences of 128 rows, forward: 195 us a call, and 191 without the small shares; one
// sequence and the gradients the same.)
__device__ __forceinline__ float gate_of(float f)
{
    const bool small = fabsf(f) > 87.33f;                // (126 ln 2 = 87.337)
    const float e = __builtin_amdgcn_exp2f(fmaf(-1.44269504f, fabsf(f), small ? 64.f : 0.f));
    return copysignf(e * __builtin_amdgcn_rcpf((small ? 0x1p64f : 1.f) + e), f);
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

// A lane has 32 values of every input: of 16 bits two columns, so that it reads four bytes of a row, and half as many rows.  (Forward, 65,536 x 2048 in bfloat16,
// one sequence: one column and 32 rows 225 us, two and 16 rows 184 when first measured.  The gradient has three inputs and a pass more: with two
// columns, its wavefronts in pairs that share a tile's rows, it takes 330 to 550 us instead of 315.  Two wavefronts to a workgroup are slower in both.)
template <typename T, bool BACKWARD> struct ScanShape {
    static constexpr int V = BACKWARD ? 1 : 4 / (int)sizeof(T), COLS = 64 * V, ROWS = SCAN_KEPT / V;
    static constexpr int WAVES = 4 * V, THREADS = 64 * WAVES, TILE = ROWS * WAVES;
    // wavefronts of a SIMD, as registers allow (gradients in 16 bits, 65,536 x 2048 in sequences of 128 rows: three 293 us, four 268)
    static constexpr int HELD = BACKWARD && sizeof(T) == 4 ? 3 : 4;
    static constexpr int MORE_LDS = V == 1 ? 16384 : 0;  // LDS besides with which there are three workgroups to a compute unit
    static constexpr bool LINES = !BACKWARD || sizeof(T) == 4;             // there are registers for both kinds of loads
};
// (200,000 x 16 in float32, 1563 tiles in one column block: 8 and 64 take 41 us, 8 and 16 or 16 and 16 take 84 to 88, 8 and 128 the same 41; with 16 and 64,
// 65,536 x 2048 in bfloat16 takes 231 and 343 us instead of 206 and 308, for registers, when measured.)
constexpr int SCAN_GROUP = 8, SCAN_RUN = 64;             // tiles whose products are joined, and tiles from one state that is handed on to the next
constexpr int SCAN_TICKET = 32;                          // places from one column block's ticket to the next: lines of their own

typedef unsigned u32_at_2 __attribute__((aligned(2)));

// A lane's columns of a tile, counted from the tile's first: rows are given by uniform pointers to that one.  Lanes past the last column read
// some column that is there and store nothing.
template <typename T, typename S> struct ScanLane {
    static constexpr int V = S::V, ROWS = S::ROWS;
    unsigned first;                          // the tile's first column
    int e, left;                             // the lane's first column; columns from the tile's first to the last one, or the tile's
    __device__ __forceinline__ ScanLane(unsigned block, unsigned d) : first(block * S::COLS), e((threadIdx.x & 63) * V) { left = min(d - first, (unsigned)S::COLS); }
    __device__ __forceinline__ bool here() const { return e < left; }
    __device__ __forceinline__ bool odd() const { return V == 2 && (left & 1); }          // the last column has no neighbour
    // The lane's values of a wavefront's rows: the last of `many` again in place of those that are not there.
    template <typename L> static __device__ __forceinline__ void each_row(int many, L load)
    {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            asm volatile("" : "+s"(many));               // (one row's pointer after the other: all of them at once are too many scalars)
            load(r, r + 1 < many);
        }
    }
    // `lines`: rows are whole lines of the cache, which no other column block reads, and are not kept there.
    __device__ __forceinline__ void load(const T *row, int64_t ld, int many, bool lines, unsigned (&out)[ROWS]) const
    {
        const T *p = row + first;
        if (V == 2 && left == 1) {
            each_row(many, [&](int r, bool further) {
                out[r] = *(const uint16_t *)p;
                p += further ? ld : 0;
            });
            return;
        }
        typedef typename std::conditional<V * sizeof(T) == 4, u32_at_2, uint16_t>::type word;
        // (a column that has no neighbour comes with the one before it)
        const unsigned off = e + V <= left ? e : left - V;
        if (S::LINES && lines)
            each_row(many, [&](int r, bool further) {
                out[r] = __builtin_nontemporal_load((const word *)(p + off));
                p += further ? ld : 0;
            });
        else
            each_row(many, [&](int r, bool further) {
                out[r] = *(const word *)(p + off);
                p += further ? ld : 0;
            });
        if (odd()) {
            const int bits = e + 1 == left ? 16 : 0;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) out[r] >>= bits;
        }
    }
    static __device__ __forceinline__ void values(unsigned x, float (&out)[V])
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
    // `row`: the tile's first column; only lanes that have one.  EDGE: the last column may have no neighbour.
    template <bool EDGE> __device__ __forceinline__ void store(T *row, const float (&in)[V]) const
    {
        if constexpr (V == 1) __builtin_nontemporal_store((T)in[0], row + (unsigned)e);
        else {
            T v[2] = {(T)in[0], (T)in[1]};
            unsigned x;
            __builtin_memcpy(&x, v, 4);
            if (EDGE && e + 1 == left) row[(unsigned)e] = v[0];
            else __builtin_nontemporal_store(x, (u32_at_2 *)(row + (unsigned)e));
        }
    }
    // Row j of floats (of a null pointer: zeros).
    __device__ __forceinline__ void load_floats(const float *p, int64_t j, int64_t d, float (&out)[V]) const
    {
        const float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < V; ++v) out[v] = p ? row[(unsigned)(e + v < left ? e + v : left - 1)] : 0.f;
    }
    __device__ __forceinline__ void store_floats(float *p, int64_t j, int64_t d, const float (&in)[V]) const
    {
        float *row = p + j * d + first;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (e + v < left) row[(unsigned)(e + v)] = in[v];
    }
};

// The second input's rows, of T or packed: what a lane asks for of a wavefront's rows, and its values.
template <typename T, bool PACKED> struct ScanInput;
template <typename T> struct ScanInput<T, false> {
    template <typename S> struct Raw { unsigned x[S::ROWS]; };
    const T *p;
    int64_t ld;
    template <typename S> __device__ __forceinline__ void load(int64_t row, int64_t, int many, bool lines, const ScanLane<T, S> &at, Raw<S> &out) const
    {
        at.load(p + row * ld, ld, many, lines, out.x);
    }
    template <typename S> static __device__ __forceinline__ void values(const Raw<S> &raw, int r, float (&out)[S::V]) { ScanLane<T, S>::values(raw.x[r], out); }
};
template <typename T> struct ScanInput<T, true> {
    // step: a lane has the scale of one row and one of the tile's groups, row by row
    template <typename S> struct Raw { unsigned x[S::ROWS], step; };
    const int8_t *q;
    const uint8_t *scales;
    int64_t ld;
    template <typename S> __device__ __forceinline__ void load(int64_t row, int64_t d, int many, bool, const ScanLane<T, S> &at, Raw<S> &out) const
    {
        constexpr int V = S::V, GROUPS = S::COLS / PACK_GROUP;
        static_assert(GROUPS * S::ROWS == 64, "a lane for every scale");
        const unsigned whole = ((unsigned)d + PACK_GROUP - 1) / PACK_GROUP * PACK_GROUP;
        const int left = min(whole - at.first, (unsigned)S::COLS), lane = threadIdx.x & 63;
        const unsigned off = at.e < left ? at.e : left - V;
        const int r = lane / GROUPS, which = r < many ? r : many > 0 ? many - 1 : 0, group = lane % GROUPS;
        out.step = scales[(row + which) * (ld / PACK_GROUP) + at.first / PACK_GROUP + (group * PACK_GROUP < left ? group : 0)];
        const uint8_t *p = (const uint8_t *)q + row * ld + at.first;
        at.each_row(many, [&](int i, bool further) {
            if constexpr (V == 1) out.x[i] = p[off];
            else out.x[i] = *(const uint16_t *)(p + off);
            p += further ? ld : 0;
        });
    }
    template <typename S> static __device__ __forceinline__ void values(const Raw<S> &raw, int r, float (&out)[S::V])
    {
        constexpr int GROUPS = S::COLS / PACK_GROUP;
        const int from = GROUPS * r + (threadIdx.x & 63) / (64 / GROUPS);
        const float step = pack_step((unsigned)__builtin_amdgcn_ds_bpermute(from * 4, (int)raw.step));
#pragma unroll
        for (int v = 0; v < S::V; ++v) out[v] = (float)(int8_t)(raw.x[r] >> (8 * v)) * step;
    }
};

// Where sequences begin: sequence j has the rows from at(j) to at(j + 1).
struct ScanOrder {
    const void *offsets;                     // null: one sequence of all rows
    int wide;
    int64_t count, n;
    __device__ __forceinline__ int64_t at(int64_t j) const { return offsets ? index_at(offsets, wide, j) : j == 0 ? 0 : n; }
    // The same for a j that all lanes have in common, the lower 32 bits: scalar loads, which do not wait behind the rows' loads.
    __device__ __forceinline__ unsigned common(unsigned j) const
    {
        if (!offsets) return j == 0 ? 0u : (unsigned)n;
        return ((const __attribute__((address_space(4))) unsigned *)offsets)[wide ? 2 * (int64_t)j : (int64_t)j];
    }
    // How many of the offsets are at most t.  (Rows, columns and sequences are 32-bit numbers here, also because hipcc 7.2 has been seen to take the condition
    // of one choice between uniform 64-bit numbers for that of the next.)
    __device__ __forceinline__ unsigned up_to(unsigned t) const
    {
        unsigned lo = 0, hi = (unsigned)count + 1;
        while (lo < hi) {                                // (the distance shrinks, whatever the offsets are)
            const unsigned step = (hi - lo + 7) >> 3;
            unsigned many = 0;
#pragma unroll
            for (int k = 1; k <= 8; ++k) {
                const unsigned j = lo + k * step - 1;
                if (j < hi && common(j) <= t) ++many;
            }
            const unsigned next = lo + (many + 1) * step - 1;
            lo = min(lo + many * step, hi);
            hi = min(next, hi);
        }
        return lo;
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
    bool lines;                              // rows of T that are read are whole lines of the cache
    int looks;                               // before a wait is given up (the last: with `tickets` eight bytes further on, which a workgroup asks for first,
                                             // gradients of 30,011 x 1000 in half precision, one sequence, take 92 us instead of 86)
};

constexpr unsigned long long SCAN_NOTHING = ~0ull;       // what no product is: its lower half is no NaN of these bits

__global__ __launch_bounds__(256) static void scan_begin(unsigned *tickets, unsigned blocks, unsigned long long *words, int64_t count)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        words[i] = SCAN_NOTHING;
        if (i < blocks) tickets[i * SCAN_TICKET] = 0;    // (there are more words than column blocks)
    }
}

// What rows do to what comes into them: x becomes a x + b.  Where it does not get through, whatever it is, since a sequence begins or a gate is closed, a is
// -0: a product of shares that is too small for a number is +0, and lets what is no number through.
constexpr float SCAN_STOP = -0.f;

struct ScanProduct {
    float a, b;
    __device__ __forceinline__ float of(float x) const { return signbit(a) ? b : fmaf(a, x, b); }
    // What the rows do after `before`.
    __device__ __forceinline__ ScanProduct after(const ScanProduct &before) const { return {signbit(a) ? SCAN_STOP : a * before.a, of(before.b)}; }
    __device__ __forceinline__ unsigned long long word() const
    {
        const unsigned lo = a == a ? __float_as_uint(a) : 0x7fc00000u;
        return (unsigned long long)__float_as_uint(b) << 32 | lo;
    }
    static __device__ __forceinline__ ScanProduct from(unsigned long long w) { return {__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32))}; }
};

__device__ __forceinline__ unsigned long long scan_look(const unsigned long long *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void scan_tell(unsigned long long *p, unsigned long long w) { __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// (Every wait ends by itself, see below.  Where a workspace is written by something else meanwhile, against its rules, this one ends too, after so many looks,
// some seconds, with what is no number, and says so.)  A: the kernel's arguments, of which those for this are read where there is a
// wait, and not kept in scalar registers all along.
template <typename A>
__device__ __forceinline__ unsigned long long scan_wait(const unsigned long long *p, unsigned long long w)
{
    if (__any(w == SCAN_NOTHING)) {
        auto args = (const __attribute__((address_space(4))) A *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(args));
        bool missing = true;
        for (int left = args->looks; missing && left > 0; --left) {
            __builtin_amdgcn_s_sleep(1);
            w = scan_look(p);
            missing = __any(w == SCAN_NOTHING);
        }
        if (missing && args->flags) atomicOr(args->flags, FLAG_WAIT);
    }
    return w;
}

// What a wavefront knows of its rows: which of them are a sequence's first, a sequence's last, or of none, and in lane r the numbers of the sequences
// that begin and end with row r.  Worked out with scalars while the rows are on their way; offsets that are no rows lead to wrong marks, but to
// no place outside of the rows and the sequences.
struct ScanRows {
    unsigned starts, ends, none;
    int start, end;                          // of this lane's row
    unsigned before, behind;                 // where the sequence of the first row begins, and that of the last one ends, if not with it; else ~0
    template <typename S> __device__ __forceinline__ ScanRows(const ScanOrder &o, unsigned t0, S)
    {
        const unsigned t1 = t0 + S::ROWS, lane = threadIdx.x & 63, count = (unsigned)o.count;
        starts = ends = 0;
        start = end = 0;
        before = behind = ~0u;
        unsigned j = t0 > 0 ? o.up_to(t0 - 1) : 0;
        if (j > 0 && j <= count && o.common(j) > t0) before = o.common(j - 1);
        for (int left = S::ROWS + 1; j <= count && left > 0; --left) {     // (rows t0 to t1, where offsets ascend)
            const unsigned at = o.common(j);
            if (at > t1) break;
            // sequence j - 1 ends in front of row `at`, sequence k - 1 begins with it; those between have no rows
            if (j > 0 && at - 1 - t0 < S::ROWS) {
                ends |= 1u << (at - 1 - t0);
                end = lane == at - 1 - t0 ? (int)j - 1 : end;
            }
            unsigned k = j + 1;
            if (k <= count && o.common(k) <= at) k = max(k, o.up_to(at));
            if (k <= count && at - t0 < S::ROWS) {
                starts |= 1u << (at - t0);
                start = lane == at - t0 ? (int)k - 1 : start;
            }
            j = k;
        }
        if (j > 0 && j <= count && o.common(j - 1) < t1) behind = o.common(j);
        const unsigned lo = o.common(0), hi = min(o.common(count), (unsigned)o.n);
        const unsigned all = S::ROWS == 32 ? ~0u : (1u << S::ROWS % 32) - 1;
        const unsigned row = t0 + (lane & (S::ROWS - 1));
        none = (unsigned)__ballot(row < lo || row >= hi) & all;
        starts &= ~none;
        ends &= ~none;
    }
};

// What sequences without rows get, each from one tile, and a look at all offsets.
template <typename S, typename F>
__device__ __forceinline__ void scan_empty(const ScanOrder &o, unsigned tile, unsigned tiles, bool check, int *flags, F empty)
{
    bool wrong = false;
    for (int64_t j0 = (int64_t)tile * S::THREADS; j0 < o.count; j0 += (int64_t)tiles * S::THREADS) {
        const int64_t j = j0 + threadIdx.x;
        bool none = false;
        if (j < o.count) {
            const int64_t lo = o.at(j), hi = o.at(j + 1);
            none = lo == hi;
            wrong |= lo < 0 || hi < lo || hi > o.n;
        }
        for (unsigned long long left = __ballot(none); left; left &= left - 1) empty(j0 + (threadIdx.x & ~63) + __builtin_ctzll(left));
    }
    if (check && wrong && flags) atomicOr(flags, FLAG_OFFSETS);
}

// How states go from tile to tile of a column block, q being a tile's number in the order in which tiles are taken, and `from` the one whose product
// lets nothing through that is needed (from >= q: nothing comes in, the tile's own product lets nothing through).
//
// A tile tells its product; the last one of SCAN_GROUP tiles tells theirs, joined; the last one of SCAN_RUN tiles hands on the state that comes out.  What
// comes into a tile is, in this order, the state handed on from the run before, the products of the run's groups before its own (`far`), and those of
// the tiles before it in its own (`near`): a state goes through a long sequence in steps of SCAN_RUN tiles, everything else of which has been joined
// by then.  Three wavefronts look for the three.
//
// Tiles are taken in the order of their column block's tickets: whoever waits does so for tiles with earlier tickets, whose workgroups have begun.
// These tell their products without waiting, groups once the products of the group are told, and states after all that is before them.
// So every wait ends.  What is joined, and in which order, follows from the offsets alone.  A word is told whole, and says by itself whether it
// has been.
template <typename A, int V>
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
                for (int v = 0; v < V; ++v) x[v] = ScanProduct::from(scan_wait<A>(p + k * line + v * 64, w[k][v])).after(x[v]);
    }
}

// By the first wavefront: tells the tile's product and, with the last of the group, the group's.
template <typename T, bool PACKED, int V>
__device__ __forceinline__ void scan_near(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned from, const ScanProduct (&own)[V], ScanProduct (&near)[V])
{
    const int64_t line = (int64_t)a.blocks * 64 * V, at = (int64_t)block * 64 * V + (threadIdx.x & 63);
    const unsigned group = q / SCAN_GROUP;
#pragma unroll
    for (int v = 0; v < V; ++v) scan_tell(a.products + q * line + at + v * 64, own[v].word());
    scan_join<Scan<T, PACKED>, V>(a.products + at, line, max(from, group * SCAN_GROUP), q, near);
    if (q % SCAN_GROUP == SCAN_GROUP - 1)
#pragma unroll
        for (int v = 0; v < V; ++v) scan_tell(a.groups + group * line + at + v * 64, own[v].after(near[v]).word());
}

template <typename T, bool PACKED, int V>
__device__ __forceinline__ void scan_far(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned from, ScanProduct (&far)[V])
{
    const int64_t line = (int64_t)a.blocks * 64 * V, at = (int64_t)block * 64 * V + (threadIdx.x & 63);
    scan_join<Scan<T, PACKED>, V>(a.groups + at, line, max(from / SCAN_GROUP, q / SCAN_RUN * (SCAN_RUN / SCAN_GROUP)), q / SCAN_GROUP, far);
}

template <typename T, bool PACKED, int V>
__device__ __forceinline__ void scan_handed(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned from, float (&x)[V])
{
    const int64_t line = (int64_t)a.blocks * 64 * V;
    const unsigned run = q / SCAN_RUN;
    if (from >= run * SCAN_RUN) return;
    const unsigned long long *p = a.handed + (int64_t)(run - 1) * line + (int64_t)block * 64 * V + (threadIdx.x & 63);
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = __uint_as_float((unsigned)scan_wait<Scan<T, PACKED>>(p + v * 64, scan_look(p + v * 64)));
}

// The workgroup's column block and tile.  Tickets, those of each column block for themselves, give tiles in the order in which workgroups begin.
// Workgroups go to the chip's eight L2 partitions in turn: those of one take neighbouring column blocks first, whose rows meet in lines of the cache, and
// then whatever is left (there are as many workgroups as tiles, so that each finds one: all blocks are used up only when every tile is taken).
template <typename S> __device__ __forceinline__ void scan_unit(const S &a, unsigned &block, unsigned &q)
{
    __shared__ unsigned found[2];
    if (!a.tickets) {
        block = blockIdx.x;
        q = 0;
        return;
    }
    if (threadIdx.x == 0) {
        const unsigned part = blockIdx.x & 7, begin = a.blocks * (uint64_t)part / 8, many = max(a.blocks * (uint64_t)(part + 1) / 8 - begin, (uint64_t)1);
        unsigned b = begin + (blockIdx.x >> 3) % many, tile;
        for (unsigned tried = 0; (tile = atomicAdd(a.tickets + b * SCAN_TICKET, 1u)) >= a.tiles && tried < a.blocks; ++tried) b = b + 1 < a.blocks ? b + 1 : 0;
        found[0] = b;
        found[1] = tile;
    }
    __syncthreads();
    block = __builtin_amdgcn_readfirstlane(found[0]);
    q = __builtin_amdgcn_readfirstlane(found[1]);
}

// What the wavefronts of a workgroup tell one another.
template <typename S> struct ScanShared {
    static constexpr int V = S::V;
    ScanProduct products[S::WAVES][V][64], own[V][64], near[V][64], far[V][64];
    float handed[V][64];
    unsigned from;
    // What comes into the wavefront's rows.  p: its product; mine: `from` of the wavefront whose rows come first, backwards the last one's.  All
    // wavefronts together.
    template <bool BACKWARD, typename T, bool PACKED>
    __device__ __forceinline__ void join(const Scan<T, PACKED> &a, unsigned q, unsigned block, unsigned mine, int wave, const ScanProduct (&p)[V], float (&x)[V])
    {
        const int lane = threadIdx.x & 63;
        if (wave == (BACKWARD ? S::WAVES - 1 : 0)) from = mine;
#pragma unroll
        for (int v = 0; v < V; ++v) products[wave][v][lane] = p[v];
        __syncthreads();
        if (a.tickets) {
            const unsigned first = __builtin_amdgcn_readfirstlane(from);
            if (wave == 0) {
                ScanProduct all[V], k[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    all[v] = products[BACKWARD ? S::WAVES - 1 : 0][v][lane];
                    k[v] = {1.f, 0.f};
#pragma unroll
                    for (int w = 1; w < S::WAVES; ++w) all[v] = products[BACKWARD ? S::WAVES - 1 - w : w][v][lane].after(all[v]);
                    own[v][lane] = all[v];
                }
                scan_near<T, PACKED, V>(a, q, block, first, all, k);
#pragma unroll
                for (int v = 0; v < V; ++v) near[v][lane] = k[v];
            } else if (wave == 1) {
                ScanProduct k[V];
#pragma unroll
                for (int v = 0; v < V; ++v) k[v] = {1.f, 0.f};
                scan_far<T, PACKED, V>(a, q, block, first, k);
#pragma unroll
                for (int v = 0; v < V; ++v) far[v][lane] = k[v];
            } else if (wave == 2) {
                float k[V] = {};
                scan_handed<T, PACKED, V>(a, q, block, first, k);
#pragma unroll
                for (int v = 0; v < V; ++v) handed[v][lane] = k[v];
            }
            __syncthreads();
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = a.tickets ? near[v][lane].after(far[v][lane]).of(handed[v][lane]) : 0.f;
            if (a.tickets && wave == S::WAVES - 1 && q % SCAN_RUN == SCAN_RUN - 1)
                scan_tell(a.handed + ((int64_t)(q / SCAN_RUN) * a.blocks + block) * 64 * V + lane + v * 64, __float_as_uint(own[v][lane].of(x[v])));
        }
        // and what the wavefronts in front of this one do to it
        if constexpr (BACKWARD) {
            for (int w = S::WAVES - 1; w > wave; --w)
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = products[w][v][lane].of(x[v]);
        } else {
            for (int w = 0; w < wave; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = products[w][v][lane].of(x[v]);
        }
    }
};

// States or gradients of sequences that begin or end among the wavefront's rows, each in the place of its row: a lane's own, read and written by no other.
template <typename S> struct ScanEdges {
    static constexpr int V = S::V;
    float place[S::ROWS][V][64];
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
    // Fetches them for the rows of `which`, whose sequences the lanes' numbers are; zeros of a null pointer.
    template <typename L> __device__ __forceinline__ void fetch(unsigned which, int number, const float *from, int64_t d, const L &at)
    {
        constexpr int AHEAD = 4;
        while (which) {
            float x[AHEAD][V];
            unsigned left = which;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (left) at.load_floats(from, __builtin_amdgcn_readlane(number, __builtin_ctz(left)), d, x[k]);
                left &= left - 1;
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (which) put(__builtin_ctz(which), x[k]);
                which &= which - 1;
            }
        }
    }
    template <typename L> __device__ __forceinline__ void store(unsigned which, int number, float *to, int64_t d, const L &at) const
    {
        for (; which; which &= which - 1) {
            const int r = __builtin_ctz(which);
            float x[V];
            get(r, x);
            at.store_floats(to, __builtin_amdgcn_readlane(number, r), d, x);
        }
    }
};

// The same value, of which the compiler does not know that it is: it is worked out here, and not where it is used from what it is made of, and what an
// earlier pass worked out of it is worked out again, instead of all of that being kept (the gradients: 161 registers, with these 120).
template <typename X> __device__ __forceinline__ void scan_anew(X &x) { asm volatile("" : "+v"(x)); }

// f(whether there is something that makes rows special)
template <typename F>
__device__ __forceinline__ void scan_rows(bool special, F f)
{
    if (special) f(std::true_type());
    else f(std::false_type());
}

// f(r, whether rows are special, whether there may be an edge) for all rows, BACKWARD from the last one on: eight at a time, without looks at each where
// none of them is one of `edges`.  (Looked at one by one, gradients of 65,536 x 2048 in bfloat16 take 317 instead of 309 us; with one look for all, sequences
// of 100 rows 345 instead of 315, when measured.)
template <int ROWS, bool BACKWARD, typename F>
__device__ __forceinline__ void scan_each(bool special, unsigned edges, F f)
{
    constexpr int EACH = 8;
    if (special) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) f(BACKWARD ? ROWS - 1 - k : k, std::true_type(), std::true_type());
    } else {
#pragma unroll
        for (int k0 = 0; k0 < ROWS; k0 += EACH)
            scan_rows(edges >> (BACKWARD ? ROWS - EACH - k0 : k0) & ((1u << EACH) - 1), [&](auto edge) __attribute__((always_inline)) {
#pragma unroll
                for (int k = k0; k < k0 + EACH; ++k) f(BACKWARD ? ROWS - 1 - k : k, std::false_type(), edge);
            });
    }
}

// The gates of the wavefront's rows, and whether one of them is closed.
template <typename T, typename S>
__device__ __forceinline__ bool scan_gates(const unsigned (&fs)[S::ROWS], float (&g)[S::ROWS][S::V])
{
    float least = 1.f;
#pragma unroll
    for (int r = 0; r < S::ROWS; ++r) {
        float f[S::V];
        ScanLane<T, S>::values(fs[r], f);
#pragma unroll
        for (int v = 0; v < S::V; ++v) {
            g[r][v] = gate_of(f[v]);
            scan_anew(g[r][v]);
            least = fminf(least, fabsf(g[r][v]));
        }
        if (r % (4 / S::V) == 4 / S::V - 1) __builtin_amdgcn_sched_barrier(0);             // (not all rows at once: there are no registers for that)
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
__global__ __launch_bounds__((ScanShape<T, false>::THREADS), (ScanShape<T, false>::HELD)) void scan_forward(const Scan<T, PACKED> a)
{
    typedef ScanShape<T, false> S;
    constexpr int V = S::V, ROWS = S::ROWS;
    __shared__ ScanShared<S> told;
    __shared__ ScanEdges<S> all_edges[S::WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ScanEdges<S> &edges = all_edges[wave];
    unsigned block, q;
    scan_unit(a, block, q);
    if (q >= a.tiles) return;
    const ScanLane<T, S> at(block, (unsigned)a.d);
    // (rows and columns are fewer than 2^31; wavefronts behind the last row have that one, as rows of no sequence, and store nothing)
    const unsigned n = (unsigned)a.order.n, t = q * S::TILE + wave * ROWS;
    const int many = t < n ? min(n - t, (unsigned)ROWS) : 0;
    const int64_t t0 = t, from = many > 0 ? t : n - 1;
    unsigned fs[ROWS];
    typename ScanInput<T, PACKED>::template Raw<S> us;
    at.load(a.f + from * a.ldf, a.ldf, many, a.lines, fs);
    a.u.load(from, a.d, many, a.lines, at, us);
    const ScanRows rows(a.order, t, S());
    edges.fetch(rows.starts, rows.start, a.h0, a.d, at);
    // every row as h = A h + B, the first one of a sequence with A = 0, and with it those of none
    float A[ROWS][V], B[ROWS][V];
    const bool closed = scan_gates<T, S>(fs, A) || rows.none;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float u[V];
        a.u.template values<S>(us, r, u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const GateShares g = gate_shares(A[r][v]);
            A[r][v] = g.a;
            B[r][v] = share_of<true>(g.c, u[v]);
        }
    }
    if (rows.starts | rows.none)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (rows.starts >> r & 1) {
                float h[V];
                edges.get(r, h);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    B[r][v] = gate_step<true>(A[r][v], h[v], B[r][v]);
                    A[r][v] = 0.f;
                }
            }
            if (rows.none >> r & 1)
#pragma unroll
                for (int v = 0; v < V; ++v) A[r][v] = B[r][v] = 0.f;
        }
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    scan_each<ROWS, false>(closed, rows.starts, [&](int r, auto special, auto edge) __attribute__((always_inline)) {
        constexpr bool SPECIAL = decltype(special)::value;
        const bool starts = decltype(edge)::value && (rows.starts >> r & 1);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (starts || (SPECIAL && A[r][v] == 0.f)) p[v] = {SCAN_STOP, B[r][v]};
            else p[v] = {p[v].a * A[r][v], fmaf(A[r][v], p[v].b, B[r][v])};
        }
    });
    float h[V];
    told.template join<false>(a, q, block, rows.before / S::TILE, wave, p, h);
    if (many > 0) {
        if (a.states && t0 % SCAN_KEPT == 0) {
            float enters[V];
#pragma unroll
            for (int v = 0; v < V; ++v) enters[v] = rows.none & 1 ? 0.f : h[v];
            if (rows.starts & 1) edges.get(0, enters);
            at.store_floats(a.states, t0 / SCAN_KEPT, a.d, enters);
        }
        const unsigned ends = a.last ? rows.ends : 0;
        T *y = a.y + t0 * a.ldy + at.first;
        if (at.here())
            scan_each<ROWS, false>(closed || many < ROWS || at.odd(), rows.starts | ends, [&](int r, auto special, auto edge) __attribute__((always_inline)) {
                constexpr bool SPECIAL = decltype(special)::value, EDGE = decltype(edge)::value;
                if (SPECIAL && r >= many) return;
                if (EDGE && (rows.starts >> r & 1))
#pragma unroll
                    for (int v = 0; v < V; ++v) h[v] = 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = gate_step<SPECIAL>(A[r][v], h[v], B[r][v]);
                at.template store<SPECIAL>(y, h);
                y += a.ldy;
                if (EDGE && (ends >> r & 1)) edges.put(r, h);
            });
        edges.store(ends, rows.end, a.last, a.d, at);
    }
    scan_empty<S>(a.order, q, a.tiles, block == 0, a.flags, [&](int64_t j) {
        float h[V];
        if (!a.last) return;
        at.load_floats(a.h0, j, a.d, h);
        at.store_floats(a.last, j, a.d, h);
    });
}

template <typename T, bool PACKED>
__global__ __launch_bounds__((ScanShape<T, true>::THREADS), (ScanShape<T, true>::HELD)) void scan_backward(const Scan<T, PACKED> a)
{
    typedef ScanShape<T, true> S;
    constexpr int V = S::V, ROWS = S::ROWS;
    __shared__ ScanShared<S> told;
    __shared__ ScanEdges<S> all_edges[S::WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ScanEdges<S> &edges = all_edges[wave];
    unsigned block, q;
    scan_unit(a, block, q);
    if (q >= a.tiles) return;
    const unsigned tile = a.tiles - 1 - q;
    const ScanLane<T, S> at(block, (unsigned)a.d);
    const unsigned n = (unsigned)a.order.n, t = tile * S::TILE + wave * ROWS;
    const int many = t < n ? min(n - t, (unsigned)ROWS) : 0;
    const int64_t t0 = t, from = many > 0 ? t : n - 1;
    unsigned fs[ROWS], dys[ROWS];
    typename ScanInput<T, PACKED>::template Raw<S> us;
    float h[V];
    at.load(a.f + from * a.ldf, a.ldf, many, a.lines, fs);
    a.u.load(from, a.d, many, a.lines, at, us);
    at.load_floats(a.states, from / SCAN_KEPT, a.d, h);
    at.load(a.dy + from * a.lddy, a.lddy, many, a.lines, dys);
    const ScanRows rows(a.order, t, S());
    edges.fetch(rows.starts, rows.start, a.h0, a.d, at);
    float g[ROWS][V], wide[ROWS][V];       // gates, and h_{t-1} - u_t
    const bool closed = scan_gates<T, S>(fs, g) || rows.none;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float u[V];
        if (rows.starts >> r & 1) edges.get(r, h);
        a.u.template values<S>(us, r, u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const GateShares shares = gate_shares(g[r][v]);
            wide[r][v] = h[v] - u[v];
            scan_anew(wide[r][v]);
            h[v] = gate_step<true>(shares.a, h[v], share_of<true>(shares.c, u[v]));
        }
    }
    edges.fetch(rows.ends, rows.end, a.dlast, a.d, at);
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
    // (dy of two rows in one register, where it is of 16 bits)
    constexpr int PER = sizeof(T) == 2 ? 2 : 1;
    unsigned two[ROWS / PER];
#pragma unroll
    for (int i = 0; i < ROWS / PER; ++i) {
        two[i] = PER == 2 ? dys[i * PER] | dys[i * PER + PER - 1] << 16 : dys[i];
        scan_anew(two[i]);
    }
    auto dy_of = [&](int r, float (&dy)[V]) __attribute__((always_inline)) {
        if constexpr (PER == 1) at.values(two[r], dy);
        else if constexpr (__is_same(T, bf16)) dy[0] = __uint_as_float(r % 2 ? two[r / 2] & 0xffff0000u : two[r / 2] << 16);
        else {
            f16 v[2];
            __builtin_memcpy(v, &two[r / 2], 4);
            dy[0] = (float)v[r % 2];
        }
    };
    // x: what goes from a row to the one before, a G
    ScanProduct p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.f, 0.f};
    auto back = [&](int r, auto special, auto edge) __attribute__((always_inline)) {
        constexpr bool SPECIAL = decltype(special)::value;
        float dy[V];
        if (decltype(edge)::value && (rows.ends >> r & 1)) {
            float x[V];
            edges.get(r, x);
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] = {SCAN_STOP, x[v]};
        }
        dy_of(r, dy);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float share = gate_shares(g[r][v]).a;
            if (SPECIAL && (share == 0.f || (rows.none >> r & 1))) p[v] = {SCAN_STOP, 0.f};
            else p[v] = {p[v].a * share, share * (p[v].b + dy[v])};
        }
    };
    scan_each<ROWS, true>(closed, rows.ends, back);
    float x[V];
    told.template join<true>(a, q, block, rows.behind == ~0u ? q : a.tiles - 1 - (rows.behind - 1) / S::TILE, wave, p, x);
    if (many > 0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {                 // (not kept from the pass above)
            if (r % PER == 0) scan_anew(two[r / PER]);
#pragma unroll
            for (int v = 0; v < V; ++v) scan_anew(g[r][v]);
        }
        const unsigned starts = a.dh0 ? rows.starts : 0;
        T *df_row = a.df + (t0 + many - 1) * a.lddf + at.first, *du_row = a.du + (t0 + many - 1) * a.lddu + at.first;
        auto give = [&](int r, auto special, auto edge) __attribute__((always_inline)) {
            constexpr bool SPECIAL = decltype(special)::value, EDGE = decltype(edge)::value;
            if (SPECIAL && r >= many) return;
            if (EDGE && (rows.ends >> r & 1)) edges.get(r, x);
            float dy[V], df[V], du[V];
            dy_of(r, dy);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float G = x[v] + dy[v];
                const GateShares shares = gate_shares(g[r][v]);
                df[v] = share_of<SPECIAL>(shares.a * shares.c, G * wide[r][v]);
                du[v] = share_of<SPECIAL>(shares.c, G);
                x[v] = share_of<SPECIAL>(shares.a, G);
                if (SPECIAL && (rows.none >> r & 1)) df[v] = du[v] = x[v] = 0.f;
            }
            at.template store<SPECIAL>(df_row, df);
            at.template store<SPECIAL>(du_row, du);
            df_row -= a.lddf;
            du_row -= a.lddu;
            if (EDGE && (starts >> r & 1)) edges.put(r, x);
        };
        if (at.here()) scan_each<ROWS, true>(closed || many < ROWS, rows.ends | starts, give);
        edges.store(starts, rows.start, a.dh0, a.d, at);
    }
    scan_empty<S>(a.order, q, a.tiles, block == 0, a.flags, [&](int64_t j) {
        float x[V];
        if (!a.dh0) return;
        at.load_floats(a.dlast, j, a.d, x);
        at.store_floats(a.dh0, j, a.d, x);
    });
}

// state = a state + (1 - a) u, y = state, one row of every sequence.  A thread has one vector of a row.  The bound is the memory: 2048 x 4096 in bfloat16
// 20 to 22 us (5.4 to 5.9 TB/s); a few rows are a launch, 2.6 us for 4 x 1024.
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
