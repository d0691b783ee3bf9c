// Rows of a table looked up by token, and the gradient of the table by sorted tokens.
//
//   out[i] = scale table[id_i];  a negative id gives zeros
//   dtable[v] = scale sum over the i with id_i = v, in ascending i, of dout[i];  negative ids count nowhere
//
// The gradient first orders the tokens by id, those of one id by their place, so that the sums have one order whatever the
// timing.  Then `embed_grad_runs` goes through the sorted tokens in pieces of one length, whatever the popularity of the ids: it adds up the
// runs of equal ids in 32-bit floats and stores a table row where the run lies inside the piece; what a piece holds of a run
// that goes on into other pieces it leaves aside, and `embed_grad_join` adds these up.  Rows that no token has are stored as
// zeros by workgroups of the same launch.  The bound is the memory: dout is read once, the table's gradient written once.
#pragma once
#include "elements.hpp"

namespace chicle_train {

constexpr int EMBED_THREADS = 256;

// Thread groups of `lanes` take a row each; columns go in steps of lanes * VEC.
template <typename T>
__global__ __launch_bounds__(EMBED_THREADS) void embed_rows(const T *__restrict__ table, int64_t ld, int64_t n_rows, const void *__restrict__ ids,
                                                            int wide, T *__restrict__ out, int64_t ldo, int64_t n, int64_t d, int lanes, float scale, int *flags)
{
    constexpr int V = Elem<T>::VEC;
    const int64_t i = (int64_t)blockIdx.x * (EMBED_THREADS / lanes) + threadIdx.x / lanes;
    if (i >= n) return;
    const int64_t id = index_at(ids, wide, i);
    const bool has = id >= 0 && id < n_rows;
    if (id >= n_rows && threadIdx.x % lanes == 0 && flags) atomicOr(flags, FLAG_ID_RANGE);
    const T *src = table + (has ? id : 0) * ld;
    T *dst = out + i * ldo;
    for (int64_t c = (int64_t)(threadIdx.x % lanes) * V; c < d; c += (int64_t)lanes * V) {
        float u[V];
        if (has) load_vec(src, c, d, u);
#pragma unroll
        for (int k = 0; k < V; ++k) u[k] = has ? u[k] * scale : 0.f;
        store_vec(dst, c, d, u);
    }
}

// ---- tokens in the order of their ids -------------------------------------------------------------------------------

// Keys are the ids; one that is negative or past the table becomes n_rows, which sorts behind all rows.
__device__ __forceinline__ unsigned token_key(const void *ids, int wide, int64_t i, int64_t n_rows, int *flags)
{
    const int64_t id = index_at(ids, wide, i);
    if (id >= n_rows && flags) atomicOr(flags, FLAG_ID_RANGE);
    return id >= 0 && id < n_rows ? (unsigned)id : (unsigned)n_rows;
}

// The bit of every row that some token has.  Bits are only ever set, so a stale word costs an atomic and no more.
__device__ __forceinline__ void mark_row(unsigned *seen, unsigned key, int64_t n_rows)
{
    if (seen && (int64_t)key < n_rows) {
        const unsigned bit = 1u << (key & 31);
        if (!(__hip_atomic_load(&seen[key >> 5], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & bit)) atomicOr(&seen[key >> 5], bit);
    }
}

constexpr int SORT_ONE = 4096;               // tokens that one workgroup sorts by itself

// One workgroup: a bitonic network over (key, place) in LDS.
__global__ __launch_bounds__(1024) void sort_tokens_one(const void *__restrict__ ids, int wide, int n, int64_t n_rows, unsigned *__restrict__ keys_out,
                                                        unsigned *__restrict__ places_out, unsigned *seen, int64_t seen_words, int *flags)
{
    __shared__ unsigned long long s[SORT_ONE];
    int size = 1;
    while (size < n) size <<= 1;
    for (int i = threadIdx.x; i < size; i += 1024)
        s[i] = i < n ? ((unsigned long long)token_key(ids, wide, i, n_rows, flags) << 32) | (unsigned)i : ~0ull;
    if (seen)
        for (int64_t i = threadIdx.x; i < seen_words; i += 1024) seen[i] = 0u;
    __threadfence();
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = threadIdx.x; i < size / 2; i += 1024) {
                const int a = 2 * i - (i & (j - 1)), b = a + j;
                const unsigned long long x = s[a], y = s[b];
                if ((x > y) == ((a & k) == 0)) { s[a] = y; s[b] = x; }
            }
            __syncthreads();
        }
    for (int i = threadIdx.x; i < n; i += 1024) {
        const unsigned key = (unsigned)(s[i] >> 32);
        keys_out[i] = key;
        places_out[i] = (unsigned)s[i];
        if (i == 0 || (unsigned)(s[i - 1] >> 32) != key) mark_row(seen, key, n_rows);
    }
}

// More tokens: passes over digits of the key, the lowest first, each of which keeps the order of equal digits.  A workgroup
// takes SORT_TILE tokens, wavefront w of it the w-th quarter, 64 tokens at a time in their order.
constexpr int SORT_TILE = 2048, SORT_WAVES = 4, SORT_THREADS = 64 * SORT_WAVES, SORT_BITS = 10, SORT_BINS = 1 << SORT_BITS;

struct SortPass {
    const void *ids;             // first pass: the tokens themselves
    const unsigned *keys_in, *places_in;
    unsigned *keys_out, *places_out;
    unsigned *count;             // [bin][workgroup], then where the bin's tokens of the workgroup go
    unsigned *seen;              // last pass
    int64_t n, n_rows, seen_words;
    int wide, shift, bins, tiles, first, last;
    int *flags;
};

__device__ __forceinline__ unsigned sort_key(const SortPass &p, int64_t i, bool flag)
{
    return p.first ? token_key(p.ids, p.wide, i, p.n_rows, flag ? p.flags : nullptr) : p.keys_in[i];
}

// Every lane's number of lower lanes with the same digit, and the number of all lanes with it; lanes without a token have the
// digit `bins` or above and take part in nothing.
__device__ __forceinline__ void match_digit(unsigned digit, bool live, int bits, int &lower, int &all)
{
    unsigned long long same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long ones = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? ones : ~ones;
    }
    const int lane = threadIdx.x & 63;
    lower = __popcll(same & ((1ull << lane) - 1));
    all = __popcll(same);
}

__global__ __launch_bounds__(SORT_THREADS) void sort_count(SortPass p)
{
    __shared__ unsigned s[SORT_BINS];
    for (int i = threadIdx.x; i < p.bins; i += SORT_THREADS) s[i] = 0u;
    if (p.first && p.seen)
        for (int64_t i = (int64_t)blockIdx.x * SORT_THREADS + threadIdx.x; i < p.seen_words; i += (int64_t)gridDim.x * SORT_THREADS) p.seen[i] = 0u;
    __syncthreads();
    const int64_t a = (int64_t)blockIdx.x * SORT_TILE, end = min(p.n, a + SORT_TILE);
    for (int64_t i = a + threadIdx.x; i < end; i += SORT_THREADS) atomicAdd(&s[(sort_key(p, i, true) >> p.shift) & (p.bins - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < p.bins; i += SORT_THREADS) p.count[(int64_t)i * p.tiles + blockIdx.x] = s[i];
}

// Exclusive sums over bins * tiles counts, by one workgroup.
__global__ __launch_bounds__(1024) void sort_offsets(unsigned *count, int64_t total)
{
    __shared__ unsigned s[16];
    unsigned carry = 0;
    for (int64_t base = 0; base < total; base += 4096) {
        unsigned v[4], sum = 0;
        const int64_t at = base + (int64_t)threadIdx.x * 4;
        for (int k = 0; k < 4; ++k) { v[k] = at + k < total ? count[at + k] : 0u; sum += v[k]; }
        unsigned up = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned t = __shfl_up(up, o);
            if ((int)(threadIdx.x & 63) >= o) up += t;
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 63) s[threadIdx.x >> 6] = up;
        __syncthreads();
        unsigned before = carry + up - sum, all = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < (int)(threadIdx.x >> 6)) before += s[w];
            all += s[w];
        }
        carry += all;
        for (int k = 0; k < 4; ++k)
            if (at + k < total) { count[at + k] = before; before += v[k]; }
    }
}

__global__ __launch_bounds__(SORT_THREADS) void sort_scatter(SortPass p, int bits)
{
    __shared__ unsigned s[SORT_WAVES][SORT_BINS];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += SORT_THREADS) (&s[0][0])[i] = 0u;
    __syncthreads();
    constexpr int STEPS = SORT_TILE / SORT_THREADS;
    const int64_t a = (int64_t)blockIdx.x * SORT_TILE + wave * (SORT_TILE / SORT_WAVES);
    unsigned key[STEPS], rank[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const int64_t i = a + k * 64 + lane;
        const bool live = i < p.n;
        key[k] = live ? sort_key(p, i, false) : 0u;
        const unsigned digit = (key[k] >> p.shift) & (p.bins - 1);
        int lower, all;
        match_digit(digit, live, bits, lower, all);
        const unsigned before = s[wave][digit];
        rank[k] = before + lower;
        __builtin_amdgcn_wave_barrier();
        if (live && lower == 0) s[wave][digit] = before + all;
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.bins; i += SORT_THREADS) {
        unsigned t = p.count[(int64_t)i * p.tiles + blockIdx.x];
        for (int w = 0; w < SORT_WAVES; ++w) { const unsigned c = s[w][i]; s[w][i] = t; t += c; }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const int64_t i = a + k * 64 + lane;
        if (i >= p.n) continue;
        const unsigned at = s[wave][(key[k] >> p.shift) & (p.bins - 1)] + rank[k];
        p.keys_out[at] = key[k];
        p.places_out[at] = p.first ? (unsigned)i : p.places_in[i];
        if (p.last) mark_row(p.seen, key[k], p.n_rows);
    }
}

// ---- sums over runs of equal ids ------------------------------------------------------------------------------------

struct EmbedGrad {
    const unsigned *keys, *places, *seen;    // sorted; seen is null where the sums are added to what the table's gradient holds
    float *head, *tail;                      // [piece][d]: what a piece holds of a run that began before it, or that goes on behind it
    int64_t n, d, n_rows, ldo, ldd;
    int piece, lanes, run_blocks;            // tokens of a piece, threads of a piece
    float scale;
};

template <typename T>
__device__ __forceinline__ void give_row(const EmbedGrad &p, T *__restrict__ out, int64_t row, int64_t c, float *sum)
{
    constexpr int V = Elem<T>::VEC;
    T *dst = out + row * p.ldo;
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] *= p.scale;
    if (!p.seen) {
        float old[V];
        load_vec(dst, c, p.d, old);
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] += old[k];
    }
    store_vec(dst, c, p.d, sum);
}

// Workgroups [0, run_blocks): EMBED_THREADS / lanes pieces each, by blocks of lanes * VEC columns (blockIdx.y).  The rest: rows that no
// token has, 32 rows (a word of `seen`) at a time.
template <typename T>
__global__ __launch_bounds__(EMBED_THREADS) void embed_grad_runs(EmbedGrad p, const T *__restrict__ dout, T *__restrict__ out)
{
    constexpr int V = Elem<T>::VEC, AHEAD = 8;
    const int64_t c = ((int64_t)blockIdx.y * p.lanes + threadIdx.x % p.lanes) * V;
    if ((int)blockIdx.x >= p.run_blocks) {
        const int groups = EMBED_THREADS / p.lanes, group = threadIdx.x / p.lanes;
        const int64_t words = (p.n_rows + 31) / 32;
        if (c >= p.d) return;
        const float zero[V] = {};
        for (int64_t w = blockIdx.x - p.run_blocks; w < words; w += gridDim.x - p.run_blocks) {
            const unsigned seen = p.seen[w];
            for (int b = group; b < 32; b += groups) {
                const int64_t row = w * 32 + b;
                if (row < p.n_rows && !(seen >> b & 1)) store_vec(out + row * p.ldo, c, p.d, zero);
            }
        }
        return;
    }
    const int64_t piece = (int64_t)blockIdx.x * (EMBED_THREADS / p.lanes) + threadIdx.x / p.lanes;
    const int64_t a = piece * p.piece, end = min(p.n, a + p.piece);
    if (a >= p.n || c >= p.d) return;
    float sum[V] = {};
    unsigned key = p.keys[a];
    bool from_before = a > 0 && p.keys[a - 1] == key;
    for (int64_t t = a; t < end; t += AHEAD) {
        float u[AHEAD][V];
        unsigned ks[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const int64_t at = min(t + q, end - 1);
            ks[q] = p.keys[at];
            load_vec(dout + (int64_t)p.places[at] * p.ldd, c, p.d, u[q]);
        }
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            if (t + q >= end) break;
            if (ks[q] != key) {                          // the run before ends inside the piece
                if (from_before) {
                    if ((int64_t)key < p.n_rows)
#pragma unroll
                        for (int k = 0; k < V; ++k)
                            if (c + k < p.d) p.head[piece * p.d + c + k] = sum[k];
                } else if ((int64_t)key < p.n_rows) give_row(p, out, key, c, sum);
                key = ks[q];
                from_before = false;
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += u[q][k];
        }
    }
    if ((int64_t)key >= p.n_rows) return;
    const bool goes_on = end < p.n && p.keys[end] == key;
    if (!from_before && !goes_on) give_row(p, out, key, c, sum);
    else {
        float *dst = (from_before ? p.head : p.tail) + piece * p.d;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (c + k < p.d) dst[c + k] = sum[k];
    }
}

// Runs over several pieces: tail of the piece where the run begins, heads of the pieces up to the one where it ends.  A workgroup
// looks at one piece and one block of 64 * VEC columns; its wavefronts take every JOIN_WAVES-th of the run's pieces.
constexpr int JOIN_WAVES = 4;

template <typename T>
__global__ __launch_bounds__(64 * JOIN_WAVES) void embed_grad_join(EmbedGrad p, T *__restrict__ out)
{
    constexpr int V = Elem<T>::VEC;
    const int64_t piece = blockIdx.x, end = (piece + 1) * p.piece;
    if (end >= p.n) return;
    const unsigned key = p.keys[end - 1];
    if (p.keys[end] != key || (int64_t)key >= p.n_rows) return;
    const int64_t a = piece * p.piece;
    if (a > 0 && p.keys[a - 1] == key && p.keys[a] == key) return;     // the run began before: another piece's work
    int64_t lo = piece + 1, hi = (p.n - 1) / p.piece;                  // last piece that begins with this id
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (p.keys[mid * p.piece] == key) lo = mid;
        else hi = mid - 1;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = ((int64_t)blockIdx.y * 64 + lane) * V;
    float sum[V] = {};
    if (c < p.d)
        for (int64_t q = piece + wave; q <= lo; q += JOIN_WAVES) {
            const float *src = (q == piece ? p.tail : p.head) + q * p.d;
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (c + k < p.d) sum[k] += src[c + k];
        }
    __shared__ float s[JOIN_WAVES][64][V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[wave][lane][k] = sum[k];
    __syncthreads();
    if (wave || c >= p.d) return;
    for (int w = 1; w < JOIN_WAVES; ++w)
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] += s[w][lane][k];
    give_row(p, out, key, c, sum);
}

}  // namespace chicle_train
