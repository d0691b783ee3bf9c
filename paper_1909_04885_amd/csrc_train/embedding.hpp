// Rows of a table looked up by token, and the gradient of the table by sorted tokens.
//
//   out[i] = scale table[id_i];  a negative id gives zeros
//   dtable[v] = scale sum over the i with id_i = v of dout[i];  negative ids count nowhere
//
// The gradient first orders the tokens by id, those of one id by their place, so that the sums have one order whatever the
// timing: ascending i inside a piece, then the pieces, ascending too, or, of sixteen and more, sixteen sums of every sixteenth.  Then
// `embed_grad_runs` goes through the sorted tokens in pieces of one length, whatever the popularity of the ids: it adds up the runs of
// equal ids in 32-bit floats and stores a table row where the run lies inside the piece; what a piece holds of a run that goes on
// into other pieces it leaves aside, and `embed_grad_join` adds these up.  Rows that no token has are stored as zeros by
// workgroups of the same launch.
//
// The bound is the memory: dout is read once, the table's gradient written once.  Lookup of 16,001 x 2048 in half precision: 17 us
// (4.9 TB/s).  Gradient of 131,072 tokens into 128,000 x 2048 in bfloat16: 229 us (4.6 TB/s; sorting 36, sums and zeros 173, joining 20);
// of 30,011 into 200,000 x 256 in 32 bits: 72 us (3.3 TB/s; sorting 29).  Below some thousand tokens four launches and the passes of
// the sort are what it takes: 64 tokens of 256 into 32,000 rows 19 us.
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

// seen[v] = 1 for every row v that some token has: all who mark a row store the same byte.  seen_bytes is a multiple of sixteen.
__device__ __forceinline__ void clear_seen(uint8_t *seen, int64_t seen_bytes, int64_t thread, int64_t threads)
{
    if (seen)
        for (int64_t i = thread * 16; i < seen_bytes; i += threads * 16) *(u32x4 *)(seen + i) = u32x4{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ void mark_seen(uint8_t *seen, unsigned key, int64_t n_rows)
{
    if (seen && (int64_t)key < n_rows) seen[key] = 1;
}

constexpr int SORT_BITS = 10, SORT_BINS = 1 << SORT_BITS;      // of a digit

// Every lane's number of lower lanes with the same digit, and the number of all lanes with it; lanes without a token count nowhere.
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

// As many tokens as one workgroup sorts by itself, in one launch: passes over digits of the key, the lowest first, each of which keeps the order
// of equal digits.  A wavefront holds STEPS times 64 tokens in their order; where its tokens of a digit go follows from what the
// wavefronts hold of every digit.
constexpr int SORT_ONE_THREADS = 1024, SORT_ONE_WAVES = SORT_ONE_THREADS / 64, SORT_ONE = 4 * SORT_ONE_THREADS;

template <int STEPS>
__global__ __launch_bounds__(SORT_ONE_THREADS) void sort_tokens_one(const void *__restrict__ ids, int wide, int n, int64_t n_rows, int passes, int bits,
                                                                    unsigned *__restrict__ keys_out, unsigned *__restrict__ places_out, uint8_t *seen,
                                                                    int64_t seen_bytes, int *flags)
{
    constexpr int ALL = STEPS * SORT_ONE_THREADS;
    __shared__ unsigned keys[ALL];
    __shared__ uint16_t places[ALL];
    __shared__ uint16_t count[SORT_ONE_WAVES][SORT_BINS];
    __shared__ unsigned totals[SORT_ONE_WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = wave * 64 * STEPS + lane, bin = threadIdx.x, mask = (1 << bits) - 1;
    unsigned key[STEPS];
    int place[STEPS], rank[STEPS];
    clear_seen(seen, seen_bytes, threadIdx.x, SORT_ONE_THREADS);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        place[s] = first + s * 64;
        key[s] = place[s] < n ? token_key(ids, wide, place[s], n_rows, flags) : 0u;
    }
    __syncthreads();                                     // (cleared before anything is marked)
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
        if (place[s] < n) mark_seen(seen, key[s], n_rows);
    for (int pass = 0; pass < passes; ++pass) {
        for (int i = threadIdx.x; i < SORT_ONE_WAVES * SORT_BINS / 2; i += SORT_ONE_THREADS) ((unsigned *)&count[0][0])[i] = 0u;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int digit = key[s] >> (pass * bits) & mask;
            int lower, all;
            match_digit(digit, first + s * 64 < n, bits, lower, all);
            rank[s] = count[wave][digit] + lower;
            __builtin_amdgcn_wave_barrier();
            if (first + s * 64 < n && lower == 0) count[wave][digit] = (uint16_t)(rank[s] + all);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        unsigned sum = 0;
        for (int w = 0; w < SORT_ONE_WAVES; ++w) sum += count[w][bin];
        unsigned up = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned t = __shfl_up(up, o);
            if (lane >= o) up += t;
        }
        if (lane == 63) totals[wave] = up;
        __syncthreads();
        unsigned at = up - sum;
        for (int w = 0; w < wave; ++w) at += totals[w];
        for (int w = 0; w < SORT_ONE_WAVES; ++w) { const unsigned c = count[w][bin]; count[w][bin] = (uint16_t)at; at += c; }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            if (first + s * 64 < n) {
                const int to = count[wave][key[s] >> (pass * bits) & mask] + rank[s];
                keys[to] = key[s];
                places[to] = (uint16_t)place[s];
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            if (first + s * 64 < n) { key[s] = keys[first + s * 64]; place[s] = places[first + s * 64]; }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
        if (first + s * 64 < n) { keys_out[first + s * 64] = key[s]; places_out[first + s * 64] = place[s]; }
}

// More tokens: passes over digits of the key, the lowest first, each of which keeps the order of equal digits.  A workgroup
// takes a tile of tokens, wavefront w of it the w-th part, 64 tokens at a time in their order.  There are at most
// SORT_MOST_TILES tiles: every workgroup adds up by itself what the tiles before it hold of each digit, which saves a launch
// between the counts and the scatter.
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES;
constexpr int SORT_LEAST_TILE = 2048, SORT_MOST_TILES = 128;

struct SortPass {
    const void *ids;             // first pass: the tokens themselves
    const unsigned *keys_in, *places_in;
    unsigned *keys_out, *places_out;
    unsigned *count;             // [tile][bin]
    int64_t n, n_rows, tile;     // tokens of a tile: a multiple of SORT_THREADS
    int wide, shift, bits, tiles, first;
    int *flags;
    uint8_t *seen;               // null where no rows are filled with zeros
    int64_t seen_bytes;
};

__device__ __forceinline__ unsigned sort_key(const SortPass &p, int64_t i, bool flag)
{
    return p.first ? token_key(p.ids, p.wide, i, p.n_rows, flag ? p.flags : nullptr) : p.keys_in[i];
}

__global__ __launch_bounds__(SORT_THREADS) void sort_count(SortPass p)
{
    __shared__ unsigned s[SORT_BINS];
    const int bins = 1 << p.bits;
    for (int i = threadIdx.x; i < bins; i += SORT_THREADS) s[i] = 0u;
    __syncthreads();
    if (p.first) clear_seen(p.seen, p.seen_bytes, (int64_t)blockIdx.x * SORT_THREADS + threadIdx.x, (int64_t)gridDim.x * SORT_THREADS);
    const int64_t a = (int64_t)blockIdx.x * p.tile, end = min(p.n, a + p.tile);
    for (int64_t i = a + threadIdx.x; i < end; i += SORT_THREADS) atomicAdd(&s[(sort_key(p, i, true) >> p.shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += SORT_THREADS) p.count[(int64_t)blockIdx.x * bins + i] = s[i];
}

__global__ __launch_bounds__(SORT_THREADS) void sort_scatter(SortPass p)
{
    __shared__ unsigned s[SORT_WAVES][SORT_BINS];        // a wavefront's tokens of a digit, then where its next one goes
    __shared__ unsigned totals[SORT_WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, bins = 1 << p.bits, mask = bins - 1;
    for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += SORT_THREADS) (&s[0][0])[i] = 0u;
    __syncthreads();
    const int64_t part = p.tile / SORT_WAVES, a = (int64_t)blockIdx.x * p.tile + wave * part, end = min(p.n, a + part);
    for (int64_t i = a + lane; i < end; i += 64) atomicAdd(&s[wave][(sort_key(p, i, false) >> p.shift) & mask], 1u);
    // Two neighbouring bins to a thread: what earlier tiles hold of them, and what all tiles do.
    constexpr int EACH = SORT_BINS / SORT_THREADS;
    unsigned before[EACH] = {}, total[EACH] = {}, sum = 0;
    constexpr int BATCH = 16;                            // tiles whose counts are asked for together
    if ((int)threadIdx.x * EACH < bins)
        for (int t = 0; t < p.tiles; t += BATCH) {
            unsigned c[BATCH][EACH];
#pragma unroll
            for (int q = 0; q < BATCH; ++q)
#pragma unroll
                for (int k = 0; k < EACH; ++k) c[q][k] = p.count[min(t + q, p.tiles - 1) * bins + min((int)threadIdx.x * EACH + k, mask)];
#pragma unroll
            for (int q = 0; q < BATCH; ++q)
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const unsigned v = t + q < p.tiles && (int)threadIdx.x * EACH + k < bins ? c[q][k] : 0u;
                    total[k] += v;
                    if (t + q < (int)blockIdx.x) before[k] += v;
                }
        }
#pragma unroll
    for (int k = 0; k < EACH; ++k) sum += total[k];
    unsigned up = sum;
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned t = __shfl_up(up, o);
        if (lane >= o) up += t;
    }
    if (lane == 63) totals[wave] = up;
    __syncthreads();
    unsigned at = up - sum;
    for (int w = 0; w < wave; ++w) at += totals[w];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int bin = threadIdx.x * EACH + k;
        unsigned t = at + before[k];
        if (bin < bins)
            for (int w = 0; w < SORT_WAVES; ++w) { const unsigned c = s[w][bin]; s[w][bin] = t; t += c; }
        at += total[k];
    }
    __syncthreads();
    for (int64_t base = a; base < end; base += 64) {
        const int64_t i = base + lane;
        const bool live = i < end;
        const unsigned key = live ? sort_key(p, i, false) : 0u, digit = (key >> p.shift) & mask;
        int lower, all;
        match_digit(digit, live, p.bits, lower, all);
        const unsigned next = s[wave][digit];
        __builtin_amdgcn_wave_barrier();
        if (live && lower == 0) s[wave][digit] = next + all;
        __builtin_amdgcn_wave_barrier();
        if (live) {
            p.keys_out[next + lower] = key;
            p.places_out[next + lower] = p.first ? (unsigned)i : p.places_in[i];
            if (p.first) mark_seen(p.seen, key, p.n_rows);
        }
    }
}

// ---- sums over runs of equal ids ------------------------------------------------------------------------------------

constexpr int ZERO_BYTES = 16384;            // of the rows that a workgroup fills with zeros
constexpr int ZERO_AHEAD = 4;

struct EmbedGrad {
    const unsigned *keys, *places;           // sorted
    float *head, *tail;                      // [piece][ldp]: what a piece holds of a run that began before it, or that goes on behind it
    int64_t n, d, n_rows, ldo, ldd, ldp;
    int piece, lanes;                        // tokens and threads of a piece
    int run_blocks, zero_blocks, zero_rows;  // zero_rows: to a workgroup
    int accumulate;
    const uint8_t *seen;
    float scale;
};

template <typename T>
__device__ __forceinline__ void give_row(const EmbedGrad &p, T *__restrict__ out, int64_t row, int64_t c, float *sum)
{
    constexpr int V = Elem<T>::VEC;
    T *dst = out + row * p.ldo;
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] *= p.scale;
    if (p.accumulate) {
        float old[V];
        load_vec(dst, c, p.d, old);
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] += old[k];
    }
    store_vec(dst, c, p.d, sum);
}

// Zeros for the rows that no token has, a few rows to a workgroup: neighbouring workgroups then store side by side, which is faster than
// long stretches of rows each (524 MB in 75 instead of 144 us).
template <typename T>
__device__ __forceinline__ void zero_rows(const EmbedGrad &p, int block, int64_t c, T *__restrict__ out)
{
    constexpr int V = Elem<T>::VEC;
    const int groups = EMBED_THREADS / p.lanes;
    const float zero[V] = {};
    const int64_t r0 = (int64_t)block * p.zero_rows, end = min(p.n_rows, r0 + p.zero_rows);
    if (c >= p.d) return;
    for (int64_t row = r0 + threadIdx.x / p.lanes; row < end; row += ZERO_AHEAD * groups) {
        bool seen[ZERO_AHEAD];                           // (asked for together)
#pragma unroll
        for (int q = 0; q < ZERO_AHEAD; ++q) seen[q] = row + q * groups >= end || p.seen[row + q * groups];
#pragma unroll
        for (int q = 0; q < ZERO_AHEAD; ++q)
            if (!seen[q]) store_vec<T, true>(out + (row + q * groups) * p.ldo, c, p.d, zero);
    }
}

// The work of run_blocks workgroups that add up pieces of tokens, EMBED_THREADS / lanes pieces each, and then of zero_blocks that store
// zeros: the pieces' long chains begin first and end among the others (30011 tokens into 200000 x 256: 76 us; in turn, 88).  blockIdx.y:
// blocks of lanes * VEC columns of the pieces.
template <typename T>
__global__ __launch_bounds__(EMBED_THREADS) void embed_grad_runs(EmbedGrad p, const T *__restrict__ dout, T *__restrict__ out)
{
    constexpr int V = Elem<T>::VEC, AHEAD = 16;
    extern __shared__ uint2 tokens[];                    // (id, place) of the workgroup's pieces
    const int64_t b = blockIdx.x;
    if (b >= p.run_blocks) {
        zero_rows(p, (int)(b - p.run_blocks), ((int64_t)blockIdx.y * p.lanes + threadIdx.x % p.lanes) * V, out);
        return;
    }
    const int groups = EMBED_THREADS / p.lanes, group = threadIdx.x / p.lanes;
    const int64_t piece0 = b * groups, t0 = piece0 * p.piece;
    for (int i = threadIdx.x; i < groups * p.piece && t0 + i < p.n; i += EMBED_THREADS) tokens[i] = make_uint2(p.keys[t0 + i], p.places[t0 + i]);
    const int64_t piece = piece0 + group, a = piece * p.piece;
    const int many = (int)min((int64_t)p.piece, p.n - a);
    const unsigned before = many > 0 && a > 0 ? p.keys[a - 1] : 0u, after = many > 0 && a + many < p.n ? p.keys[a + many] : 0u;
    __syncthreads();
    const int64_t c = ((int64_t)blockIdx.y * p.lanes + threadIdx.x % p.lanes) * V;
    if (many <= 0 || c >= p.d) return;
    const uint2 *mine = tokens + group * p.piece;
    float sum[V] = {};
    unsigned key = mine[0].x;
    bool from_before = a > 0 && before == key;
    auto leave = [&](float *part) {
        float *dst = part + piece * p.ldp + c;           // (rows of parts are padded to whole vectors)
#pragma unroll
        for (int k = 0; k < V; k += 4) *(float4 *)(dst + k) = make_float4(sum[k], sum[k + 1], sum[k + 2], sum[k + 3]);
    };
    for (int t = 0; t < many; t += AHEAD) {
        u32x4 u[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
            u[q] = ask_raw<T, true>(dout + (int64_t)mine[min(t + q, many - 1)].y * p.ldd, c, p.d);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            if (t + q >= many) break;
            const unsigned next = mine[t + q].x;
            if (next != key) {                           // the run before ends inside the piece
                if ((int64_t)key < p.n_rows) {
                    if (from_before) leave(p.head);
                    else give_row(p, out, key, c, sum);
                }
                key = next;
                from_before = false;
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] = 0.f;
            }
            float w[V];
            unpack<T>(settle<T>(u[q], c, p.d), w);
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += w[k];
        }
    }
    if ((int64_t)key >= p.n_rows) return;
    const bool goes_on = a + many < p.n && after == key;
    if (from_before) leave(p.head);
    else if (goes_on) leave(p.tail);
    else give_row(p, out, key, c, sum);
}

// Runs over several pieces: tail of the piece where the run begins, heads of the pieces up to the one where it ends.  A workgroup
// looks at JOIN_PIECES pieces and one block of JOIN_COLUMNS columns.  A wavefront adds up the run that begins in its piece, or, where
// that is long, all wavefronts take its pieces in turn.
constexpr int JOIN_WAVES = 16, JOIN_PIECES = JOIN_WAVES, JOIN_LONG = 16, JOIN_COLUMNS = 256;

// The sum of the parts of pieces first, first + step, .. up to last of the run that begins in piece `begin`, four columns to a lane.
__device__ __forceinline__ float4 sum_of_parts(const EmbedGrad &p, int64_t begin, int64_t first, int64_t last, int step, int64_t c)
{
    constexpr int AHEAD = 8;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t q = first; q <= last; q += (int64_t)step * AHEAD) {
        float4 u[AHEAD];
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            const int64_t at = min(q + h * step, last);
            u[h] = *(const float4 *)((at == begin ? p.tail : p.head) + at * p.ldp + c);
        }
#pragma unroll
        for (int h = 0; h < AHEAD; ++h)
            if (q + h * step <= last) { sum.x += u[h].x; sum.y += u[h].y; sum.z += u[h].z; sum.w += u[h].w; }
    }
    return sum;
}

// The last piece behind `piece` that begins with `key`; the one behind does.  Sorted: those that begin with it come first.
__device__ __forceinline__ int64_t last_piece(const EmbedGrad &p, int64_t piece, int64_t pieces, unsigned key, int lane)
{
    int64_t last = piece + 1;
    for (int stride = 64 * 64; stride >= 1; stride /= 64)
        for (;;) {                                       // sixty-four probes, a stride apart
            const int64_t at = last + (int64_t)(lane + 1) * stride;
            const unsigned long long same = __ballot(at < pieces && p.keys[min(at, pieces - 1) * p.piece] == key);
            last += (int64_t)__popcll(same) * stride;
            if (~same) break;
        }
    return last;
}

template <typename T>
__device__ __forceinline__ void give_columns(const EmbedGrad &p, T *__restrict__ out, int64_t row, int64_t c, float4 sum)
{
    T *dst = out + row * p.ldo + c;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < p.d) dst[k] = (T)(v[k] * p.scale + (p.accumulate ? (float)dst[k] : 0.f));
}

template <typename T>
__global__ __launch_bounds__(64 * JOIN_WAVES) void embed_grad_join(EmbedGrad p, T *__restrict__ out)
{
    __shared__ float4 s[JOIN_WAVES][64];
    __shared__ int64_t lasts[JOIN_WAVES];                // last piece of a long run, or 0
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.y * JOIN_COLUMNS + lane * 4, pieces = (p.n + p.piece - 1) / p.piece;
    const int64_t piece = (int64_t)blockIdx.x * JOIN_PIECES + wave, a = piece * p.piece, end = a + p.piece;
    int64_t last = 0;
    unsigned key = 0;
    if (end < p.n) {
        key = p.keys[end - 1];
        const bool began_before = a > 0 && p.keys[a] == key && p.keys[a - 1] == key;
        if (p.keys[end] == key && (int64_t)key < p.n_rows && !began_before) last = last_piece(p, piece, pieces, key, lane);
    }
    const bool is_long = last - piece >= JOIN_LONG;
    if (lane == 0) lasts[wave] = is_long ? last : 0;
    if (last > 0 && !is_long && c < p.d) give_columns(p, out, key, c, sum_of_parts(p, piece, piece, last, 1, c));
    __syncthreads();
    for (int w = 0; w < JOIN_WAVES; ++w) {
        const int64_t begin = (int64_t)blockIdx.x * JOIN_PIECES + w;
        last = lasts[w];
        if (last == 0) continue;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < p.d) sum = sum_of_parts(p, begin, begin + wave, last, JOIN_WAVES, c);
        s[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && c < p.d) {
            for (int v = 1; v < JOIN_WAVES; ++v) {
                const float4 t = s[v][lane];
                sum.x += t.x; sum.y += t.y; sum.z += t.z; sum.w += t.w;
            }
            give_columns(p, out, p.keys[last * p.piece], c, sum);
        }
        __syncthreads();
    }
}

}  // namespace chicle_train
