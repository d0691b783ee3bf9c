// Entry points of include/chicle_train.h: checks of arguments, workspace layout, launches.
#include <hip/hip_runtime.h>
#include <string.h>
#include <algorithm>
#include <memory>
#include <new>
#include "../../include/chicle_train.h"
#include "clip.hpp"
#include "elements.hpp"
#include "embedding.hpp"
#include "entry.hpp"
#include "layer_norm.hpp"
#include "softmax_loss.hpp"

using namespace chicle_train;

namespace {

constexpr int64_t CLIP_PIECE = 8192;                     // values of a tensor that a workgroup takes at a time
constexpr int64_t CLIP_FEW_PIECES = 4096;                // up to here the norm costs the scaling workgroups less than a launch

// Whether two of the tensors that are written overlap: workgroups would scale there beside each other, each what another may have scaled.
int check_apart(void *const *out, const int64_t *sizes, const int32_t *types, int count)
{
    struct Range { uintptr_t begin, end; };
    std::unique_ptr<Range[]> r(new (std::nothrow) Range[count]);
    if (!r) return fail(CHICLE_ENOMEM, "no host memory for %d tensors", count);
    int many = 0;
    for (int k = 0; k < count; ++k)
        if (sizes[k] > 0) r[many++] = {(uintptr_t)out[k], (uintptr_t)out[k] + (uintptr_t)sizes[k] * size_of(types[k])};
    std::sort(r.get(), r.get() + many, [](const Range &a, const Range &b) { return a.begin < b.begin; });
    for (int k = 1; k < many; ++k)
        if (r[k].begin < r[k - 1].end) return fail(CHICLE_EINVAL, "memory that is written twice, by tensors that overlap");
    return CHICLE_OK;
}

// ---- layer norm -----------------------------------------------------------------------------------------------------

constexpr int LN_FORWARD_VALUES = 32, LN_GRAD_VALUES = 16;
// Workgroups of the gradient: whole rounds of what the compute units hold at once, up to this many.  At 65,536 x 4096 in 16 bits,
// where 768 are held, 768 take 306 us and 1024 (a round and a third) 390 us.  In us, up to 256 / 512 / 768 / this many: 65,536 x 4096 in 16 bits
// 599 / 345 / 298 / 298, 30,000 x 4096 in 32 bits 330 / 255 / 253 / 263, 9001 x 1537 88 / 55 / 50 / 48, 4096 x 1024 32 / 23 / 23 / 23.  What it costs is the
// parts' bytes in short batches of wide rows: 4096 x 4096 in 16 bits 52 / 44 / 47 / 47, in 32 58 / 52 / 52 / 64, 1024 x 16,384 in 16 bits 59 / 88 / 117 / 150.
constexpr int LN_GRAD_GRID = 1024;

int64_t layer_norm_parts(int64_t n, int64_t d, int32_t type)
{
    const RowShape s = row_shape(d, 16 / size_of(type), LN_GRAD_VALUES, LN_GRAD_VALUES);
    const int64_t g = ceil_div(n, s.threads / s.lanes);
    return g < LN_GRAD_GRID ? g : LN_GRAD_GRID;
}

// ---- products -------------------------------------------------------------------------------------------------------

// The long side of a wavefront's part lies along j where A lies by k, since turning costs reads, and along i for the loss, whose sums go
// along i.
typedef MmConfig<256, 256, 2, 4, 1> MmWide;
typedef MmConfig<256, 256, 4, 2, 1> MmWideByK;
typedef MmConfig<128, 128, 2, 2, 2> MmMiddle;
typedef MmConfig<128, 64, 2, 2, 3> MmThin;
constexpr int MM_PARTS_I = 2;                            // wavefronts along i of the loss's tiles

enum { WIDE, MIDDLE, THIN };

int mm_tile_i(int c) { return c == WIDE ? 256 : 128; }
int mm_tile_j(int c) { return c == WIDE ? 256 : c == MIDDLE ? 128 : 64; }

// 16 bits: large tiles read the least and feed the matrix cores best (1300 against 1000 TFLOP/s of the middle ones), where they fill the chip:
// losses of 512 rows of 1024 and 16,000 classes (126 large tiles) 25 us in middle and 69 in large ones, 700 rows and 20,000 (237) 44 and 41.
// 32 bits: the matrix cores are the bound whatever the tile, and what counts is how much of the tiles lies past the last row, and that they share
// out well: gradients of 333 rows of 250 and 20,000 classes 168 us in middle and 160 in thin tiles, 1000 rows of 1024 and 10,000 597 and
// 578, 4096 rows of 512 and 30,000 3323 and 3481 (tiles of 64 x 64: 163, 616, 3670).
// `splittable`: the sum is long and may be divided, from 256 slices on.  Gradients in us, middle / large tiles, 1024 columns: 512 rows (8 large tiles) and
// 50,000 classes 405 / 401, 2048 rows (32) 1386 / 1314, 4096 rows (64) 2656 / 2500, with 16,000 classes (500 slices) 848 / 803, with 12,000
// (375) 661 / 661, with 6000 (188) 365 / 361.
int mm_choose(int size, int64_t rows_i, int64_t rows_j, bool splittable = false)
{
    if (rows_j <= 64) return THIN;
    const int64_t tiles = ceil_div(rows_i, 256) * ceil_div(rows_j, 256);
    if (size == 2) return tiles >= (splittable ? 32 : 192) ? WIDE : MIDDLE;
    const int64_t middle = ceil_div(rows_j, 128);
    return middle * 2 == ceil_div(rows_j, 64) && middle * ceil_div(rows_i, 128) >= 4 * CUS ? MIDDLE : THIN;
}

// f(C()) with the tile; W is the large one of the 16-bit types
template <typename T, typename W, typename F>
int with_config(int c, F f)
{
    if constexpr (sizeof(T) == 2)
        if (c == WIDE) return f(W());
    return c == MIDDLE ? f(MmMiddle()) : f(MmThin());
}

// ---- softmax loss: where everything lies ------------------------------------------------------------------------------

struct LossPlan {
    int64_t n, d, classes, ldk;          // ldk: length of laid-out rows along d
    int config;
    bool few, few_grad, tiles, kept, lay_x, lay_w;   // few: of the loss, of the gradient; tiles: something goes by products; kept: the logits
    int loss_splits;                     // of the loss's sums, more than 1 where tiles are few
    int few_blocks, few_passes, few_chunk, few_lds, few_each, few_grad_blocks;
    // gradient: pieces of the classes, or, with logits kept, of the rows
    int64_t piece, piece_rows, ldz, ldg, ldp;        // ldz, ldg: length of the rows of the logits and of G; ldp: of the rows of dx's parts
    int64_t rows_x, rows_g;                          // rows of the laid-out x and of G: whole slices
    int pieces, splits, config_dx, config_dw;
    void *x, *w, *g;
    float *logits, *parts, *rest_parts, *lse, *picked, *power;
    float2 *tile_sums;
    size_t bytes;
};

// 8192 rows of 2048 and 128,000 classes in 16 bits with a quarter of it: 23.0 ms, this 23.0, four times as much 23.3.
constexpr int64_t LOSS_PIECE_BYTES = (int64_t)1 << 30;   // both planes of G of a piece of the classes, or more of long batches
// 16,384 rows of 512 and 50,000 classes in 32 bits with a quarter of it: 24.1 ms, this 22.4, four times as much 22.3.
constexpr int64_t LOSS_KEPT_BYTES = (int64_t)1 << 30;    // logits of a piece of the rows
constexpr int64_t LOSS_MOST = (int64_t)1 << 22, LOSS_MOST_D = (int64_t)1 << 21, LOSS_MOST_CLASSES = (int64_t)1 << 23;

// Rows 1024 bytes apart, or a multiple of that, meet in few channels of the L2: half a slice more.
int64_t spread(int64_t ld, int size) { return ld * size % 1024 == 0 ? ld + MM_ROW / size : ld; }

// Classes at the end of a piece whose tiles of dw are split: those past the last whole round of tiles, where they are less than half a round
// (the gradients of 4096 rows of 1024 and 50,021 classes 2503 instead of 2676 us).
int64_t dw_rest(int config, int64_t d, int64_t classes, int64_t slices)
{
    const int64_t across = ceil_div(d, 256), tiles = across * ceil_div(classes, 256), over = tiles % CUS;
    if (config != WIDE || tiles < CUS || over == 0 || over * 2 > CUS || slices < 16) return 0;
    const int64_t rest = classes - tiles / CUS * CUS / across * 256;
    return across * ceil_div(rest, 256) * 2 > CUS ? 0 : rest;
}

// Up to how many rows the loss reads w as it lies instead of by products; with the gradient too, so that both give the same loss.
// In us, 50,000 classes, as it lies / by products.  16 bits, w aligned: 4 rows of 1024 33 / 25, 64 rows 48 / 26; w not aligned, so that products need
// it laid out first: 1 row of 1001 46 / 60, 33 rows 55 / 62, but with the gradient, which needs that anyway, 16 rows 168 / 144.
// 32 bits, aligned: 16 rows of 1024 60 / 86, 24 rows 86 / 84; not aligned: 32 rows of 1001 94 / 149, with the gradient 323 / 303, 48 rows
// 134 / 150 and 392 / 329.
int64_t few_rows(int size, bool aligned)
{
    if (size == 4) return aligned ? FEW_ROWS / 2 : FEW_ROWS;
    return aligned ? 0 : FEW_ROWS / 2;
}

LossPlan loss_plan(const void *x, int64_t ldx, const void *w, int64_t ldw, int64_t n, int64_t d, int64_t classes, int32_t type, bool grad, void *workspace)
{
    LossPlan p = {};
    p.bytes = ALIGN;
    if (n == 0) return p;                                // (nothing to lay out)
    p.n = n; p.d = d; p.classes = classes;
    const int size = size_of(type), planes = size == 2 ? MM_PLANES<bf16, true> : MM_PLANES<float, true>;
    const int64_t slice = MM_ROW / size;
    // rows that are whole slices of aligned chunks are read where they are
    auto as_is = [&](const void *q, int64_t ld) { return d % slice == 0 && ld * size % 16 == 0 && (uintptr_t)q % 16 == 0 && ld < LOSS_MOST_D; };
    p.few = n <= few_rows(size, as_is(w, ldw));
    // (16 bits: 4 rows of 1024 and 50,000 classes 78 us this way, 116 by products, 8 rows 109 and 117, of 4096 and 8000 classes 118 and 92, of 1001 and
    // 50,000 188 and 166; 32 bits: 8 rows 167 and 208)
    p.few_grad = grad && n <= (size == 4 ? FEW_GRAD_ROWS : FEW_GRAD_ROWS / 2);
    p.config = mm_choose(size, classes, n);
    p.loss_splits = 1;
    if (!p.few) {
        // Tiles that leave much of the chip idle, and sums long enough to be divided.  In us, divided / not, 16 bits: 128 rows of 4096 and
        // 1000 classes (8 tiles) 19 / 45, 256 and 3000 (48) 37 / 47, 8000 classes of 128 rows (63) 49 / 46, of 256 rows of 2048 (126) 39 / 28.
        // 32 bits: 512 rows of 2048 and 4000 classes (128) 91 / 144.
        const int64_t tiles = ceil_div(classes, mm_tile_i(p.config)) * ceil_div(n, mm_tile_j(p.config)), slices = ceil_div(d, slice), room = 2 * CUS;
        if (tiles * (size == 4 ? 1 : 4) <= CUS && slices >= 16) {
            const int64_t most = room / tiles < slices / 4 ? room / tiles : slices / 4;
            p.loss_splits = (int)ceil_div(slices, ceil_div(slices, most));
        }
    }
    p.kept = grad && (p.few || size == 4 || p.config != WIDE);
    p.tiles = !p.few || (grad && !p.few_grad);
    p.lay_w = p.tiles && !as_is(w, ldw);
    p.piece_rows = n;
    Carver c(workspace);
    p.picked = c.take<float>(n);
    if (grad) p.lse = c.take<float>(n);
    if (p.few) {
        const int64_t batch = slice / 2 * FEW_AHEAD, all = round_up(d, batch), per_column = n * size, spare = 16 / size;
        p.few_chunk = (int)all;
        if ((all + spare) * per_column > 72 * 1024) p.few_chunk = (int)((72 * 1024 / per_column - spare) / batch * batch);
        const int64_t sums = FEW_THREADS / 64 * FEW_ROWS * (int64_t)sizeof(float2), lds = (p.few_chunk + spare) * per_column;
        p.few_lds = (int)(lds > sums ? lds : sums);
        const int64_t blocks = ceil_div(ceil_div(classes, 16), FEW_THREADS / 64);
        p.few_blocks = (int)(blocks < 2048 ? blocks : 2048);
        p.few_passes = (int)ceil_div(blocks, p.few_blocks);
        p.tile_sums = c.take<float2>(n * p.few_blocks);
    }
    p.ldz = round_up(classes, 256) + 32;                 // (whole tiles, and not a multiple of 1024 bytes)
    if (p.kept && !p.few && p.loss_splits == 1) {        // as many rows as the logits have room for, at least a tile's
        const int64_t most = LOSS_KEPT_BYTES / (p.ldz * 4) / 256 * 256;
        p.pieces = (int)ceil_div(n, most < 256 ? 256 : most);
        p.piece_rows = round_up(ceil_div(n, p.pieces), 256);
        p.pieces = (int)ceil_div(n, p.piece_rows);
        if (p.piece_rows > n) p.piece_rows = n;
    }
    if (p.few_grad) {
        p.few_each = (int)(round_up(ceil_div(classes, 1024), 8));
        p.few_grad_blocks = (int)ceil_div(classes, p.few_each);
        p.ldp = round_up(d, 8);
        p.logits = c.take<float>(n * p.ldz * p.loss_splits);
        p.parts = c.take<float>(p.few_grad_blocks * n * p.ldp);
    }
    if (p.loss_splits > 1 && !grad) p.logits = c.take<float>(n * p.ldz * p.loss_splits);
    if (!p.few && p.loss_splits == 1) p.tile_sums = c.take<float2>(p.piece_rows * ceil_div(classes, mm_tile_i(p.config)) * MM_PARTS_I);
    if (p.tiles) {
        p.ldk = spread(round_up(d, slice), size);
        p.rows_x = grad ? round_up(n, slice) : n;
        // (rows without a label are zeros for the product over rows; and x is read often where there are many rows)
        p.lay_x = grad || !as_is(x, ldx) || (p.config == WIDE && spread(ldx, size) != ldx);
        p.x = p.lay_x ? c.take<char>(p.rows_x * p.ldk * size) : (char *)x;
        p.w = p.lay_w ? c.take<char>(classes * p.ldk * size) : (char *)w;
    }
    if (grad && !p.few_grad) {
        p.power = c.take<float>(2);
        if (p.kept) {
            p.piece = classes;
            if (p.few || p.loss_splits > 1) p.pieces = 1;
        } else {
            // At least a round of dw's large tiles to a piece, or eight classes to a column, so that long batches do not come in small pieces: 65,536
            // rows of 1024 and 128,000 classes 143 ms without (4096 classes to a piece), 105 with (8192), 131,072 rows of 1024 438 and 210, of 512
            // (64,000 classes) 191 and 116, 65,536 rows of 2048 99 and 92.
            const int64_t least = std::min<int64_t>(8 * d, CUS * 256 * 256 / d);
            int64_t most = std::max(LOSS_PIECE_BYTES / (planes * size * p.rows_x), least) / 256 * 256;
            most = most < 256 ? 256 : most;
            p.pieces = (int)ceil_div(classes, most);
            p.piece = round_up(ceil_div(classes, p.pieces), 256);
            p.pieces = (int)ceil_div(classes, p.piece);
            if (p.piece > classes) p.piece = classes;
        }
        p.rows_g = round_up(p.piece_rows, slice);
        p.ldg = size == 4 ? p.ldz : spread(round_up(p.piece, slice), size);        // (in 32 bits the logits themselves become G)
        p.ldp = round_up(d, 4);
        const int64_t slices = ceil_div(p.piece, slice) * planes;
        p.config_dx = mm_choose(size, d, p.piece_rows, slices >= 256);
        const int64_t tiles = ceil_div(d, mm_tile_i(p.config_dx)) * ceil_div(p.piece_rows, mm_tile_j(p.config_dx));
        const int64_t room = CUS * (p.config_dx == WIDE ? 1 : 2);
        int64_t splits = tiles >= room ? 1 : room / tiles;
        if (splits > slices / 8) splits = slices / 8;
        splits = splits < 1 ? 1 : splits;
        p.splits = (int)ceil_div(slices, ceil_div(slices, splits));
        p.config_dw = mm_choose(size, d, p.piece);
        if (p.kept) p.logits = c.take<float>(p.rows_g * p.ldz * p.loss_splits);
        p.g = size == 4 ? (void *)p.logits : c.take<char>(planes * p.rows_g * p.ldg * size);
        p.parts = c.take<float>(p.piece_rows * p.ldp * p.splits);
        if (p.config_dw == WIDE) p.rest_parts = c.take<float>((int64_t)CUS * 256 * 256);     // (splits of the last tiles of dw, a round of them)
    }
    p.bytes = c.total();
    return p;
}

int loss_check(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *labels, int32_t wide, int64_t n, int64_t d, int64_t classes,
               int32_t type)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (n < 0 || d < 1 || classes < 1 || n >= LOSS_MOST || d >= LOSS_MOST_D || classes >= LOSS_MOST_CLASSES)
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, classes %lld", (long long)n, (long long)d, (long long)classes);
    if (ceil_div(classes, 128) * ceil_div(n, 64) > INT32_MAX / 2) return fail(CHICLE_EINVAL, "too many rows times classes");
    if (ldx < d || ldw < d) return fail(CHICLE_EINVAL, "a row distance is shorter than a row");
    const int s = size_of(type);
    if (!placed(w, s) || (n > 0 && (!placed(x, s) || !placed(labels, wide ? 8 : 4)))) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    return CHICLE_OK;
}

int64_t grid_of(int64_t items, int threads, int64_t most)
{
    const int64_t g = ceil_div(items, threads);
    return g < 1 ? 1 : g < most ? g : most;
}

template <typename T>
int loss_lay_rows(const T *in, int64_t ldi, void *out, int64_t ld, int64_t rows, int64_t rows_out, int64_t cols, const LossRows *labels, hipStream_t stream)
{
    lay_rows<T><<<(unsigned)grid_of(rows_out * (ld / MM_CHUNK<T>), 256, 16384), 256, 0, stream>>>(in, ldi, (T *)out, ld, rows, rows_out, cols,
                                                                                                 labels ? labels->labels : nullptr, labels ? labels->wide : 0,
                                                                                                 labels ? labels->classes : 0);
    return launched("lay_rows");
}

template <typename T>
int run_sum_parts(const float *parts, int64_t ld, int64_t copy, int copies, T *out, int64_t ldo, int64_t rows, int64_t cols, const float *scale, hipStream_t stream,
                  const LossRows &labels = LossRows())
{
    // (several threads to a place where there are many copies to add up: 82 copies of 333 x 252 in 7 instead of 24 us)
    if (copies >= 16) sum_parts<T, 8><<<(unsigned)grid_of(rows * (ld / 4), 32, 32768), 256, 0, stream>>>(parts, ld, copy, copies, out, ldo, rows, cols, scale, labels);
    else sum_parts<T, 1><<<(unsigned)grid_of(rows * (ld / 4), 256, 32768), 256, 0, stream>>>(parts, ld, copy, copies, out, ldo, rows, cols, scale, labels);
    return launched("sum_parts");
}

template <typename T>
MmShape mm_shape(const MmOperand &a, const MmOperand &b, int64_t k, int config, int splits, int planes = 1, int64_t plane = 0)
{
    MmShape s;
    s.a = a; s.b = b;
    s.plane = plane;
    s.slices = (int)ceil_div(k, MM_K<T>) * planes;
    s.tiles_i = (int)ceil_div(a.rows, mm_tile_i(config));
    s.tiles_j = (int)ceil_div(b.rows, mm_tile_j(config));
    s.per_split = (int)ceil_div(s.slices, splits);
    s.splits = (int)ceil_div(s.slices, s.per_split);     // (none is empty; at most `splits`)
    return s;
}

template <typename C> unsigned mm_grid(const MmShape &s)
{
    const int64_t units = (int64_t)s.tiles_i * s.tiles_j * s.splits;
    return (unsigned)(units < CUS * C::PER_CU ? units : CUS * C::PER_CU);
}

// Rows of one call or of a piece of them: `rows` begins with the piece's first row.
LossRows rows_from(const LossRows &all, int64_t first, int64_t many)
{
    LossRows r = all;
    r.labels = (const char *)all.labels + first * (all.wide ? 8 : 4);
    r.n = (int)many;
    if (all.lse) r.lse = all.lse + first;
    if (all.weight) r.weight = all.weight + first;
    r.picked = all.picked + first;
    return r;
}

// lse and loss of a piece of the rows, whose laid-out x begins at `first`; logits: null, or where they are kept
template <typename T>
int run_loss(const LossPlan &p, const T *x, int64_t ldx, const T *w, int64_t ldw, const LossRows &all, int64_t first, int64_t many, float *logits,
             float *loss, float *lse, int32_t *flags, hipStream_t stream)
{
    const LossRows rows = rows_from(all, first, many);
    int parts;
    if (p.few) {
        auto kernel = loss_few<T, 1>;
        if constexpr (sizeof(T) == 4)
            if (p.n > 16) kernel = loss_few<T, 2>;
        TRY(allow_lds(kernel, p.few_lds));
        kernel<<<(unsigned)p.few_blocks, FEW_THREADS, p.few_lds, stream>>>(x, ldx, w, ldw, p.d, rows, p.few_chunk, p.few_passes, logits, p.ldz);
        TRY(launched("loss_few"));
        parts = p.few_blocks;
    } else {
        const int64_t ldx_in = p.lay_x ? p.ldk : ldx;
        const MmOperand a = {p.w, p.lay_w ? p.ldk : ldw, (int)p.classes, 0}, b = {(const T *)p.x + first * ldx_in, ldx_in, (int)many, 0};
        const MmShape s = mm_shape<T>(a, b, p.d, p.config, p.loss_splits);
        if (p.loss_splits > 1) {
            const int64_t copy = (p.rows_g ? p.rows_g : p.n) * p.ldz;
            TRY(with_config<T, MmMiddle>(p.config, [&](auto c) {
                typedef decltype(c) C;
                auto kernel = product_parts<T, C, false, false>;
                TRY(allow_lds(kernel, C::LDS));
                kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, p.logits, p.ldz, copy);
                return launched("product_parts");
            }));
            loss_join<<<(unsigned)many, 256, 0, stream>>>(rows, p.logits, p.ldz, copy, s.splits, loss + first, lse + first, flags);
            return launched("loss_join");
        }
        TRY(with_config<T, MmWide>(p.config, [&](auto c) {
            typedef decltype(c) C;
            auto kernel = loss_tiles<T, C, sizeof(T) == 4 || !std::is_same<C, MmWide>::value>;
            TRY(allow_lds(kernel, C::LDS));
            kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, rows, logits, p.ldz);
            return launched("loss_tiles");
        }));
        parts = s.tiles_i * MM_PARTS_I;
    }
    loss_rows<<<(unsigned)ceil_div(many, 4), 256, 0, stream>>>(rows, parts, loss + first, lse + first, flags);
    return launched("loss_rows");
}

// dx and dw of G of rows [row0, row0 + rows) and classes [class0, class0 + classes), dx in `copies` parts.  A piece that is not the first adds
// what all pieces share: in 32 bits, pieces of the rows, dw, in 16 bits, pieces of the classes, the parts of dx.
template <typename T>
int run_loss_products(const LossPlan &p, int64_t row0, int64_t rows, const T *w, int64_t ldw, int64_t class0, int64_t classes, int64_t ldg, T *dw,
                      int64_t lddw, const float *inverse, bool add, int &copies, hipStream_t stream)
{
    constexpr int planes = MM_PLANES<T, true>;
    const int64_t rows_g = round_up(rows, MM_K<T>), plane = p.rows_g * ldg;
    const MmOperand x_by_k = {(const T *)p.x + row0 * p.ldk, p.ldk, (int)p.d, (int)rows_g}, w_by_k = {w + class0 * ldw, ldw, (int)p.d, (int)classes};
    const MmOperand g_rows = {p.g, ldg, (int)rows, 0};
    TRY(with_config<T, MmWideByK>(p.config_dx, [&](auto c) {
        typedef decltype(c) C;
        const MmShape s = mm_shape<T>(w_by_k, g_rows, classes, p.config_dx, p.splits, planes, plane);
        auto kernel = product_parts<T, C, true, false>;
        if constexpr (sizeof(T) == 2)
            if (add) kernel = product_parts<T, C, true, false, true>;
        TRY(allow_lds(kernel, C::LDS));
        kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, p.parts, p.ldp, p.piece_rows * p.ldp);
        if (copies < s.splits) copies = s.splits;        // (the first piece's: no later one has more classes)
        return launched("product_parts");
    }));
    // dw: the last classes' tiles, where a few of them would keep the chip for another round, go by splits of the sum
    const int64_t rest = dw_rest(p.config_dw, p.d, classes, rows_g / MM_K<T> * planes), most = classes - rest;
    const MmOperand g_most = {p.g, ldg, (int)most, (int)rows_g}, g_rest = {(const T *)p.g + most, ldg, (int)rest, (int)rows_g};
    TRY(with_config<T, MmWideByK>(p.config_dw, [&](auto c) {
        typedef decltype(c) C;
        const MmShape s = mm_shape<T>(x_by_k, g_most, rows_g, p.config_dw, 1, planes, plane);
        auto kernel = product_out<T, C, false>;
        if constexpr (sizeof(T) == 4)
            if (add) kernel = product_out<T, C, true>;
        TRY(allow_lds(kernel, C::LDS));
        kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, dw + class0 * lddw, lddw, inverse);
        return launched("product_out");
    }));
    if (rest == 0) return CHICLE_OK;
    if constexpr (sizeof(T) == 2) {
        typedef MmWideByK C;
        const MmShape s = mm_shape<T>(x_by_k, g_rest, rows_g, WIDE, (int)(CUS / (ceil_div(p.d, 256) * ceil_div(rest, 256))), planes, plane);
        auto kernel = product_parts<T, C, true, true>;
        TRY(allow_lds(kernel, C::LDS));
        kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, p.rest_parts, p.ldp, rest * p.ldp);
        TRY(launched("product_parts"));
        return run_sum_parts<T>(p.rest_parts, p.ldp, rest * p.ldp, s.splits, dw + (class0 + most) * lddw, lddw, rest, p.d, inverse, stream);
    }
    return CHICLE_OK;
}

template <typename T>
int run_loss_lay(const LossPlan &p, const T *x, int64_t ldx, const T *w, int64_t ldw, const LossRows *labels, hipStream_t stream)
{
    if (p.tiles && p.lay_x) TRY(loss_lay_rows<T>(x, ldx, p.x, p.ldk, p.n, p.rows_x, p.d, labels, stream));
    if (p.tiles && p.lay_w) TRY(loss_lay_rows<T>(w, ldw, p.w, p.ldk, p.classes, p.classes, p.d, nullptr, stream));
    return CHICLE_OK;
}

template <typename T>
int run_loss_grad(const LossPlan &p, const T *x, int64_t ldx, const T *w, int64_t ldw, LossRows &rows, float *loss, T *dx, int64_t lddx, T *dw,
                  int64_t lddw, int32_t *flags, hipStream_t stream)
{
    rows.lse = p.lse;
    TRY(run_loss_lay<T>(p, x, ldx, w, ldw, &rows, stream));
    if (p.few_grad) {
        TRY(run_loss<T>(p, x, ldx, w, ldw, rows, 0, p.n, p.logits, loss, p.lse, flags, stream));
        const dim3 grid((unsigned)p.few_grad_blocks, (unsigned)ceil_div(p.d, 256 * Elem<T>::VEC));
        auto kernel = p.n == 1 ? loss_grad_few<T, 1> : p.n == 2 ? loss_grad_few<T, 2> : loss_grad_few<T, 4>;
        if constexpr (sizeof(T) == 4)
            if (p.n > 4) kernel = loss_grad_few<T, 8>;
        kernel<<<grid, 256, 0, stream>>>(x, ldx, w, ldw, p.d, rows, p.few_each, p.logits, p.ldz, dw, lddw, p.parts, p.ldp);
        TRY(launched("loss_grad_few"));
        return run_sum_parts<T>(p.parts, p.ldp, p.n * p.ldp, p.few_grad_blocks, dx, lddx, p.n, p.d, nullptr, stream, rows);
    }
    const float *inverse = nullptr;
    if (std::is_same<T, f16>::value) {
        loss_power<<<1, 1024, 0, stream>>>(rows, 16384.f, p.power);
        TRY(launched("loss_power"));
        rows.power = p.power;
        inverse = p.power + 1;
    }
    const T *w_in = (const T *)p.w;
    const int64_t ldw_in = p.lay_w ? p.ldk : ldw;
    if (p.kept) {
        for (int64_t first = 0; first < p.n; first += p.piece_rows) {
            const int64_t many = p.n - first < p.piece_rows ? p.n - first : p.piece_rows;
            TRY(run_loss<T>(p, x, ldx, w, ldw, rows, first, many, p.logits, loss, p.lse, flags, stream));
            const dim3 grid((unsigned)round_up(many, MM_K<T>), (unsigned)grid_of(p.ldg, 1024, 64));
            loss_grad_kept<T><<<grid, 256, 0, stream>>>(p.logits, p.ldz, rows_from(rows, first, many), (T *)p.g, p.ldg, p.rows_g * p.ldg);
            TRY(launched("loss_grad_kept"));
            int copies = 0;
            TRY(run_loss_products<T>(p, first, many, w_in, ldw_in, 0, p.classes, p.ldg, dw, lddw, inverse, first > 0, copies, stream));
            TRY(run_sum_parts<T>(p.parts, p.ldp, p.piece_rows * p.ldp, copies, dx + first * lddx, lddx, many, p.d, inverse, stream,
                                   rows_from(rows, first, many)));
        }
        return CHICLE_OK;
    }
    if constexpr (sizeof(T) == 2) {
        TRY(run_loss<T>(p, x, ldx, w, ldw, rows, 0, p.n, nullptr, loss, p.lse, flags, stream));
        int copies = 0;
        for (int64_t first = 0; first < p.classes; first += p.piece) {
            const int64_t many = p.classes - first < p.piece ? p.classes - first : p.piece, ldg = spread(round_up(many, MM_K<T>), 2);
            const MmOperand w_rows = {w_in + first * ldw_in, ldw_in, (int)many, 0}, x_rows = {p.x, p.ldk, (int)p.n, 0};
            const int config = mm_choose(2, many, p.n);
            TRY(with_config<T, MmWide>(config, [&](auto c) {
                typedef decltype(c) C;
                const MmShape s = mm_shape<T>(w_rows, x_rows, p.d, config, 1);
                auto kernel = loss_grad_tiles<T, C>;
                TRY(allow_lds(kernel, C::LDS));
                kernel<<<mm_grid<C>(s), C::THREADS, C::LDS, stream>>>(s, rows, (int)first, (int)many, (T *)p.g, ldg, p.rows_g * ldg, (int)p.rows_g);
                return launched("loss_grad_tiles");
            }));
            TRY(run_loss_products<T>(p, 0, p.n, w_in, ldw_in, first, many, ldg, dw, lddw, inverse, first > 0, copies, stream));
        }
        return run_sum_parts<T>(p.parts, p.ldp, p.n * p.ldp, copies, dx, lddx, p.n, p.d, inverse, stream, rows);
    }
    return CHICLE_OK;
}

// ---- embedding gradient -----------------------------------------------------------------------------------------------

constexpr int64_t EMBED_MOST_D = (1 << 23) - 1;          // blocks of columns are a grid's second dimension

struct EmbedPlan {
    int64_t pieces, tile, ldp, seen_bytes;
    int piece, tiles, passes, digit;
    bool one;                            // one workgroup sorts
    unsigned *keys[2], *places[2], *count;
    uint8_t *seen;
    float *head, *tail;
    size_t bytes;
};

EmbedPlan embed_plan(int64_t n, int64_t d, int64_t n_rows, void *workspace)
{
    EmbedPlan p = {};
    // A piece is a chain of its tokens, 0.3 us each, and what it leaves is to be joined.  In us, into 32,000 rows, pieces of 8 / 16 / 32: 500 tokens
    // of 64 18.5 / 19.7 / 23.1, 8000 of 256 39 / 41 / 45, 4000 of 1024 45 / 44 / 45, 16,000 of 1024 54 / 48 / 52; 131,072 of 2048 16 / 32: 288 / 252.
    p.piece = n * d <= (int64_t)1 << 21 ? 8 : n * d <= (int64_t)1 << 24 ? 16 : 32;
    p.pieces = ceil_div(n, p.piece);
    p.ldp = round_up(d, 8);
    int bits = 1;
    while (((int64_t)1 << bits) <= n_rows) ++bits;       // keys are 0 .. n_rows
    p.passes = (int)ceil_div(bits, SORT_BITS);
    p.digit = (int)ceil_div(bits, p.passes);
    p.one = n <= SORT_ONE;                               // (64 tokens 24 us in one launch, 29 in several; 4000 tokens 36 and 45)
    p.tile = round_up(ceil_div(n, SORT_MOST_TILES), SORT_LEAST_TILE);
    p.tiles = n ? (int)ceil_div(n, p.tile) : 0;
    Carver c(workspace);
    for (int k = 0; k < (p.one ? 1 : 2); ++k) { p.keys[k] = c.take<unsigned>(n); p.places[k] = c.take<unsigned>(n); }
    if (!p.one) p.count = c.take<unsigned>((int64_t)p.tiles << p.digit);
    p.seen_bytes = round_up(n_rows, 16);
    p.seen = c.take<uint8_t>(p.seen_bytes);
    p.head = c.take<float>(p.pieces * p.ldp);
    p.tail = c.take<float>(p.pieces * p.ldp);
    p.bytes = c.total();
    return p;
}

}  // namespace

extern "C" {

const char *chicle_train_last_error(void) { return last_error; }

size_t chicle_softmax_loss_bytes(const void *x, int64_t ldx, const void *w, int64_t ldw, int64_t n, int64_t d, int64_t classes, int32_t type,
                                 int32_t with_grad)
{
    if (!type_ok(type) || n < 0 || d < 1 || classes < 1 || n >= LOSS_MOST || d >= LOSS_MOST_D || classes >= LOSS_MOST_CLASSES) return 0;
    return loss_plan(x, ldx, w, ldw, n, d, classes, type, with_grad != 0, nullptr).bytes;
}

int chicle_softmax_loss(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *labels, int32_t wide, int64_t n, int64_t d,
                        int64_t classes, int32_t type, float *loss, float *lse, void *workspace, size_t workspace_bytes, int32_t *flags,
                        void *hip_stream)
{
    TRY(loss_check(x, ldx, w, ldw, labels, wide, n, d, classes, type));
    if (n == 0) return CHICLE_OK;
    if (!placed(loss, 4) || !placed(lse, 4)) return fail(CHICLE_EINVAL, "a null or misplaced output");
    TRY(check_workspace(workspace, workspace_bytes, loss_plan(x, ldx, w, ldw, n, d, classes, type, false, nullptr).bytes));
    const LossPlan p = loss_plan(x, ldx, w, ldw, n, d, classes, type, false, workspace);
    LossRows rows = {labels, wide, (int)n, (int)classes, nullptr, nullptr, nullptr, p.tile_sums, p.picked};
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        TRY(run_loss_lay<T>(p, (const T *)x, ldx, (const T *)w, ldw, nullptr, (hipStream_t)hip_stream));
        return run_loss<T>(p, (const T *)x, ldx, (const T *)w, ldw, rows, 0, n, nullptr, loss, lse, flags, (hipStream_t)hip_stream);
    });
}

int chicle_softmax_loss_grad(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *labels, int32_t wide, const float *row_weight,
                             int64_t n, int64_t d, int64_t classes, int32_t type, float *loss, void *dx, int64_t lddx, void *dw, int64_t lddw,
                             void *workspace, size_t workspace_bytes, int32_t *flags, void *hip_stream)
{
    TRY(loss_check(x, ldx, w, ldw, labels, wide, n, d, classes, type));
    const int s = size_of(type);
    if (lddx < d || lddw < d) return fail(CHICLE_EINVAL, "a row distance is shorter than a row");
    if (!placed(dw, s) || (n > 0 && (!placed(dx, s) || !placed(loss, 4) || !placed(row_weight, 4)))) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    hipStream_t stream = (hipStream_t)hip_stream;
    if (n == 0)                                          // no row: the classes' gradient is zero
        return with_type(type, [&](auto t) {
            typedef decltype(t) T;
            return run_sum_parts<T>(nullptr, round_up(d, 4), 0, 0, (T *)dw, lddw, classes, d, nullptr, stream);
        });
    TRY(check_workspace(workspace, workspace_bytes, loss_plan(x, ldx, w, ldw, n, d, classes, type, true, nullptr).bytes));
    const LossPlan p = loss_plan(x, ldx, w, ldw, n, d, classes, type, true, workspace);
    LossRows rows = {labels, wide, (int)n, (int)classes, nullptr, row_weight, nullptr, p.tile_sums, p.picked};
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return run_loss_grad<T>(p, (const T *)x, ldx, (const T *)w, ldw, rows, loss, (T *)dx, lddx, (T *)dw, lddw, flags, stream);
    });
}

int chicle_embed(const void *table, int64_t ld, int64_t n_rows, const void *ids, int32_t wide, int64_t n, int64_t d, int32_t type, float scale,
                 void *out, int64_t ldo, int32_t *flags, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (n < 0 || d < 1 || n_rows < 1 || n > INT32_MAX || n_rows > INT32_MAX || d > EMBED_MOST_D || ld < d || ldo < d)
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, n_rows %lld, or a row distance", (long long)n, (long long)d, (long long)n_rows);
    if (n == 0) return CHICLE_OK;
    const int s = size_of(type);
    if (!placed(table, s) || !placed(out, s) || !placed(ids, wide ? 8 : 4)) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    const int lanes = pow2_at_least(ceil_div(d, 16 / s), EMBED_THREADS);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_rows(n, EMBED_THREADS / lanes, [&](int64_t first, int64_t many, unsigned grid) {
            embed_rows<T><<<grid, EMBED_THREADS, 0, (hipStream_t)hip_stream>>>(
                (const T *)table, ld, n_rows, (const char *)ids + first * (wide ? 8 : 4), wide, (T *)out + first * ldo, ldo, many, d, lanes, scale, flags);
            return launched("embed_rows");
        });
    });
}

size_t chicle_embed_grad_bytes(int64_t n, int64_t d, int64_t n_rows)
{
    if (n < 0 || d < 1 || n_rows < 1 || n > INT32_MAX || n_rows >= INT32_MAX || d > EMBED_MOST_D) return 0;
    return embed_plan(n, d, n_rows, nullptr).bytes;
}

int chicle_embed_grad(const void *ids, int32_t wide, const void *dout, int64_t ldd, int64_t n, int64_t d, int64_t n_rows, int32_t type, float scale,
                      int32_t accumulate, void *dtable, int64_t ldo, void *workspace, size_t workspace_bytes, int32_t *flags, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (n < 0 || d < 1 || n_rows < 1 || n > INT32_MAX || n_rows >= INT32_MAX || d > EMBED_MOST_D || ldd < d || ldo < d)
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, n_rows %lld, or a row distance", (long long)n, (long long)d, (long long)n_rows);
    const int s = size_of(type);
    if (!placed(dtable, s) || (n > 0 && (!placed(dout, s) || !placed(ids, wide ? 8 : 4)))) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    hipStream_t stream = (hipStream_t)hip_stream;
    if (n == 0 && accumulate) return CHICLE_OK;
    if (n == 0)
        return with_type(type, [&](auto t) {
            typedef decltype(t) T;
            return run_sum_parts<T>(nullptr, round_up(d, 4), 0, 0, (T *)dtable, ldo, n_rows, d, nullptr, stream);
        });
    TRY(check_workspace(workspace, workspace_bytes, embed_plan(n, d, n_rows, nullptr).bytes));
    const EmbedPlan p = embed_plan(n, d, n_rows, workspace);
    uint8_t *seen = accumulate ? nullptr : p.seen;
    int last = 0;
    if (p.one) {
        auto kernel = n <= SORT_ONE_THREADS ? sort_tokens_one<1> : sort_tokens_one<4>;
        kernel<<<1, SORT_ONE_THREADS, 0, stream>>>(ids, wide, (int)n, n_rows, p.passes, p.digit, p.keys[0], p.places[0], seen, p.seen_bytes, flags);
        TRY(launched("sort_tokens_one"));
    } else
        for (int k = 0; k < p.passes; ++k) {
            const SortPass q = {ids, p.keys[(k + 1) & 1], p.places[(k + 1) & 1], p.keys[k & 1], p.places[k & 1], p.count, n, n_rows, p.tile,
                                wide, k * p.digit, p.digit, p.tiles, k == 0, flags, seen, p.seen_bytes};
            sort_count<<<(unsigned)p.tiles, SORT_THREADS, 0, stream>>>(q);
            TRY(launched("sort_count"));
            sort_scatter<<<(unsigned)p.tiles, SORT_THREADS, 0, stream>>>(q);
            TRY(launched("sort_scatter"));
            last = k & 1;
        }
    const int vec = 16 / s;
    EmbedGrad g;
    g.keys = p.keys[last]; g.places = p.places[last];
    g.head = p.head; g.tail = p.tail;
    g.n = n; g.d = d; g.n_rows = n_rows; g.ldo = ldo; g.ldd = ldd; g.ldp = p.ldp;
    g.lanes = pow2_at_least(ceil_div(d, vec), EMBED_THREADS);
    const int groups = EMBED_THREADS / g.lanes;
    // Where a workgroup has one piece and two to a compute unit are left, still longer ones.  In us, pieces of 32 / 64: 2048 columns of 16 bits into
    // 2000 rows, 16,000 tokens 48 / 55, 24,000 57 / 58, 32,768 65 / 62, 48,000 81 / 77; into 128,000 rows 16,000 130 / 130, 32,768 146 / 141, 65,536
    // 178 / 170, 131,072 247 / 226; 4096 columns 16,000 100 / 108, 65,536 205 / 188; 600 columns of 32 bits 28,000 57 / 62, 48,000 69 / 69, 1024
    // columns 65,536 104 / 99.  131,072 tokens of 512 in 16 bits (four pieces to a workgroup): 80 / 81.
    g.piece = groups == 1 && p.pieces >= 4 * CUS && p.piece == 32 ? 64 : p.piece;
    const int64_t pieces = ceil_div(n, g.piece);
    g.run_blocks = (int)ceil_div(pieces, groups);
    g.zero_rows = (int)(d * s >= ZERO_BYTES ? 1 : ZERO_BYTES / (d * s));
    while (g.run_blocks + ceil_div(n_rows, g.zero_rows) >= (int64_t)1 << 24) g.zero_rows *= 2;     // (a launch has fewer than 2^32 threads)
    g.zero_blocks = accumulate ? 0 : (int)ceil_div(n_rows, g.zero_rows);
    g.seen = seen;
    g.accumulate = accumulate;
    g.scale = scale;
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const dim3 grid((unsigned)(g.run_blocks + g.zero_blocks), (unsigned)ceil_div(d, (int64_t)g.lanes * vec));
        embed_grad_runs<T><<<grid, EMBED_THREADS, (size_t)groups * g.piece * sizeof(uint2), stream>>>(g, (const T *)dout, (T *)dtable);
        TRY(launched("embed_grad_runs"));
        if (pieces > 1) {
            const dim3 join((unsigned)ceil_div(pieces - 1, JOIN_PIECES), (unsigned)ceil_div(d, JOIN_COLUMNS));
            embed_grad_join<T><<<join, 64 * JOIN_WAVES, 0, stream>>>(g, (T *)dtable);
            TRY(launched("embed_grad_join"));
        }
        return (int)CHICLE_OK;
    });
}

int chicle_layer_norm(const void *x, int64_t ldx, const void *gamma, const void *beta, int64_t n, int64_t d, int32_t type, float eps,
                      void *y, int64_t ldy, float *mean, float *rstd, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (n < 0 || d < 1 || n > INT32_MAX || d > INT32_MAX || ldx < d || ldy < d || !(eps >= 0.f))
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, a row distance or eps", (long long)n, (long long)d);
    if (n == 0) return CHICLE_OK;
    const int s = size_of(type);
    if (!placed(x, s) || !placed(y, s) || !placed(gamma, s) || !placed(beta, s) || !placed(mean, 4) || !placed(rstd, 4))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    const RowShape r = row_shape(d, 16 / s, LN_FORWARD_VALUES / 2, LN_FORWARD_VALUES);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_vectors(r.vectors, [&](auto v) {
            constexpr int NV = decltype(v)::value;
            if constexpr (NV * Elem<T>::VEC <= LN_FORWARD_VALUES) {
                auto kernel = r.threads > 256 ? layer_norm_rows<T, NV, LN_MOST_THREADS> : layer_norm_rows<T, NV, 256>;
                return with_rows(n, r.threads / r.lanes, [&](int64_t first, int64_t many, unsigned grid) {
                    kernel<<<grid, r.threads, 0, (hipStream_t)hip_stream>>>((const T *)x + first * ldx, ldx, (const T *)gamma, (const T *)beta,
                                                                            (T *)y + first * ldy, ldy, mean + first, rstd + first, many, d, r.lanes, eps);
                    return launched("layer_norm_rows");
                });
            }
            return (int)CHICLE_OK;
        });
    });
}

size_t chicle_layer_norm_grad_bytes(int64_t n, int64_t d, int32_t type)
{
    if (!type_ok(type) || n < 0 || d < 1 || n > INT32_MAX || d > INT32_MAX) return 0;
    Carver c(nullptr);
    c.take<float>(layer_norm_parts(n, d, type) * 2 * d);
    return c.total();
}

int chicle_layer_norm_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *gamma, const float *mean, const float *rstd,
                           int64_t n, int64_t d, int32_t type, void *dx, int64_t lddx, void *dgamma, void *dbeta, void *workspace,
                           size_t workspace_bytes, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (n < 0 || d < 1 || n > INT32_MAX || d > INT32_MAX || ldx < d || lddy < d || lddx < d)
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, or a row distance", (long long)n, (long long)d);
    const int s = size_of(type);
    if (!placed(gamma, s) || !placed(dgamma, s) || !placed(dbeta, s) ||
        (n > 0 && (!placed(dy, s) || !placed(x, s) || !placed(dx, s) || !placed(mean, 4) || !placed(rstd, 4))))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    int64_t parts = layer_norm_parts(n, d, type);
    TRY(check_workspace(workspace, workspace_bytes, chicle_layer_norm_grad_bytes(n, d, type)));
    Carver c(workspace);
    float *part = c.take<float>(parts * 2 * d);
    const RowShape r = row_shape(d, 16 / s, LN_GRAD_VALUES, LN_GRAD_VALUES);
    hipStream_t stream = (hipStream_t)hip_stream;
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        if (parts > 0)
            TRY(with_vectors(r.vectors, [&](auto v) {
                constexpr int NV = decltype(v)::value;
                if constexpr (NV * Elem<T>::VEC <= LN_GRAD_VALUES) {
                    auto kernel = r.threads > 256 ? layer_norm_grad_rows<T, NV, LN_MOST_THREADS> : layer_norm_grad_rows<T, NV, 256>;
                    const size_t lds = (size_t)r.threads * Elem<T>::VEC * sizeof(float);
                    int resident = 0;
                    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, r.threads, lds) != hipSuccess || resident < 1) resident = 1;
                    const int64_t round = std::min<int64_t>((int64_t)resident * CUS, LN_GRAD_GRID);
                    parts = std::min(parts, LN_GRAD_GRID / round * round);
                    kernel<<<(unsigned)parts, r.threads, lds, stream>>>(
                        (const T *)dy, lddy, (const T *)x, ldx, (const T *)gamma, mean, rstd, (T *)dx, lddx, part, n, d, r.lanes);
                }
                return launched("layer_norm_grad_rows");
            }));
        return with_rows(2 * d, LN_SUM_COLUMNS, [&](int64_t first, int64_t, unsigned grid) {
            layer_norm_grad_sums<T><<<grid, 1024, 0, stream>>>(part, (int)parts, d, first, (T *)dgamma, (T *)dbeta);
            return launched("layer_norm_grad_sums");
        });
    });
}

size_t chicle_clip_grads_bytes(int32_t count)
{
    (void)count;
    Carver c(nullptr);
    c.take<double>(CLIP_MOST_PARTS);
    return c.total();
}

int chicle_clip_grads(const void *const *in, void *const *out, const int64_t *sizes, const int32_t *types, int32_t count, float max_norm,
                      float *norm, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (count < 0 || count > 100000 || (count > 0 && (!in || !sizes || !types))) return fail(CHICLE_EINVAL, "no tensors, or too many");
    if (!placed(norm, 4)) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    if (out && !(max_norm >= 0.f)) return fail(CHICLE_EINVAL, "max_norm must not be negative");
    int many[3] = {0, 0, 0};
    int64_t pieces_all = 0;
    for (int k = 0; k < count; ++k) {
        if (!type_ok(types[k]) || sizes[k] < 0) return fail(CHICLE_EINVAL, "tensor %d: unknown type or negative size", k);
        const int s = size_of(types[k]);
        if (sizes[k] > 0 && (!placed(in[k], s) || (out && !placed(out[k], s)))) return fail(CHICLE_EINVAL, "tensor %d: a null or misplaced pointer", k);
        if (sizes[k] > 0) ++many[types[k]];
        pieces_all += ceil_div(sizes[k], CLIP_PIECE);
    }
    if (pieces_all > INT32_MAX / 2) return fail(CHICLE_EINVAL, "too many values");
    if (out) TRY(check_apart(out, sizes, types, count));
    TRY(check_workspace(workspace, workspace_bytes, chicle_clip_grads_bytes(count)));
    Carver c(workspace);
    double *part = c.take<double>(CLIP_MOST_PARTS);
    hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t launches = ceil_div(many[0], CLIP_TENSORS) + ceil_div(many[1], CLIP_TENSORS) + ceil_div(many[2], CLIP_TENSORS);
    const int most = launches ? (int)(CLIP_MOST_PARTS / launches) : 0;
    int parts = 0;
    bool apart = false;
    for (int scale = 0; scale < (out ? 2 : 1); ++scale) {
        int first = 0;
        for (int type = 0; type < 3; ++type)
            for (int k = 0; k < count;) {
                ClipTable t;
                t.tensors = 0;
                t.first_piece[0] = 0;
                t.first_part = first;
                for (; k < count && t.tensors < CLIP_TENSORS; ++k) {
                    if (types[k] != type || sizes[k] == 0) continue;
                    t.in[t.tensors] = in[k];
                    t.out[t.tensors] = out ? out[k] : nullptr;
                    t.count[t.tensors] = sizes[k];
                    t.first_piece[t.tensors + 1] = t.first_piece[t.tensors] + (int32_t)ceil_div(sizes[k], CLIP_PIECE);
                    ++t.tensors;
                }
                if (!t.tensors) continue;
                const int pieces = t.first_piece[t.tensors], grid = scale || pieces < most ? pieces : most;
                first += grid;
                TRY(with_type(type, [&](auto e) {
                    typedef decltype(e) T;
                    if (scale) clip_scale<T><<<grid, CLIP_THREADS, 0, stream>>>(t, CLIP_PIECE, part, apart ? 0 : parts, max_norm, norm);
                    else squares<T><<<grid, CLIP_THREADS, 0, stream>>>(t, CLIP_PIECE, part);
                    return launched("clip");
                }));
            }
        if (!scale) {
            parts = first;
            apart = !out || parts == 0 || pieces_all > CLIP_FEW_PIECES;
            if (apart) {
                norm_only<<<1, CLIP_THREADS, 0, stream>>>(part, parts, norm);
                TRY(launched("norm_only"));
            }
        }
    }
    return CHICLE_OK;
}

int chicle_train_take_flags(int32_t *flags, int32_t *out, void *hip_stream)
{
    if (!placed(flags, 4) || !placed(out, 4)) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    take_flags<<<1, 1, 0, (hipStream_t)hip_stream>>>(flags, out);
    return launched("take_flags");
}

}  // extern "C"
