// Entry points of include/chicle_train.h for layers over sequences: rows in 8 bits, root-mean-square norm, gated recurrence.
#include <algorithm>
#include "entry.hpp"
#include "gated_scan.hpp"
#include "packed.hpp"
#include "rms_norm.hpp"

using namespace chicle_train;

// How often a scan's tile looks for what another one tells it before it gives up; less than this only where that is tested.
extern "C" int32_t chicle_scan_looks = 1 << 22;

namespace {

// Packed rows of d columns: both pointers, rows a multiple of 32 bytes apart.
bool packed_ok(const void *q, const void *scales, int64_t ld, int64_t d)
{
    return placed(q, 16) && scales && ld >= round_up(d, PACK_GROUP) && ld % PACK_GROUP == 0;
}

Packed packed_rows(void *q, void *scales, int64_t ld) { return Packed{(int8_t *)q, (uint8_t *)scales, ld}; }
Packed packed_from(const Packed &p, int64_t row) { return p.q ? Packed{p.q + row * p.ld, p.scales + row * (p.ld / PACK_GROUP), p.ld} : p; }

bool sizes_ok(int64_t n, int64_t d) { return n >= 0 && d >= 1 && n <= INT32_MAX && d <= INT32_MAX; }

// Whether n rows of two tensors share no memory, given where they begin, their distance and their length in bytes: one ends before the other begins, or each
// row of one lies between two rows of the other.
bool rows_apart(const void *a, int64_t lda, int64_t la, const void *b, int64_t ldb, int64_t lb, int64_t n)
{
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    if (pa + (n - 1) * lda + la <= pb || pb + (n - 1) * ldb + lb <= pa) return true;
    if (lda != ldb) return false;
    const int64_t shift = pb >= pa ? (int64_t)((pb - pa) % lda) : lda - 1 - (int64_t)((pa - pb - 1) % lda);
    return shift >= la && shift + lb <= lda;
}

// f(first row, rows, workgroups) for all n rows of `per_row` vectors.
template <typename F>
int with_vectors_of_rows(int64_t n, int64_t per_row, F f)
{
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 31) / per_row);
    for (int64_t first = 0; first < n; first += most) {
        const int64_t many = std::min(most, n - first);
        TRY(f(first, many, (unsigned)ceil_div(many * per_row, PACK_THREADS * PACK_EACH)));
    }
    return CHICLE_OK;
}

// ---- root-mean-square norm --------------------------------------------------------------------------------------------

constexpr int RMS_FORWARD_VALUES = 32, RMS_GRAD_VALUES = 16;
// Workgroups of the gradient: whole rounds of what the compute units hold at once, up to RMS_GRAD_GRID, and with RMS_GRAD_ROWS rows each where there are more
// than one round's, since each has a row of sums to write and to read again.  In us, 1 / 8 / 16 / 32 rows, 16 bits: 4000 x 16,000 177 / 127 / 126 / 127,
// 1024 x 16,384 98 / 50 / 50 / 50, 10,143 x 10,061 313 / 311 / 289 / 280, 9000 x 5000 114 / 114 / 105 / 105; 32 bits: 30,000 x 4096 354 / 355 / 353 / 344.
constexpr int RMS_GRAD_GRID = 1024, RMS_GRAD_ROWS = 32;

RowShape rms_shape(int64_t d, int32_t type, int first_values, int most_values)
{
    const int vec = 16 / size_of(type);
    RowShape s = row_shape(d, vec, first_values, most_values);
    if (s.lanes < PACK_GROUP / vec) s.lanes = PACK_GROUP / vec;            // (whole groups of columns)
    return s;
}

int64_t rms_norm_parts(int64_t n, int64_t d, int32_t type)
{
    const RowShape s = rms_shape(d, type, RMS_GRAD_VALUES, RMS_GRAD_VALUES);
    return std::min<int64_t>(ceil_div(n, s.threads / s.lanes), RMS_GRAD_GRID);
}

template <typename T, bool PACKED>
int run_rms_norm_grad(RmsGrad<T, PACKED> a, const RowShape &r, int64_t parts, T *dgamma, hipStream_t stream)
{
    if (parts > 0)
        TRY(with_vectors(r.vectors, [&](auto v) {
            constexpr int NV = decltype(v)::value;
            if constexpr (NV * Elem<T>::VEC <= RMS_GRAD_VALUES) {
                auto kernel = r.threads > 256 ? rms_norm_grad_rows<T, NV, LN_MOST_THREADS, PACKED> : rms_norm_grad_rows<T, NV, 256, PACKED>;
                // (sums of the workgroup's groups, or gamma)
                const size_t lds = std::max<size_t>((size_t)r.threads * Elem<T>::VEC * sizeof(float), (size_t)NV * r.threads * 16);
                if (lds >= 64 * 1024 - LN_MOST_THREADS) TRY(allow_lds(kernel, (int)lds));
                int resident = 0;
                if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, r.threads, lds) != hipSuccess || resident < 1) resident = 1;
                const int64_t round = std::min<int64_t>((int64_t)resident * CUS, RMS_GRAD_GRID);
                const int64_t most = std::min<int64_t>(RMS_GRAD_GRID, ceil_div(a.n, RMS_GRAD_ROWS * (r.threads / r.lanes)));
                parts = std::min(parts, std::max<int64_t>(1, most / round) * round);
                kernel<<<(unsigned)parts, r.threads, lds, stream>>>(a);
            }
            return launched("rms_norm_grad_rows");
        }));
    return with_rows(a.d, LN_SUM_COLUMNS, [&](int64_t first, int64_t, unsigned grid) {
        rms_norm_grad_sums<T><<<grid, 1024, 0, stream>>>(a.part, (int)parts, a.d, first, dgamma);
        return launched("rms_norm_grad_sums");
    });
}

// ---- gated recurrence -------------------------------------------------------------------------------------------------

// f(whether u is packed)
template <typename F>
int with_packed(bool packed, F f)
{
    return packed ? f(std::true_type()) : f(std::false_type());
}

template <typename T, bool PACKED> ScanInput<T, PACKED> scan_input(const void *u, int64_t ldu, const void *scales)
{
    if constexpr (PACKED) return {(const int8_t *)u, (const uint8_t *)scales, ldu};
    else return {(const T *)u, ldu};
}

// Tiles, and what workgroups hand on in the workspace: tickets, then words.
struct ScanPlan {
    int64_t tiles, blocks, words;
    unsigned *tickets;
    unsigned long long *products, *groups, *handed;
    size_t bytes;
};

template <typename S>
ScanPlan scan_plan(int64_t n, int64_t d, void *workspace)
{
    ScanPlan p = {};
    const int64_t columns = S::COLS;
    p.tiles = n > 0 ? ceil_div(n, S::TILE) : 1;
    p.blocks = ceil_div(d, columns);
    Carver c(workspace);
    if (p.tiles > 1) {
        const int64_t line = p.blocks * columns, groups = ceil_div(p.tiles, SCAN_GROUP), runs = ceil_div(p.tiles, SCAN_RUN);
        p.words = (p.tiles + groups + runs) * line;
        p.tickets = c.take<unsigned>(p.blocks * SCAN_TICKET);
        p.products = c.take<unsigned long long>(p.words);
        p.groups = p.products + p.tiles * line;
        p.handed = p.groups + groups * line;
    }
    p.bytes = c.total();
    return p;
}

ScanPlan scan_plan(int64_t n, int64_t d, int32_t type, bool backward)
{
    if (type == CHICLE_F32) return backward ? scan_plan<ScanShape<float, true>>(n, d, nullptr) : scan_plan<ScanShape<float, false>>(n, d, nullptr);
    return backward ? scan_plan<ScanShape<bf16, true>>(n, d, nullptr) : scan_plan<ScanShape<bf16, false>>(n, d, nullptr);
}

// Clears what is handed on, and launches the kernel.
template <bool BACKWARD, typename T, bool PACKED>
int run_scan(Scan<T, PACKED> a, void *workspace, hipStream_t stream)
{
    typedef ScanShape<T, BACKWARD> S;
    if (a.order.n == 0) {
        if (a.order.count == 0) return CHICLE_OK;
        scan_nothing<<<(unsigned)std::min<int64_t>(ceil_div(a.order.count * a.d, 256), 16384), 256, 0, stream>>>(a.order, BACKWARD ? a.dlast : a.h0,
                                                                                                               BACKWARD ? a.dh0 : a.last, a.d, a.flags);
        return launched("scan_nothing");
    }
    const ScanPlan p = scan_plan<S>(a.order.n, a.d, workspace);
    // Gradients of 30,011 rows in sequences of 100, rows that are no whole lines kept in the caches / not: 1000 columns of 16 bits 92 / 116 us, of 32 144 / 165;
    // 9001 rows of 1537 columns of 32 bits 80 / 96.  Whole lines, 65,536 x 2048 of 16 bits: forward 195 / 188, gradients 309 / 300 (where there are registers for
    // one kind only), 65,536 x 1024 of 32 bits 168 / 162 and 266 / 257.
    auto lines = [](const T *q, int64_t ld) { return (uintptr_t)q % 128 == 0 && ld * sizeof(T) % 128 == 0; };
    a.lines = lines(a.f, a.ldf) && (!BACKWARD || lines(a.dy, a.lddy));
    if constexpr (!PACKED) a.lines = a.lines && lines(a.u.p, a.u.ld);
    a.tiles = (unsigned)p.tiles;
    a.blocks = (unsigned)p.blocks;
    if (p.tiles > 1) {
        a.tickets = p.tickets;
        a.products = p.products;
        a.groups = p.groups;
        a.handed = p.handed;
        a.looks = chicle_scan_looks;
        scan_begin<<<(unsigned)std::min<int64_t>(ceil_div(p.words, 256), 2048), 256, 0, stream>>>(p.tickets, a.blocks, p.products, p.words);
        TRY(launched("scan_begin"));
    }
    const unsigned grid = (unsigned)(p.tiles * p.blocks);
    // Rows that meet in lines: three workgroups to a compute unit, so that a line is still there when the next column block comes for its part.  Calls of
    // gradients, three / four, 16 bits: 30,011 x 1000 in sequences of 100 rows 90 / 93 us, in one 87 / 92, 90,000 x 300 in sequences of 300 98 / 106, 5000 x 4099 in
    // one 77 / 88, 20,000 x 700 in sequences of 50 63 / 60; forward, 32 bits: 200,000 x 16 in one 43 / 46, 30,011 x 1000 in sequences of 100 80 / 75.
    const size_t lds = a.lines ? 0 : S::MORE_LDS;
    if constexpr (BACKWARD) scan_backward<T, PACKED><<<grid, S::THREADS, lds, stream>>>(a);
    else scan_forward<T, PACKED><<<grid, S::THREADS, lds, stream>>>(a);
    return launched(BACKWARD ? "scan_backward" : "scan_forward");
}

int scan_check(const void *f, int64_t ldf, const void *u, int64_t ldu, const void *u_scales, const void *offsets, int32_t wide, int64_t sequences,
               const void *h0, const void *states, int64_t n, int64_t d, int32_t type)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldf < d || ldu < d || sequences < 0 || sequences > INT32_MAX || (!offsets && sequences != 1))
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, sequences %lld, or a row distance", (long long)n, (long long)d, (long long)sequences);
    // (a launch has fewer than 2^32 threads)
    const ScanPlan p = scan_plan(n, d, type, false), q = scan_plan(n, d, type, true);
    if (p.tiles * p.blocks >= (int64_t)1 << 23 || q.tiles * q.blocks >= (int64_t)1 << 23) return fail(CHICLE_EINVAL, "too many values");
    const int s = size_of(type);
    if ((offsets && !placed(offsets, wide ? 8 : 4)) || (h0 && !placed(h0, 4)) || (states && !placed(states, 4)))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    if (n > 0 && (!placed(f, s) || (u_scales ? !packed_ok(u, u_scales, ldu, d) : !placed(u, s)))) return fail(CHICLE_EINVAL, "a null or misplaced input");
    return CHICLE_OK;
}

}  // namespace

extern "C" {

int chicle_pack8(const void *x, int64_t ldx, int64_t n, int64_t d, int32_t type, void *q, void *scales, int64_t ldq, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldx < d) return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, or a row distance", (long long)n, (long long)d);
    if (n == 0) return CHICLE_OK;
    if (!placed(x, size_of(type)) || !packed_ok(q, scales, ldq, d)) return fail(CHICLE_EINVAL, "a null or misplaced pointer, or packed rows too near");
    const Packed p = packed_rows(q, scales, ldq);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int per_row = (int)(round_up(d, PACK_GROUP) / Elem<T>::VEC);
        return with_vectors_of_rows(n, per_row, [&](int64_t first, int64_t many, unsigned grid) {
            pack_rows<T><<<grid, PACK_THREADS, 0, (hipStream_t)hip_stream>>>((const T *)x + first * ldx, ldx, many, d, per_row, packed_from(p, first));
            return launched("pack_rows");
        });
    });
}

int chicle_unpack8(const void *q, const void *scales, int64_t ldq, int64_t n, int64_t d, int32_t type, void *out, int64_t ldo, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldo < d) return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, or a row distance", (long long)n, (long long)d);
    if (n == 0) return CHICLE_OK;
    if (!placed(out, size_of(type)) || !packed_ok(q, scales, ldq, d)) return fail(CHICLE_EINVAL, "a null or misplaced pointer, or packed rows too near");
    const Packed p = packed_rows((void *)q, (void *)scales, ldq);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int per_row = (int)(round_up(d, PACK_GROUP) / Elem<T>::VEC);
        return with_vectors_of_rows(n, per_row, [&](int64_t first, int64_t many, unsigned grid) {
            unpack_rows<T><<<grid, PACK_THREADS, 0, (hipStream_t)hip_stream>>>(packed_from(p, first), many, d, per_row, (T *)out + first * ldo, ldo);
            return launched("unpack_rows");
        });
    });
}

int chicle_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *gamma, int64_t n, int64_t d, int32_t type, float eps,
                    void *sum, int64_t ldsum, void *y, int64_t ldy, void *y_scales, void *sum8, void *sum8_scales, int64_t ldsum8, float *rstd,
                    void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldx < d || (residual && ldres < d) || (sum && ldsum < d) || ldy < d || !(eps >= 0.f))
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, a row distance or eps", (long long)n, (long long)d);
    if (n == 0) return CHICLE_OK;
    const int s = size_of(type);
    if (!placed(x, s) || (residual && !placed(residual, s)) || !placed(gamma, s) || (sum && !placed(sum, s)) || !placed(rstd, 4) ||
        (y_scales ? !packed_ok(y, y_scales, ldy, d) : !placed(y, s)) || (sum8 && !packed_ok(sum8, sum8_scales, ldsum8, d)))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer, or packed rows too near");
    const RowShape r = rms_shape(d, type, RMS_FORWARD_VALUES / 2, RMS_FORWARD_VALUES);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_vectors(r.vectors, [&](auto v) {
            constexpr int NV = decltype(v)::value;
            if constexpr (NV * Elem<T>::VEC <= RMS_FORWARD_VALUES) {
                auto kernel = r.threads > 256 ? rms_norm_rows<T, NV, LN_MOST_THREADS> : rms_norm_rows<T, NV, 256>;
                return with_rows(n, r.threads / r.lanes, [&](int64_t first, int64_t many, unsigned grid) {
                    RmsRows<T> a;
                    a.x = (const T *)x + first * ldx;
                    a.residual = residual ? (const T *)residual + first * ldres : nullptr;
                    a.gamma = (const T *)gamma;
                    a.sum = sum ? (T *)sum + first * ldsum : nullptr;
                    a.y = y_scales ? nullptr : (T *)y + first * ldy;
                    a.rstd = rstd + first;
                    a.y8 = packed_from(packed_rows(y_scales ? y : nullptr, y_scales, ldy), first);
                    a.sum8 = packed_from(packed_rows(sum8, sum8_scales, ldsum8), first);
                    a.ldx = ldx; a.ldres = ldres; a.ldsum = ldsum; a.ldy = ldy;
                    a.n = many; a.d = d;
                    a.lanes = r.lanes;
                    a.eps = eps;
                    kernel<<<grid, r.threads, 0, (hipStream_t)hip_stream>>>(a);
                    return launched("rms_norm_rows");
                });
            }
            return (int)CHICLE_OK;
        });
    });
}

size_t chicle_rms_norm_grad_bytes(int64_t n, int64_t d, int32_t type)
{
    if (!type_ok(type) || !sizes_ok(n, d)) return 0;
    Carver c(nullptr);
    c.take<float>(rms_norm_parts(n, d, type) * d);
    return c.total();
}

int chicle_rms_norm_grad(const void *dy, int64_t lddy, const void *sum, int64_t ldsum, const void *sum_scales, const void *gamma, const float *rstd,
                         const void *dsum, int64_t lddsum, int64_t n, int64_t d, int32_t type, void *dx, int64_t lddx, void *dgamma, void *workspace,
                         size_t workspace_bytes, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldsum < d || lddy < d || lddx < d || (dsum && lddsum < d))
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, or a row distance", (long long)n, (long long)d);
    const int s = size_of(type);
    if (!placed(gamma, s) || !placed(dgamma, s) ||
        (n > 0 && (!placed(dy, s) || !placed(dx, s) || !placed(rstd, 4) || (dsum && !placed(dsum, s)) ||
                   (sum_scales ? !packed_ok(sum, sum_scales, ldsum, d) : !placed(sum, s)))))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer, or packed rows too near");
    TRY(check_workspace(workspace, workspace_bytes, chicle_rms_norm_grad_bytes(n, d, type)));
    const RowShape r = rms_shape(d, type, RMS_GRAD_VALUES, RMS_GRAD_VALUES);
    const int64_t parts = rms_norm_parts(n, d, type);
    Carver c(workspace);
    float *part = c.take<float>(parts * d);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_packed(sum_scales != nullptr, [&](auto packed) {
            constexpr bool PACKED = decltype(packed)::value;
            RmsGrad<T, PACKED> a;
            if constexpr (PACKED) a.r = {(const int8_t *)sum, (const uint8_t *)sum_scales, ldsum};
            else a.r = {(const T *)sum, ldsum};
            a.dy = (const T *)dy; a.dr = (const T *)dsum; a.gamma = (const T *)gamma;
            a.rstd = rstd;
            a.dx = (T *)dx;
            a.part = part;
            a.lddy = lddy; a.lddr = lddsum; a.lddx = lddx;
            a.n = n; a.d = d;
            a.lanes = r.lanes;
            return run_rms_norm_grad<T, PACKED>(a, r, parts, (T *)dgamma, (hipStream_t)hip_stream);
        });
    });
}

size_t chicle_gated_scan_bytes(int64_t n, int64_t d, int32_t type)
{
    if (!type_ok(type) || !sizes_ok(n, d)) return 0;
    return std::max(scan_plan(n, d, type, false).bytes, scan_plan(n, d, type, true).bytes);
}

int chicle_gated_scan(const void *f, int64_t ldf, const void *u, int64_t ldu, const void *u_scales, const void *offsets, int32_t wide, int64_t sequences,
                      const float *h0, int64_t n, int64_t d, int32_t type, void *y, int64_t ldy, float *last, float *states, void *workspace,
                      size_t workspace_bytes, int32_t *flags, void *hip_stream)
{
    TRY(scan_check(f, ldf, u, ldu, u_scales, offsets, wide, sequences, h0, states, n, d, type));
    if (ldy < d) return fail(CHICLE_EINVAL, "a row distance is shorter than a row");
    if ((n > 0 && !placed(y, size_of(type))) || (last && !placed(last, 4))) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    TRY(check_workspace(workspace, workspace_bytes, chicle_gated_scan_bytes(n, d, type)));
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_packed(u_scales != nullptr, [&](auto packed) {
            constexpr bool PACKED = decltype(packed)::value;
            Scan<T, PACKED> a = {};
            a.u = scan_input<T, PACKED>(u, ldu, u_scales);
            a.order = {offsets, wide, sequences, n};
            a.f = (const T *)f; a.h0 = h0; a.states = states; a.last = last; a.y = (T *)y;
            a.ldf = ldf; a.ldy = ldy; a.d = d;
            a.flags = flags;
            return run_scan<false>(a, workspace, (hipStream_t)hip_stream);
        });
    });
}

int chicle_gated_scan_grad(const void *f, int64_t ldf, const void *u, int64_t ldu, const void *u_scales, const void *offsets, int32_t wide,
                           int64_t sequences, const float *h0, const float *states, const void *dy, int64_t lddy, const float *dlast, int64_t n, int64_t d,
                           int32_t type, void *df, int64_t lddf, void *du, int64_t lddu, float *dh0, void *workspace, size_t workspace_bytes,
                           int32_t *flags, void *hip_stream)
{
    TRY(scan_check(f, ldf, u, ldu, u_scales, offsets, wide, sequences, h0, states, n, d, type));
    if (lddy < d || lddf < d || lddu < d) return fail(CHICLE_EINVAL, "a row distance is shorter than a row");
    const int s = size_of(type);
    if ((n > 0 && (!placed(dy, s) || !placed(df, s) || !placed(du, s) || !states)) || (dlast && !placed(dlast, 4)) || (dh0 && !placed(dh0, 4)))
        return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    TRY(check_workspace(workspace, workspace_bytes, chicle_gated_scan_bytes(n, d, type)));
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_packed(u_scales != nullptr, [&](auto packed) {
            constexpr bool PACKED = decltype(packed)::value;
            Scan<T, PACKED> a = {};
            a.u = scan_input<T, PACKED>(u, ldu, u_scales);
            a.order = {offsets, wide, sequences, n};
            a.f = (const T *)f; a.dy = (const T *)dy; a.h0 = h0; a.dlast = dlast; a.states = (float *)states; a.dh0 = dh0;
            a.df = (T *)df; a.du = (T *)du;
            a.ldf = ldf; a.lddy = lddy; a.lddf = lddf; a.lddu = lddu; a.d = d;
            a.flags = flags;
            return run_scan<true>(a, workspace, (hipStream_t)hip_stream);
        });
    });
}

int chicle_gated_step(const void *f, int64_t ldf, const void *u, int64_t ldu, float *state, int64_t ldstate, int64_t n, int64_t d, int32_t type, void *y,
                      int64_t ldy, void *hip_stream)
{
    if (!type_ok(type)) return fail(CHICLE_EINVAL, "unknown type %d", type);
    if (!sizes_ok(n, d) || ldf < d || ldu < d || ldstate < d || ldy < d)
        return fail(CHICLE_EINVAL, "sizes n %lld, d %lld, or a row distance", (long long)n, (long long)d);
    if (n == 0) return CHICLE_OK;
    const int s = size_of(type);
    if (!placed(f, s) || !placed(u, s) || !placed(y, s) || !placed(state, 4)) return fail(CHICLE_EINVAL, "a null or misplaced pointer");
    // (another thread may have written there what this one still has to read)
    auto apart = [&](const void *p, int64_t ld) { return rows_apart(state, ldstate * 4, d * 4, p, ld * s, d * s, n); };
    if (!apart(f, ldf) || !apart(u, ldu) || !apart(y, ldy)) return fail(CHICLE_EINVAL, "state overlaps another tensor");
    const int lanes = pow2_at_least(ceil_div(d, 16 / s), STEP_THREADS);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        return with_rows(n, STEP_THREADS / lanes, [&](int64_t first, int64_t many, unsigned grid) {
            scan_step<T><<<grid, STEP_THREADS, 0, (hipStream_t)hip_stream>>>((const T *)f + first * ldf, ldf, (const T *)u + first * ldu, ldu,
                                                                             state + first * ldstate, ldstate, (T *)y + first * ldy, ldy, many, d, lanes);
            return launched("scan_step");
        });
    });
}

}  // extern "C"
