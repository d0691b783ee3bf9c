// Products of 16-bit matrices whose rows both run along the summed index: C[j][i] = sum_k A[i][k] B[j][k], on the matrix cores.
//
// A workgroup forms a tile of BM x BN values of C.  Slices of 64 k of both operands go from global memory straight into LDS,
// the next slice while the present one is multiplied; sixteen-byte chunks of an LDS row are permuted by the row's number,
// so that the sixteen rows that a wavefront reads side by side lie in different banks.  Sums are held in 32-bit floats.
//
// 32-bit operands are three 16-bit planes whose sum they are exactly (leading, middle and last eight bits of the
// significand, bfloat16 each).  Six of the nine products of planes are formed; the three that are left out are below 2^-24 of
// the product together, less than its rounding.
//
// Rows past the end of an operand are read as its last row; what they give is never stored.  k is a multiple of 64.
#pragma once
#include "elements.hpp"

namespace chicle_train {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Mfma;
template <> struct Mfma<bf16> {
    typedef bf16x8 frag;
    static __device__ __forceinline__ f32x4 mul(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<f16> {
    typedef f16x8 frag;
    static __device__ __forceinline__ f32x4 mul(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

constexpr int MM_K = 64;                     // k of a slice
constexpr int MM_CHUNKS = MM_K / 8;          // sixteen-byte chunks of a slice's row

struct MmOperand {
    const void *p;
    int64_t ld, plane;                       // elements from row to row, from plane to plane
    int rows;
};

struct MmShape {
    MmOperand a, b;
    int k_slices;                            // of one plane
    int planes;                              // 1 or 3
    int tiles_i, tiles_j, splits;            // grid: tiles_i * tiles_j * splits workgroups
};

// Planes of the products that are formed, four bits each.
__device__ __forceinline__ int mm_plane_a(int s) { return (0x201100 >> (4 * s)) & 3; }
__device__ __forceinline__ int mm_plane_b(int s) { return (0x021010 >> (4 * s)) & 3; }

struct MmTile { int i, j, split, first, last; };   // slices [first, last) of this workgroup, over all products of planes

// Workgroups go to the chip's eight L2 partitions in turn: each partition gets a run of tiles, eight tiles of i by a band of j at a time.
__device__ __forceinline__ MmTile mm_tile(const MmShape &s)
{
    const int total = s.tiles_i * s.tiles_j, grid = total * s.splits;
    const int xcd = blockIdx.x & 7, q = grid >> 3, r = grid & 7;
    const int at = xcd * q + min(xcd, r) + (blockIdx.x >> 3);
    MmTile t;
    t.split = at / total;
    const int n = at - t.split * total;
    const int band = n / (8 * s.tiles_j), wide = min(8, s.tiles_i - band * 8), in = n - band * 8 * s.tiles_j;
    t.i = band * 8 + in % wide;
    t.j = in / wide;
    const int slices = s.k_slices * (s.planes == 1 ? 1 : 6);
    t.first = (int)((int64_t)slices * t.split / s.splits);
    t.last = (int)((int64_t)slices * (t.split + 1) / s.splits);
    return t;
}

template <int BM, int BN, int WAVES_I, int WAVES_J> struct MmConfig {
    static constexpr int THREADS = 64 * WAVES_I * WAVES_J;
    static constexpr int MI = BM / WAVES_I / 16, NJ = BN / WAVES_J / 16;
    static constexpr int LDS = 2 * (BM + BN) * MM_K * 2;       // bytes, both buffers
    static constexpr int TILE_I = BM, TILE_J = BN, W_I = WAVES_I, W_J = WAVES_J;
};

template <int ROWS, int THREADS>
__device__ __forceinline__ void mm_offsets(const MmOperand &o, int row0, int *off)
{
#pragma unroll
    for (int it = 0; it < ROWS * MM_CHUNKS / THREADS; ++it) {
        const int c = it * THREADS + threadIdx.x, r = c / MM_CHUNKS, chunk = (c % MM_CHUNKS) ^ (r % MM_CHUNKS);
        off[it] = (int)(min(r, o.rows - 1 - row0) * o.ld) * 2 + chunk * 16;
    }
}

template <int ROWS, int THREADS>
__device__ __forceinline__ void mm_fetch(const char *base, const int *off, char *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int it = 0; it < ROWS * MM_CHUNKS / THREADS; ++it)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + off[it]),
                                         (__attribute__((address_space(3))) void *)(lds + (it * THREADS + wave * 64) * 16), 16, 0, 0);
}

// acc[mi][nj][r] = C[j][i] at i = i0 + (wave_i * MI + mi) * 16 + 4 * (lane / 16) + r, j = j0 + (wave_j * NJ + nj) * 16 + lane % 16
template <typename T, typename C>
__device__ __forceinline__ void mm_multiply(const MmShape &s, const MmTile &t, char *lds, f32x4 (&acc)[C::MI][C::NJ])
{
    constexpr int TH = C::THREADS, BM = C::TILE_I, BN = C::TILE_J;
    constexpr int ROW = MM_K * 2, BUF = (BM + BN) * ROW;
    int off_a[BM * MM_CHUNKS / TH], off_b[BN * MM_CHUNKS / TH];
    mm_offsets<BM, TH>(s.a, t.i * BM, off_a);
    mm_offsets<BN, TH>(s.b, t.j * BN, off_b);
    const char *pa = (const char *)s.a.p + (int64_t)t.i * BM * s.a.ld * 2, *pb = (const char *)s.b.p + (int64_t)t.j * BN * s.b.ld * 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = wave / C::W_J, wj = wave % C::W_J;
    const int ra = (wi * C::MI * 16 + (lane & 15)) * ROW, rb = (wj * C::NJ * 16 + (lane & 15)) * ROW;
    auto fetch = [&](int slice, int buf) {
        const int seg = s.planes == 1 ? 0 : slice / s.k_slices, k = slice - seg * s.k_slices;
        const int64_t ka = (int64_t)k * ROW + mm_plane_a(seg) * s.a.plane * 2, kb = (int64_t)k * ROW + mm_plane_b(seg) * s.b.plane * 2;
        mm_fetch<BM, TH>(pa + ka, off_a, lds + buf * BUF);
        mm_fetch<BN, TH>(pb + kb, off_b, lds + buf * BUF + BM * ROW);
    };
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
        for (int j = 0; j < C::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (t.first >= t.last) return;
    fetch(t.first, 0);
    for (int slice = t.first; slice < t.last; ++slice) {
        const int buf = (slice - t.first) & 1;
        __syncthreads();                                 // the slice has arrived, and everybody is done with the other buffer
        if (slice + 1 < t.last) fetch(slice + 1, buf ^ 1);
        const char *la = lds + buf * BUF, *lb = la + BM * ROW;
#pragma unroll
        for (int kk = 0; kk < MM_K / 32; ++kk) {
            const int chunk = ((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
            typename Mfma<T>::frag a[C::MI], b[C::NJ];
#pragma unroll
            for (int i = 0; i < C::MI; ++i) a[i] = *(const typename Mfma<T>::frag *)(la + ra + i * 16 * ROW + chunk);
#pragma unroll
            for (int j = 0; j < C::NJ; ++j) b[j] = *(const typename Mfma<T>::frag *)(lb + rb + j * 16 * ROW + chunk);
#pragma unroll
            for (int i = 0; i < C::MI; ++i)
#pragma unroll
                for (int j = 0; j < C::NJ; ++j) acc[i][j] = Mfma<T>::mul(a[i], b[j], acc[i][j]);
        }
    }
}

}  // namespace chicle_train
