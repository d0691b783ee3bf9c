// Products of 16-bit matrices whose rows both run along the summed index: C[j][i] = sum_k A[i][k] B[j][k], on the matrix cores.
//
// A workgroup forms tiles of C one after the other.  Slices of 64 k of both operands go from global memory straight into LDS, the next
// slice while the present one is multiplied, and the next tile's first slice while the last of this one is and while what
// follows the product is done; sixteen-byte chunks of an LDS row are permuted by the row's number, so that the rows that a
// wavefront reads side by side lie in different banks.  Sums are held in 32-bit floats.
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

constexpr int MM_K = 64, MM_CHUNKS = MM_K / 8, MM_ROW = MM_K * 2;   // k of a slice, sixteen-byte chunks and bytes of its row

struct MmOperand {
    const void *p;
    int64_t ld, plane;                       // elements from row to row, from plane to plane
    int rows;
};

struct MmShape {
    MmOperand a, b;
    int k;                                   // of one plane, whole slices
    int planes;                              // 1 or 3
    int tiles_i, tiles_j, splits, per_split; // per_split: slices of a split of the sum
};

// Planes of the products that are formed, four bits each.
__device__ __forceinline__ int mm_plane_a(int s) { return (0x201100 >> (4 * s)) & 3; }
__device__ __forceinline__ int mm_plane_b(int s) { return (0x021010 >> (4 * s)) & 3; }

struct MmTile { int i, j, split; };

// Workgroups go to the chip's eight L2 partitions in turn: each partition gets a run of tiles, eight tiles of i by a band of j at a time.
__device__ __forceinline__ MmTile mm_tile(const MmShape &s, unsigned unit)
{
    const unsigned total = s.tiles_i * s.tiles_j, all = total * s.splits;
    const unsigned xcd = unit & 7, q = all >> 3, r = all & 7;
    unsigned n = xcd * q + min(xcd, r) + (unit >> 3);
    MmTile t;
    t.split = s.splits > 1 ? n / total : 0;
    n -= t.split * total;
    const unsigned band = n / (8u * s.tiles_j), wide = min(8u, (unsigned)s.tiles_i - band * 8), in = n - band * 8 * s.tiles_j;
    t.j = wide == 8 ? in >> 3 : in / wide;
    t.i = band * 8 + (in - t.j * wide);
    return t;
}

// A tile of BM x BN by WAVES_I x WAVES_J wavefronts; BLOCKS workgroups to a compute unit.
template <int BM, int BN, int WAVES_I, int WAVES_J, int BLOCKS> struct MmConfig {
    static constexpr int THREADS = 64 * WAVES_I * WAVES_J, PER_CU = BLOCKS, PER_SIMD = BLOCKS * THREADS / 256;
    static constexpr int MI = BM / WAVES_I / 16, NJ = BN / WAVES_J / 16;
    static constexpr int TILE_I = BM, TILE_J = BN, W_I = WAVES_I, W_J = WAVES_J;
    static constexpr int BUFFER = (BM + BN) * MM_ROW;
    static constexpr int EXTRA = WAVES_I * BN * 8;             // LDS of what follows the product
    static constexpr int LDS = 2 * BUFFER + EXTRA;             // bytes
    static constexpr int LOADS_A = BM * MM_CHUNKS / THREADS, LOADS_B = BN * MM_CHUNKS / THREADS;
    static_assert(LDS * BLOCKS <= 160 * 1024, "the workgroups of a compute unit fit");
};

// Where chunk c of row r lies in its row: any eight and any sixteen neighbouring rows have a chunk in different banks.
__device__ __forceinline__ int mm_place(int r, int c) { return c ^ (r & 7) ^ (r >> 3 & 1); }

template <int LOADS, int THREADS>
__device__ __forceinline__ void mm_offsets(const MmOperand &o, int row0, int *off)
{
#pragma unroll
    for (int it = 0; it < LOADS; ++it) {
        const int c = it * THREADS + threadIdx.x, r = c / MM_CHUNKS;
        off[it] = min(r, o.rows - 1 - row0) * (int)o.ld * 2 + mm_place(r, c % MM_CHUNKS) * 16;
    }
}

template <int LOADS, int THREADS>
__device__ __forceinline__ void mm_fetch(const char *base, const int *off, char *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int it = 0; it < LOADS; ++it)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + off[it]),
                                         (__attribute__((address_space(3))) void *)(lds + (it * THREADS + wave * 64) * 16), 16, 0, 0);
}

// What is fetched next: slice `at` of product of planes `seg`, `left` slices from the end of unit `unit`.
template <typename C> struct MmFetcher {
    unsigned unit, units;
    int seg, at, left, per_plane, all_slices;
    int off_a[C::LOADS_A], off_b[C::LOADS_B];
    const char *pa, *pb, *qa, *qb;

    __device__ __forceinline__ void planes(const MmShape &s)
    {
        qa = pa + mm_plane_a(seg) * s.a.plane * 2;
        qb = pb + mm_plane_b(seg) * s.b.plane * 2;
    }
    __device__ __forceinline__ void open(const MmShape &s)
    {
        const MmTile t = mm_tile(s, unit);
        mm_offsets<C::LOADS_A, C::THREADS>(s.a, t.i * C::TILE_I, off_a);
        mm_offsets<C::LOADS_B, C::THREADS>(s.b, t.j * C::TILE_J, off_b);
        pa = (const char *)s.a.p + (int64_t)t.i * C::TILE_I * s.a.ld * 2;
        pb = (const char *)s.b.p + (int64_t)t.j * C::TILE_J * s.b.ld * 2;
        const int first = t.split * s.per_split;
        seg = s.planes == 1 ? 0 : first / per_plane;
        at = first - seg * per_plane;
        left = min(s.per_split, all_slices - first);
        planes(s);
    }
    __device__ __forceinline__ void fetch(const MmShape &s, char *lds)
    {
        if (unit >= units) return;
        mm_fetch<C::LOADS_A, C::THREADS>(qa + (int64_t)at * MM_ROW, off_a, lds);
        mm_fetch<C::LOADS_B, C::THREADS>(qb + (int64_t)at * MM_ROW, off_b, lds + C::TILE_I * MM_ROW);
        if (--left == 0) {
            unit += gridDim.x;
            if (unit < units) open(s);
        } else if (++at == per_plane) {
            at = 0;
            ++seg;
            planes(s);
        }
    }
};

// Calls done(tile, acc, extra) for every tile of this workgroup, extra being C::EXTRA bytes of LDS:
// acc[mi][nj][r] = C[j][i] at i = i0 + (wave_i * MI + mi) * 16 + 4 * (lane / 16) + r, j = j0 + (wave_j * NJ + nj) * 16 + lane % 16
template <typename T, typename C, typename F>
__device__ __forceinline__ void mm_tiles(const MmShape &s, const F &done)
{
    extern __shared__ __align__(16) char lds[];
    typedef typename Mfma<T>::frag frag;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / C::W_J, wj = wave % C::W_J;
    const int ra = (wi * C::MI * 16 + (lane & 15)) * MM_ROW, rb = (C::TILE_I + wj * C::NJ * 16 + (lane & 15)) * MM_ROW;
    MmFetcher<C> next;
    next.unit = blockIdx.x;
    next.units = s.tiles_i * s.tiles_j * s.splits;
    next.per_plane = s.k / MM_K;
    next.all_slices = next.per_plane * (s.planes == 1 ? 1 : 6);
    if (next.unit < next.units) next.open(s);
    next.fetch(s, lds);
    int buf = 0;
    for (unsigned unit = blockIdx.x; unit < next.units; unit += gridDim.x) {
        const MmTile t = mm_tile(s, unit);
        const int slices = min(s.per_split, next.all_slices - t.split * s.per_split);
        f32x4 acc[C::MI][C::NJ];
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
#pragma unroll
            for (int j = 0; j < C::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int slice = 0; slice < slices; ++slice) {
            __syncthreads();                             // the slice has arrived, and everybody is done with the other buffer
            next.fetch(s, lds + (buf ^ 1) * C::BUFFER);
            const char *l = lds + buf * C::BUFFER;
            buf ^= 1;
#pragma unroll
            for (int kk = 0; kk < MM_K / 32; ++kk) {
                const int chunk = mm_place(lane & 15, kk * 4 + (lane >> 4)) * 16;
                frag a[C::MI], b[C::NJ];
#pragma unroll
                for (int j = 0; j < C::NJ; ++j) b[j] = *(const frag *)(l + rb + j * 16 * MM_ROW + chunk);
#pragma unroll
                for (int i = 0; i < C::MI; ++i) a[i] = *(const frag *)(l + ra + i * 16 * MM_ROW + chunk);
#pragma unroll
                for (int i = 0; i < C::MI; ++i)
#pragma unroll
                    for (int j = 0; j < C::NJ; ++j) acc[i][j] = Mfma<T>::mul(a[i], b[j], acc[i][j]);
            }
        }
        done(t, acc, lds + 2 * C::BUFFER);
    }
}

}  // namespace chicle_train
