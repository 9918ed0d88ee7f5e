// Orthogonalised updates: every matrix G of a list is replaced by five steps of an odd polynomial in
// X, from X = G / (|G| + eps) with the Frobenius norm, which moves all singular values near one:
//
//   A = X X^T,  X <- (a I + b A + c A A) X,   (a, b, c) = (3.4445, -4.7750, 2.0315)
//
// on the side of fewer rows r <= c: a matrix of more rows than columns is turned on the way in and
// out.  A step costs r^2 c + r^3 operations for A and its square, of which half the tiles are computed
// (both are symmetric), and 2 r^2 c for the product with X.
//
//   k_orth_norm    sums of squares of pieces (float64), and the list as a table for the others
//   k_orth_load    X / (|X| + eps) as operands, turned where rows exceed columns
//   k_orth_product the three products of a step, one launch each over every matrix's tiles
//
// Small singular values grow 3.4 times a step, almost 500 times in all, and errors of X with them, so
// operands carry 22 bits: a value times 2^12 is the sum of two half floats (the rounded value and its
// rounded remainder, 11 bits each), and a product the three part products of weight 2^-11 and more,
// summed in float32; the fourth is below 2^-22 of |x||y|.  Three bfloat16 parts would take six
// products for the same.  Half floats hold the range: the singular values of X stay below 1.21 and
// those of the polynomial's matrix below 3.45, and so do all entries; what lies below 2^-36 is lost.
#pragma once
#include "ts3_clip.h"   // sums of squares
#include "ts3_cross.h"  // LDS tiles and their reads

namespace ts3 {

constexpr float ORTH_A = 3.4445f, ORTH_B = -4.7750f, ORTH_C = 2.0315f;
constexpr float ORTH_SCALE = 4096.f;  // of a value held in two half floats

// A tensor of the list: nb matrices, wide form r x c, padded to rp x cp (multiples of 64).
struct OrthEntry {
    const void *src;
    void *dst;
    int64_t x, a;             // half floats before its X and its A in their buffers
    int32_t r, c, nb, flags;  // ORTH_TURNED, ORTH_BF16
    int32_t piece, load, gram, update;  // first workgroups of the launches
};
enum { ORTH_TURNED = 1, ORTH_BF16 = 2 };
constexpr int ORTH_BATCH = 60;  // entries that fit a launch's arguments
struct OrthBatch {
    OrthEntry e[ORTH_BATCH];
    int32_t count, first;  // entries before these
};
__host__ __device__ __forceinline__ int orth_pad(int n) { return (n + 63) & ~63; }

// Pieces of a matrix that its squares are summed by.
constexpr int64_t ORTH_PIECE = 8192;
__host__ __device__ __forceinline__ int orth_pieces(int64_t n) {
    const int64_t p = (n + ORTH_PIECE - 1) / ORTH_PIECE;
    return p < 256 ? (int)p : 256;
}

// sums[workgroup] = the squares of its piece.  The first workgroup of each entry copies it to the table.
__global__ __launch_bounds__(256) void k_orth_norm(const OrthBatch t, OrthEntry *__restrict__ table, double *__restrict__ sums) {
    __shared__ double lds[4];
    const int wg = blockIdx.x + t.e[0].piece;
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (t.e[m].piece <= wg) lo = m;
        else hi = m;
    }
    const OrthEntry &e = t.e[lo];
    if (wg == e.piece && threadIdx.x < sizeof(OrthEntry) / 4)
        reinterpret_cast<uint32_t *>(table + t.first + lo)[threadIdx.x] = reinterpret_cast<const uint32_t *>(&e)[threadIdx.x];
    const int64_t n = (int64_t)e.r * e.c;
    const int np = orth_pieces(n), i = wg - e.piece, mat = i / np;
    const int64_t per = (n + np - 1) / np, a = (int64_t)(i % np) * per, b = a + per < n ? a + per : n;
    const int64_t at = mat * n + a;
    const double s = b <= a ? 0.0
                     : e.flags & ORTH_BF16 ? clip_squares((const bf16_t *)e.src + at, b - a)
                                           : clip_squares((const float *)e.src + at, b - a);
    const double sum = clip_block_sum(s, lds);
    if (threadIdx.x == 0) sums[wg] = sum;
}

// The entry that workgroup `wg` of a launch belongs to; `first` picks the launch's count.
template <typename F> __device__ __forceinline__ int orth_find(const OrthEntry *table, int count, int wg, F first, int *lds) {
    for (int i = threadIdx.x; i < count; i += 256)
        if (first(table[i]) <= wg && (i + 1 == count || first(table[i + 1]) > wg)) *lds = i;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(*lds);
}

__device__ __forceinline__ void orth_split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// A 64 x 64 tile of X from G, through LDS where the matrix is turned; zero in the padding.
__global__ __launch_bounds__(256) void k_orth_load(const OrthEntry *__restrict__ table, int count,
                                                   const double *__restrict__ sums, double eps, _Float16 *__restrict__ x) {
    __shared__ int found;
    __shared__ double lds[4];
    __shared__ float tile[64][65];
    const int ei = orth_find(table, count, blockIdx.x, [](const OrthEntry &e) { return e.load; }, &found);
    const OrthEntry e = table[ei];
    const int rt = orth_pad(e.r) / 64, ct = orth_pad(e.c) / 64, per = rt * ct;
    const int i = blockIdx.x - e.load, mat = i / per, tr = i % per / ct, tc = i % per % ct;
    const int64_t n = (int64_t)e.r * e.c, cp = orth_pad(e.c), plane = (int64_t)orth_pad(e.r) * cp;
    const int np = orth_pieces(n);
    double s = 0.0;
    for (int k = threadIdx.x; k < np; k += 256) s += sums[e.piece + mat * np + k];
    const double f = (double)ORTH_SCALE / (sqrt(clip_block_sum(s, lds)) + eps);
    const bool turned = e.flags & ORTH_TURNED;
    const int h = turned ? e.c : e.r, w = turned ? e.r : e.c;  // as stored
    const int y0 = 64 * (turned ? tc : tr), x0 = 64 * (turned ? tr : tc), lx = threadIdx.x & 63;
#pragma unroll 4
    for (int ly = threadIdx.x >> 6; ly < 64; ly += 4) {
        const bool in = y0 + ly < h && x0 + lx < w;
        const int64_t at = mat * n + (in ? (int64_t)(y0 + ly) * w + x0 + lx : 0);
        const float v = e.flags & ORTH_BF16 ? to_float(((const bf16_t *)e.src)[at]) : ((const float *)e.src)[at];
        tile[turned ? lx : ly][turned ? ly : lx] = in ? (float)((double)v * f) : 0.f;
    }
    __syncthreads();
    _Float16 *const to = x + e.x + mat * 2 * plane;
#pragma unroll
    for (int k = threadIdx.x; k < 512; k += 256) {
        const int row = k >> 3, c = (k & 7) * 8;
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            _Float16 a, b;
            orth_split(tile[row][c + j], a, b);
            hi[j] = a;
            lo[j] = b;
        }
        const int64_t o = (int64_t)(64 * tr + row) * cp + 64 * tc + c;
        *reinterpret_cast<f16x8 *>(to + o) = hi;
        *reinterpret_cast<f16x8 *>(to + plane + o) = lo;
    }
}

// Two half-float parts of an operand; d += a b of the three part products that count, smallest first.
struct Halves {
    f16x8 hi, lo;
};
__device__ __forceinline__ f32x16 mma_half(const f16x8 &a, const f16x8 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16x8 as_half(const bf16x8 &v) { return __builtin_bit_cast(f16x8, v); }

enum OrthKind { ORTH_GRAM, ORTH_SQUARE, ORTH_UPDATE };

// ROWS rows of 32 K values, or 32 rows of K with ROWS columns: both parts, through registers.
template <int ROWS, bool COLS> struct OrthTile {
    static constexpr int PLANE = ROWS * 64, BYTES = 2 * PLANE, DP = COLS ? ROWS : 32, NPC = DP / 8;
    static constexpr int ITEMS = ROWS * 4 / 256;
    u32x4 r[2][ITEMS];
    __device__ __forceinline__ void load(const _Float16 *p, int64_t pitch, int64_t plane) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + k * 256;
            const _Float16 *const q = p + (int64_t)(i / NPC) * pitch + i % NPC * 8;
            r[0][k] = *reinterpret_cast<const u32x4 *>(q);
            r[1][k] = *reinterpret_cast<const u32x4 *>(q + plane);
        }
    }
    __device__ __forceinline__ void store(unsigned char *tile) const {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + k * 256, row = i / NPC;
            unsigned char *const to = tile + row * (DP * 2) + ((i % NPC ^ cross_swz<DP>(row)) << 4);
            *reinterpret_cast<u32x4 *>(to) = r[0][k];
            *reinterpret_cast<u32x4 *>(to + PLANE) = r[1][k];
        }
    }
};

// Result tile D[TS x TS] = sum over K of A_op B_op, K in steps of 32, four waves of TS/2 x TS/2.
//   ORTH_GRAM    A = X X^T: both operands rows of X; the tiles on and below the diagonal, each also
//                written mirrored
//   ORTH_SQUARE  a I + b A + c A A: both operands rows of A (symmetric); likewise
//   ORTH_UPDATE  the transpose of (that) X: first operand the columns of X, second rows of the matrix
// The first operand's rows are in the order of gated_row, so that a lane holds 16 consecutive ones of a
// column: 16 consecutive elements of a row of what is written.  Rows past the padding are of other
// matrices or behind the last (the buffers end with room for them) and reach no result that is kept.
template <int KIND, int TS>
__global__ __launch_bounds__(256, 2) void k_orth_product(const OrthEntry *__restrict__ table, int count,
                                                      const _Float16 *__restrict__ xs, const _Float16 *__restrict__ as,
                                                      _Float16 *__restrict__ to, bool last) {
    constexpr int NB = TS / 64;  // 32 x 32 blocks a wave's side
    constexpr bool UPDATE = KIND == ORTH_UPDATE;
    using TileA = OrthTile<TS, UPDATE>;
    using TileB = OrthTile<TS, false>;
    __shared__ __align__(16) unsigned char lds[2][TileA::BYTES + TileB::BYTES];
    __shared__ int found;
    const int ei = orth_find(table, count, blockIdx.x, [](const OrthEntry &e) { return UPDATE ? e.update : e.gram; }, &found);
    const OrthEntry e = table[ei];
    const int rp = orth_pad(e.r), cp = orth_pad(e.c), nr = (rp + TS - 1) / TS, nc = (cp + TS - 1) / TS;
    const int64_t xplane = (int64_t)rp * cp, aplane = (int64_t)rp * rp;
    int i = blockIdx.x - (UPDATE ? e.update : e.gram), ti, tj;
    const int per = UPDATE ? nr * nc : nr * (nr + 1) / 2, mat = i / per;
    i %= per;
    if constexpr (UPDATE) {
        ti = i / nr;  // of columns of X
        tj = i % nr;  // of rows
    } else {
        ti = (int)((sqrtf(8.f * i + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > i) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= i) ++ti;
        tj = i - ti * (ti + 1) / 2;
    }
    const _Float16 *const x = xs + e.x + mat * 2 * xplane, *const a = as + e.a + mat * 2 * aplane;
    const _Float16 *pa, *pb;
    int64_t sa, sb, la, lb, stepa;
    int K;
    if constexpr (KIND == ORTH_GRAM) pa = x + (int64_t)ti * TS * cp, pb = x + (int64_t)tj * TS * cp, la = lb = cp, sa = sb = xplane, K = cp, stepa = 32;
    else if constexpr (KIND == ORTH_SQUARE) pa = a + (int64_t)ti * TS * rp, pb = a + (int64_t)tj * TS * rp, la = lb = rp, sa = sb = aplane, K = rp, stepa = 32;
    else pa = x + ti * TS, pb = a + (int64_t)tj * TS * rp, la = cp, lb = rp, sa = xplane, sb = aplane, K = rp, stepa = 32 * (int64_t)cp;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, wi = wave >> 1, wj = wave & 1;
    const CrossRowRead<32> rowsA(lane);
    const int brow = lane & 31, bbase = brow * 64 | ((g ^ cross_swz<32>(brow)) << 4);
    f32x16 d[NB][NB];
#pragma unroll
    for (int p = 0; p < NB; ++p)
#pragma unroll
        for (int q = 0; q < NB; ++q) d[p][q] = f32x16{};
    TileA ta;
    TileB tb;
    ta.load(pa, la, sa);
    tb.load(pb, lb, sb);
    ta.store(lds[0]);
    tb.store(lds[0] + TileA::BYTES);
    __syncthreads();
    for (int k = 0; k < K; k += 32) {
        const unsigned char *const al = lds[k >> 5 & 1], *const bl = al + TileA::BYTES;
        if (k + 32 < K) {
            pa += stepa;
            pb += 32;
            ta.load(pa, la, sa);
            tb.load(pb, lb, sb);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Parts<2> fa[NB];
            f16x8 bh[NB], bo[NB];
#pragma unroll
            for (int p = 0; p < NB; ++p) {
                // K rows 16 ks + 8 g: half ks of row block 0, whose groups lie 16 rows apart
                if constexpr (UPDATE) {
                    const int db = wi * NB + p, j = lane & 15, gi = 4 * ((lane >> 4) & 1) + (j & 3), grp = 4 * (gi & 1) + (gi >> 1);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        s16x4 v[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int row = 16 * ks + 8 * g + 4 * h + (j >> 2);
                            v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(al + q * TileA::PLANE + row * (TS * 2) +
                                       (((4 * db + (grp >> 1)) ^ cross_swz<TS>(row)) << 4) + 8 * (grp & 1)));
                        }
                        typedef short s16x8 __attribute__((ext_vector_type(8)));
                        const s16x8 w = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
                        fa[p].p[q] = __builtin_bit_cast(bf16x8, w);
                    }
                } else {
                    rowsA.template read<2>(al, TileA::PLANE, wi * NB + p, ks, fa[p]);
                }
            }
#pragma unroll
            for (int q = 0; q < NB; ++q) {
                const unsigned char *const b = bl + (wj * NB + q) * 2048 + (bbase ^ (ks << 5));
                bh[q] = *reinterpret_cast<const f16x8 *>(b);
                bo[q] = *reinterpret_cast<const f16x8 *>(b + TileB::PLANE);
            }
#pragma unroll
            for (int t = 0; t < 3; ++t)
#pragma unroll
                for (int p = 0; p < NB; ++p)
#pragma unroll
                    for (int q = 0; q < NB; ++q)
                        d[p][q] = mma_half(as_half(fa[p].p[t == 0]), t == 1 ? bo[q] : bh[q], d[p][q]);
        }
        if (k + 32 < K) {
            unsigned char *const next = lds[(k >> 5 & 1) ^ 1];
            ta.store(next);
            tb.store(next + TileA::BYTES);
        }
        __syncthreads();
    }
    // values times 2^24; written times 2^12
#pragma unroll
    for (int p = 0; p < NB; ++p)
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int i0 = ti * TS + (wi * NB + p) * 32 + 16 * g, j = tj * TS + (wj * NB + q) * 32 + (lane & 31);
            float v[16];
            if constexpr (UPDATE) {
                // row j of X, columns i0 .. + 15
                if (j >= rp || i0 >= cp) continue;
                if (last) {
                    if (j >= e.r) continue;
                    const bool turned = e.flags & ORTH_TURNED;
                    const int64_t n = (int64_t)e.r * e.c;
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        if (i0 + t >= e.c) continue;
                        const float o = d[p][q][t] * (1.f / (ORTH_SCALE * ORTH_SCALE));
                        const int64_t at = mat * n + (turned ? (int64_t)(i0 + t) * e.r + j : (int64_t)j * e.c + i0 + t);
                        if (e.flags & ORTH_BF16) ((bf16_t *)e.dst)[at] = from_float<bf16_t>(o);
                        else ((float *)e.dst)[at] = o;
                    }
                    continue;
                }
            } else if (i0 >= rp || j >= rp) continue;
#pragma unroll
            for (int t = 0; t < 16; ++t) v[t] = d[p][q][t] * (1.f / ORTH_SCALE);
            const int64_t pitch = UPDATE ? cp : rp, plane = UPDATE ? xplane : aplane;
            const int64_t o = (int64_t)j * pitch + i0;
            _Float16 *const base = to + (UPDATE ? e.x + mat * 2 * xplane : e.a + mat * 2 * aplane);
            if constexpr (KIND == ORTH_SQUARE) {
                // A is symmetric: its row j holds the column that this lane has
#pragma unroll
                for (int h = 0; h < 16; h += 8) {
                    const f16x8 ah = *reinterpret_cast<const f16x8 *>(a + o + h), al = *reinterpret_cast<const f16x8 *>(a + aplane + o + h);
#pragma unroll
                    for (int t = 0; t < 8; ++t)
                        v[h + t] = ORTH_C * v[h + t] + ORTH_B * ((float)ah[t] + (float)al[t]) + (i0 + h + t == j && j < e.r ? ORTH_A * ORTH_SCALE : 0.f);
                }
            }
            f16x8 hi[2], lo[2];
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                _Float16 s, u;
                orth_split(v[t], s, u);
                hi[t >> 3][t & 7] = s;
                lo[t >> 3][t & 7] = u;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                *reinterpret_cast<f16x8 *>(base + o + 8 * h) = hi[h];
                *reinterpret_cast<f16x8 *>(base + plane + o + 8 * h) = lo[h];
            }
            if constexpr (!UPDATE)
                if (ti != tj)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        const int64_t m = (int64_t)(i0 + t) * rp + j;
                        base[m] = hi[t >> 3][t & 7];
                        base[plane + m] = lo[t >> 3][t & 7];
                    }
        }
}

}  // namespace ts3
