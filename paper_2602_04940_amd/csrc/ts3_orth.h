// Orthogonalised updates: every matrix G of a list is replaced by five steps of an odd polynomial in
// X, from X = G / (|G| + eps) with the Frobenius norm, which moves all singular values near one:
//
//   A = X X^T,  X <- (a I + b A + c A A) X,   (a, b, c) = (3.4445, -4.7750, 2.0315)
//
// on the side of fewer rows r <= c: a matrix of more rows than columns is turned on the way in and
// out.  A step costs r^2 c + r^3 operations for A and its square, of which half the tiles are computed
// (both are symmetric), and 2 r^2 c for the product with X.
//
//   k_orth_small   matrices of up to 64 x 64: all of it in one workgroup's LDS
// and for the others
//   k_orth_norm    sums of squares of pieces (float64); the list as a table, and the table's entry of each
//                  workgroup, for the launches that follow
//   k_orth_load    X / (|X| + eps) as operands, turned where rows exceed columns
//   k_orth_stream, k_orth_product   the three products of a step, one launch each over every matrix's tiles, of
//                  128 or, where those are few, of 64
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
#include "ts3_orth_rules.h"

namespace ts3 {

constexpr float ORTH_A = 3.4445f, ORTH_B = -4.7750f, ORTH_C = 2.0315f;
constexpr float ORTH_SCALE = 4096.f;  // of a value held in two half floats

// Launches after the first.  Of a small matrix, the first does nothing but this table, and `load` is its
// workgroup of k_orth_small.
enum OrthLaunch { ORTH_AT_LOAD, ORTH_AT_GRAM, ORTH_AT_UPDATE };
constexpr int ORTH_BATCH = 60;  // entries that fit a launch's arguments
struct OrthBatch {
    OrthEntry e[ORTH_BATCH];
    int32_t count, first;  // entries before these
};

// Pieces of a matrix that its squares are summed by.
constexpr int64_t ORTH_PIECE = 8192;
__host__ __device__ __forceinline__ int orth_pieces(int64_t n) {
    const int64_t p = (n + ORTH_PIECE - 1) / ORTH_PIECE;
    return p < 256 ? (int)p : 256;
}

// sums[workgroup] = the squares of its piece.  The first workgroup of each entry copies it to the table
// and its number to those of the later launches' workgroups (maps[launch][workgroup], up to `end`).
struct OrthMaps {
    int32_t *of[3];
    int32_t end[3];
};
__global__ __launch_bounds__(256) void k_orth_norm(const OrthBatch t, OrthEntry *__restrict__ table, const OrthMaps maps,
                                                   double *__restrict__ sums) {
    __shared__ double lds[4];
    const int wg = blockIdx.x + t.e[0].piece;
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (t.e[m].piece <= wg) lo = m;
        else hi = m;
    }
    const OrthEntry &e = t.e[lo];
    if (wg == e.piece) {
        if (threadIdx.x < sizeof(OrthEntry) / 4)
            reinterpret_cast<uint32_t *>(table + t.first + lo)[threadIdx.x] = reinterpret_cast<const uint32_t *>(&e)[threadIdx.x];
        const bool more = lo + 1 < t.count;
        const int from[3] = {e.load, e.gram, e.update};
        const int to[3] = {more ? t.e[lo + 1].load : maps.end[0], more ? t.e[lo + 1].gram : maps.end[1],
                           more ? t.e[lo + 1].update : maps.end[2]};
#pragma unroll
        for (int k = 0; k < 3; ++k)
            for (int i = from[k] + threadIdx.x; i < to[k]; i += 256) maps.of[k][i] = t.first + lo;
    }
    if (e.c <= ORTH_SMALL) return;
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

__device__ __forceinline__ void orth_split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// X and A lie in blocks of 32 columns, their rows one after another: what a step of 32 K reads of any of
// them is whole lines, whichever way round.
__device__ __forceinline__ int64_t orth_at(int row, int col, int rp) { return (int64_t)(col >> 5) * rp * 32 + row * 32 + (col & 31); }

// A 64 x 64 tile of X from G, through LDS where the matrix is turned; zero in the padding.
__global__ __launch_bounds__(256) void k_orth_load(const OrthEntry *__restrict__ table, const int32_t *__restrict__ map,
                                                   const double *__restrict__ sums, double eps, _Float16 *__restrict__ x) {
    __shared__ double lds[4];
    __shared__ float tile[64][65];
    const OrthEntry e = table[map[blockIdx.x]];
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
        const int64_t o = orth_at(64 * tr + row, 64 * tc + c, orth_pad(e.r));
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

// ROWS rows of 32 K values, or 32 rows of K with ROWS columns: both parts, through registers.  `block` is the
// distance of a block of 32 columns from the next.
template <int ROWS, bool COLS> struct OrthTile {
    static constexpr int PLANE = ROWS * 64, BYTES = 2 * PLANE, DP = COLS ? ROWS : 32;
    static constexpr int ITEMS = ROWS * 4 / 256;
    u32x4 r[2][ITEMS];
    __device__ __forceinline__ void load(int tid, const _Float16 *p, int64_t block, int64_t plane) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = tid + k * 256;
            const _Float16 *const q = COLS ? p + (i >> 7) * block + (i & 127) * 8 : p + i * 8;
            r[0][k] = *reinterpret_cast<const u32x4 *>(q);
            r[1][k] = *reinterpret_cast<const u32x4 *>(q + plane);
        }
    }
    __device__ __forceinline__ void store(int tid, unsigned char *tile) const {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = tid + k * 256, row = COLS ? i >> 2 & 31 : i >> 2, pc = COLS ? (i >> 7) * 4 + (i & 3) : i & 3;
            unsigned char *const to = tile + row * (DP * 2) + ((pc ^ cross_swz<DP>(row)) << 4);
            *reinterpret_cast<u32x4 *>(to) = r[0][k];
            *reinterpret_cast<u32x4 *>(to + PLANE) = r[1][k];
        }
    }
};

// Operand of columns 32 db .. + 31 (in gated_row order) of a tile of rows of W, rows 16 ks + 8 (lane / 32) .. + 7
// as its K slots.
template <int W> __device__ __forceinline__ void orth_cols(const unsigned char *tile, int plane, int db, int ks, Parts<2> &f) {
    const int lane = threadIdx.x & 63, j = lane & 15, gi = 4 * ((lane >> 4) & 1) + (j & 3), group = 4 * (gi & 1) + (gi >> 1);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        s16x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = 16 * ks + 8 * (lane >> 5) + 4 * h + (j >> 2);
            v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + q * plane + row * (W * 2) +
                       (((4 * db + (group >> 1)) ^ cross_swz<W>(row)) << 4) + 8 * (group & 1)));
        }
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 w = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
        f.p[q] = __builtin_bit_cast(bf16x8, w);
    }
}

// A tile of a product: where its operands start, and whose it is.
template <int KIND, int TS> struct OrthJob {
    static constexpr bool UPDATE = KIND == ORTH_UPDATE;
    OrthEntry e;
    int mat, ti, tj, K;
    const _Float16 *pa, *pb;
    int64_t block, sa, sb, stepa, stepb;  // a block of 32 columns; of the operands: parts' distances, steps of 32 K
    __device__ __forceinline__ OrthJob(const OrthEntry *table, const int32_t *map, const _Float16 *xs, const _Float16 *as, int wg)
        : e(table[map[wg]]) {
        const int rp = orth_pad(e.r), cp = orth_pad(e.c), nr = (rp + TS - 1) / TS, nc = (cp + TS - 1) / TS;
        const int64_t xplane = (int64_t)rp * cp, aplane = (int64_t)rp * rp;
        int i = wg - (UPDATE ? e.update : e.gram);
        const int per = UPDATE ? nr * nc : nr * (nr + 1) / 2;
        mat = i / per;
        i %= per;
        if constexpr (UPDATE) {
            ti = i / nr;  // of columns of X
            tj = i % nr;  // of rows
        } else {
            ti = (int)((sqrtf(8.f * i + 1.f) - 1.f) * 0.5f);
            while (ti * (ti + 1) / 2 > i) --ti;
            while ((ti + 1) * (ti + 2) / 2 <= i) ++ti;
            ti = __builtin_amdgcn_readfirstlane(ti);
            tj = i - ti * (ti + 1) / 2;
        }
        const _Float16 *const x = xs + e.x + mat * 2 * xplane, *const a = as + e.a + mat * 2 * aplane;
        block = (int64_t)rp * 32;
        stepa = stepb = block;
        if constexpr (KIND == ORTH_GRAM) pa = x + ti * TS * 32, pb = x + tj * TS * 32, sa = sb = xplane, K = cp;
        else if constexpr (KIND == ORTH_SQUARE) pa = a + ti * TS * 32, pb = a + tj * TS * 32, sa = sb = aplane, K = rp;
        else pa = x + ti * (TS / 32) * block, pb = a + tj * TS * 32, sa = xplane, sb = aplane, K = rp, stepa = 32 * 32;
    }
};

// The tile that workgroup i of a launch takes: eight in a row, of one matrix mostly, which read the same
// lines, on one XCD, and such rows dealt out over the XCDs (in the order of their sums' length).
__device__ __forceinline__ int orth_tile(int i, int n) {
    constexpr int ROW = 8, ALL = 8 * ROW;
    const int first = i / ALL * ALL, in = i - first;
    return first + ALL <= n ? first + (in & 7) * ROW + (in >> 3) : i;
}

// A wave's result, rows r0 .. and columns c0 .. of the tile, where it goes.
template <int KIND, int TS, int NA, int NB>
__device__ __forceinline__ void orth_write(const OrthJob<KIND, TS> &job, const f32x16 (&d)[NA][NB], const _Float16 *as, _Float16 *to,
                                           bool last, int r0, int c0) {
    constexpr bool UPDATE = KIND == ORTH_UPDATE;
    const int lane = threadIdx.x & 63, g = lane >> 5;
    const OrthEntry &e = job.e;
    const int mat = job.mat, rp = orth_pad(e.r), cp = orth_pad(e.c);
    const int64_t xplane = (int64_t)rp * cp, aplane = (int64_t)rp * rp;
    const _Float16 *const a = as + e.a + mat * 2 * aplane;
    // values times 2^24; written times 2^12
#pragma unroll
    for (int p = 0; p < NA; ++p)
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int i0 = job.ti * TS + r0 + p * 32 + 16 * g, j = job.tj * TS + c0 + q * 32 + (lane & 31);
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
            const int64_t plane = UPDATE ? xplane : aplane, o = orth_at(j, i0, rp);
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
                if (job.ti != job.tj)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        const int64_t m = orth_at(i0 + t, j, rp);
                        base[m] = hi[t >> 3][t & 7];
                        base[plane + m] = lo[t >> 3][t & 7];
                    }
        }
}

// Result tiles D[64 x 64] = sum over K of A_op B_op, K in steps of 32, four waves of 32 x 32.
//   ORTH_GRAM    A = X X^T: both operands rows of X; the tiles on and below the diagonal, each also
//                written mirrored
//   ORTH_SQUARE  a I + b A + c A A: both operands rows of A (symmetric); likewise
//   ORTH_UPDATE  the transpose of (that) X: first operand the columns of X, second rows of the matrix
// The first operand's rows are in the order of gated_row, so that a lane holds 16 consecutive ones of a
// column: 16 consecutive elements of a row of what is written.  Rows past the padding are of other
// matrices or behind the last (the buffers end with room for them) and reach no result that is kept.
//
// A workgroup takes every gridDim.x-th tile.  The steps of its tiles are one stream: two are on their way in
// registers and one in each half of LDS, those of the next tile asked for before this one is written.
// Where tiles are few, GROUPS groups of four waves each take every GROUPS-th pair of steps of one tile (the
// grid then has a workgroup for each), and the first adds their sums in order.
//
// The three products of six matrices of 128 x 128 to 512 take 7, 5 and 5 us, a launch's and a chain of loads'
// latency; those of 144 of 256 x 256 to 1024 39 and 22 us (k_orth_stream has the third: 62), with matrix cores on
// 33 and 24% of the cycles: of a tile's four to sixteen pairs of steps the first waits for memory and an
// epilogue follows the last.
template <int KIND, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS, 4) void k_orth_product(const OrthEntry *__restrict__ table, const int32_t *__restrict__ map,
                                                      int tiles, const _Float16 *__restrict__ xs,
                                                      const _Float16 *__restrict__ as, _Float16 *__restrict__ to, bool last) {
    constexpr int TS = 64;
    constexpr bool UPDATE = KIND == ORTH_UPDATE;
    using Job = OrthJob<KIND, TS>;
    using TileA = OrthTile<TS, UPDATE>;
    using TileB = OrthTile<TS, false>;
    constexpr int STAGE = TileA::BYTES + TileB::BYTES;
    static_assert((GROUPS - 1) * TS * TS * 4 <= GROUPS * 2 * STAGE, "the groups' sums go where the operands were");
    __shared__ __align__(16) unsigned char all_lds[GROUPS][2][STAGE];
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
    unsigned char *const lds[2] = {all_lds[group][0], all_lds[group][1]};
    const int lane = threadIdx.x & 63, wave = tid >> 6, g = lane >> 5, wi = wave >> 1, wj = wave & 1;
    const CrossRowRead<32> rowsA(lane);
    const int brow = lane & 31, bbase = brow * 64 | ((g ^ cross_swz<32>(brow)) << 4);
    int at = blockIdx.x;
    Job job(table, map, xs, as, orth_tile(at, tiles)), next = job;
    TileA ta[2];
    TileB tb[2];
    // pairs of steps of `next` that this group has not yet asked for; K is a multiple of 64
    auto pairs = [&](const Job &j) { return (j.K / 64 - group + GROUPS - 1) / GROUPS; };
    auto start = [&](Job &j) {
        j.pa += group * 2 * j.stepa;
        j.pb += group * 2 * j.stepb;
    };
    int left = pairs(next);
    start(next);
    auto fetch = [&](auto half) {
        constexpr int H = decltype(half)::value;
        ta[H].load(tid, next.pa, next.block, next.sa);
        tb[H].load(tid, next.pb, next.block, next.sb);
        constexpr int ON = H == 0 ? 1 : 2 * GROUPS - 1;
        next.pa += ON * next.stepa;
        next.pb += ON * next.stepb;
        left -= H;
    };
    auto put = [&](auto half) {
        constexpr int H = decltype(half)::value;
        ta[H].store(tid, lds[H]);
        tb[H].store(tid, lds[H] + TileA::BYTES);
    };
    f32x16 d[1][1];
    auto compute = [&](auto half) {
        const unsigned char *const al = lds[decltype(half)::value], *const bl = al + TileA::BYTES;
        Parts<2> fa[2];
        f16x8 bh[2], bo[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if constexpr (UPDATE) orth_cols<TS>(al, TileA::PLANE, wi, ks, fa[ks]);
            else rowsA.template read<2>(al, TileA::PLANE, wi, ks, fa[ks]);
            const unsigned char *const b = bl + wj * 2048 + (bbase ^ (ks << 5));
            bh[ks] = *reinterpret_cast<const f16x8 *>(b);
            bo[ks] = *reinterpret_cast<const f16x8 *>(b + TileB::PLANE);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int t = 0; t < 3; ++t) d[0][0] = mma_half(as_half(fa[ks].p[t == 0]), t == 1 ? bo[ks] : bh[ks], d[0][0]);
    };
    using H0 = std::integral_constant<int, 0>;
    using H1 = std::integral_constant<int, 1>;
    if (left > 0) {
        fetch(H0{});
        fetch(H1{});
        put(H0{});
    }
    __syncthreads();
    for (;;) {
        const int then = at + gridDim.x, mine = pairs(job), rounds = (job.K / 64 + GROUPS - 1) / GROUPS;
        d[0][0] = f32x16{};
        for (int k = 0; k < rounds; ++k) {
            if (GROUPS == 1 && left == 0 && then < tiles) {
                next = Job(table, map, xs, as, orth_tile(then, tiles));
                left = pairs(next);
            }
            const bool more = left > 0, here = GROUPS == 1 || k < mine;
            if (more) fetch(H0{});
            if (here) {
                compute(H0{});
                put(H1{});
            }
            __syncthreads();
            if (more) fetch(H1{});
            if (here) compute(H1{});
            if (more) put(H0{});
            __syncthreads();
        }
        if constexpr (GROUPS > 1) {
            float *const sums = reinterpret_cast<float *>(&all_lds[0][0][0]) + tid;
            if (group > 0)
#pragma unroll
                for (int v = 0; v < 16; ++v) sums[(group - 1) * 4096 + v * 256] = d[0][0][v];
            __syncthreads();
            if (group > 0) return;
#pragma unroll
            for (int i = 0; i < GROUPS - 1; ++i) {
#pragma unroll
                for (int v = 0; v < 16; ++v) d[0][0][v] += sums[i * 4096 + v * 256];
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        orth_write<KIND, TS, 1, 1>(job, d, as, to, last, wi * 32, wj * 32);
        if (GROUPS > 1 || then >= tiles) break;
        job = next;
        at = then;
    }
}

// The same with tiles of 128 x 128, eight waves of 64 x 32 each and a workgroup per compute unit.  The steps are
// copied to LDS directly, four stages of 32 KB, and read from there into registers a step before their use:
// one barrier a step parts the copies, the reads and the products of different steps, which go on side by
// side.  X X^T of four matrices of 1003 x 4095, in us (128 steps, 41 of matrix core time): through registers
// 102 (of which without the loads and LDS writes 57), copied and read in the step of use 98 (without the
// copies 81, without reads and products 50), in this form 89, with matrix cores on 55% of the cycles.
template <int KIND>
__global__ __launch_bounds__(512, 2) void k_orth_stream(const OrthEntry *__restrict__ table, const int32_t *__restrict__ map, int tiles,
                                                        const _Float16 *__restrict__ xs, const _Float16 *__restrict__ as,
                                                        _Float16 *__restrict__ to, bool last) {
    constexpr int TS = 128, PLANE = TS * 64, OPERAND = 2 * PLANE, STAGE = 2 * OPERAND, STAGES = 4;
    constexpr bool UPDATE = KIND == ORTH_UPDATE;
    using Job = OrthJob<KIND, TS>;
    __shared__ __align__(16) unsigned char lds[STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
    const int wi = wave >> 2, wj = wave & 3;
    int at = blockIdx.x, then = at + gridDim.x;
    Job job(table, map, xs, as, orth_tile(at, tiles)), next = job;
    // A stage is 32 copies of 1 KB, 16 per operand; wave w makes 2w and 2w + 1 of each: rows 16 c .. + 15 of a part (four
    // pieces a row), of columns 4 c .. + 3 of the 32 K (sixteen pieces a row).  A lane fetches the piece that
    // belongs where its 16 bytes land.
    const uint32_t row_off = (lane >> 2) * 64 + (((lane & 3) ^ cross_swz<32>(lane >> 2)) << 4);
    const int part = wave >> 2, chunk = 2 * wave & 7;
    uint32_t col_off[2];
    const _Float16 *pa, *pb;
    int left, ahead = 0, to_fill = 0, to_use = 0;  // steps of `next` to ask for; asked for and not done; stages
    auto aim = [&]() {
        pa = next.pa + part * next.sa + chunk * (UPDATE ? 128 : 512);
        pb = next.pb + part * next.sb + chunk * 512;
        left = next.K / 32;
        if constexpr (UPDATE)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int k = 4 * (chunk + e) + (lane >> 4), piece = (lane & 15) ^ cross_swz<128>(k);
                col_off[e] = (uint32_t)((piece >> 2) * next.block * 2 + (4 * e + (lane >> 4)) * 64 + (piece & 3) * 16);
            }
    };
    aim();
    auto issue = [&]() {
        if (left == 0) {
            if (then >= tiles) return;
            next = Job(table, map, xs, as, orth_tile(then, tiles));
            then += gridDim.x;
            aim();
        }
        const uint32_t base = lds_addr(&lds[to_fill][0]) + wave * 2048;
        // a copy's offset counts in LDS too
        dma16s<0>(UPDATE ? col_off[0] : row_off, pa, base);
        if constexpr (UPDATE) dma16s<0>(col_off[1], pa, base + 1024);
        else dma16s<1024>(row_off, pa, base);
        dma16s<0>(row_off, pb, base + OPERAND);
        dma16s<1024>(row_off, pb, base + OPERAND);
        pa += next.stepa;
        pb += next.stepb;
        to_fill = (to_fill + 1) & (STAGES - 1);
        --left;
        ++ahead;
    };
    const CrossRowRead<32> rowsA(lane);
    const int brow = lane & 31, bbase = brow * 64 | ((g ^ cross_swz<32>(brow)) << 4);
    f32x16 d[2][1];
    Parts<2> fa[2][2][2];  // [parity of the step][K half][rows]
    f16x8 bh[2][2], bo[2][2];
    auto read = [&](auto parity, int stage) {
        constexpr int H = decltype(parity)::value;
        const unsigned char *const al = lds[stage], *const bl = al + OPERAND + wj * 2048;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bh[H][ks] = *reinterpret_cast<const f16x8 *>(bl + (bbase ^ (ks << 5)));
            bo[H][ks] = *reinterpret_cast<const f16x8 *>(bl + PLANE + (bbase ^ (ks << 5)));
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                if constexpr (UPDATE) orth_cols<TS>(al, PLANE, wi * 2 + p, ks, fa[H][ks][p]);
                else rowsA.template read<2>(al, PLANE, wi * 2 + p, ks, fa[H][ks][p]);
            }
        }
    };
    auto multiply = [&](auto parity, int ks) {
        constexpr int H = decltype(parity)::value;
#pragma unroll
        for (int t = 0; t < 3; ++t)
#pragma unroll
            for (int p = 0; p < 2; ++p)
                d[p][0] = mma_half(as_half(fa[H][ks][p].p[t == 0]), t == 1 ? bo[H][ks] : bh[H][ks], d[p][0]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // Step t, whose operands are in registers: the copies of step t + 1 have landed everywhere and the stage of
    // step t has been read, so that step t + 4 may take its place.  Copies land in order, four of the wave's a
    // step; stores do not, and are waited for after a tile (`all`).
    auto step = [&](auto parity, bool all) {
        constexpr int H = decltype(parity)::value;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (all || ahead <= 2) wait_vmcnt<0>();
        else if (ahead == 3) wait_vmcnt<4>();
        else wait_vmcnt<8>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        --ahead;
        to_use = (to_use + 1) & (STAGES - 1);
        if (ahead > 0) read(std::integral_constant<int, 1 - H>{}, to_use);
        __builtin_amdgcn_sched_barrier(0);
        multiply(parity, 0);  // the matrix cores first, or they wait for the copies' scalar work in every step
        issue();
        multiply(parity, 1);
    };
    using H0 = std::integral_constant<int, 0>;
    using H1 = std::integral_constant<int, 1>;
    for (int i = 0; i < STAGES; ++i) issue();
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(H0{}, 0);
    for (;;) {
        d[0][0] = d[1][0] = f32x16{};
        for (int k = 0; k < job.K; k += 64) {
            step(H0{}, k == 0);
            step(H1{}, false);
        }
        orth_write<KIND, TS, 2, 1>(job, d, as, to, last, wi * 64, wj * 32);
        at += gridDim.x;
        if (at >= tiles) break;
        job = Job(table, map, xs, as, orth_tile(at, tiles));
    }
}

// A matrix of at most 64 x 64 per workgroup: norm, steps and result without leaving it.  Four waves, a
// 32 x 32 block of each product each; X, A and the polynomial's matrix lie in LDS as two parts of rows of
// 64 half floats.  A chain of fifteen products with a barrier each: 16 us for 24 matrices, 28 for 576 (32 x 32).
__global__ __launch_bounds__(256, 3) void k_orth_small(const OrthEntry *__restrict__ table, const int32_t *__restrict__ map, int first,
                                                    int steps, double eps) {
    constexpr int PLANE = 64 * 128;
    __shared__ __align__(16) unsigned char lds[3][2 * PLANE];
    __shared__ double sums[4];
    const int wg = first + blockIdx.x;
    const OrthEntry e = table[map[wg]];
    const int mat = wg - e.load, n = e.r * e.c;
    const bool turned = e.flags & ORTH_TURNED;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, wi = wave >> 1, wj = wave & 1;
    // thread's row and sixteen columns
    const int row = tid >> 2, c0 = (tid & 3) * 16;
    float v[16];
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const bool in = row < e.r && c0 + k < e.c;
        const int64_t at = (int64_t)mat * n + (in ? turned ? (c0 + k) * e.r + row : row * e.c + c0 + k : 0);
        const float x = e.flags & ORTH_BF16 ? to_float(((const bf16_t *)e.src)[at]) : ((const float *)e.src)[at];
        v[k] = in ? x : 0.f;
        s += (double)v[k] * v[k];
    }
    const double f = (double)ORTH_SCALE / (sqrt(clip_block_sum(s, sums)) + eps);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = row < e.r && c0 + k < e.c ? (float)((double)v[k] * f) : 0.f;
    // row j of a buffer, columns i0 .. + 15
    auto write = [](unsigned char *buffer, int j, int i0, const float (&x)[16]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f16x8 hi, lo;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                _Float16 a, b;
                orth_split(x[8 * h + k], a, b);
                hi[k] = a;
                lo[k] = b;
            }
            unsigned char *const p = buffer + j * 128 + (((i0 / 8 + h) ^ cross_swz<64>(j)) << 4);
            *reinterpret_cast<f16x8 *>(p) = hi;
            *reinterpret_cast<f16x8 *>(p + PLANE) = lo;
        }
    };
    write(lds[0], row, c0, v);
    __syncthreads();
    const CrossRowRead<64> rows(lane);
    const int brow = 32 * wj + (lane & 31), bbase = brow * 128 | ((g ^ cross_swz<64>(brow)) << 4);
    // rows of a (in gated_row order; its columns where COLS) times rows of b
    auto product = [&](const unsigned char *a, const unsigned char *b, auto cols) {
        // the part products in chains of their own: a wave alone waits for each before the next of its chain
        f32x16 d{}, d1{}, d2{};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            Parts<2> fa;
            if constexpr (decltype(cols)::value) orth_cols<64>(a, PLANE, wi, ks, fa);
            else rows.template read<2>(a, PLANE, wi, ks, fa);
            const f16x8 bh = *reinterpret_cast<const f16x8 *>(b + (bbase ^ (ks << 5)));
            const f16x8 bo = *reinterpret_cast<const f16x8 *>(b + PLANE + (bbase ^ (ks << 5)));
            d2 = mma_half(as_half(fa.p[1]), bh, d2);
            d1 = mma_half(as_half(fa.p[0]), bo, d1);
            d = mma_half(as_half(fa.p[0]), bh, d);
        }
        d1 += d2;
        return d += d1;
    };
    const int i0 = 32 * wi + 16 * g;
    for (int step = 0; step < steps; ++step) {
        f32x16 d = product(lds[0], lds[0], std::false_type{});
        float x[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k] = d[k] * (1.f / ORTH_SCALE);
        write(lds[1], brow, i0, x);
        __syncthreads();
        d = product(lds[1], lds[1], std::false_type{});
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // A is symmetric: its row holds the column that this lane has
            const unsigned char *const p = lds[1] + brow * 128 + (((i0 / 8 + h) ^ cross_swz<64>(brow)) << 4);
            const f16x8 ah = *reinterpret_cast<const f16x8 *>(p), al = *reinterpret_cast<const f16x8 *>(p + PLANE);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[8 * h + k] = ORTH_C * (d[8 * h + k] * (1.f / ORTH_SCALE)) + ORTH_B * ((float)ah[k] + (float)al[k]) +
                               (i0 + 8 * h + k == brow ? ORTH_A * ORTH_SCALE : 0.f);
        }
        write(lds[2], brow, i0, x);
        __syncthreads();
        d = product(lds[0], lds[2], std::true_type{});
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k] = d[k] * (1.f / ORTH_SCALE);
        if (step + 1 == steps) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                if (brow >= e.r || i0 + k >= e.c) continue;
                const int64_t at = (int64_t)mat * n + (turned ? (i0 + k) * e.r + brow : brow * e.c + i0 + k);
                const float o = x[k] * (1.f / ORTH_SCALE);
                if (e.flags & ORTH_BF16) ((bf16_t *)e.dst)[at] = from_float<bf16_t>(o);
                else ((float *)e.dst)[at] = o;
            }
        } else {
            __syncthreads();  // the columns have been read
            write(lds[0], brow, i0, x);
            __syncthreads();
        }
    }
}

}  // namespace ts3
