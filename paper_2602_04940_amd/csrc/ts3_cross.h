// Attention from points to the states of an encoder, and its gradient.  For a point's head with
// query q and the states' keys k_j and values v_j:
//
//   s_j = scale q.k_j over the states that are there,  lse = log sum_j e^s_j,  p_j = e^(s_j - lse)
//   out = sum_j p_j v_j
//
// and for L = sum(g * out),
//
//   dp_j = g.v_j,  ds_j = p_j (dp_j - g.out),  dq = scale sum_j ds_j k_j,
//   dk_j = scale sum over queries of ds_j q,  dv_j = sum over queries of p_j g
//
// Query heads that share keys and values are rows of one product: with G of them per shared head,
// row r of a sample and shared head is head r % G of point r / G.  So a group's keys and values are
// read once, and the sums over rows of dk and dv are over the group's heads too.
//
//   k_cross_fwd    scores, softmax with a running maximum and sum, and the weighted values, for
//                  32 or 64 rows per wave against tiles of states in LDS
//   k_cross_join   joins the parts of rows whose states were split over workgroups
//   k_cross_dq     g.out and dq for 32 rows per wave, the scores computed again
//   k_cross_dkv    dk and dv for 32 states per wave against tiles of rows in LDS
//   k_cross_sum    sums of split gradients, in the splits' order
//
// Products are 32x32x16 with the operand conventions of ts3_gated.h, bfloat16 as it is (P = 1),
// float32 as three bfloat16 parts (P = 3).  Scores are computed transposed, rows the states in
// the order of gated_row and columns the queries: a lane then holds 16 consecutive states of one
// query, which are, as they lie, the K slots of the product with the values, and a query's
// maximum and sum are in two lanes.  The values' operand is read from LDS transposed.
// In bfloat16 the weights p and the slopes ds are rounded once, as operands of the next product;
// their sums, and every other quantity, are float32.
#pragma once
#include "ts3_gated.h"  // operands, parts, storage types

namespace ts3 {

// LDS tile: rows of DP values in 16-byte pieces, piece c of row R at c ^ cross_swz(R).  Reads of 16
// rows' pieces (ds_read_b128; rows distinct mod 16 in a cycle) and transposing reads of four rows' 64
// bytes then touch all 64 banks once.
template <int DP> __device__ __forceinline__ constexpr int cross_swz(int row) {
    if constexpr (DP == 16) return (row >> 3) & 1;
    else if constexpr (DP == 32) return (row >> 2) & 3;
    else if constexpr (DP == 64) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return ((row & 3) << 2) | ((row >> 2) & 3);
}

// A tile of ROWS rows, P planes of parts, filled by THREADS threads through registers.
template <int P, int DP, int ROWS, int THREADS> struct CrossTile {
    using T = typename GatedIO<P>::T;
    static constexpr int NPC = DP / 8, PLANE = ROWS * DP * 2, BYTES = P * PLANE;
    static constexpr int TOTAL = ROWS * NPC, ITEMS = (TOTAL + THREADS - 1) / THREADS;
    u32x4 r[ITEMS][P == 1 ? 1 : 2];

    // at(row): the row's address, always readable.  Columns past D are zero.
    template <typename F> __device__ __forceinline__ void load(int D, F at) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + k * THREADS, row = i / NPC % ROWS, c = i % NPC * 8;
            const T *const p = at(row) + (c < D ? c : 0);
#pragma unroll
            for (int h = 0; h < (P == 1 ? 1 : 2); ++h)
                r[k][h] = *reinterpret_cast<const u32x4 *>(p + 4 * h);
        }
    }
    // there(row): whether the row is there; others are zero, whatever they hold.
    template <typename F> __device__ __forceinline__ void store(unsigned char *tile, int D, F there) const {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + k * THREADS, row = i / NPC, pc = i % NPC;
            if (TOTAL % THREADS && i >= TOTAL) continue;
            const bool in = pc * 8 < D && there(row);
            unsigned char *const to = tile + row * (DP * 2) + ((pc ^ cross_swz<DP>(row)) << 4);
            if constexpr (P == 1) {
                *reinterpret_cast<u32x4 *>(to) = in ? r[k][0] : u32x4{0, 0, 0, 0};
            } else {
                float v[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) v[t] = in ? __uint_as_float(r[k][t >> 2][t & 3]) : 0.f;
                Parts<3> f;
                split8(v, f);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<bf16x8 *>(to + q * PLANE) = f.p[q];
            }
        }
    }
};

// Operand of 32 rows (gated_row order) of a tile and columns 16 ks .. + 15 as its K slots.
template <int DP> struct CrossRowRead {
    int base;
    __device__ __forceinline__ CrossRowRead(int lane) {
        const int row = gated_row<32>(0, lane & 31);
        base = row * (DP * 2) | (((lane >> 5) ^ cross_swz<DP>(row)) << 4);
    }
    template <int P> __device__ __forceinline__ void read(const unsigned char *tile, int plane, int sub, int ks, Parts<P> &f) const {
        const unsigned char *const p = tile + sub * (32 * DP * 2) + (base ^ (ks << 5));
#pragma unroll
        for (int q = 0; q < P; ++q) f.p[q] = *reinterpret_cast<const bf16x8 *>(p + q * plane);
    }
};
// Operand of columns 32 db .. + 31 of a tile (in gated_row order) and rows 32 sub + 16 (lane / 32) + 8 s
// .. + 7 as its K slots: what a lane holds of a result of the other products.  With DP = 16 the columns
// past 15 repeat the first.
template <int DP> struct CrossColRead {
    int base[2][2];
    __device__ __forceinline__ CrossColRead(int lane) {
        const int j = lane & 15, gi = 4 * ((lane >> 4) & 1) + (j & 3);
        const int group = (4 * (gi & 1) + (gi >> 1)) & (DP == 16 ? 3 : 7);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 16 * (lane >> 5) + 8 * s + 4 * h + (j >> 2);
                base[s][h] = row * (DP * 2) + (((group >> 1) ^ cross_swz<DP>(row)) << 4) + 8 * (group & 1);
            }
    }
    template <int P>
    __device__ __forceinline__ void read(const unsigned char *tile, int plane, int sub, int s, int db, Parts<P> &f) const {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const unsigned char *const p = tile + sub * (32 * DP * 2) + q * plane;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + (base[s][0] ^ (db << 6))));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + (base[s][1] ^ (db << 6))));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            f.p[q] = __builtin_bit_cast(bf16x8, v);
        }
    }
};

// Strides in elements: of a sample, a row (point or state) and a head.
struct CrossView {
    const void *p;
    int64_t sb, sr, sh;
};
struct CrossArgs {
    CrossView q, k, v, g, out;
    const int32_t *lengths;     // [B] or NULL
    const unsigned char *mask;  // [B][S] or NULL; 0 is absent
    int32_t B, N, S, H, G, D;   // G query heads share a head of keys and values
    float scale;
    int32_t splits, per;        // of a loop: parts, and tiles per part
    float *lse, *delta;         // [B][H][N]
    void *to, *to2;             // results (out, dq, or dk and dv), contiguous
    float *part, *part2;        // of split loops
    __device__ __forceinline__ int heads() const { return H / G; }
    __device__ __forceinline__ int rows() const { return N * G; }
};
__device__ __forceinline__ float *cross_stat(float *p, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : r / A.G, h = hk * A.G + (A.G == 1 ? 0 : r % A.G);
    return p + ((int64_t)b * A.H + h) * A.N + n;
}
template <typename T>
__device__ __forceinline__ const T *cross_row(const CrossView &v, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : r / A.G, h = hk * A.G + (A.G == 1 ? 0 : r % A.G);
    return (const T *)v.p + b * v.sb + n * v.sr + h * v.sh;
}
// Row r of a contiguous [B][N][H][D] result.
template <typename T> __device__ __forceinline__ T *cross_to(T *p, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : r / A.G, h = hk * A.G + (A.G == 1 ? 0 : r % A.G);
    return p + (((int64_t)b * A.N + n) * A.H + h) * A.D;
}
// States of sample b that may be there: those before its length.
__device__ __forceinline__ int cross_length(const CrossArgs &A, int b) {
    if (!A.lengths) return A.S;
    const int n = A.lengths[b];
    return n < 0 ? 0 : n > A.S ? A.S : n;
}
// Which workgroup does what: (b, block of rows or states, shared head, split), the split innermost
// and then the head, so that consecutive workgroups, which share an L2, read the same lines.
struct CrossAt {
    int b, hk, blk, split;
    __device__ __forceinline__ CrossAt(const CrossArgs &A, int blocks) {
        int i = xcd_remap(blockIdx.x, gridDim.x);
        split = i % A.splits;
        i /= A.splits;
        hk = i % A.heads();
        i /= A.heads();
        blk = i % blocks;
        b = i / blocks;
    }
};

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

template <int P, int DP, int W> constexpr int cross_tile() { return P == 1 && !(W == 1 && DP == 128) ? 64 : 32; }

// A row's 16 ks + 8 (lane / 32) .. + 7 as operand columns; zero past D.
template <int P, int DP>
__device__ __forceinline__ void cross_load_row(const typename GatedIO<P>::T *row, int D, bool in, Parts<P> (&f)[DP / 16]) {
    const int g = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        const int c = 16 * ks + 8 * g;
        load_parts(row + (c < D ? c : 0), f[ks]);
        if (!(in && c < D))
#pragma unroll
            for (int q = 0; q < P; ++q) f[ks].p[q] = bf16x8{};
    }
}

// Which of the tile's states from `first` are there; bit j is state first + j.
__device__ __forceinline__ uint64_t cross_present(const CrossArgs &A, unsigned char m, int first, int len, int tile) {
    const int j = threadIdx.x & 63;
    return __ballot(j < tile && first + j < len && m);
}
__device__ __forceinline__ unsigned char cross_mask(const CrossArgs &A, int b, int first, int len) {
    const int j = first + (threadIdx.x & 63);
    return A.mask ? A.mask[(int64_t)b * A.S + (j < len ? j : 0)] : 1;
}

// Workgroup (b, hk, block, split): 32 NQ rows per wave, W waves, against the split's tiles of
// states.  The next tile is on its way to registers while this one is used, and goes to the other
// half of LDS after it.
template <int P, int DP, int NQ, int W>
__global__ __launch_bounds__(64 * W) void k_cross_fwd(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TK = cross_tile<P, DP, W>(), SUB = TK / 32, KS = DP / 16, DB = (DP + 31) / 32;
    using Tile = CrossTile<P, DP, TK, 64 * W>;
    __shared__ __align__(16) unsigned char lds[2][2][Tile::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D, R = A.rows();
    const CrossAt at(A, (R + 32 * NQ * W - 1) / (32 * NQ * W));
    const int len = cross_length(A, at.b), tiles = (len + TK - 1) / TK;
    const int t0 = at.split * A.per, t1 = min(tiles, t0 + A.per);
    const int r0 = (at.blk * W + wave) * 32 * NQ + (lane & 31);
    const T *const kb = (const T *)A.k.p + at.b * A.k.sb + at.hk * A.k.sh;
    const T *const vb = (const T *)A.v.p + at.b * A.v.sb + at.hk * A.v.sh;
    Parts<P> qf[NQ][KS];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int r = r0 + 32 * i;
        cross_load_row<P, DP>(cross_row<T>(A.q, A, at.b, at.hk, min(r, R - 1)), D, true, qf[i]);
    }
    typename Mat<32>::D o[NQ][DB];
    float m[NQ], l[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[i][d] = typename Mat<32>::D{};
    }
    const float scale2 = A.scale * LOG2E;
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile kt, vt;
    auto fetch = [&](int t) {
        const int first = t * TK;
        kt.load(D, [&](int row) { return kb + (int64_t)min(first + row, len - 1) * A.k.sr; });
        vt.load(D, [&](int row) { return vb + (int64_t)min(first + row, len - 1) * A.v.sr; });
        return cross_mask(A, at.b, first, len);
    };
    auto put = [&](int t, uint64_t there) {
        kt.store(lds[t & 1][0], D, [&](int row) { return (there >> row & 1) != 0; });
        vt.store(lds[t & 1][1], D, [&](int row) { return (there >> row & 1) != 0; });
    };
    uint64_t there = 0;
    if (t0 < t1) {
        const unsigned char mb = fetch(t0);
        there = cross_present(A, mb, t0 * TK, len, TK);
        put(t0, there);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        unsigned char mb = 0;
        if (t + 1 < t1) mb = fetch(t + 1);
        const unsigned char *const kl = lds[t & 1][0], *const vl = lds[t & 1][1];
        if (there) {
            typename Mat<32>::D s[NQ][SUB];
#pragma unroll
            for (int i = 0; i < NQ; ++i)
#pragma unroll
                for (int u = 0; u < SUB; ++u) s[i][u] = typename Mat<32>::D{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    Parts<P> a;
                    rows.template read<P>(kl, Tile::PLANE, u, ks, a);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) mma_parts<32, P>(s[i][u], a, qf[i][ks]);
                }
            const bool whole = there == (TK == 64 ? ~0ull : (1ull << TK) - 1);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                float mx = -INFINITY;
                if (!whole)
#pragma unroll
                    for (int u = 0; u < SUB; ++u) {
                        const uint32_t bits = (uint32_t)(there >> (32 * u)) >> (16 * g);
#pragma unroll
                        for (int v = 0; v < 16; ++v) s[i][u][v] = bits >> v & 1 ? s[i][u][v] : -INFINITY;
                    }
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[i][u][v]);
                const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale2;
                const float mn = fmaxf(m[i], mx), base = mn == -INFINITY ? 0.f : mn;
                const float alpha = fast_exp2(m[i] - base);
                m[i] = mn;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        s[i][u][v] = fast_exp2(fmaf(s[i][u][v], scale2, -base));
                        sum += s[i][u][v];
                    }
                l[i] = l[i] * alpha + sum;
                if (__any(alpha != 1.f))
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[i][d] *= alpha;
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Parts<P> w[NQ];
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = s[i][u][8 * h + e];
                        to_parts(x, w[i]);
                    }
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        Parts<P> a;
                        cols.template read<P>(vl, Tile::PLANE, u, h, d, a);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) mma_parts<32, P>(o[i][d], a, w[i]);
                    }
                }
        }
        if (t + 1 < t1) {
            there = cross_present(A, mb, (t + 1) * TK, len, TK);
            put(t + 1, there);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int r = r0 + 32 * i;
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[i]), __float_as_uint(l[i]), false, false);
        const float sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
        if (r >= R) continue;
        if (A.splits == 1) {
            // no state: weights of zero, whose sum is minus infinity in the logarithm
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T *const to = cross_to((T *)A.to, A, at.b, at.hk, r);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int c = 32 * d + 16 * g;
                float x[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = o[i][d][v] * inv;
                if (c < D) store_row<16>(to + c, x);
            }
            if (g == 0) *cross_stat(A.lse, A, at.b, at.hk, r) = sum == 0.f ? -INFINITY : (m[i] + log2f(sum)) * LN2;
        } else {
            // part[split][b][hk][r][DP + 2]: unscaled sums, their maximum and their weights' sum
            const int64_t row = (((int64_t)at.split * A.B + at.b) * A.heads() + at.hk) * R + r;
            float *const to = A.part + row * (DP + 4);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int c = 32 * d + 16 * g;
                float x[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = o[i][d][v];
                if (c < D) store_row<16>(to + c, x);
            }
            if (g == 0) {
                to[DP] = m[i];
                to[DP + 1] = sum;
            }
        }
    }
}

// A row per workgroup: the splits' parts scaled to the largest maximum and added, 256 / DP at a
// time, then these in order.
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_join(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int NG = 256 / DP;
    __shared__ float acc[NG][DP], sums[NG], tops[4];
    const int R = A.rows(), tid = threadIdx.x, c = tid % DP, q = tid / DP;
    const int64_t bhr = blockIdx.x, step = (int64_t)A.B * A.heads() * R * (DP + 4);
    const int r = (int)(bhr % R), hk = (int)(bhr / R % A.heads()), b = (int)(bhr / R / A.heads());
    const float *const part = A.part + bhr * (DP + 4);
    float top = -INFINITY;
    for (int s = tid; s < A.splits; s += 256) top = fmaxf(top, part[s * step + DP]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float base = top == -INFINITY ? 0.f : top;
    float v = 0.f, sum = 0.f;
    const bool in = c < A.D;
#pragma unroll 4
    for (int s = q; s < A.splits; s += NG) {
        const float *const p = part + s * step;
        const float w = fast_exp2(p[DP] - base);
        v += w * (in ? p[c] : 0.f);
        sum += w * p[DP + 1];
    }
    acc[q][c] = v;
    if (c == 0) sums[q] = sum;
    __syncthreads();
    if (q) return;
    sum = 0.f;
    v = 0.f;
    for (int i = 0; i < NG; ++i) {
        sum += sums[i];
        v += acc[i][c];
    }
    if (in) cross_to((T *)A.to, A, b, hk, r)[c] = from_float<T>(sum == 0.f ? 0.f : v / sum);
    if (c == 0) *cross_stat(A.lse, A, b, hk, r) = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
}

// delta = g.out of the rows, and their dq: as the forward's loop, with the values as a second
// operand of rows and the keys read transposed.
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_dq(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TK = P == 1 && DP < 128 ? 64 : 32, SUB = TK / 32, KS = DP / 16, DB = (DP + 31) / 32;
    using Tile = CrossTile<P, DP, TK, 256>;
    __shared__ __align__(16) unsigned char lds[2][2][Tile::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D, R = A.rows();
    const CrossAt at(A, (R + 127) / 128);
    const int len = cross_length(A, at.b), tiles = (len + TK - 1) / TK;
    const int t0 = at.split * A.per, t1 = min(tiles, t0 + A.per);
    const int r = at.blk * 128 + wave * 32 + (lane & 31), rc = min(r, R - 1);
    const T *const kb = (const T *)A.k.p + at.b * A.k.sb + at.hk * A.k.sh;
    const T *const vb = (const T *)A.v.p + at.b * A.v.sb + at.hk * A.v.sh;
    Parts<P> qf[KS], gf[KS];
    const T *const grow = cross_row<T>(A.g, A, at.b, at.hk, rc), *const orow = cross_row<T>(A.out, A, at.b, at.hk, rc);
    cross_load_row<P, DP>(cross_row<T>(A.q, A, at.b, at.hk, rc), D, true, qf);
    cross_load_row<P, DP>(grow, D, true, gf);
    float delta = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int c = 16 * ks + 8 * g;
        if (c < D)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta += to_float(grow[c + e]) * to_float(orow[c + e]);
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(delta), __float_as_uint(delta), false, false);
    delta = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (r < R && g == 0 && at.split == 0) *cross_stat(A.delta, A, at.b, at.hk, r) = delta;
    const float scale2 = A.scale * LOG2E, lse2 = *cross_stat(A.lse, A, at.b, at.hk, rc) * LOG2E;
    typename Mat<32>::D o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = typename Mat<32>::D{};
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile kt, vt;
    auto fetch = [&](int t) {
        const int first = t * TK;
        kt.load(D, [&](int row) { return kb + (int64_t)min(first + row, len - 1) * A.k.sr; });
        vt.load(D, [&](int row) { return vb + (int64_t)min(first + row, len - 1) * A.v.sr; });
        return cross_mask(A, at.b, first, len);
    };
    auto put = [&](int t, uint64_t there) {
        kt.store(lds[t & 1][0], D, [&](int row) { return (there >> row & 1) != 0; });
        vt.store(lds[t & 1][1], D, [&](int row) { return (there >> row & 1) != 0; });
    };
    uint64_t there = 0;
    if (t0 < t1) {
        const unsigned char mb = fetch(t0);
        there = cross_present(A, mb, t0 * TK, len, TK);
        put(t0, there);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        unsigned char mb = 0;
        if (t + 1 < t1) mb = fetch(t + 1);
        const unsigned char *const kl = lds[t & 1][0], *const vl = lds[t & 1][1];
        if (there)
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                typename Mat<32>::D s{}, dp{};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    Parts<P> a;
                    rows.template read<P>(kl, Tile::PLANE, u, ks, a);
                    mma_parts<32, P>(s, a, qf[ks]);
                    rows.template read<P>(vl, Tile::PLANE, u, ks, a);
                    mma_parts<32, P>(dp, a, gf[ks]);
                }
                const uint32_t bits = (uint32_t)(there >> (32 * u)) >> (16 * g);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p = fast_exp2(fmaf(s[8 * h + e], scale2, -lse2));
                        x[e] = bits >> (8 * h + e) & 1 ? p * (dp[8 * h + e] - delta) : 0.f;
                    }
                    Parts<P> w;
                    to_parts(x, w);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        Parts<P> a;
                        cols.template read<P>(kl, Tile::PLANE, u, h, d, a);
                        mma_parts<32, P>(o[d], a, w);
                    }
                }
            }
        if (t + 1 < t1) {
            there = cross_present(A, mb, (t + 1) * TK, len, TK);
            put(t + 1, there);
        }
        __syncthreads();
    }
    if (r >= R) return;
    float *const part = A.part + ((((int64_t)at.split * A.B + at.b) * A.heads() + at.hk) * R + r) * DP;
    T *const to = cross_to((T *)A.to, A, at.b, at.hk, r);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int c = 32 * d + 16 * g;
        float x[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = o[d][v] * A.scale;
        if (c < D) {
            if (A.splits == 1) store_row<16>(to + c, x);
            else store_row<16>(part + c, x);
        }
    }
}

// dk and dv of 32 states per wave, four waves, summed over the split's tiles of rows (queries and
// their output gradients in LDS with the rows' lse and delta).
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_dkv(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TR = P == 1 && DP < 128 ? 64 : 32, SUB = TR / 32, KS = DP / 16, DB = (DP + 31) / 32;
    using Tile = CrossTile<P, DP, TR, 256>;
    __shared__ __align__(16) unsigned char lds[2][2][Tile::BYTES];
    __shared__ __align__(16) float stat[2][2][TR];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D, R = A.rows();
    const CrossAt at(A, (A.S + 127) / 128);
    const int len = cross_length(A, at.b), tiles = (R + TR - 1) / TR;
    const int j = at.blk * 128 + wave * 32 + (lane & 31), jc = min(j, A.S - 1);
    const bool there = j < len && (!A.mask || A.mask[(int64_t)at.b * A.S + jc]);
    // a block of absent states has nothing to sum
    const int t0 = at.split * A.per, t1 = at.blk * 128 < len ? min(tiles, t0 + A.per) : t0;
    Parts<P> kf[KS], vf[KS];
    cross_load_row<P, DP>((const T *)A.k.p + at.b * A.k.sb + jc * A.k.sr + at.hk * A.k.sh, D, there, kf);
    cross_load_row<P, DP>((const T *)A.v.p + at.b * A.v.sb + jc * A.v.sr + at.hk * A.v.sh, D, there, vf);
    typename Mat<32>::D dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = typename Mat<32>::D{};
    const float scale2 = A.scale * LOG2E;
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile qt, gt;
    float st = 0.f;
    auto fetch = [&](int t) {
        const int first = t * TR;
        qt.load(D, [&](int row) { return cross_row<T>(A.q, A, at.b, at.hk, min(first + row, R - 1)); });
        gt.load(D, [&](int row) { return cross_row<T>(A.g, A, at.b, at.hk, min(first + row, R - 1)); });
        if (threadIdx.x < 2 * TR) {
            const int row = first + threadIdx.x % TR;
            // past the last row the weights are e^-inf
            if (threadIdx.x < TR) st = row < R ? *cross_stat(A.lse, A, at.b, at.hk, row) * LOG2E : INFINITY;
            else st = row < R ? *cross_stat(A.delta, A, at.b, at.hk, row) : 0.f;
        }
    };
    auto put = [&](int t) {
        const int first = t * TR;
        qt.store(lds[t & 1][0], D, [&](int row) { return first + row < R; });
        gt.store(lds[t & 1][1], D, [&](int row) { return first + row < R; });
        if (threadIdx.x < 2 * TR) stat[t & 1][threadIdx.x / TR][threadIdx.x % TR] = st;
    };
    if (t0 < t1) {
        fetch(t0);
        put(t0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) fetch(t + 1);
        const unsigned char *const ql = lds[t & 1][0], *const gl = lds[t & 1][1];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            typename Mat<32>::D s{}, dp{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Parts<P> a;
                rows.template read<P>(ql, Tile::PLANE, u, ks, a);
                mma_parts<32, P>(s, a, kf[ks]);
                rows.template read<P>(gl, Tile::PLANE, u, ks, a);
                mma_parts<32, P>(dp, a, vf[ks]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const int row = 32 * u + 16 * g + 8 * h + e;
                    const f32x4 ls = *reinterpret_cast<const f32x4 *>(&stat[t & 1][0][row]);
                    const f32x4 de = *reinterpret_cast<const f32x4 *>(&stat[t & 1][1][row]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = there ? fast_exp2(fmaf(s[8 * h + e + i], scale2, -ls[i])) : 0.f;
                        x[e + i] = p;
                        y[e + i] = p * (dp[8 * h + e + i] - de[i]);
                    }
                }
                Parts<P> w, z;
                to_parts(x, w);
                to_parts(y, z);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    Parts<P> a;
                    cols.template read<P>(gl, Tile::PLANE, u, h, d, a);
                    mma_parts<32, P>(dv[d], a, w);
                    cols.template read<P>(ql, Tile::PLANE, u, h, d, a);
                    mma_parts<32, P>(dk[d], a, z);
                }
            }
        }
        if (t + 1 < t1) put(t + 1);
        __syncthreads();
    }
    if (j >= A.S) return;
    const int64_t row = ((int64_t)at.b * A.S + j) * A.heads() + at.hk, all = (int64_t)A.B * A.S * A.heads();
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int c = 32 * d + 16 * g;
        float x[16], y[16];
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            x[v] = there ? dk[d][v] * A.scale : 0.f;
            y[v] = there ? dv[d][v] : 0.f;
        }
        if (c >= D) continue;
        if (A.splits == 1) {
            store_row<16>((T *)A.to + row * D + c, x);
            store_row<16>((T *)A.to2 + row * D + c, y);
        } else {
            store_row<16>(A.part + (at.split * all + row) * D + c, x);
            store_row<16>(A.part2 + (at.split * all + row) * D + c, y);
        }
    }
}

// out[i] = the splits' values of element i, in order.  Of dq the parts lie [b][hk][r][DP], of dk and dv as
// the results do.
template <int P, int DP, bool DQ> __global__ __launch_bounds__(256) void k_cross_sum(const CrossArgs A, int64_t count) {
    using T = typename GatedIO<P>::T;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    if constexpr (DQ) {
        const int64_t bhr = i / DP;
        const int c = (int)(i % DP), R = A.rows();
        if (c >= A.D) return;
        float v = 0.f;
#pragma unroll 8
        for (int s = 0; s < A.splits; ++s) v += A.part[s * count + i];
        cross_to((T *)A.to, A, (int)(bhr / R / A.heads()), (int)(bhr / R % A.heads()), (int)(bhr % R))[c] = from_float<T>(v);
    } else {
        const float *const p = blockIdx.y ? A.part2 : A.part;
        float v = 0.f;
#pragma unroll 8
        for (int s = 0; s < A.splits; ++s) v += p[s * count + i];
        ((T *)(blockIdx.y ? A.to2 : A.to))[i] = from_float<T>(v);
    }
}

}  // namespace ts3
