// The norms around a block with its gate and residual scale, and their gradient, over rows of C
// values: the branch's output f is normalised, gated, scaled and added to the stream x, and the
// sum is normalised again for the next branch.
//
//   h = LN(f),  m = h gamma_post + beta_post,  s = 1 / (1 + e^-gate)
//   y = x + scale s m,   out = LN(y) gamma_pre + beta_pre
//
// and for L = sum(gy * y) + sum(gn * out), with k = LN(y), e = gn gamma_pre,
//
//   dx = dy = gy + rstd(y) (e - mean(e) - k mean(e k)),   dgamma_pre = sum gn k,  dbeta_pre = sum gn
//   dscale = sum dy s m,   dgate = dy scale m s (1 - s),   d = dy scale s
//   dgamma_post = sum d h,  dbeta_post = sum d,  df = rstd(f) (i - mean(i) - h mean(i h)),  i = d gamma_post
//
// Both move each row once and are bound by that (the sums are over rows).  Rows lie over lanes as
// in ts3_norm.h: a group of LG lanes holds one, K pieces of V values each.  The forward reaches 4.6 to 4.9 TB/s
// (1M gated rows of 256 in bfloat16 0.55 ms); the backward has five rows to read and twice the arithmetic,
// and asks in bfloat16 for the next row before this one's (1.14 -> 0.88 ms, 4.7 TB/s, vector instructions on all cycles;
// 2M float32 rows of 128 1.30 ms, 4.7 TB/s).
#pragma once
#include "ts3_norm.h"

namespace ts3 {

// V consecutive values of a row, as they lie in memory and as floats.
template <typename T, int V> struct RawPiece;
template <> struct RawPiece<float, 4> {
    f32x4 u;
    __device__ __forceinline__ void load(const float *p) { u = *reinterpret_cast<const f32x4 *>(p); }
    __device__ __forceinline__ void get(float (&v)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = u[i];
    }
};
template <int V> struct RawPiece<bf16_t, V> {
    uint32_t u[V / 2];
    __device__ __forceinline__ void load(const bf16_t *p) {
        if constexpr (V == 8) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = x[i];
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(p);
            u[0] = x.x;
            u[1] = x.y;
        }
    }
    __device__ __forceinline__ void get(float (&v)[V]) const {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};
template <int V, typename T> __device__ __forceinline__ void store_piece(T *p, const float (&v)[V]) {
    if constexpr (sizeof(T) == 2 && V == 4)
        *reinterpret_cast<uint2 *>(p) = uint2{__builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[0], (__bf16)v[1]}),
                                              __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2], (__bf16)v[3]})};
    else store_row<V>(p, v);
}

// s = 1 / (1 + e^-a) and s (1 - s), the latter without the cancellation of 1 - s.  The product
// a log2(e) is taken in two parts, so that the exponential is good to a rounding or two for any a.
// An infinite a gives 0 or 1, a NaN itself.
__device__ __forceinline__ float gate_sigmoid(float a, float &slope) {
    const float b = a < -110.f ? -110.f : a > 200.f ? 200.f : a;  // keeps NaN; e^110 is infinite, e^-200 zero
    constexpr float L = 1.44269502f, LL = 1.92596303e-8f;         // log2(e) in two parts
    const float h = -b * L, l = fmaf(-b, L, -h) - b * LL;
    const float e = fast_exp2(h) * fmaf(l, 0.693147182f, 1.f), s = fast_rcp(1.f + e);  // within an ulp
    slope = s * (e > 0x1p100f ? 1.f : e * s);
    return s;
}

struct SandwichParams {
    const float *gamma_post, *beta_post, *scale, *gamma_pre, *beta_pre;  // the last two may be NULL
};

// The columns that a lane holds, and a parameter's values there.  FULL: the lanes hold C columns and no
// more, and nothing is masked.
template <int LG, int K, int V, bool FULL> struct SandwichCols {
    bool in[K];
    int col[K];
    __device__ __forceinline__ SandwichCols(int sub, int C) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            in[k] = FULL || (k * LG + sub) * V < C;
            col[k] = in[k] ? (k * LG + sub) * V : 0;
        }
    }
    __device__ __forceinline__ void load(const float *p, float (&v)[K][V]) const {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = p ? p[col[k] + i] : 0.f;
    }
    template <typename T> __device__ __forceinline__ void fetch(const T *p, int64_t at, RawPiece<T, V> (&raw)[K]) const {
        if (p)
#pragma unroll
            for (int k = 0; k < K; ++k) raw[k].load(p + at + col[k]);
    }
    template <typename T> __device__ __forceinline__ void get(const T *p, const RawPiece<T, V> (&raw)[K], float (&v)[K][V]) const {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (p) raw[k].get(v[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = p && in[k] ? v[k][i] : 0.f;
        }
    }
    template <typename T> __device__ __forceinline__ void store(T *p, int64_t at, const float (&v)[K][V]) const {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (in[k]) store_piece(p + at + col[k], v[k]);
    }
};

// gate may be NULL (s = 1), and out (no second norm).  y may be x.
template <typename T, int V, int LG, int K, bool FULL>
__global__ __launch_bounds__(256) void k_sandwich_fwd(const T *__restrict__ f, const T *x, const T *__restrict__ gate,
                                                      const SandwichParams p, int64_t n, int C, float eps, T *y,
                                                      T *__restrict__ out) {
    constexpr int RW = 64 / LG;
    const int lane = threadIdx.x & 63;
    const SandwichCols<LG, K, V, FULL> cols(lane % LG, C);
    float gp[K][V], bp[K][V], sc[K][V], gn[K][V], bn[K][V];
    cols.load(p.gamma_post, gp);
    cols.load(p.beta_post, bp);
    cols.load(p.scale, sc);
    cols.load(p.gamma_pre, gn);
    cols.load(p.beta_pre, bn);
    const int64_t step = (int64_t)gridDim.x * 4 * RW;
    for (int64_t r0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * RW; r0 < n; r0 += step) {
        const int64_t row = r0 + lane / LG;
        const bool live = row < n;
        const int64_t at = (live ? row : n - 1) * C;
        RawPiece<T, V> rf[K], rx[K], ra[K];
        cols.fetch(f, at, rf);
        cols.fetch(x, at, rx);
        cols.fetch(gate, at, ra);
        float v[K][V], w[K][V], a[K][V];
        cols.get(f, rf, v);
        cols.get(x, rx, w);
        cols.get(gate, ra, a);
        const float rstd = norm_stats<LG, K, V>(v, cols.in, (float)C, eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float slope, m = (v[k][i] * rstd * gp[k][i] + bp[k][i]) * sc[k][i];
                if (gate) m *= gate_sigmoid(a[k][i], slope);
                w[k][i] = cols.in[k] ? w[k][i] + m : 0.f;
            }
        if (live) cols.store(y, at, w);
        if (!out) continue;
        const float rs = norm_stats<LG, K, V>(w, cols.in, (float)C, eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) w[k][i] = w[k][i] * rs * gn[k][i] + bn[k][i];
        if (live) cols.store(out, at, w);
    }
}

// e becomes rstd (e - mean(e) - v mean(e v)) for the normalised row v: LayerNorm's gradient.
template <int LG, int K, int V>
__device__ __forceinline__ void norm_slope(float (&e)[K][V], const float (&v)[K][V], float rstd, float invC) {
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            m1 += e[k][i];
            m2 += e[k][i] * v[k][i];
        }
    m1 = group_sum<LG>(m1) * invC;
    m2 = group_sum<LG>(m2) * invC;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) e[k][i] = rstd * (e[k][i] - m1 - v[k][i] * m2);
}

// The five column sums, in the order of part[block][5][C]: dgamma_post, dbeta_post, dscale, dgamma_pre,
// dbeta_pre.  gy, gate and gn may be NULL (zero; s = 1; no second norm, y is then not read); dx may be gy.
constexpr int SANDWICH_SUMS = 5;
template <typename T> struct SandwichGrads {
    const T *f, *y, *gy, *gn, *gate;
    T *df, *dx, *dgate;
    int64_t n;
    int C;
    float eps;
    float *part;
};
template <typename T, int V, int LG, int K, bool FULL>
__global__ __launch_bounds__(256) void k_sandwich_bwd(const SandwichGrads<T> A, const SandwichParams p) {
    constexpr int RW = 64 / LG, W = LG * K * V;
    __shared__ float sums[4][W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, C = A.C;
    const float invC = 1.f / C;
    const SandwichCols<LG, K, V, FULL> cols(lane % LG, C);
    float gp[K][V], bp[K][V], sc[K][V], gn[K][V], s[SANDWICH_SUMS][K][V];
    cols.load(p.gamma_post, gp);
    cols.load(p.beta_post, bp);
    cols.load(p.scale, sc);
    cols.load(A.gn ? p.gamma_pre : nullptr, gn);
#pragma unroll
    for (int j = 0; j < SANDWICH_SUMS; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][k][i] = 0.f;
    const int64_t step = (int64_t)gridDim.x * 4 * RW;
    // The next row's loads go out before this row's arithmetic, in bfloat16: float32, with half the arithmetic a
    // byte, waits for memory anyway, and loses to more registers (2M rows of 128 1.31 against 1.37 ms).
    constexpr bool EARLY = sizeof(T) == 2;
    RawPiece<T, V> rf[K], rd[K], ra[K], ry[K], re[K];
    auto fetch = [&](int64_t r0) {
        const int64_t row = r0 + lane / LG, at = (row < A.n ? row : A.n - 1) * C;
        cols.fetch(A.f, at, rf);
        cols.fetch(A.gy, at, rd);
        cols.fetch(A.gate, at, ra);
        if (A.gn) {
            cols.fetch(A.y, at, ry);
            cols.fetch(A.gn, at, re);
        }
    };
    const int64_t first = ((int64_t)blockIdx.x * 4 + wave) * RW;
    if (EARLY && first < A.n) fetch(first);
    for (int64_t r0 = first; r0 < A.n; r0 += step) {
        const int64_t row = r0 + lane / LG;
        const bool live = row < A.n;
        const int64_t at = (live ? row : A.n - 1) * C;
        float v[K][V], w[K][V], d[K][V], e[K][V], a[K][V];
        if constexpr (!EARLY) fetch(r0);
        cols.get(A.f, rf, v);
        cols.get(A.gy, rd, d);
        cols.get(A.gate, ra, a);
        if (A.gn) {
            cols.get(A.y, ry, w);
            cols.get(A.gn, re, e);
        }
        if (EARLY && r0 + step < A.n) fetch(r0 + step);
        if (A.gn) {
            const float rs = norm_stats<LG, K, V>(w, cols.in, (float)C, A.eps);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    w[k][i] *= rs;
                    if (live) {
                        s[3][k][i] += e[k][i] * w[k][i];
                        s[4][k][i] += e[k][i];
                    }
                    e[k][i] *= gn[k][i];
                }
            norm_slope<LG, K, V>(e, w, rs, invC);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) d[k][i] += e[k][i];
        }
        if (live) cols.store(A.dx, at, d);
        const float rstd = norm_stats<LG, K, V>(v, cols.in, (float)C, A.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] *= rstd;
                d[k][i] = cols.in[k] ? d[k][i] : 0.f;
                const float m = v[k][i] * gp[k][i] + bp[k][i];
                float slope = 0.f, g = 1.f;
                if (A.gate) g = gate_sigmoid(a[k][i], slope);
                const float t = d[k][i] * sc[k][i] * g;
                a[k][i] = d[k][i] * sc[k][i] * m * slope;
                if (live) {
                    s[0][k][i] += t * v[k][i];
                    s[1][k][i] += t;
                    s[2][k][i] += d[k][i] * g * m;
                }
                e[k][i] = t * gp[k][i];
            }
        if (A.gate && live) cols.store(A.dgate, at, a);
        norm_slope<LG, K, V>(e, v, rstd, invC);
        if (live) cols.store(A.df, at, e);
    }
    // the wave's row groups, then the four waves
#pragma unroll
    for (int j = 0; j < SANDWICH_SUMS; ++j) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int m = LG; m < 64; m <<= 1) s[j][k][i] += __shfl_xor(s[j][k][i], m);
                if (lane < LG) sums[wave][(k * LG + lane % LG) * V + i] = s[j][k][i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += 256)
            A.part[((int64_t)blockIdx.x * SANDWICH_SUMS + j) * C + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
        __syncthreads();
    }
}

// The sums from those of the blocks: a workgroup takes 16 of the 5C columns, 16 threads each, in
// a fixed order.  A sum that is not wanted has no destination.
struct SandwichSums {
    float *to[SANDWICH_SUMS];
};
__global__ __launch_bounds__(256) void k_sandwich_join(const float *__restrict__ part, int nblk, int C, const SandwichSums d) {
    __shared__ double s[16][17];
    const int c = threadIdx.x & 15, q = threadIdx.x >> 4, at = blockIdx.x * 16 + c;
    double v = 0.0;
#pragma unroll 8
    for (int b = q; b < nblk; b += 16) v += part[(int64_t)b * SANDWICH_SUMS * C + at];
    s[q][c] = v;
    __syncthreads();
    if (q) return;
    for (int i = 1; i < 16; ++i) v += s[i][c];
    float *const to = d.to[at / C];
    if (to) to[at % C] = (float)v;
}

}  // namespace ts3
