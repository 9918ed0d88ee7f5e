// The residual LayerNorm of a pre-norm block and its gradient, over rows of C values:
//
//   y = x + r,  h = (y - mean(y)) rstd(y),  out = h gamma + beta      (biased variance)
//   dx = r + rstd (e - mean(e) - h mean(e h)),  e = g gamma
//   dgamma = sum over rows of g h,  dbeta = sum over rows of g
//
// Both move each row once and are bound by that.  A group of LG lanes holds a row, K pieces of
// 16 bytes each, so that every load and store of a wave is whole lines and the row sums are a
// few lane exchanges; statistics are taken from the registers, the variance about the mean.
#pragma once
#include "ts3_gated.h"  // storage types

namespace ts3 {

// Sum over groups of LG lanes (a power of two); every lane gets its group's.
template <int LG> __device__ __forceinline__ float group_sum(float v) {
    if constexpr (LG >= 2) v += dpp<0xB1>(v);    // quad_perm [1,0,3,2]
    if constexpr (LG >= 4) v += dpp<0x4E>(v);    // quad_perm [2,3,0,1]
    if constexpr (LG >= 8) v += dpp<0x141>(v);   // row_half_mirror
    if constexpr (LG >= 16) v += dpp<0x140>(v);  // row_mirror
    if constexpr (LG >= 32) {
        auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if constexpr (LG >= 64) {
        auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    return v;
}

template <typename T> struct Piece;  // 16 bytes of a row
template <> struct Piece<bf16_t> {
    static constexpr int V = 8;
    __device__ static __forceinline__ void load(const bf16_t *p, float (&v)[8]) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};
template <> struct Piece<float> {
    static constexpr int V = 4;
    __device__ static __forceinline__ void load(const float *p, float (&v)[4]) {
        const f32x4 u = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = u[i];
    }
};

// mean and 1 / sqrt(variance + eps) of the row in v, which is left centred (0 past C).  The mean
// is divided, not multiplied by 1/C: where the spread is below sqrt(eps), its rounding is scaled up.
template <int LG, int K, int V>
__device__ __forceinline__ float norm_stats(float (&v)[K][V], const bool (&in)[K], float C, float eps) {
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s += v[k][i];
    const float mean = group_sum<LG>(s) / C;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[k][i] = in[k] ? v[k][i] - mean : 0.f;
            q += v[k][i] * v[k][i];
        }
    return 1.f / sqrtf(group_sum<LG>(q) / C + eps);
}

// r may be NULL (then y, if not NULL, is a copy of x).
template <typename T, int LG, int K>
__global__ __launch_bounds__(256) void k_norm_fwd(const T *x, const T *r, const float *__restrict__ gamma,
                                                  const float *__restrict__ beta, int64_t n, int C, float eps, T *y,
                                                  T *__restrict__ out) {
    constexpr int V = Piece<T>::V, RW = 64 / LG;
    const int lane = threadIdx.x & 63, sub = lane % LG;
    float gm[K][V], bt[K][V];
    bool in[K];
    int col[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        in[k] = (k * LG + sub) * V < C;
        col[k] = in[k] ? (k * LG + sub) * V : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            gm[k][i] = gamma[col[k] + i];
            bt[k][i] = beta[col[k] + i];
        }
    }
    const int64_t step = (int64_t)gridDim.x * 4 * RW;
    for (int64_t r0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * RW; r0 < n; r0 += step) {
        const int64_t row = r0 + lane / LG;
        const bool live = row < n;
        const int64_t at = (live ? row : n - 1) * C;
        float v[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Piece<T>::load(x + at + col[k], v[k]);
            if (r) {
                float w[V];
                Piece<T>::load(r + at + col[k], w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[k][i] += w[i];
            }
            if (live && in[k] && y) store_row<V>(y + at + col[k], v[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = in[k] ? v[k][i] : 0.f;
        }
        const float rstd = norm_stats<LG, K, V>(v, in, (float)C, eps);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = v[k][i] * rstd * gm[k][i] + bt[k][i];
            if (live && in[k]) store_row<V>(out + at + col[k], o);
        }
    }
}

// Column sums of the block's rows go to part[block][2][C] (dgamma, dbeta).
template <typename T, int LG, int K>
__global__ __launch_bounds__(256) void k_norm_bwd(const T *__restrict__ y, const T *g, const T *r,
                                                  const float *__restrict__ gamma, int64_t n, int C, float eps, T *dx,
                                                  float *__restrict__ part) {
    constexpr int V = Piece<T>::V, RW = 64 / LG, W = LG * K * V;
    __shared__ float sums[4][2][W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LG;
    const float invC = 1.f / C;
    float gm[K][V], sg[K][V], sb[K][V];
    bool in[K];
    int col[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        in[k] = (k * LG + sub) * V < C;
        col[k] = in[k] ? (k * LG + sub) * V : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            gm[k][i] = gamma[col[k] + i];
            sg[k][i] = sb[k][i] = 0.f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * 4 * RW;
    for (int64_t r0 = ((int64_t)blockIdx.x * 4 + wave) * RW; r0 < n; r0 += step) {
        const int64_t row = r0 + lane / LG;
        const bool live = row < n;
        const int64_t at = (live ? row : n - 1) * C;
        float v[K][V], e[K][V], w[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Piece<T>::load(y + at + col[k], v[k]);
            Piece<T>::load(g + at + col[k], e[k]);
            if (r) Piece<T>::load(r + at + col[k], w[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] = in[k] ? v[k][i] : 0.f;
                e[k][i] = in[k] && live ? e[k][i] : 0.f;
                if (!r) w[k][i] = 0.f;
            }
        }
        const float rstd = norm_stats<LG, K, V>(v, in, (float)C, eps);
        float m1 = 0.f, m2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] *= rstd;
                if (live) {
                    sg[k][i] += e[k][i] * v[k][i];
                    sb[k][i] += e[k][i];
                }
                e[k][i] *= gm[k][i];
                m1 += e[k][i];
                m2 += e[k][i] * v[k][i];
            }
        m1 = group_sum<LG>(m1) * invC;
        m2 = group_sum<LG>(m2) * invC;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[k][i] += rstd * (e[k][i] - m1 - v[k][i] * m2);
            if (live && in[k]) store_row<V>(dx + at + col[k], w[k]);
        }
    }
    // the wave's row groups, then the four waves
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int m = LG; m < 64; m <<= 1) {
                sg[k][i] += __shfl_xor(sg[k][i], m);
                sb[k][i] += __shfl_xor(sb[k][i], m);
            }
            if (lane < LG) {
                sums[wave][0][(k * LG + sub) * V + i] = sg[k][i];
                sums[wave][1][(k * LG + sub) * V + i] = sb[k][i];
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * C; i += 256) {
        const int which = i >= C, c = which ? i - C : i;
        part[(int64_t)blockIdx.x * 2 * C + i] =
            (sums[0][which][c] + sums[1][which][c]) + (sums[2][which][c] + sums[3][which][c]);
    }
}

// dgamma and dbeta from the blocks' sums: a workgroup takes 16 of the 2C columns, 16 threads
// each, in a fixed order.
__global__ __launch_bounds__(256) void k_norm_join(const float *__restrict__ part, int nblk, int C,
                                                   float *__restrict__ dgamma, float *__restrict__ dbeta) {
    __shared__ float s[16][17];
    const int c = threadIdx.x & 15, q = threadIdx.x >> 4, at = blockIdx.x * 16 + c;
    float v = 0.f;
#pragma unroll 8
    for (int b = q; b < nblk; b += 16) v += part[(int64_t)b * 2 * C + at];
    s[q][c] = v;
    __syncthreads();
    if (q) return;
    for (int i = 1; i < 16; ++i) v += s[i][c];
    if (at < C) dgamma[at] = v;
    else dbeta[at - C] = v;
}

}  // namespace ts3
