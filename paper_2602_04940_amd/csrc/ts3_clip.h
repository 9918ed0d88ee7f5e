// The global norm of a list of tensors and the list scaled to it:
//
//   norm = sqrt(sum of the squares of every element),  dst = src * min(1, max_norm / norm)
//
// Two passes over the data, both bound by it: k_clip_sums leaves one sum of squares per piece
// of a tensor, k_clip_scale adds them up again in every workgroup (in one order: a few thousand
// sums cost less than a launch of their own) and scales its piece.  Squares and their sums are
// float64, so no float32 gradient overflows or vanishes in them.
//
// The tensors come as kernel arguments, CLIP_BATCH per launch: nothing is copied to the device
// and a captured launch keeps its list.
#pragma once
#include "ts3_gated.h"  // storage types

namespace ts3 {

constexpr int CLIP_BATCH = 96;
struct ClipBatch {
    const void *src[CLIP_BATCH];
    void *dst[CLIP_BATCH];
    int64_t n[CLIP_BATCH];             // elements, times two, plus one for bfloat16
    int32_t first[CLIP_BATCH + 1];     // first piece of each tensor in the launch
    int32_t count;
};

// The tensor that holds piece b, and the piece's elements [a, e).
__device__ __forceinline__ int clip_find(const ClipBatch &t, int b, int64_t piece, int64_t &a, int64_t &e) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (t.first[m] <= b) lo = m;
        else hi = m;
    }
    const int64_t n = t.n[lo] >> 1;
    a = (int64_t)(b - t.first[lo]) * piece;
    e = a + piece < n ? a + piece : n;
    return lo;
}
// Elements before the first 16-byte boundary of p, at most n.
template <typename T> __device__ __forceinline__ int64_t clip_head(const T *p, int64_t n) {
    const int64_t h = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int64_t)sizeof(T);
    return h < n ? h : n;
}
// Sum over the workgroup's 256 threads, in one order; every thread gets it.
__device__ __forceinline__ double clip_block_sum(double s, double *lds) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T> __device__ __forceinline__ double clip_squares(const T *p, int64_t n) {
    constexpr int V = 16 / sizeof(T);
    const int64_t head = clip_head(p, n), vecs = (n - head) / V;
    double s = 0.0;
    if (threadIdx.x < head) {
        const double v = to_float(p[threadIdx.x]);
        s += v * v;
    }
    const u32x4 *const q = reinterpret_cast<const u32x4 *>(p + head);
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < vecs; i += 256) {
        const u32x4 u = q[i];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if constexpr (sizeof(T) == 4) {
                const double v = __uint_as_float(u[t]);
                s += v * v;
            } else {
                const double v = __uint_as_float(u[t] << 16), w = __uint_as_float(u[t] & 0xffff0000u);
                s += v * v;
                s += w * w;
            }
        }
    }
    const int64_t tail = head + vecs * V + threadIdx.x;
    if (tail < n) {
        const double v = to_float(p[tail]);
        s += v * v;
    }
    return s;
}

// sums[base + b] = the squares of piece b of the launch.
__global__ __launch_bounds__(256) void k_clip_sums(const ClipBatch t, int64_t piece, int base, double *__restrict__ sums) {
    __shared__ double lds[4];
    int64_t a, e;
    const int i = clip_find(t, blockIdx.x, piece, a, e);
    const double s = t.n[i] & 1 ? clip_squares((const bf16_t *)t.src[i] + a, e - a)
                                : clip_squares((const float *)t.src[i] + a, e - a);
    const double sum = clip_block_sum(s, lds);
    if (threadIdx.x == 0) sums[base + blockIdx.x] = sum;
}

template <typename T> __device__ __forceinline__ void clip_scale(const T *p, T *d, int64_t n, float scale) {
    constexpr int V = 16 / sizeof(T);
    // Where source and destination lie differently about the 16-byte boundaries, elements go one by one.
    const bool same = (((uintptr_t)p ^ (uintptr_t)d) & 15) == 0;
    const int64_t head = same ? clip_head(p, n) : n, vecs = (n - head) / V;
    for (int64_t i = threadIdx.x; i < head; i += 256) d[i] = from_float<T>(to_float(p[i]) * scale);
    const u32x4 *const q = reinterpret_cast<const u32x4 *>(p + head);
    u32x4 *const o = reinterpret_cast<u32x4 *>(d + head);
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < vecs; i += 256) {
        u32x4 u = q[i];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if constexpr (sizeof(T) == 4) u[t] = __float_as_uint(__uint_as_float(u[t]) * scale);
            else
                u[t] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(__uint_as_float(u[t] << 16) * scale),
                                                           (__bf16)(__uint_as_float(u[t] & 0xffff0000u) * scale)});
        }
        o[i] = u;
    }
    const int64_t tail = head + vecs * V + threadIdx.x;
    if (tail < n) d[tail] = from_float<T>(to_float(p[tail]) * scale);
}

// dst = src * min(1, max_norm / norm) from the `total` sums of every launch; the first launch
// writes the norm.  In place, a piece that needs no scaling is left alone.
__global__ __launch_bounds__(256) void k_clip_scale(const ClipBatch t, int64_t piece, int total, float max_norm,
                                                    const double *__restrict__ sums, float *__restrict__ norm) {
    __shared__ double lds[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < total; i += 256) s += sums[i];
    const double nrm = sqrt(clip_block_sum(s, lds));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)nrm;
    if (t.count == 0) return;
    const float scale = nrm > (double)max_norm ? (float)((double)max_norm / nrm) : 1.f;
    int64_t a, e;
    const int i = clip_find(t, blockIdx.x, piece, a, e);
    if (scale == 1.f && t.src[i] == t.dst[i]) return;
    if (t.n[i] & 1) clip_scale((const bf16_t *)t.src[i] + a, (bf16_t *)t.dst[i] + a, e - a, scale);
    else clip_scale((const float *)t.src[i] + a, (float *)t.dst[i] + a, e - a, scale);
}

}  // namespace ts3
