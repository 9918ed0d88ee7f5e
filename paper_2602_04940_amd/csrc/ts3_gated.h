// Kernels of the gated feed-forward and of its gradient:
//
//   a = x Wg + bg,  u = x Wu + bu,  h = act(a) * u,  out = h Wd + bd
//
// and, for L = sum(g * out),
//
//   dh = g Wd^T,  da = dh * u * act'(a),  du = dh * act(a),
//   dx = da Wg^T + du Wu^T,  dWg = x^T da,  dWu = x^T du,  dWd = h^T g,
//   dbg, dbu, dbd = the column sums of da, du and g.
//
//   k_gated_load   the weights as matrix-core operands, by chunks of 32 hidden units
//   k_gated_fwd    the whole feed-forward in one kernel: the hidden layer never leaves
//                  the registers
//   k_gated_join   sums of outputs whose hidden units were split over workgroups
//   k_gated_dx     recomputes the hidden layer, gives dx, and leaves da, du and h of a
//                  tile of points in the store
//   k_gated_dw     the three weight gradients of the tile: products over its points
//   k_gated_grads  sums over the splits of the points, in index order
//
// Operands of bfloat16 are used as they are; float32 ones are sums of three bfloat16
// parts, six part products each (ts3_device.h).  Sums are float32.  Between the products,
// a hidden value is rounded once to bfloat16 (P = 1) or split exactly (P = 3).
//
// Every product is 32x32x16 (MT = 32) or 16x16x32 (MT = 16), lane l holding row or column
// l % MT and K slots 8 (l / MT) .. +7, and NV = MT/2 values per lane of a 32 x MT result
// (rows 32, in one or two tiles).  Operand rows are laid out so that these are the
// consecutive rows NV (l / MT) .. + NV - 1: a result's values then are, as they lie, the K
// slots of the next product's operand (no exchange between lanes, none through LDS), and
// what is stored of a point is 16 to 64 consecutive bytes per lane.
#pragma once
#include "ts3_device.h"
#include "ts3_pass1.h"  // transposing LDS reads

namespace ts3 {

typedef __attribute__((ext_vector_type(16))) float f32x16;

template <int MT> struct Mat;
template <> struct Mat<32> {
    static constexpr int KI = 16, HT = 1, KF = 2, NV = 16;  // K of a product; tiles, K steps of 32 rows
    typedef f32x16 D;
    __device__ static __forceinline__ void mma(D &d, const bf16x8 &a, const bf16x8 &b) {
        d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, d, 0, 0, 0);
    }
};
template <> struct Mat<16> {
    static constexpr int KI = 32, HT = 2, KF = 1, NV = 8;
    typedef f32x4 D;
    __device__ static __forceinline__ void mma(D &d, const bf16x8 &a, const bf16x8 &b) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0);
    }
};
// Which of 32 rows operand row i of tile t holds, so that lane group q holds rows NV q ..
// + NV - 1 of the result in order.
template <int MT> __host__ __device__ constexpr int gated_row(int t, int i) {
    return MT == 32 ? 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3) : 8 * (i >> 2) + 4 * t + (i & 3);
}

// A result of 32 rows by MT columns.
template <int MT> struct Rows32 {
    typename Mat<MT>::D d[Mat<MT>::HT];
    __device__ __forceinline__ float get(int v) const {
        if constexpr (MT == 32) return d[0][v];
        else return d[v >> 2][v & 3];
    }
    __device__ __forceinline__ void set(int v, float x) {
        if constexpr (MT == 32) d[0][v] = x;
        else d[v >> 2][v & 3] = x;
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int v = 0; v < Mat<MT>::NV; ++v) set(v, 0.f);
    }
};

__device__ __forceinline__ void to_parts(const float (&v)[8], Parts<1> &f) {
#pragma unroll
    for (int t = 0; t < 8; ++t) f.p[0][t] = (__bf16)v[t];
}
__device__ __forceinline__ void to_parts(const float (&v)[8], Parts<3> &f) { split8(v, f); }

// d += a b, the part products smallest first.
template <int MT, int P>
__device__ __forceinline__ void mma_parts(typename Mat<MT>::D &d, const Parts<P> &a, const Parts<P> &b) {
    using PP = PartProducts<P, P>;
#pragma unroll
    for (int q = 0; q < PP::N; ++q) Mat<MT>::mma(d, a.p[PP::I[q]], b.p[PP::J[q]]);
}

// Layout of the operands: chunks of 32 hidden units, six sections each and the chunk's
// biases, every fragment 1 KiB (64 lanes x 8 K slots) and the P parts of one in a row.
//   D        rows channels, K hidden: Wd      fragment (cb * HT + t) * KF + s
//   bias     1 KiB: bg[32], bu[32] as float32
//   G, U, H  rows hidden, K channels: Wg, Wu, Wd^T   fragment t * KS + ks
//   XG, XU   rows channels, K hidden: Wg, Wu  as D
// The forward reads (bias, G, U) and D, the backward (bias, G, U, H) and (XG, XU).
template <int P, int CP, int MT> struct GatedOps {
    using M = Mat<MT>;
    static constexpr int KS = CP / M::KI, CB = CP / 32;
    static constexpr int SEC = CP * 64 * P;
    static constexpr int BIAS = SEC, G = SEC + 1024, U = G + SEC, H = U + SEC, XG = H + SEC, XU = XG + SEC,
                         CHUNK = XU + SEC;
};

enum { GATED_SILU = 0, GATED_GELU = 1 };

// act(a) and act'(a).  SiLU: a s, s = 1 / (1 + e^-a); slope s + a s (1 - s).  GELU: a Phi(a);
// slope Phi + a phi.  For bfloat16 (P = 1), Phi by Abramowitz & Stegun 7.1.26: a polynomial in
// t = 1 / (1 + p |z|) times e^(-z^2), z = a / sqrt 2, whose exponential is also the density's;
// within 7.5e-8 of Phi.  That is not enough for float32, where the slope crosses zero (a =
// -0.75): there Phi comes from erfc.  For a very negative a, e^-a overflows to infinity and s = 0.
template <int P, bool SLOPE> __device__ __forceinline__ float gated_act(int kind, float a, float &slope) {
    constexpr float LOG2E = 1.44269504f;
    if (kind == GATED_SILU) {
        const float s = fast_rcp(1.f + fast_exp2(-LOG2E * a));
        const float y = a * s;
        if (SLOPE) slope = s + (y - y * s);
        return y;
    }
    float phi, e = 0.f;
    if (P == 1 || SLOPE) e = fast_exp2((-0.5f * LOG2E) * (a * a));
    if constexpr (P == 1) {
        const float t = fast_rcp(1.f + (0.3275911f * 0.70710678f) * fabsf(a));
        float q = 0.5f * 1.061405429f;
        q = q * t + 0.5f * -1.453152027f;
        q = q * t + 0.5f * 1.421413741f;
        q = q * t + 0.5f * -0.284496736f;
        q = q * t + 0.5f * 0.254829592f;
        q = q * t * e;
        phi = a < 0.f ? q : 1.f - q;
    } else {
        phi = 0.5f * erfcf(-0.70710678f * a);
    }
    if (SLOPE) slope = phi + a * (0.39894228f * e);
    return a * phi;
}

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<bf16_t>(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ bf16_t from_float<bf16_t>(float v) {
    return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)v)};
}
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }

// Storage type of an operand of P parts.
template <int P> struct GatedIO { typedef bf16_t T; };
template <> struct GatedIO<3> { typedef float T; };

// Eight consecutive elements of a row as an operand.
__device__ __forceinline__ void load_parts(const bf16_t *p, Parts<1> &f) { f.p[0] = *reinterpret_cast<const bf16x8 *>(p); }
__device__ __forceinline__ void load_parts(const float *p, Parts<3> &f) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split8(v, f);
}
// N consecutive values of a row, 16 bytes a time.
template <int N> __device__ __forceinline__ void store_row(bf16_t *p, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
        bf16x8 b;
#pragma unroll
        for (int t = 0; t < 8; ++t) b[t] = (__bf16)v[i + t];
        *reinterpret_cast<bf16x8 *>(p + i) = b;
    }
}
template <int N> __device__ __forceinline__ void store_row(float *p, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// The operands of every chunk from Wg, Wu [C][F] and Wd [F][C], and bd; channels past C and
// hidden units past F are zero.  One thread per eight K slots.
template <int P, int CP, int MT>
__global__ __launch_bounds__(256) void k_gated_load(const typename GatedIO<P>::T *__restrict__ Wg,
                                                    const typename GatedIO<P>::T *__restrict__ bg,
                                                    const typename GatedIO<P>::T *__restrict__ Wu,
                                                    const typename GatedIO<P>::T *__restrict__ bu,
                                                    const typename GatedIO<P>::T *__restrict__ Wd,
                                                    const typename GatedIO<P>::T *__restrict__ bd, int C, int F,
                                                    unsigned char *__restrict__ ops, float *__restrict__ bdp) {
    using O = GatedOps<P, CP, MT>;
    using M = Mat<MT>;
    constexpr int NF = O::SEC / (1024 * P);  // fragments of a section
    const int chunk = blockIdx.x;
    unsigned char *const base = ops + (size_t)chunk * O::CHUNK;
    for (int i = threadIdx.x + blockIdx.y * 256; i < 6 * NF * 64; i += gridDim.y * 256) {
        const int l = i & 63, f = (i >> 6) % NF, sec = i / (64 * NF);  // D, G, U, H, XG, XU
        const int row = l % MT, q = l / MT;
        float v[8];
        if (sec >= 1 && sec <= 3) {
            const int t = f / O::KS, ks = f % O::KS;
            const int hid = 32 * chunk + gated_row<MT>(t, row);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = M::KI * ks + 8 * q + j;
                const bool in = c < C && hid < F;
                v[j] = !in ? 0.f
                           : to_float(sec == 1 ? Wg[(size_t)c * F + hid] : sec == 2 ? Wu[(size_t)c * F + hid]
                                                                                     : Wd[(size_t)hid * C + c]);
            }
        } else {
            const int s = f % M::KF, t = f / M::KF % M::HT, cb = f / (M::KF * M::HT);
            const int c = 32 * cb + gated_row<MT>(t, row);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int hid = 32 * chunk + M::NV * q + 8 * s + j;
                const bool in = c < C && hid < F;
                v[j] = !in ? 0.f
                           : to_float(sec == 0 ? Wd[(size_t)hid * C + c] : sec == 4 ? Wg[(size_t)c * F + hid]
                                                                                     : Wu[(size_t)c * F + hid]);
            }
        }
        Parts<P> parts;
        to_parts(v, parts);
        unsigned char *const to = base + (sec == 0 ? 0 : 1024 + sec * O::SEC) + f * P * 1024 + l * 16;
#pragma unroll
        for (int p = 0; p < P; ++p) *reinterpret_cast<bf16x8 *>(to + p * 1024) = parts.p[p];
    }
    if (blockIdx.y == 0) {
        float *const bias = reinterpret_cast<float *>(base + O::BIAS);
        const int i = threadIdx.x, hid = 32 * chunk + (i & 31);
        const typename GatedIO<P>::T *const b = i < 32 ? bg : bu;
        bias[i] = i < 64 && b && hid < F ? to_float(b[hid]) : 0.f;
        if (chunk == 0 && i < CP) bdp[i] = bd && i < C ? to_float(bd[i]) : 0.f;
    }
}

// What the waves of a workgroup copy into LDS: BYTES (a multiple of 1 KiB) from src.
template <int BYTES, int WAVES> __device__ __forceinline__ void gated_stage(const unsigned char *src, uint32_t to, int wave, int lane) {
    constexpr int PIECES = BYTES / 1024;
#pragma unroll
    for (int k = 0; k < (PIECES + WAVES - 1) / WAVES; ++k)
        if (PIECES % WAVES == 0 || wave + k * WAVES < PIECES)
            dma16(src + (wave + k * WAVES) * 1024 + lane * 16, to + (wave + k * WAVES) * 1024);
}
__device__ __forceinline__ void gated_sync() {
    wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// Fragment f of a section staged at `sec`.
template <int P> __device__ __forceinline__ void lds_parts(const unsigned char *sec, int f, int lane, Parts<P> &a) {
#pragma unroll
    for (int p = 0; p < P; ++p) a.p[p] = *reinterpret_cast<const bf16x8 *>(sec + (f * P + p) * 1024 + lane * 16);
}

// The rows of NP x MT points as operands whose columns are points: K slots 8q .. of step ks
// are channels KI ks + 8q ...  Rows past n repeat row n - 1, channels past C are zero.
template <int P, int CP, int MT, int NP>
__device__ __forceinline__ void gated_rows(const typename GatedIO<P>::T *x, int64_t p0, int64_t n, int C,
                                           int lane, Parts<P> (&xf)[NP][CP / Mat<MT>::KI]) {
#pragma unroll
    for (int np = 0; np < NP; ++np) {
        const int64_t p = p0 + np * MT + lane % MT;
        const typename GatedIO<P>::T *const row = x + (p < n ? p : n - 1) * C;
#pragma unroll
        for (int ks = 0; ks < CP / Mat<MT>::KI; ++ks) {
            const int c = Mat<MT>::KI * ks + 8 * (lane / MT);
            if (c < C) load_parts(row + c, xf[np][ks]);
            else
#pragma unroll
                for (int s = 0; s < P; ++s) xf[np][ks].p[s] = bf16x8{};
        }
    }
}

// r[np] += section (rows hidden, K channels) times the points' rows.
template <int P, int CP, int MT, int NP>
__device__ __forceinline__ void gated_hidden(const unsigned char *sec, const Parts<P> (&xf)[NP][CP / Mat<MT>::KI], int lane,
                                             Rows32<MT> (&r)[NP]) {
    constexpr int KS = CP / Mat<MT>::KI;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < Mat<MT>::HT; ++t) {
            Parts<P> a;
            lds_parts(sec, t * KS + ks, lane, a);
#pragma unroll
            for (int np = 0; np < NP; ++np) mma_parts<MT, P>(r[np].d[t], a, xf[np][ks]);
        }
}
// acc[cb][np] += section (rows channels, K hidden) times hidden values.
template <int P, int CP, int MT, int NP>
__device__ __forceinline__ void gated_channels(const unsigned char *sec, const Parts<P> (&hf)[NP][Mat<MT>::KF], int lane,
                                               Rows32<MT> (&acc)[CP / 32][NP]) {
    using M = Mat<MT>;
#pragma unroll
    for (int s = 0; s < M::KF; ++s)
#pragma unroll
        for (int cb = 0; cb < CP / 32; ++cb)
#pragma unroll
            for (int t = 0; t < M::HT; ++t) {
                Parts<P> a;
                lds_parts(sec, (cb * M::HT + t) * M::KF + s, lane, a);
#pragma unroll
                for (int np = 0; np < NP; ++np) mma_parts<MT, P>(acc[cb][np].d[t], a, hf[np][s]);
            }
}
// The chunk's bias (which: 0 of the gate, 1 of the other map) as a result's first value.
template <int MT, int NP> __device__ __forceinline__ void gated_bias(const unsigned char *bias, int which, int lane, Rows32<MT> (&r)[NP]) {
    constexpr int NV = Mat<MT>::NV;
    const f32x4 *const b = reinterpret_cast<const f32x4 *>(bias + which * 128 + (lane / MT) * NV * 4);
#pragma unroll
    for (int v = 0; v < NV; v += 4) {
        const f32x4 w = b[v / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int np = 0; np < NP; ++np) r[np].set(v + i, w[i]);
    }
}

// Shapes of the two kernels that walk the hidden units: product shape, point tiles per wave,
// and the workgroups per compute unit that the registers are cut for.  The rows of wide
// float32 points fill the registers with 16 points per wave in the backward (MT = 16).
template <int P, int CP> struct GatedShape {
    static constexpr int MT = P == 3 && CP > 128 ? 16 : 32, NP = 32 / MT, WAVES = 4, PTS = WAVES * NP * MT;
    static constexpr int OCC = P == 1 ? 2 : CP <= 64 ? 2 : 1;
};
template <int P, int CP> struct GatedShapeX {
    static constexpr int MT = GatedShape<P, CP>::MT, NP = 1, WAVES = 4, PTS = WAVES * NP * MT;
    static constexpr int OCC = P == 1 && CP <= 128 ? 2 : P == 3 && CP <= 64 ? 2 : 1;
    // Where the five sections of a chunk do not fit LDS, they pass one by one through three slots.
    static constexpr bool RING = 1024 + 5 * CP * 64 * P > 160 * 1024;
    static constexpr int SLOT = 1024 + CP * 64 * P;
    static constexpr int LDS = RING ? 3 * SLOT : 1024 + 5 * CP * 64 * P;
};

// out = act(x Wg + bg) * (x Wu + bu) Wd + bd.  Workgroup (block b, split s) = (id / S, id % S)
// takes PTS points and chunks per*s .. of the hidden units; with S = 1 it writes out, else its
// sums to part[s][point][CP].
// A wave keeps its points' rows as operands and their output sums in registers, and walks the
// chunks: both products into the hidden layer, the activation, the product out of it.  (G, U)
// and D of a chunk have one LDS slot each; each is copied while the other's products run.
// out may be x: rows are read by their own workgroup alone, before its first barrier.
template <int P, int CP>
__global__ __launch_bounds__(256, (GatedShape<P, CP>::OCC)) void k_gated_fwd(
    const typename GatedIO<P>::T *x, int64_t n, int C, const unsigned char *__restrict__ ops, int nchunk, int per, int S,
    int act, const float *__restrict__ bdp, typename GatedIO<P>::T *out,
    float *__restrict__ part) {
    using Sh = GatedShape<P, CP>;
    constexpr int MT = Sh::MT, NP = Sh::NP, WAVES = Sh::WAVES;
    using M = Mat<MT>;
    using O = GatedOps<P, CP, MT>;
    constexpr int ABYTES = 1024 + 2 * O::SEC, NV = M::NV;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[ABYTES + O::SEC];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * NP * MT;
    const uint32_t la = lds_addr(lds), lb = la + ABYTES;
    const unsigned char *const sa = lds, *const sb = lds + ABYTES;

    gated_stage<ABYTES, WAVES>(ops + (size_t)j0 * O::CHUNK + O::BIAS, la, wave, lane);
    Parts<P> xf[NP][O::KS];
    gated_rows<P, CP, MT, NP>(x, p0, n, C, lane, xf);
    Rows32<MT> acc[O::CB][NP];
#pragma unroll
    for (int cb = 0; cb < O::CB; ++cb)
#pragma unroll
        for (int np = 0; np < NP; ++np) acc[cb][np].zero();
    gated_sync();
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
        gated_stage<O::SEC, WAVES>(ops + (size_t)j * O::CHUNK, lb, wave, lane);
        Rows32<MT> a[NP], u[NP];
        gated_bias<MT, NP>(sa, 0, lane, a);
        gated_bias<MT, NP>(sa, 1, lane, u);
        gated_hidden<P, CP, MT, NP>(sa + 1024, xf, lane, a);
        gated_hidden<P, CP, MT, NP>(sa + 1024 + O::SEC, xf, lane, u);
        Parts<P> hf[NP][M::KF];
#pragma unroll
        for (int np = 0; np < NP; ++np)
#pragma unroll
            for (int s = 0; s < M::KF; ++s) {
                float h[8], slope;
#pragma unroll
                for (int t = 0; t < 8; ++t) h[t] = gated_act<P, false>(act, a[np].get(8 * s + t), slope) * u[np].get(8 * s + t);
                to_parts(h, hf[np][s]);
            }
        gated_sync();  // D(j) is in LDS, (G, U)(j) read by all
        if (j + 1 < j1) gated_stage<ABYTES, WAVES>(ops + (size_t)(j + 1) * O::CHUNK + O::BIAS, la, wave, lane);
        gated_channels<P, CP, MT, NP>(sb, hf, lane, acc);
        gated_sync();  // (G, U)(j+1) is in LDS, D(j) read by all
    }
#pragma unroll
    for (int np = 0; np < NP; ++np) {
        const int64_t p = p0 + np * MT + lane % MT;
        if (p >= n) continue;
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb) {
            const int c = 32 * cb + NV * (lane / MT);
            float v[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = acc[cb][np].get(i);
            if (S > 1) store_row<NV>(part + ((int64_t)split * n + p) * CP + c, v);
            else if (c < C) {
#pragma unroll
                for (int i = 0; i < NV; ++i) v[i] += bdp[c + i];
                store_row<NV>(out + p * C + c, v);
            }
        }
    }
}

// out[p][c] = b[c] + sum over s of part[s][p][c], in the order of s.  Four channels a thread.
template <int P, int CP>
__global__ __launch_bounds__(256) void k_gated_join(const float *__restrict__ part, int64_t n, int C, int S,
                                                    const float *__restrict__ b, typename GatedIO<P>::T *__restrict__ out) {
    const int64_t total = n * (C / 4);
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t p = i / (C / 4);
        const int c = (int)(i % (C / 4)) * 4;
        f32x4 v = b ? *reinterpret_cast<const f32x4 *>(b + c) : f32x4{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < S; ++s) {
            const f32x4 w = *reinterpret_cast<const f32x4 *>(part + ((int64_t)s * n + p) * CP + c);
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] += w[t];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) out[p * C + c + t] = from_float<typename GatedIO<P>::T>(v[t]);
    }
}

// dx of n points (the first nb * PTS of the store's rows), and da, du, h in the store:
// store[m][chunk][tp][32], m = 0 da, 1 du, 2 h; rows of points past n are zero.  Grid, splits
// and LDS slots as k_gated_fwd, with (G, U, H) and (XG, XU).
template <int P, int CP>
__global__ __launch_bounds__(256, (GatedShapeX<P, CP>::OCC)) void k_gated_dx(
    const typename GatedIO<P>::T *__restrict__ x, const typename GatedIO<P>::T *__restrict__ g, int64_t n, int C,
    const unsigned char *__restrict__ ops, int nchunk, int per, int S, int act, int64_t tp,
    typename GatedIO<P>::T *__restrict__ store, typename GatedIO<P>::T *__restrict__ dx, float *__restrict__ part) {
    using T = typename GatedIO<P>::T;
    using Sh = GatedShapeX<P, CP>;
    constexpr int MT = Sh::MT, NP = Sh::NP, WAVES = Sh::WAVES;
    using M = Mat<MT>;
    using O = GatedOps<P, CP, MT>;
    constexpr int ABYTES = 1024 + 3 * O::SEC, BBYTES = 2 * O::SEC, NV = M::NV;
    // Stores of a chunk, issued after its copies: all of them may be in flight while those are waited for.
    constexpr int STORES = NP * 3 * NV * (int)sizeof(T) / 16;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Sh::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * NP * MT;
    const uint32_t la = lds_addr(lds);

    Parts<P> xf[NP][O::KS], gf[NP][O::KS];
    Rows32<MT> acc[O::CB][NP];
    Rows32<MT> a[NP], u[NP], dh[NP];
    Parts<P> daf[NP][M::KF], duf[NP][M::KF];
    auto start = [&]() {
        gated_rows<P, CP, MT, NP>(x, p0, n, C, lane, xf);
        gated_rows<P, CP, MT, NP>(g, p0, n, C, lane, gf);
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb)
#pragma unroll
            for (int np = 0; np < NP; ++np) acc[cb][np].zero();
    };
    // da, du and h of chunk j: the next products' operands, and their rows of the store.
    auto slopes = [&](int j) {
#pragma unroll
        for (int np = 0; np < NP; ++np) {
            const int64_t p = p0 + np * MT + lane % MT;
            const bool in = p < n;
            float da[NV], du[NV], h[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float slope;
                const float uv = u[np].get(v), d = in ? dh[np].get(v) : 0.f;
                const float y = gated_act<P, true>(act, a[np].get(v), slope);
                h[v] = in ? y * uv : 0.f;
                du[v] = d * y;
                da[v] = d * uv * slope;
            }
#pragma unroll
            for (int s = 0; s < M::KF; ++s) {
                float t0[8], t1[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    t0[t] = da[8 * s + t];
                    t1[t] = du[8 * s + t];
                }
                to_parts(t0, daf[np][s]);
                to_parts(t1, duf[np][s]);
            }
            asm volatile("" ::: "memory");
            T *const row = store + ((int64_t)j * tp + p) * 32 + NV * (lane / MT);
            const int64_t plane = (int64_t)nchunk * tp * 32;
            store_row<NV>(row, da);
            store_row<NV>(row + plane, du);
            store_row<NV>(row + 2 * plane, h);
        }
        asm volatile("" ::: "memory");
    };
    auto biases = [&](const unsigned char *bias) {
        gated_bias<MT, NP>(bias, 0, lane, a);
        gated_bias<MT, NP>(bias, 1, lane, u);
#pragma unroll
        for (int np = 0; np < NP; ++np) dh[np].zero();
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if constexpr (!Sh::RING) {
        const uint32_t lb = la + ABYTES;
        const unsigned char *const sa = lds, *const sb = lds + ABYTES;
        gated_stage<ABYTES, WAVES>(ops + (size_t)j0 * O::CHUNK + O::BIAS, la, wave, lane);
        start();
        gated_sync();
#pragma unroll 1
        for (int j = j0; j < j1; ++j) {
            gated_stage<BBYTES, WAVES>(ops + (size_t)j * O::CHUNK + O::XG, lb, wave, lane);
            biases(sa);
            gated_hidden<P, CP, MT, NP>(sa + 1024, xf, lane, a);
            gated_hidden<P, CP, MT, NP>(sa + 1024 + O::SEC, xf, lane, u);
            gated_hidden<P, CP, MT, NP>(sa + 1024 + 2 * O::SEC, gf, lane, dh);
            slopes(j);
            wait_vmcnt<STORES>();
            barrier();  // (XG, XU)(j) is in LDS, (G, U, H)(j) read by all
            if (j + 1 < j1) gated_stage<ABYTES, WAVES>(ops + (size_t)(j + 1) * O::CHUNK + O::BIAS, la, wave, lane);
            gated_channels<P, CP, MT, NP>(sb, daf, lane, acc);
            gated_channels<P, CP, MT, NP>(sb + O::SEC, duf, lane, acc);
            gated_sync();  // (G, U, H)(j+1) is in LDS, (XG, XU)(j) read by all
        }
    } else {
        // Step i = 5 (j - j0) + q reads section q of chunk j (bias and G, U, H, XG, XU) from slot
        // i % 3; the copies of step i + 2 are issued in step i, those of i + 1 waited for at its
        // end: the newest PER copies of the wave may still be in flight.
        constexpr int PER = O::SEC / 1024 / WAVES;
        static_assert(O::SEC % (1024 * WAVES) == 0, "every wave issues as many copies of a section");
        const int steps = 5 * (j1 - j0);
        auto issue = [&](int i) {
            const int j = j0 + i / 5, q = i % 5;
            const unsigned char *const src = ops + (size_t)j * O::CHUNK + O::G + q * O::SEC;
            const uint32_t to = la + (i % 3) * Sh::SLOT + 1024;
            if (q == 0 && wave == 0) dma16(src - 1024 + lane * 16, to - 1024);
            gated_stage<O::SEC, WAVES>(src, to, wave, lane);
        };
        auto next = [&](int i) {  // ends step i
            if (i + 2 < steps) wait_vmcnt<PER>();
            else wait_vmcnt<0>();
            barrier();
        };
        issue(0);
        issue(1);
        start();
        next(-1);
#pragma unroll 1
        for (int j = j0; j < j1; ++j) {
            const int i = 5 * (j - j0);
            auto slot = [&](int q) { return lds + ((i + q) % 3) * Sh::SLOT + 1024; };
            if (i + 2 < steps) issue(i + 2);
            biases(slot(0) - 1024);
            gated_hidden<P, CP, MT, NP>(slot(0), xf, lane, a);
            next(i);
            if (i + 3 < steps) issue(i + 3);
            gated_hidden<P, CP, MT, NP>(slot(1), xf, lane, u);
            next(i + 1);
            if (i + 4 < steps) issue(i + 4);
            gated_hidden<P, CP, MT, NP>(slot(2), gf, lane, dh);
            slopes(j);
            next(i + 2);
            if (i + 5 < steps) issue(i + 5);
            gated_channels<P, CP, MT, NP>(slot(3), daf, lane, acc);
            next(i + 3);
            if (i + 6 < steps) issue(i + 6);
            gated_channels<P, CP, MT, NP>(slot(4), duf, lane, acc);
            next(i + 4);
        }
    }
#pragma unroll
    for (int np = 0; np < NP; ++np) {
        const int64_t p = p0 + np * MT + lane % MT;
        if (p >= n) continue;
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb) {
            const int c = 32 * cb + NV * (lane / MT);
            float v[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = acc[cb][np].get(i);
            if (S > 1) store_row<NV>(part + ((int64_t)split * n + p) * CP + c, v);
            else if (c < C) store_row<NV>(dx + p * C + c, v);
        }
    }
}

// Shape of the weight gradients' kernel: a wave's result is 64 hidden units by CTW tiles of
// 32 channels, four waves cover HB hidden units by CP channels.
template <int P, int CP> struct GatedDw {
    static constexpr int WC = CP > 128 ? 2 : 1, WH = 4 / WC, HB = 64 * WH, CTW = CP / 32 / WC;
    static constexpr int HPL = HB / 32, PL = HPL + CP / 32;  // planes of 32 columns
    static constexpr int KP = P == 1 ? 32 : 16;              // points per step
    static constexpr int SLOTS = P == 1 ? 3 : 2;
    static constexpr int PLB = KP * 64;                      // bytes of a plane (of one part)
    static constexpr int SLOT = PL * PLB * P;
    static constexpr int PIECES = P == 1 ? PL * 2 : PL * 2;  // 1 KiB copies (P = 1), 16-row-by-64-byte loads
    static constexpr int PER = (PIECES + 3) / 4;
    static_assert(CP % 64 == 0, "two channel waves share CP evenly");
};

// One operand whose K slots are points: columns 32 of plane at `plane` (rows of 64 bytes),
// K slots 8q .. of the 16 points from row r0.  Lanes 0..31 and 32..63 read 256 consecutive
// bytes each.
__device__ __forceinline__ bf16x8 plane_tr(const unsigned char *plane, int r0, int lane) {
    const int j = lane & 15;
    const unsigned char *lo = plane + (r0 + 8 * (lane >> 5) + (j >> 2)) * 64 + 32 * ((lane >> 4) & 1) + 8 * (j & 3);
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lo);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lo + 256));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
}
// Sum of the first `count` slots.
__device__ __forceinline__ float sum_slots(const bf16x8 &v, int count = 8) {
    const u32x4 u = __builtin_bit_cast(u32x4, v);
    float w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[2 * i] = __uint_as_float(u[i] << 16);
        w[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    if (count < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < count ? w[i] : 0.f;
    return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
}

// The weight gradients of the tile's points: for m = 0 (dWg), 1 (dWu): sum of da or du times
// x; for 2 (dWd): of h times g.  Workgroup (m, hidden block hb, split sp) with sp outermost
// sums points per*sp .. + per - 1 (per a multiple of KP) into part[sp][m][nchunk * 32][CP] and
// bpart[sp][m][max(nchunk * 32, CP)] (sums of da, du; for m = 2 of g), added to what is there
// unless `first`.  Rows of x and g past n repeat row n - 1, against zeros of the store in the
// products.  The biases' sums run over as many terms as there are points: float64.
template <int P, int CP>
__global__ __launch_bounds__(256, 2) void k_gated_dw(const typename GatedIO<P>::T *__restrict__ x,
                                                     const typename GatedIO<P>::T *__restrict__ g, int64_t n, int C,
                                                     const typename GatedIO<P>::T *__restrict__ store, int nchunk,
                                                     int64_t tp, int64_t per, int nhb, int first,
                                                     float *__restrict__ part, float *__restrict__ bpart) {
    using T = typename GatedIO<P>::T;
    using S = GatedDw<P, CP>;
    constexpr int KP = S::KP, HPL = S::HPL, PL = S::PL, CTW = S::CTW;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::SLOTS * S::SLOT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wid = blockIdx.x;
    const int hb = wid % nhb, m = wid / nhb % 3, sp = wid / (3 * nhb);
    const int hi = wave / S::WC, ci = wave % S::WC;
    const int64_t a0 = (int64_t)sp * per, a1 = a0 + per < tp ? a0 + per : tp;
    const int nk = a0 < a1 ? (int)((a1 - a0) / KP) : 0;
    const T *const cols = m == 2 ? g : x;
    const T *const hid = store + (int64_t)m * nchunk * tp * 32;
    const int FP = nchunk * 32, BW = FP > CP ? FP : CP;

    // Piece k of a step: 16 points by one plane; lane l takes row l/4, 16 bytes (P = 1) or row
    // l/4, 32 bytes of floats (P = 3).
    auto source = [&](int k, int64_t p0) -> const T * {
        const int pl = k % PL, half = k / PL;  // half: which 16 of 32 points (P = 1), or 16 of 32 columns (P = 3)
        const int row = P == 1 ? 16 * half + (lane >> 2) : lane >> 2;
        const int col = P == 1 ? 8 * (lane & 3) : 16 * half + 4 * (lane & 3);
        if (pl < HPL) {
            int ch = hb * HPL + pl;
            ch = ch < nchunk ? ch : nchunk - 1;
            return hid + ((int64_t)ch * tp + p0 + row) * 32 + col;
        }
        int64_t p = p0 + row;
        p = p < n ? p : n - 1;
        const int c = 32 * (pl - HPL) + col;
        return cols + p * C + (c < C ? c : 0);  // channels past C: any, never stored
    };
    f32x16 acc[2][CTW];
    double bsum[2] = {0.0, 0.0}, gsum[CTW];
    const bool bh = m < 2 && ci == 0, bc = m == 2 && hb == 0 && hi == 0;
    float *const bp = bpart + ((int64_t)sp * 3 + m) * BW;
    float *const wp = part + (((int64_t)sp * 3 + m) * FP + hb * S::HB + hi * 64) * CP + ci * CTW * 32;
    auto hidden_in = [&](int t) { return hb * S::HB + hi * 64 + t * 32 < FP; };
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < CTW; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * t + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                acc[t][c][r] = first || !hidden_in(t) ? 0.f : wp[(int64_t)row * CP + 32 * c + (lane & 31)];
            }
#pragma unroll
    for (int c = 0; c < CTW; ++c) gsum[c] = 0.0;

    auto products = [&](const unsigned char *slot, int64_t left) {  // points up to row n of this step's rows
#pragma unroll
        for (int r0 = 0; r0 < KP; r0 += 16) {
            Parts<P> af[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p) af[t].p[p] = plane_tr(slot + ((2 * hi + t) * P + p) * S::PLB, r0, lane);
            if (bh)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int p = 0; p < P; ++p) bsum[t] += sum_slots(af[t].p[p]);
#pragma unroll
            for (int c = 0; c < CTW; ++c) {
                Parts<P> bf;
#pragma unroll
                for (int p = 0; p < P; ++p) bf.p[p] = plane_tr(slot + ((HPL + ci * CTW + c) * P + p) * S::PLB, r0, lane);
                if (bc) {
                    const int64_t in = left - r0 - 8 * (lane >> 5);
#pragma unroll
                    for (int p = 0; p < P; ++p) gsum[c] += sum_slots(bf.p[p], in < 8 ? (int)in : 8);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) mma_parts<32, P>(acc[t][c], af[t], bf);
            }
        }
    };
    if constexpr (P == 1) {
        const uint32_t base = lds_addr(lds);
        auto issue = [&](int k) {
#pragma unroll
            for (int i = 0; i < S::PER; ++i) {
                const int pc = wave * S::PER + i;
                if (S::PIECES % 4 == 0 || pc < S::PIECES)
                    dma16(source(pc, a0 + (int64_t)k * KP),
                          base + (k % S::SLOTS) * S::SLOT + (pc % PL) * S::PLB + (pc / PL) * 1024);
            }
        };
        static_assert(S::PIECES % 4 == 0, "every wave issues as many copies");
        if (nk > 0) issue(0);
        if (nk > 1) issue(1);
#pragma unroll 1
        for (int k = 0; k < nk; ++k) {
            if (k + 1 < nk) wait_vmcnt<S::PER>();
            else wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();  // step k is in LDS; step k - 1's slot read by all
            asm volatile("" ::: "memory");
            if (k + 2 < nk) issue(k + 2);
            products(lds + (k % S::SLOTS) * S::SLOT, n - a0 - (int64_t)k * KP);
        }
    } else {
        f32x4 st[S::PER];
        auto fetch = [&](int k) {
#pragma unroll
            for (int i = 0; i < S::PER; ++i)
                st[i] = *reinterpret_cast<const f32x4 *>(source(wave * S::PER + i, a0 + (int64_t)k * KP));
        };
        auto put = [&](int k) {
#pragma unroll
            for (int i = 0; i < S::PER; ++i) {
                const int pc = wave * S::PER + i, pl = pc % PL;
                unsigned char *to = lds + (k % S::SLOTS) * S::SLOT + pl * P * S::PLB + (lane >> 2) * 64 + 32 * (pc / PL) + 8 * (lane & 3);
                typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
                u32x2 w[3];
#pragma unroll
                for (int t = 0; t < 4; t += 2) {
                    const uint32_t h = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)st[i][t], (__bf16)st[i][t + 1]});
                    const float r0 = st[i][t] - __uint_as_float(h << 16), r1 = st[i][t + 1] - __uint_as_float(h & 0xffff0000u);
                    const uint32_t md = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)r0, (__bf16)r1});
                    w[0][t >> 1] = h;
                    w[1][t >> 1] = md;
                    w[2][t >> 1] = __builtin_bit_cast(
                        uint32_t, bf16x2{(__bf16)(r0 - __uint_as_float(md << 16)), (__bf16)(r1 - __uint_as_float(md & 0xffff0000u))});
                }
#pragma unroll
                for (int p = 0; p < P; ++p) *reinterpret_cast<u32x2 *>(to + p * S::PLB) = w[p];
            }
        };
        static_assert(S::PIECES % 4 == 0, "every wave loads as many pieces");
        if (nk > 0) {
            fetch(0);
            put(0);
        }
#pragma unroll 1
        for (int k = 0; k < nk; ++k) {
            if (k + 1 < nk) fetch(k + 1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();  // step k is in LDS; step k - 1's slot read by all
            asm volatile("" ::: "memory");
            products(lds + (k % S::SLOTS) * S::SLOT, n - a0 - (int64_t)k * KP);
            if (k + 1 < nk) put(k + 1);
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (!hidden_in(t)) continue;
#pragma unroll
        for (int c = 0; c < CTW; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * t + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                wp[(int64_t)row * CP + 32 * c + (lane & 31)] = acc[t][c][r];
            }
        if (bh) {
            const float s = (float)(bsum[t] + __shfl_xor(bsum[t], 32));
            float *const to = bp + hb * S::HB + hi * 64 + t * 32 + (lane & 31);
            if (lane < 32) *to = first ? s : *to + s;
        }
    }
    if (bc)
#pragma unroll
        for (int c = 0; c < CTW; ++c) {
            const float s = (float)(gsum[c] + __shfl_xor(gsum[c], 32));
            float *const to = bp + (ci * CTW + c) * 32 + (lane & 31);
            if (lane < 32) *to = first ? s : *to + s;
        }
}

// The gradients from the splits' sums, in index order: block (hidden tile of 32, channel tile
// of 32, m), 256 threads.  dWg and dWu are [C][F], dWd [F][C].
template <int P, int CP>
__global__ __launch_bounds__(256) void k_gated_grads(const float *__restrict__ part, const float *__restrict__ bpart, int SP,
                                                     int nchunk, int C, int F, typename GatedIO<P>::T *__restrict__ dWg,
                                                     typename GatedIO<P>::T *__restrict__ dWu,
                                                     typename GatedIO<P>::T *__restrict__ dWd,
                                                     typename GatedIO<P>::T *__restrict__ dbg,
                                                     typename GatedIO<P>::T *__restrict__ dbu,
                                                     typename GatedIO<P>::T *__restrict__ dbd) {
    using T = typename GatedIO<P>::T;
    __shared__ float tile[32][33];
    const int ht = blockIdx.x, ct = blockIdx.y, m = blockIdx.z;
    const int FP = nchunk * 32, BW = FP > CP ? FP : CP;
    const int col = threadIdx.x & 31, r8 = threadIdx.x >> 5;
    const int64_t stride = (int64_t)3 * FP * CP;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    const float *src = part + ((int64_t)m * FP + 32 * ht + r8) * CP + 32 * ct + col;
    for (int s = 0; s < SP; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += src[s * stride + (int64_t)8 * i * CP];
    if (m == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int f = 32 * ht + r8 + 8 * i, c = 32 * ct + col;
            if (f < F && c < C) dWd[(int64_t)f * C + c] = from_float<T>((float)v[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[r8 + 8 * i][col] = (float)v[i];
        __syncthreads();
        T *const to = m ? dWu : dWg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int f = 32 * ht + col, c = 32 * ct + r8 + 8 * i;
            if (f < F && c < C) to[(int64_t)c * F + f] = from_float<T>(tile[col][r8 + 8 * i]);
        }
    }
    // Column sums: by the first channel tile's blocks (da, du), the first hidden tile's (g).
    if (threadIdx.x < 32 && (m == 2 ? ht == 0 : ct == 0)) {
        const int at = 32 * (m == 2 ? ct : ht) + col;
        double s = 0.0;
        for (int i = 0; i < SP; ++i) s += bpart[((int64_t)i * 3 + m) * BW + at];
        T *const to = m == 0 ? dbg : m == 1 ? dbu : dbd;
        if (at < (m == 2 ? C : F)) to[at] = from_float<T>((float)s);
    }
}

}  // namespace ts3
