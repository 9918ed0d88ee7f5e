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
//   k_gated_slopes, k_gated_slopes3, k_gated_dx_wide   the same in two kernels, for bfloat16 points
//                  wider than 128 and float32 ones of 65 to 128 channels
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

// d[i] += a[i] b[i] for N results in turn, the part products smallest first: a product that adds
// to the one before it takes twice as long.
// `beside(q)` is issued after part product q of each.
template <int MT, int P, int N, typename F>
__device__ __forceinline__ void mma_parts_in_turn(typename Mat<MT>::D *const (&d)[N], const Parts<P> (&a)[N],
                                                  const Parts<P> *const (&b)[N], F beside) {
    using PP = PartProducts<P, P>;
#pragma unroll
    for (int q = 0; q < PP::N; ++q) {
#pragma unroll
        for (int i = 0; i < N; ++i) Mat<MT>::mma(*d[i], a[i].p[PP::I[q]], b[i]->p[PP::J[q]]);
        beside(q);
        // The compiler would put each result's products back into a row, and what goes beside them
        // before them: only loads, stores and scalar instructions may pass here.
        if constexpr (P > 1) __builtin_amdgcn_sched_barrier(0x094);
    }
}
template <int MT, int P, int N>
__device__ __forceinline__ void mma_parts_in_turn(typename Mat<MT>::D *const (&d)[N], const Parts<P> (&a)[N],
                                                  const Parts<P> *const (&b)[N]) {
    mma_parts_in_turn<MT, P, N>(d, a, b, [](int) {});
}
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

// act(a) and act'(a), the same in the forward and the backward.  SiLU: a s, s = 1 / (1 + e^-a); slope
// s + a s (1 - s).  For a very negative a, e^-a overflows to infinity and s = 0.  GELU: a Phi(a);
// slope Phi + a phi.  The exponentials are the hardware's, of a product rounded to float32: good to
// some |a| 2^-24 of themselves in SiLU, a^2 2^-24 in GELU.
// Float32 takes Phi from erfc and the density from its exponential.
// Bfloat16 takes Phi(-z) = e^(-z^2/2) Q(t), t = 1 / (1 + p z), z = |a|, whose exponential is also the
// density's.  Q is a polynomial of five terms without a constant, fitted here with p by a linear
// program on z up to 13.3: minimax of the relative error for Phi(-z) < 0.01, of the absolute one
// for smaller z.  Phi is within 1.7e-6, which the slope needs where it crosses zero (a = -0.75), and
// GELU within 1.3e-4 of itself down to a = -13, a fifteenth of a bfloat16 rounding of the hidden value
// (2e-3).  Below, where GELU leaves the normal float32 numbers, e vanishes.  A logistic form,
// Phi ~ 1 / (1 + 2^-u) with u an odd polynomial of four terms, takes 365 us instead of 380 (forward of
// 250,000 points at C = 256, F = 1024) but holds relative to GELU only as far as a = -4.8.
template <int P, int ACT, bool SLOPE> __device__ __forceinline__ float gated_act(float a, float &slope) {
    constexpr float LOG2E = 1.44269504f;
    if constexpr (ACT == GATED_SILU) {
        const float s = fast_rcp(1.f + fast_exp2(-LOG2E * a));
        const float y = a * s;
        if (SLOPE) slope = s + (y - y * s);
        return y;
    } else {
        float phi, e = 0.f;
        if (P == 1 || SLOPE) e = fast_exp2((-0.5f * LOG2E) * (a * a));
        if constexpr (P == 1) {
            const float t = fast_rcp(1.f + 0.358239511f * fabsf(a));
            float q = -0.0928955438f;
            q = q * t + 0.241391272f;
            q = q * t + 0.0510493026f;
            q = q * t + 0.158779151f;
            q = q * t + 0.141674645f;
            q = q * t * e;
            phi = a < 0.f ? q : 1.f - q;
        } else {
            phi = 0.5f * erfcf(-0.70710678f * a);
        }
        if (SLOPE) slope = phi + a * (0.39894228f * e);
        return a * phi;
    }
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
            dma16s<0>(lane * 16, src + (wave + k * WAVES) * 1024, to + (wave + k * WAVES) * 1024);
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
// are channels KI ks + 8q ...  Rows past n and channels past C are zero.
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
            load_parts(row + (c < C ? c : 0), xf[np][ks]);  // no branch: the loads leave together
#pragma unroll
            for (int s = 0; s < P; ++s) xf[np][ks].p[s] = c < C && p < n ? xf[np][ks].p[s] : bf16x8{};
        }
    }
}

// r[np] += section (rows hidden, K channels) times the points' rows, K step ks.
template <int P, int CP, int MT, int NP>
__device__ __forceinline__ void gated_hidden(const unsigned char *sec, const Parts<P> (&xf)[NP][CP / Mat<MT>::KI], int ks,
                                             int lane, Rows32<MT> (&r)[NP]) {
#pragma unroll
    for (int t = 0; t < Mat<MT>::HT; ++t) {
        Parts<P> a;
        lds_parts(sec, t * (CP / Mat<MT>::KI) + ks, lane, a);
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
        for (int cb = 0; cb < CP / 32; cb += 2)
#pragma unroll
            for (int t = 0; t < M::HT; ++t) {
                Parts<P> a[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) lds_parts(sec, ((cb + i) * M::HT + t) * M::KF + s, lane, a[i]);
#pragma unroll
                for (int np = 0; np < NP; ++np)
                    mma_parts_in_turn<MT, P, 2>({&acc[cb][np].d[t], &acc[cb + 1][np].d[t]}, a, {&hf[np][s], &hf[np][s]});
            }
}
// Order of a region of N products that read one operand each from LDS (P = 1), and PRE reads
// before them: D operands are on their way ahead of the product that uses them.  Left to itself
// the compiler reads one or two ahead, less than the reads' latency beside other waves' reads.
template <int PRE, int N, int D> __device__ __forceinline__ void gated_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, PRE + D, 0);
#pragma unroll
    for (int i = 0; i < N - D; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, D, 0);
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
    static constexpr int OCC = P == 1 || CP <= 128 ? 2 : 1;
};
template <int P, int CP> struct GatedShapeX {
    static constexpr int MT = GatedShape<P, CP>::MT, WAVES = 4, PTS = WAVES * MT;
    static constexpr int OCC = P == 3 && CP > 64 ? 1 : 2;
    static constexpr int LDS_MAX = 160 * 1024 / OCC, A = 1024 + 3 * CP * 64 * P, B = 2 * CP * 64 * P;
    // Where the five sections of a chunk do not fit LDS, they pass one by one through three slots.
    static constexpr bool RING = A + B > LDS_MAX;
    static constexpr int SLOT = 1024 + CP * 64 * P;
    static constexpr int ASLOTS = 2 * A + B <= LDS_MAX ? 2 : 1;
    static constexpr int LDS = RING ? 3 * SLOT : ASLOTS * A + B;
};

// Sums of a workgroup that takes a split of the hidden units: sheet (split * nb + block) of
// part, 16 bytes of every lane after another as they lie in the registers; of the `points`
// points of the wave that there are.
template <int CP, int MT, int NP>
__device__ __forceinline__ void gated_put_sums(const Rows32<MT> (&acc)[CP / 32][NP], float *sheet, int wave, int lane,
                                               int64_t points) {
    constexpr int NV = Mat<MT>::NV;
    float *const to = sheet + wave * (NP * MT * CP) + lane * 4;
#pragma unroll
    for (int np = 0; np < NP; ++np)
        if (np * MT + lane % MT < points)
#pragma unroll
            for (int cb = 0; cb < CP / 32; ++cb)
#pragma unroll
            for (int v = 0; v < NV; v += 4)
                *reinterpret_cast<f32x4 *>(to + ((cb * NP + np) * NV + v) * 64) =
                    f32x4{acc[cb][np].get(v), acc[cb][np].get(v + 1), acc[cb][np].get(v + 2), acc[cb][np].get(v + 3)};
}

// out = b + the splits' sums, in the order of the splits; b may be NULL.  A thread takes four
// channels of a point that one lane held.  Grid: a wave for each of nb * PTS * CP / 256 such pieces.
template <int P, int CP, int MT, int NP>
__global__ __launch_bounds__(256) void k_gated_join(const float *__restrict__ part, int64_t n, int C, int S, int nb,
                                                    const float *__restrict__ b, typename GatedIO<P>::T *__restrict__ out) {
    constexpr int NV = Mat<MT>::NV, V4 = NV / 4, CB = CP / 32, PTS = 4 * NP * MT;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, piece = (int)(w % (V4 * NP * CB));
    const int v = piece % V4 * 4, np = piece / V4 % NP, cb = piece / (V4 * NP), wave = (int)(w / (V4 * NP * CB) % 4);
    const int64_t blk = w / (V4 * NP * CB * 4), p = blk * PTS + (wave * NP + np) * MT + lane % MT;
    const int c = 32 * cb + NV * (lane / MT) + v;
    if (blk >= nb || p >= n || c >= C) return;
    f32x4 sum = b ? *reinterpret_cast<const f32x4 *>(b + c) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float *src = part + blk * PTS * CP + wave * (NP * MT * CP) + ((cb * NP + np) * NV + v) * 64 + lane * 4;
#pragma unroll 8
    for (int s = 0; s < S; ++s) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(src + (int64_t)s * nb * PTS * CP);
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] += x[t];
    }
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
    if constexpr (P == 3) *reinterpret_cast<f32x4 *>(out + p * C + c) = sum;
    else
        *reinterpret_cast<bf16x4 *>(out + p * C + c) = bf16x4{(__bf16)sum[0], (__bf16)sum[1], (__bf16)sum[2], (__bf16)sum[3]};
}

// out = act(x Wg + bg) * (x Wu + bu) Wd + bd.  Workgroup (block b, split s) = (id / S, id % S)
// takes PTS points and chunks per*s .. of the hidden units; with S = 1 it writes out, else its
// sums to sheet (s, b) of part.
// A wave keeps its points' rows as operands and their output sums in registers, and walks the
// chunks: both products into the hidden layer, the activation, the product out of it.  (G, U)
// have one LDS slot, free for the next chunk's once every wave's products into the hidden layer
// are done, D two where they fit.
// HW = 2, for calls that do not fill the chip: twice the waves on the same points, the second
// half on every other chunk, its sums added through LDS at the end.
// out may be x: rows are read by their own workgroup alone, before its first barrier.
template <int P, int CP, int ACT, int HW>
__global__ __launch_bounds__(256 * HW, (GatedShape<P, CP>::OCC)) void k_gated_fwd(
    const typename GatedIO<P>::T *x, int64_t n, int C, const unsigned char *__restrict__ ops, int nchunk, int per, int S,
    const float *__restrict__ bdp, typename GatedIO<P>::T *out, float *__restrict__ part) {
    using Sh = GatedShape<P, CP>;
    constexpr int MT = Sh::MT, NP = Sh::NP, WAVES = Sh::WAVES;
    using M = Mat<MT>;
    using O = GatedOps<P, CP, MT>;
    constexpr int ABYTES = 1024 + 2 * O::SEC, NV = M::NV, AHEAD = CP > 192 ? 4 : 6;
    constexpr int DSLOTS = ABYTES + 2 * O::SEC <= 80 * 1024 ? 2 : 1;  // two workgroups per compute unit
    constexpr int HALF = ABYTES + DSLOTS * O::SEC, SUMS = HW == 2 ? WAVES * NP * MT * CP * 4 : 0;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[HW * HALF > SUMS ? HW * HALF : SUMS];
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wave = wid % WAVES, half = wid / WAVES;
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * NP * MT;
    const uint32_t la = lds_addr(lds) + half * HALF, lb = la + ABYTES;
    const unsigned char *const sa = lds + half * HALF, *const sb = sa + ABYTES;
    auto slot = [&](int i) { return DSLOTS == 2 ? (i & 1) * O::SEC : 0; };  // of the half's i-th chunk
    auto issue_a = [&](int i) {
        gated_stage<ABYTES, WAVES>(ops + (size_t)(j0 + HW * i + half) * O::CHUNK + O::BIAS, la, wave, lane);
    };
    auto issue_d = [&](int i) {
        gated_stage<O::SEC, WAVES>(ops + (size_t)(j0 + HW * i + half) * O::CHUNK, lb + slot(i), wave, lane);
    };
    const int steps = (j1 - j0 + HW - 1) / HW, mine = (j1 - j0 - half + HW - 1) / HW;  // the half's own chunks

    if (mine > 0) {
        issue_a(0);
        if (DSLOTS == 2) issue_d(0);
    }
    Parts<P> xf[NP][O::KS];
    gated_rows<P, CP, MT, NP>(x, p0, n, C, lane, xf);
    Rows32<MT> acc[O::CB][NP];
#pragma unroll
    for (int cb = 0; cb < O::CB; ++cb)
#pragma unroll
        for (int np = 0; np < NP; ++np) acc[cb][np].zero();
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        gated_sync();  // (G, U), and with two slots D, of chunk i are in LDS; D of chunk i - 1 is read by all
        if (HW == 2 && i >= mine) {
            barrier();
            continue;
        }
        if (DSLOTS == 1) issue_d(i);
        else if (i + 1 < mine) issue_d(i + 1);
        Rows32<MT> a[NP], u[NP];
        gated_bias<MT, NP>(sa, 0, lane, a);
        gated_bias<MT, NP>(sa, 1, lane, u);
#pragma unroll
        for (int ks = 0; ks < O::KS; ++ks)
#pragma unroll
            for (int t = 0; t < M::HT; ++t) {
                Parts<P> w[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) lds_parts(sa + 1024 + k * O::SEC, t * O::KS + ks, lane, w[k]);
#pragma unroll
                for (int np = 0; np < NP; ++np)
                    mma_parts_in_turn<MT, P, 2>({&a[np].d[t], &u[np].d[t]}, w, {&xf[np][ks], &xf[np][ks]});
            }
        if constexpr (P == 1) gated_ahead<8, 2 * O::KS, AHEAD>();
        if (DSLOTS == 1) wait_vmcnt<0>();
        barrier();  // (G, U) of chunk i are read by all; with one slot, D is in LDS
        // The wave that has its vector work before it goes first, or the two of a SIMD share each phase
        // in step and neither's products run beside the other's activation (1M bfloat16 points at
        // C = 256, F = 1024: SiLU 1.40 -> 1.34 ms, GELU 1.525 -> 1.515; the other way round 1.43).
        __builtin_amdgcn_s_setprio(1);
        if (i + 1 < mine) issue_a(i + 1);
        Parts<P> hf[NP][M::KF];
#pragma unroll
        for (int np = 0; np < NP; ++np)
#pragma unroll
            for (int s = 0; s < M::KF; ++s) {
                float h[8], slope;
#pragma unroll
                for (int t = 0; t < 8; ++t) h[t] = gated_act<P, ACT, false>(a[np].get(8 * s + t), slope) * u[np].get(8 * s + t);
                to_parts(h, hf[np][s]);
            }
        gated_channels<P, CP, MT, NP>(sb + slot(i), hf, lane, acc);
        if constexpr (P == 1) gated_ahead<0, O::CB * M::KF, AHEAD>();
        __builtin_amdgcn_s_setprio(0);
    }
    if constexpr (HW == 2) {
        barrier();  // the last operands are read by all
        if (half == 1) gated_put_sums<CP, MT, NP>(acc, reinterpret_cast<float *>(lds), wave, lane, NP * MT);
        barrier();
        if (half == 1) return;
        const float *const sums = reinterpret_cast<float *>(lds) + wave * (NP * MT * CP) + lane * 4;
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb)
#pragma unroll
            for (int np = 0; np < NP; ++np)
#pragma unroll
                for (int v = 0; v < NV; v += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(sums + ((cb * NP + np) * NV + v) * 64);
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[cb][np].set(v + t, acc[cb][np].get(v + t) + w[t]);
                }
    }
    if (S > 1) {
        gated_put_sums<CP, MT, NP>(acc, part + (split * (int64_t)(gridDim.x / S) + blk) * Sh::PTS * CP, wave, lane, n - p0);
        return;
    }
#pragma unroll
    for (int np = 0; np < NP; ++np) {
        const int64_t p = p0 + np * MT + lane % MT;
        if (p >= n) continue;
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb) {
            const int c = 32 * cb + NV * (lane / MT);
            if (c >= C) continue;
            float v[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = acc[cb][np].get(i) + bdp[c + i];
            store_row<NV>(out + p * C + c, v);
        }
    }
}

// Sums over the 32 points (lanes 0..31 and 32..63) of 16 values of da and du each, as they are
// before bfloat16 rounds them: summed as the store holds them, every point's rounding stays in
// dbg and dbu (1.6 times the error of the output's own rounding, measured at 50 to 500 points).
// Each step adds two lanes and merges two values into the halves that this frees, so the 32
// values take 77 instructions instead of 160: add() leaves value i of da in the lower and of du
// in the upper row of 16, store() merges the 16 that are left.  Lane l ends with value l & 15 of
// its half, of du if l & 16.
struct GatedColumns {
    float r[16];
    __device__ __forceinline__ void add(int v, float da, float du) {
        auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(da), __float_as_uint(du), false, false);
        r[v] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    template <int CTRL, int N> __device__ __forceinline__ void merge(int lane) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float a = r[i] + dpp<CTRL>(r[i]), b = r[i + N] + dpp<CTRL>(r[i + N]);
            r[i] = lane & N ? b : a;
        }
    }
    // To row w of chunk j: cols[m][chunk][rows][32], m = 0 da, 1 du.
    __device__ __forceinline__ void store(float *cols, int nchunk, int j, int64_t rows, int64_t w, int lane) {
        merge<0x128, 8>(lane);  // row_ror:8
        merge<0x141, 4>(lane);  // row_half_mirror
        merge<0x4E, 2>(lane);   // quad_perm [2,3,0,1]
        merge<0xB1, 1>(lane);   // quad_perm [1,0,3,2]
        const int m = (lane >> 4) & 1;
        cols[(((int64_t)m * nchunk + j) * rows + w) * 32 + 16 * (lane >> 5) + (lane & 15)] = r[0];
    }
};

// The store holds da, du and h (m = 0, 1, 2) by chunks and blocks of 32 points, each as the lanes
// of a 32 x 32 result hold it, 16 bytes of every lane after another: store[m][chunk][tp / 32][1024],
// so that a wave writes and reads whole lines.  By rows of 32 hidden units, 16 bytes of a lane to a
// row, the slopes of 350,000 float32 points at C = 128, F = 512 took 1.03 ms instead of 0.90, a
// training step of 100,000 at C = 64 336 us instead of 291.
// Place in its block of hidden unit h (a multiple of the 16 bytes' values) of point p.
template <int P> __host__ __device__ constexpr int gated_at(int p, int h) {
    constexpr int V = P == 1 ? 8 : 4;
    return (h % 16 / V * 64 + h / 16 * 32 + p) * V;
}
// Eight values of a lane at their place.
__device__ __forceinline__ void gated_put(bf16_t *at, const float (&v)[8]) { store_row<8>(at, v); }
__device__ __forceinline__ void gated_put(float *at, const float (&v)[8]) {
    *reinterpret_cast<f32x4 *>(at) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4 *>(at + 256) = f32x4{v[4], v[5], v[6], v[7]};
}

// The hidden layer of a chunk before the activation, and the gradient of its output.
template <int MT> struct GatedHidden {
    Rows32<MT> a[1], u[1], dh[1];
};

// dx of n points (the first nb * PTS of the store's), and da, du, h in the store; values of points
// past n are zero.  In bfloat16 also the sums of da and du over 32 points each, in cols
// (GatedColumns).  Grid and splits as k_gated_fwd.
// (G, U, H) have two LDS slots where they fit, else one, (XG, XU) have one; copies are issued a
// phase ahead.
template <int P, int CP, int ACT>
__global__ __launch_bounds__(256, (GatedShapeX<P, CP>::OCC)) void k_gated_dx(
    const typename GatedIO<P>::T *__restrict__ x, const typename GatedIO<P>::T *__restrict__ g, int64_t n, int C,
    const unsigned char *__restrict__ ops, int nchunk, int per, int S, int64_t tp,
    typename GatedIO<P>::T *__restrict__ store, float *__restrict__ cols, typename GatedIO<P>::T *__restrict__ dx,
    float *__restrict__ part) {
    using T = typename GatedIO<P>::T;
    using Sh = GatedShapeX<P, CP>;
    constexpr int MT = Sh::MT, WAVES = Sh::WAVES;
    using M = Mat<MT>;
    using O = GatedOps<P, CP, MT>;
    constexpr int NV = M::NV, KS = O::KS;
    // Stores of a chunk: they are issued after its copies and may stay in flight while those are waited for.
    constexpr int STORES = 3 * NV * (int)sizeof(T) / 16 + (P == 1);
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Sh::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * MT, p = p0 + lane % MT;
    const bool in = p < n;
    const uint32_t la = lds_addr(lds);

    // A float32 product on the matrix cores comes out low by some 2^-28 of its terms, whatever its
    // sign: nothing to a value, but dbu, a sum over millions of them, was off by 4e-6 of itself. So
    // odd points' g is negated on the way in and dh back, and the sums over points lose it.
    const uint32_t flip = P == 3 && (lane & 1) ? 0x80008000u : 0u;
    const float sign = P == 3 && (lane & 1) ? -1.f : 1.f;
    Parts<P> xf[1][KS], gf[1][KS];
    Rows32<MT> acc[O::CB][1];
    Parts<P> daf[1][M::KF], duf[1][M::KF];
    auto start = [&]() {
        gated_rows<P, CP, MT, 1>(x, p0, n, C, lane, xf);
        gated_rows<P, CP, MT, 1>(g, p0, n, C, lane, gf);
        if constexpr (P == 3)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int s = 0; s < P; ++s)
                    gf[0][ks].p[s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, gf[0][ks].p[s]) ^ flip);
#pragma unroll
        for (int cb = 0; cb < O::CB; ++cb) acc[cb][0].zero();
    };
    auto biases = [&](GatedHidden<MT> &c, const unsigned char *bias) {
        gated_bias<MT, 1>(bias, 0, lane, c.a);
        gated_bias<MT, 1>(bias, 1, lane, c.u);
        c.dh[0].zero();
    };
    // K step ks of the three products into the hidden layer, from their sections at sec.
    auto hidden = [&](GatedHidden<MT> &c, const unsigned char *sec, int ks) {
#pragma unroll
        for (int t = 0; t < M::HT; ++t) {
            Parts<P> w[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) lds_parts(sec + i * O::SEC, t * KS + ks, lane, w[i]);
            mma_parts_in_turn<MT, P, 3>({&c.a[0].d[t], &c.u[0].d[t], &c.dh[0].d[t]}, w, {&xf[0][ks], &xf[0][ks], &gf[0][ks]});
        }
    };
    // da, du and h of values v0 .. v1 - 1 of chunk j; each eight, as they are complete, become
    // the next products' operands and go to the store.
    float da[8], du[8], h[8];
    GatedColumns sums;
    auto slopes = [&](GatedHidden<MT> &c, int j, int v0, int v1) {
#pragma unroll
        for (int v = v0; v < v1; ++v) {
            float slope;
            const float uv = c.u[0].get(v), d = P == 3 ? sign * c.dh[0].get(v) : c.dh[0].get(v);
            const float y = gated_act<P, ACT, true>(c.a[0].get(v), slope);
            h[v & 7] = in ? y * uv : 0.f;
            du[v & 7] = d * y;
            da[v & 7] = d * uv * slope;
            if constexpr (P == 1) sums.add(v, da[v & 7], du[v & 7]);
            if ((v & 7) == 7) {
                to_parts(da, daf[0][v >> 3]);
                to_parts(du, duf[0][v >> 3]);
                T *const at = store + ((int64_t)j * tp + p / 32 * 32) * 32 + gated_at<P>(p % 32, NV * (lane / MT) + (v & ~7));
                const int64_t plane = (int64_t)nchunk * tp * 32;
                gated_put(at, da);
                gated_put(at + plane, du);
                gated_put(at + 2 * plane, h);
            }
        }
        if constexpr (P == 1)
            if (v1 == NV) sums.store(cols, nchunk, j, tp / 32, p0 / 32, lane);
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if constexpr (!Sh::RING) {
        constexpr int AP = Sh::A / 1024 / WAVES;  // copies of (G, U, H) that every wave issues at least
        const uint32_t lb = la + Sh::ASLOTS * Sh::A;
        const unsigned char *const sb = lds + Sh::ASLOTS * Sh::A;
        auto slot = [&](int j) { return Sh::ASLOTS == 2 ? ((j - j0) & 1) * Sh::A : 0; };
        auto issue = [&](int j) { gated_stage<Sh::A, WAVES>(ops + (size_t)j * O::CHUNK + O::BIAS, la + slot(j), wave, lane); };
        GatedHidden<MT> c;
        issue(j0);
        start();
#pragma unroll 1
        for (int j = j0; j < j1; ++j) {
            wait_vmcnt<0>();
            barrier();  // (G, U, H)(j) is in LDS; chunk j - 1 is read by all
            gated_stage<Sh::B, WAVES>(ops + (size_t)j * O::CHUNK + O::XG, lb, wave, lane);
            const bool more = j + 1 < j1;
            if (Sh::ASLOTS == 2 && more) issue(j + 1);
            const unsigned char *const sec = lds + slot(j) + 1024;
            biases(c, sec - 1024);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) hidden(c, sec, ks);
            slopes(c, j, 0, NV);
            asm volatile("" ::: "memory");
            if (Sh::ASLOTS == 2 && more) wait_vmcnt<AP + STORES>();
            else wait_vmcnt<STORES>();
            barrier();  // (XG, XU)(j) is in LDS, (G, U, H)(j) read by all
            if (Sh::ASLOTS == 1 && more) issue(j + 1);
            gated_channels<P, CP, MT, 1>(sb, daf, lane, acc);
            gated_channels<P, CP, MT, 1>(sb + O::SEC, duf, lane, acc);
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
        GatedHidden<MT> c;
#pragma unroll 1
        for (int j = j0; j < j1; ++j) {
            const int i = 5 * (j - j0);
            auto slot = [&](int q) { return lds + ((i + q) % 3) * Sh::SLOT + 1024; };
            if (i + 2 < steps) issue(i + 2);
            biases(c, slot(0) - 1024);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) gated_hidden<P, CP, MT, 1>(slot(0), xf, ks, lane, c.a);
            next(i);
            if (i + 3 < steps) issue(i + 3);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) gated_hidden<P, CP, MT, 1>(slot(1), xf, ks, lane, c.u);
            next(i + 1);
            if (i + 4 < steps) issue(i + 4);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) gated_hidden<P, CP, MT, 1>(slot(2), gf, ks, lane, c.dh);
            slopes(c, j, 0, NV);
            asm volatile("" ::: "memory");
            next(i + 2);
            if (i + 5 < steps) issue(i + 5);
            gated_channels<P, CP, MT, 1>(slot(3), daf, lane, acc);
            next(i + 3);
            if (i + 6 < steps) issue(i + 6);
            gated_channels<P, CP, MT, 1>(slot(4), duf, lane, acc);
            next(i + 4);
        }
    }
    if (S > 1) {
        gated_put_sums<CP, MT, 1>(acc, part + (split * (int64_t)(gridDim.x / S) + blk) * Sh::PTS * CP, wave, lane, n - p0);
        return;
    }
    if (!in) return;
#pragma unroll
    for (int cb = 0; cb < O::CB; ++cb) {
        const int c = 32 * cb + NV * (lane / MT);
        if (c >= C) continue;
        float v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = acc[cb][0].get(i);
        store_row<NV>(dx + p * C + c, v);
    }
}

// Where the rows (x and g) and the sums of dx fill a wave's registers together, one wave per SIMD
// would have to do all (bfloat16 at CP = 256: 8,900 cycles per chunk, of 2,560 of products;
// float32 at CP = 128: 350,000 points of F = 512 in 1.53 ms, of 0.68 of products).  There the
// backward takes two kernels: the slopes without the sums, and dx, which reads da and du back
// from the store, on two waves per SIMD (float32: 0.85 + 0.47 ms).  Where one kernel has two waves
// per SIMD it is faster: a bfloat16 step of 300,000 points at C = 128, F = 512 takes 0.76 ms, in two
// kernels 0.80, at C = 64, F = 256 0.33 and 0.38.  Float32 rows of more than 128 channels fill 288
// registers and more beside the 96 of two chunks' results, which k_gated_slopes3 has no room for:
// they stay with the one kernel and its ring of sections (not tried otherwise; a step of 100,003
// points at C = 256, F = 683 takes 2.58 ms, at C = 192, F = 512 1.48 ms).
template <int P, int CP> struct GatedWide {
    static constexpr bool USE = P == 1 ? CP > 128 : CP == 128;
    static constexpr int WAVES = 4, PTS = WAVES * 32;
    static constexpr int SEC = CP * 64 * P, A = 1024 + 3 * SEC;
};

// da, du, h (and cols) of chunks per*s .. of PTS points, as k_gated_dx leaves them, bfloat16.
// One LDS slot: the next chunk is copied while the slopes of this one are computed, beside the
// SIMD's other wave.
template <int CP, int ACT>
__global__ __launch_bounds__(256, 2) void k_gated_slopes(const bf16_t *__restrict__ x, const bf16_t *__restrict__ g,
                                                         int64_t n, int C, const unsigned char *__restrict__ ops,
                                                         int nchunk, int per, int S, int64_t tp,
                                                         bf16_t *__restrict__ store, float *__restrict__ cols) {
    using Sh = GatedWide<1, CP>;
    using O = GatedOps<1, CP, 32>;
    constexpr int WAVES = Sh::WAVES, KS = O::KS;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Sh::A];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * 32, p = p0 + lane % 32;
    const bool in = p < n;
    const uint32_t la = lds_addr(lds);
    auto issue = [&](int j) { gated_stage<Sh::A, WAVES>(ops + (size_t)j * O::CHUNK + O::BIAS, la, wave, lane); };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    issue(j0);
    Parts<1> xf[1][KS], gf[1][KS];
    gated_rows<1, CP, 32, 1>(x, p0, n, C, lane, xf);
    gated_rows<1, CP, 32, 1>(g, p0, n, C, lane, gf);
    const int64_t plane = (int64_t)nchunk * tp * 32;
    Rows32<32> a[1], u[1], dh[1];
    auto slopes = [&](int j) {
        asm volatile("" ::: "memory");
        bf16_t *const at = store + ((int64_t)j * tp + p0) * 32 + lane * 8;
        GatedColumns sums;
#pragma unroll
        for (int v0 = 0; v0 < 16; v0 += 8) {
            float da[8], du[8], h[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                float slope;
                const float uv = u[0].get(v0 + v), d = dh[0].get(v0 + v);
                const float y = gated_act<1, ACT, true>(a[0].get(v0 + v), slope);
                h[v] = in ? y * uv : 0.f;
                du[v] = d * y;
                da[v] = d * uv * slope;
                sums.add(v0 + v, da[v], du[v]);
            }
            gated_put(at + v0 * 64, da);
            gated_put(at + plane + v0 * 64, du);
            gated_put(at + 2 * plane + v0 * 64, h);
        }
        sums.store(cols, nchunk, j, tp / 32, p0 / 32, lane);
        asm volatile("" ::: "memory");
    };
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
        // The copies of chunk j are older than the seven stores of chunk j - 1.
        if (j > j0) wait_vmcnt<7>();
        else wait_vmcnt<0>();
        barrier();  // chunk j is in LDS
        const unsigned char *const sec = lds + 1024;
        gated_bias<32, 1>(lds, 0, lane, a);
        gated_bias<32, 1>(lds, 1, lane, u);
        dh[0].zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            gated_hidden<1, CP, 32, 1>(sec, xf, ks, lane, a);
            gated_hidden<1, CP, 32, 1>(sec + O::SEC, xf, ks, lane, u);
            gated_hidden<1, CP, 32, 1>(sec + 2 * O::SEC, gf, ks, lane, dh);
        }
        gated_ahead<8, 3 * KS, 8>();
        barrier();  // chunk j is read by all
        if (j + 1 < j1) issue(j + 1);
        slopes(j);
    }
}

// The same in float32, on one wave per SIMD, which issues its vector work beside its own products
// or not at all: the products into the hidden layer of chunk j + 1 are interleaved with the slopes
// of chunk j, some values after each K step.  Two LDS slots, copies a chunk ahead.
template <int CP, int ACT>
__global__ __launch_bounds__(256, 1) void k_gated_slopes3(const float *__restrict__ x, const float *__restrict__ g,
                                                          int64_t n, int C, const unsigned char *__restrict__ ops,
                                                          int nchunk, int per, int S, int64_t tp,
                                                          float *__restrict__ store) {
    using Sh = GatedWide<3, CP>;
    using O = GatedOps<3, CP, 32>;
    constexpr int WAVES = Sh::WAVES, KS = O::KS, NV = 16, STORES = 3 * NV * 4 / 16;
    static_assert(NV == 2 * KS, "two values beside each K step");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * Sh::A];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int64_t p0 = blk * Sh::PTS + wave * 32, p = p0 + lane % 32;
    const bool in = p < n;
    const uint32_t la = lds_addr(lds);
    auto slot = [&](int j) { return ((j - j0) & 1) * Sh::A; };
    auto issue = [&](int j) { gated_stage<Sh::A, WAVES>(ops + (size_t)j * O::CHUNK + O::BIAS, la + slot(j), wave, lane); };
    issue(j0);
    Parts<3> xf[1][KS], gf[1][KS];
    gated_rows<3, CP, 32, 1>(x, p0, n, C, lane, xf);
    gated_rows<3, CP, 32, 1>(g, p0, n, C, lane, gf);
    // As in k_gated_dx: odd points' g is negated on the way in and dh back.
    const uint32_t flip = lane & 1 ? 0x80008000u : 0u;
    const float sign = lane & 1 ? -1.f : 1.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int s = 0; s < 3; ++s)
            gf[0][ks].p[s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, gf[0][ks].p[s]) ^ flip);
    auto biases = [&](GatedHidden<32> &c, const unsigned char *bias) {
        gated_bias<32, 1>(bias, 0, lane, c.a);
        gated_bias<32, 1>(bias, 1, lane, c.u);
        c.dh[0].zero();
    };
    typedef Parts<3> Fragments[3];
    auto load = [&](Fragments &w, const unsigned char *sec, int ks) {
#pragma unroll
        for (int i = 0; i < 3; ++i) lds_parts(sec + i * O::SEC, ks, lane, w[i]);
    };
    auto hidden = [&](GatedHidden<32> &c, const Fragments &w, int ks, auto beside) {
        mma_parts_in_turn<32, 3, 3>({&c.a[0].d[0], &c.u[0].d[0], &c.dh[0].d[0]}, w, {&xf[0][ks], &xf[0][ks], &gf[0][ks]},
                                    beside);
    };
    const int64_t plane = (int64_t)nchunk * tp * 32;
    float da[4], du[4], h[4];
    auto slopes = [&](GatedHidden<32> &c, int j, int v0, int v1) {
#pragma unroll
        for (int v = v0; v < v1; ++v) {
            float slope;
            const float uv = c.u[0].get(v), d = sign * c.dh[0].get(v);
            const float y = gated_act<3, ACT, true>(c.a[0].get(v), slope);
            h[v & 3] = in ? y * uv : 0.f;
            du[v & 3] = d * y;
            da[v & 3] = d * uv * slope;
            if ((v & 3) == 3) {
                float *const at = store + ((int64_t)j * tp + p0) * 32 + (v & ~3) * 64 + lane * 4;
                store_row<4>(at, da);
                store_row<4>(at + plane, du);
                store_row<4>(at + 2 * plane, h);
            }
        }
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Slopes of chunk j in c; `next` gets the hidden layer of chunk j + 1.
    auto step = [&](GatedHidden<32> &c, GatedHidden<32> &next, int j) {
        if (j > j0) wait_vmcnt<STORES>();  // the copies of chunk j + 1 are older than the stores of chunk j - 1
        else wait_vmcnt<0>();
        barrier();  // chunk j + 1 is in LDS, chunk j read by all
        if (j + 2 < j1) issue(j + 2);
        const unsigned char *const sec = lds + slot(j + 1) + 1024;
        Fragments w[2];
        load(w[0], sec, 0);
        biases(next, sec - 1024);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            __builtin_amdgcn_sched_barrier(0);  // K step by K step: left to itself the compiler gathers the slopes
            if (ks + 1 < KS) load(w[(ks + 1) & 1], sec, ks + 1);
            hidden(next, w[ks & 1], ks, [&](int q) {
                const int at = ks * NV / KS + q / 3;
                if (q % 3 == 1) slopes(c, j, at, at + 1);
            });
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    GatedHidden<32> c0, c1;
    gated_sync();
    if (j0 + 1 < j1) issue(j0 + 1);
    biases(c0, lds);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        Fragments w;
        load(w, lds + 1024, ks);
        hidden(c0, w, ks, [](int) {});
    }
    int j = j0;
#pragma unroll 1
    for (; j + 2 < j1; j += 2) {
        step(c0, c1, j);
        step(c1, c0, j + 1);
    }
    if (j + 1 < j1) {
        step(c0, c1, j);
        slopes(c1, j + 1, 0, NV);
    } else {
        slopes(c0, j, 0, NV);
    }
}

// Eight values of a point in the store as an operand, as they were loaded.
template <int P> struct GatedRaw {
    u32x4 v[P == 1 ? 1 : 2];
    __device__ __forceinline__ void load(const typename GatedIO<P>::T *p) {
        v[0] = *reinterpret_cast<const u32x4 *>(p);
        if constexpr (P == 3) v[1] = *reinterpret_cast<const u32x4 *>(p + 256);
    }
    // Makes the compiler wait for the load here: it does not know of the copies that are issued
    // after this and would wait for some of them at the first use.
    __device__ __forceinline__ void arrived() {
        asm volatile("" : "+v"(v[0]));
        if constexpr (P == 3) asm volatile("" : "+v"(v[1]));
    }
    __device__ __forceinline__ void parts(Parts<P> &f) const {
        if constexpr (P == 1) f.p[0] = __builtin_bit_cast(bf16x8, v[0]);
        else {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = __uint_as_float(v[i / 4][i & 3]);
            split8(t, f);
        }
    }
};

// dx = da Wg^T + du Wu^T from the store, over chunks per*s ..; sums to dx or part as k_gated_fwd.
// A step takes SPS of the sections XG and XU of a chunk: in bfloat16 both, in two LDS slots, the
// copies issued one step ahead; in float32 one, in three slots, two steps ahead.  A chunk's da and
// du of a point lie in the store as the lane's operands; they are on their way two steps ahead.
template <int P, int CP>
__global__ __launch_bounds__(256, 2) void k_gated_dx_wide(int64_t n, int C, const unsigned char *__restrict__ ops,
                                                          int nchunk, int per, int S, int64_t tp,
                                                          const typename GatedIO<P>::T *__restrict__ store,
                                                          typename GatedIO<P>::T *__restrict__ dx,
                                                          float *__restrict__ part) {
    using T = typename GatedIO<P>::T;
    using Sh = GatedWide<P, CP>;
    using O = GatedOps<P, CP, 32>;
    constexpr int WAVES = Sh::WAVES, SPS = P == 1 ? 2 : 1, SLOTS = P == 1 ? 2 : 3, BYTES = SPS * Sh::SEC;
    constexpr int PER = BYTES / 1024 / WAVES, LOADS = SPS * 2 * (P == 1 ? 1 : 2);
    static_assert(BYTES % (1024 * WAVES) == 0, "every wave issues as many copies");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[SLOTS * BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t blk = blockIdx.x / S;
    const int split = blockIdx.x % S;
    const int j0 = split * per, j1 = j0 + per < nchunk ? j0 + per : nchunk;
    const int steps = (j1 - j0) * 2 / SPS;
    const int64_t p0 = blk * Sh::PTS + wave * 32, p = p0 + lane % 32;
    const uint32_t la = lds_addr(lds);
    auto issue = [&](int i) {
        const unsigned char *const src = ops + (size_t)(j0 + i * SPS / 2) * O::CHUNK + O::XG + (i * SPS & 1) * Sh::SEC;
        gated_stage<BYTES, WAVES>(src, la + i % SLOTS * BYTES, wave, lane);
    };
    const int64_t plane = (int64_t)nchunk * tp * 32;
    typedef GatedRaw<P> Raws[SPS][2];
    auto fetch = [&](int i, Raws &f) {
        const T *const at = store + ((int64_t)(j0 + i * SPS / 2) * tp + p0) * 32 + lane * (P == 1 ? 8 : 4);
#pragma unroll
        for (int m = 0; m < SPS; ++m)
#pragma unroll
            for (int s = 0; s < 2; ++s) f[m][s].load(at + ((i * SPS & 1) + m) * plane + 512 * s);
    };
    Rows32<32> acc[O::CB][1];
#pragma unroll
    for (int cb = 0; cb < O::CB; ++cb) acc[cb][0].zero();
    Raws f[3];
    issue(0);
    fetch(0, f[0]);
    if (steps > 1) {
        if (SLOTS == 3) issue(1);
        asm volatile("" ::: "memory");
        fetch(1, f[1]);
    }
    auto step = [&](Raws &now, Raws &then, int i) {
        asm volatile("" ::: "memory");
        // what was issued for step i + 1 may be in flight
        if (i + 1 < steps) wait_vmcnt<LOADS + (SLOTS == 3 ? PER : 0)>();
        else wait_vmcnt<0>();
#pragma unroll
        for (int m = 0; m < SPS; ++m)
#pragma unroll
            for (int s = 0; s < 2; ++s) now[m][s].arrived();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // step i's sections are in LDS, step i - 1's read by all
        asm volatile("" ::: "memory");
        if (i + SLOTS - 1 < steps) issue(i + SLOTS - 1);
        if (i + 2 < steps) fetch(i + 2, then);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int m = 0; m < SPS; ++m) {
            Parts<P> hf[1][2];
#pragma unroll
            for (int s = 0; s < 2; ++s) now[m][s].parts(hf[0][s]);
            gated_channels<P, CP, 32, 1>(lds + i % SLOTS * BYTES + m * Sh::SEC, hf, lane, acc);
        }
        if constexpr (P == 1) gated_ahead<0, 4 * O::CB, 6>();
    };
    int i = 0;
#pragma unroll 1
    for (; i + 2 < steps; i += 3) {
        step(f[0], f[2], i);
        step(f[1], f[0], i + 1);
        step(f[2], f[1], i + 2);
    }
    if (i < steps) step(f[0], f[2], i);
    if (i + 1 < steps) step(f[1], f[0], i + 1);
    if (S > 1) {
        gated_put_sums<CP, 32, 1>(acc, part + (split * (int64_t)(gridDim.x / S) + blk) * Sh::PTS * CP, wave, lane, n - p0);
        return;
    }
    if (p >= n) return;
#pragma unroll
    for (int cb = 0; cb < O::CB; ++cb) {
        const int c = 32 * cb + 16 * (lane / 32);
        if (c >= C) continue;
        float v[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) v[t] = acc[cb][0].get(t);
        store_row<16>(dx + p * C + c, v);
    }
}

// Shape of the weight gradients' kernel: a wave's result is 64 hidden units by CTW tiles of
// 32 channels, W waves cover HB hidden units by CP channels.
// Four waves leave room for two workgroups per compute unit; eight, one workgroup of as many waves,
// read two thirds of the bytes per product and have LDS for copies three steps ahead instead of
// two (USE8: bfloat16, where the copies go to LDS directly, at the widths whose pieces divide by
// eight): 250,000 points at C = 256, F = 1024 took 517 us instead of 548.
template <int P, int CP, int W> struct GatedDw {
    static constexpr int WC = CP > 128 ? 2 : 1, WH = W / WC, HB = 64 * WH, CTW = CP / 32 / WC;
    static constexpr int HPL = HB / 32, PL = HPL + CP / 32;  // planes of 32 columns
    static constexpr int KP = P == 1 ? 32 : 16;              // points per step
    static constexpr int SLOTS = P == 3 ? 2 : W == 8 ? 4 : 3;
    static constexpr int PLB = KP * 64;                      // bytes of a plane (of one part)
    static constexpr int SLOT = PL * PLB * P;
    static constexpr int PIECES = PL * 2;                    // 1 KiB copies (P = 1), 16-row-by-64-byte loads
    static constexpr int PER = PIECES / W;
    static_assert(CP % 64 == 0, "two channel waves share CP evenly");
    static_assert(PIECES % W == 0, "every wave issues as many copies or loads");
};
template <int P, int CP> struct GatedDwWide {
    static constexpr bool USE8 = P == 1 && CP % 128 == 0;
};

// One operand whose K slots are points: columns 32 of plane at `plane`, K slots 8q .. of the 16
// points from row r0.  Lanes 0..31 and 32..63 read 256 consecutive bytes each: four rows of 64
// bytes, or (PIECES) the four 16-byte pieces of the rows one after another, four rows each, in the
// order columns 0, 16, 8, 24, as they come from the store.
template <bool PIECES> __device__ __forceinline__ bf16x8 plane_tr(const unsigned char *plane, int r0, int lane) {
    const int j = lane & 15, h = (lane >> 4) & 1;
    const unsigned char *lo = plane + (r0 + 8 * (lane >> 5)) * 64 +
                              (PIECES ? (j & 2) * 64 + h * 64 + (j >> 2) * 16 + 8 * (j & 1) : (j >> 2) * 64 + 32 * h + 8 * (j & 3));
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lo);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lo + 256));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
}
// s plus the eight slots of v.
__device__ __forceinline__ float sum_slots(const bf16x8 &v, float s) {
    const bf16x2 one{(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int i = 0; i < 8; i += 2) s = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{v[i], v[i + 1]}, one, s, false);
    return s;
}
// The weight gradients of the tile's points: for m = 0 (dWg), 1 (dWu): sum of da or du times
// x; for 2 (dWd): of h times g.  Workgroup (m, hidden block hb, split sp) with sp outermost
// sums points per*sp .. + per - 1 (per a multiple of 32) into part[sp][m][nchunk * 32][CP] and
// bpart[sp][m][max(nchunk * 32, CP)] (sums of da, du; for m = 2 of g), added to what is there
// unless `first` (at the end: short chains of sums round less).  Rows past n are read from
// `zeros` (16 bytes).
// SUMS: column sums that the workgroup takes as it reads its operands, of the hidden columns
// (1), of the channels (2) or none (0).  Every wave takes them, wanted or not: beside the
// products they are free, branches around them are not.  In bfloat16 those of the hidden
// columns come from cols instead, after the products.
template <int P, int CP> struct GatedDwArgs {
    const typename GatedIO<P>::T *x, *g, *store;
    const float *cols;
    int64_t n, tp, per;
    int C, nchunk, nhb, first;
    const unsigned char *zeros;
    float *part, *bpart;
};
template <int P, int CP, int W, int SUMS>
__device__ __forceinline__ void gated_dw(const GatedDwArgs<P, CP> &A, unsigned char *lds, int m, int hb, int sp) {
    using T = typename GatedIO<P>::T;
    using S = GatedDw<P, CP, W>;
    constexpr int KP = S::KP, HPL = S::HPL, PL = S::PL, CTW = S::CTW;
    const int64_t n = A.n, tp = A.tp, per = A.per;
    const int C = A.C, nchunk = A.nchunk, first = A.first;
    const T *const store = A.store;
    const unsigned char *const zeros = A.zeros;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int hi = wave / S::WC, ci = wave % S::WC;
    const int64_t a0 = (int64_t)sp * per, a1 = a0 + per < tp ? a0 + per : tp;
    const int nk = a0 < a1 ? (int)((a1 - a0) / KP) : 0;
    const T *const cols = m == 2 ? A.g : A.x;
    const T *const hid = store + (int64_t)m * nchunk * tp * 32;
    const int FP = nchunk * 32, BW = FP > CP ? FP : CP;

    // Piece k of a step: 16 points by one plane of 32 columns (P = 1: half k / PL of the points) or
    // 16 points by 16 columns (P = 3: half k / PL of the plane).  Lane l takes 16 bytes of row l / 4
    // of x and g; of the store, where four lanes in a row are four points, of row hrow.
    // The wave's pieces are a uniform base, which moves on with the steps (in the store by a block
    // of 32 points, for P = 3 in two unequal steps), and a lane's offset.
    const int hrow = (lane >> 4) * 4 + (lane & 3), hq = (lane >> 2) & 3;
    const unsigned char *base[S::PER];
    uint32_t voff[S::PER];
    int64_t inc[S::PER], inc2[S::PER];
    constexpr int E = (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < S::PER; ++i) {
        const int k = wave * S::PER + i, pl = k % PL, half = k / PL;
        const int row = P == 1 ? 16 * half + (lane >> 2) : lane >> 2;
        const int col = P == 1 ? 8 * (lane & 3) : 16 * half + 4 * (lane & 3);
        if (pl < HPL) {
            int ch = hb * HPL + pl;
            ch = ch < nchunk ? ch : nchunk - 1;  // its products are not stored
            base[i] = (const unsigned char *)(hid + ((int64_t)ch * tp + a0) * 32);
            voff[i] = (P == 1 ? gated_at<P>(16 * half + hrow, 16 * (hq & 1) + 8 * (hq >> 1)) : gated_at<P>(hrow, 16 * half + 4 * hq)) * E;
            inc[i] = P == 1 ? 1024 * E : gated_at<P>(16, 0) * E;
            inc2[i] = 1024 * E - inc[i];
        } else {  // channels past C repeat others; their products are not stored
            const int c = 32 * (pl - HPL) < C ? 32 * (pl - HPL) : 0;
            base[i] = (const unsigned char *)(cols + a0 * C + c);
            voff[i] = (row * C + (c + col < C ? col : col & 15)) * E;
            inc[i] = inc2[i] = (int64_t)KP * C * E;
        }
    }
    // Address of piece i at step k for a step that passes row n, by lane.
    auto ragged = [&](int i, int k) {
        const int pl = (wave * S::PER + i) % PL, half = (wave * S::PER + i) / PL;
        const int64_t p = a0 + (int64_t)k * KP + (P == 1 ? 16 * half : 0) + (lane >> 2);
        return pl >= HPL && p >= n ? zeros : base[i] + voff[i];
    };
    f32x16 acc[2][CTW];
    double bsum[2] = {0.0, 0.0}, gsum[CTW];
    const bool bh = P == 3 && SUMS == 1 && ci == 0, bc = SUMS == 2 && hi == 0;
    float *const bp = A.bpart + ((int64_t)sp * 3 + m) * BW;
    float *const wp = A.part + (((int64_t)sp * 3 + m) * FP + hb * S::HB + hi * 64) * CP + ci * CTW * 32;
    auto hidden_in = [&](int t) { return hb * S::HB + hi * 64 + t * 32 < FP; };
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < CTW; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[t][c][r] = 0.f;
#pragma unroll
    for (int c = 0; c < CTW; ++c) gsum[c] = 0.0;

    auto step = [&](int k) {
        const unsigned char *const slot = lds + (k % S::SLOTS) * S::SLOT;
        float bs[2] = {0.f, 0.f}, gs[CTW];
#pragma unroll
        for (int c = 0; c < CTW; ++c) gs[c] = 0.f;
#pragma unroll
        for (int r0 = 0; r0 < KP; r0 += 16) {
            Parts<P> af[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    af[t].p[p] = plane_tr<P == 1>(slot + ((2 * hi + t) * P + p) * S::PLB, r0, lane);
                    if constexpr (P == 3 && SUMS == 1) bs[t] = sum_slots(af[t].p[p], bs[t]);
                }
#pragma unroll
            for (int c = 0; c < CTW; ++c) {
                Parts<P> bf;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    bf.p[p] = plane_tr<false>(slot + ((HPL + ci * CTW + c) * P + p) * S::PLB, r0, lane);
                    if constexpr (SUMS == 2) gs[c] = sum_slots(bf.p[p], gs[c]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) mma_parts<32, P>(acc[t][c], af[t], bf);  // in turn they gain nothing here
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) bsum[t] += bs[t];
#pragma unroll
        for (int c = 0; c < CTW; ++c) gsum[c] += gs[c];
    };
    if constexpr (P == 1) {
        const uint32_t l0 = lds_addr(lds);
        auto issue = [&](int k) {  // k = 0, 1, 2, ... in turn
            const bool whole = a0 + (int64_t)(k + 1) * KP <= n;
#pragma unroll
            for (int i = 0; i < S::PER; ++i) {
                const int pc = wave * S::PER + i;
                const uint32_t to = l0 + (k % S::SLOTS) * S::SLOT + (pc % PL) * S::PLB + (pc / PL) * 1024;
                if (whole) dma16s<0>(voff[i], base[i], to);
                else dma16(ragged(i, k), to);
                base[i] += inc[i];
            }
        };
        constexpr int AHEAD = S::SLOTS - 1;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k < nk) issue(k);
#pragma unroll 1
        for (int k = 0; k < nk; ++k) {
            if (k + AHEAD - 1 < nk) wait_vmcnt<(AHEAD - 1) * S::PER>();
            else wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();  // step k is in LDS; step k - 1's slot read by all
            asm volatile("" ::: "memory");
            if (k + AHEAD < nk) issue(k + AHEAD);
            step(k);
        }
    } else {
        f32x4 st[S::PER];
        auto fetch = [&](int k) {  // k = 0, 1, 2, ... in turn
            const bool whole = a0 + (int64_t)(k + 1) * KP <= n;
#pragma unroll
            for (int i = 0; i < S::PER; ++i) {
                st[i] = *reinterpret_cast<const f32x4 *>(whole ? base[i] + voff[i] : ragged(i, k));
                base[i] += k & 1 ? inc2[i] : inc[i];
            }
        };
        auto put = [&](int k) {
#pragma unroll
            for (int i = 0; i < S::PER; ++i) {
                const int pc = wave * S::PER + i, pl = pc % PL;
                const int at = pl < HPL ? hrow * 64 + 8 * hq : (lane >> 2) * 64 + 8 * (lane & 3);
                unsigned char *to = lds + (k % S::SLOTS) * S::SLOT + pl * P * S::PLB + at + 32 * (pc / PL);
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
            step(k);
            if (k + 1 < nk) put(k + 1);
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (!hidden_in(t)) continue;
        float *const to = wp + (int64_t)(32 * t + 4 * (lane >> 5)) * CP + (lane & 31);
#pragma unroll
        for (int c = 0; c < CTW; ++c) {
            if (!first)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][c][r] += to[(8 * (r >> 2) + (r & 3)) * CP + 32 * c];
#pragma unroll
            for (int r = 0; r < 16; ++r) to[(8 * (r >> 2) + (r & 3)) * CP + 32 * c] = acc[t][c][r];
        }
        if (bh) {
            const float s = (float)(bsum[t] + __shfl_xor(bsum[t], 32));
            float *const to = bp + hb * S::HB + hi * 64 + t * 32 + (lane & 31);
            if (lane < 32) *to = first ? s : *to + s;
        }
    }
    if constexpr (P == 1 && SUMS == 1) {
        // Rows of 32 points and chunks of the split: eight lanes a row, TPC a chunk.
        static_assert(KP == 32, "a split is whole rows of cols");
        constexpr int TPC = 64 * W / HPL;
        const int ch = hb * HPL + threadIdx.x / TPC, row = threadIdx.x % TPC / 8, c4 = 4 * (threadIdx.x & 7);
        if (ch < nchunk) {
            const float *const src = A.cols + (((int64_t)m * nchunk + ch) * (tp / 32) + a0 / 32) * 32 + c4;
            double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 8
            for (int k = row; k < nk; k += TPC / 8) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(src + (int64_t)k * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += v[i];
            }
#pragma unroll
            for (int x = 8; x < TPC; x <<= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += __shfl_xor(s[i], x);
            if (row == 0) {
                float *const to = bp + ch * 32 + c4;
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = first ? (float)s[i] : (float)(to[i] + s[i]);
            }
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

template <int P, int CP, int W> __global__ __launch_bounds__(64 * W, 2) void k_gated_dw(const GatedDwArgs<P, CP> A) {
    using S = GatedDw<P, CP, W>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::SLOTS * S::SLOT];
    // The workgroups of one split, which read the same rows of x and g, share an XCD and its L2.
    const int wid = xcd_remap(blockIdx.x, gridDim.x);
    const int hb = wid % A.nhb, m = wid / A.nhb % 3, sp = wid / (3 * A.nhb);
    if (m < 2) gated_dw<P, CP, W, 1>(A, lds, m, hb, sp);
    else if (hb == 0) gated_dw<P, CP, W, 2>(A, lds, m, hb, sp);
    else gated_dw<P, CP, W, 0>(A, lds, m, hb, sp);
}

// The gradients from the splits' sums: block (hidden tile of 32, channel tile of 32, m), four
// groups of 256 threads, each a quarter of the splits in order, then the groups in order.  dWg
// and dWu are [C][F], dWd [F][C].
template <int P, int CP>
__global__ __launch_bounds__(1024) void k_gated_grads(const float *__restrict__ part, const float *__restrict__ bpart, int SP,
                                                      int nchunk, int C, int F, typename GatedIO<P>::T *__restrict__ dWg,
                                                      typename GatedIO<P>::T *__restrict__ dWu,
                                                      typename GatedIO<P>::T *__restrict__ dWd,
                                                      typename GatedIO<P>::T *__restrict__ dbg,
                                                      typename GatedIO<P>::T *__restrict__ dbu,
                                                      typename GatedIO<P>::T *__restrict__ dbd) {
    using T = typename GatedIO<P>::T;
    constexpr int GROUPS = 4;
    __shared__ double sums[GROUPS][32][33];
    const int ht = blockIdx.x, ct = blockIdx.y, m = blockIdx.z;
    const int FP = nchunk * 32, BW = FP > CP ? FP : CP;
    const int q = threadIdx.x >> 8, col = threadIdx.x & 31, r8 = (threadIdx.x >> 5) & 7;
    const int per = (SP + GROUPS - 1) / GROUPS, s0 = q * per, s1 = s0 + per < SP ? s0 + per : SP;
    const int64_t stride = (int64_t)3 * FP * CP;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    const float *src = part + ((int64_t)m * FP + 32 * ht + r8) * CP + 32 * ct + col;
#pragma unroll 8
    for (int s = s0; s < s1; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += src[s * stride + (int64_t)8 * i * CP];
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[q][r8 + 8 * i][col] = v[i];
    // Column sums: by the first channel tile's blocks (da, du), the first hidden tile's (g).
    const bool columns = m == 2 ? ht == 0 : ct == 0;
    const int at = 32 * (m == 2 ? ct : ht) + col;
    if (columns && r8 == 0) {
        double s = 0.0;
#pragma unroll 8
        for (int i = s0; i < s1; ++i) s += bpart[((int64_t)i * 3 + m) * BW + at];
        sums[q][col][32] = s;
    }
    __syncthreads();
    const int a = threadIdx.x >> 5, b = threadIdx.x & 31;  // one value a thread, b along the gradient's rows
    const int f = 32 * ht + (m == 2 ? a : b), c = 32 * ct + (m == 2 ? b : a);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) sum += m == 2 ? sums[i][a][b] : sums[i][b][a];
    if (f < F && c < C) {
        if (m == 2) dWd[(int64_t)f * C + c] = from_float<T>((float)sum);
        else (m ? dWu : dWg)[(int64_t)c * F + f] = from_float<T>((float)sum);
    }
    if (columns && threadIdx.x < 32 && at < (m == 2 ? C : F)) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) s += sums[i][col][32];
        (m == 0 ? dbg : m == 1 ? dbu : dbd)[at] = from_float<T>((float)s);
    }
}

}  // namespace ts3
