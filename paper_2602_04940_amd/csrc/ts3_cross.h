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
//                  32 rows per wave against tiles of states in LDS
//   k_cross_join, k_cross_join_few   join the parts of rows whose states were split over workgroups
//   k_cross_dq     g.out and dq for 32 rows per wave, the scores computed again
//   k_cross_dkv    dk and dv for 32 states per wave against tiles of rows in LDS
//   k_cross_sum, k_cross_sum_dq   sums of split gradients, in the splits' order
//
// Products are 32x32x16 with the operand conventions of ts3_gated.h, bfloat16 as it is (P = 1),
// float32 as three bfloat16 parts (P = 3), both exactly: scores are scaled in float32, by the instruction that
// takes the base or the logarithm of the sum from them.  (Scaled beforehand, in accumulators that start from those,
// they would leave the matrix cores as exponents; but 16 bits of a scaled bfloat16 operand put lse off by 1.3e-3 at
// scores of 300, and sums that start from a logarithm of 14 lose three bits of scores of one: float32 gradients were
// off by 1.2e-6 to 1.8e-6 of their size, now by 0.7e-6, and took as long.)  Scores are computed transposed, rows the states in
// the order of gated_row and columns the queries: a lane then holds 16 consecutive states of one
// query, which are, as they lie, the K slots of the product with the values, and a query's
// maximum and sum are in two lanes.  The values' operand is read from LDS transposed.
// In bfloat16 the weights p and the slopes ds are rounded once, as operands of the next product;
// their sums, and every other quantity, are float32.  With p in two bfloat16 parts out would be off by its own rounding
// alone, 0.0017 of its size in the mean square in place of 0.0024, for twice the products with the values and
// the parting of every weight: 1M rows of 8 heads of 32 and 512 states 0.80 -> 1.17 ms.
#pragma once
#include "ts3_gated.h"  // operands, parts, storage types

namespace ts3 {

// Eight consecutive values of a row.
__device__ __forceinline__ void load8f(const bf16_t *p, float (&v)[8]) {
    const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8f(const float *p, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 u = *reinterpret_cast<const f32x4 *>(p + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * h + i] = u[i];
    }
}

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
    static constexpr int STEP = THREADS / NPC;  // rows from one item of a thread to its next
    u32x4 r[ITEMS][P == 1 ? 1 : 2];

    __device__ __forceinline__ static int row0() { return threadIdx.x / NPC % ROWS; }
    __device__ __forceinline__ static int col0(int D) {
        const int c = threadIdx.x % NPC * 8;
        return c < D ? c : 0;  // columns past D are read from the first and dropped
    }
    __device__ __forceinline__ void item(int k, const T *p) {
#pragma unroll
        for (int h = 0; h < (P == 1 ? 1 : 2); ++h) r[k][h] = *reinterpret_cast<const u32x4 *>(p + 4 * h);
    }
    // Items at equal steps from the thread's first, rows past `end` read from `safe` instead.
    __device__ __forceinline__ void load(const T *p, int64_t step, int end, const T *safe) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) item(k, row0() + k * STEP < end ? p + k * step : safe);
    }
    // at(row): the row's address, always readable.
    template <typename F> __device__ __forceinline__ void load(int D, F at) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) item(k, at((threadIdx.x + k * THREADS) / NPC % ROWS) + col0(D));
    }
    // there(row): whether the row is there; others are zero, whatever they hold.  `all`: every row is.
    template <typename F> __device__ __forceinline__ void store(unsigned char *tile, int D, bool all, F there) const {
        const bool cin = threadIdx.x % NPC * 8 < D;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + k * THREADS, row = i / NPC, pc = i % NPC;
            if (TOTAL % THREADS && i >= TOTAL) continue;
            unsigned char *const to = tile + row * (DP * 2) + ((pc ^ cross_swz<DP>(row)) << 4);
            u32x4 v[P == 1 ? 1 : 2];
#pragma unroll
            for (int h = 0; h < (P == 1 ? 1 : 2); ++h) v[h] = r[k][h];
            if (!(all && D == DP)) {
                asm volatile("");  // a branch, not selections
                const bool in = cin && there(row);
#pragma unroll
                for (int h = 0; h < (P == 1 ? 1 : 2); ++h) v[h] = in ? v[h] : u32x4{0, 0, 0, 0};
            }
            if constexpr (P == 1) {
                *reinterpret_cast<u32x4 *>(to) = v[0];
            } else {
                float x[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) x[t] = __uint_as_float(v[t >> 2][t & 3]);
                Parts<3> f;
                split8(x, f);
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

// Division by a number that the host knows, exact for 32-bit operands: the upper half of the product
// with floor(2^64 / d) + 1.
struct CrossDiv {
    uint32_t d;
    uint64_t m;
    __host__ CrossDiv(uint32_t d = 1) : d(d), m(~uint64_t(0) / d + 1) {}
    // d = 1 gives m = 0 (2^64)
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return m ? (uint32_t)__umul64hi(n, m) : n; }
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
    CrossDiv by_splits, by_heads, by_blocks, by_G;
    float *lse, *delta;         // [B][H][N]
    void *to, *to2;             // results (out, dq, or dk and dv), contiguous
    float *part, *part2;        // of split loops
    __device__ __forceinline__ int heads() const { return (int)by_heads.d; }
    __device__ __forceinline__ int rows() const { return N * G; }
};
__device__ __forceinline__ float *cross_stat(float *p, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : (int)A.by_G((uint32_t)r), h = hk * A.G + r - n * A.G;
    return p + ((int64_t)b * A.H + h) * A.N + n;
}
template <typename T>
__device__ __forceinline__ const T *cross_row(const CrossView &v, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : (int)A.by_G((uint32_t)r), h = hk * A.G + r - n * A.G;
    return (const T *)v.p + b * v.sb + n * v.sr + h * v.sh;
}
// Row r of a contiguous [B][N][H][D] result.
template <typename T> __device__ __forceinline__ T *cross_to(T *p, const CrossArgs &A, int b, int hk, int r) {
    const int n = A.G == 1 ? r : (int)A.by_G((uint32_t)r), h = hk * A.G + r - n * A.G;
    return p + (((int64_t)b * A.N + n) * A.H + h) * A.D;
}
// States of sample b that may be there: those before its length.
__device__ __forceinline__ int cross_length(const CrossArgs &A, int b) {
    if (!A.lengths) return A.S;
    const int n = A.lengths[b];
    return n < 0 ? 0 : n > A.S ? A.S : n;
}
// Which workgroup does what: (b, block of rows or states, shared head, split), the split innermost and then
// the head.  Consecutive workgroups go to different XCDs, and so does a long sample's work: with the workgroups of
// an L2 next to each other, the XCDs with the short samples end early (8 samples of 9,000 rows and up to 2,000
// states, 4 heads of 64: 177 against 117 us, with the gradient 704 against 545), one row's long states come
// through half of the XCDs (8 heads of 32 and 100,003 states 42 against 24 us), and nothing is gained (72,000 rows
// of 2,000 states 194 against 192 us): states are few bytes a product.
struct CrossAt {
    int b, hk, blk, split;
    __device__ __forceinline__ explicit CrossAt(const CrossArgs &A) {
        const uint32_t i = blockIdx.x, j = A.by_splits(i), k = A.by_heads(j), l = A.by_blocks(k);
        split = (int)(i - j * A.by_splits.d);
        hk = (int)(j - k * A.by_heads.d);
        blk = (int)(k - l * A.by_blocks.d);
        b = (int)l;
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

// The sum of two lanes' values, 32 apart.
__device__ __forceinline__ float both_halves(float v) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ float dot2(bf16x2 a, bf16x2 b, float c) { return __builtin_amdgcn_fdot2_f32_bf16(a, b, c, false); }
__device__ __forceinline__ f32x16 splat16(float v) { return f32x16{v, v, v, v, v, v, v, v, v, v, v, v, v, v, v, v}; }

// Which of the tile's states from `first` are there; bit j is state first + j.
__device__ __forceinline__ uint64_t cross_present(const CrossArgs &A, unsigned char m, int first, int len, int tile) {
    const int j = threadIdx.x & 63;
    return __ballot(j < tile && first + j < len && m);
}
__device__ __forceinline__ unsigned char cross_mask(const CrossArgs &A, int b, int first, int len) {
    const int j = first + (threadIdx.x & 63);
    return A.mask ? A.mask[(int64_t)b * A.S + (j < len ? j : 0)] : 1;
}

// 32 rows of a wave on their way through the states.
//
// The exponents are taken against a base per row, which need not be the maximum.  It is zero where the
// row's first 32 states have a sum of weights of 2^-16 at least then, or else their maximum; afterwards
// only what lies so far above that a lane's sum of 16 weights reaches 2^40 moves it.  The 32 states are
// then done over, and the maximum is not looked for otherwise.  In float32 and bfloat16 the weights'
// precision does not depend on the base.
template <int P, int DP> struct CrossRows {
    using T = typename GatedIO<P>::T;
    static constexpr int KS = DP / 16, DB = (DP + 31) / 32;
    Parts<P> qf[KS];
    f32x16 o[DB];
    float base, l;
    float low;  // what a sum has to reach: something while a row has no base yet, then nothing

    // Row r, one past the last read as the last.
    __device__ __forceinline__ void begin(const CrossArgs &A, const CrossAt &at, int r) {
        cross_load_row<P, DP>(cross_row<T>(A.q, A, at.b, at.hk, min(r, A.rows() - 1)), A.D, true, qf);
        base = l = 0.f;
        low = 0x1p-16f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    }
    // The states 32 u .. + 31 of a tile of keys and one of values; bit j of `here` is whether j is there.
    __device__ __forceinline__ void step(const unsigned char *kl, const unsigned char *vl, int plane, int u, uint32_t here,
                                         const CrossRowRead<DP> &rows, const CrossColRead<DP> &cols, float scale2, int g) {
        if (here == 0) return;
        f32x16 s;
        // exponents against the base, absent states' at minus infinity
        auto scores = [&]() {
            s = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Parts<P> a;
                rows.template read<P>(kl, plane, u, ks, a);
                mma_parts<32, P>(s, a, qf[ks]);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = fmaf(s[v], scale2, -base);
            if (here != ~0u) {
                uint32_t bits = here >> (16 * g);
                asm("" : "+v"(bits));  // or the bits are taken apart where no state is absent, too
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v] = bits >> v & 1 ? s[v] : -INFINITY;
            }
        };
        float sum;
        Parts<P> w[2];
#pragma unroll 1
        for (bool again = false;; again = true) {
            scores();
            sum = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = fast_exp2(s[8 * h + e]);
                    sum += x[e];
                }
                to_parts(x, w[h]);
            }
            if (again) break;
            const unsigned out = !(sum < 0x1p40f && sum >= low);
            if (!__any(out)) {
                low = 0.f;
                break;
            }
            scores();
            // a row moves by its own sums alone: the others' results do not depend on it
            const auto sw = __builtin_amdgcn_permlane32_swap(out, out, false, false);
            const bool moves = sw[0] | sw[1], have = low == 0.f;
            float mx = -INFINITY;
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
            const auto mw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(mw[0]), __uint_as_float(mw[1]));
            const float up = !moves || mx == -INFINITY ? 0.f : have ? fmaxf(mx, 0.f) : mx;
            const float alpha = have ? fast_exp2(-up) : 1.f;
            if (!moves || mx > -INFINITY) low = 0.f;
            base += up;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= alpha;
        }
        l += sum;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                Parts<P> a;
                cols.template read<P>(vl, plane, u, h, d, a);
                mma_parts<32, P>(o[d], a, w[h]);
            }
    }
    __device__ __forceinline__ void finish(const CrossArgs &A, const CrossAt &at, int r, int g) const {
        const int R = A.rows();
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        const float sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
        if (r >= R) return;
        if (A.splits == 1) {
            // no state: weights of zero, whose sum is minus infinity in the logarithm
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T *const to = cross_to((T *)A.to, A, at.b, at.hk, r);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int c = 32 * d + 16 * g;
                float x[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = o[d][v] * inv;
                if (c < A.D) store_row<16>(to + c, x);
            }
            if (g == 0) *cross_stat(A.lse, A, at.b, at.hk, r) = sum == 0.f ? -INFINITY : (base + log2f(sum)) * LN2;
        } else {
            // part[split][b][hk][r][DP + 4]: unscaled sums, their base and their weights' sum
            const int64_t row = (((int64_t)at.split * A.B + at.b) * A.heads() + at.hk) * R + r;
            float *const to = A.part + row * (DP + 4);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int c = 32 * d + 16 * g;
                float x[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = o[d][v];
                if (c < A.D) store_row<16>(to + c, x);
            }
            if (g == 0) {
                to[DP] = sum == 0.f ? -INFINITY : base;
                to[DP + 1] = sum;
            }
        }
    }
};

// What bounds it: the vector ALU (50,003 float32 rows and 8 heads of 16 against 1,000 states 0.26 ms, a fifth of
// them masked 0.28: vector instructions on 82% of the cycles, most of them parting weights in three, matrix cores on
// 41%), and for the few rows of a wave alone (W = 1) the loads of states (one row of 4 samples of 100,003 states, two heads
// of 64 each, 43 us with the join, 4.8 TB/s; of samples of different lengths 37 us, 3.4 TB/s, as the longest outlasts the others).
//
// Workgroup (b, hk, block, split): 32 rows per wave, W waves, against the split's tiles of
// states.  The next tile is on its way to registers while this one is used, and goes to the other
// half of LDS after it (a wave alone needs one half: its own reads come first).
template <int P, int DP, int W>
__global__ __launch_bounds__(64 * W, W == 4 ? (DP * P <= 32 ? 4 : DP * P <= 96 ? 2 : 1) : 1) void k_cross_fwd(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TK = cross_tile<P, DP, W>(), SUB = TK / 32, HALVES = W == 1 ? 1 : 2;
    using Tile = CrossTile<P, DP, TK, 64 * W>;
    __shared__ __align__(16) unsigned char lds[HALVES][2][Tile::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D;
    const CrossAt at(A);
    const int len = cross_length(A, at.b), tiles = (len + TK - 1) / TK;
    const int t0 = at.split * A.per, t1 = min(tiles, t0 + A.per);
    const int r0 = (at.blk * W + wave) * 32 + (lane & 31);
    const T *const kb = (const T *)A.k.p + at.b * A.k.sb + at.hk * A.k.sh;
    const T *const vb = (const T *)A.v.p + at.b * A.v.sb + at.hk * A.v.sh;
    CrossRows<P, DP> q;
    q.begin(A, at, r0);
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile kt, vt;
    const T *const kz = kb + Tile::col0(D), *const vz = vb + Tile::col0(D);
    const T *kp = kz + ((int64_t)Tile::row0() + (int64_t)t0 * TK) * A.k.sr, *vp = vz + ((int64_t)Tile::row0() + (int64_t)t0 * TK) * A.v.sr;
    const int64_t ks = TK * A.k.sr, vs = TK * A.v.sr;
    auto fetch = [&](int t) {
        const int first = t * TK;
        kt.load(kp, Tile::STEP * A.k.sr, len - first, kz);
        vt.load(vp, Tile::STEP * A.v.sr, len - first, vz);
        kp += ks;
        vp += vs;
        return cross_mask(A, at.b, first, len);
    };
    constexpr uint64_t ALL = TK == 64 ? ~0ull : (1ull << TK) - 1;
    // absent values are cleared, which weights of zero multiply; absent keys' scores are replaced
    auto put = [&](int t, uint64_t there) {
        kt.store(lds[t & (HALVES - 1)][0], D, true, [](int) { return true; });
        vt.store(lds[t & (HALVES - 1)][1], D, there == ALL, [&](int row) { return (there >> row & 1) != 0; });
    };
    uint64_t there = 0;
    unsigned char mb = 0;
    if (t0 < t1) {
        mb = fetch(t0);
        there = cross_present(A, mb, t0 * TK, len, TK);
        put(t0, there);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) mb = fetch(t + 1);
        const unsigned char *const kl = lds[t & (HALVES - 1)][0], *const vl = lds[t & (HALVES - 1)][1];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            q.step(kl, vl, Tile::PLANE, u, u ? (uint32_t)(there >> 32) : (uint32_t)there, rows, cols, A.scale * LOG2E, g);
        if constexpr (HALVES == 1) __syncthreads();
        if (t + 1 < t1) {
            there = cross_present(A, mb, (t + 1) * TK, len, TK);
            put(t + 1, there);
        }
        __syncthreads();
    }
    q.finish(A, at, r0, g);
}

// The same for many rows and few states: a sample's and head's states all lie in LDS, and the
// workgroup's W waves go through blocks of 32 rows, with neither loads of states nor barriers between
// them.  Of the blocks, A.per workgroups (at.blk) take every one in turn, and a workgroup's waves the next
// one each: dealt out beforehand, the waves of a SIMD, which do not run equally fast, would end
// apart (a quarter of the waves' time idle in the forward).  1M rows of 8 heads of 32 and 512 states
// 0.79 to 0.83 ms, 640 TFLOP/s: the vector ALU is busy on all cycles (a multiply-add, an exponential, a sum and half a
// conversion per score), matrix cores on 32%.
template <int P, int DP, int WAVES> struct CrossAll {
    static constexpr int TK = cross_tile<P, DP, WAVES>(), W = WAVES;
    using Tile = CrossTile<P, DP, TK, 64 * W>;
    static constexpr int TILE = 2 * Tile::BYTES, BATCH = 2;
    static constexpr int LDS = 160 * 1024;      // a workgroup per compute unit
    static constexpr bool FITS = DP * P <= 64;  // within the registers of so many waves
    static constexpr int64_t bytes(int64_t S) { return (S + TK - 1) / TK * (TILE + 8) + 8; }
    // The first row of the wave's next block.
    __device__ static __forceinline__ int64_t next(const CrossArgs &A, const CrossAt &at, int *taken) {
        int i = 0;
        if ((threadIdx.x & 63) == 0) i = atomicAdd(taken, 1);
        return ((int64_t)__builtin_amdgcn_readfirstlane(i) * A.per + at.blk) * 32;
    }
    // Keys, values (absent ones cleared) and presence of the tiles.
    __device__ static __forceinline__ void fill(const CrossArgs &A, const CrossAt &at, int len, unsigned char *tiles, uint64_t *present) {
        using T = typename GatedIO<P>::T;
        const int n = (len + TK - 1) / TK, D = A.D;
        const T *const kb = (const T *)A.k.p + at.b * A.k.sb + at.hk * A.k.sh;
        const T *const vb = (const T *)A.v.p + at.b * A.v.sb + at.hk * A.v.sh;
        for (int t = 0; t < n; t += BATCH) {
            Tile kt[BATCH], vt[BATCH];
            unsigned char m[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int first = (t + i) * TK;
                kt[i].load(D, [&](int row) { return kb + (int64_t)min(first + row, len - 1) * A.k.sr; });
                vt[i].load(D, [&](int row) { return vb + (int64_t)min(first + row, len - 1) * A.v.sr; });
                m[i] = cross_mask(A, at.b, first, len);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (t + i >= n) break;
                const uint64_t there = cross_present(A, m[i], (t + i) * TK, len, TK);
                auto in = [&](int row) { return (there >> row & 1) != 0; };
                kt[i].store(tiles + (t + i) * TILE, D, false, in);
                vt[i].store(tiles + (t + i) * TILE + Tile::BYTES, D, false, in);
                if (threadIdx.x == 0) present[t + i] = there;
            }
        }
        __syncthreads();
    }
};
template <int P, int DP>
__global__ __launch_bounds__(1024, 4) void k_cross_fwd_all(const CrossArgs A) {
    using All = CrossAll<P, DP, 16>;
    extern __shared__ __align__(16) unsigned char all_lds[];
    const CrossAt at(A);
    const int lane = threadIdx.x & 63, g = lane >> 5, R = A.rows();
    const int len = cross_length(A, at.b), n = (len + All::TK - 1) / All::TK;
    uint64_t *const present = (uint64_t *)(all_lds + (size_t)((A.S + All::TK - 1) / All::TK) * All::TILE);
    int *const taken = (int *)(present + (A.S + All::TK - 1) / All::TK);
    if (threadIdx.x == 0) *taken = 0;
    All::fill(A, at, len, all_lds, present);
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    for (int64_t first; (first = All::next(A, at, taken)) < R;) {
        const int r0 = (int)first;
        CrossRows<P, DP> q;
        q.begin(A, at, r0 + (lane & 31));
        for (int t = 0; t < n; ++t) {
            const uint64_t there = present[t];
            const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)there), hi = __builtin_amdgcn_readfirstlane((uint32_t)(there >> 32));
            const unsigned char *const kl = all_lds + t * All::TILE;
            q.step(kl, kl + All::Tile::BYTES, All::Tile::PLANE, 0, lo, rows, cols, A.scale * LOG2E, g);
            if constexpr (All::TK == 64) q.step(kl, kl + All::Tile::BYTES, All::Tile::PLANE, 1, hi, rows, cols, A.scale * LOG2E, g);
        }
        q.finish(A, at, r0 + (lane & 31), g);
    }
}

// Few parts: a row per DP / 4 lanes, which take the splits' parts in order, scaled to the largest base.
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_join_few(const CrossArgs A, int64_t count) {
    using T = typename GatedIO<P>::T;
    constexpr int LG = DP / 4;
    const int64_t bhr = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LG, step = count * (DP + 4);
    const int c = 4 * (threadIdx.x % LG), R = A.rows();
    if (bhr >= count || c >= A.D) return;
    const float *const part = A.part + bhr * (DP + 4);
    float top = -INFINITY;
    for (int s = 0; s < A.splits; ++s) top = fmaxf(top, part[s * step + DP]);
    const float base = top == -INFINITY ? 0.f : top;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int s = 0; s < A.splits; ++s) {
        const float *const p = part + s * step;
        const float w = fast_exp2(p[DP] - base);
        v += w * *reinterpret_cast<const f32x4 *>(p + c);
        sum += w * p[DP + 1];
    }
    const int b = (int)(bhr / R / A.heads()), hk = (int)(bhr / R % A.heads()), r = (int)(bhr % R);
    T *const to = cross_to((T *)A.to, A, b, hk, r) + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = from_float<T>(sum == 0.f ? 0.f : v[i] / sum);
    if (c == 0) *cross_stat(A.lse, A, b, hk, r) = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
}
// Many: a row per workgroup, 1024 / DP splits at a time by as many groups of lanes, then the groups' sums in
// order.
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_join(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int LG = DP / 4, NG = 256 / LG;
    __shared__ __align__(16) float acc[NG][DP];
    __shared__ float sums[NG], tops[4];
    const int R = A.rows(), tid = threadIdx.x, c = 4 * (tid % LG), q = tid / LG;
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
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    const bool in = c < A.D;
#pragma unroll 8
    for (int s = q; s < A.splits; s += NG) {
        const float *const p = part + s * step;
        const f32x4 x = *reinterpret_cast<const f32x4 *>(p + (in ? c : 0));
        const float w = fast_exp2(p[DP] - base);
        v += w * x;
        sum += w * p[DP + 1];
    }
    *reinterpret_cast<f32x4 *>(&acc[q][c]) = v;
    if (c == 0) sums[q] = sum;
    __syncthreads();
    if (tid >= DP) return;
    sum = 0.f;
    float y = 0.f;
    for (int i = 0; i < NG; ++i) {
        sum += sums[i];
        y += acc[i][tid];
    }
    if (tid < A.D) cross_to((T *)A.to, A, b, hk, r)[tid] = from_float<T>(sum == 0.f ? 0.f : y / sum);
    if (tid == 0) *cross_stat(A.lse, A, b, hk, r) = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
}

// 32 rows of a wave: dq from the states they go through, the values being a second operand of rows and the
// keys read transposed, and delta = g.out.
//
// In bfloat16 out is rounded, and delta from it is off by 2^-8 of |g| |out|, which where a row's weight lies on few
// states is much of dp - delta.  It is what the slopes x = p (dp - delta) start from, but the loop takes sum x and
// sum p k beside sum x k, in float32: the first is what delta is off by, and dk is computed from the better one; and
// their product is what dq is off by.  Taken from the rounded slopes instead, which sum x k has, the first also is what
// their roundings add to dq through the mean key, as sum x k - sum x sum p k is sum x (k - mean k): keys around 4 with a
// spread of one put dq off by 0.0070 of its size before, now by 0.0023, and keys around zero by 0.0024 and 0.0022
// (0.0017 of it dq's own rounding).  In float32 sum p k would cost six products more, where the roundings
// are 2^-24.
//
// 250,001 points of 512 states, 8 heads of 32, take k_cross_dq_all 0.35 ms, vector instructions on 78% of the cycles
// and matrix cores on 39%.
template <int P, int DP> struct CrossSlopes {
    using T = typename GatedIO<P>::T;
    static constexpr int KS = DP / 16, DB = (DP + 31) / 32;
    static constexpr bool MEND = P == 1;
    Parts<P> qf[KS], gf[KS];
    f32x16 o[DB], dstart;         // dstart: minus delta from out
    float start;                  // minus the logarithm of the sum
    f32x16 means[MEND ? DB : 1];  // sum p k
    float rest, rounded;          // of the lane's states, sum p (dp - delta from out), and of its roundings
    __device__ __forceinline__ void begin(const CrossArgs &A, const CrossAt &at, int r, int g) {
        const int rc = min(r, A.rows() - 1), D = A.D;
        const T *const grow = cross_row<T>(A.g, A, at.b, at.hk, rc), *const orow = cross_row<T>(A.out, A, at.b, at.hk, rc);
        cross_load_row<P, DP>(cross_row<T>(A.q, A, at.b, at.hk, rc), D, true, qf);
        cross_load_row<P, DP>(grow, D, true, gf);
        float delta = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = 16 * ks + 8 * g;
            float x[8], y[8], d = 0.f;
            load8f(grow + (c < D ? c : 0), x);
            load8f(orow + (c < D ? c : 0), y);
#pragma unroll
            for (int e = 0; e < 8; ++e) d += x[e] * y[e];
            delta += c < D ? d : 0.f;
        }
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(delta), __float_as_uint(delta), false, false);
        delta = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
        start = -LOG2E * *cross_stat(A.lse, A, at.b, at.hk, rc);
        dstart = splat16(-delta);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            o[d] = f32x16{};
            if constexpr (MEND) means[d] = f32x16{};
        }
        rest = rounded = 0.f;
    }
    __device__ __forceinline__ void step(const unsigned char *kl, const unsigned char *vl, int plane, int u, uint32_t here,
                                         const CrossRowRead<DP> &rows, const CrossColRead<DP> &cols, float scale2, int g) {
        if (here == 0) return;
        f32x16 s{}, dp = dstart;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Parts<P> a;
            rows.template read<P>(kl, plane, u, ks, a);
            mma_parts<32, P>(s, a, qf[ks]);
            rows.template read<P>(vl, plane, u, ks, a);
            mma_parts<32, P>(dp, a, gf[ks]);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = fast_exp2(fmaf(s[v], scale2, start));
        if (here != ~0u) {
            uint32_t bits = here >> (16 * g);
            asm("" : "+v"(bits));
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[v] = bits >> v & 1 ? s[v] : 0.f;
                dp[v] = bits >> v & 1 ? dp[v] : 0.f;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[8], y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = s[8 * h + e];
                x[e] = y[e] * dp[8 * h + e];
                if constexpr (MEND) rest += x[e];
            }
            Parts<P> w, z;
            to_parts(x, w);
            if constexpr (MEND) {
                to_parts(y, z);
#pragma unroll
                for (int e = 0; e < 8; e += 2) rounded = dot2(bf16x2{w.p[0][e], w.p[0][e + 1]}, bf16x2{(__bf16)1.f, (__bf16)1.f}, rounded);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                Parts<P> a;
                cols.template read<P>(kl, plane, u, h, d, a);
                mma_parts<32, P>(o[d], a, w);
                if constexpr (MEND) mma_parts<32, P>(means[d], a, z);
            }
        }
    }
    // Parts of split loops hold sum p (dp - delta from out) k, that of p k and the two without k, a row of 2 DP + 4.
    __device__ __forceinline__ void finish(const CrossArgs &A, const CrossAt &at, int r, int g) const {
        const int R = A.rows();
        const float off = both_halves(rest), sum = both_halves(rounded);
        if (r >= R) return;
        float *const part = A.part + ((((int64_t)at.split * A.B + at.b) * A.heads() + at.hk) * R + r) * (2 * DP + 4);
        T *const to = cross_to((T *)A.to, A, at.b, at.hk, r);
        if (g == 0) {
            if (A.splits == 1 || at.split == 0) *cross_stat(A.delta, A, at.b, at.hk, r) = (A.splits == 1 ? off : 0.f) - dstart[0];
            if (MEND && A.splits > 1) part[2 * DP] = off, part[2 * DP + 1] = sum;
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const int c = 32 * d + 16 * g;
            float x[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                x[v] = o[d][v];
                if constexpr (MEND)
                    if (A.splits == 1) x[v] -= sum * means[d][v];
                x[v] *= A.splits == 1 ? A.scale : 1.f;
            }
            if (c >= A.D) continue;
            if (A.splits == 1) {
                store_row<16>(to + c, x);
                continue;
            }
            store_row<16>(part + c, x);
            if constexpr (MEND) {
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = means[d][v];
                store_row<16>(part + DP + c, x);
            }
        }
    }
};

// As k_cross_fwd, and as k_cross_fwd_all.
template <int P, int DP> __global__ __launch_bounds__(256, DP * P <= 96 ? 2 : 1) void k_cross_dq(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TK = P == 1 && DP < 128 ? 64 : 32, SUB = TK / 32;
    using Tile = CrossTile<P, DP, TK, 256>;
    __shared__ __align__(16) unsigned char lds[2][2][Tile::BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D;
    const CrossAt at(A);
    const int len = cross_length(A, at.b), tiles = (len + TK - 1) / TK;
    const int t0 = at.split * A.per, t1 = min(tiles, t0 + A.per);
    const int r = at.blk * 128 + wave * 32 + (lane & 31);
    const T *const kb = (const T *)A.k.p + at.b * A.k.sb + at.hk * A.k.sh;
    const T *const vb = (const T *)A.v.p + at.b * A.v.sb + at.hk * A.v.sh;
    CrossSlopes<P, DP> q;
    q.begin(A, at, r, g);
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile kt, vt;
    const T *const kz = kb + Tile::col0(D), *const vz = vb + Tile::col0(D);
    const T *kp = kz + ((int64_t)Tile::row0() + (int64_t)t0 * TK) * A.k.sr, *vp = vz + ((int64_t)Tile::row0() + (int64_t)t0 * TK) * A.v.sr;
    const int64_t ks = TK * A.k.sr, vs = TK * A.v.sr;
    auto fetch = [&](int t) {
        const int first = t * TK;
        kt.load(kp, Tile::STEP * A.k.sr, len - first, kz);
        vt.load(vp, Tile::STEP * A.v.sr, len - first, vz);
        kp += ks;
        vp += vs;
        return cross_mask(A, at.b, first, len);
    };
    constexpr uint64_t ALL = TK == 64 ? ~0ull : (1ull << TK) - 1;
    // absent keys are cleared, which slopes of zero multiply; absent values' slopes are replaced
    auto put = [&](int t, uint64_t there) {
        kt.store(lds[t & 1][0], D, there == ALL, [&](int row) { return (there >> row & 1) != 0; });
        vt.store(lds[t & 1][1], D, true, [](int) { return true; });
    };
    uint64_t there = 0;
    unsigned char mb = 0;
    if (t0 < t1) {
        mb = fetch(t0);
        there = cross_present(A, mb, t0 * TK, len, TK);
        put(t0, there);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) mb = fetch(t + 1);
        const unsigned char *const kl = lds[t & 1][0], *const vl = lds[t & 1][1];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            q.step(kl, vl, Tile::PLANE, u, u ? (uint32_t)(there >> 32) : (uint32_t)there, rows, cols, A.scale * LOG2E, g);
        if (t + 1 < t1) {
            there = cross_present(A, mb, (t + 1) * TK, len, TK);
            put(t + 1, there);
        }
        __syncthreads();
    }
    q.finish(A, at, r, g);
}
// As many waves as the registers allow: with sum p k, bfloat16 heads of 64 spill at 12 (the whole gradient of
// 100,003 points of 256 states and 4 heads 277 us, at 8 waves 211).
template <int WIDTH> constexpr int CROSS_DQ_WAVES = WIDTH <= 48 ? 12 : 8;
template <int P, int DP>
__global__ __launch_bounds__(64 * CROSS_DQ_WAVES<DP * P>, CROSS_DQ_WAVES<DP * P> / 4) void k_cross_dq_all(const CrossArgs A) {
    using All = CrossAll<P, DP, CROSS_DQ_WAVES<DP * P>>;
    extern __shared__ __align__(16) unsigned char all_lds[];
    const CrossAt at(A);
    const int lane = threadIdx.x & 63, g = lane >> 5, R = A.rows();
    const int len = cross_length(A, at.b), n = (len + All::TK - 1) / All::TK;
    uint64_t *const present = (uint64_t *)(all_lds + (size_t)((A.S + All::TK - 1) / All::TK) * All::TILE);
    int *const taken = (int *)(present + (A.S + All::TK - 1) / All::TK);
    if (threadIdx.x == 0) *taken = 0;
    All::fill(A, at, len, all_lds, present);
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    for (int64_t first; (first = All::next(A, at, taken)) < R;) {
        const int r0 = (int)first;
        CrossSlopes<P, DP> q;
        q.begin(A, at, r0 + (lane & 31), g);
        for (int t = 0; t < n; ++t) {
            const uint64_t there = present[t];
            const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)there), hi = __builtin_amdgcn_readfirstlane((uint32_t)(there >> 32));
            const unsigned char *const kl = all_lds + t * All::TILE;
            q.step(kl, kl + All::Tile::BYTES, All::Tile::PLANE, 0, lo, rows, cols, A.scale * LOG2E, g);
            if constexpr (All::TK == 64) q.step(kl, kl + All::Tile::BYTES, All::Tile::PLANE, 1, hi, rows, cols, A.scale * LOG2E, g);
        }
        q.finish(A, at, r0 + (lane & 31), g);
    }
}

// dk and dv of 32 states per wave, four waves, summed over the split's tiles of rows (queries and
// their output gradients in LDS with the rows' lse and delta).  250,001 points and 512 states, 8 heads of 32 in
// bfloat16: 0.34 ms, the vector ALU busy on 64% of the cycles, matrix cores on 40%, waves waiting for LDS on 20%: the two or
// three waves a SIMD that the sums leave room for take turns more than they overlap.
template <int P, int DP> __global__ __launch_bounds__(256, DP * P <= 64 ? 2 : 1) void k_cross_dkv(const CrossArgs A) {
    using T = typename GatedIO<P>::T;
    constexpr int TR = P == 1 && DP < 128 ? 64 : 32, SUB = TR / 32, KS = DP / 16, DB = (DP + 31) / 32;
    using Tile = CrossTile<P, DP, TR, 256>;
    __shared__ __align__(16) unsigned char lds[2][2][Tile::BYTES];
    __shared__ __align__(16) float stat[2][2][TR];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, D = A.D, R = A.rows();
    const CrossAt at(A);
    const int len = cross_length(A, at.b), tiles = (R + TR - 1) / TR;
    const int j = at.blk * 128 + wave * 32 + (lane & 31), jc = min(j, A.S - 1);
    const bool there = j < len && (!A.mask || A.mask[(int64_t)at.b * A.S + jc]);
    // a block of absent states has nothing to sum
    const int t0 = at.split * A.per, t1 = at.blk * 128 < len ? min(tiles, t0 + A.per) : t0;
    const float scale2 = A.scale * LOG2E;
    Parts<P> kf[KS], vf[KS];
    cross_load_row<P, DP>((const T *)A.k.p + at.b * A.k.sb + jc * A.k.sr + at.hk * A.k.sh, D, there, kf);
    cross_load_row<P, DP>((const T *)A.v.p + at.b * A.v.sb + jc * A.v.sr + at.hk * A.v.sh, D, there, vf);
    typename Mat<32>::D dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = typename Mat<32>::D{};
    const CrossRowRead<DP> rows(lane);
    const CrossColRead<DP> cols(lane);
    Tile qt, gt;
    float st = 0.f;
    // Where G divides 16, a thread's rows keep their head from item to item and tile to tile.
    const bool even = 16 % A.G == 0;
    const int64_t pts = even ? TR / A.G : 0, ptk = even ? Tile::STEP / A.G : 0;  // points a tile, and an item
    const T *const qz = cross_row<T>(A.q, A, at.b, at.hk, 0) + Tile::col0(D), *const gz = cross_row<T>(A.g, A, at.b, at.hk, 0) + Tile::col0(D);
    const T *qp = cross_row<T>(A.q, A, at.b, at.hk, Tile::row0() + t0 * TR) + Tile::col0(D);
    const T *gp = cross_row<T>(A.g, A, at.b, at.hk, Tile::row0() + t0 * TR) + Tile::col0(D);
    float *const stats = threadIdx.x < TR ? A.lse : A.delta, *const sz = cross_stat(stats, A, at.b, at.hk, 0);
    const float *sp = cross_stat(stats, A, at.b, at.hk, (int)threadIdx.x % TR + t0 * TR);
    auto fetch = [&](int t) {
        const int first = t * TR;
        if (even) {
            qt.load(qp, ptk * A.q.sr, R - first, qz);
            gt.load(gp, ptk * A.g.sr, R - first, gz);
            if (threadIdx.x < 2 * TR) st = *(first + (int)threadIdx.x % TR < R ? sp : sz);
            qp += pts * A.q.sr;
            gp += pts * A.g.sr;
            sp += pts;
        } else {
            qt.load(D, [&](int row) { return cross_row<T>(A.q, A, at.b, at.hk, min(first + row, R - 1)); });
            gt.load(D, [&](int row) { return cross_row<T>(A.g, A, at.b, at.hk, min(first + row, R - 1)); });
            if (threadIdx.x < 2 * TR) st = *cross_stat(stats, A, at.b, at.hk, min(first + (int)threadIdx.x % TR, R - 1));
        }
    };
    auto put = [&](int t) {
        const int first = t * TR;
        const bool all = first + TR <= R;
        qt.store(lds[t & 1][0], D, all, [&](int row) { return first + row < R; });
        gt.store(lds[t & 1][1], D, all, [&](int row) { return first + row < R; });
        if (threadIdx.x < 2 * TR) {
            // negated, as the accumulators start; past the last row the weights are e^-inf
            const int row = threadIdx.x % TR;
            const bool lse = threadIdx.x < TR, in = first + row < R;
            stat[t & 1][lse ? 0 : 1][row] = lse ? in ? -LOG2E * st : -INFINITY : in ? -st : 0.f;
        }
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
            // what an absent state's column holds stays in it, and is dropped at the end
            f32x16 s, dp, ls;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int row = 32 * u + 16 * g + e;
                const f32x4 x = *reinterpret_cast<const f32x4 *>(&stat[t & 1][0][row]);
                const f32x4 y = *reinterpret_cast<const f32x4 *>(&stat[t & 1][1][row]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ls[e + i] = x[i];
                    dp[e + i] = y[i];
                }
            }
            s = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Parts<P> a;
                rows.template read<P>(ql, Tile::PLANE, u, ks, a);
                mma_parts<32, P>(s, a, kf[ks]);
                rows.template read<P>(gl, Tile::PLANE, u, ks, a);
                mma_parts<32, P>(dp, a, vf[ks]);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[v] = fast_exp2(fmaf(s[v], scale2, ls[v]));
                dp[v] *= s[v];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = s[8 * h + e];
                    y[e] = dp[8 * h + e];
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

// dk and dv: the splits' values of element i, in order.
template <typename T> __global__ __launch_bounds__(256) void k_cross_sum(const CrossArgs A, int64_t count) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    const float *const p = blockIdx.y ? A.part2 : A.part;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < A.splits; ++s) v += p[s * count + i];
    ((T *)(blockIdx.y ? A.to2 : A.to))[i] = from_float<T>(v);
}
// dq from the splits' parts, in order, and delta: DP threads a row.
template <int P, int DP> __global__ __launch_bounds__(256) void k_cross_sum_dq(const CrossArgs A, int64_t count) {
    using T = typename GatedIO<P>::T;
    const int64_t bhr = ((int64_t)blockIdx.x * 256 + threadIdx.x) / DP;
    const int c = threadIdx.x % DP, R = A.rows();
    if (bhr >= count || c >= A.D) return;
    const float *const p = A.part + bhr * (2 * DP + 4);
    const int64_t step = count * (2 * DP + 4);
    float v = 0.f, m = 0.f, off = 0.f, sum = 0.f;
#pragma unroll 8
    for (int s = 0; s < A.splits; ++s) {
        v += p[s * step + c];
        if constexpr (P == 1) {
            m += p[s * step + DP + c];
            off += p[s * step + 2 * DP];
            sum += p[s * step + 2 * DP + 1];
        }
    }
    const int b = (int)(bhr / R / A.heads()), hk = (int)(bhr / R % A.heads()), r = (int)(bhr % R);
    cross_to((T *)A.to, A, b, hk, r)[c] = from_float<T>(A.scale * (v - sum * m));
    if (P == 1 && c == 0) *cross_stat(A.delta, A, b, hk, r) += off;
}

}  // namespace ts3
