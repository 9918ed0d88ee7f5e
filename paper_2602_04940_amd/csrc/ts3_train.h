// Host side of the training operators: the gated feed-forward (ts3_gated.h), the residual
// LayerNorm (ts3_norm.h) and the clipping by the global norm (ts3_clip.h).  Included once, at
// the end of ts3.hip, for its error helpers.
#pragma once
#include "ts3_clip.h"
#include "ts3_gated.h"
#include "ts3_gated_rules.h"
#include "ts3_norm.h"

struct ts3_gated {
    ts3_gated_desc desc{};
    int32_t P = 1, nchunk = 0;   // operand parts; chunks of 32 hidden units
    bool loaded = false;
    unsigned char *ops = nullptr;  // GatedOps
    float *bd = nullptr;           // [CP]
    float *part = nullptr;         // sums of split outputs, a sheet of PTS x CP per workgroup
    Workspace store;               // da, du, h of a tile
    Workspace wpart;               // sums of the weight gradients' splits
    Workspace bpart;               // and of the biases'
    int64_t bytes = 0;
};
struct ts3_norm {
    ts3_norm_desc desc{};
    float *part = nullptr;  // [NORM_BLOCKS][2][C]
};
struct ts3_clip {
    double *sums = nullptr;  // [CLIP_PIECES + CLIP_TENSORS]
};

namespace {

// Calls fn(P, CP) as integral constants for the operand parts and the padded width.
template <typename F> auto gated_dispatch(const ts3_gated *h, F fn) {
    auto with = [&](auto p) {
        switch ((h->desc.C + 63) / 64) {
            case 1: return fn(p, ic<64>{});
            case 2: return fn(p, ic<128>{});
            case 3: return fn(p, ic<192>{});
            default: return fn(p, ic<256>{});
        }
    };
    return h->P == 1 ? with(ic<1>{}) : with(ic<3>{});
}

constexpr int64_t GATED_TILE_MAX = 1 << 24;

// Bytes that a call reads or writes.
struct Range {
    const void *p;
    int64_t bytes;
};
bool overlap(const Range &a, const Range &b) {
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    return a.p && b.p && pa < pb + (uintptr_t)b.bytes && pb < pa + (uintptr_t)a.bytes;
}
// Overlaps that are not the same array.
bool overlap_in_part(const Range &a, const Range &b) { return a.p != b.p && overlap(a, b); }
bool aligned16(std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if ((uintptr_t)p & 15) return false;
    return true;
}

constexpr int NORM_BLOCKS = 1024;

// Calls run(LG, K): lanes per row and 16-byte pieces per lane.
template <typename T, typename F> void norm_dispatch(int C, F run) {
    const int pieces = C / Piece<T>::V;
    if constexpr (sizeof(T) == 4)
        if (pieces > 64) return run(ic<64>{}, ic<2>{});
    if (pieces > 32) return run(ic<64>{}, ic<1>{});
    if (pieces > 16) return run(ic<32>{}, ic<1>{});
    if (pieces > 8) return run(ic<16>{}, ic<1>{});
    if (pieces > 4) return run(ic<8>{}, ic<1>{});
    if (pieces > 2) return run(ic<4>{}, ic<1>{});
    run(ic<2>{}, ic<1>{});
}

template <typename T> void launch_norm_fwd(const ts3_norm_desc &d, const void *x, const void *r, const float *gamma,
                                           const float *beta, int64_t n, void *y, void *out, hipStream_t st) {
    auto run = [&](auto lg, auto k) {
        constexpr int LG = decltype(lg)::value, K = decltype(k)::value;
        const int64_t rows = 4 * (64 / LG);
        const unsigned grid = (unsigned)std::min<int64_t>((n + rows - 1) / rows, (int64_t)16 * device_cu_count());
        hipLaunchKernelGGL((k_norm_fwd<T, LG, K>), dim3(grid), dim3(256), 0, st, (const T *)x, (const T *)r, gamma, beta,
                           n, d.C, d.eps, (T *)y, (T *)out);
    };
    norm_dispatch<T>(d.C, run);
}

template <typename T> int launch_norm_bwd(const ts3_norm_desc &d, const void *y, const void *g, const void *r,
                                          const float *gamma, int64_t n, void *dx, float *part, hipStream_t st) {
    int blocks = 0;
    auto run = [&](auto lg, auto k) {
        constexpr int LG = decltype(lg)::value, K = decltype(k)::value;
        const int64_t rows = 4 * (64 / LG);
        blocks = (int)std::min<int64_t>((n + rows - 1) / rows, NORM_BLOCKS);
        if (blocks)
            hipLaunchKernelGGL((k_norm_bwd<T, LG, K>), dim3(blocks), dim3(256), 0, st, (const T *)y, (const T *)g,
                               (const T *)r, gamma, n, d.C, d.eps, (T *)dx, part);
    };
    norm_dispatch<T>(d.C, run);
    return blocks;
}

constexpr int CLIP_TENSORS = 16384, CLIP_PIECES = 16384;
constexpr int64_t CLIP_PIECE = 8192;  // least elements of a piece

// Tensors of one type that lie one after another, source and destination alike.
struct ClipRun {
    const char *src;
    char *dst;
    int64_t n;
    int32_t dtype;
    int64_t bytes() const { return n * (dtype == TS3_BF16 ? 2 : 4); }
};

// Whether a written array shares a byte with another read or written one: such elements would be scaled
// twice, or not at all, by what the workgroups come to first.
bool clip_overlaps(const std::vector<ClipRun> &runs, bool writes_in_place) {
    struct Access {
        uintptr_t a, e;
        bool write;
    };
    std::vector<Access> acc;
    acc.reserve(2 * runs.size());
    auto add = [&](const void *p, const ClipRun &r, bool write) {
        acc.push_back(Access{(uintptr_t)p, (uintptr_t)p + (uintptr_t)r.bytes(), write});
    };
    for (const ClipRun &r : runs) {
        if (r.src != r.dst) add(r.src, r, false);
        add(r.dst, r, r.src != r.dst || writes_in_place);
    }
    auto before = [](const Access &x, const Access &y) { return x.a < y.a; };
    if (!std::is_sorted(acc.begin(), acc.end(), before)) std::sort(acc.begin(), acc.end(), before);
    uintptr_t any = 0, written = 0;  // ends of what came so far
    for (const Access &x : acc) {
        if (x.a < (x.write ? any : written)) return true;
        any = std::max(any, x.e);
        if (x.write) written = std::max(written, x.e);
    }
    return false;
}

}  // namespace

extern "C" {

ts3_status ts3_gated_create(const ts3_gated_desc *desc, ts3_gated **out) {
    if (!desc || !out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    if (desc->C <= 0 || desc->F <= 0)
        return fail(TS3_ERR_INVALID_ARG, "C and F must be positive (got %d, %d)", desc->C, desc->F);
    if (desc->activation != TS3_SILU && desc->activation != TS3_GELU)
        return fail(TS3_ERR_INVALID_ARG, "activation %d is not TS3_SILU or TS3_GELU", desc->activation);
    if (desc->io_dtype != TS3_FP32 && desc->io_dtype != TS3_BF16)
        return fail(TS3_ERR_INVALID_ARG, "io_dtype %d is not TS3_FP32 or TS3_BF16", desc->io_dtype);
    if (desc->C % 16 || desc->C > 256 || desc->F > 65536)
        return fail(TS3_ERR_UNSUPPORTED, "no kernel for C=%d, F=%d (C a multiple of 16 up to 256, F up to 65536)",
                    desc->C, desc->F);
    ts3_gated *h = new (std::nothrow) ts3_gated();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->desc = *desc;
    h->P = desc->io_dtype == TS3_BF16 ? 1 : 3;
    h->nchunk = (desc->F + 31) / 32;
    ts3_status s = gated_dispatch(h, [&](auto p, auto cp) {
        constexpr int P = decltype(p)::value, CP = decltype(cp)::value;
        const int64_t ops = (int64_t)h->nchunk * GatedOps<P, CP, GatedShape<P, CP>::MT>::CHUNK;
        // a round of workgroups of the kernel with the largest blocks of points
        const int64_t part = (int64_t)device_cu_count() * std::max(GatedShape<P, CP>::PTS, GatedWide<P, CP>::PTS) * CP * 4;
        ts3_status st = device_alloc((void **)&h->ops, ops);
        if (st == TS3_OK) st = device_alloc((void **)&h->bd, CP * 4);
        if (st == TS3_OK) st = device_alloc((void **)&h->part, part);
        h->bytes = ops + CP * 4 + part;
        return st;
    });
    if (s != TS3_OK) {
        ts3_gated_free(h);
        return s;
    }
    *out = h;
    return TS3_OK;
}

ts3_status ts3_gated_free(ts3_gated *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    for (void *p : {(void *)h->ops, (void *)h->bd, (void *)h->part}) (void)hipFree(p);
    for (Workspace *w : {&h->store, &h->wpart, &h->bpart}) w->free();
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_gated_bytes(const ts3_gated *h, int64_t *bytes) {
    if (!h || !bytes) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *bytes = h->bytes;
    return TS3_OK;
}

ts3_status ts3_gated_load(ts3_gated *h, const ts3_gated_weights *w, void *stream) {
    if (!h || !w) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (!w->Wg || !w->Wu || !w->Wd) return fail(TS3_ERR_INVALID_ARG, "Wg, Wu or Wd is NULL");
    const uintptr_t type = h->P == 1 ? 1 : 3;
    for (const void *p : {w->Wg, w->bg, w->Wu, w->bu, w->Wd, w->bd})
        if ((uintptr_t)p & type) return fail(TS3_ERR_INVALID_ARG, "a weight is not aligned to its type");
    gated_dispatch(h, [&](auto p, auto cp) {
        constexpr int P = decltype(p)::value, CP = decltype(cp)::value;
        using T = typename GatedIO<P>::T;
        constexpr int FRAGS = 6 * CP * 64 / 1024;  // of a chunk; a wave each
        hipLaunchKernelGGL((k_gated_load<P, CP, GatedShape<P, CP>::MT>), dim3(h->nchunk, FRAGS / 4), dim3(256), 0,
                           (hipStream_t)stream, (const T *)w->Wg, (const T *)w->bg, (const T *)w->Wu, (const T *)w->bu,
                           (const T *)w->Wd, (const T *)w->bd, h->desc.C, h->desc.F, h->ops, h->bd);
    });
    LAUNCH_CHECK("gated operands");
    h->loaded = true;
    return TS3_OK;
}

ts3_status ts3_gated_forward(ts3_gated *h, const void *x, int64_t n, void *out, void *stream) {
    if (!h) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 required");
    if (!h->loaded) return fail(TS3_ERR_BAD_STATE, "no weights loaded");
    if (n == 0) return TS3_OK;
    if (!x || !out || !aligned16({x, out}))
        return fail(TS3_ERR_INVALID_ARG, "x and out must be 16-byte aligned device pointers");
    const int64_t rows = n * h->desc.C * (h->P == 1 ? 2 : 4);
    if (overlap_in_part({x, rows}, {out, rows})) return fail(TS3_ERR_INVALID_ARG, "out overlaps x in part");
    return gated_dispatch(h, [&](auto p, auto cp) -> ts3_status {
        constexpr int P = decltype(p)::value, CP = decltype(cp)::value;
        using T = typename GatedIO<P>::T;
        constexpr int PTS = GatedShape<P, CP>::PTS;
        const int C = h->desc.C, cus = device_cu_count();
        hipStream_t st = (hipStream_t)stream;
        for (int64_t p0 = 0; p0 < n; p0 += MAX_WGS * PTS) {
            const int64_t m = std::min<int64_t>(n - p0, MAX_WGS * PTS), nb = (m + PTS - 1) / PTS;
            const int S = gated_splits(m, nb, h->nchunk, P, CP, cus), per = (h->nchunk + S - 1) / S;
            T *const to = (T *)out + p0 * C;
            const bool silu = h->desc.activation == TS3_SILU;
            auto launch = [&](auto hw) {
                constexpr int HW = decltype(hw)::value;
                const auto kernel = silu ? &k_gated_fwd<P, CP, GATED_SILU, HW> : &k_gated_fwd<P, CP, GATED_GELU, HW>;
                hipLaunchKernelGGL(kernel, dim3((unsigned)(nb * S)), dim3(256 * HW), 0, st, (const T *)x + p0 * C, m, C,
                                   h->ops, h->nchunk, per, S, h->bd, to, h->part);
            };
            if constexpr (GatedShape<P, CP>::OCC == 2)
                if (gated_halves<P, CP>(nb * S, per, cus) == 2) launch(ic<2>{});
                else launch(ic<1>{});
            else launch(ic<1>{});
            LAUNCH_CHECK("gated forward");
            if (S > 1) {
                using Sh = GatedShape<P, CP>;
                hipLaunchKernelGGL((k_gated_join<P, CP, Sh::MT, Sh::NP>), dim3((unsigned)(nb * (Sh::PTS / 4 * CP / 256))),
                                   dim3(256), 0, st, h->part, m, C, S, (int)nb, h->bd, to);
                LAUNCH_CHECK("gated join");
            }
        }
        return TS3_OK;
    });
}

ts3_status ts3_gated_backward(ts3_gated *h, const void *x, const void *g, int64_t n, int64_t tile, void *dx,
                              const ts3_gated_grads *gr, void *stream) {
    if (!h || !gr) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0 || tile <= 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 and tile > 0 required");
    if (!h->loaded) return fail(TS3_ERR_BAD_STATE, "no weights loaded");
    if (!gr->dWg || !gr->dbg || !gr->dWu || !gr->dbu || !gr->dWd || !gr->dbd)
        return fail(TS3_ERR_INVALID_ARG, "a gradient pointer is NULL");
    const uintptr_t type = h->P == 1 ? 1 : 3;
    for (const void *p : {gr->dWg, gr->dbg, gr->dWu, gr->dbu, gr->dWd, gr->dbd})
        if ((uintptr_t)p & type) return fail(TS3_ERR_INVALID_ARG, "a gradient is not aligned to its type");
    if (n > 0 && (!x || !g || !dx || !aligned16({x, g, dx})))
        return fail(TS3_ERR_INVALID_ARG, "x, g and dx must be 16-byte aligned device pointers");
    // dx is written while other points' x and g are read, the gradients at the end.
    const int64_t e = h->P == 1 ? 2 : 4, C = h->desc.C, F = h->desc.F;
    const Range dxr{n > 0 ? dx : nullptr, n * C * e};
    if (overlap(dxr, {x, dxr.bytes}) || overlap(dxr, {g, dxr.bytes}))
        return fail(TS3_ERR_INVALID_ARG, "dx may not overlap x or g (the weight gradients read them after dx is written)");
    const Range outs[] = {dxr, {gr->dWg, C * F * e}, {gr->dWu, C * F * e}, {gr->dWd, C * F * e}, {gr->dbg, F * e},
                          {gr->dbu, F * e}, {gr->dbd, C * e}};
    for (const Range &a : outs)
        for (const Range &b : outs)
            if (&a < &b && overlap(a, b)) return fail(TS3_ERR_INVALID_ARG, "dx and the gradients may not overlap one another");
    return gated_dispatch(h, [&](auto p, auto cp) -> ts3_status {
        constexpr int P = decltype(p)::value, CP = decltype(cp)::value;
        using T = typename GatedIO<P>::T;
        constexpr bool WIDE = GatedWide<P, CP>::USE;
        constexpr int PTS = WIDE ? GatedWide<P, CP>::PTS : GatedShapeX<P, CP>::PTS;
        const int C = h->desc.C, F = h->desc.F, nchunk = h->nchunk, FP = nchunk * 32, BW = std::max(FP, CP), cus = device_cu_count();
        const int W = gated_dw_waves<P, CP>(nchunk), HB = GatedDw<P, CP, 4>::HB / 4 * W, nhb = (FP + HB - 1) / HB;
        hipStream_t st = (hipStream_t)stream;
        // k_gated_load leaves zeros after the 64 biases of a chunk's block.
        const unsigned char *const zeros = h->ops + GatedOps<P, CP, GatedShape<P, CP>::MT>::BIAS + 256;
        const int64_t step = std::min(std::min(tile, GATED_TILE_MAX), std::max<int64_t>(n, 1));
        const int SP = n > 0 ? gated_point_splits<P, CP>(nchunk, step, cus) : 0;
        if (n > 0) {
            // da, du and h of a tile, and in bfloat16 the sums of da and du over 32 points each
            const int64_t rows = (step + PTS - 1) / PTS * PTS;
            const int64_t need = rows * 3 * FP * (int64_t)sizeof(T) + (P == 1 ? rows / 32 * 2 * FP * 4 : 0);
            const int most = gated_point_splits<P, CP>(nchunk, GATED_TILE_MAX, cus);
            const int64_t wbytes = (int64_t)most * 3 * FP * CP * 4, bbytes = (int64_t)most * 3 * BW * 4;
            ts3_status s = h->wpart.reserve(wbytes, st, h->bytes);
            if (s == TS3_OK) s = h->bpart.reserve(bbytes, st, h->bytes);
            if (s == TS3_OK) s = h->store.reserve(need, st, h->bytes);
            if (s != TS3_OK) return s;
        }
        T *const store = (T *)h->store.p;
        float *const wpart = (float *)h->wpart.p, *const bpart = (float *)h->bpart.p;
        for (int64_t t0 = 0; t0 < n; t0 += step) {
            const int64_t m = std::min(step, n - t0), nb = (m + PTS - 1) / PTS, tp = nb * PTS;
            const int S = gated_splits(m, nb, nchunk, P, CP, cus), per = (nchunk + S - 1) / S;
            const T *const xt = (const T *)x + t0 * C, *const gt = (const T *)g + t0 * C;
            T *const dxt = (T *)dx + t0 * C;
            const bool silu = h->desc.activation == TS3_SILU;
            float *const cols = P == 1 ? (float *)(store + tp * 3 * FP) : nullptr;
            if constexpr (WIDE) {
                const dim3 grid((unsigned)(nb * S));
                if constexpr (P == 1) {
                    const auto slopes = silu ? &k_gated_slopes<CP, GATED_SILU> : &k_gated_slopes<CP, GATED_GELU>;
                    hipLaunchKernelGGL(slopes, grid, dim3(256), 0, st, xt, gt, m, C, h->ops, nchunk, per, S, tp,
                                       store, cols);
                } else {
                    const auto slopes = silu ? &k_gated_slopes3<CP, GATED_SILU> : &k_gated_slopes3<CP, GATED_GELU>;
                    hipLaunchKernelGGL(slopes, grid, dim3(256), 0, st, xt, gt, m, C, h->ops, nchunk, per, S, tp,
                                       store);
                }
                LAUNCH_CHECK("gated slopes");
                hipLaunchKernelGGL((k_gated_dx_wide<P, CP>), grid, dim3(256), 0, st, m, C, h->ops, nchunk,
                                   per, S, tp, (const T *)store, dxt, h->part);
            } else {
                const auto kernel = silu ? &k_gated_dx<P, CP, GATED_SILU> : &k_gated_dx<P, CP, GATED_GELU>;
                hipLaunchKernelGGL(kernel, dim3((unsigned)(nb * S)), dim3(256), 0, st, xt, gt, m, C, h->ops, nchunk, per,
                                   S, tp, store, cols, dxt, h->part);
            }
            LAUNCH_CHECK("gated dx");
            if (S > 1) {
                hipLaunchKernelGGL((k_gated_join<P, CP, GatedShape<P, CP>::MT, 1>), dim3((unsigned)(nb * (PTS / 4 * CP / 256))),
                                   dim3(256), 0, st, h->part, m, C, S, (int)nb, (const float *)nullptr, dxt);
                LAUNCH_CHECK("gated join");
            }
            const int64_t pps = ((tp + SP - 1) / SP + 31) / 32 * 32;
            const GatedDwArgs<P, CP> a{xt, gt, store, cols, m, tp, pps, C, nchunk, nhb, t0 == 0, zeros, wpart, bpart};
            auto dw = &k_gated_dw<P, CP, 4>;
            if constexpr (GatedDwWide<P, CP>::USE8)
                if (W == 8) dw = &k_gated_dw<P, CP, 8>;
            hipLaunchKernelGGL(dw, dim3((unsigned)(3 * nhb * SP)), dim3(64 * W), 0, st, a);
            LAUNCH_CHECK("gated weight gradients");
        }
        hipLaunchKernelGGL((k_gated_grads<P, CP>), dim3(nchunk, (C + 31) / 32, 3), dim3(1024), 0, st, wpart, bpart,
                           SP, nchunk, C, F, (T *)gr->dWg, (T *)gr->dWu, (T *)gr->dWd, (T *)gr->dbg, (T *)gr->dbu,
                           (T *)gr->dbd);
        LAUNCH_CHECK("gated gradient sums");
        return TS3_OK;
    });
}

ts3_status ts3_norm_create(const ts3_norm_desc *desc, ts3_norm **out) {
    if (!desc || !out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    if (desc->C <= 0) return fail(TS3_ERR_INVALID_ARG, "C must be positive (got %d)", desc->C);
    if (desc->io_dtype != TS3_FP32 && desc->io_dtype != TS3_BF16)
        return fail(TS3_ERR_INVALID_ARG, "io_dtype %d is not TS3_FP32 or TS3_BF16", desc->io_dtype);
    if (!(desc->eps >= 0.f) || std::isinf(desc->eps)) return fail(TS3_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (desc->C % 16 || desc->C > 512)
        return fail(TS3_ERR_UNSUPPORTED, "no kernel for C=%d (a multiple of 16 up to 512)", desc->C);
    ts3_norm *h = new (std::nothrow) ts3_norm();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->desc = *desc;
    ts3_status s = device_alloc((void **)&h->part, (int64_t)NORM_BLOCKS * 2 * desc->C * 4);
    if (s != TS3_OK) {
        delete h;
        return s;
    }
    *out = h;
    return TS3_OK;
}

ts3_status ts3_norm_free(ts3_norm *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    (void)hipFree(h->part);
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_norm_forward(ts3_norm *h, const void *x, const void *r, const float *gamma, const float *beta, int64_t n,
                            void *y, void *out, void *stream) {
    if (!h) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 required");
    if (n == 0) return TS3_OK;
    if (!x || !gamma || !beta || !out) return fail(TS3_ERR_INVALID_ARG, "x, gamma, beta or out is NULL");
    if (!aligned16({x, r, y, out})) return fail(TS3_ERR_INVALID_ARG, "x, r, y and out must be 16-byte aligned");
    const int64_t rows = n * h->desc.C * (h->desc.io_dtype == TS3_BF16 ? 2 : 4), row = (int64_t)h->desc.C * 4;
    const Range yr{y, rows}, outr{out, rows};
    for (const void *p : {x, r, (const void *)y})
        if (overlap(outr, {p, rows})) return fail(TS3_ERR_INVALID_ARG, "out may not overlap x, r or y");
    for (const void *p : {x, r})
        if (overlap_in_part(yr, {p, rows})) return fail(TS3_ERR_INVALID_ARG, "y overlaps x or r in part");
    for (const float *p : {gamma, beta})
        if (overlap(outr, {p, row}) || overlap(yr, {p, row}))
            return fail(TS3_ERR_INVALID_ARG, "y and out may not overlap gamma or beta");
    const auto launch = h->desc.io_dtype == TS3_BF16 ? &launch_norm_fwd<bf16_t> : &launch_norm_fwd<float>;
    launch(h->desc, x, r, gamma, beta, n, y, out, (hipStream_t)stream);
    LAUNCH_CHECK("norm forward");
    return TS3_OK;
}

ts3_status ts3_norm_backward(ts3_norm *h, const void *y, const void *g, const void *gr, const float *gamma, int64_t n,
                             void *dx, float *dgamma, float *dbeta, void *stream) {
    if (!h) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 required");
    if (!dgamma || !dbeta) return fail(TS3_ERR_INVALID_ARG, "dgamma or dbeta is NULL");
    if (n > 0 && (!y || !g || !gamma || !dx)) return fail(TS3_ERR_INVALID_ARG, "y, g, gamma or dx is NULL");
    if (!aligned16({y, g, gr, dx})) return fail(TS3_ERR_INVALID_ARG, "y, g, gr and dx must be 16-byte aligned");
    const int64_t rows = n * h->desc.C * (h->desc.io_dtype == TS3_BF16 ? 2 : 4), row = (int64_t)h->desc.C * 4;
    const Range dxr{n > 0 ? dx : nullptr, rows};
    if (overlap(dxr, {y, rows})) return fail(TS3_ERR_INVALID_ARG, "dx may not overlap y");
    if (overlap_in_part(dxr, {g, rows}) || overlap_in_part(dxr, {gr, rows}))
        return fail(TS3_ERR_INVALID_ARG, "dx overlaps g or gr in part");
    if (overlap(dxr, {gamma, row}) || overlap(dxr, {dgamma, row}) || overlap(dxr, {dbeta, row}) ||
        overlap({dgamma, row}, {dbeta, row}))
        return fail(TS3_ERR_INVALID_ARG, "dx may not overlap gamma, dgamma or dbeta, nor these two each other");
    const auto launch = h->desc.io_dtype == TS3_BF16 ? &launch_norm_bwd<bf16_t> : &launch_norm_bwd<float>;
    const int blocks = launch(h->desc, y, g, gr, gamma, n, dx, h->part, (hipStream_t)stream);
    LAUNCH_CHECK("norm backward");
    hipLaunchKernelGGL(k_norm_join, dim3(2 * h->desc.C / 16), dim3(256), 0, (hipStream_t)stream, h->part, blocks,
                       h->desc.C, dgamma, dbeta);
    LAUNCH_CHECK("norm column sums");
    return TS3_OK;
}

ts3_status ts3_clip_create(ts3_clip **out) {
    if (!out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    ts3_clip *h = new (std::nothrow) ts3_clip();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    ts3_status s = device_alloc((void **)&h->sums, (int64_t)(CLIP_PIECES + CLIP_TENSORS) * 8);
    if (s != TS3_OK) {
        delete h;
        return s;
    }
    *out = h;
    return TS3_OK;
}

ts3_status ts3_clip_free(ts3_clip *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    (void)hipFree(h->sums);
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_clip_gradients(ts3_clip *h, const ts3_clip_tensor *tensors, int32_t count, float max_norm, float *norm,
                              void *stream) {
    if (!h || (!tensors && count > 0)) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (count < 0 || count > CLIP_TENSORS)
        return fail(TS3_ERR_INVALID_ARG, "0 <= count <= %d required (got %d)", CLIP_TENSORS, count);
    if (!(max_norm > 0.f)) return fail(TS3_ERR_INVALID_ARG, "max_norm must be > 0");
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        const ts3_clip_tensor &t = tensors[i];
        if (t.dtype != TS3_FP32 && t.dtype != TS3_BF16)
            return fail(TS3_ERR_INVALID_ARG, "tensor %d: dtype %d is not TS3_FP32 or TS3_BF16", i, t.dtype);
        if (t.n < 0 || t.n > (int64_t(1) << 48)) return fail(TS3_ERR_INVALID_ARG, "tensor %d: 0 <= n <= 2^48 required", i);
        if (t.n == 0) continue;
        const uintptr_t type = t.dtype == TS3_BF16 ? 1 : 3;
        if (!t.src || !t.dst || (((uintptr_t)t.src | (uintptr_t)t.dst) & type))
            return fail(TS3_ERR_INVALID_ARG, "tensor %d: a pointer is NULL or not aligned to its type", i);
        total += t.n;
    }
    hipStream_t st = (hipStream_t)stream;
    try {
        std::vector<ClipRun> runs;
        int last[2] = {-1, -1};  // the newest run of each type
        for (int32_t i = 0; i < count; ++i) {
            const ts3_clip_tensor &t = tensors[i];
            if (t.n == 0) continue;
            const int64_t e = t.dtype == TS3_BF16 ? 2 : 4;
            if (last[t.dtype] >= 0) {
                ClipRun &r = runs[(size_t)last[t.dtype]];
                if (r.src + r.n * e == t.src && r.dst + r.n * e == t.dst) {
                    r.n += t.n;
                    continue;
                }
            }
            last[t.dtype] = (int)runs.size();
            runs.push_back(ClipRun{(const char *)t.src, (char *)t.dst, t.n, t.dtype});
        }
        if (clip_overlaps(runs, !std::isinf(max_norm)))
            return fail(TS3_ERR_INVALID_ARG, "a destination overlaps another tensor (the same one twice, or views of one array)");
        // A multiple of 8 elements, so that pieces keep their tensor's alignment.
        const int64_t piece = std::max(CLIP_PIECE, (total + CLIP_PIECES - 1) / CLIP_PIECES / 8 * 8 + 8);
        std::vector<ClipBatch> batches;
        int pieces = 0;
        for (size_t i = 0; i < runs.size(); ++i) {
            if (i % CLIP_BATCH == 0) batches.emplace_back();
            ClipBatch &b = batches.back();
            const int k = b.count++;
            b.src[k] = runs[i].src;
            b.dst[k] = runs[i].dst;
            b.n[k] = runs[i].n * 2 + (runs[i].dtype == TS3_BF16);
            const int np = (int)((runs[i].n + piece - 1) / piece);
            b.first[k + 1] = b.first[k] + np;
            pieces += np;
        }
        int base = 0;
        for (const ClipBatch &b : batches) {
            const int np = b.first[b.count];
            hipLaunchKernelGGL(k_clip_sums, dim3(np), dim3(256), 0, st, b, piece, base, h->sums);
            LAUNCH_CHECK("clip sums");
            base += np;
        }
        if (batches.empty()) batches.emplace_back();  // the norm of nothing
        for (const ClipBatch &b : batches) {
            hipLaunchKernelGGL(k_clip_scale, dim3(std::max(1, b.first[b.count])), dim3(256), 0, st, b, piece, pieces,
                               max_norm, h->sums, &b == &batches.front() ? norm : nullptr);
            LAUNCH_CHECK("clip scale");
        }
    } catch (const std::bad_alloc &) {
        return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    }
    return TS3_OK;
}

}  // extern "C"
