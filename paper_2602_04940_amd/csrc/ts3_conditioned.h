// Host side of the operators of a conditioned block: attention to an encoder's states (ts3_cross.h), the
// norms around a block (ts3_sandwich.h) and orthogonalised updates (ts3_orth.h); how their calls are
// cut is in ts3_cross_rules.h and ts3_orth_rules.h.  Included once, after
// ts3_train.h, for its helpers and those of ts3.hip.
#pragma once
#include "ts3_cross_rules.h"
#include "ts3_orth.h"
#include "ts3_sandwich.h"

struct ts3_cross {
    ts3_cross_desc desc{};
    Workspace part;   // parts of split loops
    Workspace delta;  // the backward's g.out
    bool lds = false;  // whether the kernels that fill a compute unit's LDS may
    int64_t bytes = 0;
};
struct ts3_sandwich {
    ts3_sandwich_desc desc{};
    float *part = nullptr;  // [NORM_BLOCKS][SANDWICH_SUMS][C]
};
struct ts3_orth {
    ts3_orth_desc desc{};
    Workspace work;
    int64_t bytes = 0;
};

namespace {

// Calls run(LG, K, FULL): lanes per row and pieces of V values per lane, and whether these are C.
template <int V, typename F> void sandwich_dispatch(int C, F run) {
    auto with = [&](auto lg, auto k) {
        if (C == decltype(lg)::value * decltype(k)::value * V) run(lg, k, std::true_type{});
        else run(lg, k, std::false_type{});
    };
    const int pieces = C / V;
    if constexpr (V == 4)
        if (pieces > 64) return with(ic<64>{}, ic<2>{});
    if (pieces > 32) return with(ic<64>{}, ic<1>{});
    if (pieces > 16) return with(ic<32>{}, ic<1>{});
    if (pieces > 8) return with(ic<16>{}, ic<1>{});
    if (pieces > 4) return with(ic<8>{}, ic<1>{});
    if (pieces > 2) return with(ic<4>{}, ic<1>{});
    with(ic<2>{}, ic<1>{});
}

// Calls fn(P, DP) for the operand parts and the padded head width.
template <typename F> auto cross_dispatch(const ts3_cross_desc &d, F fn) {
    auto with = [&](auto p) {
        if (d.D <= 16) return fn(p, ic<16>{});
        if (d.D <= 32) return fn(p, ic<32>{});
        if (d.D <= 64) return fn(p, ic<64>{});
        return fn(p, ic<128>{});
    };
    return d.io_dtype == TS3_BF16 ? with(ic<1>{}) : with(ic<3>{});
}

// Elements from a view's first to behind its last; 0 where a side is.
int64_t view_extent(const ts3_view &v, int64_t B, int64_t rows, int64_t heads, int64_t D) {
    if (B <= 0 || rows <= 0) return 0;
    return (B - 1) * v.batch + (rows - 1) * v.row + (heads - 1) * v.head + D;
}
constexpr int64_t CROSS_STRIDE_MAX = int64_t(1) << 40;

ts3_status cross_check_view(const char *name, const ts3_view &v, int64_t extent, int64_t size) {
    if (extent == 0) return TS3_OK;
    if (!v.p || ((uintptr_t)v.p & 15)) return fail(TS3_ERR_INVALID_ARG, "%s must be a 16-byte aligned device pointer", name);
    for (int64_t s : {v.batch, v.row, v.head})
        if (s < 0 || s > CROSS_STRIDE_MAX || s * size % 16)
            return fail(TS3_ERR_INVALID_ARG, "%s: strides must be multiples of 16 bytes, from 0 to 2^40 elements", name);
    return TS3_OK;
}

// Checks what forward and backward share, and fills the kernels' arguments.
ts3_status cross_inputs(const ts3_cross *h, const ts3_cross_inputs &in, CrossArgs &A) {
    if (in.B < 0 || in.N < 0 || in.S < 0) return fail(TS3_ERR_INVALID_ARG, "B, N and S must be >= 0");
    const int64_t B = in.B, N = in.N, S = in.S, H = h->desc.H, HK = h->desc.Hkv, D = h->desc.D;
    if (!cross_fits({B, HK, N * (H / HK), S, false}))
        return fail(TS3_ERR_UNSUPPORTED, "no launch for B=%lld, N=%lld, S=%lld", (long long)B, (long long)N, (long long)S);
    const int64_t size = h->desc.io_dtype == TS3_BF16 ? 2 : 4;
    for (const ts3_view *v : {&in.q, &in.k, &in.v}) {
        const bool q = v == &in.q;
        ts3_status s = cross_check_view(q ? "q" : v == &in.k ? "k" : "v", *v, view_extent(*v, B, q ? N : S, q ? H : HK, D), size);
        if (s != TS3_OK) return s;
    }
    if ((uintptr_t)in.lengths & 3) return fail(TS3_ERR_INVALID_ARG, "lengths is not aligned to its type");
    auto view = [](const ts3_view &v) { return CrossView{v.p, v.batch, v.row, v.head}; };
    A = CrossArgs{};
    A.q = view(in.q), A.k = view(in.k), A.v = view(in.v);
    A.lengths = in.lengths;
    A.mask = in.mask;
    A.B = in.B, A.N = in.N, A.S = in.S, A.H = h->desc.H, A.G = h->desc.H / h->desc.Hkv, A.D = h->desc.D;
    A.scale = h->desc.scale > 0.f ? h->desc.scale : (float)(1.0 / std::sqrt((double)h->desc.D));
    A.by_heads = CrossDiv((uint32_t)h->desc.Hkv);
    A.by_G = CrossDiv((uint32_t)A.G);
    return TS3_OK;
}
// Refuses outputs that overlap an input or one another.
ts3_status cross_overlaps(std::initializer_list<Range> ins, std::initializer_list<Range> outs) {
    for (const Range *o = outs.begin(); o != outs.end(); ++o) {
        for (const Range &i : ins)
            if (overlap(*o, i)) return fail(TS3_ERR_INVALID_ARG, "an output overlaps an input");
        for (const Range *p = outs.begin(); p != o; ++p)
            if (overlap(*o, *p)) return fail(TS3_ERR_INVALID_ARG, "outputs overlap one another");
    }
    return TS3_OK;
}
CrossSize cross_size(const CrossArgs &A) { return {A.B, A.H / A.G, (int64_t)A.N * A.G, A.S, A.lengths != nullptr}; }
void cross_cut_by(CrossArgs &A, int64_t blocks, const CrossCut &cut) {
    A.per = (int32_t)cut.per;
    A.splits = (int32_t)cut.splits;
    A.by_splits = CrossDiv((uint32_t)A.splits);
    A.by_blocks = CrossDiv((uint32_t)std::max<int64_t>(blocks, 1));
}

template <int P, int DP> ts3_status cross_allow_lds(ts3_cross *h) {
    if (h->lds) return TS3_OK;
    HIP_TRY(hipFuncSetAttribute((const void *)&k_cross_fwd_all<P, DP>, hipFuncAttributeMaxDynamicSharedMemorySize, ATTN_LDS_MAX));
    HIP_TRY(hipFuncSetAttribute((const void *)&k_cross_dq_all<P, DP>, hipFuncAttributeMaxDynamicSharedMemorySize, ATTN_LDS_MAX));
    h->lds = true;
    return TS3_OK;
}

}  // namespace

extern "C" {

ts3_status ts3_cross_create(const ts3_cross_desc *desc, ts3_cross **out) {
    if (!desc || !out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    if (desc->H <= 0 || desc->Hkv <= 0 || desc->D <= 0)
        return fail(TS3_ERR_INVALID_ARG, "H, Hkv and D must be positive (got %d, %d, %d)", desc->H, desc->Hkv, desc->D);
    if (desc->H % desc->Hkv) return fail(TS3_ERR_INVALID_ARG, "H=%d is not a multiple of Hkv=%d", desc->H, desc->Hkv);
    if (desc->io_dtype != TS3_FP32 && desc->io_dtype != TS3_BF16)
        return fail(TS3_ERR_INVALID_ARG, "io_dtype %d is not TS3_FP32 or TS3_BF16", desc->io_dtype);
    if (!(desc->scale >= 0.f) || std::isinf(desc->scale)) return fail(TS3_ERR_INVALID_ARG, "scale must be finite and >= 0");
    if (desc->D % 16 || desc->D > 128 || desc->H > 1024)
        return fail(TS3_ERR_UNSUPPORTED, "no kernel for H=%d, D=%d (D a multiple of 16 up to 128, H up to 1024)", desc->H, desc->D);
    ts3_cross *h = new (std::nothrow) ts3_cross();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->desc = *desc;
    *out = h;
    return TS3_OK;
}

ts3_status ts3_cross_free(ts3_cross *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    h->part.free();
    h->delta.free();
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_cross_bytes(const ts3_cross *h, int64_t *bytes) {
    if (!h || !bytes) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *bytes = h->bytes;
    return TS3_OK;
}

ts3_status ts3_cross_forward(ts3_cross *h, const ts3_cross_inputs *in, void *out, float *lse, void *stream) {
    if (!h || !in) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    CrossArgs A;
    ts3_status s = cross_inputs(h, *in, A);
    if (s != TS3_OK) return s;
    if (A.B == 0 || A.N == 0) return TS3_OK;
    if (!out || ((uintptr_t)out & 15) || !lse || ((uintptr_t)lse & 3))
        return fail(TS3_ERR_INVALID_ARG, "out must be a 16-byte aligned device pointer, lse one aligned to its type");
    const int64_t e = h->desc.io_dtype == TS3_BF16 ? 2 : 4, rows = (int64_t)A.B * A.N * A.H, HK = h->desc.Hkv;
    s = cross_overlaps({{A.q.p, e * view_extent(in->q, A.B, A.N, A.H, A.D)}, {A.k.p, e * view_extent(in->k, A.B, A.S, HK, A.D)},
                        {A.v.p, e * view_extent(in->v, A.B, A.S, HK, A.D)}, {A.lengths, 4 * (int64_t)A.B},
                        {A.mask, (int64_t)A.B * A.S}},
                       {{out, rows * A.D * e}, {lse, rows * 4}});
    if (s != TS3_OK) return s;
    A.to = out;
    A.lse = lse;
    return cross_dispatch(h->desc, [&](auto p, auto dp) -> ts3_status {
        constexpr int P = decltype(p)::value, DP = decltype(dp)::value;
        const int64_t R = (int64_t)A.N * A.G, bh = (int64_t)A.B * HK;
        hipStream_t st = (hipStream_t)stream;
        const CrossPlan plan = cross_forward_plan<P, DP>(cross_size(A), device_cu_count());
        cross_cut_by(A, plan.blocks, plan.cut);
        const int64_t wgs = bh * plan.blocks * plan.cut.splits;
        using All = CrossAll<P, DP, 16>;
        if constexpr (All::FITS) if (plan.kind == CROSS_ALL) {
            if (ts3_status r = cross_allow_lds<P, DP>(h); r != TS3_OK) return r;
            const unsigned lds = (unsigned)All::bytes(A.S);
            hipLaunchKernelGGL((k_cross_fwd_all<P, DP>), dim3((unsigned)wgs), dim3(64 * All::W), lds, st, A);
            LAUNCH_CHECK("cross attention");
            return TS3_OK;
        }
        if (plan.join != CROSS_WHOLE) {
            ts3_status r = h->part.reserve(A.splits * bh * R * (DP + 4) * 4, st, h->bytes);
            if (r != TS3_OK) return r;
            A.part = (float *)h->part.p;
        }
        if constexpr (DP * P <= 192)
            if (plan.kind == CROSS_ONE) hipLaunchKernelGGL((k_cross_fwd<P, DP, 1>), dim3((unsigned)wgs), dim3(64), 0, st, A);
        if (plan.kind == CROSS_FOUR) hipLaunchKernelGGL((k_cross_fwd<P, DP, 4>), dim3((unsigned)wgs), dim3(256), 0, st, A);
        LAUNCH_CHECK("cross attention");
        const int64_t count = bh * R;
        if (plan.join == CROSS_JOIN_FEW)
            hipLaunchKernelGGL((k_cross_join_few<P, DP>), dim3((unsigned)((count * (DP / 4) + 255) / 256)), dim3(256), 0, st, A, count);
        else if (plan.join == CROSS_JOIN)
            hipLaunchKernelGGL((k_cross_join<P, DP>), dim3((unsigned)count), dim3(256), 0, st, A);
        LAUNCH_CHECK("cross attention join");
        return TS3_OK;
    });
}

ts3_status ts3_cross_backward(ts3_cross *h, const ts3_cross_inputs *in, const void *out, const float *lse, const ts3_view *g,
                              void *dq, void *dk, void *dv, void *stream) {
    if (!h || !in || !g) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    CrossArgs A;
    ts3_status s = cross_inputs(h, *in, A);
    if (s != TS3_OK) return s;
    const int64_t e = h->desc.io_dtype == TS3_BF16 ? 2 : 4, HK = h->desc.Hkv, B = A.B, N = A.N, S = A.S, H = A.H, D = A.D;
    const int64_t rows = B * N * H, states = B * S * HK, gx = view_extent(*g, B, N, H, D);
    s = cross_check_view("g", *g, gx, e);
    if (s != TS3_OK) return s;
    if (rows > 0 && (!out || !lse || !dq || !aligned16({out, dq}) || ((uintptr_t)lse & 3)))
        return fail(TS3_ERR_INVALID_ARG, "out and dq must be 16-byte aligned device pointers, lse one aligned to its type");
    if (states > 0 && (!dk || !dv || !aligned16({dk, dv})))
        return fail(TS3_ERR_INVALID_ARG, "dk and dv must be 16-byte aligned device pointers");
    s = cross_overlaps({{A.q.p, e * view_extent(in->q, B, N, H, D)}, {A.k.p, e * view_extent(in->k, B, S, HK, D)},
                        {A.v.p, e * view_extent(in->v, B, S, HK, D)}, {A.lengths, 4 * B}, {A.mask, B * S}, {g->p, e * gx},
                        {out, rows * D * e}, {lse, rows * 4}},
                       {{dq, rows * D * e}, {dk, states * D * e}, {dv, states * D * e}});
    if (s != TS3_OK) return s;
    if (B == 0) return TS3_OK;
    A.g = CrossView{g->p, g->batch, g->row, g->head};
    A.out = CrossView{out, N * H * D, H * D, D};
    A.lse = const_cast<float *>(lse);
    return cross_dispatch(h->desc, [&](auto p, auto dp) -> ts3_status {
        constexpr int P = decltype(p)::value, DP = decltype(dp)::value;
        const int64_t R = N * A.G, bh = B * HK;
        hipStream_t st = (hipStream_t)stream;
        const CrossBackwardPlan plan = cross_backward_plan<P, DP>(cross_size(A), device_cu_count());
        CrossArgs Q = A, V = A;
        cross_cut_by(Q, plan.qblocks, plan.q);
        cross_cut_by(V, plan.vblocks, plan.v);
        const int64_t qwgs = bh * plan.qblocks * plan.q.splits, vwgs = bh * plan.vblocks * plan.v.splits;
        using All = CrossAll<P, DP, CROSS_DQ_WAVES<DP * P>>;
        const int64_t qn = bh * R * (2 * DP + 4), vn = states * D;
        // one after the other: the parts share their memory
        const int64_t need = std::max(Q.splits > 1 ? Q.splits * qn * 4 : 0, V.splits > 1 ? 2 * V.splits * vn * 4 : 0);
        ts3_status r = h->part.reserve(need, st, h->bytes);
        if (r == TS3_OK) r = h->delta.reserve(rows * 4, st, h->bytes);
        if (r != TS3_OK) return r;
        Q.part = V.part = (float *)h->part.p;
        V.part2 = V.part + V.splits * vn;
        Q.delta = V.delta = (float *)h->delta.p;
        Q.to = dq;
        if (R > 0 && plan.kind == CROSS_ALL) {
            if constexpr (All::FITS) {
                if (ts3_status r = cross_allow_lds<P, DP>(h); r != TS3_OK) return r;
                hipLaunchKernelGGL((k_cross_dq_all<P, DP>), dim3((unsigned)qwgs), dim3(64 * All::W), (unsigned)All::bytes(S), st, Q);
            }
            LAUNCH_CHECK("cross attention dq");
        } else if (R > 0) {
            hipLaunchKernelGGL((k_cross_dq<P, DP>), dim3((unsigned)qwgs), dim3(256), 0, st, Q);
            LAUNCH_CHECK("cross attention dq");
            if (Q.splits > 1) {
                hipLaunchKernelGGL((k_cross_sum_dq<P, DP>), dim3((unsigned)((bh * R * DP + 255) / 256)), dim3(256), 0, st, Q, bh * R);
                LAUNCH_CHECK("cross attention dq sums");
            }
        }
        if (S > 0) {
            V.to = dk;
            V.to2 = dv;
            hipLaunchKernelGGL((k_cross_dkv<P, DP>), dim3((unsigned)vwgs), dim3(256), 0, st, V);
            LAUNCH_CHECK("cross attention dk and dv");
            if (V.splits > 1) {
                hipLaunchKernelGGL((k_cross_sum<typename GatedIO<P>::T>), dim3((unsigned)((vn + 255) / 256), 2), dim3(256), 0, st, V, vn);
                LAUNCH_CHECK("cross attention dk and dv sums");
            }
        }
        return TS3_OK;
    });
}

ts3_status ts3_sandwich_create(const ts3_sandwich_desc *desc, ts3_sandwich **out) {
    if (!desc || !out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    if (desc->C <= 0) return fail(TS3_ERR_INVALID_ARG, "C must be positive (got %d)", desc->C);
    if (desc->io_dtype != TS3_FP32 && desc->io_dtype != TS3_BF16)
        return fail(TS3_ERR_INVALID_ARG, "io_dtype %d is not TS3_FP32 or TS3_BF16", desc->io_dtype);
    if (!(desc->eps >= 0.f) || std::isinf(desc->eps)) return fail(TS3_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (desc->C % 16 || desc->C > 512)
        return fail(TS3_ERR_UNSUPPORTED, "no kernel for C=%d (a multiple of 16 up to 512)", desc->C);
    ts3_sandwich *h = new (std::nothrow) ts3_sandwich();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->desc = *desc;
    ts3_status s = device_alloc((void **)&h->part, (int64_t)NORM_BLOCKS * SANDWICH_SUMS * desc->C * 4);
    if (s != TS3_OK) {
        delete h;
        return s;
    }
    *out = h;
    return TS3_OK;
}

ts3_status ts3_sandwich_free(ts3_sandwich *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    (void)hipFree(h->part);
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_sandwich_forward(ts3_sandwich *h, const void *f, const void *x, const void *gate, const ts3_sandwich_params *p,
                                int64_t n, void *y, void *out, void *stream) {
    if (!h || !p) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 required");
    if (n == 0) return TS3_OK;
    if (!f || !x || !y || !p->gamma_post || !p->beta_post || !p->scale)
        return fail(TS3_ERR_INVALID_ARG, "f, x, y, gamma_post, beta_post or scale is NULL");
    if (out ? !p->gamma_pre || !p->beta_pre : p->gamma_pre || p->beta_pre)
        return fail(TS3_ERR_INVALID_ARG, "out, gamma_pre and beta_pre come together or not at all");
    if (!aligned16({f, x, gate, y, out})) return fail(TS3_ERR_INVALID_ARG, "f, x, gate, y and out must be 16-byte aligned");
    const int64_t rows = n * h->desc.C * (h->desc.io_dtype == TS3_BF16 ? 2 : 4), row = (int64_t)h->desc.C * 4;
    const Range yr{y, rows}, outr{out, rows};
    if (overlap_in_part(yr, {x, rows})) return fail(TS3_ERR_INVALID_ARG, "y overlaps x in part");
    if (overlap(outr, {x, rows}) || overlap(outr, yr)) return fail(TS3_ERR_INVALID_ARG, "out may not overlap x or y");
    for (const void *q : {f, gate})
        if (overlap(yr, {q, rows}) || overlap(outr, {q, rows}))
            return fail(TS3_ERR_INVALID_ARG, "y and out may not overlap f or gate");
    for (const float *q : {p->gamma_post, p->beta_post, p->scale, p->gamma_pre, p->beta_pre})
        if (overlap(yr, {q, row}) || overlap(outr, {q, row}))
            return fail(TS3_ERR_INVALID_ARG, "y and out may not overlap a parameter");
    const SandwichParams sp{p->gamma_post, p->beta_post, p->scale, p->gamma_pre, p->beta_pre};
    auto launch = [&](auto type) {
        using T = decltype(type);
        constexpr int V = Piece<T>::V;
        sandwich_dispatch<V>(h->desc.C, [&](auto lg, auto k, auto full) {
            constexpr int LG = decltype(lg)::value, K = decltype(k)::value;
            const int64_t per = 4 * (64 / LG);
            const unsigned grid = (unsigned)std::min<int64_t>((n + per - 1) / per, (int64_t)8 * device_cu_count());
            hipLaunchKernelGGL((k_sandwich_fwd<T, V, LG, K, decltype(full)::value>), dim3(grid), dim3(256), 0, (hipStream_t)stream, (const T *)f,
                               (const T *)x, (const T *)gate, sp, n, h->desc.C, h->desc.eps, (T *)y, (T *)out);
        });
    };
    if (h->desc.io_dtype == TS3_BF16) launch(bf16_t{});
    else launch(float{});
    LAUNCH_CHECK("sandwich norm forward");
    return TS3_OK;
}

ts3_status ts3_sandwich_backward(ts3_sandwich *h, const void *f, const void *y, const void *gate, const void *gy, const void *gn,
                                 const ts3_sandwich_params *p, int64_t n, void *df, void *dx, void *dgate,
                                 const ts3_sandwich_grads *d, void *stream) {
    if (!h || !p || !d) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (n < 0) return fail(TS3_ERR_INVALID_ARG, "n >= 0 required");
    if (!d->gamma_post || !d->beta_post || !d->scale) return fail(TS3_ERR_INVALID_ARG, "a parameter's gradient is NULL");
    if (n > 0 && (gn ? !d->gamma_pre || !d->beta_pre : d->gamma_pre || d->beta_pre))
        return fail(TS3_ERR_INVALID_ARG, "gn and the gradients of gamma_pre and beta_pre come together or not at all");
    if (n > 0) {
        if (!f || !df || !dx || !p->gamma_post || !p->beta_post || !p->scale)
            return fail(TS3_ERR_INVALID_ARG, "f, df, dx, gamma_post, beta_post or scale is NULL");
        if (!gy && !gn) return fail(TS3_ERR_INVALID_ARG, "gy and gn are both NULL");
        if (gn && (!y || !p->gamma_pre)) return fail(TS3_ERR_INVALID_ARG, "gn needs y and gamma_pre");
        if (!gate != !dgate) return fail(TS3_ERR_INVALID_ARG, "gate and dgate come together or not at all");
    }
    if (!aligned16({f, y, gate, gy, gn, df, dx, dgate}))
        return fail(TS3_ERR_INVALID_ARG, "f, y, gate, gy, gn, df, dx and dgate must be 16-byte aligned");
    const int64_t rows = n * h->desc.C * (h->desc.io_dtype == TS3_BF16 ? 2 : 4), row = (int64_t)h->desc.C * 4;
    const Range outs[] = {{n ? df : nullptr, rows}, {n ? dx : nullptr, rows}, {n ? dgate : nullptr, rows}, {d->gamma_post, row},
                          {d->beta_post, row}, {d->scale, row}, {d->gamma_pre, row}, {d->beta_pre, row}};
    for (const Range &a : outs) {
        for (const Range &b : outs)
            if (&a < &b && overlap(a, b)) return fail(TS3_ERR_INVALID_ARG, "the gradients may not overlap one another");
        if (n > 0)
            for (const void *q : {f, y, gate, gy, gn})
                if (overlap(a, {q, rows}) && !(q == dx && q == gy && a.p == dx))
                    return fail(TS3_ERR_INVALID_ARG, "a gradient overlaps an input (dx may be gy)");
        for (const float *q : {p->gamma_post, p->beta_post, p->scale, p->gamma_pre})
            if (overlap(a, {q, row})) return fail(TS3_ERR_INVALID_ARG, "a gradient overlaps a parameter");
    }
    const SandwichParams sp{p->gamma_post, p->beta_post, p->scale, p->gamma_pre, p->beta_pre};
    int blocks = 0;
    auto launch = [&](auto type) {
        using T = decltype(type);
        const SandwichGrads<T> A{(const T *)f, (const T *)y, (const T *)gy, (const T *)gn, (const T *)gate, (T *)df, (T *)dx,
                                 (T *)dgate, n, h->desc.C, h->desc.eps, h->part};
        auto run = [&](auto v) {
            constexpr int V = decltype(v)::value;
            sandwich_dispatch<V>(h->desc.C, [&](auto lg, auto k, auto full) {
                constexpr int LG = decltype(lg)::value, K = decltype(k)::value;
                const int64_t per = 4 * (64 / LG);
                blocks = (int)std::min<int64_t>((n + per - 1) / per, NORM_BLOCKS);
                if (blocks)
                    hipLaunchKernelGGL((k_sandwich_bwd<T, V, LG, K, decltype(full)::value>), dim3(blocks), dim3(256), 0,
                                       (hipStream_t)stream, A, sp);
            });
        };
        // Eight bfloat16 values a lane take 190 registers, two waves a SIMD: 1.25 ms for 1M gated rows of 256, with
        // four 0.91; but wider rows would have two pieces a lane (500,000 of 512: 1.15 ms with eight, 3.6 TB/s).
        if constexpr (sizeof(T) == 2)
            if (h->desc.C > 256) return run(ic<8>{});
        run(ic<4>{});
    };
    if (h->desc.io_dtype == TS3_BF16) launch(bf16_t{});
    else launch(float{});
    LAUNCH_CHECK("sandwich norm backward");
    const SandwichSums sums{{d->gamma_post, d->beta_post, d->scale, d->gamma_pre, d->beta_pre}};
    hipLaunchKernelGGL(k_sandwich_join, dim3(SANDWICH_SUMS * h->desc.C / 16), dim3(256), 0, (hipStream_t)stream, h->part, blocks,
                       h->desc.C, sums);
    LAUNCH_CHECK("sandwich norm column sums");
    return TS3_OK;
}

ts3_status ts3_orth_create(const ts3_orth_desc *desc, ts3_orth **out) {
    if (!desc || !out) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *out = nullptr;
    if (desc->steps < 1 || desc->steps > 64) return fail(TS3_ERR_INVALID_ARG, "1 <= steps <= 64 required (got %d)", desc->steps);
    if (!(desc->eps >= 0.f) || std::isinf(desc->eps)) return fail(TS3_ERR_INVALID_ARG, "eps must be finite and >= 0");
    ts3_orth *h = new (std::nothrow) ts3_orth();
    if (!h) return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->desc = *desc;
    *out = h;
    return TS3_OK;
}

ts3_status ts3_orth_free(ts3_orth *h) {
    if (!h) return TS3_OK;
    hipError_t e = hipDeviceSynchronize();
    h->work.free();
    delete h;
    if (e != hipSuccess) return fail(TS3_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
    return TS3_OK;
}

ts3_status ts3_orth_bytes(const ts3_orth *h, int64_t *bytes) {
    if (!h || !bytes) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    *bytes = h->bytes;
    return TS3_OK;
}

ts3_status ts3_orth_matrices(ts3_orth *h, const ts3_matrix *matrices, int32_t count, void *stream) {
    constexpr int32_t SIDE = 32768, COUNT = 16384;
    if (!h || (!matrices && count > 0)) return fail(TS3_ERR_INVALID_ARG, "NULL argument");
    if (count < 0 || count > COUNT) return fail(TS3_ERR_INVALID_ARG, "0 <= count <= %d required (got %d)", COUNT, count);
    for (int32_t i = 0; i < count; ++i) {
        const ts3_matrix &m = matrices[i];
        if (m.dtype != TS3_FP32 && m.dtype != TS3_BF16)
            return fail(TS3_ERR_INVALID_ARG, "tensor %d: dtype %d is not TS3_FP32 or TS3_BF16", i, m.dtype);
        if (m.rows < 0 || m.cols < 0 || m.batch < 0) return fail(TS3_ERR_INVALID_ARG, "tensor %d: a size is negative", i);
        if (!m.rows || !m.cols || !m.batch) continue;
        if (m.rows > SIDE || m.cols > SIDE)
            return fail(TS3_ERR_UNSUPPORTED, "tensor %d: no kernel for a %d x %d matrix (sides up to %d)", i, m.rows, m.cols, SIDE);
        if ((int64_t)m.rows * m.cols > (int64_t(1) << 40) / m.batch)
            return fail(TS3_ERR_UNSUPPORTED, "tensor %d: no launch for so many or so large matrices", i);
        const uintptr_t type = m.dtype == TS3_BF16 ? 1 : 3;
        if (!m.src || !m.dst || (((uintptr_t)m.src | (uintptr_t)m.dst) & type))
            return fail(TS3_ERR_INVALID_ARG, "tensor %d: a pointer is NULL or not aligned to its type", i);
    }
    hipStream_t st = (hipStream_t)stream;
    try {
        std::vector<OrthEntry> list;
        std::vector<ClipRun> runs;
        for (int32_t i = 0; i < count; ++i) {
            const ts3_matrix &m = matrices[i];
            if (!m.rows || !m.cols || !m.batch) continue;
            OrthEntry e{};
            e.src = m.src;
            e.dst = m.dst;
            e.r = std::min(m.rows, m.cols);
            e.c = std::max(m.rows, m.cols);
            e.nb = m.batch;
            e.flags = (m.rows > m.cols ? ORTH_TURNED : 0) | (m.dtype == TS3_BF16 ? ORTH_BF16 : 0);
            list.push_back(e);
            runs.push_back(ClipRun{(const char *)m.src, (char *)m.dst, (int64_t)m.rows * m.cols * m.batch, m.dtype});
        }
        if (runs.empty()) return TS3_OK;
        if (clip_overlaps(runs, true))
            return fail(TS3_ERR_INVALID_ARG, "a result overlaps another tensor (the same one twice, or views of one array)");
        // The longest sums first, and the small matrices behind the others.
        std::stable_sort(list.begin(), list.end(), [](const OrthEntry &p, const OrthEntry &q) { return p.c > q.c; });
        const int64_t cus = device_cu_count();
        const OrthShape shape[2] = {orth_shape(list.data(), list.size(), false, cus), orth_shape(list.data(), list.size(), true, cus)};
        int64_t x = 0, a = 0, slack = 0, n[4] = {0, 0, 0, 0}, big = 0;
        for (OrthEntry &e : list) {
            const int64_t rp = orth_pad(e.r), cp = orth_pad(e.c);
            const bool is_small = e.c <= ORTH_SMALL;
            e.x = x;
            e.a = a;
            e.piece = (int32_t)n[0], e.load = (int32_t)n[1], e.gram = (int32_t)n[2], e.update = (int32_t)n[3];
            if (!is_small) {
                x += 2 * e.nb * rp * cp;
                a += 2 * e.nb * rp * rp;
                slack = std::max(slack, 64 * cp + 64);
            }
            n[0] += is_small ? 1 : (int64_t)e.nb * orth_pieces((int64_t)e.r * e.c);
            n[1] += is_small ? e.nb : e.nb * (rp / 64) * (cp / 64);
            n[2] += orth_tiles(e, shape[0].side, false);
            n[3] += orth_tiles(e, shape[1].side, true);
            if (!is_small) big = n[1];
            for (int64_t k : n)
                if (k >= int64_t(1) << 23) return fail(TS3_ERR_UNSUPPORTED, "no launch for so many or so large matrices");
        }
        auto align = [](int64_t v) { return (v + 255) & ~int64_t(255); };
        int64_t need = 0;
        auto place = [&](int64_t bytes) {
            const int64_t at = need;
            need += align(bytes);
            return at;
        };
        const int nl = (int)list.size();
        const int64_t at_table = place((int64_t)nl * (int64_t)sizeof(OrthEntry)), at_sums = place(n[0] * 8);
        const int64_t at_maps[3] = {place(n[1] * 4), place(n[2] * 4), place(n[3] * 4)};
        const int64_t at_x[2] = {place((x + slack) * 2), place((x + slack) * 2)};
        const int64_t at_a = place((a + slack) * 2), at_b = place((a + slack) * 2);
        ts3_status s = h->work.reserve(need, st, h->bytes);
        if (s != TS3_OK) return s;
        unsigned char *const w = (unsigned char *)h->work.p;
        OrthEntry *const table = (OrthEntry *)(w + at_table);
        double *const sums = (double *)(w + at_sums);
        _Float16 *const xs[2] = {(_Float16 *)(w + at_x[0]), (_Float16 *)(w + at_x[1])};
        _Float16 *const as = (_Float16 *)(w + at_a), *const bs = (_Float16 *)(w + at_b);
        OrthMaps maps{};
        for (int k = 0; k < 3; ++k) maps.of[k] = (int32_t *)(w + at_maps[k]);
        for (int first = 0; first < nl; first += ORTH_BATCH) {
            OrthBatch b{};
            b.first = first;
            b.count = std::min(ORTH_BATCH, nl - first);
            std::copy(list.begin() + first, list.begin() + first + b.count, b.e);
            const bool more = first + b.count < nl;
            const OrthEntry &next = list[(size_t)(more ? first + b.count : 0)];
            maps.end[ORTH_AT_LOAD] = more ? next.load : (int32_t)n[1];
            maps.end[ORTH_AT_GRAM] = more ? next.gram : (int32_t)n[2];
            maps.end[ORTH_AT_UPDATE] = more ? next.update : (int32_t)n[3];
            const int64_t wgs = (more ? next.piece : n[0]) - b.e[0].piece;
            hipLaunchKernelGGL(k_orth_norm, dim3((unsigned)wgs), dim3(256), 0, st, b, table, maps, sums);
            LAUNCH_CHECK("orthogonalisation norms");
        }
        const double eps = h->desc.eps;
        if (n[1] > big) {
            hipLaunchKernelGGL(k_orth_small, dim3((unsigned)(n[1] - big)), dim3(256), 0, st, table, maps.of[ORTH_AT_LOAD], (int)big,
                               h->desc.steps, eps);
            LAUNCH_CHECK("orthogonalisation of small matrices");
        }
        if (big == 0) return TS3_OK;
        hipLaunchKernelGGL(k_orth_load, dim3((unsigned)big), dim3(256), 0, st, table, maps.of[ORTH_AT_LOAD], sums, eps, xs[0]);
        LAUNCH_CHECK("orthogonalisation operands");
        auto product = [&](auto kind, const OrthShape &sh, int64_t count, const int32_t *map, const _Float16 *px, const _Float16 *pa,
                           _Float16 *out, bool last) {
            constexpr int KIND = decltype(kind)::value;
            const auto kernel = sh.side == 128 ? &k_orth_stream<KIND> : sh.groups == 1 ? &k_orth_product<KIND, 1> : &k_orth_product<KIND, 4>;
            const int64_t most = sh.side == 128 ? cus : sh.groups == 1 ? 4 * cus : count;
            const int threads = sh.side == 128 ? 512 : 256 * sh.groups;
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(count, most)), dim3(threads), 0, st, table, map, (int)count, px, pa, out,
                               last);
        };
        for (int i = 0; i < h->desc.steps; ++i) {
            const _Float16 *const from = xs[i & 1];
            product(ic<ORTH_GRAM>{}, shape[0], n[2], maps.of[ORTH_AT_GRAM], from, as, as, false);
            product(ic<ORTH_SQUARE>{}, shape[0], n[2], maps.of[ORTH_AT_GRAM], from, as, bs, false);
            product(ic<ORTH_UPDATE>{}, shape[1], n[3], maps.of[ORTH_AT_UPDATE], from, bs, xs[i & 1 ^ 1], i + 1 == h->desc.steps);
            LAUNCH_CHECK("orthogonalisation products");
        }
    } catch (const std::bad_alloc &) {
        return fail(TS3_ERR_OUT_OF_MEMORY, "host allocation failed");
    }
    return TS3_OK;
}

}  // extern "C"
