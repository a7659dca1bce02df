// The gated feed-forward block and its gradient: which products they are, how the products are cut, the workspace and the
// C entry points.  The products are in ffn_mfma16.h, ffn_f32.hip and, for few rows, ffn_few.hip.
//
//   forward : h = act(x w_in^T) (gate, up in one product, FFN_GATE), out = h w_out^T
//   gradient: [dgate | dup], h from dout w_out (FFN_GRAD); dx = [dgate | dup] w_in; dw_in = [dgate | dup]^T x;
//             dw_out = dout^T h; column sums for the biases
#include "ffn.h"

namespace gmpgr {

// Joins the slices of a product that was cut along k and applies its epilogue: 8 columns a thread.
template <int KIND, int EPI> __global__ void __launch_bounds__(256) ffn_finish_kernel(FfnArgs p) {
    constexpr int W = 8;
    const int64_t across = (p.N + W - 1) / W, total = across * p.M, width = EPI == FFN_GATE ? 2 * (int64_t)p.N : p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / across;
        const int n = (int)(i - m * across) * W, left = p.N - n;
        float s[W] = {}, u[W] = {}, v[W];
        const FfnRow<W> r = {};
#pragma unroll 4
        for (int c = 0; c < p.splits; ++c) {
            const float *q = p.part + ((int64_t)c * p.M + m) * width + n;
            load_cols<W>(q, left, v);
#pragma unroll
            for (int e = 0; e < W; ++e) s[e] += v[e];
            if (EPI == FFN_GATE) {
                load_cols<W>(q + p.N, left, v);
#pragma unroll
                for (int e = 0; e < W; ++e) u[e] += v[e];
            }
        }
        ffn_epilogue<KIND, EPI, W>(p, m, n, s, u, r);
    }
}

template <int KIND> static int launch_finish(const FfnArgs &a, int epi, hipStream_t stream) {
    const int64_t groups = ((int64_t)((a.N + 7) / 8) * a.M + 255) / 256;
    auto fn = epi == FFN_GATE ? ffn_finish_kernel<KIND, FFN_GATE> : ffn_finish_kernel<KIND, FFN_STORE>;
    hipLaunchKernelGGL(fn, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

// The cut that a simple account says is fastest: rounds of workgroups over 256 compute units, each of which holds a_unit of
// them, a round as many steps of 64 k as a slice has and a start and an end; a last round that leaves units with fewer
// workgroups is that much shorter; and for slices the writing and reading of the parts and one more launch.  Fitted to
// measured products: of 8192 x 8192 x 2048 (FFN_GRAD) 449 us in tiles of 256, 478 in tiles of 128; 8192 x 8192 x 2048
// (FFN_GATE) 562 and 793, 4096 x 2048 x 2048 63 and 68; 4096 x 2048 x 2048 (FFN_STORE) 40 in two slices of k and 35; 8192 x
// 2048 x 16384 442 and 569.  It is up to 20 % low for products that end inside a tile and a round: of 1537 x 2 x 2731 x 1003 in
// fp16 (FFN_GATE) it says 40 us, which take 50 (and of the other tile 44, which is as near), of 1537 x 2731 x 777 (FFN_GRAD)
// 34, which take 43, of 2048 x 1300 x 256 in fp32 (FFN_GRAD) 27, which take 33.
struct FfnTileCost {
    int rows, cols, a_unit;
    double step, ends[3];  // microseconds of 64 k, of the start and the end by epilogue, with a_unit of them at work
};
static const FfnTileCost FFN_TILES16[] = {{256, 256, 1, 1.7, {13.0, 17.0, 50.0}}, {128, 128, 2, 1.1, {4.0, 6.0, 20.0}}};
static const FfnTileCost FFN_TILES32[] = {{128, 128, 2, 9.3, {6.0, 6.0, 12.0}}, {64, 64, 4, 5.1, {5.0, 5.0, 10.0}}};

FfnCut ffn_cut(int kind, int64_t M, int64_t N, int64_t K, int epi) {
    FfnCut best = {128, 128, 1};
    double least = 0.0;
    for (int i = 0; i < 2; ++i) {
        FfnTileCost c = kind == ANN_F32 ? FFN_TILES32[i] : FFN_TILES16[i];
        if (c.rows == 64 && epi == FFN_GATE) c.rows = 128, c.a_unit = 2;  // gate and up of a column are one wave's
        const int64_t cols = epi == FFN_GATE ? c.cols / 2 : c.cols, tiles = ((M + c.rows - 1) / c.rows) * ((N + cols - 1) / cols);
        // FFN_GRAD is not cut along k: its column sums are its tiles'
        for (int s = 1; s <= 16 && (s == 1 || (s <= K / 256 && epi != FFN_GRAD)); s += s < 4 ? 1 : 2) {
            const int64_t slots = 256 * c.a_unit, groups = tiles * s, rounds = groups / slots, rest = groups % slots;
            const double steps = (double)((K + 64 * s - 1) / (64 * s));
            double last = (double)((rest + 255) / 256) / c.a_unit;
            if (rest > 0 && last < 1.0) last += 0.1;
            double t = ((double)rounds + last) * steps * c.step + (double)(rounds + (rest > 0)) * c.ends[s > 1 ? FFN_STORE : epi];
            if (s > 1)  // the parts come out of the caches, what the epilogue reads and writes does not
                t += 4.0 + (double)M * (double)N * (8.0 * s * (epi == FFN_GATE ? 2 : 1) / 1.0e7 + (epi == FFN_GATE ? 12.0 / 4.0e6 : 0.0));
            if (least == 0.0 || t < least) least = t, best = {c.rows, c.cols, s};
        }
    }
    return best;
}

size_t ffn_part_floats(int kind, int64_t M, int64_t N, int64_t K, int epi) {
    const int s = ffn_cut(kind, M, N, K, epi).splits;
    return s > 1 ? (size_t)s * (size_t)M * (size_t)N * (epi == FFN_GATE ? 2 : 1) : 0;
}

int launch_ffn_product(const FfnProduct &product, float *part, hipStream_t stream) {
    FfnProduct p = product;
    FfnArgs &a = p.args;
    const FfnCut cut = ffn_cut(p.kind, a.M, a.N, a.K, p.epi);
    a.k_slice = cut.splits == 1 ? a.K : (int32_t)((((int64_t)a.K + cut.splits - 1) / cut.splits + 63) / 64 * 64);
    a.splits = (int32_t)(((int64_t)a.K + a.k_slice - 1) / a.k_slice);
    a.part = a.splits > 1 ? part : nullptr;
    const int rc = p.kind == ANN_F32    ? launch_ffn32(p, cut.cols, stream)
                   : p.kind == ANN_BF16 ? launch_ffn16<ANN_BF16>(p, cut.cols, stream)
                                        : launch_ffn16<ANN_F16>(p, cut.cols, stream);
    if (rc != ANN_OK || a.splits == 1) return rc;
    return p.kind == ANN_F32    ? launch_finish<ANN_F32>(a, p.epi, stream)
           : p.kind == ANN_BF16 ? launch_finish<ANN_BF16>(a, p.epi, stream)
                                : launch_finish<ANN_F16>(a, p.epi, stream);
}

struct Region {
    size_t total = 0;
    size_t take(size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) & ~(size_t)255;
        return at;
    }
};
// Parts of a workspace.  x, w_in, w_out, dout: copies of operands whose rows the 16-bit kernels cannot load as they lie (an
// odd width, stride or address); kept free for every call, because a workspace is sized before the addresses are known.
struct FfnPlan {
    size_t x, w_in, w_out, dout, dpre, h, h_rest, part, cols, total;
    int64_t D8, F8, O8, ld_pre;  // row strides of the copies, of h and of dpre (fp32: as wide as the rows)
    int64_t gate_parts, out_parts;  // cols: sums over blocks of rows, [gate_parts][2 F] for b_in's gradient, [out_parts][O]
};
// Few rows: h in two 16-bit parts (both products are the few rows' then).
static bool ffn_h_rest(int64_t M, int dtype) { return dtype != ANN_F32 && M <= ffn_few(dtype, FFN_STORE); }
static size_t most(size_t a, size_t b) { return a > b ? a : b; }

static FfnPlan ffn_plan(int64_t M, int64_t D, int64_t F, int64_t O, int dtype, bool gradient) {
    Region r;
    FfnPlan p = {};
    const size_t e = elem_bytes(dtype);
    const bool pack = dtype != ANN_F32;
    const int64_t to = pack ? 8 : 1;
    p.D8 = (D + to - 1) / to * to, p.F8 = (F + to - 1) / to * to, p.O8 = (O + to - 1) / to * to;
    p.ld_pre = (2 * F + to - 1) / to * to;
    p.h = r.take((size_t)M * p.F8 * e);
    p.h_rest = r.take(ffn_h_rest(M, dtype) && !gradient ? (size_t)M * p.F8 * e : 0);
    const bool few_in = !gradient && M <= ffn_few(dtype, FFN_GATE), few_out = !gradient && M <= ffn_few(dtype, FFN_STORE);
    if (pack && !few_in) {
        p.x = r.take((size_t)M * p.D8 * e);
        p.w_in = r.take((size_t)2 * F * p.D8 * e);
    }
    if (pack && !few_out) p.w_out = r.take((size_t)O * p.F8 * e);
    size_t n = 0;
    if (!gradient) {
        if (!few_in) n = ffn_part_floats(dtype, M, F, D, FFN_GATE);
        if (!few_out) n = most(n, ffn_part_floats(dtype, M, O, F, FFN_STORE));
    } else {
        if (pack) p.dout = r.take((size_t)M * p.O8 * e);
        p.dpre = r.take((size_t)M * p.ld_pre * e);
        n = ffn_part_floats(dtype, M, D, 2 * F, FFN_STORE);
        n = most(n, ffn_part_floats(dtype, 2 * F, D, M, FFN_STORE));
        n = most(n, ffn_part_floats(dtype, O, F, M, FFN_STORE));
    }
    p.part = r.take(sizeof(float) * n);
    if (gradient) {
        p.gate_parts = pack ? ffn_col_blocks(M, ffn_cut(dtype, M, F, O, FFN_GRAD).rows) : column_sum_parts(M, 2 * F);
        p.out_parts = column_sum_parts(M, O);
        p.cols = r.take(sizeof(float) * ((size_t)p.gate_parts * 2 * F + (size_t)p.out_parts * O));
    }
    p.total = r.total + 256;
    return p;
}

// An operand as the product's kernels take it: itself, or its copy in the workspace, which the call's one packing launch makes.
struct Rows {
    const void *p;
    int64_t ld;
};
static Rows ffn_rows(int dtype, const void *p, int64_t ld, int64_t rows, int64_t width, char *copy, int64_t ld_copy, PadRows *pads) {
    if (dtype == ANN_F32 || ffn_direct(p, ld, width)) return {p, ld};
    pads->item[pads->n++] = {p, ld, rows, width, copy, ld_copy};
    return {copy, ld_copy};
}

static bool ffn_sizes(int64_t M, int32_t D, int32_t F, int32_t O, int32_t dtype) {
    // M is the k of the weights' gradients, which the kernels count in 32 bits up to three steps past its end, and with 2^29
    // rows in tiles of 64 a launch has 2^31 threads
    const int32_t w = 1 << 20;
    if (M < 0 || M > (1 << 29) || D < 1 || D > w || F < 1 || F > w || O < 1 || O > w || !row_dtype(dtype)) {
        set_error("need 0 <= M <= 2^29, widths 1 .. 2^20, dtype ANN_F32, ANN_BF16 or ANN_F16 (got M=%lld, %d, %d, %d, dtype %d)",
                  (long long)M, D, F, O, dtype);
        return false;
    }
    return true;
}
static bool ffn_array(const char *name, const void *p, size_t align, bool may_be_null) {
    if ((!p && !may_be_null) || (uintptr_t)p % align) {
        set_error("%s must %sbe aligned to its elements", name, may_be_null ? "" : "not be null and must ");
        return false;
    }
    return true;
}
static bool ffn_stride(const char *name, int64_t ld, int64_t width) {
    if (ld < width || ld > (int64_t)1 << 32) {
        set_error("%s = %lld, need %lld .. 2^32", name, (long long)ld, (long long)width);
        return false;
    }
    return true;
}
static bool ffn_workspace(const void *ws, size_t have, size_t need, int *rc) {
    if (!ws || (uintptr_t)ws % 256) {
        set_error("workspace_dev must not be null and must be 256-byte aligned");
        *rc = ANN_EINVAL;
        return false;
    }
    if (have < need) {
        set_error("workspace of %zu bytes, %zu needed", have, need);
        *rc = ANN_EWORKSPACE;
        return false;
    }
    return true;
}

}  // namespace gmpgr

using namespace gmpgr;

extern "C" {

size_t ann_gated_ffn_workspace_bytes(int64_t M, int32_t d_in, int32_t d_hidden, int32_t d_out, int32_t dtype) {
    return ffn_sizes(M, d_in, d_hidden, d_out, dtype) ? ffn_plan(M, d_in, d_hidden, d_out, dtype, false).total : 0;
}

size_t ann_gated_ffn_backward_workspace_bytes(int64_t M, int32_t d_in, int32_t d_hidden, int32_t d_out, int32_t dtype) {
    return ffn_sizes(M, d_in, d_hidden, d_out, dtype) ? ffn_plan(M, d_in, d_hidden, d_out, dtype, true).total : 0;
}

int ann_gated_ffn(const void *x_dev, int64_t ld_x, const void *w_in_dev, const void *b_in_dev, const void *w_out_dev,
                  const void *b_out_dev, int64_t M, int32_t d_in, int32_t d_hidden, int32_t d_out, int32_t act,
                  int32_t dtype, void *out_dev, int64_t ld_out, float *pre_dev, void *workspace_dev,
                  size_t workspace_bytes, void *stream) {
    int rc = ANN_EINVAL;
    if (!ffn_sizes(M, d_in, d_hidden, d_out, dtype)) return rc;
    if (act < ANN_SILU || act > ANN_RELU) {
        set_error("unknown activation %d", act);
        return rc;
    }
    if (M == 0) return ANN_OK;
    const size_t e = elem_bytes(dtype);
    if (!ffn_array("x_dev", x_dev, e, false) || !ffn_array("w_in_dev", w_in_dev, e, false) ||
        !ffn_array("w_out_dev", w_out_dev, e, false) || !ffn_array("out_dev", out_dev, e, false) ||
        !ffn_array("b_in_dev", b_in_dev, e, true) || !ffn_array("b_out_dev", b_out_dev, e, true) ||
        !ffn_array("pre_dev", pre_dev, 4, true) || !ffn_stride("ld_x", ld_x, d_in) || !ffn_stride("ld_out", ld_out, d_out))
        return rc;
    if (rows_overlap(x_dev, ld_x, d_in, out_dev, ld_out, d_out, M, e)) {
        set_error("out_dev must not overlap x_dev");
        return rc;
    }
    const FfnPlan plan = ffn_plan(M, d_in, d_hidden, d_out, dtype, false);
    if (!ffn_workspace(workspace_dev, workspace_bytes, plan.total, &rc)) return rc;
    char *ws = (char *)workspace_dev;
    hipStream_t s = (hipStream_t)stream;
    const bool few_in = M <= ffn_few(dtype, FFN_GATE), few_out = M <= ffn_few(dtype, FFN_STORE);
    Rows x = {x_dev, ld_x}, w_in = {w_in_dev, d_in}, w_out = {w_out_dev, d_hidden};
    PadRows pads = {};
    if (!few_in) {
        x = ffn_rows(dtype, x_dev, ld_x, M, d_in, ws + plan.x, plan.D8, &pads);
        w_in = ffn_rows(dtype, w_in_dev, d_in, (int64_t)2 * d_hidden, d_in, ws + plan.w_in, plan.D8, &pads);
    }
    if (!few_out) w_out = ffn_rows(dtype, w_out_dev, d_hidden, d_out, d_hidden, ws + plan.w_out, plan.F8, &pads);
    rc = launch_pad_rows(pads, s);
    if (rc != ANN_OK) return rc;
    FfnProduct p = {};
    p.kind = dtype, p.epi = FFN_GATE, p.a_rows = true, p.b_rows = true;
    p.args.A = x.p, p.args.lda = x.ld, p.args.B = w_in.p, p.args.ldb = w_in.ld;
    p.args.M = (int32_t)M, p.args.N = d_hidden, p.args.K = d_in, p.args.up = d_hidden;
    p.args.C = ws + plan.h, p.args.ldc = plan.F8, p.args.pad = dtype != ANN_F32;
    p.args.bias = b_in_dev, p.args.pre = pre_dev, p.args.act = act;
    void *rest = ffn_h_rest(M, dtype) ? ws + plan.h_rest : nullptr;
    p.args.h = rest, p.args.ldh = plan.F8;
    rc = few_in ? launch_ffn_few(p, s) : launch_ffn_product(p, (float *)(ws + plan.part), s);
    if (rc != ANN_OK) return rc;
    FfnProduct q = {};
    q.kind = dtype, q.epi = FFN_STORE, q.a_rows = true, q.b_rows = true;
    q.args.A = ws + plan.h, q.args.A_rest = rest, q.args.lda = plan.F8, q.args.B = w_out.p, q.args.ldb = w_out.ld;
    q.args.M = (int32_t)M, q.args.N = d_out, q.args.K = d_hidden;
    q.args.C = out_dev, q.args.ldc = ld_out, q.args.bias = b_out_dev;
    return few_out ? launch_ffn_few(q, s) : launch_ffn_product(q, (float *)(ws + plan.part), s);
}

int ann_gated_ffn_backward(const void *dout_dev, int64_t ld_dout, const void *x_dev, int64_t ld_x, const float *pre_dev,
                           const void *w_in_dev, const void *w_out_dev, int64_t M, int32_t d_in, int32_t d_hidden,
                           int32_t d_out, int32_t act, int32_t dtype, void *dx_dev, int64_t ld_dx, void *dw_in_dev,
                           void *db_in_dev, void *dw_out_dev, void *db_out_dev, void *workspace_dev,
                           size_t workspace_bytes, void *stream) {
    int rc = ANN_EINVAL;
    if (!ffn_sizes(M, d_in, d_hidden, d_out, dtype)) return rc;
    if (act < ANN_SILU || act > ANN_RELU) {
        set_error("unknown activation %d", act);
        return rc;
    }
    const size_t e = elem_bytes(dtype);
    if (!ffn_array("dx_dev", dx_dev, e, true) || !ffn_array("dw_in_dev", dw_in_dev, e, true) ||
        !ffn_array("db_in_dev", db_in_dev, e, true) || !ffn_array("dw_out_dev", dw_out_dev, e, true) ||
        !ffn_array("db_out_dev", db_out_dev, e, true))
        return rc;
    hipStream_t s = (hipStream_t)stream;
    if (M == 0) {
        rc = dw_in_dev ? launch_zero(dw_in_dev, (int64_t)2 * d_hidden * d_in, dtype, s) : ANN_OK;
        if (rc == ANN_OK && db_in_dev) rc = launch_zero(db_in_dev, (int64_t)2 * d_hidden, dtype, s);
        if (rc == ANN_OK && dw_out_dev) rc = launch_zero(dw_out_dev, (int64_t)d_out * d_hidden, dtype, s);
        if (rc == ANN_OK && db_out_dev) rc = launch_zero(db_out_dev, d_out, dtype, s);
        return rc;
    }
    if (!ffn_array("dout_dev", dout_dev, e, false) || !ffn_array("x_dev", x_dev, e, false) ||
        !ffn_array("pre_dev", pre_dev, 4, false) || !ffn_array("w_in_dev", w_in_dev, e, false) ||
        !ffn_array("w_out_dev", w_out_dev, e, false) || !ffn_stride("ld_dout", ld_dout, d_out) ||
        !ffn_stride("ld_x", ld_x, d_in) || (dx_dev && !ffn_stride("ld_dx", ld_dx, d_in)))
        return rc;
    if (dx_dev && (rows_overlap(dx_dev, ld_dx, d_in, dout_dev, ld_dout, d_out, M, e) ||
                   rows_overlap(dx_dev, ld_dx, d_in, x_dev, ld_x, d_in, M, e))) {
        set_error("dx_dev must not overlap dout_dev or x_dev");
        return rc;
    }
    const FfnPlan plan = ffn_plan(M, d_in, d_hidden, d_out, dtype, true);
    if (!ffn_workspace(workspace_dev, workspace_bytes, plan.total, &rc)) return rc;
    char *ws = (char *)workspace_dev;
    float *part = (float *)(ws + plan.part);
    void *dpre = ws + plan.dpre, *h = ws + plan.h;
    const bool hidden = dx_dev || dw_in_dev || db_in_dev;  // the gradient of gate and up is wanted
    Rows dout = {dout_dev, ld_dout}, x = {x_dev, ld_x}, w_in = {w_in_dev, d_in}, w_out = {w_out_dev, d_hidden};
    PadRows pads = {};
    if (hidden || dw_out_dev) {
        dout = ffn_rows(dtype, dout_dev, ld_dout, M, d_out, ws + plan.dout, plan.O8, &pads);
        w_out = ffn_rows(dtype, w_out_dev, d_hidden, d_out, d_hidden, ws + plan.w_out, plan.F8, &pads);
    }
    if (dx_dev) w_in = ffn_rows(dtype, w_in_dev, d_in, (int64_t)2 * d_hidden, d_in, ws + plan.w_in, plan.D8, &pads);
    if (dw_in_dev) x = ffn_rows(dtype, x_dev, ld_x, M, d_in, ws + plan.x, plan.D8, &pads);
    rc = launch_pad_rows(pads, s);
    if (rc == ANN_OK && (hidden || dw_out_dev)) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_GRAD, p.a_rows = true, p.b_rows = false;
        p.args.A = dout.p, p.args.lda = dout.ld, p.args.B = w_out.p, p.args.ldb = w_out.ld;
        p.args.M = (int32_t)M, p.args.N = d_hidden, p.args.K = d_out;
        p.args.C = dpre, p.args.ldc = plan.ld_pre, p.args.up = d_hidden, p.args.pad = dtype != ANN_F32;
        p.args.h = dw_out_dev ? h : nullptr, p.args.ldh = plan.F8;
        p.args.pre = const_cast<float *>(pre_dev), p.args.act = act;
        p.args.cols = db_in_dev && dtype != ANN_F32 ? (float *)(ws + plan.cols) : nullptr;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dx_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = true, p.b_rows = false;
        p.args.A = dpre, p.args.lda = plan.ld_pre, p.args.B = w_in.p, p.args.ldb = w_in.ld;
        p.args.M = (int32_t)M, p.args.N = d_in, p.args.K = 2 * d_hidden;
        p.args.C = dx_dev, p.args.ldc = ld_dx;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dw_in_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = false, p.b_rows = false;
        p.args.A = dpre, p.args.lda = plan.ld_pre, p.args.B = x.p, p.args.ldb = x.ld;
        p.args.M = 2 * d_hidden, p.args.N = d_in, p.args.K = (int32_t)M;
        p.args.C = dw_in_dev, p.args.ldc = d_in;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dw_out_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = false, p.b_rows = false;
        p.args.A = dout.p, p.args.lda = dout.ld, p.args.B = h, p.args.ldb = plan.F8;
        p.args.M = d_out, p.args.N = d_hidden, p.args.K = (int32_t)M;
        p.args.C = dw_out_dev, p.args.ldc = d_hidden;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && (db_in_dev || db_out_dev)) {
        ColumnSums sums = {};
        float *gate = (float *)(ws + plan.cols), *out = gate + plan.gate_parts * 2 * d_hidden;
        // in 16 bits the sums over blocks of rows are there: of the values before their rounding
        if (db_in_dev)
            sums.item[sums.n++] = {dtype == ANN_F32 ? dpre : nullptr, (int64_t)2 * d_hidden, plan.ld_pre, db_in_dev, gate, plan.gate_parts};
        if (db_out_dev) sums.item[sums.n++] = {dout_dev, d_out, ld_dout, db_out_dev, out, plan.out_parts};
        rc = launch_column_sums(sums, M, dtype, s);
    }
    return rc;
}

}  // extern "C"
