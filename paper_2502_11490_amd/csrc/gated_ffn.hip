// The gated feed-forward block and its gradient: which products they are, how the products are cut, the workspace and the
// C entry points.  The products are in ffn_mfma16.h and ffn_f32.hip.
//
//   forward : h = act(x w_in^T) (gate, up in one product, FFN_GATE), out = h w_out^T
//   gradient: [dgate | dup], h from dout w_out (FFN_GRAD); dx = [dgate | dup] w_in; dw_in = [dgate | dup]^T x;
//             dw_out = dout^T h; column sums for the biases
#include "ffn.h"

namespace gmpgr {

// Joins the slices of a product that was cut along k and applies its epilogue: four columns a thread.
template <int KIND, int EPI> __global__ void __launch_bounds__(256) ffn_finish_kernel(FfnArgs p) {
    const int64_t quads = (p.N + 3) / 4, total = quads * p.M, width = EPI == FFN_GATE ? 2 * (int64_t)p.N : p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int n = (int)(i - m * quads) * 4, left = p.N - n;
        float s[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f}, v[4];
        for (int c = 0; c < p.splits; ++c) {
            const float *q = p.part + ((int64_t)c * p.M + m) * width + n;
            load4(q, left, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
            if (EPI == FFN_GATE) {
                load4(q + p.N, left, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] += v[e];
            }
        }
        ffn_epilogue<KIND, EPI>(p, m, n, s, u);
    }
}

template <int KIND> static int launch_finish(const FfnArgs &a, int epi, hipStream_t stream) {
    const int64_t groups = ((int64_t)((a.N + 3) / 4) * a.M + 255) / 256;
    auto fn = epi == FFN_GATE   ? ffn_finish_kernel<KIND, FFN_GATE>
              : epi == FFN_GRAD ? ffn_finish_kernel<KIND, FFN_GRAD>
                                : ffn_finish_kernel<KIND, FFN_STORE>;
    hipLaunchKernelGGL(fn, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

// Slices of k: enough workgroups for two a compute unit where the tiles alone are not, each slice with 4 or more steps
// of 64, and at most 16 (each costs a write and a read of the whole result in fp32).
int ffn_splits(int kind, int64_t M, int64_t N, int64_t K, int epi) {
    const int64_t cols = epi == FFN_GATE ? 64 : 128, tiles = ((M + 127) / 128) * ((N + cols - 1) / cols);
    (void)kind;
    int64_t s = 512 / (tiles < 1 ? 1 : tiles);
    if (s > K / 256) s = K / 256;
    if (s > 16) s = 16;
    return s < 1 ? 1 : (int)s;
}

size_t ffn_part_floats(int kind, int64_t M, int64_t N, int64_t K, int epi) {
    const int s = ffn_splits(kind, M, N, K, epi);
    return s > 1 ? (size_t)s * (size_t)M * (size_t)N * (epi == FFN_GATE ? 2 : 1) : 0;
}

int launch_ffn_product(const FfnProduct &product, float *part, hipStream_t stream) {
    FfnProduct p = product;
    FfnArgs &a = p.args;
    const int s = ffn_splits(p.kind, a.M, a.N, a.K, p.epi);
    a.k_slice = (int32_t)((((int64_t)a.K + s - 1) / s + 63) / 64 * 64);
    if (s == 1) a.k_slice = a.K;
    a.splits = (int32_t)(((int64_t)a.K + a.k_slice - 1) / a.k_slice);
    a.part = a.splits > 1 ? part : nullptr;
    const int rc = p.kind == ANN_F32    ? launch_ffn32(p, stream)
                   : p.kind == ANN_BF16 ? launch_ffn16<ANN_BF16>(p, stream)
                                        : launch_ffn16<ANN_F16>(p, stream);
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
struct ForwardPlan {
    size_t h, part, total;
};
struct BackwardPlan {
    size_t dpre, h, part, total;
};
static size_t most(size_t a, size_t b) { return a > b ? a : b; }

static ForwardPlan forward_plan(int64_t M, int64_t D, int64_t F, int64_t O, int dtype) {
    Region r;
    ForwardPlan p;
    p.h = r.take((size_t)M * F * elem_bytes(dtype));
    p.part = r.take(sizeof(float) * most(ffn_part_floats(dtype, M, F, D, FFN_GATE), ffn_part_floats(dtype, M, O, F, FFN_STORE)));
    p.total = r.total + 256;
    return p;
}
static BackwardPlan backward_plan(int64_t M, int64_t D, int64_t F, int64_t O, int dtype) {
    Region r;
    BackwardPlan p;
    p.dpre = r.take((size_t)M * 2 * F * elem_bytes(dtype));
    p.h = r.take((size_t)M * F * elem_bytes(dtype));
    size_t n = ffn_part_floats(dtype, M, F, O, FFN_GRAD);
    n = most(n, ffn_part_floats(dtype, M, D, 2 * F, FFN_STORE));
    n = most(n, ffn_part_floats(dtype, 2 * F, D, M, FFN_STORE));
    n = most(n, ffn_part_floats(dtype, O, F, M, FFN_STORE));
    n = most(n, (size_t)column_sum_parts(M, 2 * F) * 2 * F);
    n = most(n, (size_t)column_sum_parts(M, O) * O);
    p.part = r.take(sizeof(float) * n);
    p.total = r.total + 256;
    return p;
}

static bool ffn_sizes(int64_t M, int32_t D, int32_t F, int32_t O, int32_t dtype) {
    const int32_t w = 1 << 20;
    if (M < 0 || M > 0x7fffffffll || D < 1 || D > w || F < 1 || F > w || O < 1 || O > w || !row_dtype(dtype)) {
        set_error("need 0 <= M < 2^31, widths 1 .. 2^20, dtype ANN_F32, ANN_BF16 or ANN_F16 (got M=%lld, %d, %d, %d, dtype %d)",
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
static bool overlap(const void *a, int64_t rows_a, int64_t ld_a, int64_t w_a, const void *b, int64_t rows_b, int64_t ld_b,
                    int64_t w_b, size_t e) {
    const uintptr_t a0 = (uintptr_t)a, a1 = a0 + (size_t)((rows_a - 1) * ld_a + w_a) * e;
    const uintptr_t b0 = (uintptr_t)b, b1 = b0 + (size_t)((rows_b - 1) * ld_b + w_b) * e;
    return a0 < b1 && b0 < a1;
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
    return ffn_sizes(M, d_in, d_hidden, d_out, dtype) ? forward_plan(M, d_in, d_hidden, d_out, dtype).total : 0;
}

size_t ann_gated_ffn_backward_workspace_bytes(int64_t M, int32_t d_in, int32_t d_hidden, int32_t d_out, int32_t dtype) {
    return ffn_sizes(M, d_in, d_hidden, d_out, dtype) ? backward_plan(M, d_in, d_hidden, d_out, dtype).total : 0;
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
    if (overlap(x_dev, M, ld_x, d_in, out_dev, M, ld_out, d_out, e)) {
        set_error("out_dev must not overlap x_dev");
        return rc;
    }
    const ForwardPlan plan = forward_plan(M, d_in, d_hidden, d_out, dtype);
    if (!ffn_workspace(workspace_dev, workspace_bytes, plan.total, &rc)) return rc;
    char *ws = (char *)workspace_dev;
    hipStream_t s = (hipStream_t)stream;
    FfnProduct p = {};
    p.kind = dtype, p.epi = FFN_GATE, p.a_rows = true, p.b_rows = true;
    p.args.A = x_dev, p.args.lda = ld_x, p.args.B = w_in_dev, p.args.ldb = d_in;
    p.args.M = (int32_t)M, p.args.N = d_hidden, p.args.K = d_in;
    p.args.C = ws + plan.h, p.args.ldc = d_hidden, p.args.bias = b_in_dev, p.args.pre = pre_dev, p.args.act = act;
    rc = launch_ffn_product(p, (float *)(ws + plan.part), s);
    if (rc != ANN_OK) return rc;
    FfnProduct q = {};
    q.kind = dtype, q.epi = FFN_STORE, q.a_rows = true, q.b_rows = true;
    q.args.A = ws + plan.h, q.args.lda = d_hidden, q.args.B = w_out_dev, q.args.ldb = d_hidden;
    q.args.M = (int32_t)M, q.args.N = d_out, q.args.K = d_hidden;
    q.args.C = out_dev, q.args.ldc = ld_out, q.args.bias = b_out_dev;
    return launch_ffn_product(q, (float *)(ws + plan.part), s);
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
    if (dx_dev && (overlap(dx_dev, M, ld_dx, d_in, dout_dev, M, ld_dout, d_out, e) ||
                   overlap(dx_dev, M, ld_dx, d_in, x_dev, M, ld_x, d_in, e))) {
        set_error("dx_dev must not overlap dout_dev or x_dev");
        return rc;
    }
    const BackwardPlan plan = backward_plan(M, d_in, d_hidden, d_out, dtype);
    if (!ffn_workspace(workspace_dev, workspace_bytes, plan.total, &rc)) return rc;
    char *ws = (char *)workspace_dev;
    float *part = (float *)(ws + plan.part);
    void *dpre = ws + plan.dpre, *h = ws + plan.h;
    rc = ANN_OK;
    if (dx_dev || dw_in_dev || db_in_dev || dw_out_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_GRAD, p.a_rows = true, p.b_rows = false;
        p.args.A = dout_dev, p.args.lda = ld_dout, p.args.B = w_out_dev, p.args.ldb = d_hidden;
        p.args.M = (int32_t)M, p.args.N = d_hidden, p.args.K = d_out;
        p.args.C = dpre, p.args.ldc = (int64_t)2 * d_hidden, p.args.h = dw_out_dev ? h : nullptr;
        p.args.pre = const_cast<float *>(pre_dev), p.args.act = act;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dx_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = true, p.b_rows = false;
        p.args.A = dpre, p.args.lda = (int64_t)2 * d_hidden, p.args.B = w_in_dev, p.args.ldb = d_in;
        p.args.M = (int32_t)M, p.args.N = d_in, p.args.K = 2 * d_hidden;
        p.args.C = dx_dev, p.args.ldc = ld_dx;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dw_in_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = false, p.b_rows = false;
        p.args.A = dpre, p.args.lda = (int64_t)2 * d_hidden, p.args.B = x_dev, p.args.ldb = ld_x;
        p.args.M = 2 * d_hidden, p.args.N = d_in, p.args.K = (int32_t)M;
        p.args.C = dw_in_dev, p.args.ldc = d_in;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && dw_out_dev) {
        FfnProduct p = {};
        p.kind = dtype, p.epi = FFN_STORE, p.a_rows = false, p.b_rows = false;
        p.args.A = dout_dev, p.args.lda = ld_dout, p.args.B = h, p.args.ldb = d_hidden;
        p.args.M = d_out, p.args.N = d_hidden, p.args.K = (int32_t)M;
        p.args.C = dw_out_dev, p.args.ldc = d_hidden;
        rc = launch_ffn_product(p, part, s);
    }
    if (rc == ANN_OK && db_in_dev)
        rc = launch_column_sum(dpre, M, (int64_t)2 * d_hidden, (int64_t)2 * d_hidden, dtype, db_in_dev, dtype, part, s);
    if (rc == ANN_OK && db_out_dev) rc = launch_column_sum(dout_dev, M, d_out, ld_dout, dtype, db_out_dev, dtype, part, s);
    return rc;
}

}  // extern "C"
