// Products of the gated feed-forward block: what they take and their epilogues.
#pragma once

#include "rows.h"

namespace gmpgr {

// What becomes of a product's sums.
enum FfnEpi {
    FFN_STORE = 0,  // C = sum + bias
    FFN_GATE = 1,   // columns in pairs (gate, up): C = act(gate) * up, and the sums themselves to pre
    FFN_GRAD = 2,   // the sum is dh: C = [dh * up * act'(gate) | dh * act(gate)], h = act(gate) * up
};

// C [M][N] = sum over k < K of A(m, k) B(n, k); where an operand's k are contiguous it is [rows][ld], else [k][ld].
struct FfnArgs {
    const void *A, *B;
    const void *A_rest;   // few rows: what A's rounding left over, added to it in the products (null = nothing)
    int64_t lda, ldb;
    int32_t M, N, K;      // FFN_GATE: N = d_hidden, B has rows 0 .. N - 1 for the gate, up .. up + N - 1 for up
    int32_t up;           // FFN_GRAD: C has the gate's columns from 0 and up's from `up` on
    void *C;
    int64_t ldc;
    const void *bias;     // [N], FFN_GATE: [2 N]; null = none
    float *pre;           // [M][2 N]: FFN_GATE writes it (null = not), FFN_GRAD reads it
    void *h;              // [M][ldh], FFN_GRAD writes h; FFN_GATE what C's rounding leaves over (null = not)
    int64_t ldh;
    bool pad;             // C's rows are padded (to 8 columns) for the next product: zeros go behind the last column
    float *cols;          // [row blocks][2 N], FFN_GRAD in 16 bits writes its column sums over blocks of rows (null = not)
    int32_t act;
    // sums over slices of k: slice s writes part[s][M][N or 2 N] in place of the epilogue
    float *part;
    int32_t splits, k_slice;
    int32_t tiles_m, tiles_n;
};

// The activation and its derivative.  exp() in fp32 rows, the hardware's base-2 exponential in the 16-bit ones (2^-22
// against the type's 2^-11 or 2^-8).
template <int KIND> __device__ __forceinline__ float ffn_exp(float z) {
    return KIND == ANN_F32 ? expf(z) : __builtin_amdgcn_exp2f(1.4426950408889634f * z);
}
template <int KIND> __device__ __forceinline__ float ffn_sigmoid(float z) {
    return KIND == ANN_F32 ? 1.0f / (1.0f + expf(-z)) : sigmoid_hw(z);
}
// W of them; the choice is the same for the whole call, so it is taken once.
template <int KIND, int W, bool SLOPE>
__device__ __forceinline__ void ffn_act_each(int act, const float *z, float *value, float *slope) {
    if (act == ANN_SILU || act == ANN_SIGMOID) {
        const bool silu = act == ANN_SILU;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float sig = ffn_sigmoid<KIND>(z[i]);
            value[i] = silu ? z[i] * sig : sig;
            if (SLOPE) {
                // 1 - sig = exp(-z) sig, which keeps its bits where sig is near 1; exp(-z) overflows where sig is 0
                const float e = ffn_exp<KIND>(-z[i]), t = sig * (e < __builtin_inff() ? e * sig : 1.0f);
                slope[i] = silu ? sig + z[i] * t : t;
            }
        }
    } else if (act == ANN_GELU) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float cdf = 0.5f * erfcf(z[i] * -0.70710678118654752f);  // as (1 + erf) / 2 it would end at z = -5
            value[i] = z[i] * cdf;
            if (SLOPE) slope[i] = cdf + z[i] * (0.39894228040143268f * ffn_exp<KIND>(-0.5f * z[i] * z[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            value[i] = z[i] <= 0.f ? 0.f : z[i];  // NaN stays NaN
            if (SLOPE) slope[i] = z[i] > 0.f ? 1.f : 0.f;
        }
    }
}

// W consecutive elements (8 to 32 bytes), the first `left` of them.
template <typename T, int W> struct __attribute__((packed, aligned(sizeof(T)))) PackOf {
    typedef T type __attribute__((ext_vector_type(W)));
    type v;
};
template <int W, typename T> __device__ __forceinline__ void load_cols(const T *p, int left, float *v) {
    constexpr int P = W * sizeof(T) > 16 ? 16 / sizeof(T) : W;  // elements of an access
    if (left >= W) {
#pragma unroll
        for (int i = 0; i < W; i += P) {
            const typename PackOf<T, P>::type t = reinterpret_cast<const PackOf<T, P> *>(p + i)->v;
#pragma unroll
            for (int j = 0; j < P; ++j) v[i + j] = (float)t[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}
template <int W, typename T> __device__ __forceinline__ void store_cols(T *p, int left, const float *v) {
    constexpr int P = W * sizeof(T) > 16 ? 16 / sizeof(T) : W;
    if (left >= W) {
#pragma unroll
        for (int i = 0; i < W; i += P) {
            typename PackOf<T, P>::type t;
#pragma unroll
            for (int j = 0; j < P; ++j) t[j] = (T)v[i + j];
            reinterpret_cast<PackOf<T, P> *>(p + i)->v = t;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

// What an epilogue reads of row m for W columns from n on; fetched ahead of the sums where that hides its way.
template <int W> struct FfnRow {
    float gate[W], up[W];
};
template <int W, int EPI, bool INSIDE = false>
__device__ __forceinline__ void ffn_row(const FfnArgs &p, int64_t m, int n, FfnRow<W> &r) {
    if (EPI == FFN_GRAD) {
        const float *__restrict__ q = p.pre + m * 2 * p.N + n;
        load_cols<W>(q, INSIDE ? W : p.N - n, r.gate);
        load_cols<W>(q + p.N, INSIDE ? W : p.N - n, r.up);
    }
}

struct FfnTrue {
    static constexpr bool value = true;
};
struct FfnFalse {
    static constexpr bool value = false;
};

// W consecutive columns from n on of row m (the caller has m < M, n < N); `up` for FFN_GATE only.  INSIDE: all of the
// tile's columns are inside, so that nothing is padded either.  dgate, dup: what FFN_GRAD writes, before its rounding.
template <int KIND, int EPI, int W, bool INSIDE = false>
__device__ __forceinline__ void ffn_epilogue(const FfnArgs &p, int64_t m, int n, const float *sum, const float *up,
                                             const FfnRow<W> &r, float *dgate = nullptr, float *dup = nullptr) {
    using T = typename ElemOf<KIND>::type;
    const int left = INSIDE ? W : p.N - n;
    T *C = (T *)p.C + m * p.ldc + n;
    float v[W], w[W];
    if (EPI == FFN_STORE) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = sum[i];
        if (p.bias) {
            load_cols<W>((const T *)p.bias + n, left, w);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] += w[i];
        }
        store_cols<W>(C, left, v);
    } else if (EPI == FFN_GATE) {
        float g[W], u[W];
#pragma unroll
        for (int i = 0; i < W; ++i) g[i] = sum[i], u[i] = up[i];
        if (p.bias) {
            load_cols<W>((const T *)p.bias + n, left, v);
            load_cols<W>((const T *)p.bias + p.N + n, left, w);
#pragma unroll
            for (int i = 0; i < W; ++i) g[i] += v[i], u[i] += w[i];
        }
        if (p.pre) {
            float *q = p.pre + m * 2 * p.N + n;
            store_cols<W>(q, left, g);
            store_cols<W>(q + p.N, left, u);
        }
        ffn_act_each<KIND, W, false>(p.act, g, v, nullptr);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= u[i];
        store_cols<W>(C, left, v);
        if (p.h) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float kept = (float)(T)v[i];
                v[i] = __builtin_isinf(kept) ? 0.f : v[i] - kept;
            }
            store_cols<W>((T *)p.h + m * p.ldh + n, left, v);
        }
        if (!INSIDE && p.pad && left <= W)
            for (int64_t i = p.N; i < p.ldc; ++i) ((T *)p.C + m * p.ldc)[i] = (T)0.f;
    } else {
        float a[W], slope[W];
        ffn_act_each<KIND, W, true>(p.act, r.gate, a, slope);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[i] = sum[i] * r.up[i] * slope[i];
            w[i] = sum[i] * a[i];
            a[i] *= r.up[i];
            if (dgate) dgate[i] = v[i], dup[i] = w[i];
        }
        store_cols<W>(C, left, v);
        store_cols<W>(C + p.up, left, w);
        if (!INSIDE && p.pad && left <= W)
            for (int64_t i = p.up + p.N; i < p.ldc; ++i) ((T *)p.C + m * p.ldc)[i] = (T)0.f;
        if (p.h) store_cols<W>((T *)p.h + m * p.ldh + n, left, a);
    }
}

// The tile and slice of a workgroup.  Workgroups go round the 8 XCDs in turn; each XCD gets a run of consecutive tiles,
// which lie in blocks 8 tiles of rows high, so that the tiles an XCD works on at a time share rows and columns in its L2.
struct FfnTile {
    int m, n, split;
};
__device__ __forceinline__ FfnTile ffn_tile(const FfnArgs &p) {
    const int total = gridDim.x, q = total >> 3, r = total & 7, xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    int id = xcd * q + (xcd < r ? xcd : r) + at;
    const int tiles = p.tiles_m * p.tiles_n;
    FfnTile t;
    t.split = id / tiles;
    id -= t.split * tiles;
    const int band = id / (8 * p.tiles_n), first = band * 8;
    const int high = p.tiles_m - first < 8 ? p.tiles_m - first : 8;
    id -= band * 8 * p.tiles_n;
    t.n = id / high;
    t.m = first + id - t.n * high;
    return t;
}

// One product: a_rows / b_rows = the operand's k are contiguous.
struct FfnProduct {
    FfnArgs args;
    int kind, epi;
    bool a_rows, b_rows;
};
// How it is cut: tiles of rows x cols (FFN_GATE: half as many columns of C), k in `splits` slices.
struct FfnCut {
    int rows, cols, splits;
};
FfnCut ffn_cut(int kind, int64_t M, int64_t N, int64_t K, int epi);
// Row blocks of FfnArgs::cols: two a tile.
inline int64_t ffn_col_blocks(int64_t M, int tile) { return (M + tile - 1) / tile * 2; }
size_t ffn_part_floats(int kind, int64_t M, int64_t N, int64_t K, int epi);  // what launch_ffn_product needs as `part`
int launch_ffn_product(const FfnProduct &p, float *part, hipStream_t stream);

template <int KIND> int launch_ffn16(const FfnProduct &p, int tile, hipStream_t stream);  // ffn_bf16.hip, ffn_f16.hip
int launch_ffn32(const FfnProduct &p, int cols, hipStream_t stream);                      // ffn_f32.hip

// ffn_few.hip: the same for few rows, both operands' k contiguous, any alignment; FFN_STORE and FFN_GATE, no slices.
// Up to how many rows they are taken, with the kernels' times (few rows / tiles and the joining of their slices, us) at the
// lines, for 2048 -> 2 x 8192 -> 2048, 1024 -> 2 x 4096 -> 1024 and 512 -> 2 x 2048 -> 128, four blocks' weights in turn:
//   FFN_GATE, 16 bits, 64: 23 / 24, 10 / 14 and 6 / 10 with 64 rows; more have no kernel here.
//   FFN_GATE, fp32, 16: 36 / 84, 11 / 28 and 7 / 18 with 16 rows; more would gain too (with 64 rows 61 / 82, 21 / 29, 12 / 19), but
//     have no kernel here.
//   FFN_STORE, 16 bits, 8, up to where h comes in two parts: 14 / 16, 8 / 10 and 6 / 9 with 8 rows.  With h in one part the lead
//     ends later: 15 / 16, 8 / 11 and 5 / 9 with 9 rows, 17 / 16, 9 / 11 and 6 / 9 with 16.
//   FFN_STORE, fp32, 16: with 8 rows 24 / 31, 10 / 13 and 6 / 11, with 9 33 / 30, 15 / 13 and 9 / 13, with 16 37 / 30, 17 / 13 and
//     10 / 13: from 9 rows on narrow outputs gain what wide ones lose.
constexpr int ffn_few(int kind, int epi) { return kind == ANN_F32 ? 16 : epi == FFN_GATE ? 64 : 8; }
int launch_ffn_few(const FfnProduct &p, hipStream_t stream);

// 16-bit operands as launch_ffn16 takes them: 16-byte aligned rows, the contiguous extent a multiple of 8, and 256 rows
// within 2^30 bytes.
inline bool ffn_direct(const void *p, int64_t ld, int64_t width) {
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && width % 8 == 0 && ld <= (int64_t)1 << 21;
}
// rows.hip: up to four copies out [rows][ld_out] = in [rows][width], zeros in the columns behind, of 16-bit elements, in one launch
struct PadRows {
    struct Item {
        const void *in;
        int64_t ld_in, rows, width;
        void *out;
        int64_t ld_out;
    } item[4];
    int n;
};
int launch_pad_rows(const PadRows &p, hipStream_t stream);

}  // namespace gmpgr
