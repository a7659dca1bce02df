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
    int64_t lda, ldb;
    int32_t M, N, K;      // FFN_GATE: N = d_hidden, B has 2 N rows
    void *C;
    int64_t ldc;
    const void *bias;     // [N], FFN_GATE: [2 N]; null = none
    float *pre;           // [M][2 N]: FFN_GATE writes it (null = not), FFN_GRAD reads it
    void *h;              // [M][N], FFN_GRAD writes it (null = not)
    int32_t act;
    // sums over slices of k: slice s writes part[s][M][N or 2 N] in place of the epilogue
    float *part;
    int32_t splits, k_slice;
    int32_t tiles_m, tiles_n;
};

struct ActValue {
    float value, slope;
};

// The activation and its derivative.  exp() in fp32 rows, the hardware's base-2 exponential in the 16-bit ones (2^-22
// against the type's 2^-11 or 2^-8).
template <int KIND> __device__ __forceinline__ float ffn_exp(float z) {
    return KIND == ANN_F32 ? expf(z) : __builtin_amdgcn_exp2f(1.4426950408889634f * z);
}
template <int KIND> __device__ __forceinline__ float ffn_sigmoid(float z) {
    return KIND == ANN_F32 ? 1.0f / (1.0f + expf(-z)) : sigmoid_hw(z);
}
template <int KIND> __device__ __forceinline__ ActValue ffn_act(int act, float z) {
    if (act == ANN_RELU) return {z > 0.f ? z : (z <= 0.f ? 0.f : z), z > 0.f ? 1.f : 0.f};  // NaN stays NaN
    if (act == ANN_GELU) {
        const float cdf = 0.5f * (1.0f + erff(z * 0.70710678118654752f));
        return {z * cdf, cdf + z * (0.39894228040143268f * ffn_exp<KIND>(-0.5f * z * z))};
    }
    const float sig = ffn_sigmoid<KIND>(z);
    if (act == ANN_SILU) return {z * sig, sig * (1.0f + z * (1.0f - sig))};
    return {sig, sig * (1.0f - sig)};
}

// Four consecutive elements, the first `left` of them.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Pack4 {
    typedef T type __attribute__((ext_vector_type(4)));
    type v;
};
template <typename T> __device__ __forceinline__ void store4(T *p, int left, const float *v) {
    if (left >= 4) {
        typename Pack4<T>::type o = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        reinterpret_cast<Pack4<T> *>(p)->v = o;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}
template <typename T> __device__ __forceinline__ void load4(const T *p, int left, float *v) {
    if (left >= 4) {
        const typename Pack4<T>::type t = reinterpret_cast<const Pack4<T> *>(p)->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}

// Four consecutive columns n .. n + 3 of row m (the caller has m < M, n < N); `up` for FFN_GATE only.
template <int KIND, int EPI>
__device__ __forceinline__ void ffn_epilogue(const FfnArgs &p, int64_t m, int n, const float *sum, const float *up) {
    using T = typename ElemOf<KIND>::type;
    const int left = p.N - n;
    T *C = (T *)p.C + m * p.ldc + n;
    float v[4], w[4];
    if (EPI == FFN_STORE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = sum[i];
        if (p.bias) {
            load4((const T *)p.bias + n, left, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += w[i];
        }
        store4(C, left, v);
    } else if (EPI == FFN_GATE) {
        float g[4], u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = sum[i], u[i] = up[i];
        if (p.bias) {
            load4((const T *)p.bias + n, left, v);
            load4((const T *)p.bias + p.N + n, left, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] += v[i], u[i] += w[i];
        }
        if (p.pre) {
            float *q = p.pre + m * 2 * p.N + n;
            store4(q, left, g);
            store4(q + p.N, left, u);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ffn_act<KIND>(p.act, g[i]).value * u[i];
        store4(C, left, v);
    } else {
        float g[4], u[4], h[4];
        const float *q = p.pre + m * 2 * p.N + n;
        load4(q, left, g);
        load4(q + p.N, left, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const ActValue a = ffn_act<KIND>(p.act, g[i]);
            h[i] = a.value * u[i];
            v[i] = sum[i] * u[i] * a.slope;
            w[i] = sum[i] * a.value;
        }
        store4(C, left, v);
        store4(C + p.N, left, w);
        if (p.h) store4((T *)p.h + m * p.N + n, left, h);
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

// One product; layouts: a_rows / b_rows = the operand's k are contiguous.  part: ffn_part_floats() floats.
struct FfnProduct {
    FfnArgs args;
    int kind, epi;
    bool a_rows, b_rows;
};
int ffn_splits(int kind, int64_t M, int64_t N, int64_t K, int epi);
size_t ffn_part_floats(int kind, int64_t M, int64_t N, int64_t K, int epi);
int launch_ffn_product(const FfnProduct &p, float *part, hipStream_t stream);

template <int KIND> int launch_ffn16(const FfnProduct &p, hipStream_t stream);  // ffn_bf16.hip, ffn_f16.hip
int launch_ffn32(const FfnProduct &p, hipStream_t stream);                      // ffn_f32.hip

}  // namespace gmpgr
