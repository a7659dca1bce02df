// Products of the gated feed-forward block in fp32, on the matrix cores' fp32 instruction.
//
// A workgroup of 4 waves forms a 128 x 128 tile, a wave 64 x 64 of it out of 32 x 32 x 2 instructions (64 cycles each, so
// the four LDS reads of one float a lane that feed four of them cost next to nothing).  16 of the k at a time lie in
// LDS as [k][row], two buffers, loaded through registers.  Lines are 160 floats apart: the two k that a wave reads at a
// time lie on the two halves of the banks.
#include "ffn.h"

namespace gmpgr {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int F32_BK = 16, F32_LINE = 160, F32_TILE = 128;

template <bool KROWS, bool GATE> struct Operand32 {
    const float *base;
    int64_t ld;
    int32_t rows, up;

    __device__ __forceinline__ void init(const void *p, int64_t ld_, int row0, int rows_, int up_) {
        ld = ld_, rows = rows_ - row0, up = up_;
        base = (const float *)p + (KROWS ? row0 * ld : (int64_t)row0);
    }
    // GATE: rows of the tile go 32 of the gate, the same 32 of up, and so on
    __device__ __forceinline__ int64_t source_row(int r) const {
        if (!GATE) return r < rows ? r : rows - 1;
        const int f = (r >> 6) * 32 + (r & 31);
        return (int64_t)(f < rows ? f : rows - 1) + ((r >> 5) & 1 ? up : 0);
    }
    // 128 x 16 floats as 512 pieces of 4, two a thread
    __device__ __forceinline__ void load(f32x4v *regs, int k0, int K) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = i * 256 + threadIdx.x;
            const int r = KROWS ? c >> 2 : (c & 31) * 4, k = k0 + (KROWS ? (c & 3) * 4 : c >> 5);
            const float *p = KROWS ? base + source_row(r) * ld + k : base + k * ld + r;
            float v[4];
            load_cols<4>(p, KROWS ? K - k : k < K ? rows - r : 0, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) regs[i][e] = v[e];
        }
    }
    static __device__ __forceinline__ void put(float *lds, const f32x4v *regs) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = i * 256 + threadIdx.x;
            if (KROWS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[((c & 3) * 4 + e) * F32_LINE + (c >> 2)] = regs[i][e];
            } else {
                *(f32x4v *)(lds + (c >> 5) * F32_LINE + (c & 31) * 4) = regs[i];
            }
        }
    }
};

template <bool A_ROWS, bool B_ROWS, int EPI> __global__ void __launch_bounds__(256) ffn_mfma32_kernel(FfnArgs p) {
    constexpr bool GATE = EPI == FFN_GATE;
    constexpr int COLS = GATE ? F32_TILE / 2 : F32_TILE, SIZE = F32_BK * F32_LINE;
    __shared__ __attribute__((aligned(16))) float lds[2][2][SIZE];
    const FfnTile t = ffn_tile(p);
    const int m0 = t.m * F32_TILE, n0 = t.n * COLS;
    const int k_first = t.split * p.k_slice, K = k_first + p.k_slice < p.K ? k_first + p.k_slice : p.K;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    Operand32<A_ROWS, false> a;
    Operand32<B_ROWS, GATE> b;
    a.init(p.A, p.lda, m0, p.M, 0);
    b.init(p.B, p.ldb, n0, p.N, p.up);
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    f32x4v ra[2], rb[2];
    a.load(ra, k_first, K);
    b.load(rb, k_first, K);
    a.put(lds[0][0], ra);
    b.put(lds[0][1], rb);
    __syncthreads();
    int buffer = 0;
    for (int k = k_first; k < K; k += F32_BK) {
        const bool more = k + F32_BK < K;
        if (more) {
            a.load(ra, k + F32_BK, K);
            b.load(rb, k + F32_BK, K);
        }
        const float *la = lds[buffer][0] + (lane >> 5) * F32_LINE + wm + (lane & 31);
        const float *lb = lds[buffer][1] + (lane >> 5) * F32_LINE + wn + (lane & 31);
#pragma unroll
        for (int kk = 0; kk < F32_BK; kk += 2) {
            float fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) fa[i] = la[kk * F32_LINE + i * 32], fb[i] = lb[kk * F32_LINE + i * 32];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[j], fa[i], acc[i][j], 0, 0, 0);
        }
        if (more) {
            a.put(lds[buffer ^ 1][0], ra);
            b.put(lds[buffer ^ 1][1], rb);
        }
        __syncthreads();
        buffer ^= 1;
    }
    // A lane has columns 8 q + 4 (lane / 32) .. + 3 of row lane % 32 of every 32 x 32 piece.
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + wm + i * 32 + (lane & 31);
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 2; j += GATE ? 2 : 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + (GATE ? wn / 2 : wn + j * 32) + q * 8 + (lane >> 5) * 4;
                if (n >= p.N) continue;
                float s[4], u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = acc[i][j][q * 4 + e], u[e] = GATE ? acc[i][1][q * 4 + e] : 0.f;
                if (p.part) {
                    const int64_t width = GATE ? 2 * (int64_t)p.N : p.N;
                    float *o = p.part + ((int64_t)t.split * p.M + m) * width + n;
                    store_cols<4>(o, p.N - n, s);
                    if (GATE) store_cols<4>(o + p.N, p.N - n, u);
                } else {
                    FfnRow<4> r;
                    ffn_row<4, EPI>(p, m, n, r);
                    ffn_epilogue<ANN_F32, EPI, 4>(p, m, n, s, u, r);
                }
            }
    }
}

template <bool A_ROWS, bool B_ROWS, int EPI> static int launch_tile32(FfnArgs a, hipStream_t stream) {
    constexpr int COLS = EPI == FFN_GATE ? F32_TILE / 2 : F32_TILE;
    a.tiles_m = (a.M + F32_TILE - 1) / F32_TILE;
    a.tiles_n = (a.N + COLS - 1) / COLS;
    const int64_t total = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    if (total > 0x7fffffff) {
        set_error("a product of %d x %d has too many tiles", a.M, a.N);
        return ANN_ENOTIMPL;
    }
    auto fn = ffn_mfma32_kernel<A_ROWS, B_ROWS, EPI>;
    hipLaunchKernelGGL(fn, dim3((unsigned)total), dim3(256), 0, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

int launch_ffn32(const FfnProduct &p, hipStream_t stream) {
    if (p.epi == FFN_GATE) return launch_tile32<true, true, FFN_GATE>(p.args, stream);
    if (p.epi == FFN_GRAD) return launch_tile32<true, false, FFN_GRAD>(p.args, stream);
    if (p.a_rows && p.b_rows) return launch_tile32<true, true, FFN_STORE>(p.args, stream);
    if (p.a_rows) return launch_tile32<true, false, FFN_STORE>(p.args, stream);
    return launch_tile32<false, false, FFN_STORE>(p.args, stream);
}

}  // namespace gmpgr
