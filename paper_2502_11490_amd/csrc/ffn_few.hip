// Products of the gated feed-forward block for few rows (one request, a handful of them): C = x w^T with M <= 64.
//
// Bound by reading w once; nothing of it is used twice, so it goes from memory straight into the registers of the
// matrix instruction.  A wave takes 16 RT rows of w (FFN_GATE: of the gate, and the same of up) and every KW-th step of
// the k, a workgroup's KW waves the others, joined in LDS in order.  A step is 128 bytes of every row: lane l has the 32
// bytes l / 16 of row l % 16, of w as of x, and the instruction's k are numbered accordingly on both sides; a line of w is
// read whole, by 4 lanes, at whatever address it begins.  With 4 (8) rows of x at most, the instruction's 16 rows are 4
// (8) rows in 4 (2) slices of a step: four times the workgroups, so that few columns still occupy every compute unit, and of
// the 16 x 16 sums the blocks on the diagonal are added.  h comes in two 16-bit parts, its rounding and what that leaves
// over: the instructions are idle anyway, and out is then as near as from an fp32 h.  Several steps' loads are on their way together.
// One bf16 row through 2048 -> 2 x 8192 (67 MB): 13 to 14 us, 4.7 to 5.1 TB/s; 8192 -> 2048 (34 MB): 9.3 to 10 us, 3.3 to 3.6
// TB/s (without slices 11.6 us, with h in one part 8.5 us).  In fp32: 31 us (134 MB, 4.3 TB/s) and 16 us (67 MB, 4.3 TB/s).
#include "ffn.h"

namespace gmpgr {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 rows by 128 bytes of k, as the matrix instruction takes them: the lane's 32 bytes.
template <int KIND> struct FewFrag {
    using T = typename ElemOf<KIND>::type;
    using P = typename Pack16<T>::type;
    static constexpr int V = VEC<T>, K = 8 * V;  // elements of 16 bytes, k of a step
    P part[2];
    // the step's k begin at k and are `step` many, the lane's at `first` of them and at 2 V times its number of 16
    __device__ __forceinline__ void load(const T *row, int k, int first, int step, int K_end) {
        const int at = k + first + ((threadIdx.x & 63) >> 4) * 2 * V;
        if (k + step <= K_end) {  // the whole wave: nothing ends inside the step
            part[0] = load16(row + at);
            part[1] = load16(row + at + V);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < V; ++i) part[h][i] = at + h * V + i < K_end ? row[at + h * V + i] : (T)0.f;
        }
    }
    static __device__ __forceinline__ f32x4 product(const FewFrag &w, const FewFrag &x, f32x4 sum) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (KIND == ANN_BF16) {
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[h], x.part[h], sum, 0, 0, 0);
            } else if constexpr (KIND == ANN_F16) {
                sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.part[h], x.part[h], sum, 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sum = __builtin_amdgcn_mfma_f32_16x16x4f32(w.part[h][i], x.part[h][i], sum, 0, 0, 0);
            }
        }
        return sum;
    }
};

// REST: A_rest is there.
template <int KIND, int EPI, int S, int MT, int RT, bool REST>
__global__ void __launch_bounds__(MT > 1 ? 512 : 1024) ffn_few_kernel(FfnArgs p) {
    using T = typename ElemOf<KIND>::type;
    using Frag = FewFrag<KIND>;
    constexpr int HALVES = EPI == FFN_GATE ? 2 : 1, TILES = HALVES * RT * MT, AHEAD = MT > 1 ? 2 : 4, R = 16 / S;
    extern __shared__ __attribute__((aligned(16))) char few_lds[];
    f32x4 *const joined = (f32x4 *)few_lds;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6, l = lane & 15;
    const int n0 = blockIdx.x * R * RT, first = l / R * Frag::K;  // first: the lane's slice of a step
    const T *w[HALVES * RT], *x[MT];
    const int64_t rest = REST ? (const T *)p.A_rest - (const T *)p.A : 0;
#pragma unroll
    for (int i = 0; i < HALVES * RT; ++i) {
        const int n = n0 + i % RT * R + l % R;
        w[i] = (const T *)p.B + ((int64_t)(n < p.N ? n : p.N - 1) + (i >= RT ? p.up : 0)) * p.ldb;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = (const T *)p.A + (int64_t)(i * 16 + l % R < p.M ? i * 16 + l % R : p.M - 1) * p.lda;
    f32x4 sum[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    // steps go round the waves
    const int stride = waves * S * Frag::K;
    for (int k = wave * S * Frag::K; k < p.K; k += AHEAD * stride) {
        Frag fw[AHEAD][HALVES * RT], fx[AHEAD][MT], fr[REST ? AHEAD : 1][MT];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int at = k + a * stride;
            if (at < p.K) {
#pragma unroll
                for (int i = 0; i < HALVES * RT; ++i) fw[a][i].load(w[i], at, first, S * Frag::K, p.K);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    fx[a][i].load(x[i], at, first, S * Frag::K, p.K);
                    if (REST) fr[REST ? a : 0][i].load(x[i] + rest, at, first, S * Frag::K, p.K);
                }
            }
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if (k + a * stride < p.K)
#pragma unroll
                for (int i = 0; i < HALVES * RT; ++i)
#pragma unroll
                    for (int j = 0; j < MT; ++j) {
                        sum[i * MT + j] = Frag::product(fw[a][i], fx[a][j], sum[i * MT + j]);
                        if (REST) sum[i * MT + j] = Frag::product(fw[a][i], fr[REST ? a : 0][j], sum[i * MT + j]);
                    }
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) joined[(wave * TILES + i) * 64 + lane] = sum[i];
    __syncthreads();
    // A lane of a 16 x 16 piece has rows 4 (lane / 16) .. + 3 of w and row lane % 16 of x.  With slices, row s R + n of
    // w's side belongs with row s R + m of x's: only the R x R blocks on the diagonal count, and they add up.
    constexpr int QUADS = R / 4 * R;  // of R x R outputs
    for (int i = threadIdx.x; i < RT * MT * QUADS; i += blockDim.x) {
        const int tile = i / QUADS, at = i % QUADS, row = at % R, quad = at / R;
        const int m = tile % MT * 16 + row, n = n0 + tile / MT * R + quad * 4;
        if (m >= p.M || n >= p.N) continue;
        f32x4 sum_g = f32x4{0.f, 0.f, 0.f, 0.f}, sum_u = sum_g;
        for (int v = 0; v < waves; ++v)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int from = (s * (R / 4) + quad) * 16 + s * R + row;
                sum_g += joined[(v * TILES + tile) * 64 + from];
                if (EPI == FFN_GATE) sum_u += joined[(v * TILES + RT * MT + tile) * 64 + from];
            }
        const float a[4] = {sum_g[0], sum_g[1], sum_g[2], sum_g[3]}, b[4] = {sum_u[0], sum_u[1], sum_u[2], sum_u[3]};
        FfnRow<4> r;
        ffn_epilogue<KIND, EPI, 4>(p, m, n, a, b, r);
    }
}

template <int KIND, int EPI, int S, int MT, int RT, bool REST = false> static int launch_few(const FfnArgs &a, hipStream_t stream) {
    constexpr int TILES = (EPI == FFN_GATE ? 2 : 1) * RT * MT, ROWS = 16 / S * RT, STEP = FewFrag<KIND>::K * S;
    const int64_t groups = ((int64_t)a.N + ROWS - 1) / ROWS, steps = ((int64_t)a.K + STEP - 1) / STEP;
    // waves of a workgroup: 16 a compute unit in all, each with a step or more, their sums within 64 KB
    int waves = 4;
    while (waves < (MT > 1 ? 8 : 16) && groups * waves < 4096 && waves < steps && waves * 2 * TILES <= 64) waves *= 2;
    hipLaunchKernelGGL((ffn_few_kernel<KIND, EPI, S, MT, RT, REST>), dim3((unsigned)groups), dim3(waves * 64),
                       (size_t)waves * TILES * 1024, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

template <int KIND, int EPI> static int launch_few_rows(const FfnArgs &a, hipStream_t stream) {
    if constexpr (EPI == FFN_STORE && KIND != ANN_F32) {
        if (a.M <= 4) return launch_few<KIND, EPI, 4, 1, 1, true>(a, stream);
        if (a.M <= 8) return launch_few<KIND, EPI, 2, 1, 1, true>(a, stream);
    } else {
        if (a.M <= 4) return launch_few<KIND, EPI, 4, 1, 1>(a, stream);
        if (a.M <= 8) return launch_few<KIND, EPI, 2, 1, 1>(a, stream);
        if (a.M <= 16) return launch_few<KIND, EPI, 1, 1, 1>(a, stream);
    }
    if constexpr (ffn_few(KIND, EPI) > 16) {
        // 32 columns a workgroup, which read x half as often, where that still occupies every compute unit
        if (a.N < 32 * 256) return a.M <= 32 ? launch_few<KIND, EPI, 1, 2, 1>(a, stream) : launch_few<KIND, EPI, 1, 4, 1>(a, stream);
        return a.M <= 32 ? launch_few<KIND, EPI, 1, 2, 2>(a, stream) : launch_few<KIND, EPI, 1, 4, 2>(a, stream);
    }
    set_error("%d rows are too many for this kernel", a.M);
    return ANN_EINVAL;
}

int launch_ffn_few(const FfnProduct &p, hipStream_t stream) {
    const bool gate = p.epi == FFN_GATE;
    if (p.kind == ANN_F32) return gate ? launch_few_rows<ANN_F32, FFN_GATE>(p.args, stream) : launch_few_rows<ANN_F32, FFN_STORE>(p.args, stream);
    if (p.kind == ANN_BF16) return gate ? launch_few_rows<ANN_BF16, FFN_GATE>(p.args, stream) : launch_few_rows<ANN_BF16, FFN_STORE>(p.args, stream);
    return gate ? launch_few_rows<ANN_F16, FFN_GATE>(p.args, stream) : launch_few_rows<ANN_F16, FFN_STORE>(p.args, stream);
}

}  // namespace gmpgr
