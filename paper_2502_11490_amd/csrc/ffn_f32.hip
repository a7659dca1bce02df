// Products of the gated feed-forward block in fp32, on the matrix cores' fp32 instruction.
//
// A workgroup of 4 waves forms a BM x BN tile, a wave a quarter of it out of 32 x 32 x 2 instructions (64 cycles each, so
// the LDS reads that feed them cost next to nothing).  32 of the k at a time lie in LDS, two buffers, loaded through
// registers: a line of 128 bytes of every row.  Of every 8 k the lower half of a wave takes the first 4 and the upper
// half the others, an instruction one of each: an operand whose k are contiguous then lies as [row][32 k], lines 36
// floats apart, and gives a lane its 4 in one read of 16 bytes (16 lanes on 16 different sets of banks); one whose rows
// are contiguous lies as [k][row], lines 8 floats longer than the tile, so that the two halves' k lie on the two halves of
// the banks.
// 8192 x 1024 x 4096: 610 us, 113 TFLOP/s, in tiles of 128, 674 in tiles of 64; those keep the last round of middling products
// short: 2048 x 1300 x 256 (FFN_GRAD) 33 us against 41.
#include "ffn.h"

namespace gmpgr {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int F32_BK = 32;

// A tile of ROWS rows by 32 k.
template <bool KROWS, bool GATE, int ROWS> struct Operand32 {
    static constexpr int PASSES = ROWS * F32_BK / 4 / 256, LINE = KROWS ? F32_BK + 4 : ROWS + 8, ACROSS = ROWS / 4;
    static constexpr int SIZE = (KROWS ? ROWS : F32_BK) * LINE;
    const float *base;
    int64_t ld;
    int32_t rows, up;
    int64_t offset[PASSES];  // elements from the tile's first row at the step's first k

    __device__ __forceinline__ void init(const void *p, int64_t ld_, int row0, int rows_, int up_) {
        ld = ld_, rows = rows_ - row0, up = up_;
        base = (const float *)p + (KROWS ? row0 * ld : (int64_t)row0);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = i * 256 + threadIdx.x;
            offset[i] = KROWS ? source_row(piece_row(c)) * ld + piece_k(c) : piece_k(c) * ld + piece_row(c);
        }
    }
    // GATE: rows of the tile go 32 of the gate, the same 32 of up, and so on; rows behind the last one repeat it
    __device__ __forceinline__ int64_t source_row(int r) const {
        if (!GATE) return r < rows ? r : rows - 1;
        const int f = (r >> 6) * 32 + (r & 31);
        return (int64_t)(f < rows ? f : rows - 1) + ((r >> 5) & 1 ? up : 0);
    }
    static __device__ __forceinline__ int piece_row(int c) { return KROWS ? c / (F32_BK / 4) : c % ACROSS * 4; }
    static __device__ __forceinline__ int piece_k(int c) { return KROWS ? c % (F32_BK / 4) * 4 : c / ACROSS; }
    // The tile's pieces of 4 floats, PASSES a thread.  Whether anything ends inside the step is one question for the
    // workgroup: with a test per piece the compiler waits for each before it asks for the next.
    __device__ __forceinline__ void load(f32x4v *regs, int k0, int K) const {
        if (k0 + F32_BK <= K && (KROWS || rows >= ROWS)) {
            const float *from = KROWS ? base + k0 : base + k0 * ld;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) regs[i] = reinterpret_cast<const PackOf<float, 4> *>(from + offset[i])->v;
            return;
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = i * 256 + threadIdx.x, r = piece_row(c), k = k0 + piece_k(c);
            const float *p = KROWS ? base + source_row(r) * ld + k : base + k * ld + r;
            const int left = KROWS ? K - k : k < K ? rows - r : 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) regs[i][e] = e < left ? p[e] : 0.f;
        }
    }
    static __device__ __forceinline__ void put(float *lds, const f32x4v *regs) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = i * 256 + threadIdx.x;
            *(f32x4v *)(lds + (KROWS ? c / (F32_BK / 4) * LINE + c % (F32_BK / 4) * 4 : c / ACROSS * LINE + c % ACROSS * 4)) = regs[i];
        }
    }
    // The lane's row (row0 + lane % 32) of the 8 k from k on: 4 of them, one an instruction.
    static __device__ __forceinline__ f32x4v frag(const float *lds, int row0, int k) {
        const int lane = threadIdx.x & 63, r = row0 + (lane & 31);
        k += (lane >> 5) * 4;
        if (KROWS) return *(const f32x4v *)(lds + r * LINE + k);
        return f32x4v{lds[k * LINE + r], lds[(k + 1) * LINE + r], lds[(k + 2) * LINE + r], lds[(k + 3) * LINE + r]};
    }
};

template <bool A_ROWS, bool B_ROWS, int EPI, int BM, int BN> __global__ void __launch_bounds__(256, 2) ffn_mfma32_kernel(FfnArgs p) {
    constexpr bool GATE = EPI == FFN_GATE;
    constexpr int COLS = GATE ? BN / 2 : BN;
    // waves as 2 x 2; GATE with 64 columns (32 of the gate, the same 32 of up): 4 x 1, so that a wave has both
    constexpr int WN = GATE && BN == 64 ? 1 : 2, WM = 4 / WN, MW = BM / WM / 32, NW = BN / WN / 32;
    using OpA = Operand32<A_ROWS, false, BM>;
    using OpB = Operand32<B_ROWS, GATE, BN>;
    constexpr int SIZE_A = OpA::SIZE, BUFFER = SIZE_A + OpB::SIZE;
    extern __shared__ __attribute__((aligned(16))) float lds32[];
    const FfnTile t = ffn_tile(p);
    const int m0 = t.m * BM, n0 = t.n * COLS;
    const int k_first = t.split * p.k_slice, K = k_first + p.k_slice < p.K ? k_first + p.k_slice : p.K;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    OpA a;
    OpB b;
    a.init(p.A, p.lda, m0, p.M, 0);
    b.init(p.B, p.ldb, n0, p.N, p.up);
    f32x16 acc[MW][NW];
#pragma unroll
    for (int i = 0; i < MW; ++i)
#pragma unroll
        for (int j = 0; j < NW; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    f32x4v ra[OpA::PASSES], rb[OpB::PASSES];
    a.load(ra, k_first, K);
    b.load(rb, k_first, K);
    a.put(lds32, ra);
    b.put(lds32 + SIZE_A, rb);
    __syncthreads();
    int buffer = 0;
    for (int k = k_first; k < K; k += F32_BK) {
        const bool more = k + F32_BK < K;
        if (more) {
            a.load(ra, k + F32_BK, K);
            b.load(rb, k + F32_BK, K);
        }
        const float *now = lds32 + buffer * BUFFER;
#pragma unroll
        for (int kk = 0; kk < F32_BK; kk += 8) {
            f32x4v fa[MW], fb[NW];
#pragma unroll
            for (int i = 0; i < MW; ++i) fa[i] = OpA::frag(now, wm + i * 32, kk);
#pragma unroll
            for (int j = 0; j < NW; ++j) fb[j] = OpB::frag(now + SIZE_A, wn + j * 32, kk);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MW; ++i)
#pragma unroll
                    for (int j = 0; j < NW; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[j][e], fa[i][e], acc[i][j], 0, 0, 0);
        }
        if (more) {
            a.put(lds32 + (buffer ^ 1) * BUFFER, ra);
            b.put(lds32 + (buffer ^ 1) * BUFFER + SIZE_A, rb);
        }
        __syncthreads();
        buffer ^= 1;
    }
    // A lane has columns 8 q + 4 (lane / 32) .. + 3 of row lane % 32 of every 32 x 32 piece.
#pragma unroll
    for (int i = 0; i < MW; ++i) {
        const int64_t m = m0 + wm + i * 32 + (lane & 31);
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < NW; j += GATE ? 2 : 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + (GATE ? wn / 2 : wn + j * 32) + q * 8 + (lane >> 5) * 4;
                if (n >= p.N) continue;
                float s[4], u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = acc[i][j][q * 4 + e], u[e] = GATE ? acc[i][NW - 1][q * 4 + e] : 0.f;
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

template <bool A_ROWS, bool B_ROWS, int EPI, int BM, int BN> static int launch_tile32(FfnArgs a, hipStream_t stream) {
    constexpr int COLS = EPI == FFN_GATE ? BN / 2 : BN;
    constexpr size_t LDS = 2 * (Operand32<A_ROWS, false, BM>::SIZE + Operand32<B_ROWS, EPI == FFN_GATE, BN>::SIZE) * sizeof(float);
    static std::atomic<uint32_t> done{0};
    auto fn = ffn_mfma32_kernel<A_ROWS, B_ROWS, EPI, BM, BN>;
    int device = 0;
    ANN_HIP_TRY(hipGetDevice(&device));
    const int rc = raise_lds_limit((const void *)fn, LDS, device, done);
    if (rc != ANN_OK) return rc;
    a.tiles_m = (a.M + BM - 1) / BM;
    a.tiles_n = (a.N + COLS - 1) / COLS;
    const int64_t total = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    if (total > 0x7fffffff) {
        set_error("a product of %d x %d has too many tiles", a.M, a.N);
        return ANN_ENOTIMPL;
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)total), dim3(256), LDS, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}
template <bool A_ROWS, bool B_ROWS, int EPI> static int launch_layout32(const FfnArgs &a, int cols, hipStream_t stream) {
    return cols == 128 ? launch_tile32<A_ROWS, B_ROWS, EPI, 128, 128>(a, stream)
                       : launch_tile32<A_ROWS, B_ROWS, EPI, EPI == FFN_GATE ? 128 : 64, 64>(a, stream);
}

int launch_ffn32(const FfnProduct &p, int cols, hipStream_t stream) {
    if (p.epi == FFN_GATE) return launch_layout32<true, true, FFN_GATE>(p.args, cols, stream);
    if (p.epi == FFN_GRAD) return launch_layout32<true, false, FFN_GRAD>(p.args, cols, stream);
    if (p.a_rows && p.b_rows) return launch_layout32<true, true, FFN_STORE>(p.args, cols, stream);
    if (p.a_rows) return launch_layout32<true, false, FFN_STORE>(p.args, cols, stream);
    return launch_layout32<false, false, FFN_STORE>(p.args, cols, stream);
}

}  // namespace gmpgr
