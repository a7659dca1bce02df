// Products of the gated feed-forward block in the 16-bit types, on the matrix cores.
//
// A workgroup forms a BM x BN tile of C; its WM x WN waves each a part of (BM / WM) x (BN / WN) out of 16 x 16 x 32
// matrix instructions.  64 of the k at a time lie in LDS, in two buffers: the next ones are on their way while the
// present ones are multiplied.  An operand whose k are contiguous lies as [row][64 k], 128 bytes a row in 8 pieces
// of 16, piece c at place c ^ (row & 7), and is read a piece a lane; one whose rows are contiguous lies as [64 k][rows],
// and is read by the transposing LDS read (16 lanes fetch 4 k of 16 rows and get 4 k of a row each), its pieces at
// c ^ 2 ((k & 3) | (k >> 3 & 1) << 2), which puts the eight k that half a wave reads at a time on eight different sets of banks.
// FAST: global memory is loaded straight into LDS (16 bytes a lane, addresses in lane order, so the
// permutation is in what a lane loads); it needs 16-byte aligned rows.  Otherwise through registers, any alignment.
#pragma once

#include "ffn.h"

namespace gmpgr {

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int KIND> struct Frag16;
template <> struct Frag16<ANN_BF16> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(type a, type b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Frag16<ANN_F16> {
    typedef _Float16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(type a, type b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

constexpr int FFN_BK = 64;
constexpr uint32_t FFN_NOWHERE = 0x80000000u;  // an offset outside every buffer: such a load gives zeros

// One operand's tile of ROWS rows by 64 k, loaded by THREADS threads.
template <int KIND, bool KROWS, bool GATE, bool FAST, int ROWS, int THREADS>
struct Operand16 {
    using T = typename ElemOf<KIND>::type;
    static constexpr int PASSES = ROWS * 8 / THREADS;
    static constexpr int BYTES = ROWS * FFN_BK * 2;
    static constexpr int ACROSS = ROWS / 8;  // pieces of a line of [64 k][rows]

    const T *base;   // the tile's first row at k = 0
    int64_t ld;
    int32_t rows;    // rows of the operand from the tile's first on; GATE: of one half
    int32_t up;      // GATE: rows from a gate row to its up row
    uint32_t offset[FAST ? PASSES : 1];

    // Piece c of the tile: which row (or first row) and k of the tile it holds.
    static __device__ __forceinline__ int piece_row(int c) {
        return KROWS ? c >> 3 : ((c & (ACROSS - 1)) ^ swizzle(c / ACROSS)) * 8;
    }
    static __device__ __forceinline__ int piece_k(int c) { return KROWS ? ((c & 7) ^ ((c >> 3) & 7)) * 8 : c / ACROSS; }
    static __device__ __forceinline__ int swizzle(int k) { return 2 * ((k & 3) | ((k >> 3) & 1) << 2); }
    // GATE: rows of the tile go 16 of the gate, the same 16 of up, and so on
    __device__ __forceinline__ int64_t source_row(int r) const {
        if (!GATE) return r < rows ? r : rows - 1;
        const int f = (r >> 5) * 16 + (r & 15);
        return (int64_t)(f < rows ? f : rows - 1) + ((r >> 4) & 1 ? up : 0);
    }

    __device__ __forceinline__ void init(const void *p, int64_t ld_, int row0, int rows_, int up_) {
        ld = ld_, rows = rows_ - row0, up = up_;
        base = (const T *)p + (KROWS ? row0 * ld : (int64_t)row0);
        if (FAST)
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int c = i * THREADS + threadIdx.x, r = piece_row(c), k = piece_k(c);
                offset[i] = KROWS ? (uint32_t)((source_row(r) * ld + k) * 2)
                                  : r < rows ? (uint32_t)((k * ld + r) * 2) : FFN_NOWHERE;
            }
    }

    // FAST: sends for the pieces from k0 on (those at k >= K: zeros)
    __device__ __forceinline__ void fetch(char *lds, int k0, int K) const {
        const T *from = KROWS ? base + k0 : base + k0 * ld;
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)from, 0, 0x7fffffff, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const uint32_t o = k0 + piece_k(i * THREADS + threadIdx.x) < K ? offset[i] : FFN_NOWHERE;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LdsPtr)(lds + (i * THREADS + wave * 64) * 16), 16, o, 0, 0, 0);
        }
    }

    // otherwise: into registers, and from them into LDS
    __device__ __forceinline__ void load(s16x8 *regs, int k0, int K) const {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = i * THREADS + threadIdx.x, r = piece_row(c), k = k0 + piece_k(c);
            const T *p = KROWS ? base + source_row(r) * ld + k : base + k * ld + r;
            const int left = KROWS ? K - k : k < K ? rows - r : 0;
            s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
            if (left >= 8) {
                v = __builtin_bit_cast(s16x8, load16(p));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) v[j] = __builtin_bit_cast(short, p[j]);
            }
            regs[i] = v;
        }
    }
    static __device__ __forceinline__ void put(char *lds, const s16x8 *regs) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) *(s16x8 *)(lds + (i * THREADS + threadIdx.x) * 16) = regs[i];
    }

    // The operand of a matrix instruction: rows row0 .. row0 + 15 (a lane's: row0 + lane % 16), k 32 ks + 8 (lane / 16) + 0 .. 7
    static __device__ __forceinline__ typename Frag16<KIND>::type frag(const char *lds, int row0, int ks) {
        const int lane = threadIdx.x & 63, kg = lane >> 4, l = lane & 15;
        if (KROWS) {
            const int r = row0 + l;
            return *(const typename Frag16<KIND>::type *)(lds + r * 128 + (((ks * 4 + kg) ^ (r & 7)) << 4));
        }
        const int k = ks * 32 + kg * 8 + (l >> 2);
        const int place = ((row0 >> 3) + ((l >> 1) & 1)) ^ (2 * ((l >> 2) | (kg & 1) << 2));
        const char *p = lds + k * (ROWS * 2) + place * 16 + (l & 1) * 8;
        typedef __attribute__((address_space(3))) s16x4 *Quad;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad)(p + 4 * ROWS * 2));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(typename Frag16<KIND>::type, v);
    }
};

template <int KIND, bool A_ROWS, bool B_ROWS, bool FAST, int EPI, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM *WN * 64) ffn_mfma16_kernel(FfnArgs p) {
    constexpr int THREADS = WM * WN * 64, MT = BM / WM / 16, NT = BN / WN / 16;
    constexpr bool GATE = EPI == FFN_GATE;
    constexpr int COLS = GATE ? BN / 2 : BN;  // columns of C
    using OpA = Operand16<KIND, A_ROWS, false, FAST, BM, THREADS>;
    using OpB = Operand16<KIND, B_ROWS, GATE, FAST, BN, THREADS>;
    constexpr int BUFFER = OpA::BYTES + OpB::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const FfnTile t = ffn_tile(p);
    const int m0 = t.m * BM, n0 = t.n * COLS;
    const int k_first = t.split * p.k_slice, K = k_first + p.k_slice < p.K ? k_first + p.k_slice : p.K;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    OpA a;
    OpB b;
    a.init(p.A, p.lda, m0, p.M, 0);
    b.init(p.B, p.ldb, n0, p.N, p.N);

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    s16x8 ra[FAST ? 1 : OpA::PASSES], rb[FAST ? 1 : OpB::PASSES];
    if (FAST) {
        a.fetch(lds, k_first, K);
        b.fetch(lds + OpA::BYTES, k_first, K);
    } else {
        a.load(ra, k_first, K);
        b.load(rb, k_first, K);
        OpA::put(lds, ra);
        OpB::put(lds + OpA::BYTES, rb);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int buffer = 0;
    for (int k = k_first; k < K; k += FFN_BK) {
        char *now = lds + buffer * BUFFER, *next = lds + (buffer ^ 1) * BUFFER;
        const bool more = k + FFN_BK < K;
        if (more) {
            if (FAST) {
                a.fetch(next, k + FFN_BK, K);
                b.fetch(next + OpA::BYTES, k + FFN_BK, K);
            } else {
                a.load(ra, k + FFN_BK, K);
                b.load(rb, k + FFN_BK, K);
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            typename Frag16<KIND>::type fa[MT], fb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[j] = OpB::frag(now + OpA::BYTES, wn + j * 16, ks);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[i] = OpA::frag(now, wm + i * 16, ks);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = Frag16<KIND>::mfma(fb[j], fa[i], acc[i][j]);
        }
        if (!FAST && more) {
            OpA::put(next, ra);
            OpB::put(next + OpA::BYTES, rb);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        buffer ^= 1;
    }

    // A lane has columns 4 (lane / 16) .. + 3 of row lane % 16 of every 16 x 16 piece.
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + wm + i * 16 + (lane & 15);
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < NT; j += GATE ? 2 : 1) {
            const int n = n0 + (GATE ? (wn + j * 16) / 2 : wn + j * 16) + (lane >> 4) * 4;
            if (n >= p.N) continue;
            float s[4], u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = acc[i][j][e], u[e] = GATE ? acc[i][j + (GATE ? 1 : 0)][e] : 0.f;
            if (p.part) {
                const int64_t width = GATE ? 2 * (int64_t)p.N : p.N;
                float *q = p.part + ((int64_t)t.split * p.M + m) * width + n;
                store4(q, p.N - n, s);
                if (GATE) store4(q + p.N, p.N - n, u);
            } else {
                ffn_epilogue<KIND, EPI>(p, m, n, s, u);
            }
        }
    }
}

template <int KIND, bool A_ROWS, bool B_ROWS, bool FAST, int EPI, int BM, int BN, int WM, int WN>
int launch_tile16(FfnArgs a, hipStream_t stream) {
    constexpr size_t LDS = 2 * (size_t)(BM + BN) * FFN_BK * 2;
    constexpr int COLS = EPI == FFN_GATE ? BN / 2 : BN;
    static std::atomic<uint32_t> done{0};
    auto fn = ffn_mfma16_kernel<KIND, A_ROWS, B_ROWS, FAST, EPI, BM, BN, WM, WN>;
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
    hipLaunchKernelGGL(fn, dim3((unsigned)total), dim3(WM * WN * 64), LDS, stream, a);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

// Rows that 16-byte loads straight into LDS can take: 16-byte aligned, pieces that do not straddle an end, and offsets
// inside a tile that fit 31 bits.
inline bool direct_operand(const void *p, int64_t ld, bool k_rows, int64_t rows, int64_t K, int64_t up) {
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && (k_rows ? K : rows) % 8 == 0 && ((k_rows ? up : 0) + 256) * ld < ((int64_t)1 << 30);
}

template <int KIND, bool A_ROWS, bool B_ROWS, int EPI> int launch_layout16(const FfnArgs &a, hipStream_t stream) {
    const bool fast = direct_operand(a.A, a.lda, A_ROWS, a.M, a.K, 0) &&
                      direct_operand(a.B, a.ldb, B_ROWS, a.N, a.K, EPI == FFN_GATE ? a.N : 0);
    return fast ? launch_tile16<KIND, A_ROWS, B_ROWS, true, EPI, 128, 128, 2, 2>(a, stream)
                : launch_tile16<KIND, A_ROWS, B_ROWS, false, EPI, 128, 128, 2, 2>(a, stream);
}

template <int KIND> int launch_ffn16(const FfnProduct &p, hipStream_t stream) {
    if (p.epi == FFN_GATE) return launch_layout16<KIND, true, true, FFN_GATE>(p.args, stream);
    if (p.epi == FFN_GRAD) return launch_layout16<KIND, true, false, FFN_GRAD>(p.args, stream);
    if (p.a_rows && p.b_rows) return launch_layout16<KIND, true, true, FFN_STORE>(p.args, stream);
    if (p.a_rows) return launch_layout16<KIND, true, false, FFN_STORE>(p.args, stream);
    return launch_layout16<KIND, false, false, FFN_STORE>(p.args, stream);
}

}  // namespace gmpgr
