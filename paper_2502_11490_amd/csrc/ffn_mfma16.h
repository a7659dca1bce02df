// Products of the gated feed-forward block in the 16-bit types, on the matrix cores.
//
// A workgroup of 4 waves forms a BM x BN tile of C, a wave a quarter of it out of 16 x 16 x 32 matrix instructions.  64
// of the k at a time lie in LDS, in two buffers.  A step goes in two halves of 32 k: while the matrix cores work on
// one half's operands the next half's are read from LDS into a second set of registers, and half way through a
// step, when every wave has read the last of the present buffer and the next one is there, one barrier lets the loads of
// the step after next go out into it.  They have a whole step to arrive.
//   An operand whose k are contiguous lies as [row][64 k], 128 bytes a row in 8 pieces of 16, piece c at place
// c ^ (row & 7), and is read a piece a lane; one whose rows are contiguous lies as [64 k][rows], and is read by the
// transposing LDS read (16 lanes fetch 4 k of 16 rows and get 4 k of a row each), its pieces at
// c ^ 2 ((k & 3) | (k >> 3 & 1) << 2), which puts the eight k that half a wave reads at a time on eight different sets of
// banks.  Global memory is loaded straight into LDS, 16 bytes a lane with addresses in lane order, so the permutation
// is in what a lane loads; operands have 16-byte aligned rows and a contiguous extent that is a multiple of 8 (the
// host packs those that do not).
//   bf16 products M x N x K, in tiles of 256 and, forced, of 128: 8192 x 2048 x 8192 243 us (1.13 PFLOP/s) and 287; with w as
// [k][row], 8192 x 2048 x 16384, 442 us (1.24) and 569; with both as [k][row], 16384 x 2048 x 8192, 473 us (1.16) and 556;
// FFN_GATE 8192 x 2 8192 x 2048 562 us (0.98) and 793; FFN_GRAD 8192 x 8192 x 2048, whose epilogue moves 0.94 GB, 449 and 478.
// (Averages of ten passes; other cards and runs are up to 4 % slower.)
// With the loop's loads into LDS taken out the first three are 197, 406 and 444 us: the matrix instructions bound them, under
// that load's clock, and the loads add 6 to 23 %.  Two workgroups of the 128 tile share a compute unit: 4096 x 2048 x 2048
// 35 us, where the 256 tile has to cut k in two to occupy the units, 40 us and the joining.
#pragma once

#include "ffn.h"
#include "keys.h"  // wave_lds_fence

namespace gmpgr {

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int KIND> struct Frag16;
// The sums stay where they are: the instruction as a statement whose sum is one accumulation register group in place.  (As a
// builtin, with all 256 accumulation registers taken, the compiler moves the groups about: 140 copies a step.)  The
// statement is opaque to the compiler's wait states: its operands come from LDS reads, and the loop ends with the wait states
// of its last sums; the compiled code is tested for both.  (Two wait states in every statement instead: 3 % more time.)
template <> struct Frag16<ANN_BF16> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void mfma(type a, type b, f32x4 &c) {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};
template <> struct Frag16<ANN_F16> {
    typedef _Float16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void mfma(type a, type b, f32x4 &c) {
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
};

constexpr int FFN_BK = 64;
constexpr uint32_t FFN_NOWHERE = 0x80000000u;  // an offset outside every buffer: such a load gives zeros

// One operand's tile of ROWS rows by 64 k, loaded by 256 threads.
template <int KIND, bool KROWS, bool GATE, int ROWS> struct Operand16 {
    using T = typename ElemOf<KIND>::type;
    using Frag = typename Frag16<KIND>::type;
    static constexpr int PASSES = ROWS * 8 / 256;
    static constexpr int BYTES = ROWS * FFN_BK * 2;
    static constexpr int ACROSS = ROWS / 8;  // pieces of a line of [64 k][rows]

    const T *base;   // the tile's first row at k = 0
    int64_t ld;
    int32_t piece_k;             // KROWS: the k of this thread's pieces (of all passes)
    uint32_t offset[PASSES];     // bytes from the tile's first row at the step's first k

    static __device__ __forceinline__ int swizzle(int k) { return 2 * ((k & 3) | ((k >> 3) & 1) << 2); }

    // row0: first row of the tile, rows: of the operand (GATE: of one half, up: rows from a gate row to its up row).
    // GATE: rows of the tile go 16 of the gate, the same 16 of up, and so on.  Rows behind the last one repeat it.
    __device__ __forceinline__ void init(const void *p, int64_t ld_, int row0, int rows, int up) {
        ld = ld_;
        base = (const T *)p + (KROWS ? row0 * ld : (int64_t)row0);
        // a wave's pieces of a pass are all of the gate (the first two waves) or all of up
        if (GATE) base += (int64_t)(__builtin_amdgcn_readfirstlane(threadIdx.x >> 7) * up) * ld;
        piece_k = ((threadIdx.x & 7) ^ ((threadIdx.x >> 3) & 7)) * 8;
        const int last = rows - row0 - 1;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = i * 256 + threadIdx.x;
            if (KROWS) {
                const int r = c >> 3, f = GATE ? (r >> 5) * 16 + (r & 15) : r;
                offset[i] = (uint32_t)(((int64_t)(f < last ? f : last) * ld + piece_k) * 2);
            } else {
                const int k = c / ACROSS, r = ((c & (ACROSS - 1)) ^ swizzle(k)) * 8;
                offset[i] = r <= last ? (uint32_t)((k * ld + r) * 2) : FFN_NOWHERE;
            }
        }
    }

    // The buffer of the step at k0: its pieces, and for k >= K nothing but zeros (KROWS: see past()).
    __device__ __forceinline__ i32x4 buffer(int k0, int K) const {
        const uintptr_t from = (uintptr_t)(KROWS ? base + k0 : base + k0 * ld);
        const int64_t left = (int64_t)(K - k0) * ld * 2;
        const int bytes = KROWS || left > 0x7fffffff ? 0x7fffffff : left > 0 ? (int)left : 0;
        return i32x4{(int)(uint32_t)from, (int)(uint32_t)(from >> 32) & 0xffff, bytes, 0x00020000};
    }
    __device__ __forceinline__ uint32_t past(int k0, int K) const { return KROWS && k0 + piece_k >= K ? FFN_NOWHERE : 0u; }

    // Sends for pass i of a step's pieces: 16 bytes a lane, straight into LDS.  A statement, because the compiler lets no
    // transposing LDS read go ahead of such a load; the waits are in the loop.  (m0 is the compiler's only from one
    // instruction to the next.)
    __device__ __forceinline__ void fetch(uint32_t lds, int i, i32x4 from, uint32_t past) const {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     ::"s"(lds + i * 4096), "v"(KROWS ? offset[i] | past : offset[i]), "s"(from));
    }
    __device__ __forceinline__ void fetch_all(uint32_t lds, int k0, int K) const {
        const i32x4 from = buffer(k0, K);
        const uint32_t none = past(k0, K);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) fetch(lds, i, from, none);
    }

    // The operand of a matrix instruction: rows row0 .. row0 + 15 (a lane's: row0 + lane % 16), k 32 ks + 8 (lane / 16) + 0 .. 7
    static __device__ __forceinline__ Frag frag(const char *lds, int row0, int ks) {
        const int lane = threadIdx.x & 63, kg = lane >> 4, l = lane & 15;
        if (KROWS) {
            const int r = row0 + l;
            return *(const Frag *)(lds + r * 128 + (((ks * 4 + kg) ^ (r & 7)) << 4));
        }
        const int k = ks * 32 + kg * 8 + (l >> 2);
        const int place = ((row0 >> 3) + ((l >> 1) & 1)) ^ (2 * ((l >> 2) | (kg & 1) << 2));
        const char *p = lds + k * (ROWS * 2) + place * 16 + (l & 1) * 8;
        typedef __attribute__((address_space(3))) s16x4 *Quad;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad)(p + 4 * ROWS * 2));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(Frag, v);
    }
};

template <int KIND, bool A_ROWS, bool B_ROWS, int EPI, int BM, int BN>
__global__ void __launch_bounds__(256, BM == 256 ? 1 : 2) ffn_mfma16_kernel(FfnArgs p) {
#ifdef __HIP_DEVICE_COMPILE__  // the registers that the statements name mean nothing to the host
    constexpr int MT = BM / 32, NT = BN / 32;  // 16 x 16 pieces of a wave
    constexpr bool GATE = EPI == FFN_GATE;
    constexpr int COLS = GATE ? BN / 2 : BN;   // columns of C
    using OpA = Operand16<KIND, A_ROWS, false, BM>;
    using OpB = Operand16<KIND, B_ROWS, GATE, BN>;
    using Frag = typename Frag16<KIND>::type;
    constexpr int BUFFER = OpA::BYTES + OpB::BYTES;
    constexpr int LOADS = OpA::PASSES + OpB::PASSES;
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const FfnTile t = ffn_tile(p);
    const int m0 = t.m * BM, n0 = t.n * COLS;
    const int k_first = t.split * p.k_slice, K = k_first + p.k_slice < p.K ? k_first + p.k_slice : p.K;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    OpA a;
    OpB b;
    a.init(p.A, p.lda, m0, p.M, 0);
    b.init(p.B, p.ldb, n0, p.N, p.up);

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // where this wave's pieces of a pass go
    const uint32_t lds_at = (uint32_t)(uintptr_t)(LdsPtr)lds + wave * 1024;
    a.fetch_all(lds_at, k_first, K);
    b.fetch_all(lds_at + OpA::BYTES, k_first, K);
    a.fetch_all(lds_at + BUFFER, k_first + FFN_BK, K);
    b.fetch_all(lds_at + BUFFER + OpA::BYTES, k_first + FFN_BK, K);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS) : "memory");
    Frag fa[2][MT], fb[2][NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) fb[0][j] = OpB::frag(lds + OpA::BYTES, wn + j * 16, 0);
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[0][i] = OpA::frag(lds, wm + i * 16, 0);

    int buffer = 0;
    for (int k = k_first; k < K; k += FFN_BK, buffer ^= 1) {
        const char *now = lds + buffer * BUFFER, *next = lds + (buffer ^ 1) * BUFFER;
        const uint32_t to = lds_at + buffer * BUFFER;
        const i32x4 from_a = a.buffer(k + 2 * FFN_BK, K), from_b = b.buffer(k + 2 * FFN_BK, K);
        const uint32_t past_a = a.past(k + 2 * FFN_BK, K), past_b = b.past(k + 2 * FFN_BK, K);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char *from = half ? next : now;
            if (half) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            // the matrix instructions in order, and between them one after the other what the next half needs
#pragma unroll
            for (int x = 0; x < MT * NT; ++x) {
                constexpr int READ_EACH = MT * NT / 2 / (MT + NT), LOAD_EACH = MT * NT / LOADS;
                if (half && x % LOAD_EACH == 0) {
                    const int y = x / LOAD_EACH;
                    if (y < OpA::PASSES) a.fetch(to, y, from_a, past_a);
                    else b.fetch(to + OpA::BYTES, y - OpA::PASSES, from_b, past_b);
                }
                if (x % READ_EACH == READ_EACH - 1) {
                    const int y = x / READ_EACH;
                    if (y < NT) fb[half ^ 1][y] = OpB::frag(from + OpA::BYTES, wn + y * 16, half ^ 1);
                    else if (y < NT + MT) fa[half ^ 1][y - NT] = OpA::frag(from, wm + (y - NT) * 16, half ^ 1);
                }
                Frag16<KIND>::mfma(fb[half][x % NT], fa[half][x / NT], acc[x / NT][x % NT]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        asm volatile("s_nop 15\n\ts_nop 3");  // the last sums are there before anything the compiler puts behind the loop
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads past the end write to LDS
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(acc[i][j]));
    __builtin_amdgcn_sched_barrier(0);

    // The sums go through LDS, half of the wave's rows at a time and each wave in a part of its own, and from there row after
    // row to the epilogue, a lane 4 columns of either half of the row's: the instruction leaves 4 columns of 16 rows in a
    // lane, which would be pieces of 8 bytes of 16 lines a store; so a line is one access's.  Piece q (4 columns) of row r
    // lies at q ^ (r & 15).
    __syncthreads();
    constexpr int WN = BN / 2, HALF = MT / 2 * 16;
    constexpr int WIDE = GATE ? WN / 2 : WN, LANES = WIDE / 8, ROWS = 64 / LANES;  // columns of C, lanes a row, rows at a time
    float *const mine = (float *)lds + wave * HALF * WN;
    const int lane_row = lane / LANES, c = (lane % LANES) * 4;                     // c: first of the lane's columns
    const int n = n0 + (GATE ? wn / 2 : wn) + c;
    // the piece of column c + e WIDE / 2; GATE: 16 columns of the gate, 16 of up, ...
    auto piece = [&](int e) { const int at = c + e * (WIDE / 2); return GATE ? (at >> 4) * 8 + (at & 15) / 4 : at / 4; };
    // What the epilogue reads of memory is on its way one batch of rows ahead.  A tile inside C asks nothing per lane: with a
    // test the compiler would wait for each load where the branches meet.
    constexpr int AHEAD = HALF / ROWS < 4 ? HALF / ROWS : 4;
    float cols[2][8] = {};  // FFN_GRAD: sums of the lane's columns of the gate's and of up's gradient, before they are rounded
    auto finish = [&](auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half) wave_lds_fence();  // other lanes have read the first half's sums
#pragma unroll
            for (int i = 0; i < MT / 2; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    *(f32x4 *)(mine + (i * 16 + (lane & 15)) * WN + ((j * 4 + (lane >> 4)) ^ (lane & 15)) * 4) =
                        acc[half * (MT / 2) + i][j];
            wave_lds_fence();  // what a lane reads others have written
            const int64_t m_first = m0 + wm + half * HALF + lane_row;
            FfnRow<4> row[AHEAD][2], next[AHEAD][2];
            auto fetch = [&](int r0) {
#pragma unroll
                for (int x = 0; x < AHEAD; ++x)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int64_t m = m_first + r0 + x * ROWS;
                        const int ne = n + e * (WIDE / 2);
                        if (EPI == FFN_GRAD && (INSIDE || (!p.part && m < p.M && ne < p.N)))
                            ffn_row<4, EPI, INSIDE>(p, m, ne, next[x][e]);
                    }
            };
            fetch(0);
            for (int r0 = 0; r0 < HALF; r0 += ROWS * AHEAD) {
#pragma unroll
                for (int x = 0; x < AHEAD; ++x) row[x][0] = next[x][0], row[x][1] = next[x][1];
                if (r0 + ROWS * AHEAD < HALF) fetch(r0 + ROWS * AHEAD);
#pragma unroll
                for (int x = 0; x < AHEAD; ++x)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = r0 + x * ROWS + lane_row, ne = n + e * (WIDE / 2);
                        const int64_t m = m_first + r0 + x * ROWS;
                        if (!INSIDE && (m >= p.M || ne >= p.N)) continue;
                        const f32x4 v = *(const f32x4 *)(mine + r * WN + (piece(e) ^ (r & 15)) * 4);
                        f32x4 w = f32x4{0.f, 0.f, 0.f, 0.f};
                        if (GATE) w = *(const f32x4 *)(mine + r * WN + ((piece(e) + 4) ^ (r & 15)) * 4);
                        const float s[4] = {v[0], v[1], v[2], v[3]}, u[4] = {w[0], w[1], w[2], w[3]};
                        if (!INSIDE && p.part) {
                            const int64_t width = GATE ? 2 * (int64_t)p.N : p.N;
                            float *o = p.part + ((int64_t)t.split * p.M + m) * width + ne;
                            store_cols<4>(o, p.N - ne, s);
                            if (GATE) store_cols<4>(o + p.N, p.N - ne, u);
                        } else {
                            float dg[4] = {}, du[4] = {};
                            ffn_epilogue<KIND, EPI, 4, INSIDE>(p, m, ne, s, u, row[x][e], EPI == FFN_GRAD ? dg : nullptr, du);
                            if (EPI == FFN_GRAD)
#pragma unroll
                                for (int f = 0; f < 4; ++f) cols[0][e * 4 + f] += dg[f], cols[1][e * 4 + f] += du[f];
                        }
                    }
            }
        }
    };
    if (m0 + BM <= p.M && n0 + COLS <= p.N && !p.part)
        finish(FfnTrue{});
    else
        finish(FfnFalse{});
    if (EPI == FFN_GRAD && p.cols) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) cols[h][e] += __shfl_xor(cols[h][e], o);
        if (lane_row == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int ne = n + e * (WIDE / 2);
                    if (ne < p.N)
                        store_cols<4>(p.cols + ((int64_t)t.m * 2 + (wave >> 1)) * 2 * p.N + h * p.N + ne, p.N - ne, cols[h] + e * 4);
                }
    }
#endif
}

template <int KIND, bool A_ROWS, bool B_ROWS, int EPI, int BM, int BN> int launch_tile16(FfnArgs a, hipStream_t stream) {
    constexpr size_t LDS = 2 * (size_t)(BM + BN) * FFN_BK * 2;
    constexpr int COLS = EPI == FFN_GATE ? BN / 2 : BN;
    static std::atomic<uint32_t> done{0};
    auto fn = ffn_mfma16_kernel<KIND, A_ROWS, B_ROWS, EPI, BM, BN>;
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

template <int KIND, bool A_ROWS, bool B_ROWS, int EPI>
int launch_layout16(const FfnArgs &a, int tile, hipStream_t stream) {
    return tile == 256 ? launch_tile16<KIND, A_ROWS, B_ROWS, EPI, 256, 256>(a, stream)
                       : launch_tile16<KIND, A_ROWS, B_ROWS, EPI, 128, 128>(a, stream);
}

template <int KIND> int launch_ffn16(const FfnProduct &p, int tile, hipStream_t stream) {
    if (p.epi == FFN_GATE) return launch_layout16<KIND, true, true, FFN_GATE>(p.args, tile, stream);
    if (p.epi == FFN_GRAD) return launch_layout16<KIND, true, false, FFN_GRAD>(p.args, tile, stream);
    if (p.a_rows && p.b_rows) return launch_layout16<KIND, true, true, FFN_STORE>(p.args, tile, stream);
    if (p.a_rows) return launch_layout16<KIND, true, false, FFN_STORE>(p.args, tile, stream);
    return launch_layout16<KIND, false, false, FFN_STORE>(p.args, tile, stream);
}

}  // namespace gmpgr
