// Dropout from a counter-based generator: out = residual + (kept ? x * scale : 0).
//
// The choice for element e is a pure function of (seed, draw, e), so no mask is stored: the gradient is the same call
// on the output's gradient.  Philox4x32-10 with counter (block lo, block hi, draw lo, draw hi), block = e / 8, and key
// (seed lo, seed hi ^ 0x64726F70); the constant keeps the words apart from those of the serendipity noise under the
// same seed and draw.  A block's four words give eight 16-bit numbers, low half first; element e is kept iff number
// e % 8 is >= t = round(65536 p), and kept elements are scaled by 65536 / (65536 - t): with the probability rounded to
// 2^-16 the scale is exact for the probability that is drawn.  A dropped element is selected away, never multiplied,
// so infinities and NaN in dropped places leave nothing.
//   Bound by memory: 16 bits an element make one block of 20 wide products serve 8 elements.  32768 x 4096 bf16: with
// residual 144 us, 5.6 TB/s; without 96 us, 5.6 TB/s.
#include <math.h>

#include "philox.h"
#include "rows.h"

namespace gmpgr {

template <int KIND, bool RESIDUAL>
__global__ void __launch_bounds__(256)
dropout_kernel(const typename ElemOf<KIND>::type *x, const typename ElemOf<KIND>::type *residual,
               typename ElemOf<KIND>::type *out, int64_t n, uint32_t threshold, float scale, uint32_t k0, uint32_t k1,
               uint64_t draw, const uint64_t *__restrict__ draw_dev) {
    using T = typename ElemOf<KIND>::type;
    if (draw_dev) draw += *draw_dev;
    const int64_t blocks = (n + 7) / 8, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t b = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; b < blocks; b += step) {
        const int64_t e0 = b * 8;
        const int left = n - e0 < 8 ? (int)(n - e0) : 8;
        float v[8], r[8];
#pragma unroll
        for (int i = 0; i < 8; i += VEC<T>) {
            load_floats(x + e0 + i, left - i, v + i);
            if (RESIDUAL) load_floats(residual + e0 + i, left - i, r + i);
        }
        const Philox4 w = philox4x32_10((uint32_t)b, (uint32_t)((uint64_t)b >> 32), (uint32_t)draw,
                                        (uint32_t)(draw >> 32), k0, k1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t u = i & 1 ? w.x[i / 2] >> 16 : w.x[i / 2] & 0xFFFFu;
            v[i] = u >= threshold ? v[i] * scale : 0.f;
            if (RESIDUAL) v[i] += r[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i += VEC<T>) store_floats(out + e0 + i, left - i, v + i);
    }
}

template <int KIND>
static int launch_dropout(const void *x, const void *residual, void *out, int64_t n, uint32_t threshold, uint64_t seed,
                          uint64_t draw, const uint64_t *draw_dev, hipStream_t stream) {
    using T = typename ElemOf<KIND>::type;
    const float scale = threshold >= 65536u ? 0.f : 65536.f / (float)(65536u - threshold);
    const int64_t groups = ((n + 7) / 8 + 255) / 256;
    const unsigned grid = (unsigned)(groups < (1 << 20) ? groups : (1 << 20));
    auto fn = residual ? dropout_kernel<KIND, true> : dropout_kernel<KIND, false>;
    hipLaunchKernelGGL(fn, dim3(grid), dim3(256), 0, stream, (const T *)x, (const T *)residual, (T *)out, n, threshold,
                       scale, (uint32_t)seed, (uint32_t)(seed >> 32) ^ 0x64726F70u, draw, draw_dev);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

}  // namespace gmpgr

using namespace gmpgr;

extern "C" int ann_dropout(const void *x_dev, const void *residual_dev, void *out_dev, int64_t n, int32_t dtype, double p,
                           uint64_t seed, uint64_t draw, const uint64_t *draw_dev, void *stream) {
    if (n < 0 || n > (int64_t)1 << 46 || !row_dtype(dtype) || !(p >= 0.0) || !(p <= 1.0)) {
        set_error("need 0 <= n <= 2^46, dtype ANN_F32, ANN_BF16 or ANN_F16, 0 <= p <= 1");
        return ANN_EINVAL;
    }
    if (n == 0) return ANN_OK;
    if (!x_dev || !out_dev) {
        set_error("x_dev and out_dev must not be null");
        return ANN_EINVAL;
    }
    const size_t e = elem_bytes(dtype);
    if (((uintptr_t)x_dev | (uintptr_t)residual_dev | (uintptr_t)out_dev) % e || (uintptr_t)draw_dev % 8) {
        set_error("x_dev, residual_dev and out_dev must be aligned to their elements, draw_dev to 8 bytes");
        return ANN_EINVAL;
    }
    const int64_t w = n;  // one row
    if ((out_dev != x_dev && rows_overlap(x_dev, w, w, out_dev, w, w, 1, e)) ||
        (residual_dev && out_dev != residual_dev && rows_overlap(residual_dev, w, w, out_dev, w, w, 1, e))) {
        set_error("out_dev must be x_dev or residual_dev, or must not overlap them");
        return ANN_EINVAL;
    }
    const uint32_t threshold = (uint32_t)floor(p * 65536.0 + 0.5);
    auto fn = dtype == ANN_F32 ? launch_dropout<ANN_F32> : dtype == ANN_BF16 ? launch_dropout<ANN_BF16> : launch_dropout<ANN_F16>;
    return fn(x_dev, residual_dev, out_dev, n, threshold, seed, draw, draw_dev, (hipStream_t)stream);
}
