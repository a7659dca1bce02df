// Column sums and fills shared by the operators on rows of vectors.  Sums are formed in fp32 in a fixed order (slices of
// rows, then the slices one after the other), so that a result does not change from run to run.
#include "ffn.h"

namespace gmpgr {

// part [P][width], the first n columns of which go to `first`, the others to `second`.  One thread a column and slice of
// parts; the 8 slices of a workgroup are joined in order.
template <int KIND>
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float *__restrict__ part, int64_t P, int64_t width, int64_t n,
                 typename ElemOf<KIND>::type *__restrict__ first, typename ElemOf<KIND>::type *__restrict__ second) {
    __shared__ float s[8][32];
    const int c = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    float acc = 0.f;
    if (col < width) {
        const int64_t p0 = P * y / 8, p1 = P * (y + 1) / 8;
#pragma unroll 8
        for (int64_t p = p0; p < p1; ++p) acc += part[p * width + col];
    }
    s[y][c] = acc;
    __syncthreads();
    if (y == 0 && col < width) {
#pragma unroll
        for (int i = 1; i < 8; ++i) acc += s[i][c];
        typename ElemOf<KIND>::type *out = col < n ? first : second;
        if (out) out[col < n ? col : col - n] = (typename ElemOf<KIND>::type)acc;
    }
}

static int launch_sum(const float *part, int64_t P, int64_t width, int64_t n, void *first, void *second, int dtype,
                      hipStream_t stream) {
    const dim3 grid((unsigned)((width + 31) / 32));
    if (dtype == ANN_F32)
        hipLaunchKernelGGL(sum_parts_kernel<ANN_F32>, grid, dim3(256), 0, stream, part, P, width, n, (float *)first, (float *)second);
    else if (dtype == ANN_BF16)
        hipLaunchKernelGGL(sum_parts_kernel<ANN_BF16>, grid, dim3(256), 0, stream, part, P, width, n, (__bf16 *)first, (__bf16 *)second);
    else
        hipLaunchKernelGGL(sum_parts_kernel<ANN_F16>, grid, dim3(256), 0, stream, part, P, width, n, (_Float16 *)first, (_Float16 *)second);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

int launch_sum_parts(const float *part, int64_t P, int64_t n, void *out, int dtype, hipStream_t stream) {
    return launch_sum(part, P, n, n, out, nullptr, dtype, stream);
}

int launch_sum_two(const float *part, int64_t P, int64_t n, void *first, void *second, int dtype, hipStream_t stream) {
    return launch_sum(part, P, 2 * n, n, first, second, dtype, stream);
}

__global__ void __launch_bounds__(256) zero_kernel(uint16_t *out, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0;
}

int launch_zero(void *out, int64_t n, int dtype, hipStream_t stream) {
    n *= (int64_t)elem_bytes(dtype) / 2;
    if (n == 0) return ANN_OK;
    const int64_t groups = (n + 255) / 256;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, stream, (uint16_t *)out, n);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

// A workgroup sums a slice of rows of 64 16-byte pieces of columns: 4 waves take every fourth row, joined in LDS.
template <int KIND>
__global__ void __launch_bounds__(256)
column_sum_kernel(const typename ElemOf<KIND>::type *__restrict__ in, int64_t M, int64_t n, int64_t ld,
                  float *__restrict__ part) {
    using T = typename ElemOf<KIND>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[3][64 * V];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int left = n - col < V ? (int)(n - col) : V;
    const int64_t r0 = M * blockIdx.y / gridDim.y, r1 = M * (blockIdx.y + 1) / gridDim.y;
    float acc[V] = {};
    if (left > 0)
#pragma unroll 4
        for (int64_t r = r0 + w; r < r1; r += 4) {
            float v[V];
            load_floats(in + r * ld + col, left, v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += v[i];
        }
    if (w)
#pragma unroll
        for (int i = 0; i < V; ++i) s[w - 1][i * 64 + lane] = acc[i];
    __syncthreads();
    if (w == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left)
                part[(int64_t)blockIdx.y * n + col + i] = ((acc[i] + s[0][i * 64 + lane]) + s[1][i * 64 + lane]) + s[2][i * 64 + lane];
    }
}

// Slices of rows: enough workgroups for two a compute unit, at least 32 rows each.
int64_t column_sum_parts(int64_t M, int64_t n) {
    const int64_t across = (n + 511) / 512;
    int64_t p = 512 / (across < 512 ? across : 512);
    if (p > (M + 31) / 32) p = (M + 31) / 32;
    return p < 1 ? 1 : p;
}

int launch_column_sum(const void *in, int64_t M, int64_t n, int64_t ld, int in_dtype, void *out, int dtype, float *part,
                      hipStream_t stream) {
    const int64_t P = column_sum_parts(M, n);
    const int V = (int)(16 / elem_bytes(in_dtype));
    const dim3 grid((unsigned)((n + 64 * V - 1) / (64 * V)), (unsigned)P);
    if (in_dtype == ANN_F32)
        hipLaunchKernelGGL(column_sum_kernel<ANN_F32>, grid, dim3(256), 0, stream, (const float *)in, M, n, ld, part);
    else if (in_dtype == ANN_BF16)
        hipLaunchKernelGGL(column_sum_kernel<ANN_BF16>, grid, dim3(256), 0, stream, (const __bf16 *)in, M, n, ld, part);
    else
        hipLaunchKernelGGL(column_sum_kernel<ANN_F16>, grid, dim3(256), 0, stream, (const _Float16 *)in, M, n, ld, part);
    ANN_HIP_TRY(hipGetLastError());
    return launch_sum_parts(part, P, n, out, dtype, stream);
}

// 8 elements a thread.
__global__ void __launch_bounds__(256)
pad_rows_kernel(const uint16_t *__restrict__ in, int64_t ld_in, int64_t rows, int64_t width, uint16_t *__restrict__ out, int64_t ld_out) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) Pack {
        u16x8 v;
    };
    const int64_t across = ld_out / 8, total = rows * across;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / across, c = (i - r * across) * 8, left = width - c;
        const uint16_t *p = in + r * ld_in + c;
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (left >= 8) {
            v = reinterpret_cast<const Pack *>(p)->v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) v[e] = p[e];
        }
        *(u16x8 *)(out + r * ld_out + c) = v;
    }
}

int launch_pad_rows(const void *in, int64_t ld_in, int64_t rows, int64_t width, void *out, int64_t ld_out, hipStream_t stream) {
    const int64_t groups = (rows * (ld_out / 8) + 255) / 256;
    hipLaunchKernelGGL(pad_rows_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, stream,
                       (const uint16_t *)in, ld_in, rows, width, (uint16_t *)out, ld_out);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

}  // namespace gmpgr
