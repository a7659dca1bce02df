// Column sums and fills shared by the operators on rows of vectors.  Sums are formed in fp32 in a fixed order (slices of
// rows, then the slices one after the other), so that a result does not change from run to run.
#include "ffn.h"

namespace gmpgr {

// Adds the parts of 32 columns, one thread a column and 32nd of the parts, which are joined in order.  (With eighths of 500
// parts, whose reads follow each other, 6.3 us instead of 4.)
template <int KIND>
__device__ __forceinline__ void sum_columns(const float *__restrict__ part, int64_t P, int64_t width, int64_t first_col,
                                            int64_t n, typename ElemOf<KIND>::type *first,
                                            typename ElemOf<KIND>::type *second) {
    __shared__ float s[32][32];
    const int c = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t col = first_col + c;
    float acc = 0.f;
    if (col < width) {
        const int64_t p0 = P * y / 32, p1 = P * (y + 1) / 32;
#pragma unroll 8
        for (int64_t p = p0; p < p1; ++p) acc += part[p * width + col];
    }
    s[y][c] = acc;
    __syncthreads();
    if (y == 0 && col < width) {
#pragma unroll
        for (int i = 1; i < 32; ++i) acc += s[i][c];
        typename ElemOf<KIND>::type *out = col < n ? first : second;
        if (out) out[col < n ? col : col - n] = (typename ElemOf<KIND>::type)acc;
    }
}

template <int KIND>
__global__ void __launch_bounds__(1024)
sum_two_kernel(const float *__restrict__ part, int64_t P, int64_t n, typename ElemOf<KIND>::type *first,
               typename ElemOf<KIND>::type *second) {
    sum_columns<KIND>(part, P, 2 * n, (int64_t)blockIdx.x * 32, n, first, second);
}

int launch_sum_two(const float *part, int64_t P, int64_t n, void *first, void *second, int dtype, hipStream_t stream) {
    const dim3 grid((unsigned)((2 * n + 31) / 32));
    if (dtype == ANN_F32)
        hipLaunchKernelGGL(sum_two_kernel<ANN_F32>, grid, dim3(1024), 0, stream, part, P, n, (float *)first, (float *)second);
    else if (dtype == ANN_BF16)
        hipLaunchKernelGGL(sum_two_kernel<ANN_BF16>, grid, dim3(1024), 0, stream, part, P, n, (__bf16 *)first, (__bf16 *)second);
    else
        hipLaunchKernelGGL(sum_two_kernel<ANN_F16>, grid, dim3(1024), 0, stream, part, P, n, (_Float16 *)first, (_Float16 *)second);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
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
template <int KIND> __global__ void __launch_bounds__(256) column_slices_kernel(ColumnSums::Item a, int64_t M) {
    using T = typename ElemOf<KIND>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[3][64 * V];
    const T *in = (const T *)a.in;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int left = a.n - col < V ? (a.n > col ? (int)(a.n - col) : 0) : V;
    const int64_t r0 = M * blockIdx.y / gridDim.y, r1 = M * (blockIdx.y + 1) / gridDim.y;
    float acc[V] = {};
    if (left > 0)
#pragma unroll 4
        for (int64_t r = r0 + w; r < r1; r += 4) {
            float v[V];
            load_floats(in + r * a.ld + col, left, v);
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
                a.part[(int64_t)blockIdx.y * a.n + col + i] = ((acc[i] + s[0][i * 64 + lane]) + s[1][i * 64 + lane]) + s[2][i * 64 + lane];
    }
}

template <int KIND> __global__ void __launch_bounds__(1024) sum_column_parts_kernel(ColumnSums sums, int first_groups) {
    const bool second = (int)blockIdx.x >= first_groups;
    const ColumnSums::Item &a = sums.item[second];
    sum_columns<KIND>(a.part, a.parts, a.n, (int64_t)(blockIdx.x - (second ? first_groups : 0)) * 32, a.n,
                      (typename ElemOf<KIND>::type *)a.out, nullptr);
}

// Slices of rows: enough workgroups for four a compute unit, at least 16 rows each.
int64_t column_sum_parts(int64_t M, int64_t n) {
    const int64_t across = (n + 511) / 512;
    int64_t p = 1024 / (across < 1024 ? across : 1024);
    if (p > (M + 15) / 16) p = (M + 15) / 16;
    return p < 1 ? 1 : p;
}

template <int KIND> static int launch_column_sums_of(const ColumnSums &sums, int64_t M, hipStream_t stream) {
    constexpr int64_t cols = 64 * VEC<typename ElemOf<KIND>::type>;
    for (int i = 0; i < sums.n; ++i) {
        const ColumnSums::Item &a = sums.item[i];
        if (!a.in) continue;
        hipLaunchKernelGGL(column_slices_kernel<KIND>, dim3((unsigned)((a.n + cols - 1) / cols), (unsigned)a.parts), dim3(256), 0,
                           stream, a, M);
        ANN_HIP_TRY(hipGetLastError());
    }
    const int64_t first = (sums.item[0].n + 31) / 32, all = first + (sums.n > 1 ? (sums.item[1].n + 31) / 32 : 0);
    hipLaunchKernelGGL(sum_column_parts_kernel<KIND>, dim3((unsigned)all), dim3(1024), 0, stream, sums, (int)first);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

int launch_column_sums(const ColumnSums &sums, int64_t M, int dtype, hipStream_t stream) {
    if (dtype == ANN_F32) return launch_column_sums_of<ANN_F32>(sums, M, stream);
    if (dtype == ANN_BF16) return launch_column_sums_of<ANN_BF16>(sums, M, stream);
    return launch_column_sums_of<ANN_F16>(sums, M, stream);
}

// 8 elements a thread, one array after the other.
__global__ void __launch_bounds__(256) pad_rows_kernel(PadRows p) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) Pack {
        u16x8 v;
    };
    for (int a = 0; a < p.n; ++a) {
        const PadRows::Item &t = p.item[a];
        const int64_t across = t.ld_out / 8, total = t.rows * across;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
            const int64_t r = i / across, c = (i - r * across) * 8, left = t.width - c;
            const uint16_t *from = (const uint16_t *)t.in + r * t.ld_in + c;
            u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
            if (left >= 8) {
                v = reinterpret_cast<const Pack *>(from)->v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) v[e] = from[e];
            }
            *(u16x8 *)((uint16_t *)t.out + r * t.ld_out + c) = v;
        }
    }
}

int launch_pad_rows(const PadRows &p, hipStream_t stream) {
    if (p.n == 0) return ANN_OK;
    int64_t groups = 1;
    for (int a = 0; a < p.n; ++a) {
        const int64_t g = (p.item[a].rows * (p.item[a].ld_out / 8) + 255) / 256;
        if (g > groups) groups = g;
    }
    hipLaunchKernelGGL(pad_rows_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, stream, p);
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

}  // namespace gmpgr
