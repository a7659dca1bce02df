// Layer norm of rows and its gradient.
//
//   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),  xh = (x - mean) rstd,  out = xh gamma + beta
//   g = dout gamma,  dx = rstd (g - mean_d(g) - xh mean_d(g xh)),  dgamma = sum_rows dout xh,  dbeta = sum_rows dout
//
// Everything is formed in fp32 and rounded once, to the rows' type.  Bound by memory: a row is read once into registers
// (packed, as it lies in memory), the variance is summed over the deviations from the mean that the registers give, and
// the row is written from them.  A team of threads owns a row: 2^t lanes of a wave for narrow rows, a workgroup for wide
// ones; a team takes one row after the other, so that gamma, beta and the sums of the columns' gradients stay in
// registers, and the next row is on its way while one is worked on.  Rows that no team's registers hold are read three times
// (out of the caches, mostly).
//   16384 x 4096 bf16: forward 47 us, 5.7 TB/s (without the row ahead 54); gradient 80 + 5 us, 5.0 TB/s (without 107); two
// workgroups a compute unit in the gradient keep the column sums, 2 d floats each, at 4 % of its traffic.
#include "rows.h"

namespace gmpgr {

// Sums of N floats over the team, the same in every thread.  LANES = 0: `lanes` lanes of a wave (a power of two);
// otherwise a workgroup of LANES threads, through `s` (N * LANES / 64 floats; free again at the next call's barrier).
template <int LANES, int N>
__device__ __forceinline__ void team_sum(float *v, int lanes, float *s) {
    const int most = LANES ? 64 : lanes;
    for (int o = 1; o < most; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o);
    if (LANES) {
        constexpr int W = LANES ? LANES / 64 : 1;
        __syncthreads();  // the values of the sum before have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i * W + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) t += s[i * W + w];
            v[i] = t;
        }
    }
}

template <typename T> __device__ __forceinline__ typename Pack16<T>::type load_part(const T *p, int left) {
    if (left >= VEC<T>) return load16(p);
    typename Pack16<T>::type v;
#pragma unroll
    for (int i = 0; i < VEC<T>; ++i) v[i] = i < left ? p[i] : (T)0.f;
    return v;
}
template <typename T> __device__ __forceinline__ void store_part(T *p, int left, typename Pack16<T>::type v) {
    if (left >= VEC<T>) {
        store16(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i)
            if (i < left) p[i] = v[i];
    }
}

template <int KIND, int LANES, int NV>
__global__ void __launch_bounds__(LANES ? LANES : 256)
ln_forward_kernel(const typename ElemOf<KIND>::type *x, int64_t ld_x,
                  const typename ElemOf<KIND>::type *__restrict__ gamma,
                  const typename ElemOf<KIND>::type *__restrict__ beta, typename ElemOf<KIND>::type *out, int64_t ld_out,
                  float *__restrict__ mean_out, float *__restrict__ rstd_out, int64_t M, int d, float eps, int lanes) {
    using T = typename ElemOf<KIND>::type;
    using P = typename Pack16<T>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[LANES ? LANES / 64 : 1];
    const int team_size = LANES ? LANES : lanes;
    const int lane = LANES ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int teams = LANES ? 1 : 256 / lanes;
    const float inv_d = 1.0f / (float)d;
    P gm[NV], bt[NV];
    int left[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * team_size + lane) * V;
        left[j] = d - c;
        if (left[j] > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) gm[j][i] = (T)1.f, bt[j][i] = (T)0.f;
            if (gamma) gm[j] = load_part(gamma + c, left[j]);
            if (beta) bt[j] = load_part(beta + c, left[j]);
        }
    }
    // the next row is on its way while one is worked on
    const int64_t step = (int64_t)gridDim.x * teams, mine = LANES ? 0 : threadIdx.x / lanes;
    P next[NV];
    auto fetch = [&](int64_t row) {
        if (row >= M) return;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (left[j] > 0) next[j] = load_part(x + row * ld_x + (j * team_size + lane) * V, left[j]);
    };
    fetch((int64_t)blockIdx.x * teams + mine);
    for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < M; r0 += step) {
        // teams behind the last row follow along: the lanes of a wave sum together
        const int64_t row = r0 + mine;
        const bool on = row < M;
        P raw[NV];
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = next[j];
        fetch(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (on && left[j] > 0)
#pragma unroll
                for (int i = 0; i < V; ++i) sum[0] += (float)raw[j][i];
        team_sum<LANES, 1>(sum, lanes, s);
        const float mean = sum[0] * inv_d;
        float sq[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (on && left[j] > 0)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float c = (float)raw[j][i] - mean;
                    sq[0] += i < left[j] ? c * c : 0.f;
                }
        team_sum<LANES, 1>(sq, lanes, s);
        const float rstd = 1.0f / sqrtf(sq[0] * inv_d + eps);
        if (!on) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (left[j] > 0) {
                P o;
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = (T)(((float)raw[j][i] - mean) * rstd * (float)gm[j][i] + (float)bt[j][i]);
                store_part(out + row * ld_out + (j * team_size + lane) * V, left[j], o);
            }
        if (lane == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// Rows of any width: a workgroup of 1,024 a row, read three times.
template <int KIND>
__global__ void __launch_bounds__(1024)
ln_forward_any_kernel(const typename ElemOf<KIND>::type *x, int64_t ld_x,
                      const typename ElemOf<KIND>::type *__restrict__ gamma,
                      const typename ElemOf<KIND>::type *__restrict__ beta, typename ElemOf<KIND>::type *out,
                      int64_t ld_out, float *__restrict__ mean_out, float *__restrict__ rstd_out, int64_t M, int d, float eps) {
    using T = typename ElemOf<KIND>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[16];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
        const T *p = x + row * ld_x;
        float sum[1] = {0.f}, sq[1] = {0.f}, v[V], g[V], b[V];
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            load_floats(p + c, (int)(d - c), v);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0] += v[i];
        }
        team_sum<1024, 1>(sum, 0, s);
        const float mean = sum[0] * inv_d;
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            load_floats(p + c, (int)(d - c), v);
#pragma unroll
            for (int i = 0; i < V; ++i) sq[0] += c + i < d ? (v[i] - mean) * (v[i] - mean) : 0.f;
        }
        team_sum<1024, 1>(sq, 0, s);
        const float rstd = 1.0f / sqrtf(sq[0] * inv_d + eps);
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const int left = (int)(d - c);
            load_floats(p + c, left, v);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = 1.f, b[i] = 0.f;
            if (gamma) load_floats(gamma + c, left, g);
            if (beta) load_floats(beta + c, left, b);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (v[i] - mean) * rstd * g[i] + b[i];
            store_floats(out + row * ld_out + c, left, v);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// The gradient.  Sums over a team's rows of dout xh and dout stay in registers; the teams of a workgroup are joined in
// LDS, part[workgroup][2][d] goes to memory, and sum_two_kernel adds the workgroups in order.
template <int KIND, int LANES, int NV>
__global__ void __launch_bounds__(LANES ? LANES : 256)
ln_backward_kernel(const typename ElemOf<KIND>::type *dout, int64_t ld_dout, const typename ElemOf<KIND>::type *x,
                   int64_t ld_x, const typename ElemOf<KIND>::type *__restrict__ gamma,
                   const float *__restrict__ mean_in, const float *__restrict__ rstd_in, typename ElemOf<KIND>::type *dx,
                   int64_t ld_dx, float *__restrict__ part, int64_t M, int d, int lanes) {
    using T = typename ElemOf<KIND>::type;
    using P = typename Pack16<T>::type;
    constexpr int V = VEC<T>;
    constexpr int JOIN = LANES ? 1 : 3 * 2 * NV * V * 64;
    __shared__ float s[LANES ? 2 * LANES / 64 : 1];
    __shared__ float join[JOIN];
    const int team_size = LANES ? LANES : lanes;
    const int lane = LANES ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int teams = LANES ? 1 : 256 / lanes;
    const float inv_d = 1.0f / (float)d;
    P gm[NV];
    int left[NV];
    float dg[NV][V], db[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * team_size + lane) * V;
        left[j] = d - c;
#pragma unroll
        for (int i = 0; i < V; ++i) gm[j][i] = (T)1.f, dg[j][i] = 0.f, db[j][i] = 0.f;
        if (gamma && left[j] > 0) gm[j] = load_part(gamma + c, left[j]);
    }
    // the next row is on its way while one is worked on
    const int64_t step = (int64_t)gridDim.x * teams, mine = LANES ? 0 : threadIdx.x / lanes;
    P xn[NV], yn[NV];
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](int64_t row) {
        if (row >= M) return;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (left[j] > 0) {
                const int c = (j * team_size + lane) * V;
                xn[j] = load_part(x + row * ld_x + c, left[j]);
                yn[j] = load_part(dout + row * ld_dout + c, left[j]);
            }
        mean_n = mean_in[row], rstd_n = rstd_in[row];
    };
    fetch((int64_t)blockIdx.x * teams + mine);
    for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < M; r0 += step) {
        const int64_t row = r0 + mine;
        const bool on = row < M;
        P xr[NV], yr[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) xr[j] = xn[j], yr[j] = yn[j];
        const float mean = mean_n, rstd = rstd_n;
        fetch(row + step);
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (on && left[j] > 0)
#pragma unroll
                for (int i = 0; i < V; ++i) {  // behind the row's end dout is zero
                    const float xh = ((float)xr[j][i] - mean) * rstd, y = (float)yr[j][i], g = y * (float)gm[j][i];
                    sums[0] += g;
                    sums[1] += g * xh;
                    dg[j][i] += y * xh;
                    db[j][i] += y;
                }
        if (!dx) continue;
        team_sum<LANES, 2>(sums, lanes, s);
        if (!on) continue;
        const float a = sums[0] * inv_d, b = sums[1] * inv_d;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (left[j] > 0) {
                P o;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = ((float)xr[j][i] - mean) * rstd, g = (float)yr[j][i] * (float)gm[j][i];
                    o[i] = (T)(rstd * (g - a - xh * b));
                }
                store_part(dx + row * ld_dx + (j * team_size + lane) * V, left[j], o);
            }
    }
    if (!part) return;
    if (!LANES) {
        // teams of a wave, then the waves of the workgroup
        for (int o = lanes; o < 64; o <<= 1)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dg[j][i] += __shfl_xor(dg[j][i], o);
                    db[j][i] += __shfl_xor(db[j][i], o);
                }
        const int w = threadIdx.x >> 6, wl = threadIdx.x & 63;
        if (w)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    join[(((w - 1) * NV + j) * V + i) * 128 + wl] = dg[j][i];
                    join[(((w - 1) * NV + j) * V + i) * 128 + 64 + wl] = db[j][i];
                }
        __syncthreads();
        if (w || wl >= lanes) return;
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dg[j][i] += join[((q * NV + j) * V + i) * 128 + wl];
                    db[j][i] += join[((q * NV + j) * V + i) * 128 + 64 + wl];
                }
    }
    float *o = part + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * team_size + lane) * V;
        if (left[j] > 0)
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                store_floats(o + c + i, left[j] - i, dg[j] + i);
                store_floats(o + d + c + i, left[j] - i, db[j] + i);
            }
    }
}

// dx of rows of any width: a workgroup of 1,024 a row, read twice.
template <int KIND>
__global__ void __launch_bounds__(1024)
ln_backward_any_kernel(const typename ElemOf<KIND>::type *dout, int64_t ld_dout, const typename ElemOf<KIND>::type *x,
                       int64_t ld_x, const typename ElemOf<KIND>::type *__restrict__ gamma,
                       const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
                       typename ElemOf<KIND>::type *dx, int64_t ld_dx, int64_t M, int d) {
    using T = typename ElemOf<KIND>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[32];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
        const float mean = mean_in[row], rstd = rstd_in[row];
        float sums[2] = {0.f, 0.f}, v[V], y[V], g[V];
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = 1.f;
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const int left = (int)(d - c);
            load_floats(x + row * ld_x + c, left, v);
            load_floats(dout + row * ld_dout + c, left, y);
            if (gamma) load_floats(gamma + c, left, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sums[0] += y[i] * g[i];
                sums[1] += y[i] * g[i] * ((v[i] - mean) * rstd);
            }
        }
        team_sum<1024, 2>(sums, 0, s);
        const float a = sums[0] * inv_d, b = sums[1] * inv_d;
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const int left = (int)(d - c);
            load_floats(x + row * ld_x + c, left, v);
            load_floats(dout + row * ld_dout + c, left, y);
            if (gamma) load_floats(gamma + c, left, g);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = rstd * (y[i] * g[i] - a - (v[i] - mean) * rstd * b);
            store_floats(dx + row * ld_dx + c, left, v);
        }
    }
}

// part[slice][2][d] of rows of any width: a workgroup sums a slice of rows of 64 16-byte pieces of columns.
template <int KIND>
__global__ void __launch_bounds__(256)
ln_column_grad_any_kernel(const typename ElemOf<KIND>::type *__restrict__ dout, int64_t ld_dout,
                          const typename ElemOf<KIND>::type *__restrict__ x, int64_t ld_x,
                          const float *__restrict__ mean_in, const float *__restrict__ rstd_in, float *__restrict__ part,
                          int64_t M, int d) {
    using T = typename ElemOf<KIND>::type;
    constexpr int V = VEC<T>;
    __shared__ float s[3][2 * V][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int left = col < d ? (int)(d - col) : 0;
    const int64_t r0 = M * blockIdx.y / gridDim.y, r1 = M * (blockIdx.y + 1) / gridDim.y;
    float dg[V] = {}, db[V] = {};
    if (left > 0)
        for (int64_t r = r0 + w; r < r1; r += 4) {
            float v[V], y[V];
            load_floats(x + r * ld_x + col, left, v);
            load_floats(dout + r * ld_dout + col, left, y);
            const float mean = mean_in[r], rstd = rstd_in[r];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dg[i] += y[i] * ((v[i] - mean) * rstd);
                db[i] += y[i];
            }
        }
    if (w)
#pragma unroll
        for (int i = 0; i < V; ++i) s[w - 1][i][lane] = dg[i], s[w - 1][V + i][lane] = db[i];
    __syncthreads();
    if (w) return;
    float *o = part + (int64_t)blockIdx.y * 2 * d;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < left) {
            o[col + i] = ((dg[i] + s[0][i][lane]) + s[1][i][lane]) + s[2][i][lane];
            o[d + col + i] = ((db[i] + s[0][V + i][lane]) + s[1][V + i][lane]) + s[2][V + i][lane];
        }
}

// How a row is spread over threads: enough 16-byte pieces a thread to hold it in registers, at most 4.  lanes = 0: a
// workgroup of `threads`, or (nv = 0) the kernels for any width.
struct RowPlan {
    int threads, lanes, nv;
};
static RowPlan row_plan(int64_t d, int dtype) {
    const int64_t pieces = (d * (int64_t)elem_bytes(dtype) + 15) / 16;
    if (pieces <= 64) {
        int lanes = 1;
        while (lanes < pieces) lanes <<= 1;
        return {256, lanes, 1};
    }
    if (pieces <= 128) return {256, 64, 2};
    if (pieces <= 512) return {256, 0, 2};
    if (pieces <= 1024) return {256, 0, 4};
    if (pieces <= 2048) return {1024, 0, 2};
    return {1024, 0, 0};
}

// Workgroups: at most `most`, each with the same number of rounds or one less.
static int64_t row_groups(int64_t M, const RowPlan &p, int64_t most) {
    const int64_t teams = p.lanes ? 256 / p.lanes : 1, groups = (M + teams - 1) / teams, rounds = (groups + most - 1) / most;
    return (groups + rounds - 1) / rounds;
}
// Of the gradient, where each workgroup writes 2 d sums: two of 256 threads a compute unit.
static int64_t backward_groups(int64_t M, const RowPlan &p) { return row_groups(M, p, p.threads == 1024 ? 256 : 512); }

template <int KIND>
static int launch_forward(const void *x, int64_t ld_x, const void *gamma, const void *beta, void *out, int64_t ld_out,
                          float *mean, float *rstd, int64_t M, int d, float eps, hipStream_t stream) {
    using T = typename ElemOf<KIND>::type;
    const RowPlan p = row_plan(d, KIND);
    const dim3 grid((unsigned)row_groups(M, p, p.threads == 1024 ? 512 : 2048));
    if (p.nv == 0) {
        hipLaunchKernelGGL(ln_forward_any_kernel<KIND>, grid, dim3(1024), 0, stream, (const T *)x, ld_x, (const T *)gamma,
                           (const T *)beta, (T *)out, ld_out, mean, rstd, M, d, eps);
    } else {
        auto fn = p.lanes    ? (p.nv == 1 ? ln_forward_kernel<KIND, 0, 1> : ln_forward_kernel<KIND, 0, 2>)
                  : p.threads == 256 ? (p.nv == 2 ? ln_forward_kernel<KIND, 256, 2> : ln_forward_kernel<KIND, 256, 4>)
                                     : ln_forward_kernel<KIND, 1024, 2>;
        hipLaunchKernelGGL(fn, grid, dim3(p.threads), 0, stream, (const T *)x, ld_x, (const T *)gamma, (const T *)beta,
                           (T *)out, ld_out, mean, rstd, M, d, eps, p.lanes);
    }
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

template <int KIND>
static int launch_backward(const void *dout, int64_t ld_dout, const void *x, int64_t ld_x, const void *gamma,
                           const float *mean, const float *rstd, void *dx, int64_t ld_dx, float *part, int64_t M, int d,
                           hipStream_t stream) {
    using T = typename ElemOf<KIND>::type;
    const RowPlan p = row_plan(d, KIND);
    if (p.nv == 0) {
        if (part) {  // first: dx may take the place of x or dout
            hipLaunchKernelGGL(ln_column_grad_any_kernel<KIND>,
                               dim3((unsigned)((d + 64 * VEC<T> - 1) / (64 * VEC<T>)), (unsigned)column_sum_parts(M, d)),
                               dim3(256), 0, stream, (const T *)dout, ld_dout, (const T *)x, ld_x, mean, rstd, part, M, d);
            ANN_HIP_TRY(hipGetLastError());
        }
        if (dx)
            hipLaunchKernelGGL(ln_backward_any_kernel<KIND>, dim3((unsigned)(M < 512 ? M : 512)), dim3(1024), 0, stream,
                               (const T *)dout, ld_dout, (const T *)x, ld_x, (const T *)gamma, mean, rstd, (T *)dx, ld_dx, M, d);
    } else {
        auto fn = p.lanes    ? (p.nv == 1 ? ln_backward_kernel<KIND, 0, 1> : ln_backward_kernel<KIND, 0, 2>)
                  : p.threads == 256 ? (p.nv == 2 ? ln_backward_kernel<KIND, 256, 2> : ln_backward_kernel<KIND, 256, 4>)
                                     : ln_backward_kernel<KIND, 1024, 2>;
        hipLaunchKernelGGL(fn, dim3((unsigned)backward_groups(M, p)), dim3(p.threads), 0, stream, (const T *)dout, ld_dout,
                           (const T *)x, ld_x, (const T *)gamma, mean, rstd, (T *)dx, ld_dx, part, M, d, p.lanes);
    }
    ANN_HIP_TRY(hipGetLastError());
    return ANN_OK;
}

static int64_t backward_parts(int64_t M, int d, int dtype) {
    const RowPlan p = row_plan(d, dtype);
    return p.nv ? backward_groups(M, p) : column_sum_parts(M, d);
}

static bool ln_sizes(int64_t M, int32_t d, int32_t dtype) {
    if (M < 0 || M > (int64_t)1 << 40 || d < 1 || d > 1 << 24 || !row_dtype(dtype)) {
        set_error("need 0 <= M <= 2^40, 1 <= d <= 2^24, dtype ANN_F32, ANN_BF16 or ANN_F16");
        return false;
    }
    return true;
}
static bool ln_apart(const char *names, const void *a, int64_t ld_a, const void *b, int64_t ld_b, int64_t M, int32_t d, int32_t dtype) {
    if ((a == b && ld_a == ld_b) || !rows_overlap(a, ld_a, d, b, ld_b, d, M, elem_bytes(dtype))) return true;
    set_error("%s must be the same rows or have none in common", names);
    return false;
}
static bool ln_rows(const char *name, const void *p, int64_t ld, int64_t M, int32_t d, int32_t dtype) {
    if (!p || (uintptr_t)p % elem_bytes(dtype) || ld < d || ld > (int64_t)1 << 40) {
        set_error("%s must not be null, must be aligned to its elements and have a row stride of at least d = %d (got %lld)",
                  name, d, (long long)ld);
        return false;
    }
    return true;
}

}  // namespace gmpgr

using namespace gmpgr;

extern "C" {

int ann_layer_norm(const void *x_dev, int64_t ld_x, const void *gamma_dev, const void *beta_dev, int64_t M, int32_t d,
                   int32_t dtype, double eps, void *out_dev, int64_t ld_out, float *mean_dev, float *rstd_dev, void *stream) {
    if (!ln_sizes(M, d, dtype)) return ANN_EINVAL;
    if (!(eps >= 0.0) || !(eps < 3.0e38)) {
        set_error("need a finite eps >= 0");
        return ANN_EINVAL;
    }
    if (M == 0) return ANN_OK;
    if (!ln_rows("x_dev", x_dev, ld_x, M, d, dtype) || !ln_rows("out_dev", out_dev, ld_out, M, d, dtype)) return ANN_EINVAL;
    if (!ln_apart("x_dev and out_dev", x_dev, ld_x, out_dev, ld_out, M, d, dtype)) return ANN_EINVAL;
    if (((uintptr_t)gamma_dev | (uintptr_t)beta_dev) % elem_bytes(dtype) || ((uintptr_t)mean_dev | (uintptr_t)rstd_dev) % 4) {
        set_error("gamma_dev, beta_dev, mean_dev and rstd_dev must be aligned to their elements");
        return ANN_EINVAL;
    }
    auto fn = dtype == ANN_F32 ? launch_forward<ANN_F32> : dtype == ANN_BF16 ? launch_forward<ANN_BF16> : launch_forward<ANN_F16>;
    return fn(x_dev, ld_x, gamma_dev, beta_dev, out_dev, ld_out, mean_dev, rstd_dev, M, d, (float)eps, (hipStream_t)stream);
}

size_t ann_layer_norm_backward_workspace_bytes(int64_t M, int32_t d, int32_t dtype) {
    if (!ln_sizes(M, d, dtype)) return 0;
    return 256 + (size_t)(M ? backward_parts(M, d, dtype) : 0) * 2 * (size_t)d * sizeof(float);
}

int ann_layer_norm_backward(const void *dout_dev, int64_t ld_dout, const void *x_dev, int64_t ld_x, const void *gamma_dev,
                            const float *mean_dev, const float *rstd_dev, int64_t M, int32_t d, int32_t dtype, void *dx_dev,
                            int64_t ld_dx, void *dgamma_dev, void *dbeta_dev, void *workspace_dev, size_t workspace_bytes,
                            void *stream) {
    if (!ln_sizes(M, d, dtype)) return ANN_EINVAL;
    const size_t e = elem_bytes(dtype);
    if (((uintptr_t)gamma_dev | (uintptr_t)dgamma_dev | (uintptr_t)dbeta_dev) % e) {
        set_error("gamma_dev, dgamma_dev and dbeta_dev must be aligned to their elements");
        return ANN_EINVAL;
    }
    hipStream_t s = (hipStream_t)stream;
    if (M == 0) {
        int rc = dgamma_dev ? launch_zero(dgamma_dev, d, dtype, s) : ANN_OK;
        return rc == ANN_OK && dbeta_dev ? launch_zero(dbeta_dev, d, dtype, s) : rc;
    }
    if (!ln_rows("dout_dev", dout_dev, ld_dout, M, d, dtype) || !ln_rows("x_dev", x_dev, ld_x, M, d, dtype) ||
        (dx_dev && (!ln_rows("dx_dev", dx_dev, ld_dx, M, d, dtype) ||
                    !ln_apart("dout_dev and dx_dev", dout_dev, ld_dout, dx_dev, ld_dx, M, d, dtype) ||
                    !ln_apart("x_dev and dx_dev", x_dev, ld_x, dx_dev, ld_dx, M, d, dtype))))
        return ANN_EINVAL;
    if (!mean_dev || !rstd_dev || ((uintptr_t)mean_dev | (uintptr_t)rstd_dev) % 4) {
        set_error("mean_dev and rstd_dev must not be null and must be aligned to their elements");
        return ANN_EINVAL;
    }
    const bool columns = dgamma_dev || dbeta_dev;
    const int64_t parts = backward_parts(M, d, dtype);
    if (columns && (!workspace_dev || (uintptr_t)workspace_dev % 256)) {
        set_error("workspace_dev must not be null and must be 256-byte aligned");
        return ANN_EINVAL;
    }
    if (columns && workspace_bytes < ann_layer_norm_backward_workspace_bytes(M, d, dtype)) {
        set_error("workspace of %zu bytes, %zu needed", workspace_bytes, ann_layer_norm_backward_workspace_bytes(M, d, dtype));
        return ANN_EWORKSPACE;
    }
    if (!dx_dev && !columns) return ANN_OK;
    float *part = columns ? (float *)workspace_dev : nullptr;
    auto fn = dtype == ANN_F32 ? launch_backward<ANN_F32> : dtype == ANN_BF16 ? launch_backward<ANN_BF16> : launch_backward<ANN_F16>;
    int rc = fn(dout_dev, ld_dout, x_dev, ld_x, gamma_dev, mean_dev, rstd_dev, dx_dev, ld_dx, part, M, d, s);
    if (rc != ANN_OK || !columns) return rc;
    return launch_sum_two(part, parts, d, dgamma_dev, dbeta_dev, dtype, s);
}

}  // extern "C"
