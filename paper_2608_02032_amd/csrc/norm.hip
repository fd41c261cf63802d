// norm.hip -- layer norm of the residual stream (and its form without
// centring, the RMS norm of the language model), with the residual addition
// ahead of it, and its backward.  With s = x + residual as stored,
//   mu = mean(s) (0 without centring),  r = (mean((s - mu)^2) + eps)^-1/2,
//   out = (s - mu) r (.) w + b;
// backward, with xh = (s - mu) r and g = dout (.) w:
//   dx = r (g - mean(g) - xh mean(g xh)) + dsum   (mean(g) only if centred),
//   dw = sum_rows dout (.) xh,  db = sum_rows dout.
// The mean square is taken of the deviations, never as a difference of
// squares, which would lose what a large mean leaves.
#include "dart_common.hpp"
#include "dart_internal.hpp"

namespace dart {
namespace {

__device__ __forceinline__ float block_sum(float v, float* s_red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    const int wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_red[wave] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < nw; ++i) s += s_red[i];
    return s;
}

// One block per row, which it reads once from memory and then from cache.
template <typename T>
__global__ __launch_bounds__(256) void k_layernorm(const T* x, int64_t xs, const T* res, int64_t rs,
                                                   const float* __restrict__ w,
                                                   const float* __restrict__ b, float eps, T* out,
                                                   T* sum, int64_t rows, int D, int center) {
    extern __shared__ float s_row[];
    __shared__ float s_red[4];
    const int64_t r = flat_block();
    if (r >= rows) return;
    float a = 0.f;
    for (int i = threadIdx.x; i < D; i += 256) {
        float v = to_f(x[r * xs + i]);
        if (res) v = to_f(from_f<T>(v + to_f(res[r * rs + i])));
        s_row[i] = v;
        a += v;
    }
    const float mu = center ? block_sum(a, s_red) / D : 0.f;
    float q = 0.f;
    for (int i = threadIdx.x; i < D; i += 256) q += (s_row[i] - mu) * (s_row[i] - mu);
    const float inv = 1.0f / sqrtf(block_sum(q, s_red) / D + eps);
    for (int i = threadIdx.x; i < D; i += 256) {
        const float v = s_row[i];
        out[r * D + i] = from_f<T>((v - mu) * inv * (w ? w[i] : 1.f) + (b ? b[i] : 0.f));
        if (sum) sum[r * D + i] = from_f<T>(v);
    }
}

// One block per run of rows; the sums of the weight's and the bias's gradient
// over the run stand in the block's partial row, each column with one thread.
constexpr int kNormBwdRows = 32;
template <typename T, typename GT>
__global__ __launch_bounds__(256) void k_layernorm_bwd(const T* __restrict__ x, int64_t xs,
                                                       const float* __restrict__ w, float eps,
                                                       const GT* dout, const GT* dsum, GT* dx,
                                                       float* __restrict__ part, int64_t rows, int D,
                                                       int center) {
    __shared__ float s_red[4];
    const int64_t blk = flat_block();
    const int64_t r0 = blk * kNormBwdRows;
    if (r0 >= rows) return;
    const int64_t r1 = r0 + kNormBwdRows < rows ? r0 + kNormBwdRows : rows;
    float* acc = part + blk * 2 * D;
    for (int64_t r = r0; r < r1; ++r) {
        float a = 0.f;
        for (int i = threadIdx.x; i < D; i += 256) a += to_f(x[r * xs + i]);
        const float mu = center ? block_sum(a, s_red) / D : 0.f;
        float q = 0.f, g1 = 0.f, g2 = 0.f;
        for (int i = threadIdx.x; i < D; i += 256) {
            const float d = to_f(x[r * xs + i]) - mu, g = to_f(dout[r * D + i]) * (w ? w[i] : 1.f);
            q += d * d;
            g1 += g;
            g2 += g * d;
        }
        const float inv = 1.0f / sqrtf(block_sum(q, s_red) / D + eps);
        const float m1 = center ? block_sum(g1, s_red) / D : 0.f, m2 = block_sum(g2, s_red) * inv / D;
        for (int i = threadIdx.x; i < D; i += 256) {
            const float xh = (to_f(x[r * xs + i]) - mu) * inv, go = to_f(dout[r * D + i]);
            const float g = go * (w ? w[i] : 1.f);
            const float d = inv * (g - m1 - xh * m2) + (dsum ? to_f(dsum[r * D + i]) : 0.f);
            dx[r * D + i] = from_f<GT>(d);
            acc[i] = r == r0 ? go * xh : acc[i] + go * xh;
            acc[D + i] = r == r0 ? go : acc[D + i] + go;
        }
    }
}

int64_t bwd_blocks(int64_t rows) { return (rows + kNormBwdRows - 1) / kNormBwdRows; }

template <typename T>
void run_layernorm(int64_t rows, int D, int center, const void* x, int64_t xs, const void* res, int64_t rs,
                   const float* w, const float* b, float eps, void* out, void* sum, hipStream_t st) {
    k_layernorm<T><<<flat_grid(rows, 256), 256, D * sizeof(float), st>>>(
        (const T*)x, xs, (const T*)res, rs, w, b, eps, (T*)out, (T*)sum, rows, D, center);
}

template <typename T, typename GT>
void run_layernorm_bwd(int64_t rows, int D, int center, const void* x, int64_t xs, const float* w, float eps,
                       const void* dout, const void* dsum, void* dx, float* part, hipStream_t st) {
    k_layernorm_bwd<T, GT><<<flat_grid(bwd_blocks(rows), 256), 256, 0, st>>>(
        (const T*)x, xs, w, eps, (const GT*)dout, (const GT*)dsum, (GT*)dx, part, rows, D, center);
}

}  // namespace

hipError_t launch_layernorm(int dtype, int64_t rows, int D, int center, const void* x, int64_t xs,
                            const void* res, int64_t rs, const float* w, const float* b, float eps,
                            void* out, void* sum, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    prof_begin("k_layernorm", st);
    if (dtype == 1) run_layernorm<bf16>(rows, D, center, x, xs, res, rs, w, b, eps, out, sum, st);
    else run_layernorm<float>(rows, D, center, x, xs, res, rs, w, b, eps, out, sum, st);
    prof_end(st);
    return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(int64_t rows, int D) {
    return align256(sizeof(float) * (size_t)bwd_blocks(rows) * 2 * D);
}

hipError_t launch_layernorm_bwd(int dtype, int gdtype, int64_t rows, int D, int center, const void* x,
                                int64_t xs, const float* w, float eps, const void* dout,
                                const void* dsum, void* dx, float* dw, float* db, void* ws,
                                hipStream_t st) {
    float* part = reinterpret_cast<float*>(ws);
    const int64_t nb = bwd_blocks(rows);
    if (rows > 0) {
        prof_begin("k_layernorm_bwd", st);
        if (dtype == 0) run_layernorm_bwd<float, float>(rows, D, center, x, xs, w, eps, dout, dsum, dx, part, st);
        else if (gdtype == 0) run_layernorm_bwd<bf16, float>(rows, D, center, x, xs, w, eps, dout, dsum, dx, part, st);
        else run_layernorm_bwd<bf16, bf16>(rows, D, center, x, xs, w, eps, dout, dsum, dx, part, st);
        prof_end(st);
    }
    // a partial row is one item of 2 D values: the first D are the weight's sums
    if (dw || db) sum_parts(part, nb, 2 * (int64_t)D, dw, 2 * D, D, db, st);
    return hipGetLastError();
}

}  // namespace dart
