// Layer norm, forward and backward.
#include "elements.cuh"

namespace cdadam {

constexpr int kNormBlock = 256;

// One block per row, three passes over it: mean, mean squared deviation, output.
template <typename T>
__global__ void __launch_bounds__(kNormBlock) k_norm(NormForward a)
{
    __shared__ float sh[2][kNormBlock / 32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    float s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kNormBlock) s += widen(x[j]);
    const float mean = block_sum_all<kNormBlock>(s, sh[0]) / (float)a.cols;
    s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kNormBlock) {
        const float c = widen(x[j]) - mean;
        s = fmaf(c, c, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum_all<kNormBlock>(s, sh[1]) / (float)a.cols + a.eps);
    for (int64_t j = threadIdx.x; j < a.cols; j += kNormBlock) {
        float v = (widen(x[j]) - mean) * rstd;
        if (a.weight.p) v *= any_at(a.weight, j);
        if (a.bias.p) v += any_at(a.bias, j);
        y[j] = narrow<T>(v);
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// Gradient with respect to x: one block per row, two passes.
template <typename T>
__global__ void __launch_bounds__(kNormBlock) k_norm_dx(NormBackward a)
{
    __shared__ float sh[2][kNormBlock / 32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kNormBlock) {
        const float h = widen(dy[j]) * (a.weight.p ? any_at(a.weight, j) : 1.0f);
        s1 += h;
        s2 = fmaf(h, (widen(x[j]) - mean) * rstd, s2);
    }
    s1 = block_sum_all<kNormBlock>(s1, sh[0]) / (float)a.cols;
    s2 = block_sum_all<kNormBlock>(s2, sh[1]) / (float)a.cols;
    for (int64_t j = threadIdx.x; j < a.cols; j += kNormBlock) {
        const float h = widen(dy[j]) * (a.weight.p ? any_at(a.weight, j) : 1.0f);
        const float xh = (widen(x[j]) - mean) * rstd;
        dx[j] = narrow<T>(rstd * (h - s1 - xh * s2));
    }
}

__device__ __forceinline__ void store_grad(void *p, int64_t i, int type, int accumulate, float v)
{
    if (type == 0) {
        float *q = static_cast<float *>(p) + i;
        *q = accumulate ? *q + v : v;
    } else if (type == 1) {
        bf16 *q = static_cast<bf16 *>(p) + i;
        *q = narrow<bf16>(accumulate ? widen(*q) + v : v);
    } else {
        f16 *q = static_cast<f16 *>(p) + i;
        *q = narrow<f16>(accumulate ? widen(*q) + v : v);
    }
}

// Gradients of weight and bias: a block owns 32 columns of a group, its 8 warps every eighth row.
template <typename T>
__global__ void __launch_bounds__(kNormBlock) k_norm_dw(NormBackward a)
{
    __shared__ float sw[kNormBlock / 32][33], sb[kNormBlock / 32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane, per = a.rows / a.groups, first = blockIdx.y * per;
    float w = 0.0f, b = 0.0f;
    if (j < a.cols)
        for (int64_t r = first + warp; r < first + per; r += kNormBlock / 32) {
            const float dy = widen(static_cast<const T *>(a.dy)[r * a.dy_stride + j]);
            const float x = widen(static_cast<const T *>(a.x)[r * a.x_stride + j]);
            w = fmaf(dy, (x - a.mean[r]) * a.rstd[r], w);
            b += dy;
        }
    sw[warp][lane] = w;
    sb[warp][lane] = b;
    __syncthreads();
    if (warp == 0 && j < a.cols) {
        w = b = 0.0f;
        for (int i = 0; i < kNormBlock / 32; ++i) { w += sw[i][lane]; b += sb[i][lane]; }
        if (a.dweight) store_grad(a.dweight, blockIdx.y * a.dweight_stride + j, a.grad_type, a.accumulate, w);
        if (a.dbias) store_grad(a.dbias, blockIdx.y * a.dbias_stride + j, a.grad_type, a.accumulate, b);
    }
}

int64_t layer_norm_workspace(int64_t, int64_t, int64_t) { return 0; }

void launch_layer_norm(const NormForward &a, int type, cudaStream_t st)
{
    if (a.rows == 0) return;
    const unsigned g = (unsigned)a.rows;
    if (type == 0) k_norm<float><<<g, kNormBlock, 0, st>>>(a);
    else if (type == 1) k_norm<bf16><<<g, kNormBlock, 0, st>>>(a);
    else k_norm<f16><<<g, kNormBlock, 0, st>>>(a);
}

template <typename T>
static void norm_backward(const NormBackward &a, cudaStream_t st)
{
    if (a.dweight || a.dbias) {     // before dx, which may overwrite dy or x
        const dim3 g((unsigned)((a.cols + 31) / 32), (unsigned)a.groups);
        k_norm_dw<T><<<g, kNormBlock, 0, st>>>(a);
    }
    if (a.dx && a.rows) k_norm_dx<T><<<(unsigned)a.rows, kNormBlock, 0, st>>>(a);
}

void launch_layer_norm_backward(const NormBackward &a, int type, cudaStream_t st)
{
    if (type == 0) norm_backward<float>(a, st);
    else if (type == 1) norm_backward<bf16>(a, st);
    else norm_backward<f16>(a, st);
}

}  // namespace cdadam
