// The operators around a worker's loss: what the C entry points hand to the kernels.
// Every launcher queues work on `st` and returns; errors are picked up by the caller with
// cudaGetLastError().
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace cdadam {

// Lets `kernel` be launched with `bytes` of dynamic shared memory.  Up to 48 KB, of which its static
// shared memory takes a few, that needs no call.  The limit belongs to the function and not to the
// launch, and another host thread may be between setting it and its own launch of another size:
// so every call sets the same one, the most that any launch takes, and none lowers it.  (A block has
// 227 KB; the static part is at most 3 KB, k_distill's.  A call for every launch costs the host less
// than a microsecond; nothing remembers which device has had it.)
constexpr int kSharedLimit = 216 * 1024;

template <typename F>
inline void allow_shared(F *kernel, size_t bytes)
{
    if (bytes > 40 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedLimit);
}

// Queues a kernel; false where that was refused, so that what would read its results is not queued
// either (the reason stays for the caller's cudaGetLastError()).
template <typename... P, typename... A>
inline bool queue(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess;
}

// A read-only vector of any of the three element types, widened at every access.
struct AnyVec {
    const void *p;      // NULL: not given
    int type;
};

struct NormForward {
    const void *x; int64_t x_stride;
    AnyVec weight, bias;
    int64_t rows, cols;
    float eps;
    void *y; int64_t y_stride;
    float *mean, *rstd;
    int wait_limit;     // polls; < 0: the kernels' default
};

struct NormBackward {
    const void *dy; int64_t dy_stride;
    const void *x; int64_t x_stride;
    AnyVec weight;
    const float *mean, *rstd;
    int64_t rows, cols, groups;
    void *dx; int64_t dx_stride;
    void *dweight; int64_t dweight_stride;
    void *dbias; int64_t dbias_stride;
    int grad_type, accumulate;
    float *parts;       // workspace
    int wait_limit;
};

struct Logprobs {
    const void *z; int64_t stride;
    const void *tokens;         // NULL: no logprob
    int64_t rows, vocab;
    int index64;                // tokens and ids are 64-bit
    double scale2;              // log2(e) / temperature
    int k;
    float *logprob, *entropy, *lse;
    void *top_ids; float *top_logprobs;
};

struct LogprobsBackward {
    const void *z; int64_t stride;
    const void *tokens;
    int64_t rows, vocab;
    int index64;
    double scale2, lse_scale;   // log2(e) / temperature; the same as rounded to binary32, times temperature
    float inv_temperature;
    const float *lse, *entropy, *dlogprob, *dentropy;
    void *dz; int64_t dz_stride;
};

struct Distill {
    const void *z; int64_t stride;
    const void *ids; const float *teacher;
    int64_t rows, vocab;
    int k, index64;
    double scale2;
    float inv_temperature;
    int rest;
    const float *dloss;
    float *loss;
    void *dz; int64_t dz_stride;   // dz NULL: the loss alone
    int wait_limit;
};

// A matrix of elements of the operator's type.
struct Matrix {
    void *p; int64_t stride;            // NULL: not given
};
// An 8-bit matrix and what goes with it: a step per row (rows format) or an exponent for every 32 columns of a row
// (checkpoint).
struct Rows8 {
    int8_t *p; int64_t stride;
    float *scale;
};
struct Kept8 {
    int8_t *p; int64_t stride;
    uint8_t *exponents; int64_t exponents_stride;
};

struct RmsNorm {
    Matrix x, residual;
    AnyVec weight;
    int64_t rows, cols;
    float eps;
    int normalise;      // 0: s = 1 (the rows format of x itself)
    Matrix total, y;
    Rows8 q;
    Kept8 kept;
    float *rstd;
};

struct RmsNormBackward {
    Matrix dy, x;       // x.p NULL: kept
    Kept8 kept;
    AnyVec weight;
    const float *rstd;
    Matrix dtotal;
    int64_t rows, cols, groups;
    Matrix dx;
    void *dweight; int64_t dweight_stride;
    int grad_type, accumulate;
    float *parts;       // workspace
};

struct Matmul8 {
    Rows8 x, w;
    AnyVec bias;
    int64_t tokens, channels, inner;
    void *y; int64_t y_stride;
    int wait_limit;     // polls; < 0: the kernel's default
};

// type: 0 binary32, 1 bfloat16, 2 binary16 (the CDADAM_* codes)
void launch_layer_norm(const NormForward &a, int type, cudaStream_t st);
void launch_layer_norm_backward(const NormBackward &a, int type, cudaStream_t st);
int64_t layer_norm_workspace(int64_t rows, int64_t cols, int64_t groups);
void launch_token_logprobs(const Logprobs &a, int type, cudaStream_t st);
void launch_token_logprobs_backward(const LogprobsBackward &a, int type, cudaStream_t st);
void launch_distill(const Distill &a, int type, cudaStream_t st);
void launch_rms_norm(const RmsNorm &a, int type, cudaStream_t st);
void launch_rms_norm_backward(const RmsNormBackward &a, int type, cudaStream_t st);
int64_t rms_norm_workspace(int64_t rows, int64_t cols, int64_t groups);
void launch_checkpoint8(const Matrix &x, const Kept8 &kept, int64_t rows, int64_t cols, int type, cudaStream_t st);
// values of the rows format (kept.p NULL) or of a checkpoint
void launch_restore8(const Rows8 &q, const Kept8 &kept, const Matrix &to, int64_t rows, int64_t cols, int type, cudaStream_t st);
// false: the matrices could not be described to the copy engine (the driver refused; the runtime may hold the reason)
bool launch_matmul8(const Matmul8 &a, int type, cudaStream_t st);

}  // namespace cdadam
