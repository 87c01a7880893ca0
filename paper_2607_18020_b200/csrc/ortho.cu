// Orthogonalised update of a stack of matrices by Newton-Schulz products, and the optimiser's whole
// step around it.
//
//   X = U / (|U| + eps);  `steps` times:  S = X X^T,  P = b S + c S S,  X <- a X + P X
// on the shorter side (taller matrices are turned on the way in and back on the way out).
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.775f, NS_C = 2.0315f;
constexpr int SUM_BLOCKS = 64;      // blocks that sum the squares of one matrix

// What the matrices are read from and written to.
struct OrthoIo {
    const void* grad;
    int64_t grad_matrix, grad_row;
    void* out;          // orthogonalize: result;  muon: weight
    float* momentum;    // muon only
    int rows, cols, m, n;
    bool turned, nesterov;
    float decay, keep, rate;   // momentum decay, 1 - lr wd, lr sqrt(max(1, rows / cols))
    double eps;
};

// The matrix to orthogonalise, element (r, c) of matrix k; with `momentum` already moved on.
template <typename T>
__device__ __forceinline__ float update_at(const OrthoIo& io, int64_t k, int64_t r, int64_t c) {
    const float g = to_f32<T>(((const T*)io.grad)[k * io.grad_matrix + r * io.grad_row + c]);
    if (io.momentum == nullptr) return g;
    const float mom = io.momentum[(k * io.rows + r) * io.cols + c];
    return io.nesterov ? fmaf(io.decay, mom, g) : mom;
}

// Moves the momentum on (muon) and leaves each block's sum of squares of the update, in 64 bits: the
// squares of gradients of any scale fit.
template <typename T>
__global__ void __launch_bounds__(256) ortho_square_kernel(OrthoIo io, double* __restrict__ sums) {
    pdl_wait_then_trigger();
    __shared__ double part[8];
    const int64_t k = blockIdx.x / SUM_BLOCKS, all = (int64_t)io.rows * io.cols;
    double v = 0.0;
    for (int64_t e = (int64_t)(blockIdx.x % SUM_BLOCKS) * 256 + threadIdx.x; e < all; e += SUM_BLOCKS * 256) {
        const int64_t r = e / io.cols, c = e % io.cols;
        if (io.momentum != nullptr) {
            float* mom = io.momentum + k * all + e;
            *mom = fmaf(io.decay, *mom, to_f32<T>(((const T*)io.grad)[k * io.grad_matrix + r * io.grad_row + c]));
        }
        const double u = update_at<T>(io, k, r, c);
        v += u * u;
    }
#pragma unroll
    for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(~0u, v, m);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += part[i];
        sums[blockIdx.x] = v;
    }
}

__device__ __forceinline__ float inverse_norm(const double* sums, double eps) {
    double v = 0.0;
    for (int i = 0; i < SUM_BLOCKS; ++i) v += sums[i];
    return (float)(1.0 / (sqrt(v) + eps));
}

// X (m x n) of matrix k.
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(OrthoIo io, const double* __restrict__ sums, float* __restrict__ x, int64_t all) {
    pdl_wait_then_trigger();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= all) return;
    const int64_t per = (int64_t)io.m * io.n, k = e / per, i = e % per / io.n, j = e % io.n;
    x[e] = update_at<T>(io, k, io.turned ? j : i, io.turned ? i : j) * inverse_norm(sums + k * SUM_BLOCKS, io.eps);
}

// C = alpha L R + beta D for row-major L (m x k), R (k x n), or its transpose as stored when RT.
template <bool RT>
__global__ void __launch_bounds__(256) product_kernel(const float* __restrict__ l, const float* __restrict__ r, const float* __restrict__ d,
                                                      float* __restrict__ c, int m, int n, int kk, float alpha, float beta) {
    pdl_wait_then_trigger();
    __shared__ float sl[16][65], sr[16][65];
    const int64_t which = blockIdx.z;
    l += which * m * kk; r += which * (int64_t)kk * n; d += which * (int64_t)m * n; c += which * (int64_t)m * n;
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < kk; k0 += 16) {
        for (int e = threadIdx.x; e < 1024; e += 256) {
            const int a = e / 16, b = e % 16;
            sl[b][a] = i0 + a < m && k0 + b < kk ? l[(int64_t)(i0 + a) * kk + k0 + b] : 0.f;
            if (RT) sr[b][a] = j0 + a < n && k0 + b < kk ? r[(int64_t)(j0 + a) * kk + k0 + b] : 0.f;
            else sr[e / 64][e % 64] = k0 + e / 64 < kk && j0 + e % 64 < n ? r[(int64_t)(k0 + e / 64) * n + j0 + e % 64] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sl[k][ty * 4 + a], sr[k][tx * 4 + b], acc[a][b]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ty * 4 + a, j = j0 + tx * 4 + b;
            if (i < m && j < n) c[(int64_t)i * n + j] = alpha * acc[a][b] + (beta != 0.f ? beta * d[(int64_t)i * n + j] : 0.f);
        }
}

template <typename T>
__global__ void __launch_bounds__(256) ortho_finish_kernel(OrthoIo io, const float* __restrict__ x, int64_t all) {
    pdl_wait_then_trigger();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= all) return;
    const int64_t per = (int64_t)io.rows * io.cols, k = e / per, r = e % per / io.cols, c = e % io.cols;
    const float v = x[k * per + (io.turned ? c * io.n + r : r * io.n + c)];
    T* out = (T*)io.out + e;
    *out = from_f32<T>(io.momentum == nullptr ? v : fmaf(-io.rate, v, io.keep * to_f32<T>(*out)));
}

struct OrthoSpace {
    size_t sums, x[2], s, p, total;
};
OrthoSpace space(int64_t count, int64_t m, int64_t n) {
    OrthoSpace w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    w.sums = take(count * SUM_BLOCKS * 8);
    w.x[0] = take(count * m * n * 4);
    w.x[1] = take(count * m * n * 4);
    w.s = take(count * m * m * 4);
    w.p = take(count * m * m * 4);
    w.total = at;
    return w;
}

int check(const fpde_ortho_args* a) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->steps < 0 || a->steps > 100 || !(a->eps >= 0)) return FPDE_ERR_PARAM;
    if (a->count < 0 || a->rows < 0 || a->cols < 0 || a->rows > (1 << 20) || a->cols > (1 << 20) || a->count > (1 << 20)) return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

#define FPDE_TRY(x)                           \
    do {                                      \
        const cudaError_t e_ = (x);           \
        if (e_ != cudaSuccess) return e_;     \
    } while (0)

template <typename T>
cudaError_t run(const fpde_ortho_args* a, bool muon, cudaStream_t st) {
    OrthoIo io = {};
    io.grad = a->grad; io.grad_matrix = a->grad_matrix; io.grad_row = a->grad_row;
    io.out = muon ? a->weight : a->out;
    io.momentum = muon ? a->momentum : nullptr;
    io.rows = (int)a->rows; io.cols = (int)a->cols;
    io.turned = a->rows > a->cols;
    io.m = io.turned ? io.cols : io.rows; io.n = io.turned ? io.rows : io.cols;
    io.nesterov = a->nesterov != 0;
    io.decay = (float)a->momentum_decay;
    io.keep = (float)(1.0 - a->lr * a->weight_decay);
    io.rate = (float)(a->lr * sqrt(io.rows > io.cols ? (double)io.rows / io.cols : 1.0));
    io.eps = a->eps;
    const OrthoSpace w = space(a->count, io.m, io.n);
    char* ws = (char*)a->workspace;
    double* sums = (double*)(ws + w.sums);
    float* x[2] = {(float*)(ws + w.x[0]), (float*)(ws + w.x[1])};
    float *s = (float*)(ws + w.s), *p = (float*)(ws + w.p);
    const int64_t all = a->count * (int64_t)io.m * io.n;
    const dim3 flat((unsigned)ceil_div(all, 256));
    FPDE_TRY(launch_kernel(ortho_square_kernel<T>, dim3((unsigned)(a->count * SUM_BLOCKS)), dim3(256), st, io, sums));
    FPDE_TRY(launch_kernel(ortho_start_kernel<T>, flat, dim3(256), st, io, (const double*)sums, x[0], all));
    const unsigned mt = (unsigned)ceil_div(io.m, 64), nt = (unsigned)ceil_div(io.n, 64), k = (unsigned)a->count;
    int at = 0;
    for (int i = 0; i < a->steps; ++i, at ^= 1) {
        FPDE_TRY(launch_kernel(product_kernel<true>, dim3(mt, mt, k), dim3(256), st, (const float*)x[at], (const float*)x[at],
                               (const float*)s, s, io.m, io.m, io.n, 1.f, 0.f));
        FPDE_TRY(launch_kernel(product_kernel<true>, dim3(mt, mt, k), dim3(256), st, (const float*)s, (const float*)s, (const float*)s, p,
                               io.m, io.m, io.m, NS_C, NS_B));
        FPDE_TRY(launch_kernel(product_kernel<false>, dim3(nt, mt, k), dim3(256), st, (const float*)p, (const float*)x[at],
                               (const float*)x[at], x[at ^ 1], io.m, io.n, io.m, 1.f, NS_A));
    }
    return launch_kernel(ortho_finish_kernel<T>, flat, dim3(256), st, io, (const float*)x[at], all);
}

int call(const fpde_ortho_args* a, bool muon, void* stream) {
    const int st = check(a);
    if (st != FPDE_OK) return st;
    if (a->count * a->rows * a->cols == 0) return FPDE_OK;
    const size_t e = dtype_bytes(a->dtype);
    if (a->grad == nullptr || (muon ? a->weight == nullptr || a->momentum == nullptr : a->out == nullptr)) return FPDE_ERR_NULL;
    if (!aligned(a->grad, e) || !aligned(a->out, e) || !aligned(a->weight, e) || !aligned(a->momentum, 4)) return FPDE_ERR_ALIGN;
    if (a->workspace == nullptr || !aligned(a->workspace, 256) || a->workspace_bytes < fpde_orthogonalize_workspace_bytes(a))
        return FPDE_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t err = a->dtype == FPDE_F32 ? run<float>(a, muon, s) : a->dtype == FPDE_BF16 ? run<__nv_bfloat16>(a, muon, s) : run<__half>(a, muon, s);
    return err == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
}

}  // namespace
}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_orthogonalize_workspace_bytes(const fpde_ortho_args* a) {
    if (check(a) != FPDE_OK) return 0;
    const int64_t m = a->rows < a->cols ? a->rows : a->cols, n = a->rows < a->cols ? a->cols : a->rows;
    return space(a->count, m, n).total;
}

int fpde_orthogonalize(const fpde_ortho_args* a, void* stream) { return call(a, false, stream); }
int fpde_muon_step(const fpde_ortho_args* a, void* stream) { return call(a, true, stream); }
unsigned int fpde_diag_ortho_timeouts(void) { return 0; }

}  // extern "C"
