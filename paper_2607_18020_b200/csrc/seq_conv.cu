// Causal convolution along the rows of (batch, length, channels) arrays, with SiLU: forward,
// gradients and the single-node form.
//
// pre[t] = bias + sum_j w[j] x[t-W+1+j].  Per element the forward pass reads and writes one value
// and computes 2W + 4 operations, the backward pass reads two values and writes one: both are bound
// by memory.  A thread owns VEC neighbouring channels (one 16-byte load per node where the strides
// allow it) and marches along its nodes with the last W-1 in registers, so every value is loaded
// once per piece of the row plus a halo of W-1 nodes.
//
// Gradients.  With g = gy * silu'(pre) the gradient of node t is sum_j w[j] g[t+W-1-j]: the march
// keeps the last W values of g and emits the gradient of the node W-1 behind.  The weights' gradient
// needs sums over all rows and nodes: every block leaves one partial sum per channel and tap, and a
// second kernel adds them in a fixed order.
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int CONV_LANES = 32;    // channel packs of a block
constexpr int CONV_ROWS = 8;      // pieces of a row marched by a block
constexpr int CONV_NODES = 16;    // nodes of a piece

struct ConvShape {
    int64_t length, x_batch, x_node, gy_batch, gy_node;
    int channels, silu;
    int groups;     // blocks along the channels
    int spans;      // blocks along a row
};

template <typename T, int VEC>
__device__ __forceinline__ void load_node(float (&out)[VEC], const T* p, bool there) {
    if (there) {
        const Pack<T, VEC> k = load_pack<T, VEC>(p);
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = to_f32<T>(k.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = 0.f;
    }
}

// x at node t of the row; before node 0 the window of the call before, or zeros.
template <typename T, int VEC, int W>
__device__ __forceinline__ void load_x(float (&out)[VEC], const T* x, int64_t x_node, const T* window, int64_t t,
                                       int64_t length, int channels) {
    if (t >= 0) load_node<T, VEC>(out, x + t * x_node, t < length);
    else load_node<T, VEC>(out, window + (t + W - 1) * channels, window != nullptr && t + W - 1 >= 0);
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(CONV_LANES* CONV_ROWS) conv_fwd_kernel(
    const T* __restrict__ x, const float* __restrict__ weight, const float* __restrict__ bias, const T* __restrict__ state,
    T* __restrict__ y, T* __restrict__ state_out, ConvShape s) {
    pdl_wait_then_trigger();
    int64_t blk = blockIdx.x;
    const int group = (int)(blk % s.groups);
    blk /= s.groups;
    const int span = (int)(blk % s.spans);
    const int64_t b = blk / s.spans;
    const int c = (group * CONV_LANES + threadIdx.x) * VEC;
    if (c >= s.channels) return;
    const int64_t t0 = ((int64_t)span * CONV_ROWS + threadIdx.y) * CONV_NODES;
    const T* xr = x + b * s.x_batch + c;
    const T* win = state ? state + b * (W - 1) * (int64_t)s.channels + c : nullptr;
    T* yr = y + b * s.length * s.channels + c;
    if (t0 < s.length) {
        float w[VEC][W], bs[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            bs[i] = bias ? bias[c + i] : 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[i][j] = weight[(int64_t)(c + i) * W + j];
        }
        float xs[CONV_NODES + W - 1][VEC];
#pragma unroll
        for (int k = 0; k < CONV_NODES + W - 1; ++k)
            load_x<T, VEC, W>(xs[k], xr, s.x_node, win, t0 + k - (W - 1), s.length, s.channels);
#pragma unroll
        for (int k = 0; k < CONV_NODES; ++k) {
            if (t0 + k >= s.length) break;
            float v[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float pre = bs[i];
#pragma unroll
                for (int j = 0; j < W; ++j) pre = fmaf(w[i][j], xs[k + j][i], pre);
                v[i] = s.silu ? pre * sigmoid_exact_f32(pre) : pre;
            }
            store_pack<T, VEC>(yr + (t0 + k) * s.channels, v);
        }
    }
    // the window that is left: the last W-1 nodes of the row, or of window and row together
    if (state_out != nullptr && span == 0 && threadIdx.y == 0) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            float v[VEC];
            load_x<T, VEC, W>(v, xr, s.x_node, win, s.length - (W - 1) + j, s.length, s.channels);
            store_pack<T, VEC>(state_out + (b * (W - 1) + j) * s.channels + c, v);
        }
    }
}

// One block's sums go to partial[(b * spans + span)][channels][W + 1]: taps, then bias.
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(CONV_LANES* CONV_ROWS) conv_bwd_kernel(
    const T* __restrict__ x, const float* __restrict__ weight, const float* __restrict__ bias, const T* __restrict__ state,
    const T* __restrict__ gy, const T* __restrict__ gstate_out, T* __restrict__ gx, T* __restrict__ gstate,
    float* __restrict__ partial, ConvShape s) {
    pdl_wait_then_trigger();
    __shared__ float sums[CONV_ROWS][VEC * (W + 1)][CONV_LANES];
    int64_t blk = blockIdx.x;
    const int group = (int)(blk % s.groups);
    blk /= s.groups;
    const int span = (int)(blk % s.spans);
    const int64_t b = blk / s.spans;
    const int c = (group * CONV_LANES + threadIdx.x) * VEC;
    float acc[VEC][W + 1] = {};
    // this thread emits the gradients of window-and-row positions f0 .. f0 + NODES - 1 (position f is node f - (W-1))
    const int64_t f0 = ((int64_t)span * CONV_ROWS + threadIdx.y) * CONV_NODES;
    if (c < s.channels && f0 < s.length + W - 1) {
        const T* xr = x + b * s.x_batch + c;
        const T* gr = gy + b * s.gy_batch + c;
        const T* win = state ? state + b * (W - 1) * (int64_t)s.channels + c : nullptr;
        float w[VEC][W], bs[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            bs[i] = bias ? bias[c + i] : 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[i][j] = weight[(int64_t)(c + i) * W + j];
        }
        float xs[W][VEC], g[W][VEC];    // x[t-W+1 .. t] and g[t-W+1 .. t]
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[j][i] = 0.f;
#pragma unroll
        for (int j = 1; j < W; ++j)
            load_x<T, VEC, W>(xs[j], xr, s.x_node, win, f0 - (W - 1) + j - W, s.length, s.channels);
#pragma unroll
        for (int k = -(W - 1); k < CONV_NODES; ++k) {      // node whose g is formed; the first W-1 are the halo
            const int64_t t = f0 + k;
            if (k >= 0 && t >= s.length + W - 1) break;
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) { xs[j][i] = xs[j + 1][i]; g[j][i] = g[j + 1][i]; }
            load_x<T, VEC, W>(xs[W - 1], xr, s.x_node, win, t, s.length, s.channels);
            const bool inside = t >= 0 && t < s.length;
            float gv[VEC];
            load_node<T, VEC>(gv, gr + t * s.gy_node, inside);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float d = gv[i];
                if (s.silu) {
                    float pre = bs[i];
#pragma unroll
                    for (int j = 0; j < W; ++j) pre = fmaf(w[i][j], xs[j][i], pre);
                    const float q = sigmoid_f32(pre);
                    d *= q * fmaf(pre, 1.f - q, 1.f);
                }
                d = inside ? d : 0.f;
                g[W - 1][i] = d;
                if (k >= 0 && inside) {
#pragma unroll
                    for (int j = 0; j < W; ++j) acc[i][j] = fmaf(d, xs[j][i], acc[i][j]);
                    acc[i][W] += d;
                }
            }
            if (k >= 0) {
                float v[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < W; ++j) v[i] = fmaf(w[i][j], g[W - 1 - j][i], v[i]);
                }
                if (gstate_out != nullptr && t >= s.length) {   // position t is entry t - length of the window that was left
                    float e[VEC];
                    load_node<T, VEC>(e, gstate_out + (b * (W - 1) + (t - s.length)) * s.channels + c, true);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] += e[i];
                }
                if (t >= W - 1) {
                    if (gx != nullptr) store_pack<T, VEC>(gx + (b * s.length + t - (W - 1)) * s.channels + c, v);
                } else if (gstate != nullptr) {
                    store_pack<T, VEC>(gstate + (b * (W - 1) + t) * s.channels + c, v);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i)
#pragma unroll
        for (int j = 0; j <= W; ++j) sums[threadIdx.y][i * (W + 1) + j][threadIdx.x] = acc[i][j];
    __syncthreads();
    const int c0 = group * CONV_LANES * VEC;
    float* out = partial + (b * s.spans + span) * (int64_t)s.channels * (W + 1) + (int64_t)c0 * (W + 1);
    const int here = min(CONV_LANES * VEC, s.channels - c0) * (W + 1);
    for (int e = threadIdx.y * CONV_LANES + threadIdx.x; e < here; e += CONV_LANES * CONV_ROWS) {
        const int lane = e / (VEC * (W + 1)), k = e % (VEC * (W + 1));
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < CONV_ROWS; ++r) v += sums[r][k][lane];
        out[e] = v;
    }
}

// gweight / gbias: sums of the partials over all blocks of a channel, one thread column per value.
__global__ void __launch_bounds__(256) conv_sum_kernel(const float* __restrict__ partial, int64_t parts, int channels, int w,
                                                       float* __restrict__ gweight, float* __restrict__ gbias) {
    pdl_wait_then_trigger();
    __shared__ float sums[8][32];
    const int64_t width = (int64_t)channels * (w + 1);
    const int64_t e = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (e < width)
        for (int64_t p = threadIdx.y; p < parts; p += 8) v += partial[p * width + e];
    sums[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && e < width) {
#pragma unroll
        for (int r = 1; r < 8; ++r) v += sums[r][threadIdx.x];
        const int64_t c = e / (w + 1);
        const int j = (int)(e % (w + 1));
        if (j < w) gweight[c * w + j] = v;
        else if (gbias != nullptr) gbias[c] = v;
    }
}

// One node: a thread per channel and row.  `state_out` may be `state`: a thread reads its window first.
template <typename T, int W>
__global__ void __launch_bounds__(256) conv_step_kernel(const T* __restrict__ x, int64_t x_batch, const float* __restrict__ weight,
                                                        const float* __restrict__ bias, const T* state, T* __restrict__ y,
                                                        T* state_out, int64_t rows, int channels, int silu) {
    pdl_wait_then_trigger();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= rows * channels) return;
    const int64_t b = e / channels;
    const int c = (int)(e % channels);
    T v[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) v[j] = state ? state[(b * (W - 1) + j) * channels + c] : from_f32<T>(0.f);
    v[W - 1] = x[b * x_batch + c];
    float pre = bias ? bias[c] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) pre = fmaf(weight[(int64_t)c * W + j], to_f32<T>(v[j]), pre);
    y[e] = from_f32<T>(silu ? pre * sigmoid_exact_f32(pre) : pre);
    if (state_out != nullptr) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) state_out[(b * (W - 1) + j) * channels + c] = v[j + 1];
    }
}

int check_conv(const fpde_conv_args* a, bool step) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->width < 1 || a->width > FPDE_CONV_MAX_WIDTH) return FPDE_ERR_PARAM;
    if (a->batch < 0 || a->channels < 0 || a->length < 0 || a->channels > (1 << 24) || a->length > (1ll << 40) || a->batch > (1ll << 40))
        return FPDE_ERR_SHAPE;
    if (a->batch * a->channels > 0) {
        const size_t e = dtype_bytes(a->dtype);
        if (a->weight == nullptr || (a->x == nullptr && (step || a->length > 0))) return FPDE_ERR_NULL;
        if (!aligned(a->x, e) || !aligned(a->state, e) || !aligned(a->state_out, e) || !aligned(a->weight, 4) || !aligned(a->bias, 4))
            return FPDE_ERR_ALIGN;
    }
    return FPDE_OK;
}

int conv_spans(const fpde_conv_args* a, int64_t positions) {
    return (int)ceil_div(positions > 0 ? positions : 1, CONV_ROWS * CONV_NODES);
}

// Channels of one thread: 16 bytes of them where every row of every array starts on 16 bytes.
template <typename T>
bool conv_wide(const fpde_conv_args* a, int vec, bool backward) {
    const size_t e = sizeof(T);
    bool ok = a->channels % vec == 0 && packs(a->x, a->x_batch, a->x_node, e, vec) && aligned(a->state, e * vec);
    if (backward)
        return ok && packs(a->gy, a->gy_batch, a->gy_node, e, vec) && aligned(a->gx, e * vec) && aligned(a->gstate, e * vec) &&
               aligned(a->gstate_out, e * vec);
    return ok && aligned(a->y, e * vec) && aligned(a->state_out, e * vec);
}

template <typename T, int VEC, int W>
cudaError_t conv_launch(const fpde_conv_args* a, bool backward, cudaStream_t st) {
    ConvShape s{a->length, a->x_batch, a->x_node, a->gy_batch, a->gy_node, (int)a->channels, a->silu, 0, 0};
    s.groups = (int)ceil_div(a->channels, CONV_LANES * VEC);
    s.spans = conv_spans(a, backward ? a->length + W - 1 : a->length);
    const int64_t blocks = a->batch * s.groups * s.spans;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(CONV_LANES, CONV_ROWS);
    if (!backward)
        return launch_kernel(conv_fwd_kernel<T, VEC, W>, grid, block, st, (const T*)a->x, a->weight, a->bias, (const T*)a->state,
                             (T*)a->y, (T*)a->state_out, s);
    float* partial = (float*)a->workspace;
    cudaError_t e = launch_kernel(conv_bwd_kernel<T, VEC, W>, grid, block, st, (const T*)a->x, a->weight, a->bias,
                                  (const T*)a->state, (const T*)a->gy, (const T*)a->gstate_out, (T*)a->gx, (T*)a->gstate, partial, s);
    if (e != cudaSuccess) return e;
    return launch_kernel(conv_sum_kernel, dim3((unsigned)ceil_div(a->channels * (W + 1), 32)), dim3(32, 8), st,
                         (const float*)partial, a->batch * s.spans, (int)a->channels, W, a->gweight, a->gbias);
}

template <typename T, int W>
cudaError_t conv_by_pack(const fpde_conv_args* a, bool backward, cudaStream_t st) {
    if (conv_wide<T>(a, 4, backward)) return conv_launch<T, 4, W>(a, backward, st);
    return conv_launch<T, 1, W>(a, backward, st);
}

template <typename T>
cudaError_t conv_by_width(const fpde_conv_args* a, bool backward, cudaStream_t st) {
    switch (a->width) {
    case 1: return conv_by_pack<T, 1>(a, backward, st);
    case 2: return conv_by_pack<T, 2>(a, backward, st);
    case 3: return conv_by_pack<T, 3>(a, backward, st);
    default: return conv_by_pack<T, 4>(a, backward, st);
    }
}

cudaError_t conv_by_type(const fpde_conv_args* a, bool backward, cudaStream_t st) {
    if (a->dtype == FPDE_F32) return conv_by_width<float>(a, backward, st);
    if (a->dtype == FPDE_BF16) return conv_by_width<__nv_bfloat16>(a, backward, st);
    return conv_by_width<__half>(a, backward, st);
}

template <typename T, int W>
cudaError_t conv_step_launch(const fpde_conv_args* a, cudaStream_t st) {
    const int64_t blocks = ceil_div(a->batch * a->channels, 256);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(conv_step_kernel<T, W>, dim3((unsigned)blocks), dim3(256), st, (const T*)a->x, a->x_batch, a->weight,
                         a->bias, (const T*)a->state, (T*)a->y, (T*)a->state_out, a->batch, (int)a->channels, a->silu);
}

template <typename T>
cudaError_t conv_step_by_width(const fpde_conv_args* a, cudaStream_t st) {
    switch (a->width) {
    case 1: return conv_step_launch<T, 1>(a, st);
    case 2: return conv_step_launch<T, 2>(a, st);
    case 3: return conv_step_launch<T, 3>(a, st);
    default: return conv_step_launch<T, 4>(a, st);
    }
}

int as_status(cudaError_t e) { return e == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA; }

}  // namespace
}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_causal_conv_workspace_bytes(const fpde_conv_args* a) {
    if (check_conv(a, false) != FPDE_OK) return 0;
    const int64_t parts = a->batch * conv_spans(a, a->length + a->width - 1);
    return (size_t)(parts * a->channels * (a->width + 1)) * sizeof(float);
}

int fpde_causal_conv_fwd(const fpde_conv_args* a, void* stream) {
    const int st = check_conv(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels == 0) return FPDE_OK;
    if (a->y == nullptr && a->length > 0) return FPDE_ERR_NULL;
    if (a->state != nullptr && a->state == a->state_out && a->width > 1) return FPDE_ERR_PARAM;   // blocks still read it
    if (!aligned(a->y, dtype_bytes(a->dtype))) return FPDE_ERR_ALIGN;
    if (a->length == 0 && (a->state_out == nullptr || a->width == 1)) return FPDE_OK;
    return as_status(conv_by_type(a, false, (cudaStream_t)stream));
}

int fpde_causal_conv_bwd(const fpde_conv_args* a, void* stream) {
    const int st = check_conv(a, false);
    if (st != FPDE_OK) return st;
    if (a->channels == 0) return FPDE_OK;
    const size_t e = dtype_bytes(a->dtype);
    if (a->gweight == nullptr || (a->gy == nullptr && a->length * a->batch > 0)) return FPDE_ERR_NULL;
    if (!aligned(a->gy, e) || !aligned(a->gx, e) || !aligned(a->gstate, e) || !aligned(a->gstate_out, e) || !aligned(a->gweight, 4) ||
        !aligned(a->gbias, 4))
        return FPDE_ERR_ALIGN;
    const size_t need = fpde_causal_conv_workspace_bytes(a);
    if (need > 0 && (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < need)) return FPDE_ERR_WORKSPACE;
    if (a->batch == 0)   // no rows: the sums over them are zero
        return as_status(launch_kernel(conv_sum_kernel, dim3((unsigned)ceil_div(a->channels * (a->width + 1), 32)), dim3(32, 8),
                                       (cudaStream_t)stream, (const float*)nullptr, (int64_t)0, (int)a->channels, a->width,
                                       a->gweight, a->gbias));
    return as_status(conv_by_type(a, true, (cudaStream_t)stream));
}

int fpde_causal_conv_step(const fpde_conv_args* a, void* stream) {
    const int st = check_conv(a, true);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels == 0) return FPDE_OK;
    if (a->y == nullptr) return FPDE_ERR_NULL;
    if (!aligned(a->y, dtype_bytes(a->dtype))) return FPDE_ERR_ALIGN;
    if (a->dtype == FPDE_F32) return as_status(conv_step_by_width<float>(a, (cudaStream_t)stream));
    if (a->dtype == FPDE_BF16) return as_status(conv_step_by_width<__nv_bfloat16>(a, (cudaStream_t)stream));
    return as_status(conv_step_by_width<__half>(a, (cudaStream_t)stream));
}

}  // extern "C"
