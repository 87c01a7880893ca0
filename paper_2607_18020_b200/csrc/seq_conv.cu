// Causal convolution along the rows of (batch, length, channels) arrays, with SiLU: forward,
// gradients and the single-node form.
//
// pre[t] = bias + sum_j w[j] x[t-W+1+j].  Per element the forward pass reads and writes one value
// and computes 2W + 4 operations, the backward pass reads two values and writes one: memory is the floor.
// A thread owns a pair of neighbouring channels (one where rows start on odd elements) and marches along
// its piece of a row with the last W-1 nodes in registers, so every value is loaded once per piece plus
// a halo of W-1 nodes; the nodes ahead are on their way to shared memory meanwhile.  A block has 4 pieces
// of 32 channel packs.  8 x 8192 x 2048 bf16, W = 4: forward 115 us (floor 82, 0.66 instructions a
// clock and scheduler, 45 % of the warps active), gradients 208 us (floor 123; 0.63 instructions, 28 % of the warps at 93
// registers; some 40 instructions an element for the filter, its gate, their gradients and the weights'): neither bytes nor
// issue slots are used up, both wait for latency.  Registers one group ahead instead of shared memory left too few bytes on their way: 328 and
// 587 us.
//
// Gradients.  With g = gy * silu'(pre) the gradient of node t is sum_j w[j] g[t+W-1-j]: the march
// keeps the last W values of g and emits the gradient of the node W-1 behind.  The weights' gradient
// needs sums over all rows and nodes: every block leaves one partial sum per channel and tap, and a
// second kernel adds them in a fixed order.
#include <type_traits>

#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int CONV_LANES = 32;    // channel packs of a block
constexpr int CONV_ROWS = 4;      // pieces of a row marched by a block
constexpr int CONV_THREADS = CONV_LANES * CONV_ROWS;
constexpr int GROUP = 8;          // nodes computed together
constexpr int MOST_NODES = 256;  // of a piece
constexpr int AHEAD = 2;          // groups on their way per thread and array (a power of two); four are no faster

struct ConvShape {
    int64_t length, x_batch, x_node, gy_batch, gy_node;
    int channels, silu;
    int groups;     // blocks along the channels
    int spans;      // blocks along a row
    int nodes;      // nodes of a piece (a multiple of GROUP)
};

// A thread's own nodes of one array, a few groups ahead of where it computes: 4- and 8-byte packs travel
// by cp.async into shared memory that only this thread reads (no registers held, no barrier needed),
// 2-byte ones, which cp.async does not have, through registers one group ahead.
template <typename T, int VEC>
struct Feed {
    static constexpr int BYTES = sizeof(T) * VEC;
    static constexpr bool ASYNC = BYTES >= 4;
    static constexpr int SLOTS = ASYNC ? AHEAD * GROUP : 1;
    using P = Pack<T, VEC>;
    P (*ring)[CONV_THREADS];      // [SLOTS][threads]
    P held[ASYNC ? 1 : GROUP];
    const T* p;
    int64_t node;
    int left;                     // nodes from p on that exist
    int tid;

    __device__ __forceinline__ void request(int slot) {      // the next GROUP nodes
        const T* q = p;
        if (ASYNC) {
            const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(&ring[slot * GROUP][tid]));
#pragma unroll
            for (int k = 0; k < GROUP; ++k, q += node) {
                if (k < left) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst + k * (uint32_t)(CONV_THREADS * BYTES)), "l"(q), "n"(BYTES < 4 ? 4 : BYTES) : "memory");
                else ring[slot * GROUP + k][tid] = P{};
            }
        } else {
#pragma unroll
            for (int k = 0; k < GROUP; ++k, q += node) {
                held[k] = P{};
                if (k < left) held[k] = load_pack<T, VEC>(q);
            }
        }
        p = q;
        left -= GROUP;
    }
    __device__ __forceinline__ P get(int slot, int k) const { return ASYNC ? ring[slot * GROUP + k][tid] : held[k]; }
};
__device__ __forceinline__ void feed_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void feed_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory"); }
__device__ __forceinline__ int clamp_left(int64_t n) { return n < 0 ? 0 : n > (1 << 30) ? 1 << 30 : (int)n; }

struct ConvWhere {
    int c;              // first channel of the thread
    int span;
    int64_t b, t0;      // row; first node of the thread's piece
};
template <int VEC>
__device__ __forceinline__ ConvWhere conv_where(const ConvShape& s) {
    ConvWhere w;
    int64_t blk = blockIdx.x;
    w.c = ((int)(blk % s.groups) * CONV_LANES + threadIdx.x) * VEC;
    blk /= s.groups;
    w.span = (int)(blk % s.spans);
    w.b = blk / s.spans;
    w.t0 = ((int64_t)w.span * CONV_ROWS + threadIdx.y) * s.nodes;
    return w;
}

template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> pack_at(const T* p, bool there) {
    Pack<T, VEC> k;
    if (there) return load_pack<T, VEC>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) k.v[i] = from_f32<T>(0.f);
    return k;
}

// x at node t of the row; before node 0 the window of the call before, or zeros.
template <typename T, int VEC, int W>
__device__ __forceinline__ Pack<T, VEC> x_at(const T* x, int64_t x_node, const T* window, int64_t t, int64_t length, int channels) {
    if (t >= 0) return pack_at<T, VEC>(x + t * x_node, t < length);
    return pack_at<T, VEC>(window + (t + W - 1) * channels, window != nullptr && t + W - 1 >= 0);
}

// The filters of the thread's channels, tap by tap, and their biases.
template <int VEC, int W>
__device__ __forceinline__ void load_filter(typename Lanes<VEC>::V (&w)[W], typename Lanes<VEC>::V& bs, const float* weight, const float* bias, int c) {
    float v[VEC];
#pragma unroll
    for (int j = 0; j < W; ++j) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = weight[(int64_t)(c + i) * W + j];
        w[j] = of_array(v);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = bias ? bias[c + i] : 0.f;
    bs = of_array(v);
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(CONV_THREADS) conv_fwd_kernel(
    const T* __restrict__ x, const float* __restrict__ weight, const float* __restrict__ bias, const T* __restrict__ state,
    T* __restrict__ y, T* __restrict__ state_out, ConvShape s) {
    pdl_wait_then_trigger();
    using F = Feed<T, VEC>;
    using V = typename Lanes<VEC>::V;
    __shared__ Pack<T, VEC> ring[F::SLOTS][CONV_THREADS];
    const ConvWhere at = conv_where<VEC>(s);
    const int c = at.c;
    if (c >= s.channels) return;
    const T* xr = x + at.b * s.x_batch + c;
    const T* win = state ? state + at.b * (W - 1) * (int64_t)s.channels + c : nullptr;
    if (at.t0 < s.length) {
        const int total = (int)(s.length - at.t0 < s.nodes ? s.length - at.t0 : s.nodes);
        F fx;
        fx.ring = ring; fx.p = xr + at.t0 * s.x_node; fx.node = s.x_node; fx.left = total; fx.tid = threadIdx.y * CONV_LANES + threadIdx.x;
        if (F::ASYNC) {
#pragma unroll
            for (int a = 0; a < AHEAD - 1; ++a) { fx.request(a); feed_commit(); }
        } else {
            fx.request(0);
        }
        V w[W], bs;
        load_filter<VEC, W>(w, bs, weight, bias, c);
        V xs[GROUP + W - 1];                    // the W-1 nodes before the group, then the group
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            xs[GROUP + j] = widen_v<T, VEC>(x_at<T, VEC, W>(xr, s.x_node, win, at.t0 + j - (W - 1), s.length, s.channels));
        T* yp = y + (at.b * s.length + at.t0) * s.channels + c;
        // AHEAD groups a turn: the slots are then known when this is compiled, and the window moves by renaming
        for (int turn = 0; turn < total; turn += AHEAD * GROUP)
#pragma unroll
        for (int slot = 0; slot < AHEAD; ++slot) {
            const int t = turn + slot * GROUP;
            if (t >= total) break;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) xs[j] = xs[GROUP + j];
            if (F::ASYNC) { fx.request((slot + AHEAD - 1) % AHEAD); feed_commit(); feed_wait(); }
#pragma unroll
            for (int k = 0; k < GROUP; ++k) xs[W - 1 + k] = widen_v<T, VEC>(fx.get(slot, k));
            if (!F::ASYNC) fx.request(0);
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                V pre = bs;
#pragma unroll
                for (int j = 0; j < W; ++j) pre = fma_v(w[j], xs[k + j], pre);
                if (s.silu) pre = mul_v(pre, sigmoid_v(pre));
                if (t + k < total) store_v<T, VEC>(yp + k * (int64_t)s.channels, pre);
            }
            yp += GROUP * (int64_t)s.channels;
        }
    }
    // the window that is left: the last W-1 nodes of the row, or of window and row together
    if (state_out != nullptr && at.span == 0 && threadIdx.y == 0) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            *reinterpret_cast<Pack<T, VEC>*>(state_out + (at.b * (W - 1) + j) * s.channels + c) =
                x_at<T, VEC, W>(xr, s.x_node, win, s.length - (W - 1) + j, s.length, s.channels);
    }
}

// A thread emits the gradients of window-and-row positions t0 .. t0 + nodes - 1 (position f is node
// f - (W-1)); the g of node f is formed at the same time, after a halo of W-1 nodes.
// One block's sums go to partial[(b * spans + span)][channels][W + 1]: taps, then bias.
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(CONV_THREADS) conv_bwd_kernel(
    const T* __restrict__ x, const float* __restrict__ weight, const float* __restrict__ bias, const T* __restrict__ state,
    const T* __restrict__ gy, const T* __restrict__ gstate_out, T* __restrict__ gx, T* __restrict__ gstate,
    float* __restrict__ partial, ConvShape s) {
    pdl_wait_then_trigger();
    using F = Feed<T, VEC>;
    using V = typename Lanes<VEC>::V;
    __shared__ Pack<T, VEC> ring_x[F::SLOTS][CONV_THREADS], ring_g[F::SLOTS][CONV_THREADS];
    __shared__ float sums[CONV_ROWS][VEC * (W + 1)][CONV_LANES];
    const ConvWhere at = conv_where<VEC>(s);
    const int c = at.c;
    const V zero = all_v<V>(0.f), one = all_v<V>(1.f);
    V acc[W + 1];                                  // gradients of the taps and the bias
#pragma unroll
    for (int j = 0; j <= W; ++j) acc[j] = zero;
    if (c < s.channels && at.t0 < s.length + W - 1) {
        const int total = (int)(s.length + W - 1 - at.t0 < s.nodes ? s.length + W - 1 - at.t0 : s.nodes);   // positions
        const int nodes = min(total, clamp_left(s.length - at.t0));                                          // of these, nodes that exist
        const T* xr = x + at.b * s.x_batch + c;
        const T* gr = gy + at.b * s.gy_batch + c;
        const T* win = state ? state + at.b * (W - 1) * (int64_t)s.channels + c : nullptr;
        F fx, fg;
        fx.ring = ring_x; fx.p = xr + at.t0 * s.x_node; fx.node = s.x_node;
        fg.ring = ring_g; fg.p = gr + at.t0 * s.gy_node; fg.node = s.gy_node;
        fx.left = fg.left = nodes;
        fx.tid = fg.tid = threadIdx.y * CONV_LANES + threadIdx.x;
        if (F::ASYNC) {
#pragma unroll
            for (int a = 0; a < AHEAD - 1; ++a) { fx.request(a); fg.request(a); feed_commit(); }
        } else {
            fx.request(0);
            fg.request(0);
        }
        V w[W], bs;
        load_filter<VEC, W>(w, bs, weight, bias, c);
        // g of one node from the W values of x that reach it: gy q (1 + pre (1 - q)), q the sigmoid
        auto slope = [&](V gv, const V* xv) {
            if (!s.silu) return gv;
            V pre = bs;
#pragma unroll
            for (int j = 0; j < W; ++j) pre = fma_v(w[j], xv[j], pre);
            const V q = sigmoid_v(pre), rest = fma_v(q, all_v<V>(-1.f), one);
            return mul_v(gv, mul_v(q, fma_v(pre, rest, one)));
        };
        V xs[GROUP + W - 1], g[GROUP + W - 1];                     // the W-1 nodes before the group, then the group
        {
            V h[2 * W - 2 + (W == 1)];                             // x from 2 (W-1) nodes before
#pragma unroll
            for (int j = 0; j < 2 * (W - 1); ++j)
                h[j] = widen_v<T, VEC>(x_at<T, VEC, W>(xr, s.x_node, win, at.t0 - 2 * (W - 1) + j, s.length, s.channels));
#pragma unroll
            for (int k = 0; k < W - 1; ++k) {
                const int64_t t = at.t0 - (W - 1) + k;
                const bool inside = t >= 0 && t < s.length;
                const V gv = widen_v<T, VEC>(pack_at<T, VEC>(gr + t * s.gy_node, inside));
                g[GROUP + k] = inside ? slope(gv, h + k) : zero;
                xs[GROUP + k] = h[W - 1 + k];
            }
        }
        T* gxp = gx + (at.b * s.length + at.t0 - (W - 1)) * s.channels + c;      // of the thread's first position
        for (int turn = 0; turn < total; turn += AHEAD * GROUP)
#pragma unroll
        for (int slot = 0; slot < AHEAD; ++slot) {
            const int t = turn + slot * GROUP;
            if (t >= total) break;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) { xs[j] = xs[GROUP + j]; g[j] = g[GROUP + j]; }
            if (F::ASYNC) {
                fx.request((slot + AHEAD - 1) % AHEAD);
                fg.request((slot + AHEAD - 1) % AHEAD);
                feed_commit();
                feed_wait();
            }
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                xs[W - 1 + k] = widen_v<T, VEC>(fx.get(slot, k));
                g[W - 1 + k] = widen_v<T, VEC>(fg.get(slot, k));
            }
            if (!F::ASYNC) { fx.request(0); fg.request(0); }
            // INNER: every node of the group exists and none of its positions lies in a window
            auto compute = [&](auto inner) {
                constexpr bool INNER = decltype(inner)::value;
#pragma unroll
                for (int k = 0; k < GROUP; ++k) {
                    const bool inside = INNER || t + k < nodes;
                    const V d = inside ? slope(g[W - 1 + k], xs + k) : zero;   // not a product: x may hold NaN
                    g[W - 1 + k] = d;
                    if (inside) {
#pragma unroll
                        for (int j = 0; j < W; ++j) acc[j] = fma_v(d, xs[k + j], acc[j]);
                        acc[W] = add_v(acc[W], d);
                    }
                    V v = mul_v(w[0], g[W - 1 + k]);
#pragma unroll
                    for (int j = 1; j < W; ++j) v = fma_v(w[j], g[W - 1 + k - j], v);
                    if (INNER) {
                        store_v<T, VEC>(gxp + k * (int64_t)s.channels, v);
                        continue;
                    }
                    const int64_t f = at.t0 + t + k;
                    if (t + k >= total) continue;
                    if (f >= s.length && gstate_out != nullptr)        // entry f - length of the window that was left
                        v = add_v(v, widen_v<T, VEC>(load_pack<T, VEC>(gstate_out + (at.b * (W - 1) + (f - s.length)) * s.channels + c)));
                    if (f >= W - 1) {
                        if (gx != nullptr) store_v<T, VEC>(gxp + k * (int64_t)s.channels, v);
                    } else if (gstate != nullptr) {
                        store_v<T, VEC>(gstate + (at.b * (W - 1) + f) * s.channels + c, v);
                    }
                }
            };
            if (t + GROUP <= nodes && at.t0 + t >= W - 1 && gx != nullptr) compute(std::true_type{});
            else compute(std::false_type{});
            gxp += GROUP * (int64_t)s.channels;
        }
    }
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        float v[VEC];
        to_array(v, acc[j]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sums[threadIdx.y][i * (W + 1) + j][threadIdx.x] = v[i];
    }
    __syncthreads();
    const int c0 = c - threadIdx.x * VEC;
    float* out = partial + (at.b * s.spans + at.span) * (int64_t)s.channels * (W + 1) + (int64_t)c0 * (W + 1);
    const int here = min(CONV_LANES * VEC, s.channels - c0) * (W + 1);
    for (int e = threadIdx.y * CONV_LANES + threadIdx.x; e < here; e += CONV_THREADS) {
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

// One node: a thread takes VEC neighbouring channels of `rows` rows, one after the other, and keeps their
// filter in registers.  `state_out` may be `state`: a thread reads its window first.
template <typename T, int W, int VEC>
__global__ void __launch_bounds__(128) conv_step_kernel(const T* __restrict__ x, int64_t x_batch, const float* __restrict__ weight,
                                                        const float* __restrict__ bias, const T* state, T* __restrict__ y, T* state_out,
                                                        int64_t batch, int across, int rows, int channels, int silu) {
    pdl_wait_then_trigger();
    const int c = ((int)(blockIdx.x % across) * 128 + (int)threadIdx.x) * VEC;
    if (c >= channels) return;
    float w[VEC][W], bs[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        bs[i] = bias ? bias[c + i] : 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[i][j] = weight[(int64_t)(c + i) * W + j];
    }
    const int64_t b0 = (int64_t)(blockIdx.x / across) * rows, b1 = b0 + rows < batch ? b0 + rows : batch;
#pragma unroll 2
    for (int64_t b = b0; b < b1; ++b) {
        Pack<T, VEC> v[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) v[j] = pack_at<T, VEC>(state + (b * (W - 1) + j) * channels + c, state != nullptr);
        v[W - 1] = load_pack<T, VEC>(x + b * x_batch + c);
        float pre[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            // Rounded as the formula reads, products, sum, bias, quotient, without contraction: the scan reads
            // a 16-bit y at once, and every fp32 difference turns some of its roundings.
            pre[i] = __fmul_rn(w[i][0], to_f32<T>(v[0].v[i]));
#pragma unroll
            for (int j = 1; j < W; ++j) pre[i] = __fadd_rn(pre[i], __fmul_rn(w[i][j], to_f32<T>(v[j].v[i])));
            pre[i] = __fadd_rn(pre[i], bs[i]);
            if (silu) pre[i] = __fdiv_rn(pre[i], 1.f + expf(-pre[i]));
        }
        store_pack<T, VEC>(y + b * channels + c, pre);
        if (state_out != nullptr) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Pack<T, VEC>*>(state_out + (b * (W - 1) + j) * channels + c) = v[j + 1];
        }
    }
}

int check_conv_sizes(const fpde_conv_args* a, bool step = false) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->width < 1 || a->width > FPDE_CONV_MAX_WIDTH) return FPDE_ERR_PARAM;
    if (a->batch < 0 || a->channels < 0 || a->length < 0 || a->channels > (1 << 24) || a->length > (1ll << 40) || a->batch > (1ll << 40) ||
        !product_fits(a->batch, step ? a->width : a->length + a->width, a->channels))
        return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

int check_conv(const fpde_conv_args* a, bool step) {
    const int st = check_conv_sizes(a, step);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels > 0) {
        const size_t e = dtype_bytes(a->dtype);
        if (a->weight == nullptr || (a->x == nullptr && (step || a->length > 0))) return FPDE_ERR_NULL;
        if (!aligned(a->x, e) || !aligned(a->state, e) || !aligned(a->state_out, e) || !aligned(a->weight, 4) || !aligned(a->bias, 4))
            return FPDE_ERR_ALIGN;
    }
    return FPDE_OK;
}

// Nodes of a thread's piece: long pieces re-read fewer halo nodes, short ones give a small grid more
// threads.  Doubled while there are still 1024 threads per SM.
int conv_nodes(const fpde_conv_args* a, int64_t positions) {
    int nodes = AHEAD * GROUP;
    while (nodes < MOST_NODES && a->batch * ceil_div(a->channels, 2) * ceil_div(positions, 2 * nodes) >= 148 * 1024) nodes *= 2;
    return nodes;
}
int64_t conv_spans(const fpde_conv_args* a, int64_t positions) {
    return ceil_div(positions > 0 ? positions : 1, (int64_t)CONV_ROWS * conv_nodes(a, positions));
}

// Two channels a thread where every row of every array starts on two elements.
template <typename T>
bool conv_pairs(const fpde_conv_args* a, bool backward) {
    const size_t e = sizeof(T);
    const bool ok = a->channels % 2 == 0 && packs(a->x, a->x_batch, a->x_node, e, 2) && aligned(a->state, 2 * e);
    if (backward)
        return ok && packs(a->gy, a->gy_batch, a->gy_node, e, 2) && aligned(a->gx, 2 * e) && aligned(a->gstate, 2 * e) && aligned(a->gstate_out, 2 * e);
    return ok && aligned(a->y, 2 * e) && aligned(a->state_out, 2 * e);
}

template <typename T, int VEC, int W, bool backward>
cudaError_t conv_launch(const fpde_conv_args* a, cudaStream_t st) {
    ConvShape s{a->length, a->x_batch, a->x_node, a->gy_batch, a->gy_node, (int)a->channels, a->silu, 0, 0, 0};
    s.groups = (int)ceil_div(a->channels, CONV_LANES * VEC);
    const int64_t positions = backward ? a->length + W - 1 : a->length, spans = conv_spans(a, positions);
    s.spans = (int)spans;
    s.nodes = conv_nodes(a, positions);
    const int64_t blocks = a->batch * s.groups * spans;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(CONV_LANES, CONV_ROWS);
    if constexpr (!backward)
        return launch_kernel(conv_fwd_kernel<T, VEC, W>, grid, block, st, (const T*)a->x, a->weight, a->bias, (const T*)a->state,
                             (T*)a->y, (T*)a->state_out, s);
    else {
        float* partial = (float*)a->workspace;
        cudaError_t e = launch_kernel(conv_bwd_kernel<T, VEC, W>, grid, block, st, (const T*)a->x, a->weight, a->bias,
                                      (const T*)a->state, (const T*)a->gy, (const T*)a->gstate_out, (T*)a->gx, (T*)a->gstate, partial, s);
        if (e != cudaSuccess) return e;
        return launch_kernel(conv_sum_kernel, dim3((unsigned)ceil_div(a->channels * (W + 1), 32)), dim3(32, 8), st,
                             (const float*)partial, a->batch * spans, (int)a->channels, W, a->gweight, a->gbias);
    }
}

template <typename T, int W>
cudaError_t conv_by_pack(const fpde_conv_args* a, bool backward, cudaStream_t st) {
    if (backward) return conv_pairs<T>(a, true) ? conv_launch<T, 2, W, true>(a, st) : conv_launch<T, 1, W, true>(a, st);
    return conv_pairs<T>(a, false) ? conv_launch<T, 2, W, false>(a, st) : conv_launch<T, 1, W, false>(a, st);
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

// One row a thread while the GPU is not full: latency.
int step_rows(const fpde_conv_args* a, int64_t across) { return a->batch * across >= 148 * 16 ? 4 : 1; }

template <typename T, int W, int VEC>
cudaError_t conv_step_run(const fpde_conv_args* a, cudaStream_t st) {
    const int64_t across = ceil_div(a->channels, 128 * VEC);
    const int rows = step_rows(a, across);
    const int64_t blocks = ceil_div(a->batch, rows) * across;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(conv_step_kernel<T, W, VEC>, dim3((unsigned)blocks), dim3(128), st, (const T*)a->x, a->x_batch, a->weight, a->bias,
                         (const T*)a->state, (T*)a->y, (T*)a->state_out, a->batch, (int)across, rows, (int)a->channels, a->silu);
}

bool step_pairs(const fpde_conv_args* a) {
    const size_t e = dtype_bytes(a->dtype);
    return a->channels % 2 == 0 && packs(a->x, a->x_batch, 0, e, 2) && aligned(a->y, 2 * e) && aligned(a->state, 2 * e) && aligned(a->state_out, 2 * e);
}

template <typename T, int W>
cudaError_t conv_step_launch(const fpde_conv_args* a, cudaStream_t st) {
    return step_pairs(a) ? conv_step_run<T, W, 2>(a, st) : conv_step_run<T, W, 1>(a, st);
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
    if (check_conv_sizes(a) != FPDE_OK) return 0;
    const int64_t parts = a->batch * conv_spans(a, a->length + a->width - 1);
    return (size_t)(parts * a->channels * (a->width + 1)) * sizeof(float);
}

int fpde_diag_conv_nodes(const fpde_conv_args* a, int backward) {
    return check_conv_sizes(a) != FPDE_OK ? 0 : conv_nodes(a, a->length + (backward ? a->width - 1 : 0));
}

int fpde_diag_conv_step_rows(const fpde_conv_args* a) {
    return check_conv_sizes(a, true) != FPDE_OK ? 0 : step_rows(a, ceil_div(a->channels, step_pairs(a) ? 256 : 128));
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
