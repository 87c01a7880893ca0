// Rotation of queries and keys by their position, with or without a norm of each head before it, and the
// gradients.
//
//   u = x / sqrt(mean(x^2) + eps) * weight;  y = u with pair i of its first 2 * pairs features turned by
//   position * inv_freq[i]
//
// Every element is read and written once; memory bounds it.  8 x 4096 x 32 heads x 128 bf16: forward MEASURED.
//
// A block takes a tile of nodes.  First it forms the cosines and sines of the tile's angles, once for all heads,
// in shared memory: turns = position * inv_freq / 2 pi in 64 bits, reduced there to [-1/2, 1/2], so that the
// 32-bit sine and cosine of what is left are good to their last bits at any position.  Then groups of 1 to 32
// lanes take one head of one node each.  A lane holds both members of V pairs (or 2 V features that are not
// turned), in two loads of up to 16 bytes; sums over a head are shuffles among the group's lanes.
//
// Gradients.  The rotation's is the rotation by the opposite angle: the same kernel.  With g the upstream gradient
// turned back, n = x r, r = 1 / sqrt(mean(x^2) + eps):  gx = r (g w - n mean(g w n)),  gw = sum over nodes and heads of g n.
// A lane keeps its features' share of gw in registers over all tiles of its block (a grid of fixed size), a block
// sums its groups' shares, and a second kernel the blocks', all in a fixed order.
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int THREADS = 256;
constexpr int MOST_TILE = 16;                  // nodes of a tile
constexpr int MOST_PAIRS = FPDE_HEAD_MAX_DIM / 2;
constexpr int GRAD_BLOCKS = 148 * 3;           // blocks of the gradients of the norm, at most

struct HeadView {
    const void* p;
    int64_t batch, node, head;
};

struct HeadShape {
    int64_t length, nodes, pos_batch, pos_node, offset;
    const int64_t* positions;
    const float* inv_freq;
    int heads[2];             // of q and k
    int dim, pairs, interleaved, norm;
    int lanes;                // of a group: a power of two
    int tile;                 // nodes a block takes at once
    float eps, sign;
};

struct Tile {
    int64_t batch[MOST_TILE], node[MOST_TILE];
    double position[MOST_TILE];
    alignas(16) float cosine[MOST_TILE * MOST_PAIRS];
    alignas(16) float sine[MOST_TILE * MOST_PAIRS];
};

// The nodes of the tile that starts at node `first` of all rows, and the cosines and sines of their angles.
__device__ __forceinline__ void open_tile(Tile& t, const HeadShape& s, int64_t first, int count) {
    if (threadIdx.x < count) {
        const int64_t n = first + threadIdx.x, b = n / s.length;
        t.batch[threadIdx.x] = b;
        t.node[threadIdx.x] = n - b * s.length;
        // as doubles: a position past 2^53 is rounded, and the sum cannot overflow
        const int64_t at = s.positions != nullptr ? s.positions[b * s.pos_batch + (n - b * s.length) * s.pos_node] : n - b * s.length;
        t.position[threadIdx.x] = (double)at + (double)s.offset;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count * s.pairs; i += THREADS) {
        const int n = i / s.pairs;
        // the product is rounded once, relative to its size: 1e-10 of a turn at position 10^6
        double turns = t.position[n] * ((double)s.inv_freq[i - n * s.pairs] * 0.15915494309189535);
        turns -= rint(turns);
        float c, q;
        sincospif(2.f * (float)turns, &q, &c);
        t.cosine[i] = c;
        t.sine[i] = q * s.sign;
    }
    __syncthreads();
}

// Where in its head a lane's unit lies: two packs of V features.
template <int V>
struct Unit {
    int first, second;        // features
    int pair;                 // first pair, or -1: not turned
    bool has, has_second;     // V = 1: an odd head's last feature has no second
};
template <int V>
__device__ __forceinline__ Unit<V> unit_at(const HeadShape& s, int u) {
    Unit<V> r;
    const int turned = s.pairs / V;
    if (u < turned) {
        r.pair = u * V;
        r.first = s.interleaved ? 2 * u * V : u * V;
        r.second = s.interleaved ? r.first + V : u * V + s.pairs;
    } else {
        r.pair = -1;
        r.first = 2 * u * V;
        r.second = r.first + V;
    }
    r.has = r.first < s.dim;
    r.has_second = r.second < s.dim;
    return r;
}

template <typename T, int V>
__device__ __forceinline__ void load_unit(float (&v)[2 * V], const T* head, const Unit<V>& u) {
    float a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = b[i] = 0.f;
    if (u.has) widen<T, V>(a, load_pack<T, V>(head + u.first));
    if (u.has_second) widen<T, V>(b, load_pack<T, V>(head + u.second));
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = a[i];
        v[V + i] = b[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_unit(T* head, const Unit<V>& u, const float (&v)[2 * V]) {
    float a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        a[i] = v[i];
        b[i] = v[V + i];
    }
    if (u.has) store_pack<T, V>(head + u.first, a);
    if (u.has_second) store_pack<T, V>(head + u.second, b);
}
// The unit's pairs turned by the angles of node n of the tile.
template <int V>
__device__ __forceinline__ void turn(float (&v)[2 * V], const Unit<V>& u, const Tile& t, int n, const HeadShape& s) {
    if (u.pair < 0) return;
    const Pack<float, (V > 4 ? 4 : V)>*cs = reinterpret_cast<const Pack<float, (V > 4 ? 4 : V)>*>(t.cosine + n * s.pairs + u.pair),
                                   *sn = reinterpret_cast<const Pack<float, (V > 4 ? 4 : V)>*>(t.sine + n * s.pairs + u.pair);
    constexpr int W = V > 4 ? 4 : V;
    float c[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        c[i] = cs[i / W].v[i % W];
        q[i] = sn[i / W].v[i % W];
    }
    float w[2 * V];
    if (s.interleaved) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * q[i];
            w[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * q[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[i] = v[i] * c[i] - v[V + i] * q[i];
            w[V + i] = v[V + i] * c[i] + v[i] * q[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) v[i] = w[i];
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int m = lanes / 2; m > 0; m /= 2) v += __shfl_xor_sync(~0u, v, m);
    return v;
}

template <int V, int U>
__device__ __forceinline__ void load_weight(float (&w)[U][2 * V], const float* weight, const Unit<V> (&unit)[U]) {
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = weight != nullptr && unit[k].has ? weight[unit[k].first + i] : 1.f;
            w[k][V + i] = weight != nullptr && unit[k].has_second ? weight[unit[k].second + i] : 1.f;
        }
}

template <typename T, int V, int U>
__global__ void __launch_bounds__(THREADS) head_fwd_kernel(HeadView q, HeadView k, const float* __restrict__ q_weight, const float* __restrict__ k_weight,
                                                           T* __restrict__ q_out, T* __restrict__ k_out, HeadShape s) {
    __shared__ Tile t;
    pdl_wait_then_trigger();
    const int64_t first = (int64_t)blockIdx.x * s.tile;
    const int count = (int)min((int64_t)s.tile, s.nodes - first);
    open_tile(t, s, first, count);
    const int lane = threadIdx.x & (s.lanes - 1), groups = THREADS / s.lanes, group = threadIdx.x / s.lanes;
    Unit<V> unit[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit[i] = unit_at<V>(s, lane + i * s.lanes);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const HeadView x = which ? k : q;
        T* out = which ? k_out : q_out;
        const int heads = s.heads[which];
        if (heads == 0) continue;
        float w[U][2 * V];
        if (s.norm) load_weight<V, U>(w, which ? k_weight : q_weight, unit);
        const int items = count * heads, rounds = (items + groups - 1) / groups;      // the same for all groups: their sums are warps' shuffles
#pragma unroll 2
        for (int r = 0; r < rounds; ++r) {
            const int item = group + r * groups;
            const bool in = item < items;
            const int n = in ? item / heads : 0, h = in ? item - n * heads : 0;
            const T* from = (const T*)x.p + t.batch[n] * x.batch + t.node[n] * x.node + h * x.head;
            float v[U][2 * V];
#pragma unroll
            for (int i = 0; i < U; ++i) load_unit<T, V>(v[i], from, unit[i]);
            if (s.norm) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) sum = fmaf(v[i][e], v[i][e], sum);
                const float scale = 1.f / sqrtf(group_sum(sum, s.lanes) / s.dim + s.eps);
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) v[i][e] = v[i][e] * scale * w[i][e];
            }
            if (!in) continue;
            T* to = out + ((first + n) * heads + h) * s.dim;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                turn<V>(v[i], unit[i], t, n, s);
                store_unit<T, V>(to, unit[i], v[i]);
            }
        }
    }
}

// Gradients with norm; part: (blocks, 2, dim), this block's shares of the weights' gradients.
template <typename T, int V, int U>
__global__ void __launch_bounds__(THREADS) head_bwd_kernel(HeadView q, HeadView k, HeadView gq, HeadView gk, const float* __restrict__ q_weight,
                                                           const float* __restrict__ k_weight, T* __restrict__ gx_q, T* __restrict__ gx_k,
                                                           float* __restrict__ part, HeadShape s) {
    __shared__ Tile t;
    __shared__ float shares[THREADS * U * 2 * V];
    pdl_wait_then_trigger();
    const int lane = threadIdx.x & (s.lanes - 1), groups = THREADS / s.lanes, group = threadIdx.x / s.lanes;
    Unit<V> unit[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit[i] = unit_at<V>(s, lane + i * s.lanes);
    float gw[2][U][2 * V] = {};
    for (int64_t first = (int64_t)blockIdx.x * s.tile; first < s.nodes; first += (int64_t)gridDim.x * s.tile) {
        const int count = (int)min((int64_t)s.tile, s.nodes - first);
        open_tile(t, s, first, count);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const HeadView x = which ? k : q, g = which ? gk : gq;
            T* out = which ? gx_k : gx_q;
            const int heads = s.heads[which];
            if (heads == 0) continue;
            float w[U][2 * V];
            load_weight<V, U>(w, which ? k_weight : q_weight, unit);
            const int items = count * heads, rounds = (items + groups - 1) / groups;
            for (int r = 0; r < rounds; ++r) {
                const int item = group + r * groups;
                const bool in = item < items;
                const int n = in ? item / heads : 0, h = in ? item - n * heads : 0;
                const T* from = (const T*)x.p + t.batch[n] * x.batch + t.node[n] * x.node + h * x.head;
                const T* up = (const T*)g.p + t.batch[n] * g.batch + t.node[n] * g.node + h * g.head;
                float v[U][2 * V], d[U][2 * V], sum = 0.f, along = 0.f;
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    load_unit<T, V>(v[i], from, unit[i]);
                    load_unit<T, V>(d[i], up, unit[i]);
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    turn<V>(d[i], unit[i], t, n, s);
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) sum = fmaf(v[i][e], v[i][e], sum);
                }
                const float scale = 1.f / sqrtf(group_sum(sum, s.lanes) / s.dim + s.eps);
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) {
                        v[i][e] *= scale;
                        along = fmaf(d[i][e] * w[i][e], v[i][e], along);
                        if (in) gw[which][i][e] = fmaf(d[i][e], v[i][e], gw[which][i][e]);
                    }
                along = group_sum(along, s.lanes) / s.dim;
                if (!in) continue;
                T* to = out + ((first + n) * heads + h) * s.dim;
#pragma unroll
                for (int i = 0; i < U; ++i) {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) v[i][e] = scale * fmaf(-along, v[i][e], d[i][e] * w[i][e]);
                    store_unit<T, V>(to, unit[i], v[i]);
                }
            }
        }
        __syncthreads();              // before the next tile's angles
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        // by group and feature; a feature that does not exist has no place
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (unit[i].has) shares[group * s.dim + unit[i].first + e] = gw[which][i][e];
                if (unit[i].has_second) shares[group * s.dim + unit[i].second + e] = gw[which][i][V + e];
            }
        __syncthreads();
        for (int f = threadIdx.x; f < s.dim; f += THREADS) {
            float sum = 0.f;
            for (int j = 0; j < groups; ++j) sum += shares[j * s.dim + f];
            part[((int64_t)blockIdx.x * 2 + which) * s.dim + f] = sum;
        }
    }
}

// Sums over the blocks, 8 shares at a time; no blocks: zeros.
__global__ void __launch_bounds__(256) head_sum_kernel(const float* __restrict__ part, int blocks, int dim, float* __restrict__ gq_weight,
                                                       float* __restrict__ gk_weight) {
    __shared__ double rows[8][33];
    pdl_wait_then_trigger();
    const int f = blockIdx.x * 32 + threadIdx.x;
    double sum = 0.;
    if (f < 2 * dim)
        for (int b = threadIdx.y; b < blocks; b += 8) sum += part[(int64_t)b * 2 * dim + f];
    rows[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y != 0 || f >= 2 * dim) return;
#pragma unroll
    for (int j = 1; j < 8; ++j) sum += rows[j][threadIdx.x];
    float* to = f < dim ? gq_weight : gk_weight;
    if (to != nullptr) to[f < dim ? f : f - dim] = (float)sum;
}

// ------------------------------------------------------------------------------------------- host
int check_head_sizes(const fpde_head_args* a) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->dim < 1 || a->dim > FPDE_HEAD_MAX_DIM || a->pairs < 0 || 2 * (int64_t)a->pairs > a->dim) return FPDE_ERR_PARAM;
    const int64_t most = 1 << 20;
    if (a->batch < 0 || a->length < 0 || a->q_heads < 0 || a->k_heads < 0 || a->q_heads > most || a->k_heads > most || a->batch > (1ll << 36) ||
        a->length > (1ll << 36) || !product_fits(a->batch, a->length, (a->q_heads + a->k_heads) * a->dim))
        return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

int64_t nodes_of(const fpde_head_args* a) { return a->batch * a->length; }

HeadShape head_shape(const fpde_head_args* a, int v, float sign) {
    HeadShape s = {};
    s.length = a->length;
    s.nodes = nodes_of(a);
    s.positions = a->positions;
    s.pos_batch = a->pos_batch;
    s.pos_node = a->pos_node;
    s.offset = a->offset;
    s.inv_freq = a->inv_freq;
    s.heads[0] = (int)a->q_heads;
    s.heads[1] = (int)a->k_heads;
    s.dim = (int)a->dim;
    s.pairs = a->pairs;
    s.interleaved = a->interleaved;
    s.norm = a->norm;
    s.eps = (float)a->eps;
    s.sign = sign;
    const int units = (int)ceil_div(a->dim, 2 * v);
    s.lanes = 1;
    while (s.lanes < units && s.lanes < 32) s.lanes *= 2;
    // enough blocks to fill the GPU first, then as many nodes as share a block's start
    const int64_t room = s.nodes / (148 * 8);
    s.tile = room < 1 ? 1 : room > MOST_TILE ? MOST_TILE : (int)room;
    return s;
}

int grad_blocks(const HeadShape& s) { return (int)(ceil_div(s.nodes, s.tile) < GRAD_BLOCKS ? ceil_div(s.nodes, s.tile) : GRAD_BLOCKS); }

// Elements of a pack: the most that 16 bytes, the pairs, the rest of a head and every array's alignment allow.
int pack_of(const fpde_head_args* a, const HeadView* in, int inputs, const void* out_q, const void* out_k) {
    const size_t e = dtype_bytes(a->dtype);
    for (int v = (int)(16 / e); v > 1; v /= 2) {
        bool ok = a->pairs % v == 0 && (a->dim - 2 * a->pairs) % (2 * v) == 0 && aligned(out_q, e * v) && aligned(out_k, e * v);
        for (int i = 0; i < inputs; ++i) ok = ok && packs(in[i].p, in[i].batch, in[i].node, e, v) && in[i].head % v == 0;
        if (ok) return v;
    }
    return 1;
}

struct HeadCall {
    const fpde_head_args* a;
    HeadView q, k, gq, gk;
    void *out_q, *out_k;
    float sign;
    bool grad;                // of the norm
    cudaStream_t st;
};

template <typename T, int V, int U>
cudaError_t head_launch(const HeadCall& c) {
    const HeadShape s = head_shape(c.a, V, c.sign);
    if (c.grad) {
        const int blocks = grad_blocks(s);
        const cudaError_t e = launch_kernel(head_bwd_kernel<T, V, U>, dim3(blocks), dim3(THREADS), c.st, c.q, c.k, c.gq, c.gk, c.a->q_weight,
                                            c.a->k_weight, (T*)c.out_q, (T*)c.out_k, (float*)c.a->workspace, s);
        if (e != cudaSuccess) return e;
        return launch_kernel(head_sum_kernel, dim3((unsigned)ceil_div(2 * s.dim, 32)), dim3(32, 8), c.st, (const float*)c.a->workspace, blocks, s.dim,
                             c.a->gq_weight, c.a->gk_weight);
    }
    const int64_t blocks = ceil_div(s.nodes, s.tile);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(head_fwd_kernel<T, V, U>, dim3((unsigned)blocks), dim3(THREADS), c.st, c.q, c.k, c.a->q_weight, c.a->k_weight, (T*)c.out_q,
                         (T*)c.out_k, s);
}

template <typename T>
cudaError_t head_by_pack(const HeadCall& c) {
    const HeadView in[] = {c.q, c.k, c.gq, c.gk};
    const int v = pack_of(c.a, in, c.grad ? 4 : 2, c.out_q, c.out_k);
    const int64_t units = ceil_div(c.a->dim, 2 * v);
    if constexpr (sizeof(T) == 2)
        if (v == 8) return head_launch<T, 8, 1>(c);
    if (v == 4) return head_launch<T, 4, 1>(c);
    if (v == 2) return units > 32 ? head_launch<T, 2, 2>(c) : head_launch<T, 2, 1>(c);
    return units > 64 ? head_launch<T, 1, 4>(c) : units > 32 ? head_launch<T, 1, 2>(c) : head_launch<T, 1, 1>(c);
}

int head_run(const HeadCall& c) {
    const cudaError_t e = c.a->dtype == FPDE_F32 ? head_by_pack<float>(c) : c.a->dtype == FPDE_BF16 ? head_by_pack<__nv_bfloat16>(c) : head_by_pack<__half>(c);
    return e == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
}

int check_head(const fpde_head_args* a) {
    const int st = check_head_sizes(a);
    if (st != FPDE_OK) return st;
    if (a->norm && !(a->eps >= 0. && a->eps < 1e30)) return FPDE_ERR_PARAM;
    if (nodes_of(a) > 0 && a->pairs > 0 && a->inv_freq == nullptr) return FPDE_ERR_NULL;
    if (!aligned(a->inv_freq, 4) || !aligned(a->positions, 8) || !aligned(a->q_weight, 4) || !aligned(a->k_weight, 4)) return FPDE_ERR_ALIGN;
    return FPDE_OK;
}

HeadView view_q(const fpde_head_args* a) { return {a->q_heads > 0 ? a->q : nullptr, a->q_batch, a->q_node, a->q_head}; }
HeadView view_k(const fpde_head_args* a) { return {a->k_heads > 0 ? a->k : nullptr, a->k_batch, a->k_node, a->k_head}; }
HeadView view_gq(const fpde_head_args* a) { return {a->q_heads > 0 ? a->gq : nullptr, a->gq_batch, a->gq_node, a->gq_head}; }
HeadView view_gk(const fpde_head_args* a) { return {a->k_heads > 0 ? a->gk : nullptr, a->gk_batch, a->gk_node, a->gk_head}; }

// One of q's or k's arrays: there, and on its elements, if there are such heads at all.
int check_array(const void* p, int64_t heads, size_t e) { return heads == 0 ? FPDE_OK : p == nullptr ? FPDE_ERR_NULL : aligned(p, e) ? FPDE_OK : FPDE_ERR_ALIGN; }

}  // namespace
}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_head_rotary_workspace_bytes(const fpde_head_args* a) {
    if (check_head_sizes(a) != FPDE_OK || !a->norm) return 0;
    return (size_t)GRAD_BLOCKS * 2 * a->dim * sizeof(float);
}

int fpde_head_rotary_fwd(const fpde_head_args* a, void* stream) {
    int st = check_head(a);
    if (st != FPDE_OK) return st;
    if (nodes_of(a) * (a->q_heads + a->k_heads) == 0) return FPDE_OK;
    const size_t e = dtype_bytes(a->dtype);
    if ((st = check_array(a->q, a->q_heads, e)) || (st = check_array(a->q_out, a->q_heads, e)) || (st = check_array(a->k, a->k_heads, e)) ||
        (st = check_array(a->k_out, a->k_heads, e)))
        return st;
    return head_run({a, view_q(a), view_k(a), {}, {}, a->q_out, a->k_out, 1.f, false, (cudaStream_t)stream});
}

int fpde_head_rotary_bwd(const fpde_head_args* a, void* stream) {
    int st = check_head(a);
    if (st != FPDE_OK) return st;
    const size_t e = dtype_bytes(a->dtype);
    const bool any = nodes_of(a) * (a->q_heads + a->k_heads) > 0;
    if (any && ((st = check_array(a->gq, a->q_heads, e)) || (st = check_array(a->gx_q, a->q_heads, e)) || (st = check_array(a->gk, a->k_heads, e)) ||
                (st = check_array(a->gx_k, a->k_heads, e))))
        return st;
    if (!a->norm) return any ? head_run({a, view_gq(a), view_gk(a), {}, {}, a->gx_q, a->gx_k, -1.f, false, (cudaStream_t)stream}) : FPDE_OK;
    if (any && ((st = check_array(a->q, a->q_heads, e)) || (st = check_array(a->k, a->k_heads, e)))) return st;
    if (!aligned(a->gq_weight, 4) || !aligned(a->gk_weight, 4)) return FPDE_ERR_ALIGN;
    if (!any)        // no nodes: the sums over them are zero
        return launch_kernel(head_sum_kernel, dim3((unsigned)ceil_div(2 * a->dim, 32)), dim3(32, 8), (cudaStream_t)stream, (const float*)nullptr, 0,
                             (int)a->dim, a->gq_weight, a->gk_weight) == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
    if (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < fpde_head_rotary_workspace_bytes(a)) return FPDE_ERR_WORKSPACE;
    return head_run({a, view_q(a), view_k(a), view_gq(a), view_gk(a), a->gx_q, a->gx_k, -1.f, true, (cudaStream_t)stream});
}

}  // extern "C"
