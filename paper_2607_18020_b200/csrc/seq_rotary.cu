// Rotation of queries and keys by their position, with or without a norm of each head before it, and the
// gradients.
//
//   u = x / sqrt(mean(x^2) + eps) * weight;  y = u with pair i of its first 2 * pairs features turned by
//   position * inv_freq[i]
//
// Every element is read and written once; memory bounds it.
//
// A block takes a tile of nodes.  First it forms the cosines and sines of the tile's angles, once for all heads,
// in shared memory.  An angle is counted in 2^-64 of a turn: positions are whole numbers, so inv_freq / 2 pi may lose its whole
// turns, and a 64-bit product that wraps is the angle's remainder; the 32-bit sine and cosine of that are good to their
// last bits at any position.  Then groups of 1 to 32 lanes take two neighbouring heads of a node at a time, neighbouring groups
// neighbouring heads.  A lane holds both members of V pairs (or 2 V features that are not turned), in two packs of up
// to 16 bytes; sums over a head are shuffles among the group's lanes.  The angles and the weight are read from shared
// memory for both heads at once (for one head at a time its data pipe was half busy at half of memory's rate).
//
// What a lane reads comes through places of its own in shared memory, copied there one or two items ahead: registers
// hold too little of it.  8 x 4096 nodes of 32 heads of 128 in bf16, forward with norm, floor 82 us: 146 us with the loads of one item in
// registers (24 warps an SM that load, then compute), 160 to 186 with two ahead in registers (16 warps).
//
// Gradients.  The rotation's is the rotation by the opposite angle: the same kernel.  With g the upstream gradient
// turned back, n = x r, r = 1 / sqrt(mean(x^2) + eps):  gx = r (g w - n mean(g w n)),  gw = sum over nodes and heads of g n.
// A lane keeps its features' share of gw in registers over all tiles of its block (a grid of fixed size), a block
// sums its groups' shares, and a second kernel the blocks', all in a fixed order.
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int THREADS = 256;
constexpr int MOST_TILE = 64, MOST_ANGLES = 2048;      // of a tile: nodes, and nodes times pairs
constexpr int MOST_PAIRS = FPDE_HEAD_MAX_DIM / 2;
constexpr int GRAD_BLOCKS = 148 * 2;           // blocks of the gradients of the norm, at most: two an SM

struct HeadView {
    const void* p;
    int64_t batch, node, head;
};

struct HeadShape {
    int64_t length, nodes, pos_batch, pos_node, offset;
    const int64_t* positions;
    const float* inv_freq;
    int heads0, heads1;       // of q and k
    int dim, pairs, interleaved, norm;
    int lanes;                // of a group: a power of two
    int tile;                 // nodes a block takes at once
    float eps, sign, inv_dim;
};

struct Tile {
    int64_t batch[MOST_TILE], node[MOST_TILE];
    uint64_t position[MOST_TILE], turn[MOST_PAIRS];        // turn: 2^-64 turns a node
    float sound[MOST_PAIRS];                               // 1, or NaN for a frequency that is infinite or NaN
    alignas(16) float cosine[MOST_ANGLES];
    alignas(16) float sine[MOST_ANGLES];
};

// Before the first tile: what a node turns each pair by.
__device__ __forceinline__ void open_turns(Tile& t, const HeadShape& s) {
    for (int i = threadIdx.x; i < s.pairs; i += THREADS) {
        // rounded once, relative to its size: 1e-10 of a turn at position 10^6
        double turns = (double)s.inv_freq[i] * 0.15915494309189535;
        turns -= rint(turns);
        t.turn[i] = (uint64_t)__double2ll_rn(turns * 0x1p63) << 1;
        t.sound[i] = turns - turns == 0. ? 1.f : NAN;          // a whole number cannot say it
    }
}
// The nodes of the tile that starts at node `first` of all rows.
__device__ __forceinline__ void open_nodes(Tile& t, const HeadShape& s, int64_t first, int count) {
    if (threadIdx.x < count) {
        const int64_t n = first + threadIdx.x, b = n / s.length;
        t.batch[threadIdx.x] = b;
        t.node[threadIdx.x] = n - b * s.length;
        const int64_t at = s.positions != nullptr ? s.positions[b * s.pos_batch + (n - b * s.length) * s.pos_node] : n - b * s.length;
        t.position[threadIdx.x] = (uint64_t)at + (uint64_t)s.offset;
    }
    __syncthreads();
}
// And the cosines and sines of their angles.
__device__ __forceinline__ void open_angles(Tile& t, const HeadShape& s, int count) {
    for (int i = threadIdx.x; i < count * s.pairs; i += THREADS) {
        const int n = i / s.pairs, pair = i - n * s.pairs;
        float c, q;
        sincospif((float)(int64_t)(t.position[n] * t.turn[pair]) * 0x1p-63f, &q, &c);
        t.cosine[i] = c * t.sound[pair];
        t.sine[i] = q * s.sign * t.sound[pair];
    }
    __syncthreads();
}

// Where in its head a lane's unit lies: two packs of V features.  Neighbouring lanes hold neighbouring packs, first of the first half
// of what is turned, or is not, then of the second: with a lane's two packs side by side a warp touches every 32 bytes twice (4 x 4096
// nodes of 20 heads of 128, half of them turned in pairs of neighbours, bf16: 45 us, 31 so).
template <int V>
struct Unit {
    int first, second;        // features
    int pair, other;          // first pairs: of the unit, and of its second pack where pairs are neighbours; -1: not turned
    bool has, has_second;     // V = 1: an odd head's last feature has no second
};
template <int V>
__device__ __forceinline__ Unit<V> unit_at(const HeadShape& s, int u) {
    Unit<V> r = {0, 0, -1, -1, false, false};
    const int turned = s.pairs / V, left = (s.dim - 2 * s.pairs + 2 * V - 1) / (2 * V), x = u - turned;
    if (x < 0) {
        const bool split = V == 1 && s.interleaved;        // a pair over two packs
        r.pair = V > 1 && s.interleaved ? u * V / 2 : u * V;
        r.other = s.pairs / 2 + r.pair;
        r.first = split ? 2 * u : u * V;
        r.second = split ? 2 * u + 1 : u * V + s.pairs;
        r.has = r.has_second = true;
    } else if (x < left) {
        r.first = 2 * s.pairs + x * V;
        r.second = r.first + left * V;
        r.has = true;
        r.has_second = r.second < s.dim;
    }
    if (!r.has_second) r.second = r.first;                 // a place in the weights all the same
    return r;
}

// A lane's own places in shared memory: `stage` times PACKS packs, thread by thread.
template <typename T, int V, int PACKS>
struct Ring {
    static constexpr int BYTES = V * sizeof(T);
    uint32_t at;
    __device__ __forceinline__ explicit Ring(const void* base) : at((uint32_t)__cvta_generic_to_shared(base) + threadIdx.x * BYTES) {}
    __device__ __forceinline__ uint32_t place(int stage, int pack) const { return at + (stage * PACKS + pack) * THREADS * BYTES; }
    // `from` on its way to a place; zeros if there is nothing
    __device__ __forceinline__ void ask(int stage, int pack, const T* from, bool there) const {
        const uint32_t to = place(stage, pack);
        if constexpr (BYTES == 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
        else if constexpr (BYTES >= 4)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
        else {          // too little for the copy engine's smallest
            const uint16_t v = there ? *reinterpret_cast<const uint16_t*>(from) : (uint16_t)0;
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"(v) : "memory");
        }
    }
    __device__ __forceinline__ void get(float* v, int stage, int pack) const {
        Pack<T, V> k;
        const uint32_t from = place(stage, pack);
        if constexpr (BYTES == 16) {
            uint4& x = reinterpret_cast<uint4&>(k);
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(from) : "memory");
        } else if constexpr (BYTES == 8) {
            uint2& x = reinterpret_cast<uint2&>(k);
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(from) : "memory");
        } else if constexpr (BYTES == 4) {
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(reinterpret_cast<uint32_t&>(k)) : "r"(from) : "memory");
        } else {
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(reinterpret_cast<uint16_t&>(k)) : "r"(from) : "memory");
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_f32<T>(k.v[i]);
    }
};
__device__ __forceinline__ void ring_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void ring_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
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
// A unit's angles; what is not turned has cosine 1 and sine 0, and is left alone all the same (an infinity times 0 is none).
template <int V>
struct Angles {
    float c[V], s[V];
};
template <int V>
__device__ __forceinline__ Angles<V> angles_of(const Unit<V>& u, const Tile& t, int n, const HeadShape& s) {
    constexpr int W = V > 4 ? 4 : V;
    Angles<V> a = {};
    if (u.pair < 0) return a;
    const float *cosine = t.cosine + n * s.pairs, *sine = t.sine + n * s.pairs;
    if constexpr (V > 1)
        if (s.interleaved) {
            constexpr int H = V / 2;
            const Pack<float, H> c0 = load_pack<float, H>(cosine + u.pair), c1 = load_pack<float, H>(cosine + u.other), s0 = load_pack<float, H>(sine + u.pair),
                                 s1 = load_pack<float, H>(sine + u.other);
#pragma unroll
            for (int i = 0; i < H; ++i) {
                a.c[i] = c0.v[i];
                a.c[H + i] = c1.v[i];
                a.s[i] = s0.v[i];
                a.s[H + i] = s1.v[i];
            }
            return a;
        }
#pragma unroll
    for (int i = 0; i < V; i += W) {
        const Pack<float, W> c = load_pack<float, W>(cosine + u.pair + i), q = load_pack<float, W>(sine + u.pair + i);
#pragma unroll
        for (int e = 0; e < W; ++e) {
            a.c[i + e] = c.v[e];
            a.s[i + e] = q.v[e];
        }
    }
    return a;
}
template <int V>
__device__ __forceinline__ void turn(float (&v)[2 * V], const Unit<V>& u, const Angles<V>& a, bool interleaved) {
    if (u.pair < 0) return;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float x = v[2 * i], y = v[2 * i + 1];
            v[2 * i] = x * a.c[i] - y * a.s[i];
            v[2 * i + 1] = y * a.c[i] + x * a.s[i];
        }
    } else if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const uint64_t x = pair(v[i], v[i + 1]), y = pair(v[V + i], v[V + i + 1]), c = pair(a.c[i], a.c[i + 1]), s = pair(a.s[i], a.s[i + 1]);
            unpair(fma2(x, c, mul2(y, mul2(s, both(-1.f)))), v[i], v[i + 1]);
            unpair(fma2(y, c, mul2(x, s)), v[V + i], v[V + i + 1]);
        }
    } else {
        const float x = v[0], y = v[1];
        v[0] = x * a.c[0] - y * a.s[0];
        v[1] = y * a.c[0] + x * a.s[0];
    }
}
// 1 / sqrt(x): the hardware's, with one step of Newton's
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x);
    const float d = fmaf(-x * r, r, 1.f);                  // an x of 0 has an infinite root, which it keeps
    return d - d == 0.f ? fmaf(r * 0.5f, d, r) : r;
}
template <int V, int U>
__device__ __forceinline__ float square_sum(const float (&v)[U][2 * V]) {
    uint64_t sum = both(0.f);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < 2 * V; e += 2) {
            const uint64_t x = pair(v[i][e], v[i][e + 1]);
            sum = fma2(x, x, sum);
        }
    return sum2(sum);
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int m = lanes / 2; m > 0; m /= 2) v += __shfl_xor_sync(~0u, v, m);
    return v;
}

// A unit's weights, from shared memory: there is one for every place that a lane may stand for.
template <int V>
__device__ __forceinline__ void load_weight(float (&w)[2 * V], const float* weight, const Unit<V>& u) {
    constexpr int W = V > 4 ? 4 : V;
#pragma unroll
    for (int i = 0; i < V; i += W) {
        const Pack<float, W> a = load_pack<float, W>(weight + u.first + i), b = load_pack<float, W>(weight + u.second + i);
#pragma unroll
        for (int e = 0; e < W; ++e) {
            w[i + e] = a.v[e];
            w[V + i + e] = b.v[e];
        }
    }
}

// Two heads of a node, of q or of k: an item.  The items of a tile are numbered node by node, q's before k's.
struct Items {
    int of_q, each, step_n, step_h;            // of a node's q, and of a node; from one of a group's items to its next
    __device__ __forceinline__ Items(int hq, int hk, int groups) {
        of_q = (hq + 1) / 2;
        each = of_q + (hk + 1) / 2;
        step_n = groups / each;
        step_h = groups - step_n * each;
    }
    __device__ __forceinline__ void on(int& n, int& i) const {
        n += step_n;
        i += step_h;
        if (i >= each) {
            i -= each;
            ++n;
        }
    }
};

constexpr int FWD_BLOCKS = 3;                  // resident on an SM
constexpr int STAGES = 3, GRAD_STAGES = 2;     // items of a group in shared memory: the one at hand and those on their way

template <typename T, int V, int U>
__global__ void __launch_bounds__(THREADS, FWD_BLOCKS) head_fwd_kernel(HeadView q, HeadView k, const float* __restrict__ q_weight, const float* __restrict__ k_weight,
                                                              T* __restrict__ q_out, T* __restrict__ k_out, HeadShape s) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Tile t;
    __shared__ alignas(16) float weights[2][FPDE_HEAD_MAX_DIM];
    pdl_wait_then_trigger();
    const int64_t first = (int64_t)blockIdx.x * s.tile;
    const int count = (int)min((int64_t)s.tile, s.nodes - first);
    if (s.norm)
        for (int i = threadIdx.x; i < FPDE_HEAD_MAX_DIM; i += THREADS) {
            weights[0][i] = q_weight != nullptr && i < s.dim ? q_weight[i] : 1.f;
            weights[1][i] = k_weight != nullptr && i < s.dim ? k_weight[i] : 1.f;
        }
    open_turns(t, s);
    open_nodes(t, s, first, count);
    const int lane = threadIdx.x & (s.lanes - 1), groups = THREADS / s.lanes, group = threadIdx.x / s.lanes;
    const Items items(s.heads0, s.heads1, groups);
    Unit<V> unit[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit[i] = unit_at<V>(s, lane + i * s.lanes);
    const Ring<T, V, 4 * U> ring(dynamic);
    int n = group / items.each, at = group - n * items.each, ask_n = n, ask_at = at;
    auto ask = [&](int stage) {
        const bool in = ask_n < count, of_k = ask_at >= items.of_q;
        const int node = in ? ask_n : 0, h = 2 * (of_k ? ask_at - items.of_q : ask_at), heads = of_k ? s.heads1 : s.heads0;
        const int64_t step = of_k ? k.head : q.head;
        const T* from = of_k ? (const T*)k.p + t.batch[node] * k.batch + t.node[node] * k.node + h * step
                             : (const T*)q.p + t.batch[node] * q.batch + t.node[node] * q.node + h * step;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const bool there = in && h + j < heads;
                ring.ask(stage, (2 * j) * U + i, from + j * step + unit[i].first, there && unit[i].has);
                ring.ask(stage, (2 * j + 1) * U + i, from + j * step + unit[i].second, there && unit[i].has_second);
            }
        ring_close();
        items.on(ask_n, ask_at);
    };
#pragma unroll
    for (int j = 0; j < STAGES - 1; ++j) ask(j);
    open_angles(t, s, count);
    const int rounds = (count * items.each + groups - 1) / groups;      // the same for all groups: sums are whole warps' shuffles
    int stage = 0;
#pragma unroll 1
    for (int r = 0; r < rounds; ++r, items.on(n, at)) {
        const bool in = n < count, of_k = at >= items.of_q;
        const int node = in ? n : 0, h = 2 * (of_k ? at - items.of_q : at), heads = of_k ? s.heads1 : s.heads0;
        ask(stage == 0 ? STAGES - 1 : stage - 1);
        T* to = (of_k ? k_out : q_out) + ((first + n) * heads + h) * s.dim;
        Angles<V> angles[U];
        float w[U][2 * V];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            angles[i] = angles_of<V>(unit[i], t, node, s);
            if (s.norm) load_weight<V>(w[i], weights[of_k], unit[i]);
        }
        ring_wait<STAGES - 1>();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float v[U][2 * V];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                ring.get(v[i], stage, (2 * j) * U + i);
                ring.get(v[i] + V, stage, (2 * j + 1) * U + i);
            }
            if (s.norm) {
                const uint64_t scale = both(inverse_root(fmaf(group_sum(square_sum<V, U>(v), s.lanes), s.inv_dim, s.eps)));
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int e = 0; e < 2 * V; e += 2)
                        unpair(mul2(mul2(pair(v[i][e], v[i][e + 1]), scale), pair(w[i][e], w[i][e + 1])), v[i][e], v[i][e + 1]);
            }
            if (in && h + j < heads) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    turn<V>(v[i], unit[i], angles[i], s.interleaved);
                    store_unit<T, V>(to + j * s.dim, unit[i], v[i]);
                }
            }
        }
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    ring_wait<0>();
}

// Gradients with norm, of q in the first q_blocks blocks and of k in the others; part: (blocks, dim), this block's share of its
// weight's gradient.
template <typename T, int V, int U>
__global__ void __launch_bounds__(THREADS, 2) head_bwd_kernel(HeadView q, HeadView k, HeadView gq, HeadView gk, const float* __restrict__ q_weight,
                                                              const float* __restrict__ k_weight, T* __restrict__ gx_q, T* __restrict__ gx_k,
                                                              float* __restrict__ part, int q_blocks, HeadShape s) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Tile t;
    __shared__ alignas(16) float weight[FPDE_HEAD_MAX_DIM];
    pdl_wait_then_trigger();
    const bool of_k = (int)blockIdx.x >= q_blocks;
    const int block = of_k ? blockIdx.x - q_blocks : blockIdx.x, blocks = of_k ? gridDim.x - q_blocks : q_blocks;
    const int64_t x_batch = of_k ? k.batch : q.batch, x_node = of_k ? k.node : q.node, x_head = of_k ? k.head : q.head;
    const int64_t g_batch = of_k ? gk.batch : gq.batch, g_node = of_k ? gk.node : gq.node, g_head = of_k ? gk.head : gq.head;
    const T *x = (const T*)(of_k ? k.p : q.p), *g = (const T*)(of_k ? gk.p : gq.p);
    T* out = of_k ? gx_k : gx_q;
    const int heads = of_k ? s.heads1 : s.heads0;
    const int lane = threadIdx.x & (s.lanes - 1), groups = THREADS / s.lanes, group = threadIdx.x / s.lanes;
    const Items items(heads, 0, groups);
    Unit<V> unit[U];
#pragma unroll
    for (int i = 0; i < U; ++i) unit[i] = unit_at<V>(s, lane + i * s.lanes);
    float gw[U][2 * V] = {};
    const float* given = of_k ? k_weight : q_weight;
    for (int i = threadIdx.x; i < FPDE_HEAD_MAX_DIM; i += THREADS) weight[i] = given != nullptr && i < s.dim ? given[i] : 1.f;
    open_turns(t, s);
    const Ring<T, V, 8 * U> ring(dynamic);
    for (int64_t first = (int64_t)block * s.tile; first < s.nodes; first += (int64_t)blocks * s.tile) {
        const int count = (int)min((int64_t)s.tile, s.nodes - first);
        open_nodes(t, s, first, count);
        int n = group / items.each, at = group - n * items.each, ask_n = n, ask_at = at;
        auto ask = [&](int stage) {
            const bool in = ask_n < count;
            const int node = in ? ask_n : 0, h = 2 * ask_at;
            const T *from = x + t.batch[node] * x_batch + t.node[node] * x_node + h * x_head, *up = g + t.batch[node] * g_batch + t.node[node] * g_node + h * g_head;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const bool there = in && h + j < heads;
                    ring.ask(stage, (4 * j) * U + i, from + j * x_head + unit[i].first, there && unit[i].has);
                    ring.ask(stage, (4 * j + 1) * U + i, from + j * x_head + unit[i].second, there && unit[i].has_second);
                    ring.ask(stage, (4 * j + 2) * U + i, up + j * g_head + unit[i].first, there && unit[i].has);
                    ring.ask(stage, (4 * j + 3) * U + i, up + j * g_head + unit[i].second, there && unit[i].has_second);
                }
            ring_close();
            items.on(ask_n, ask_at);
        };
#pragma unroll
        for (int j = 0; j < GRAD_STAGES - 1; ++j) ask(j);
        open_angles(t, s, count);
        const int rounds = (count * items.each + groups - 1) / groups;
        int stage = 0;
#pragma unroll 1
        for (int r = 0; r < rounds; ++r, items.on(n, at)) {
            const bool in = n < count;
            const int node = in ? n : 0, h = 2 * at;
            ask(stage == 0 ? GRAD_STAGES - 1 : stage - 1);
            T* to = out + ((first + n) * heads + h) * s.dim;
            Angles<V> angles[U];
#pragma unroll
            for (int i = 0; i < U; ++i) angles[i] = angles_of<V>(unit[i], t, node, s);
            ring_wait<GRAD_STAGES - 1>();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float v[U][2 * V], d[U][2 * V];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    ring.get(v[i], stage, (4 * j) * U + i);
                    ring.get(v[i] + V, stage, (4 * j + 1) * U + i);
                    ring.get(d[i], stage, (4 * j + 2) * U + i);
                    ring.get(d[i] + V, stage, (4 * j + 3) * U + i);
                }
                float sum = square_sum<V, U>(v);
                uint64_t dots = both(0.f);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    turn<V>(d[i], unit[i], angles[i], s.interleaved);
                    float w[2 * V];
                    load_weight<V>(w, weight, unit[i]);
#pragma unroll
                    for (int e = 0; e < 2 * V; e += 2)
                        dots = fma2(mul2(pair(d[i][e], d[i][e + 1]), pair(w[e], w[e + 1])), pair(v[i][e], v[i][e + 1]), dots);
                }
                float along = sum2(dots);
                for (int m = s.lanes / 2; m > 0; m /= 2) {
                    sum += __shfl_xor_sync(~0u, sum, m);
                    along += __shfl_xor_sync(~0u, along, m);
                }
                if (!in || h + j >= heads) continue;
                const float scale = inverse_root(fmaf(sum, s.inv_dim, s.eps));
                const uint64_t r = both(scale), back = both(-along * scale * s.inv_dim);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    float w[2 * V];
                    load_weight<V>(w, weight, unit[i]);
#pragma unroll
                    for (int e = 0; e < 2 * V; e += 2) {
                        const uint64_t n = mul2(pair(v[i][e], v[i][e + 1]), r), g = pair(d[i][e], d[i][e + 1]);
                        unpair(fma2(g, n, pair(gw[i][e], gw[i][e + 1])), gw[i][e], gw[i][e + 1]);
                        unpair(mul2(r, fma2(back, n, mul2(g, pair(w[e], w[e + 1])))), v[i][e], v[i][e + 1]);
                    }
                    store_unit<T, V>(to + j * s.dim, unit[i], v[i]);
                }
            }
            stage = stage == GRAD_STAGES - 1 ? 0 : stage + 1;
        }
        ring_wait<0>();
        __syncthreads();              // before the next tile's angles
    }
    float* shares = reinterpret_cast<float*>(dynamic);      // by group and feature; a feature that does not exist has no place
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (unit[i].has) shares[group * s.dim + unit[i].first + e] = gw[i][e];
            if (unit[i].has_second) shares[group * s.dim + unit[i].second + e] = gw[i][V + e];
        }
    __syncthreads();
    for (int f = threadIdx.x; f < s.dim; f += THREADS) {
        float sum = 0.f;
        for (int j = 0; j < groups; ++j) sum += shares[j * s.dim + f];
        part[(int64_t)blockIdx.x * s.dim + f] = sum;
    }
}

// Sums over the blocks of q and those of k, 32 rows of threads and four shares of each at a time; no blocks: zeros.
constexpr int SUM_ROWS = 32;
__global__ void __launch_bounds__(32 * SUM_ROWS) head_sum_kernel(const float* __restrict__ part, int q_blocks, int k_blocks, int dim,
                                                                 float* __restrict__ gq_weight, float* __restrict__ gk_weight) {
    __shared__ double rows[SUM_ROWS][33];
    pdl_wait_then_trigger();
    const int f = blockIdx.x * 32 + threadIdx.x, end = blockIdx.y ? q_blocks + k_blocks : q_blocks;
    double sum = 0.;
    if (f < dim)
        for (int b = (blockIdx.y ? q_blocks : 0) + threadIdx.y; b < end; b += 4 * SUM_ROWS) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = b + e * SUM_ROWS < end ? part[(int64_t)(b + e * SUM_ROWS) * dim + f] : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += v[e];
        }
    rows[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y != 0 || f >= dim) return;
#pragma unroll
    for (int j = 1; j < SUM_ROWS; ++j) sum += rows[j][threadIdx.x];
    float* to = blockIdx.y ? gk_weight : gq_weight;
    if (to != nullptr) to[f] = (float)sum;
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
    s.heads0 = (int)a->q_heads;
    s.heads1 = (int)a->k_heads;
    s.dim = (int)a->dim;
    s.pairs = a->pairs;
    s.interleaved = a->interleaved;
    s.norm = a->norm;
    s.eps = (float)a->eps;
    s.inv_dim = (float)(1. / a->dim);
    s.sign = sign;
    const int units = (int)ceil_div(a->dim, 2 * v);
    s.lanes = 1;
    while (s.lanes < units && s.lanes < 32) s.lanes *= 2;
    // whole waves of blocks with tiles as large as fit
    const int64_t most = s.pairs > MOST_ANGLES / MOST_TILE ? MOST_ANGLES / s.pairs : MOST_TILE, wave = 148 * FWD_BLOCKS, waves = ceil_div(s.nodes, wave * most);
    s.tile = (int)ceil_div(s.nodes, wave * (waves > 0 ? waves : 1));
    if (s.tile < 1) s.tile = 1;
    return s;
}

// Blocks of the gradients, divided between q and k by their heads.
void grad_blocks(const HeadShape& s, int& q, int& k) {
    const int64_t tiles = ceil_div(s.nodes, s.tile), heads = s.heads0 + s.heads1;
    const int64_t wanted = ceil_div(GRAD_BLOCKS * (int64_t)s.heads0, heads);
    q = s.heads0 == 0 ? 0 : (int)(wanted < tiles ? wanted : tiles);
    const int64_t left = s.heads0 == 0 ? GRAD_BLOCKS : GRAD_BLOCKS - wanted > 0 ? GRAD_BLOCKS - wanted : 1;
    k = s.heads1 == 0 ? 0 : (int)(left < tiles ? left : tiles);
}
cudaError_t sum_launch(const fpde_head_args* a, int q, int k, cudaStream_t st) {
    return launch_kernel(head_sum_kernel, dim3((unsigned)ceil_div(a->dim, 32), 2), dim3(32, SUM_ROWS), st, (const float*)a->workspace, q, k, (int)a->dim,
                         a->gq_weight, a->gk_weight);
}

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
        int qb, kb;
        grad_blocks(s, qb, kb);
        static std::atomic<uint64_t> done{0};
        const size_t ring = GRAD_STAGES * 8 * U * V * sizeof(T) * THREADS, shares = THREADS * U * 2 * V * sizeof(float), bytes = ring > shares ? ring : shares;
        cudaError_t e = allow_smem(head_bwd_kernel<T, V, U>, bytes, done);
        if (e != cudaSuccess) return e;
        e = launch_kernel_smem(head_bwd_kernel<T, V, U>, dim3(qb + kb), dim3(THREADS), bytes, c.st, c.q, c.k, c.gq, c.gk, c.a->q_weight, c.a->k_weight,
                               (T*)c.out_q, (T*)c.out_k, (float*)c.a->workspace, qb, s);
        return e != cudaSuccess ? e : sum_launch(c.a, qb, kb, c.st);
    }
    const int64_t blocks = ceil_div(s.nodes, s.tile);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    static std::atomic<uint64_t> done{0};
    const size_t bytes = STAGES * 4 * U * V * sizeof(T) * THREADS;
    const cudaError_t e = allow_smem(head_fwd_kernel<T, V, U>, bytes, done);
    if (e != cudaSuccess) return e;
    return launch_kernel_smem(head_fwd_kernel<T, V, U>, dim3((unsigned)blocks), dim3(THREADS), bytes, c.st, c.q, c.k, c.a->q_weight, c.a->k_weight,
                              (T*)c.out_q, (T*)c.out_k, s);
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
    return (size_t)(GRAD_BLOCKS + 1) * a->dim * sizeof(float);
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
        return sum_launch(a, 0, 0, (cudaStream_t)stream) == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
    if (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < fpde_head_rotary_workspace_bytes(a)) return FPDE_ERR_WORKSPACE;
    return head_run({a, view_q(a), view_k(a), view_gq(a), view_gk(a), a->gx_q, a->gx_k, -1.f, true, (cudaStream_t)stream});
}

}  // extern "C"
