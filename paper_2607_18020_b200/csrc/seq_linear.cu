// Linear attention with a decay for each head: forward, gradients and the single-node form.
//
//   S[t] = g S[t-1] + k[t] v[t]^T;  o[t] = scale q[t] S[t];  g = exp(log_decay)
//
// A march takes three arrays of a row and head, a (like q), b (like k) and c (like v), a chunk of nodes at a time.
// With S the state before the chunk, and i, j nodes of the chunk,
//   out_i = near sum_{j <= i} g^(i-j) (a_i . b_j) c_j + far g^(i+1-shift) a_i S
//   S <- g^n S + gain sum_j g^(n-1-j+shift) b_j c_j^T                        (n: nodes of the chunk)
// Everything is such a march:
//   o:  (q, k, v) from state, near = far = scale, gain = 1, shift = 0
//   gq: (go, v, k) from state^T, the same
//   gk: (v, go, q) from the last node to the first, from gstate^T, near = gain = scale, far = 1, shift = 1
//   gv: (k, q, go) likewise from gstate; its last state is the gradient of the first one
#include "seq_linear.cuh"

namespace fpde {
namespace {

constexpr int C = 32, THREADS = 128;

// The march of 32- and 16-bit arrays in 32 bits.  A block takes a row and head, or a piece, and up to 64 features of c, in
// chunks of 32 nodes: a, b and c in shared memory as fp32, the next chunk's on their way there (fp32 arrays: copied; 16-bit ones are
// widened when their turn comes), the state there too.  The four products run in packed arithmetic.  Registers filled from shared
// memory bind it, then instructions: 256 x 128 nodes of 4 heads of 32 in fp32, 44 us a march (with tiles of 2 x 4 for all products and
// without the skipped pairs 60; memory's floor is 10).  16 nodes a chunk would be fewer multiplications, but more barriers and half a tile
// for each thread.
template <typename T, int DA, int DC>
struct Sizes {
    static constexpr int PA = DA + 4, PC = DC + 4, PP = C + 4, STAGES = sizeof(T) == 4 && DA <= 64 ? 2 : 1;
    static constexpr int TILE = 2 * C * PA + C * PC;
    static constexpr size_t BYTES = sizeof(float) * (STAGES * TILE + DA * PC + C * PP);
};

// Rows of a chunk to shared memory, W features of pitch P, zeros where there is no node or feature.
template <typename T, int W, int P>
__device__ __forceinline__ void load_rows(float* to, const T* from, int64_t stride, int rows, int cols, bool packed) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t base = (uint32_t)__cvta_generic_to_shared(to);
        if (packed) {
#pragma unroll
            for (int i = threadIdx.x; i < C * W / 4; i += THREADS) {
                const int r = i / (W / 4), c = i % (W / 4) * 4, have = r < rows ? min(max(cols - c, 0), 4) : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + (r * P + c) * 4), "l"(have ? from + r * stride + c : from), "r"(4 * have)
                             : "memory");
            }
        } else {
            for (int i = threadIdx.x; i < C * W; i += THREADS) {
                const int r = i / W, c = i % W;
                const bool have = r < rows && c < cols;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(base + (r * P + c) * 4), "l"(have ? from + r * stride + c : from), "r"(have ? 4 : 0)
                             : "memory");
            }
        }
    } else {
        for (int i = threadIdx.x; i < C * W / 4; i += THREADS) {
            const int r = i / (W / 4), c = i % (W / 4) * 4;
            float v[4] = {};
            if (r < rows && packed && c + 4 <= cols) widen<T, 4>(v, load_pack<T, 4>(from + r * stride + c));
            else if (r < rows)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < cols) v[e] = to_f32<T>(from[r * stride + c + e]);
            *reinterpret_cast<float4*>(to + r * P + c) = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
}

// The sums of two lanes that took a half of the terms each: the lower one gets the first N / 2 rows, the upper one the others.
template <int N>
__device__ __forceinline__ void halves(uint64_t (&v)[N][2], int half) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint64_t mine = half ? v[N / 2 + i][e] : v[i][e], other = half ? v[i][e] : v[N / 2 + i][e];
            v[i][e] = add2(mine, __shfl_xor_sync(~0u, other, 16));
        }
}

__device__ __forceinline__ void lds_pairs(uint64_t (&p)[2], const float* from) {
    const float4 v = *reinterpret_cast<const float4*>(from);
    p[0] = pair(v.x, v.y);
    p[1] = pair(v.z, v.w);
}

// ENDS: only the state that a piece leaves, from zero.
template <typename T, int DA, int DC, bool ENDS>
__global__ void __launch_bounds__(THREADS, DA == 32 ? 5 : DA == 64 ? 3 : 2) march_kernel(March m, bool a_packed, bool b_packed, bool c_packed, bool out_packed) {
    using Z = Sizes<T, DA, DC>;
    extern __shared__ __align__(16) float smem[];
    float *ss = smem + Z::STAGES * Z::TILE, *sp = ss + DA * Z::PC;
    __shared__ float powers[C + 2];
    __shared__ float whole[4];                             // g^32 and that of the last chunk, each in two parts
    pdl_wait_then_trigger();
    const int tid = threadIdx.x;
    const int across = (m.dc + DC - 1) / DC, pieces = ENDS ? m.pieces - 1 : m.pieces;      // nobody starts from the last one's end
    unsigned id = blockIdx.x;
    const int c0 = (int)(id % across) * DC;
    id /= across;
    const int p = (int)(id % pieces);
    id /= pieces;
    const int64_t bt = id / (unsigned)m.heads, h = id - (unsigned)bt * (unsigned)m.heads;
    const int cols = min(DC, m.dc - c0);
    const int64_t first = p * m.piece, last = min(m.length, first + m.piece);
    const int chunks = (int)((last - first + C - 1) / C), tail = (int)(last - first) - (chunks - 1) * C;
    const int64_t dir = m.reversed ? -1 : 1, origin = m.reversed ? m.length - 1 - first : first;
    const T* a = (const T*)m.a.p + bt * m.a.batch + h * m.a.head + origin * m.a.node;
    const T* b = (const T*)m.b.p + bt * m.b.batch + h * m.b.head + origin * m.b.node;
    const T* cc = (const T*)m.c.p + bt * m.c.batch + h * m.c.head + origin * m.c.node + c0;
    auto load = [&](int c, int stage) {
        const int n = c < chunks - 1 ? C : tail;
        const int64_t at = dir * c * C;
        float* to = smem + stage * Z::TILE;
        if (!ENDS) load_rows<T, DA, Z::PA>(to, a + at * m.a.node, dir * m.a.node, n, m.da, a_packed);
        load_rows<T, DA, Z::PA>(to + C * Z::PA, b + at * m.b.node, dir * m.b.node, n, m.da, b_packed);
        load_rows<T, DC, Z::PC>(to + 2 * C * Z::PA, cc + at * m.c.node, dir * m.c.node, n, cols, c_packed);
        if constexpr (sizeof(T) == 4) asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (chunks > 0) load(0, 0);
    if (tid < C + 4) {
        const double g = power(m.log_decay[h], tid < C + 2 ? tid : tid == C + 2 ? C : max(tail, 0));
        if (tid < C + 2) {
            powers[tid] = (float)g;
        } else {
            whole[2 * (tid - C - 2)] = (float)g;
            whole[2 * (tid - C - 2) + 1] = (float)(g - (float)g);
        }
    }
    const int64_t st = (bt * m.heads + h) * m.da * m.dc;
    float* local = m.local + ((bt * m.heads + h) * m.pieces + p) * m.da * m.dc;
    const float* from = ENDS ? nullptr : m.pieces > 1 ? local : m.start != nullptr ? m.start + st : nullptr;
    const bool turned = m.pieces > 1 ? m.local_turned : m.start_turned;
    for (int i = tid; i < DA * DC; i += THREADS) {         // along the rows of what is read
        const int r = turned ? i % DA : i / DC, c = turned ? i / DA : i % DC;
        float v = 0.f;
        if (from != nullptr && r < m.da && c < cols) v = from[turned ? (c0 + c) * m.da + r : r * m.dc + c0 + c];
        ss[r * Z::PC + c] = v;
    }
    // A result is tiles of 4 x 4 to 16 x 4 a thread.  Where that leaves threads over, two lanes share a tile, each with half of the
    // terms: half the registers filled from shared memory, which is what binds this, for the tiles of 2 x 4 that would take all.
    constexpr int GC = DC / 4, HALVES = DC == 32 ? 2 : 1, GR = THREADS / GC / HALVES;
    constexpr int RO = C / GR, RS = DA / GR, MO = RO / HALVES, MS = RS / HALVES;
    static_assert(RO == 4 && THREADS == 128, "");
    const int half = HALVES == 2 ? tid >> 4 & 1 : 0, t = HALVES == 2 ? (tid & 15) | (tid >> 5) << 4 : tid;
    const int tc = t % GC * 4, tr = GR - 1 - t / GC;        // the warps with the most pairs of nodes to multiply have the fewest to sum
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const int n = c < chunks - 1 ? C : tail, stage = Z::STAGES == 2 ? c & 1 : 0;
        const float *sa = smem + stage * Z::TILE, *sb = sa + C * Z::PA, *sc = sb + C * Z::PA;
        if (Z::STAGES == 1 && c > 0) load(c, 0);
        if constexpr (sizeof(T) == 4) asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        if (Z::STAGES == 2 && c + 1 < chunks) load(c + 1, stage ^ 1);
        if (!ENDS) {
            // (a_i . b_j), 4 x 4 and half of the features a thread, with the decay between the nodes
            const int hd = tid >> 4 & 1, warp = tid / 32, td = (tid & 15) | warp << 4, j0 = td % 8, i0 = td / 8 * 4;
            uint64_t s[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = both(0.f);
            auto dots = [&](auto count) {
                constexpr int J = decltype(count)::value;
#pragma unroll 4
                for (int d = hd * (DA / 2); d < (hd + 1) * (DA / 2); d += 4) {
                    uint64_t x[4][2], y[J][2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) lds_pairs(x[i], sa + (i0 + i) * Z::PA + d);
#pragma unroll
                    for (int j = 0; j < J; ++j) lds_pairs(y[j], sb + (j0 + 8 * j) * Z::PA + d);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < J; ++j) s[i][j] = fma2(x[i][1], y[j][1], fma2(x[i][0], y[j][0], s[i][j]));
                }
            };
            if (warp < 2) dots(std::integral_constant<int, 2>());      // the rest lies behind all of the warp's nodes
            else dots(std::integral_constant<int, 4>());
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float lo = sum2(s[i][j]), hi = sum2(s[2 + i][j]);
                    const float sum = (hd ? hi : lo) + __shfl_xor_sync(~0u, hd ? lo : hi, 16);
                    const int row = i0 + 2 * hd + i, back = row - (j0 + 8 * j);
                    sp[row * Z::PP + j0 + 8 * j] = back < 0 ? 0.f : m.near * powers[max(back, 0)] * sum;
                }
            uint64_t o[RO][2];
#pragma unroll
            for (int i = 0; i < RO; ++i) o[i][0] = o[i][1] = both(0.f);
#pragma unroll 2
            for (int d = half * (DA / HALVES); d < (half + 1) * (DA / HALVES); d += 4) {
                uint64_t y[4][2];
#pragma unroll
                for (int e = 0; e < 4; ++e) lds_pairs(y[e], ss + (d + e) * Z::PC + tc);
#pragma unroll
                for (int i = 0; i < RO; ++i) {
                    const float4 x = *reinterpret_cast<const float4*>(sa + (tr * RO + i) * Z::PA + d);
                    const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[i][0] = fma2(both(xs[e]), y[e][0], o[i][0]);
                        o[i][1] = fma2(both(xs[e]), y[e][1], o[i][1]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RO; ++i) {
                const uint64_t w = both(m.far * powers[tr * RO + i + 1 - m.shift]);
                o[i][0] = mul2(o[i][0], w);
                o[i][1] = mul2(o[i][1], w);
            }
            __syncthreads();
            // rows behind a node are not looked at: they may hold anything
#pragma unroll 1
            for (int j = 4 * half; j < tr * RO; j += 4 * HALVES) {
                uint64_t y[4][2];
#pragma unroll
                for (int e = 0; e < 4; ++e) lds_pairs(y[e], sc + (j + e) * Z::PC + tc);
#pragma unroll
                for (int i = 0; i < RO; ++i) {
                    const float4 x = *reinterpret_cast<const float4*>(sp + (tr * RO + i) * Z::PP + j);
                    const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[i][0] = fma2(both(xs[e]), y[e][0], o[i][0]);
                        o[i][1] = fma2(both(xs[e]), y[e][1], o[i][1]);
                    }
                }
            }
#pragma unroll 1
            for (int j = tr * RO + half; j < (tr + 1) * RO; j += HALVES) {
                uint64_t y[2];
                lds_pairs(y, sc + j * Z::PC + tc);
#pragma unroll
                for (int i = 0; i < RO; ++i) {
                    if (j > tr * RO + i) continue;
                    const uint64_t x = both(sp[(tr * RO + i) * Z::PP + j]);
                    o[i][0] = fma2(x, y[0], o[i][0]);
                    o[i][1] = fma2(x, y[1], o[i][1]);
                }
            }
            if constexpr (HALVES == 2) halves(o, half);
            const int row = tr * RO + half * MO;
            T* out = (T*)m.out + ((bt * m.length + origin + dir * (c * C + row)) * m.heads + h) * m.dc + c0 + tc;
#pragma unroll
            for (int i = 0; i < MO; ++i, out += dir * m.heads * m.dc) {
                if (row + i >= n) continue;
                float v[4];
                unpair(o[i][0], v[0], v[1]);
                unpair(o[i][1], v[2], v[3]);
                if (out_packed && tc + 4 <= cols) store_pack<T, 4>(out, v);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (tc + e < cols) out[e] = from_f32<T>(v[e]);
            }
        }
        uint64_t u[RS][2];
#pragma unroll
        for (int i = 0; i < RS; ++i) u[i][0] = u[i][1] = both(0.f);
#pragma unroll 2
        for (int j = half; j < n; j += HALVES) {
            uint64_t y[2];
            const uint64_t w = both(m.gain * powers[n - 1 - j + m.shift]);
            lds_pairs(y, sc + j * Z::PC + tc);
            y[0] = mul2(y[0], w);
            y[1] = mul2(y[1], w);
            float x[RS];
#pragma unroll
            for (int i = 0; i < RS; i += 4) *reinterpret_cast<float4*>(x + i) = *reinterpret_cast<const float4*>(sb + j * Z::PA + tr * RS + i);
#pragma unroll
            for (int i = 0; i < RS; ++i) {
                u[i][0] = fma2(both(x[i]), y[0], u[i][0]);
                u[i][1] = fma2(both(x[i]), y[1], u[i][1]);
            }
        }
        if constexpr (HALVES == 2) halves(u, half);
        const uint64_t hi = both(whole[n == C ? 0 : 2]), lo = both(whole[n == C ? 1 : 3]);
        __syncthreads();                                   // everyone has read the state
#pragma unroll
        for (int i = 0; i < MS; ++i) {
            float* at = ss + (tr * RS + half * MS + i) * Z::PC + tc;
            uint64_t v[2];
            lds_pairs(v, at);
            float4 w;
            unpair(fma2(hi, v[0], fma2(lo, v[0], u[i][0])), w.x, w.y);
            unpair(fma2(hi, v[1], fma2(lo, v[1], u[i][1])), w.z, w.w);
            *reinterpret_cast<float4*>(at) = w;
        }
    }
    __syncthreads();
    float* to = ENDS ? local : p == m.pieces - 1 && m.end != nullptr ? m.end + st : nullptr;
    if (to == nullptr) return;
    for (int i = tid; i < DA * DC; i += THREADS) {
        const int r = i / DC, c = i % DC;
        if (r < m.da && c < cols) to[r * m.dc + c0 + c] = ss[r * Z::PC + c];
    }
}

// What each piece leaves becomes the state that each starts from; PIECES pieces at a time, so that their loads are on their way
// together: 4, or 8 where there are more (2 pieces of 64 rows and heads of 128 x 128: 7 and 14 us; 16 of 8, the whole call: 41 and 36).
constexpr int SQUARE = 16, JOINED = 4;         // features of a block either way, so that a turned state is read by whole sectors too; squares of a block
template <int PIECES>
__global__ void __launch_bounds__(SQUARE * SQUARE) join_kernel(March m) {
    __shared__ float parts[2];
    pdl_wait_then_trigger();
    const int across = (m.dc + SQUARE - 1) / SQUARE, squares = across * ((m.da + SQUARE * JOINED - 1) / (SQUARE * JOINED));
    const int64_t row = blockIdx.x / (unsigned)squares, size = (int64_t)m.da * m.dc;
    const int square = (int)(blockIdx.x - row * squares), d0 = square / across * (SQUARE * JOINED) + threadIdx.x / SQUARE,
              e = square % across * SQUARE + threadIdx.x % SQUARE;
    if (threadIdx.x == 0) {
        const double g = power(m.log_decay[row % m.heads], (double)m.piece);
        parts[0] = (float)g;
        parts[1] = (float)(g - (float)g);
    }
    float s[JOINED];
#pragma unroll
    for (int j = 0; j < JOINED; ++j) {
        const int d = d0 + j * SQUARE;
        s[j] = m.start != nullptr && d < m.da && e < m.dc ? m.start[row * size + (m.start_turned ? e * m.da + d : d * m.dc + e)] : 0.f;
    }
    __syncthreads();
    if (e >= m.dc) return;
    const float hi = parts[0], lo = parts[1];
    float* at = m.local + row * m.pieces * size + d0 * m.dc + e;
    for (int p = 0; p < m.pieces; p += PIECES, at += PIECES * size) {
        float u[PIECES][JOINED];
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int j = 0; j < JOINED; ++j) u[k][j] = p + k < m.pieces - 1 && d0 + j * SQUARE < m.da ? at[k * size + j * SQUARE * m.dc] : 0.f;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (p + k >= m.pieces) break;
#pragma unroll
            for (int j = 0; j < JOINED; ++j) {
                if (d0 + j * SQUARE < m.da) at[k * size + j * SQUARE * m.dc] = s[j];
                s[j] = fmaf(hi, s[j], fmaf(lo, s[j], u[k][j]));
            }
        }
    }
}

// One node of every row and head.  A block takes one head's state: LX lanes of V columns each, the rows over the
// rest of its threads, whose shares of the output are summed in shared memory.  Memory bounds it, the state's way there and back:
// 256 rows of 32 heads of 128 x 128, 200 us of 165.  The decay comes from 64 bits and in two parts, as in the march: rounded to 32 its error
// would be the same in every step, 3e-4 of a state after 12345 steps of a head that hardly forgets.
constexpr int STEP_THREADS = 256;
template <typename T, int V>
__global__ void __launch_bounds__(STEP_THREADS) linear_step_kernel(LinearView q, LinearView k, LinearView v, const float* __restrict__ log_decay,
                                                                   const float* state, float* state_out, T* __restrict__ o, int heads, int dk, int dv,
                                                                   int lx, float scale) {
    __shared__ float sq[FPDE_LINEAR_MAX_DIM], sk[FPDE_LINEAR_MAX_DIM], part[STEP_THREADS * V], decay[2];
    pdl_wait_then_trigger();
    const int64_t row = blockIdx.x, b = row / heads;
    const int h = (int)(row - b * heads), tid = threadIdx.x;
    if (tid < dk) {
        sq[tid] = to_f32<T>(((const T*)q.p)[b * q.batch + h * q.head + tid]) * scale;
        sk[tid] = to_f32<T>(((const T*)k.p)[b * k.batch + h * k.head + tid]);
    }
    if (tid == STEP_THREADS - 1) {                         // a thread without a feature
        const double g = power(log_decay[h], 1.);
        const float hi = (float)g;
        decay[0] = hi;
        decay[1] = hi - hi == 0.f ? (float)(g - hi) : 0.f;     // past the range of 32 bits there is no rest
    }
    const int x = tid % lx, y = tid / lx, rows = STEP_THREADS / lx, c = x * V;
    const bool in = c < dv;
    float val[V];
    if (in)
        for (int e = 0; e < V; ++e) val[e] = to_f32<T>(((const T*)v.p)[b * v.batch + h * v.head + c + e]);
    __syncthreads();
    const float hi = decay[0], lo = decay[1];
    float sum[V] = {};
    if (in) {
        const int64_t at = row * dk * dv + c;
#pragma unroll 8
        for (int d = y; d < dk; d += rows) {
            float s[V];
            if (state != nullptr) widen<float, V>(s, load_pack<float, V>(state + at + (int64_t)d * dv));
            else
                for (int e = 0; e < V; ++e) s[e] = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[e] = fmaf(hi, s[e], fmaf(lo, s[e], sk[d] * val[e]));
                sum[e] = fmaf(sq[d], s[e], sum[e]);
            }
            if (state_out != nullptr) store_pack<float, V>(state_out + at + (int64_t)d * dv, s);
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) part[(y * lx + x) * V + e] = sum[e];
    __syncthreads();
    if (tid < dv) {
        float s = 0.f;
        for (int j = 0; j < rows; ++j) s += part[j * lx * V + tid];
        o[row * dv + tid] = from_f32<T>(s);
    }
}

// ------------------------------------------------------------------------------------------- host
int check_linear_sizes(const fpde_linear_args* a, bool step = false) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->dk < 1 || a->dk > FPDE_LINEAR_MAX_DIM || a->dv < 1 || a->dv > FPDE_LINEAR_MAX_DIM) return FPDE_ERR_PARAM;
    if (a->batch < 0 || a->length < 0 || a->heads < 0 || a->heads > (1 << 24) || a->length > (1ll << 36) || a->batch > (1ll << 36) ||
        !product_fits(a->batch, step ? 1 : a->length, a->heads * (a->dk > a->dv ? a->dk : a->dv)) || !product_fits(a->batch, a->heads, a->dk * a->dv))
        return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

int check_linear(const fpde_linear_args* a, bool step) {
    const int st = check_linear_sizes(a, step);
    if (st != FPDE_OK) return st;
    if (!(a->scale - a->scale == 0.)) return FPDE_ERR_PARAM;
    if (a->batch * a->heads > 0) {
        if (a->log_decay == nullptr) return FPDE_ERR_NULL;
        if ((step || a->length > 0) && (a->q == nullptr || a->k == nullptr || a->v == nullptr)) return FPDE_ERR_NULL;
        const size_t e = dtype_bytes(a->dtype);
        const void* act[] = {a->q, a->k, a->v, a->o, a->go, a->gq, a->gk, a->gv};
        const void* par[] = {a->log_decay, a->state, a->state_out, a->gstate_out, a->gstate};
        for (const void* p : act)
            if (!aligned(p, e)) return FPDE_ERR_ALIGN;
        for (const void* p : par)
            if (!aligned(p, 4)) return FPDE_ERR_ALIGN;
    }
    return FPDE_OK;
}

// A chunk there takes as long however few of its 128 nodes and 64 or 128 features there are.  2048 rows and heads, 32-bit
// arithmetic and tensor cores: 32 features, 192 nodes 143 and 155 us, 256 nodes 186 and 158; 64 features, 40 nodes 139 and 138, 96 nodes 231
// and 144; 128 features, 24 nodes 400 and 261, 96 nodes 933 and 280.  fp16 arrays are widened to fp32: fp16 holds neither the products of
// queries and keys nor the states, and as bf16 factors its values would be two parts each, which the march is not written for.
bool on_tensor_cores(const fpde_linear_args* a, const March& m) {
    const int64_t widest = a->dk > a->dv ? a->dk : a->dv, enough = widest <= 32 ? 193 : widest <= 64 ? 40 : 24;
    if (a->dtype != FPDE_BF16 || a->length < enough) return false;
    for (const LinearView* x : {&m.a, &m.b, &m.c})
        if (!aligned(x->p, 16) || !tile_steps(*x, a->heads, a->length, a->batch)) return false;
    return true;
}

// Pieces of a row.  With more than one, all but the last are marched through twice, the first time for their ends alone, and the
// states are joined in between.  The number with the least time of waves of blocks is taken; the figures are measured
// microseconds of a chunk and of a block's start, and of two more launches and the join, which reads and writes a state for each piece.
// In 32 bits one figure stands for all widths: four blocks an SM, where 5, 3 or 2 are resident with up to 32, 64 and 128 features of a.
// `other`: a march that shares the pieces is on the tensor cores.  If only one of the two is, the one in 32 bits, which takes longer,
// decides, in whole chunks of the other.
void cut(March& m, bool gradient, bool other) {
    const bool mma = m.mma && other, wide = m.da > 64 || m.dc > 64;
    const int chunk = m.mma || other ? MMA_CHUNK : C;
    const double main = mma ? (wide ? 4.3 : 2.5) : 4.0 * (chunk / C), ends = mma ? (wide ? 2.2 : 1.2) : 2.0 * (chunk / C), start = mma ? 6. : 4.;
    const int64_t rows = m.batch * m.heads * (mma ? 1 : ceil_div(m.dc, 64)), slots = mma ? MMA_BLOCKS : 148 * 4, chunks = ceil_div(m.length, chunk);
    const double join = (double)m.batch * m.heads * m.da * m.dc * 8 / 5e6;
    const double first = gradient ? 2. / 3. : 1.;         // of three marches one uses another's states
    int64_t best = 1;
    double least = 1e300;
    for (int64_t p = 1, each; p <= chunks && p <= 1024 && rows * (p - 1) < 8 * slots; p = each > 1 ? ceil_div(chunks, each - 1) : chunks + 1) {
        each = ceil_div(chunks, p);
        // a chunk takes longer the more blocks read memory with it: 4.3 us of 128 x 128 features on 64 SMs, 5.5 on all
        const auto load = [&](int64_t blocks) { return 0.8 + 0.45 * (blocks < slots ? (double)blocks / slots : 1.); };
        double time = (double)ceil_div(rows * p, slots) * (start + each * main * load(rows * p));
        if (p > 1) time += first * ((double)ceil_div(rows * (p - 1), slots) * (start + each * ends * load(rows * (p - 1))) + 4.5 + p * join);
        if (time < least) {
            least = time;
            best = p;
        }
    }
    const int64_t each = chunks > 0 ? ceil_div(chunks, best) : 1;
    m.piece = each * chunk;
    m.pieces = (int)best;
}

size_t local_bytes(const March& m) { return m.pieces > 1 ? (size_t)m.batch * m.heads * m.pieces * m.da * m.dc * sizeof(float) : 0; }
// For the march, and for what it becomes if arrays turn out to start on no multiple of 16 bytes.
size_t most_bytes(const March& m, bool gradient, bool other) {
    size_t most = 0;
    for (const int mma : {0, 1})
        for (const int shared : {0, 1}) {
            if (mma > m.mma || shared > other) continue;
            March as = m;
            as.mma = mma;
            cut(as, gradient, shared);
            const size_t bytes = local_bytes(as);
            if (bytes > most) most = bytes;
        }
    return most;
}

March march_of(const fpde_linear_args* a) {
    March m = {};
    m.batch = a->batch;
    m.length = a->length;
    m.heads = a->heads;
    m.log_decay = a->log_decay;
    m.local = (float*)a->workspace;
    return m;
}
March march_o(const fpde_linear_args* a) {
    March m = march_of(a);
    m.a = {a->q, a->q_batch, a->q_node, a->q_head};
    m.b = {a->k, a->k_batch, a->k_node, a->k_head};
    m.c = {a->v, a->v_batch, a->v_node, a->v_head};
    m.da = (int)a->dk;
    m.dc = (int)a->dv;
    m.near = m.far = (float)a->scale;
    m.gain = 1.f;
    m.start = a->state;
    m.out = a->o;
    m.end = a->state_out;
    m.mma = on_tensor_cores(a, m);
    cut(m, false, m.mma);
    return m;
}
March march_gq(const fpde_linear_args* a) {
    March m = march_of(a);
    m.a = {a->go, a->go_batch, a->go_node, a->go_head};
    m.b = {a->v, a->v_batch, a->v_node, a->v_head};
    m.c = {a->k, a->k_batch, a->k_node, a->k_head};
    m.da = (int)a->dv;
    m.dc = (int)a->dk;
    m.near = m.far = (float)a->scale;
    m.gain = 1.f;
    m.start = a->state;
    m.start_turned = 1;
    m.out = a->gq;
    m.mma = on_tensor_cores(a, m);
    cut(m, true, m.mma);
    return m;
}
// Starts from the states that gv's march has joined, turned; its pieces are that one's.
March march_gk(const fpde_linear_args* a) {
    March m = march_of(a);
    m.a = {a->v, a->v_batch, a->v_node, a->v_head};
    m.b = {a->go, a->go_batch, a->go_node, a->go_head};
    m.c = {a->q, a->q_batch, a->q_node, a->q_head};
    m.da = (int)a->dv;
    m.dc = (int)a->dk;
    m.reversed = m.shift = 1;
    m.near = m.gain = (float)a->scale;
    m.far = 1.f;
    m.start = a->gstate_out;
    m.start_turned = m.local_turned = 1;
    m.out = a->gk;
    m.local_there = true;
    m.mma = on_tensor_cores(a, m);
    return m;
}
March march_gv(const fpde_linear_args* a, const March& gk) {
    March m = march_of(a);
    m.a = {a->k, a->k_batch, a->k_node, a->k_head};
    m.b = {a->q, a->q_batch, a->q_node, a->q_head};
    m.c = {a->go, a->go_batch, a->go_node, a->go_head};
    m.da = (int)a->dk;
    m.dc = (int)a->dv;
    m.reversed = m.shift = 1;
    m.near = m.gain = (float)a->scale;
    m.far = 1.f;
    m.start = a->gstate_out;
    m.out = a->gv;
    m.end = a->gstate;
    m.mma = on_tensor_cores(a, m);
    cut(m, true, gk.mma);
    return m;
}

#define FPDE_TRY(x)                           \
    do {                                      \
        const cudaError_t e_ = (x);           \
        if (e_ != cudaSuccess) return e_;     \
    } while (0)

template <typename T, int DA, int DC>
cudaError_t march_launch(const March& m, cudaStream_t st) {
    const size_t bytes = Sizes<T, DA, DC>::BYTES;
    const bool pa = packs(m.a.p, m.a.batch, m.a.node, sizeof(T), 4) && m.a.head % 4 == 0, pb = packs(m.b.p, m.b.batch, m.b.node, sizeof(T), 4) && m.b.head % 4 == 0,
               pc = packs(m.c.p, m.c.batch, m.c.node, sizeof(T), 4) && m.c.head % 4 == 0, po = m.dc % 4 == 0 && aligned(m.out, 4 * sizeof(T));
    const int64_t rows = m.batch * m.heads * ceil_div(m.dc, DC), blocks = rows * m.pieces;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    if (m.pieces > 1 && !m.local_there) {
        static std::atomic<uint64_t> done{0};
        FPDE_TRY(allow_smem(march_kernel<T, DA, DC, true>, bytes, done));
        FPDE_TRY(launch_kernel_smem(march_kernel<T, DA, DC, true>, dim3((unsigned)(rows * (m.pieces - 1))), dim3(THREADS), bytes, st, m, pa, pb, pc, po));
        FPDE_TRY(march_join(m, st));
    }
    static std::atomic<uint64_t> done{0};
    FPDE_TRY(allow_smem(march_kernel<T, DA, DC, false>, bytes, done));
    return launch_kernel_smem(march_kernel<T, DA, DC, false>, dim3((unsigned)blocks), dim3(THREADS), bytes, st, m, pa, pb, pc, po);
}

template <typename T>
cudaError_t march_run(const March& m, cudaStream_t st) {
    if (m.dc <= 32) return m.da <= 32 ? march_launch<T, 32, 32>(m, st) : m.da <= 64 ? march_launch<T, 64, 32>(m, st) : march_launch<T, 128, 32>(m, st);
    return m.da <= 32 ? march_launch<T, 32, 64>(m, st) : m.da <= 64 ? march_launch<T, 64, 64>(m, st) : march_launch<T, 128, 64>(m, st);
}

cudaError_t march_by_type(const fpde_linear_args* a, const March& m, cudaStream_t st) {
    cudaError_t e;
    if (m.mma && march_mma(m, st, &e)) return e;
    if (a->dtype == FPDE_F32) return march_run<float>(m, st);
    if (a->dtype == FPDE_BF16) return march_run<__nv_bfloat16>(m, st);
    return march_run<__half>(m, st);
}

template <typename T, int V>
cudaError_t step_launch(const fpde_linear_args* a, cudaStream_t st) {
    const int64_t rows = a->batch * a->heads;
    if (rows > 0x7fffffff) return cudaErrorInvalidConfiguration;
    int lx = 1;
    while (lx * V < a->dv) lx *= 2;
    return launch_kernel(linear_step_kernel<T, V>, dim3((unsigned)rows), dim3(STEP_THREADS), st, LinearView{a->q, a->q_batch, 0, a->q_head},
                         LinearView{a->k, a->k_batch, 0, a->k_head}, LinearView{a->v, a->v_batch, 0, a->v_head}, a->log_decay, a->state, a->state_out,
                         (T*)a->o, (int)a->heads, (int)a->dk, (int)a->dv, lx, (float)a->scale);
}
template <typename T>
cudaError_t step_run(const fpde_linear_args* a, cudaStream_t st) {
    return a->dv % 4 == 0 && aligned(a->state, 16) && aligned(a->state_out, 16) ? step_launch<T, 4>(a, st) : step_launch<T, 1>(a, st);
}

int as_status(cudaError_t e) { return e == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA; }

}  // namespace

cudaError_t march_join(const March& m, cudaStream_t st) {
    const int64_t blocks = m.batch * m.heads * ceil_div(m.da, SQUARE * JOINED) * ceil_div(m.dc, SQUARE);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(m.pieces > 4 ? join_kernel<8> : join_kernel<4>, dim3((unsigned)blocks), dim3(SQUARE * SQUARE), st, m);
}

}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_linear_attention_workspace_bytes(const fpde_linear_args* a, int backward) {
    if (check_linear_sizes(a) != FPDE_OK) return 0;
    fpde_linear_args b = *a;
    b.q = b.k = b.v = b.go = nullptr;              // the size is the same wherever the arrays start
    if (!backward) {
        const March m = march_o(&b);
        return most_bytes(m, false, m.mma);
    }
    const March gq = march_gq(&b), gk = march_gk(&b);
    const size_t q = most_bytes(gq, true, gq.mma), v = most_bytes(march_gv(&b, gk), true, gk.mma);
    return q > v ? q : v;
}

static int check_workspace(const fpde_linear_args* a, int backward) {
    const size_t need = fpde_linear_attention_workspace_bytes(a, backward);
    return need > 0 && (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < need) ? FPDE_ERR_WORKSPACE : FPDE_OK;
}

static int forward(const fpde_linear_args* a, int lose, void* stream) {
    int st = check_linear(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->heads == 0) return FPDE_OK;
    if (a->o == nullptr && a->length > 0) return FPDE_ERR_NULL;
    if (a->state != nullptr && a->state == a->state_out) return FPDE_ERR_PARAM;      // blocks still read it
    if ((st = check_workspace(a, 0)) != FPDE_OK) return st;
    March m = march_o(a);
    m.lose = lose;
    return as_status(march_by_type(a, m, (cudaStream_t)stream));
}

int fpde_linear_attention_fwd(const fpde_linear_args* a, void* stream) { return forward(a, 0, stream); }

int fpde_linear_attention_bwd(const fpde_linear_args* a, void* stream) {
    int st = check_linear(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->heads == 0) return FPDE_OK;
    if (a->length > 0 && (a->go == nullptr || a->gq == nullptr || a->gk == nullptr || a->gv == nullptr)) return FPDE_ERR_NULL;
    if (a->gstate != nullptr && a->gstate == a->gstate_out) return FPDE_ERR_PARAM;
    if ((st = check_workspace(a, 1)) != FPDE_OK) return st;
    const cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = march_by_type(a, march_gq(a), s);
    March gk = march_gk(a);
    const March gv = march_gv(a, gk);
    gk.pieces = gv.pieces;
    gk.piece = gv.piece;
    if (e == cudaSuccess) e = march_by_type(a, gv, s);
    if (e == cudaSuccess) e = march_by_type(a, gk, s);
    return as_status(e);
}

int fpde_linear_attention_step(const fpde_linear_args* a, void* stream) {
    const int st = check_linear(a, true);
    if (st != FPDE_OK) return st;
    if (a->batch * a->heads == 0) return FPDE_OK;
    if (a->o == nullptr) return FPDE_ERR_NULL;
    const cudaStream_t s = (cudaStream_t)stream;
    if (a->dtype == FPDE_F32) return as_status(step_run<float>(a, s));
    if (a->dtype == FPDE_BF16) return as_status(step_run<__nv_bfloat16>(a, s));
    return as_status(step_run<__half>(a, s));
}

int fpde_diag_linear_lost(const fpde_linear_args* a, int ends, void* stream) { return forward(a, ends ? 2 : 1, stream); }

unsigned int fpde_diag_linear_timeouts(void) { return march_mma_timeouts(); }

int fpde_diag_linear_form(const fpde_linear_args* a, int march) {
    if (check_linear_sizes(a) != FPDE_OK || march < 0 || march > 2) return 0;
    // an array without strides stands for dense rows of whole 16 bytes
    fpde_linear_args b = *a;
    b.q = b.k = b.v = b.go = nullptr;
    const auto rows = [&](int64_t& batch, int64_t& node, int64_t& head, int64_t width) {
        if (batch != 0 || node != 0 || head != 0) return;
        head = ceil_div(width, 8) * 8;
        node = head * b.heads;
        batch = node * b.length;
    };
    rows(b.q_batch, b.q_node, b.q_head, b.dk);
    rows(b.k_batch, b.k_node, b.k_head, b.dk);
    rows(b.v_batch, b.v_node, b.v_head, b.dv);
    rows(b.go_batch, b.go_node, b.go_head, b.dv);
    const March gk = march_gk(&b), m = march == 0 ? march_o(&b) : march == 1 ? march_gq(&b) : march_gv(&b, gk);
    return m.mma && (march < 2 || gk.mma) ? -m.pieces : m.pieces;
}

}  // extern "C"
