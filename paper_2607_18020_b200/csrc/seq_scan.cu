// Selective state space scan along the rows of (batch, length, channels) arrays: forward, gradients
// and the single-node form.
//
//   dt = softplus(delta + bias);  h[t] = exp(dt A) h[t-1] + dt u B;  y = C.h + D u;  out = y silu(z)
//
// Each (node, channel, state) costs one exponential and four multiplications or fused adds, against
// 16 bytes or less per (node, channel): with 16 states the special function unit (16 exponentials a
// clock and SM) bounds the forward pass, not memory.  8 x 2048 x 4096 x 16 bf16: 239 us of exponentials,
// 83 us of bytes, measured 531 us with that unit busy 55 to 63 % of the time; the rest is the latency of a
// march of dependent nodes at 14 warps an SM.
//
// Layout.  A thread keeps four states of one or two channels, as pairs for the packed fp32 instructions;
// S = 2, 4, 8 or 16 neighbouring lanes share their channels and the sums over states are shuffles among
// them.  Two channels a thread read B and C half as often (with one, shared memory's data pipe was 86 %
// busy) and halve the shuffles that sum gB and gC; one channel a thread gives small grids more warps.  A
// block marches through tiles of nodes: the tile's dt, dt u, B and C are brought to shared memory once, in
// fp32, by loads that run along the channels and travel one tile ahead.
//
// Long rows.  Where batch x channels gives too few blocks, a row is cut into chunks: one pass forms
// each chunk's state from zero and its sum of dt (the chunk's decay is exp(A sum dt)), a second kernel joins
// them along the row, and the march starts every chunk from its joined state.  The gradient does the
// same backwards with the adjoint state.  1 x 16384 x 1536 x 16 bf16: 309 us (one block per SM or fewer
// without chunks: 1442 us).
//
// Gradients.  With gy = gout silu(z) the adjoint state is p[t] = C gy + exp(dt[t+1] A) p[t+1]; then
//   gC = sum_c h gy, gB = sum_c p dt u, gu = dt (p.B) + D gy, gdt = sum_n p exp(dt A) h[t-1] A + u (p.B),
//   gA = sum_t p exp(dt A) h[t-1] dt.
// The forward pass stores the state before every KEEP-th node; the backward march recomputes the
// states inside such a piece in registers and walks it backwards.  It is bound by instructions: about 105
// per warp, node and four states, a fifth of them the sums over lanes; 4 x 4096 x 2048 x 16 bf16: 825 us,
// and 216 us for the chunks' ends.
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int STEP_THREADS = 128, STEP_CHANNELS = 4;      // one node: 28 us for 256 x 4096 x 16 bf16, 134 MB of states
constexpr int FWD_LANES = 32, BACK_LANES = 64;     // channels of a block with 4 lanes a channel: threads = that x 4 / NC
constexpr int FWD_UNROLL = 4;
constexpr double FWD_ENDS = 0.5, BACK_ENDS = 0.3;      // what forming the chunks' ends costs, as a share of the march
constexpr int TILE = 16;          // nodes brought to shared memory together
constexpr int KEEP = 8;           // nodes between stored states: what the backward march holds in registers
constexpr int NS = 4;             // states of a thread; it has NC = 1 or 2 channels
// resident blocks that the registers are budgeted for
__host__ __device__ constexpr int fwd_blocks(int nc) { return nc == 2 ? 7 : 5; }
__host__ __device__ constexpr int back_blocks(int nc) { return nc == 2 ? 3 : 2; }
__host__ __device__ constexpr int fwd_threads(int nc) { return FWD_LANES * 4 / nc; }
__host__ __device__ constexpr int back_threads(int nc) { return BACK_LANES * 4 / nc; }

struct ScanShape {
    int64_t length;
    int64_t u_batch, u_node, delta_batch, delta_node, z_batch, z_node, B_batch, B_node, C_batch, C_node, g_batch, g_node;
    int channels, states, softplus;
    int tiles;                    // blocks along the channels
    int chunks;                   // pieces of a row
    int chunk;                    // nodes of a piece (a multiple of TILE)
    int64_t kept_nodes;           // stored states of a row
};

template <typename T>
struct ScanIn {
    const T *u, *delta, *z, *B, *C, *gout;
    const float *A, *D, *bias;
};

struct Where {
    int tile, chunk;
    int64_t b;
};
__device__ __forceinline__ Where where(const ScanShape& s) {
    int64_t k = blockIdx.x;
    Where w;
    w.tile = (int)(k % s.tiles);
    k /= s.tiles;
    w.chunk = (int)(k % s.chunks);
    w.b = k / s.chunks;
    return w;
}

__device__ __forceinline__ float step_of(float raw, int softplus) { return softplus ? softplus_f32(raw) : raw; }

// A thread's own share of the tiles of ARRAYS activations: pack column `col` of rows r0, r0 + RP, ...  The
// next tile travels while this one is computed, by cp.async into shared memory that only this thread reads
// (no registers held, no barrier); 2-byte packs, which cp.async does not have, wait in registers.
template <typename T, int VEC, int NODES, int RP, int ARRAYS, int THREADS>
struct Feed {
    static constexpr int PER = (NODES + RP - 1) / RP, BYTES = sizeof(T) * VEC;
    static constexpr bool ASYNC = BYTES >= 4;
    using P = Pack<T, VEC>;
    struct Space { P v[ASYNC ? 2 : 1][ARRAYS][PER][THREADS]; };
    Space& space;
    const T* p[ARRAYS];                           // of row r0 of the tile to request next
    int now = 0;                                  // half that holds the current tile
    int r0;
    bool column;                                  // the thread's channels exist (zeros where not)
    P held[ASYNC ? 1 : ARRAYS][PER];
    __device__ __forceinline__ Feed(Space& where_, int r0_, bool column_) : space(where_), r0(r0_), column(column_) {
#pragma unroll
        for (int h = 0; h < (ASYNC ? 2 : 1); ++h)
#pragma unroll
            for (int a = 0; a < ARRAYS; ++a)
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    if (!column) space.v[h][a][k][threadIdx.x] = P{};
                    if (!ASYNC) held[a][k] = P{};
                }
    }
    __device__ __forceinline__ void start(int array, const T* row0, int64_t node, int col) { p[array] = row0 + r0 * node + col; }
    __device__ __forceinline__ void one(int array, int k, const T* src) {
        if (ASYNC)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(&space.v[now ^ 1][array][k][threadIdx.x]))),
                         "l"(src), "n"(BYTES < 4 ? 4 : BYTES) : "memory");
        else held[array][k] = load_pack<T, VEC>(src);
    }
    // Asks for the tile at p, of which `here` rows exist, and moves on by `advance` nodes.  Rows that do not
    // exist keep what an earlier tile left: they are masked where they are used.
    __device__ __forceinline__ void request(int array, int64_t node, int here, int advance) {
        const T* src = p[array];
        if (column) {
            if (here >= NODES && NODES % RP == 0) {
#pragma unroll
                for (int k = 0; k < PER; ++k) one(array, k, src + (int64_t)(k * RP) * node);
            } else {
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (r0 + k * RP < here) one(array, k, src + (int64_t)(k * RP) * node);
            }
        }
        p[array] = src + advance * node;
    }
    __device__ __forceinline__ void arrive() {    // what was requested becomes the current tile
        if (ASYNC) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            now ^= 1;
        } else {
#pragma unroll
            for (int a = 0; a < ARRAYS; ++a)
#pragma unroll
                for (int k = 0; k < PER; ++k) space.v[0][a][k][threadIdx.x] = held[a][k];
        }
    }
    __device__ __forceinline__ void get(float (&out)[VEC], int array, int k) const {
        widen<T, VEC>(out, space.v[ASYNC ? now : 0][array][k][threadIdx.x]);
    }
};

// The same for B and C, one state each of rows rn, rn + RN, ...: few, kept in registers.
template <typename T, int NODES, int RN>
struct States {
    static constexpr int PER = (NODES + RN - 1) / RN;
    T v[PER];
    const T* p;
    __device__ __forceinline__ void load(int64_t node, int rn, int here, bool there, int advance) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            v[k] = from_f32<T>(0.f);
            if (there && rn + k * RN < here) v[k] = p[(int64_t)(k * RN) * node];
        }
        p += advance * node;
    }
};

// Sums of N values over the lanes that differ in the bits HI .. LO of the lane number: while a lane holds
// more than one value it gives half of them away and takes its partner's share of the others.  Afterwards
// v[0 .. left) are the sums of values from .. from + left - 1 (`from` is returned).
template <int N, int HI, int LO>
__host__ __device__ constexpr int sums_left() {
    int left = N;
    for (int m = HI; m >= LO; m /= 2) left = left > 1 ? left / 2 : 1;
    return left;
}
template <int N, int HI, int LO>
__device__ __forceinline__ int sum_lanes(float (&v)[N], int lane) {
    int from = 0;
#pragma unroll
    for (int m = HI, left = N; m >= LO; m /= 2) {
        if (left > 1) {
            left /= 2;
            const bool up = lane & m;
#pragma unroll
            for (int i = 0; i < left; ++i) {
                const float send = up ? v[i] : v[left + i];
                v[i] = (up ? v[left + i] : v[i]) + __shfl_xor_sync(~0u, send, m);
            }
            from += up ? left : 0;
        } else {
            v[0] += __shfl_xor_sync(~0u, v[0], m);
        }
    }
    return from;
}

// Sums over the states of four nodes k0 .. k0+3 of the thread's channels (value NC * node + channel) to
// dst[node][channel].
template <int S, int NC, int CT>
__device__ __forceinline__ void put_sums(float (*dst)[CT], float (&v)[4 * NC], int k0, int c, int q) {
    const int from = sum_lanes<4 * NC, S / 2, 1>(v, q);
    constexpr int LEFT = sums_left<4 * NC, S / 2, 1>(), SHARE = S > 4 * NC ? S / (4 * NC) : 1;      // lanes with the same sum
    float* at = &dst[k0 + from / NC][c];
    if constexpr (LEFT >= NC && NC == 2) {
#pragma unroll
        for (int i = 0; i < LEFT / 2; ++i) *reinterpret_cast<float2*>(at + i * CT) = make_float2(v[2 * i], v[2 * i + 1]);
    } else if (SHARE == 1 || q % SHARE == 0) {
#pragma unroll
        for (int i = 0; i < LEFT; ++i) at[i * CT + from % NC] = v[i];
    }
}

__device__ __forceinline__ uint64_t exp2_pair(uint64_t v) {
    float a, b;
    unpair(v, a, b);
    return pair(exp2_f32(a), exp2_f32(b));
}

struct alignas(16) Quad {            // four floats as two pairs
    uint64_t lo, hi;
};
__device__ __forceinline__ Quad quad_at(const float* p) { return *reinterpret_cast<const Quad*>(p); }
__device__ __forceinline__ Quad quad_of(const float (&v)[NS]) { return {pair(v[0], v[1]), pair(v[2], v[3])}; }
__device__ __forceinline__ void quad_to(float (&v)[NS], const Quad& q) { unpair(q.lo, v[0], v[1]); unpair(q.hi, v[2], v[3]); }

// v[i], v[i] side by side for each channel of the thread.
template <int N>
__device__ __forceinline__ void put_twice(float2* at, const float (&v)[N]) {
    if constexpr (N == 2) *reinterpret_cast<float4*>(at) = make_float4(v[0], v[0], v[1], v[1]);
    else *at = make_float2(v[0], v[0]);
}

// The pairs of the thread's channels.
__device__ __forceinline__ void get_channels(uint64_t (&v)[2], const float2* at) {
    const Quad q = quad_at(&at->x);
    v[0] = q.lo;
    v[1] = q.hi;
}
__device__ __forceinline__ void get_channels(uint64_t (&v)[1], const float2* at) { v[0] = *reinterpret_cast<const uint64_t*>(at); }

// Four states from memory, or what stands in for those that do not exist.
__device__ __forceinline__ Quad load_states(const float* p, int n, int states, float scale) {
    float v[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) v[i] = p != nullptr && n + i < states ? p[n + i] * scale : 0.f;
    return quad_of(v);
}
__device__ __forceinline__ bool states_packed(int states) { return states % NS == 0; }
__device__ __forceinline__ void store_states(float* p, int n, int states, bool packed, const Quad& q) {
    if (packed) {     // rows of states start on 16 bytes
        if (n < states) *reinterpret_cast<Quad*>(p + n) = q;
        return;
    }
    float v[NS];
    quad_to(v, q);
#pragma unroll
    for (int i = 0; i < NS; ++i)
        if (n + i < states) p[n + i] = v[i];
}

// States that do not exist have zero A, B and C and stay zero while everything is finite; an infinite dt, dt u or gy
// makes NaN of them (0 times infinity), which the sums over states must not see.  Lanes that hold no state at all
// read dt, dt u and gy from a column of zeros behind the channels: full lanes (8, 16, 32, 64 states) lose nothing, others
// an access to shared memory (8 x 1024 x 2048 x 12 fp32 236 -> 247 us, 4 x 2048 x 2048 x 4 bf16 training 805 -> 827).  Where
// a lane's four states exist in part (PARTIAL: the number of states is no multiple of four), the others are cleared at
// every node (4 x 2048 x 1024 x 5 bf16 training 442 -> 456).  Looking for infinities first, and clearing only in the
// tiles that have them, took a second loop in the kernel and made the first one 3 to 12 % slower for every size.
constexpr int ZEROS = 2;          // columns
__device__ __forceinline__ Quad existing(const Quad& q, int n, int states) {
    float v[NS];
    quad_to(v, q);
#pragma unroll
    for (int i = 0; i < NS; ++i) v[i] = n + i < states ? v[i] : 0.f;
    return quad_of(v);
}

// ------------------------------------------------------------------------------------------ forward
template <typename T, int S, int NC, int VEC, bool ENDS>
struct FwdSpace {
    static constexpr int THREADS = fwd_threads(NC), CT = THREADS / S * NC, NP = S * NS;
    static constexpr int RP = THREADS / (CT / VEC), RN = THREADS / NP;      // rows at a time
    using Act = Feed<T, VEC, TILE, RP, ENDS ? 2 : 3, THREADS>;
    __align__(16) float2 sdt[TILE][CT + ZEROS], sdu[TILE][CT + ZEROS];      // dt, dt;  dt u, dt u: pairs as the arithmetic wants them
    __align__(16) float sb[TILE][NP], sc[ENDS ? 1 : TILE][NP];
    __align__(8) float sy[ENDS ? 1 : TILE][CT];
    typename Act::Space room;
};

// ENDS = false: the march.  ENDS = true, for rows cut into chunks: only what the join needs,
// local[b][chunk][channel][state] = state at the chunk's end when it starts from zero and
// sums[b][chunk][channel] = sum of dt.
template <typename T, int S, int NC, int VEC, bool ENDS, bool PARTIAL>
__global__ void __launch_bounds__(fwd_threads(NC), fwd_blocks(NC)) scan_fwd_kernel(ScanIn<T> in, const float* __restrict__ state, const float* __restrict__ enter,
                                                           T* __restrict__ out, float* __restrict__ state_out, float* __restrict__ kept,
                                                           float* __restrict__ local, float* __restrict__ sums, ScanShape s) {
    pdl_wait_then_trigger();
    using Space = FwdSpace<T, S, NC, VEC, ENDS>;
    using Act = typename Space::Act;
    constexpr int CT = Space::CT, NP = Space::NP, CP = CT / VEC, RP = Space::RP, RN = Space::RN;
    enum { U, DELTA, Z };
    using Bc = States<T, TILE, RN>;
    extern __shared__ __align__(16) uint8_t raw_space[];
    Space& m = *reinterpret_cast<Space*>(raw_space);
    const Where w = where(s);
    const int tid = threadIdx.x, q = tid % S, cl = tid / S * NC;
    const int c0 = w.tile * CT, c = c0 + cl, from = ENDS || q * NS < s.states ? cl : CT;      // where it reads dt and dt u
    const int64_t first = (int64_t)w.chunk * s.chunk;
    const int64_t end = first + s.chunk < s.length ? first + s.chunk : s.length;
    const int64_t per = (int64_t)s.channels * s.states;
    const int64_t at = w.b * s.chunks + w.chunk;
    Quad a2[NC], h[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int64_t cn = (int64_t)(c + k) * s.states;
        const bool mine = c + k < s.channels;
        a2[k] = load_states(mine ? in.A + cn : nullptr, q * NS, s.states, LOG2_E);
        h[k] = load_states(ENDS || !mine ? nullptr : enter ? enter + at * per + cn : state ? state + w.b * per + cn : nullptr, q * NS, s.states, 1.f);
    }
    // what this thread brings in: pack column `col` of rows r0, r0 + RP, ... and state n of rows rn, rn + RN, ...
    const int col = tid % CP * VEC, r0 = tid / CP, n = tid % NP, rn = tid / NP;
    const bool column = c0 + col < s.channels, row_n = n < s.states;
    float bias[VEC], dd[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        bias[i] = in.bias && column ? in.bias[c0 + col + i] : 0.f;
        dd[i] = in.D && column ? in.D[c0 + col + i] : 0.f;
    }
    Act act(m.room, r0, column);
    Bc bt, ct;
    act.start(U, in.u + w.b * s.u_batch + first * s.u_node + c0, s.u_node, col);
    act.start(DELTA, in.delta + w.b * s.delta_batch + first * s.delta_node + c0, s.delta_node, col);
    if constexpr (!ENDS) act.start(Z, in.z + w.b * s.z_batch + first * s.z_node + c0, s.z_node, col);
    bt.p = in.B + w.b * s.B_batch + (first + rn) * s.B_node + n;
    ct.p = in.C + w.b * s.C_batch + (first + rn) * s.C_node + n;
    auto fetch = [&](int here) {
        act.request(U, s.u_node, here, TILE);
        act.request(DELTA, s.delta_node, here, TILE);
        bt.load(s.B_node, rn, here, row_n, TILE);
        if constexpr (!ENDS) {
            if (in.z) act.request(Z, s.z_node, here, TILE);
            ct.load(s.C_node, rn, here, row_n, TILE);
        }
    };
    if (!ENDS && tid < TILE * ZEROS) m.sdt[tid / ZEROS][CT + tid % ZEROS] = m.sdu[tid / ZEROS][CT + tid % ZEROS] = make_float2(0.f, 0.f);
    float total[NC] = {};
    int left = (int)(end - first);               // nodes of the chunk from this tile on
    fetch(left);
    for (int64_t t0 = first; left > 0; t0 += TILE, left -= TILE) {
        act.arrive();
#pragma unroll
        for (int k = 0; k < Act::PER; ++k) {
            const int r = r0 + k * RP;
            if (TILE % RP != 0 && r >= TILE) break;
            float dt[VEC], u[VEC];
            act.get(u, U, k);
            act.get(dt, DELTA, k);
#pragma unroll
            for (int i = 0; i < VEC; ++i) dt[i] += bias[i];
            if (s.softplus) softplus_of<VEC>(dt);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                u[i] *= dt[i];
                if (left < TILE && r >= left) dt[i] = u[i] = 0.f;      // past the end: the state stays
            }
            put_twice<VEC>(&m.sdt[r][col], dt);
            put_twice<VEC>(&m.sdu[r][col], u);
        }
#pragma unroll
        for (int k = 0; k < Bc::PER; ++k) {
            if (TILE % RN != 0 && rn + k * RN >= TILE) break;
            m.sb[rn + k * RN][n] = to_f32<T>(bt.v[k]);
            if constexpr (!ENDS) m.sc[rn + k * RN][n] = to_f32<T>(ct.v[k]);
        }
        __syncthreads();
        if (left > TILE) fetch(left - TILE);
        const int here = left < TILE ? left : TILE;
#pragma unroll FWD_UNROLL
        for (int k0 = 0; k0 < TILE; k0 += 4) {
            if (!ENDS && kept != nullptr && k0 % KEEP == 0 && k0 < here) {
                float* dst = kept + ((w.b * s.kept_nodes + (t0 + k0) / KEEP) * s.channels + c) * s.states;
#pragma unroll
                for (int k = 0; k < NC; ++k)
                    if (c + k < s.channels) store_states(dst + k * s.states, q * NS, s.states, states_packed(s.states), h[k]);
            }
            float y[4 * NC];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const Quad b4 = quad_at(&m.sb[k0 + r][q * NS]);
                Quad c4;
                if constexpr (!ENDS) c4 = quad_at(&m.sc[k0 + r][q * NS]);
                uint64_t dt2[NC], du2[NC];
                get_channels(dt2, &m.sdt[k0 + r][from]);
                get_channels(du2, &m.sdu[k0 + r][from]);
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    h[k].lo = fma2(exp2_pair(mul2(dt2[k], a2[k].lo)), h[k].lo, mul2(du2[k], b4.lo));
                    h[k].hi = fma2(exp2_pair(mul2(dt2[k], a2[k].hi)), h[k].hi, mul2(du2[k], b4.hi));
                    if constexpr (PARTIAL) h[k] = existing(h[k], q * NS, s.states);
                    if constexpr (ENDS) {
                        float dt, same;
                        unpair(dt2[k], dt, same);
                        total[k] += dt;
                    } else {
                        y[NC * r + k] = sum2(fma2(c4.lo, h[k].lo, mul2(c4.hi, h[k].hi)));
                    }
                }
            }
            if constexpr (!ENDS) put_sums<S, NC, CT>(m.sy, y, k0, cl, q);
        }
        __syncthreads();
        if constexpr (!ENDS) {
            T* op = out + (w.b * s.length + t0 + r0) * s.channels + c0 + col;
#pragma unroll
            for (int k = 0; k < Act::PER; ++k) {
                const int r = r0 + k * RP;
                if (r >= here || !column) continue;
                // the fetch of the next tile went to the other half (2-byte packs: it is still in registers)
                float y[VEC], u[VEC], z[VEC], g[VEC];
                act.get(u, U, k);
                if (in.z) {
                    act.get(z, Z, k);
                    sigmoid_of<VEC>(g, z);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    y[i] = m.sy[r][col + i];
                    if (in.D) y[i] = fmaf(dd[i], u[i], y[i]);
                    if (in.z) y[i] *= z[i] * g[i];
                }
                store_pack<T, VEC>(op + (int64_t)(k * RP) * s.channels, y);
            }
        }
        // no barrier: the next tile writes sy only after its own first barrier, and sd, sb, sc were
        // last read before the barrier above
    }
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        if (c + k >= s.channels) continue;
        if (ENDS) {
            store_states(local + (at * s.channels + c + k) * s.states, q * NS, s.states, states_packed(s.states), h[k]);
            if (q == 0) sums[at * s.channels + c + k] = total[k];
        } else if (state_out != nullptr && w.chunk == s.chunks - 1) {
            float v[NS];
            quad_to(v, h[k]);
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (q * NS + i < s.states) state_out[w.b * per + (int64_t)(c + k) * s.states + q * NS + i] = v[i];
        }
    }
}

// Joins the chunks along a row: afterwards local[b][chunk] holds what enters the chunk (BACK: from
// behind).  One thread per (row, channel, state).
template <bool BACK>
__global__ void __launch_bounds__(256) scan_join_kernel(float* __restrict__ local, const float* __restrict__ sums,
                                                        const float* __restrict__ A, const float* __restrict__ start, int64_t rows,
                                                        ScanShape s) {
    pdl_wait_then_trigger();
    const int64_t per = (int64_t)s.channels * s.states;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= rows * per) return;
    const int64_t b = e / per, cn = e % per, c = cn / s.states;
    const float a2 = A[cn] * LOG2_E;
    float carry = start ? start[e] : 0.f;
    constexpr int AHEAD = 8;      // chunks whose values are loaded together: the chain itself is one fused add each
    for (int k0 = 0; k0 < s.chunks; k0 += AHEAD) {
        float own[AHEAD], keep[AHEAD], decay[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool there = k0 + k < s.chunks;
            const int64_t at = b * s.chunks + (BACK ? s.chunks - 1 - (k0 + k) : k0 + k);
            own[k] = there ? local[at * per + cn] : 0.f;
            decay[k] = there ? a2 * sums[at * s.channels + c] : 0.f;
            keep[k] = exp2_f32(decay[k]);
        }
        const float start_of_group = carry;
        float enters[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            enters[k] = carry;
            carry = fmaf(keep[k], carry, own[k]);         // chunks that do not exist: own and keep are 0 and 1
        }
        // What is not finite stays so, so one look at the end of a group is enough.  A chunk's decay may leave fp32's range
        // where those of its nodes do not: then it is applied in halves, and what was zero or infinite stays so, as it
        // would node by node.
        if (!(fabsf(carry) < INFINITY)) {
            carry = start_of_group;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                enters[k] = carry;
                if (keep[k] == 0.f || keep[k] == INFINITY) {
                    const float half = exp2_f32(0.5f * decay[k]);
                    const bool stays = (carry == 0.f || fabsf(carry) == INFINITY) && fabsf(decay[k]) < INFINITY;
                    carry = (stays ? carry : carry * half * half) + own[k];
                } else {
                    carry = fmaf(keep[k], carry, own[k]);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (k0 + k >= s.chunks) break;
            const int64_t at = b * s.chunks + (BACK ? s.chunks - 1 - (k0 + k) : k0 + k);
            local[at * per + cn] = enters[k];
        }
    }
}

// ----------------------------------------------------------------------------------------- backward
// What one block keeps in shared memory.
template <typename T, int S, int NC, int VEC>
struct BackSpace {
    static constexpr int THREADS = back_threads(NC), CT = THREADS / S * NC, NP = S * NS, WARPS = THREADS / 32;
    __align__(16) float2 sdt[TILE][CT + ZEROS], sdu[TILE][CT + ZEROS], sg[TILE][CT + ZEROS];     // dt, dt;  dt u, dt u;  gy, gy
    __align__(16) float sb[TILE][NP], sc[TILE][NP];
    __align__(8) float sy[TILE][CT], st[TILE][CT], sq[TILE][CT];         // C.h, p.B, sum p a h A
    float red[WARPS][TILE][2 * NP];                         // the warps' sums over channels: gB, gC
    static constexpr int RP = THREADS / (CT / VEC), RN = THREADS / NP;
    using Act = Feed<T, VEC, TILE, RP, 4, THREADS>;
    typename Act::Space room;
    Quad hold[TILE / KEEP][NC][THREADS];                    // the thread's stored states of the tile, on their way a tile ahead
};

// part_bc[tile][b][t][2 NP]: this block's share of gB and gC; part_a[b][chunk][channel][states + 2]:
// this chunk's share of gA, gD and gdelta_bias.
// ENDS = true, for rows cut into chunks: only local = what the adjoint state hands to the node before the
// chunk when nothing comes from behind it, and the sums of dt.
template <typename T, int S, int NC, int VEC, bool ENDS, bool PARTIAL>
__global__ void __launch_bounds__(back_threads(NC), back_blocks(NC)) scan_bwd_kernel(ScanIn<T> in, const float* __restrict__ kept, const float* __restrict__ enter,
                                                                const float* __restrict__ gstate_out, T* __restrict__ gu,
                                                                T* __restrict__ gdelta, T* __restrict__ gz, float* __restrict__ gstate,
                                                                float* __restrict__ part_bc, float* __restrict__ part_a,
                                                                float* __restrict__ local, float* __restrict__ sums, int64_t rows, ScanShape s) {
    pdl_wait_then_trigger();
    using Space = BackSpace<T, S, NC, VEC>;
    using Act = typename Space::Act;
    constexpr int THREADS = Space::THREADS, CT = Space::CT, NP = Space::NP, CP = CT / VEC, RP = Space::RP, RN = Space::RN;
    enum { DELTA, Z, GOUT, U };
    using Bc = States<T, TILE, RN>;
    extern __shared__ __align__(16) uint8_t raw_space[];
    Space& m = *reinterpret_cast<Space*>(raw_space);
    const Where w = where(s);
    const int tid = threadIdx.x, q = tid % S, cl = tid / S * NC, warp = tid / 32, lane = tid % 32;
    const int c0 = w.tile * CT, c = c0 + cl, from = ENDS || q * NS < s.states ? cl : CT;      // where it reads dt, dt u and gy
    const int64_t first = (int64_t)w.chunk * s.chunk;
    const int64_t end = first + s.chunk < s.length ? first + s.chunk : s.length;
    const int64_t per = (int64_t)s.channels * s.states;
    const int64_t at = w.b * s.chunks + w.chunk;
    Quad a2[NC], p[NC], ga[NC];                  // p: the adjoint state, from behind
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int64_t cn = (int64_t)(c + k) * s.states;
        const bool mine = c + k < s.channels;
        a2[k] = load_states(mine ? in.A + cn : nullptr, q * NS, s.states, LOG2_E);
        p[k] = load_states(ENDS || !mine ? nullptr : enter ? enter + at * per + cn : gstate_out ? gstate_out + w.b * per + cn : nullptr, q * NS,
                           s.states, 1.f);
        ga[k] = {0, 0};
    }
    const int col = tid % CP * VEC, r0 = tid / CP, n = tid % NP, rn = tid / NP;
    const bool column = c0 + col < s.channels, row_n = n < s.states;
    float bias[VEC], dd[VEC], gd[VEC] = {}, gbias[VEC] = {};
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        bias[i] = in.bias && column ? in.bias[c0 + col + i] : 0.f;
        dd[i] = in.D && column ? in.D[c0 + col + i] : 0.f;
    }
    const int ntiles = (int)((end - first + TILE - 1) / TILE);
    const int64_t last = first + (int64_t)(ntiles - 1) * TILE;
    Act act(m.room, r0, column);
    Bc bt, ct;
    act.start(DELTA, in.delta + w.b * s.delta_batch + last * s.delta_node + c0, s.delta_node, col);
    act.start(Z, in.z + w.b * s.z_batch + last * s.z_node + c0, s.z_node, col);
    act.start(GOUT, in.gout + w.b * s.g_batch + last * s.g_node + c0, s.g_node, col);
    act.start(U, in.u + w.b * s.u_batch + last * s.u_node + c0, s.u_node, col);
    bt.p = in.B + w.b * s.B_batch + (last + rn) * s.B_node + n;
    ct.p = in.C + w.b * s.C_batch + (last + rn) * s.C_node + n;
    auto fetch = [&](int here) {
        act.request(DELTA, s.delta_node, here, -TILE);
        if (in.z) act.request(Z, s.z_node, here, -TILE);
        act.request(GOUT, s.g_node, here, -TILE);
        ct.load(s.C_node, rn, here, row_n, -TILE);
        if constexpr (!ENDS) {
            act.request(U, s.u_node, here, -TILE);
            bt.load(s.B_node, rn, here, row_n, -TILE);
        }
    };
    // the stored states before the pieces of the tile at node t; lanes without states or channel keep zeros
    auto fetch_states = [&](int64_t t) {
#pragma unroll
        for (int piece = 0; piece < TILE / KEEP; ++piece) {
            const float* hp = kept + ((w.b * s.kept_nodes + t / KEEP + piece) * s.channels + c) * s.states;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                if (t + piece * KEEP >= end || c + k >= s.channels || q * NS >= s.states) continue;
                Quad* dst = &m.hold[piece][k][tid];
                if (states_packed(s.states))
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))),
                                 "l"(hp + k * s.states + q * NS) : "memory");
                else *dst = load_states(hp + k * s.states, q * NS, s.states, 1.f);
            }
        }
    };
    if constexpr (!ENDS) {
#pragma unroll
        for (int piece = 0; piece < TILE / KEEP; ++piece)
#pragma unroll
            for (int k = 0; k < NC; ++k) m.hold[piece][k][tid] = {0, 0};
        if (ntiles > 0) fetch_states(last);
        if (tid < TILE * ZEROS)
            m.sdt[tid / ZEROS][CT + tid % ZEROS] = m.sdu[tid / ZEROS][CT + tid % ZEROS] = m.sg[tid / ZEROS][CT + tid % ZEROS] = make_float2(0.f, 0.f);
    }
    float total[NC] = {};
    if (ntiles > 0) fetch((int)(end - last));
    for (int64_t t0 = last; t0 >= first && ntiles > 0; t0 -= TILE) {
        const int here = (int)(end - t0 < TILE ? end - t0 : TILE);
        const int top = (here - 1) / KEEP * KEEP;      // first node of the last piece that has nodes
        act.arrive();
        if constexpr (!ENDS && !Act::ASYNC) asm volatile("cp.async.wait_all;" ::: "memory");      // the stored states
#pragma unroll
        for (int k = 0; k < Act::PER; ++k) {
            const int r = r0 + k * RP;
            if (TILE % RP != 0 && r >= TILE) break;
            float dt[VEC], u[VEC], z[VEC], g[VEC], gate[VEC];
            act.get(dt, DELTA, k);
            act.get(g, GOUT, k);
            if constexpr (!ENDS) act.get(u, U, k);
#pragma unroll
            for (int i = 0; i < VEC; ++i) dt[i] += bias[i];
            if (s.softplus) softplus_of<VEC>(dt);
            if (in.z) {
                act.get(z, Z, k);
                sigmoid_of<VEC>(gate, z);
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if (in.z) g[i] *= z[i] * gate[i];
                u[i] = ENDS ? 0.f : dt[i] * u[i];
                if (here < TILE && r >= here) dt[i] = u[i] = g[i] = 0.f;      // past the end: nothing changes
            }
            put_twice<VEC>(&m.sdt[r][col], dt);
            put_twice<VEC>(&m.sg[r][col], g);
            if constexpr (!ENDS) put_twice<VEC>(&m.sdu[r][col], u);
        }
#pragma unroll
        for (int k = 0; k < Bc::PER; ++k) {
            if (TILE % RN != 0 && rn + k * RN >= TILE) break;
            if constexpr (!ENDS) m.sb[rn + k * RN][n] = to_f32<T>(bt.v[k]);
            m.sc[rn + k * RN][n] = to_f32<T>(ct.v[k]);
        }
        __syncthreads();
        if (t0 > first) fetch(TILE);
        if constexpr (ENDS) {
#pragma unroll 4
            for (int r = TILE - 1; r >= 0; --r) {
                const Quad c4 = quad_at(&m.sc[r][q * NS]);
                uint64_t dt2[NC], g2[NC];
                get_channels(dt2, &m.sdt[r][cl]);
                get_channels(g2, &m.sg[r][cl]);
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    float dt, same;
                    unpair(dt2[k], dt, same);
                    total[k] += dt;
                    p[k].lo = mul2(fma2(c4.lo, g2[k], p[k].lo), exp2_pair(mul2(dt2[k], a2[k].lo)));
                    p[k].hi = mul2(fma2(c4.hi, g2[k], p[k].hi), exp2_pair(mul2(dt2[k], a2[k].hi)));
                }
            }
            __syncthreads();
        } else {
#pragma unroll 1
            for (int base = top; base >= 0; base -= KEEP) {
                Quad hs[KEEP + 1][NC];                 // hs[r]: the state BEFORE node base + r
#pragma unroll
                for (int k = 0; k < NC; ++k) hs[0][k] = m.hold[base / KEEP][k][tid];
                if (base == 0 && t0 > first) fetch_states(t0 - TILE);
                // forward through the piece
#pragma unroll
                for (int k0 = 0; k0 < KEEP; k0 += 4) {
                    asm volatile("" ::: "memory");     // the loads of a group stay with it: hoisted ones would spill the states
                    float y[4 * NC];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = k0 + j;
                        const Quad b4 = quad_at(&m.sb[base + r][q * NS]), c4 = quad_at(&m.sc[base + r][q * NS]);
                        uint64_t dt2[NC], du2[NC];
                        get_channels(dt2, &m.sdt[base + r][from]);
                        get_channels(du2, &m.sdu[base + r][from]);
#pragma unroll
                        for (int k = 0; k < NC; ++k) {
                            hs[r + 1][k].lo = fma2(exp2_pair(mul2(dt2[k], a2[k].lo)), hs[r][k].lo, mul2(du2[k], b4.lo));
                            hs[r + 1][k].hi = fma2(exp2_pair(mul2(dt2[k], a2[k].hi)), hs[r][k].hi, mul2(du2[k], b4.hi));
                            if constexpr (PARTIAL) hs[r + 1][k] = existing(hs[r + 1][k], q * NS, s.states);
                            y[NC * j + k] = sum2(fma2(c4.lo, hs[r + 1][k].lo, mul2(c4.hi, hs[r + 1][k].hi)));
                        }
                    }
                    put_sums<S, NC, CT>(m.sy, y, base + k0, cl, q);
                }
                // and backwards
#pragma unroll
                for (int k0 = KEEP - 4; k0 >= 0; k0 -= 4) {
                    float tb[4 * NC], ta[4 * NC];
#pragma unroll
                    for (int j = 3; j >= 0; --j) {
                        const int r = k0 + j;
                        asm volatile("" ::: "memory");
                        const Quad b4 = quad_at(&m.sb[base + r][q * NS]), c4 = quad_at(&m.sc[base + r][q * NS]);
                        uint64_t dt2[NC], du2[NC], g2[NC];
                        get_channels(dt2, &m.sdt[base + r][from]);
                        get_channels(du2, &m.sdu[base + r][from]);
                        get_channels(g2, &m.sg[base + r][from]);
                        Quad vb, vc;                   // shares of gB and gC of this node, summed over the thread's channels
#pragma unroll
                        for (int k = 0; k < NC; ++k) {
                            const uint64_t g = g2[k], dt = dt2[k], du = du2[k];
                            p[k].lo = fma2(c4.lo, g, p[k].lo);
                            p[k].hi = fma2(c4.hi, g, p[k].hi);
                            if constexpr (PARTIAL) p[k] = existing(p[k], q * NS, s.states);
                            vb.lo = k == 0 ? mul2(p[k].lo, du) : fma2(p[k].lo, du, vb.lo);
                            vb.hi = k == 0 ? mul2(p[k].hi, du) : fma2(p[k].hi, du, vb.hi);
                            vc.lo = k == 0 ? mul2(hs[r + 1][k].lo, g) : fma2(hs[r + 1][k].lo, g, vc.lo);
                            vc.hi = k == 0 ? mul2(hs[r + 1][k].hi, g) : fma2(hs[r + 1][k].hi, g, vc.hi);
                            tb[NC * j + k] = sum2(fma2(p[k].lo, b4.lo, mul2(p[k].hi, b4.hi)));
                            p[k].lo = mul2(p[k].lo, exp2_pair(mul2(dt, a2[k].lo)));
                            p[k].hi = mul2(p[k].hi, exp2_pair(mul2(dt, a2[k].hi)));
                            if constexpr (PARTIAL) p[k] = existing(p[k], q * NS, s.states);
                            const uint64_t ph_lo = mul2(p[k].lo, hs[r][k].lo), ph_hi = mul2(p[k].hi, hs[r][k].hi);
                            ta[NC * j + k] = sum2(fma2(ph_lo, a2[k].lo, mul2(ph_hi, a2[k].hi)));
                            ga[k].lo = fma2(ph_lo, dt, ga[k].lo);
                            ga[k].hi = fma2(ph_hi, dt, ga[k].hi);
                        }
                        float v[2 * NS];
                        unpair(vb.lo, v[0], v[1]);
                        unpair(vb.hi, v[2], v[3]);
                        unpair(vc.lo, v[4], v[5]);
                        unpair(vc.hi, v[6], v[7]);
                        const int share = sum_lanes<2 * NS, 16, S>(v, lane);
#pragma unroll
                        for (int i = 0; i < sums_left<2 * NS, 16, S>(); ++i)
                            m.red[warp][base + r][((share + i) / NS) * NP + q * NS + (share + i) % NS] = v[i];
                    }
                    put_sums<S, NC, CT>(m.st, tb, base + k0, cl, q);
                    put_sums<S, NC, CT>(m.sq, ta, base + k0, cl, q);
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < Act::PER; ++k) {
                const int r = r0 + k * RP;
                if (r >= here || !column) continue;
                float ou[VEC], od[VEC], oz[VEC], raw[VEC], slope[VEC], z[VEC], gate[VEC], go[VEC], u[VEC];
                act.get(u, U, k);
                if (s.softplus) {
                    act.get(raw, DELTA, k);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) raw[i] += bias[i];
                    sigmoid_of<VEC>(slope, raw);
                }
                if (in.z) {
                    act.get(z, Z, k);
                    act.get(go, GOUT, k);
                    sigmoid_of<VEC>(gate, z);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float dt = m.sdt[r][col + i].x, gy = m.sg[r][col + i].x, through = m.st[r][col + i];
                    ou[i] = fmaf(dt, through, in.D ? dd[i] * gy : 0.f);      // without D there is no term, not 0 gy
                    od[i] = fmaf(u[i], through, m.sq[r][col + i] * (1.f / LOG2_E));
                    if (s.softplus) od[i] *= slope[i];
                    if (in.z) oz[i] = go[i] * (in.D ? fmaf(dd[i], u[i], m.sy[r][col + i]) : m.sy[r][col + i]) * (gate[i] * fmaf(z[i], 1.f - gate[i], 1.f));
                    gd[i] = fmaf(gy, u[i], gd[i]);
                    gbias[i] += od[i];
                }
                const int64_t o = (w.b * s.length + t0 + r) * s.channels + c0 + col;
                store_pack<T, VEC>(gu + o, ou);
                store_pack<T, VEC>(gdelta + o, od);
                if (in.z) store_pack<T, VEC>(gz + o, oz);
            }
            for (int e = tid; e < here * 2 * NP; e += THREADS) {
                const int r = e / (2 * NP), k = e % (2 * NP);
                float v = 0.f;
#pragma unroll
                for (int i = 0; i < Space::WARPS; ++i) v += m.red[i][r][k];
                part_bc[(((int64_t)w.tile * rows + w.b) * s.length + t0 + r) * (2 * NP) + k] = v;
            }
            __syncthreads();
        }
    }
    if constexpr (ENDS) {
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            if (c + k >= s.channels) continue;
            store_states(local + (at * s.channels + c + k) * s.states, q * NS, s.states, states_packed(s.states), p[k]);
            if (q == 0) sums[at * s.channels + c + k] = total[k];
        }
    } else {
        // this chunk's share of the parameters' gradients
        float* pa = part_a + (at * s.channels) * (int64_t)(s.states + 2);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            if (c + k >= s.channels) continue;
            float v[NS], e[NS];
            quad_to(v, ga[k]);
            quad_to(e, p[k]);
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (q * NS + i < s.states) {
                    pa[(int64_t)(c + k) * (s.states + 2) + q * NS + i] = v[i];
                    if (gstate != nullptr && w.chunk == 0) gstate[w.b * per + (int64_t)(c + k) * s.states + q * NS + i] = e[i];
                }
        }
        // threads tid, tid + CP, ... hold sums of the same channels
        float(*fin)[THREADS] = reinterpret_cast<float(*)[THREADS]>(raw_space);     // 2 VEC rows
        static_assert(2 * sizeof(m.sdt) >= 2 * VEC * THREADS * sizeof(float), "room for the sums of every thread");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            fin[i][tid] = gd[i];
            fin[VEC + i][tid] = gbias[i];
        }
        __syncthreads();
        if (tid < CT && c0 + tid < s.channels) {
            float v0 = 0.f, v1 = 0.f;
            for (int e = tid / VEC; e < THREADS; e += CP) { v0 += fin[tid % VEC][e]; v1 += fin[VEC + tid % VEC][e]; }
            pa[(int64_t)(c0 + tid) * (s.states + 2) + s.states] = v0;
            pa[(int64_t)(c0 + tid) * (s.states + 2) + s.states + 1] = v1;
        }
    }
}

// gB, gC: sums of part_bc over the channel tiles.
template <typename T>
__global__ void __launch_bounds__(256) scan_sum_bc_kernel(const float* __restrict__ part, int tiles, int64_t nodes, int np, int states,
                                                          T* __restrict__ gB, T* __restrict__ gC) {
    pdl_wait_then_trigger();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, all = nodes * 2 * np;
    if (e >= all) return;
    float v = 0.f;
    for (int k = 0; k < tiles; ++k) v += part[k * all + e];
    const int64_t t = e / (2 * np);
    const int n = (int)(e % (2 * np));
    if (n < np) {
        if (n < states) gB[t * states + n] = from_f32<T>(v);
    } else if (n - np < states) {
        gC[t * states + n - np] = from_f32<T>(v);
    }
}

// gA, gD, gdelta_bias: sums of part_a over rows and chunks.
__global__ void __launch_bounds__(256) scan_sum_a_kernel(const float* __restrict__ part, int64_t parts, int channels, int states,
                                                         float* __restrict__ gA, float* __restrict__ gD, float* __restrict__ gbias) {
    pdl_wait_then_trigger();
    __shared__ float sums[8][32];
    const int64_t width = (int64_t)channels * (states + 2);
    const int64_t e = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (e < width)
        for (int64_t p = threadIdx.y; p < parts; p += 8) v += part[p * width + e];
    sums[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && e < width) {
#pragma unroll
        for (int r = 1; r < 8; ++r) v += sums[r][threadIdx.x];
        const int64_t c = e / (states + 2);
        const int n = (int)(e % (states + 2));
        if (n < states) gA[c * states + n] = v;
        else if (n == states) { if (gD != nullptr) gD[c] = v; }
        else if (gbias != nullptr) gbias[c] = v;
    }
}

// ---------------------------------------------------------------------------------------- one node
// Bound by the states' traffic, 8 bytes each.  S lanes share a channel, four states each, and take four
// channels of one row at once, so that their loads are on their way together.  What is per channel (dt,
// the gate) is computed by one lane for each: the lane to which the sum over the states comes.  B and C
// of the row are loaded once per thread.  PADDED: there are fewer states than lanes hold.  state_out may be state: a thread reads what it writes.
template <typename T, int S, bool PADDED>
__global__ void __launch_bounds__(STEP_THREADS, PADDED && S > 2 ? 8 : 1) scan_step_kernel(ScanIn<T> in, const float* state, T* __restrict__ out, float* state_out,
                                                                 int across, bool packed, ScanShape s) {
    pdl_wait_then_trigger();
    constexpr int CT = STEP_THREADS / S, K = STEP_CHANNELS;           // channels next to one another
    constexpr int OWN = sums_left<K, S / 2, 1>(), SHARE = S > K ? S / K : 1;      // channels of a lane, lanes of a channel
    const int64_t b = blockIdx.x / across;
    const int lane = threadIdx.x % 32, q = threadIdx.x % S, n0 = q * NS, c0 = (int)(blockIdx.x % across) * (CT * K) + threadIdx.x / S;
    const int first = q * K / S;                                      // its first channel
    const bool mine = n0 < s.states;
    Quad h[K], a2[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = c0 + k * CT;
        const int64_t cn = (int64_t)c * s.states;
        h[k] = a2[k] = {0, 0};
        if (c >= s.channels) continue;
        if (packed) {
            if (mine && state) h[k] = quad_at(state + b * s.channels * s.states + cn + n0);
            if (mine) a2[k] = quad_at(in.A + cn + n0);
        } else {
            h[k] = load_states(state ? state + b * s.channels * s.states + cn : nullptr, n0, s.states, 1.f);
            a2[k] = load_states(in.A + cn, n0, s.states, 1.f);
        }
    }
    float dt[OWN], u[OWN], z[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int c = c0 + (first + k) * CT;
        dt[k] = u[k] = z[k] = 0.f;
        if (c < s.channels) {
            dt[k] = to_f32<T>(in.delta[b * s.delta_batch + c]) + (in.bias ? in.bias[c] : 0.f);
            u[k] = to_f32<T>(in.u[b * s.u_batch + c]);
            if (in.z) z[k] = to_f32<T>(in.z[b * s.z_batch + c]);
        }
    }
    float bv[NS], cv[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        bv[i] = n0 + i < s.states ? to_f32<T>(in.B[b * s.B_batch + n0 + i]) : 0.f;
        cv[i] = n0 + i < s.states ? to_f32<T>(in.C[b * s.C_batch + n0 + i]) : 0.f;
    }
    const Quad b4 = quad_of(bv), c4 = quad_of(cv);
#pragma unroll
    for (int k = 0; k < OWN; ++k) dt[k] = step_of(dt[k], s.softplus);
    float y[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = c0 + k * CT, owner = (lane & ~(S - 1)) + (S >= K ? k * (S / K) : k / OWN);
        const float step = __shfl_sync(~0u, dt[k % OWN], owner), du = __shfl_sync(~0u, dt[k % OWN] * u[k % OWN], owner);
        const bool live = !PADDED || mine;                            // infinities stop at lanes without a state
        const uint64_t d = both(live ? step * LOG2_E : 0.f), w = both(live ? du : 0.f);
        h[k].lo = fma2(exp2_pair(mul2(d, a2[k].lo)), h[k].lo, mul2(w, b4.lo));
        h[k].hi = fma2(exp2_pair(mul2(d, a2[k].hi)), h[k].hi, mul2(w, b4.hi));
        if (PADDED && s.states % NS != 0) h[k] = existing(h[k], n0, s.states);
        y[k] = sum2(fma2(c4.lo, h[k].lo, mul2(c4.hi, h[k].hi)));
        if (c < s.channels && state_out != nullptr) store_states(state_out + (b * s.channels + c) * s.states, n0, s.states, packed, h[k]);
    }
    sum_lanes<K, S / 2, 1>(y, q);
    if (q % SHARE != 0) return;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int c = c0 + (first + k) * CT;
        if (c >= s.channels) continue;
        if (in.D) y[k] = fmaf(in.D[c], u[k], y[k]);
        if (in.z) y[k] *= z[k] * sigmoid_f32(z[k]);
        out[b * s.channels + c] = from_f32<T>(y[k]);
    }
}

// --------------------------------------------------------------------------------------------- host
int lanes_of(int states) {
    int s = 2;
    while (s * NS < states) s *= 2;
    return s;
}

ScanShape shape_of(const fpde_scan_args* a) {
    ScanShape s = {};
    s.length = a->length;
    s.u_batch = a->u_batch; s.u_node = a->u_node;
    s.delta_batch = a->delta_batch; s.delta_node = a->delta_node;
    s.z_batch = a->z_batch; s.z_node = a->z_node;
    s.B_batch = a->B_batch; s.B_node = a->B_node;
    s.C_batch = a->C_batch; s.C_node = a->C_node;
    s.g_batch = a->gout_batch; s.g_node = a->gout_node;
    s.channels = (int)a->channels;
    s.states = a->states;
    s.softplus = a->softplus;
    return s;
}

// The plan depends on sizes only, so that the forward and the backward call agree on it.
ScanShape plan(const fpde_scan_args* a, bool backward) {
    ScanShape s = shape_of(a);
    s.tiles = (int)ceil_div(a->channels, (backward ? BACK_LANES : FWD_LANES) * 4 / lanes_of(a->states));
    s.kept_nodes = ceil_div(a->length, KEEP);
    // Chunks.  The blocks run in waves of `resident` per SM, and a wave takes as long as its nodes: the marches
    // are bound by latency, so fewer blocks on an SM are hardly faster.  Splitting adds the pass that forms
    // the chunks' ends, a share `ends_cost` of the march, and two launches, worth about 80 nodes.  The
    // cheapest number of chunks wins, the fewest of equals.  Measured against seven other numbers for each of 13 shapes, both
    // directions: within 5 % of the best of them but for the forward pass of 32 x 300 x 333 (5 chunks 65 us, none 46), 8 x 512 x 1024 (4
    // chunks 65, none 58), 2 x 8192 x 2048 (8 chunks 439, 32 400), 1 x 4096 x 256 and 1 x 65536 x 64 (10 %), and the gradients
    // of 16 x 256 x 256 (57, 53) and 1 x 512 x 2048 (62, 59).
    const int64_t length = a->length > 0 ? a->length : 1, blocks = a->batch * s.tiles;
    const int64_t resident = 148 * (backward ? back_blocks(2) : fwd_blocks(2));
    const double ends_cost = backward ? BACK_ENDS : FWD_ENDS;
    const int64_t most = ceil_div(length, 2 * TILE) < 1024 ? ceil_div(length, 2 * TILE) : 1024;
    int64_t chunk = length;
    double best = 0;
    for (int64_t k = 1; k <= most; ++k) {
        const int64_t nodes = k == 1 ? length : ceil_div(ceil_div(length, k), TILE) * TILE;
        const int64_t waves = ceil_div(blocks * ceil_div(length, nodes), resident);
        const double cost = (double)(nodes * waves) * (k == 1 ? 1 : 1 + ends_cost) + (k == 1 ? 0 : 80);
        if (k == 1 || cost < best) { best = cost; chunk = nodes; }
        if (waves > 4) break;
    }
    chunk = ceil_div(chunk, TILE) * TILE;
    if (chunk > (1 << 30)) chunk = 1 << 30;
    s.chunk = (int)chunk;
    s.chunks = (int)ceil_div(a->length > 0 ? a->length : 1, chunk);
    return s;
}

int check_scan_sizes(const fpde_scan_args* a, bool step = false) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->states < 1 || a->states > FPDE_SCAN_MAX_STATES) return FPDE_ERR_PARAM;
    if (a->batch < 0 || a->channels < 0 || a->length < 0 || a->channels > (1 << 24) || a->length > (1ll << 36) || a->batch > (1ll << 36) ||
        !product_fits(a->batch, step ? 1 : a->length, a->channels))
        return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

int check_scan(const fpde_scan_args* a, bool step) {
    const int st = check_scan_sizes(a, step);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels > 0) {
        if (a->A == nullptr) return FPDE_ERR_NULL;
        if ((step || a->length > 0) && (a->u == nullptr || a->delta == nullptr || a->B == nullptr || a->C == nullptr)) return FPDE_ERR_NULL;
        const size_t e = dtype_bytes(a->dtype);
        const void* act[] = {a->u, a->delta, a->z, a->B, a->C, a->out, a->gout, a->gu, a->gdelta, a->gz, a->gB, a->gC};
        const void* par[] = {a->A, a->D, a->delta_bias, a->state, a->state_out, a->gstate_out, a->gA, a->gD, a->gdelta_bias, a->gstate};
        for (const void* p : act)
            if (!aligned(p, e)) return FPDE_ERR_ALIGN;
        for (const void* p : par)
            if (!aligned(p, 4)) return FPDE_ERR_ALIGN;
    }
    return FPDE_OK;
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// Workspace: [local states][sums of dt] of the chunks, then [part_bc][part_a] of the backward pass.
struct ScanSpace {
    size_t local, sums, part_bc, part_a, total;
};
ScanSpace space(const fpde_scan_args* a, const ScanShape& s, bool backward) {
    ScanSpace w = {};
    const size_t per = (size_t)a->batch * s.chunks * s.channels;
    size_t at = 0;
    if (s.chunks > 1) {
        w.local = at; at += round16(per * s.states * 4);
        w.sums = at; at += round16(per * 4);
    }
    if (backward) {
        w.part_bc = at; at += round16((size_t)s.tiles * a->batch * s.length * 2 * lanes_of(s.states) * NS * 4);
        w.part_a = at; at += round16(per * (s.states + 2) * 4);
    }
    w.total = at;
    return w;
}

template <typename T>
ScanIn<T> inputs(const fpde_scan_args* a) {
    return {(const T*)a->u, (const T*)a->delta, (const T*)a->z, (const T*)a->B, (const T*)a->C, (const T*)a->gout, a->A, a->D, a->delta_bias};
}

#define FPDE_TRY(x)                           \
    do {                                      \
        const cudaError_t e_ = (x);           \
        if (e_ != cudaSuccess) return e_;     \
    } while (0)

// Two channels per load where every row of every activation starts on two elements.
template <typename T>
bool scan_pairs(const fpde_scan_args* a, bool backward) {
    const size_t e = sizeof(T);
    bool ok = a->channels % 2 == 0 && packs(a->u, a->u_batch, a->u_node, e, 2) && packs(a->delta, a->delta_batch, a->delta_node, e, 2) &&
              (a->z == nullptr || packs(a->z, a->z_batch, a->z_node, e, 2));
    if (!backward) return ok && aligned(a->out, 2 * e);
    return ok && packs(a->gout, a->gout_batch, a->gout_node, e, 2) && aligned(a->gu, 2 * e) && aligned(a->gdelta, 2 * e) && aligned(a->gz, 2 * e);
}

template <typename T, int S, int NC, int VEC>
cudaError_t run_fwd(const fpde_scan_args* a, const ScanShape& s, cudaStream_t st) {
    const ScanSpace w = space(a, s, false);
    const ScanIn<T> in = inputs<T>(a);
    const int64_t blocks = a->batch * s.tiles * s.chunks;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    float* local = nullptr;
    if (s.chunks > 1) {
        local = (float*)((char*)a->workspace + w.local);
        float* sums = (float*)((char*)a->workspace + w.sums);
        constexpr size_t bytes = sizeof(FwdSpace<T, S, 1, VEC, true>);
        static std::atomic<uint64_t> allowed{0};
        FPDE_TRY(allow_smem(scan_fwd_kernel<T, S, 1, VEC, true, false>, bytes, allowed));
        FPDE_TRY(launch_kernel_smem(scan_fwd_kernel<T, S, 1, VEC, true, false>, grid, dim3(fwd_threads(1)), bytes, st, in, (const float*)nullptr, (const float*)nullptr,
                               (T*)nullptr, (float*)nullptr, (float*)nullptr, local, sums, s));
        FPDE_TRY(launch_kernel(scan_join_kernel<false>, dim3((unsigned)ceil_div(a->batch * s.channels * s.states, 256)), dim3(256), st,
                               local, (const float*)sums, a->A, a->state, a->batch, s));
    }
    constexpr size_t bytes = sizeof(FwdSpace<T, S, NC, VEC, false>);
    auto march = [&](auto* kernel, std::atomic<uint64_t>& allowed) {
        FPDE_TRY(allow_smem(kernel, bytes, allowed));
        return launch_kernel_smem(kernel, grid, dim3(fwd_threads(NC)), bytes, st, in, a->state, (const float*)local, (T*)a->out, a->state_out,
                                  (float*)a->kept, (float*)nullptr, (float*)nullptr, s);
    };
    static std::atomic<uint64_t> whole{0}, partial{0};
    return s.states % NS == 0 ? march(scan_fwd_kernel<T, S, NC, VEC, false, false>, whole) : march(scan_fwd_kernel<T, S, NC, VEC, false, true>, partial);
}

template <typename T, int S, int NC, int VEC>
cudaError_t run_bwd(const fpde_scan_args* a, const ScanShape& s, cudaStream_t st) {
    const ScanSpace w = space(a, s, true);
    const ScanIn<T> in = inputs<T>(a);
    const int64_t blocks = a->batch * s.tiles * s.chunks;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    constexpr size_t bytes = sizeof(BackSpace<T, S, NC, VEC>);
    char* ws = (char*)a->workspace;
    float *local = nullptr, *part_bc = (float*)(ws + w.part_bc), *part_a = (float*)(ws + w.part_a);
    if (s.chunks > 1) {
        constexpr size_t ends = sizeof(BackSpace<T, S, 1, VEC>);
        local = (float*)(ws + w.local);
        float* sums = (float*)(ws + w.sums);
        static std::atomic<uint64_t> allowed{0};
        FPDE_TRY(allow_smem(scan_bwd_kernel<T, S, 1, VEC, true, false>, ends, allowed));
        FPDE_TRY(launch_kernel_smem(scan_bwd_kernel<T, S, 1, VEC, true, false>, grid, dim3(back_threads(1)), ends, st, in, (const float*)nullptr,
                                    (const float*)nullptr, (const float*)nullptr, (T*)nullptr, (T*)nullptr, (T*)nullptr, (float*)nullptr,
                                    (float*)nullptr, (float*)nullptr, local, sums, a->batch, s));
        FPDE_TRY(launch_kernel(scan_join_kernel<true>, dim3((unsigned)ceil_div(a->batch * s.channels * s.states, 256)), dim3(256), st,
                               local, (const float*)sums, a->A, a->gstate_out, a->batch, s));
    }
    auto march = [&](auto* kernel, std::atomic<uint64_t>& allowed) {
        FPDE_TRY(allow_smem(kernel, bytes, allowed));
        return launch_kernel_smem(kernel, grid, dim3(back_threads(NC)), bytes, st, in, (const float*)a->kept, (const float*)local, a->gstate_out,
                                  (T*)a->gu, (T*)a->gdelta, (T*)a->gz, a->gstate, part_bc, part_a, (float*)nullptr, (float*)nullptr, a->batch, s);
    };
    static std::atomic<uint64_t> whole{0}, partial{0};
    FPDE_TRY(s.states % NS == 0 ? march(scan_bwd_kernel<T, S, NC, VEC, false, false>, whole) : march(scan_bwd_kernel<T, S, NC, VEC, false, true>, partial));
    if (a->batch * a->length > 0)
        FPDE_TRY(launch_kernel(scan_sum_bc_kernel<T>, dim3((unsigned)ceil_div(a->batch * a->length * 2 * S * NS, 256)), dim3(256), st,
                               (const float*)part_bc, s.tiles, a->batch * a->length, S * NS, s.states, (T*)a->gB, (T*)a->gC));
    return launch_kernel(scan_sum_a_kernel, dim3((unsigned)ceil_div((int64_t)s.channels * (s.states + 2), 32)), dim3(32, 8), st,
                         (const float*)part_a, a->batch * s.chunks, s.channels, s.states, a->gA, a->gD, a->gdelta_bias);
}

template <typename T, int S>
cudaError_t run_step(const fpde_scan_args* a, cudaStream_t st) {
    const ScanShape s = shape_of(a);
    const int64_t across = ceil_div(s.channels, STEP_THREADS / S * STEP_CHANNELS), blocks = a->batch * across;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const bool packed = s.states % NS == 0 && aligned(a->state, 16) && aligned(a->state_out, 16) && aligned(a->A, 16);
    auto kernel = s.states == S * NS ? scan_step_kernel<T, S, false> : scan_step_kernel<T, S, true>;
    return launch_kernel(kernel, dim3((unsigned)blocks), dim3(STEP_THREADS), st, inputs<T>(a), a->state, (T*)a->out, a->state_out,
                         (int)across, packed, s);
}

// Up to so many blocks a march gives its threads one channel instead of two: a block then has twice the
// threads with half the work, which pays while SMs have warps to spare.  Rows of 256 nodes, bf16, us with one channel and with
// two.  16 states forward: 128 blocks 27 / 38, 256 31 / 39, 384 51 / 46, 592 51 / 47, 640 52 / 69, 896 76 / 71, 1280 91 / 99, 1792
// 130 / 122; gradients: 128 127 / 141, 256 134 / 179, 296 136 / 181, 320 211 / 184, 448 259 / 297, 640 335 / 328.  32 states
// alike.  8 states: one channel is as good or better nearly everywhere (592 51 / 59, 768 81 / 74, 1024 88 / 115; gradients 296 202 / 281,
// 640 489 / 671).  Whole waves decide, and no one number is best at every size; these are the last ones at which one
// channel wins in both types.  The pass that only forms the chunks' ends always has one (169 / 189, 216 / 213).
constexpr int64_t FWD_ONE = 148 * 4, BACK_ONE = 148 * 2;

int channels_a_thread(const fpde_scan_args* a, const ScanShape& s, bool backward) {
    return a->batch * s.tiles * s.chunks <= (backward ? BACK_ONE : FWD_ONE) ? 1 : 2;
}

enum Call { CALL_FWD, CALL_BWD, CALL_STEP };

template <typename T, int S>
cudaError_t run(const fpde_scan_args* a, Call call, cudaStream_t st) {
    if (call == CALL_FWD) {
        const ScanShape s = plan(a, false);
        const bool pairs = scan_pairs<T>(a, false);
        if (channels_a_thread(a, s, false) == 1) return pairs ? run_fwd<T, S, 1, 2>(a, s, st) : run_fwd<T, S, 1, 1>(a, s, st);
        return pairs ? run_fwd<T, S, 2, 2>(a, s, st) : run_fwd<T, S, 2, 1>(a, s, st);
    }
    if (call == CALL_BWD) {
        const ScanShape s = plan(a, true);
        const bool pairs = scan_pairs<T>(a, true);
        if (channels_a_thread(a, s, true) == 1) return pairs ? run_bwd<T, S, 1, 2>(a, s, st) : run_bwd<T, S, 1, 1>(a, s, st);
        return pairs ? run_bwd<T, S, 2, 2>(a, s, st) : run_bwd<T, S, 2, 1>(a, s, st);
    }
    return run_step<T, S>(a, st);
}

template <typename T>
cudaError_t by_lanes(const fpde_scan_args* a, Call call, cudaStream_t st) {
    switch (lanes_of(a->states)) {
    case 2: return run<T, 2>(a, call, st);
    case 4: return run<T, 4>(a, call, st);
    case 8: return run<T, 8>(a, call, st);
    default: return run<T, 16>(a, call, st);
    }
}

int dispatch(const fpde_scan_args* a, Call call, void* stream) {
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = a->dtype == FPDE_F32    ? by_lanes<float>(a, call, st)
                          : a->dtype == FPDE_BF16 ? by_lanes<__nv_bfloat16>(a, call, st)
                                                  : by_lanes<__half>(a, call, st);
    return e == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
}

int check_space(const fpde_scan_args* a, bool backward) {
    const size_t need = fpde_selective_scan_workspace_bytes(a, backward);
    return need > 0 && (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < need) ? FPDE_ERR_WORKSPACE : FPDE_OK;
}

}  // namespace
}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_selective_scan_kept_bytes(const fpde_scan_args* a) {
    if (check_scan_sizes(a) != FPDE_OK) return 0;
    return (size_t)(a->batch * ceil_div(a->length, KEEP) * a->channels * a->states) * 4;
}

size_t fpde_selective_scan_workspace_bytes(const fpde_scan_args* a, int backward) {
    if (check_scan_sizes(a) != FPDE_OK) return 0;
    return space(a, plan(a, backward != 0), backward != 0).total;
}

int fpde_diag_scan_channels(const fpde_scan_args* a, int backward) {
    return check_scan_sizes(a) != FPDE_OK ? 0 : channels_a_thread(a, plan(a, backward != 0), backward != 0);
}

int fpde_diag_scan_chunks(const fpde_scan_args* a, int backward) { return check_scan_sizes(a) != FPDE_OK ? 0 : plan(a, backward != 0).chunks; }

int fpde_selective_scan_fwd(const fpde_scan_args* a, void* stream) {
    int st = check_scan(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels == 0) return FPDE_OK;
    if (a->out == nullptr && a->length > 0) return FPDE_ERR_NULL;
    if (a->kept != nullptr && (!aligned(a->kept, 16) || a->kept_bytes < fpde_selective_scan_kept_bytes(a))) return FPDE_ERR_WORKSPACE;
    if ((st = check_space(a, false)) != FPDE_OK) return st;
    return dispatch(a, CALL_FWD, stream);
}

int fpde_selective_scan_bwd(const fpde_scan_args* a, void* stream) {
    int st = check_scan(a, false);
    if (st != FPDE_OK) return st;
    if (a->channels == 0) return FPDE_OK;
    if (a->gA == nullptr) return FPDE_ERR_NULL;
    if (a->batch * a->length > 0) {
        if (a->gout == nullptr || a->gu == nullptr || a->gdelta == nullptr || a->gB == nullptr || a->gC == nullptr || (a->z && !a->gz))
            return FPDE_ERR_NULL;
        if (a->kept == nullptr || !aligned(a->kept, 16) || a->kept_bytes < fpde_selective_scan_kept_bytes(a)) return FPDE_ERR_WORKSPACE;
    }
    if ((st = check_space(a, true)) != FPDE_OK) return st;
    if (a->batch == 0)   // no rows: the sums over them are zero
        return launch_kernel(scan_sum_a_kernel, dim3((unsigned)ceil_div(a->channels * (a->states + 2), 32)), dim3(32, 8),
                             (cudaStream_t)stream, (const float*)nullptr, (int64_t)0, (int)a->channels, a->states, a->gA, a->gD,
                             a->gdelta_bias) == cudaSuccess ? FPDE_OK : FPDE_ERR_CUDA;
    return dispatch(a, CALL_BWD, stream);
}

int fpde_selective_scan_step(const fpde_scan_args* a, void* stream) {
    const int st = check_scan(a, true);
    if (st != FPDE_OK) return st;
    if (a->batch * a->channels == 0) return FPDE_OK;
    if (a->out == nullptr) return FPDE_ERR_NULL;
    return dispatch(a, CALL_STEP, stream);
}

}  // extern "C"
