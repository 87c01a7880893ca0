// Selective state space scan along the rows of (batch, length, channels) arrays: forward, gradients
// and the single-node form.
//
//   dt = softplus(delta + bias);  h[t] = exp(dt A) h[t-1] + dt u B;  y = C.h + D u;  out = y silu(z)
//
// Each (node, channel, state) costs one exponential and four multiplications or fused adds, against
// 16 bytes or less per (node, channel): with 16 states the special function unit (16 exponentials a
// clock and SM) bounds the forward pass, not memory.
//
// Layout.  A thread keeps four states of one channel; S = 2, 4, 8 or 16 neighbouring lanes share a
// channel, so a warp covers 32/S channels and the sums over states are shuffles among S lanes.  A
// block of 128 threads marches CT = 128/S channels through tiles of nodes; the tile's dt, dt u, B and
// C are brought to shared memory once, in fp32, by loads that run along the channels.
//
// Long rows.  Where batch x channels gives too few blocks, a row is cut into chunks: one kernel forms
// each chunk's state from zero and its sum of dt (the chunk's decay is exp(A sum dt)), a second joins
// them along the row, and the march starts every chunk from its joined state.  The gradient does the
// same backwards with the adjoint state.
//
// Gradients.  With gy = gout silu(z) the adjoint state is p[t] = C gy + exp(dt[t+1] A) p[t+1]; then
//   gC = sum_c h gy, gB = sum_c p dt u, gu = dt (p.B) + D gy, gdt = sum_n p exp(dt A) h[t-1] A + u (p.B),
//   gA = sum_t p exp(dt A) h[t-1] dt.
// The forward pass stores the state before every KEEP-th node; the backward march recomputes the
// states inside such a piece in registers and walks it backwards.
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr int THREADS = 128;
constexpr int WARPS = THREADS / 32;
constexpr int TILE = 32;          // nodes of a forward tile
constexpr int KEEP = 16;          // nodes between stored states = nodes of a backward tile
constexpr int NS = 4;             // states of a thread

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

// Sum over the S lanes of a channel of four values, one per node: lane q (of S) returns the sum of
// value q & 3 for S >= 4; S = 2: v[0], v[1] become the sums of values 2 (q & 1) and 2 (q & 1) + 1.
template <int S>
__device__ __forceinline__ void sum_lanes(float (&v)[4], int q) {
    if (S == 2) {
        const bool up = q & 1;
        const float s0 = up ? v[0] : v[2], s1 = up ? v[1] : v[3];
        v[0] = (up ? v[2] : v[0]) + __shfl_xor_sync(~0u, s0, 1);
        v[1] = (up ? v[3] : v[1]) + __shfl_xor_sync(~0u, s1, 1);
        return;
    }
    const bool hi = q & 2, up = q & 1;
    const float s0 = hi ? v[0] : v[2], s1 = hi ? v[1] : v[3];
    const float a = (hi ? v[2] : v[0]) + __shfl_xor_sync(~0u, s0, 2);
    const float b = (hi ? v[3] : v[1]) + __shfl_xor_sync(~0u, s1, 2);
    v[0] = (up ? b : a) + __shfl_xor_sync(~0u, up ? a : b, 1);
#pragma unroll
    for (int m = 4; m < S; m *= 2) v[0] += __shfl_xor_sync(~0u, v[0], m);
}

// Writes the sums that sum_lanes left for nodes k0 .. k0+3 of channel c.
template <int S, int CT>
__device__ __forceinline__ void put_sums(float (*dst)[CT], const float (&v)[4], int k0, int c, int q) {
    if (S == 2) {
        dst[k0 + 2 * (q & 1)][c] = v[0];
        dst[k0 + 2 * (q & 1) + 1][c] = v[1];
    } else if (S == 4 || q < 4) {
        dst[k0 + (q & 3)][c] = v[0];
    }
}

// ------------------------------------------------------------------------------------- chunk states
// BACK = false: local[b][chunk][channel][state] = state at the chunk's end when it starts from zero,
// sums[b][chunk][channel] = sum of dt.  BACK = true: local = what the adjoint state hands to the node
// before the chunk when nothing comes from behind it.
template <typename T, int S, bool BACK>
__global__ void __launch_bounds__(THREADS) scan_local_kernel(ScanIn<T> in, float* __restrict__ local, float* __restrict__ sums,
                                                             ScanShape s) {
    pdl_wait_then_trigger();
    constexpr int CT = THREADS / S, NP = S * NS;
    __shared__ float2 sd[TILE][CT];       // dt, dt u  (BACK: dt, gy)
    __shared__ float sb[TILE][NP];        // B (BACK: C)
    const Where w = where(s);
    const int tid = threadIdx.x, q = tid % S, cl = tid / S;
    const int c0 = w.tile * CT, c = c0 + cl;
    const int64_t first = (int64_t)w.chunk * s.chunk;
    const int64_t end = first + s.chunk < s.length ? first + s.chunk : s.length;
    float a2[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int n = q * NS + i;
        a2[i] = c < s.channels && n < s.states ? in.A[(int64_t)c * s.states + n] * LOG2_E : 0.f;
        h[i] = 0.f;
    }
    float total = 0.f;
    const int ntiles = (int)((end - first + TILE - 1) / TILE);
    for (int k = 0; k < ntiles; ++k) {
        const int64_t t0 = first + (int64_t)(BACK ? ntiles - 1 - k : k) * TILE;
        const int here = (int)(end - t0 < TILE ? end - t0 : TILE);
        __syncthreads();
        for (int e = tid; e < TILE * CT; e += THREADS) {
            const int r = e / CT, lc = e % CT, ch = c0 + lc;
            float2 v = make_float2(0.f, 0.f);
            if (r < here && ch < s.channels) {
                const int64_t t = t0 + r;
                const float raw = to_f32<T>(in.delta[w.b * s.delta_batch + t * s.delta_node + ch]) + (in.bias ? in.bias[ch] : 0.f);
                v.x = step_of(raw, s.softplus);
                if (BACK) {
                    float g = to_f32<T>(in.gout[w.b * s.g_batch + t * s.g_node + ch]);
                    if (in.z) {
                        const float z = to_f32<T>(in.z[w.b * s.z_batch + t * s.z_node + ch]);
                        g *= z * sigmoid_f32(z);
                    }
                    v.y = g;
                } else {
                    v.y = v.x * to_f32<T>(in.u[w.b * s.u_batch + t * s.u_node + ch]);
                }
            }
            sd[r][lc] = v;
        }
        for (int e = tid; e < TILE * NP; e += THREADS) {
            const int r = e / NP, n = e % NP;
            const bool there = r < here && n < s.states;
            sb[r][n] = !there ? 0.f
                     : BACK   ? to_f32<T>(in.C[w.b * s.C_batch + (t0 + r) * s.C_node + n])
                              : to_f32<T>(in.B[w.b * s.B_batch + (t0 + r) * s.B_node + n]);
        }
        __syncthreads();
#pragma unroll 4
        for (int k2 = 0; k2 < TILE; ++k2) {
            const int r = BACK ? TILE - 1 - k2 : k2;     // nodes past the end have dt = 0 and add nothing
            const float2 d = sd[r][cl];
            const float4 b4 = *reinterpret_cast<const float4*>(&sb[r][q * NS]);
            const float bb[NS] = {b4.x, b4.y, b4.z, b4.w};
            total += d.x;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const float a = exp2_f32(d.x * a2[i]);
                h[i] = BACK ? a * fmaf(d.y, bb[i], h[i]) : fmaf(a, h[i], d.y * bb[i]);
            }
        }
    }
    if (c < s.channels) {
        const int64_t at = (w.b * s.chunks + w.chunk) * s.channels + c;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (q * NS + i < s.states) local[at * s.states + q * NS + i] = h[i];
        if (q == 0) sums[at] = total;
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
    for (int k = 0; k < s.chunks; ++k) {
        const int64_t at = b * s.chunks + (BACK ? s.chunks - 1 - k : k);
        const float own = local[at * per + cn];
        const float keep = exp2_f32(a2 * sums[at * s.channels + c]);
        local[at * per + cn] = carry;
        carry = fmaf(keep, carry, own);
    }
}

// ------------------------------------------------------------------------------------------ forward
template <typename T, int S>
__global__ void __launch_bounds__(THREADS) scan_fwd_kernel(ScanIn<T> in, const float* __restrict__ state, const float* __restrict__ enter,
                                                           T* __restrict__ out, float* __restrict__ state_out, float* __restrict__ kept,
                                                           ScanShape s) {
    pdl_wait_then_trigger();
    constexpr int CT = THREADS / S, NP = S * NS, PER = TILE * CT / THREADS;
    __shared__ float2 sd[TILE][CT];
    __shared__ float sb[TILE][NP], sc[TILE][NP];
    __shared__ float sy[TILE][CT];
    const Where w = where(s);
    const int tid = threadIdx.x, q = tid % S, cl = tid / S;
    const int c0 = w.tile * CT, c = c0 + cl;
    const int64_t first = (int64_t)w.chunk * s.chunk;
    const int64_t end = first + s.chunk < s.length ? first + s.chunk : s.length;
    const int64_t per = (int64_t)s.channels * s.states;
    float a2[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int n = q * NS + i;
        const bool there = c < s.channels && n < s.states;
        a2[i] = there ? in.A[(int64_t)c * s.states + n] * LOG2_E : 0.f;
        h[i] = !there  ? 0.f
               : enter ? enter[(w.b * s.chunks + w.chunk) * per + (int64_t)c * s.states + n]
               : state ? state[w.b * per + (int64_t)c * s.states + n]
                       : 0.f;
    }
    for (int64_t t0 = first; t0 < end; t0 += TILE) {
        const int here = (int)(end - t0 < TILE ? end - t0 : TILE);
        float u[PER], z[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int e = tid + k * THREADS, r = e / CT, lc = e % CT, ch = c0 + lc;
            float2 v = make_float2(0.f, 0.f);
            u[k] = z[k] = 0.f;
            if (r < here && ch < s.channels) {
                const int64_t t = t0 + r;
                const float raw = to_f32<T>(in.delta[w.b * s.delta_batch + t * s.delta_node + ch]) + (in.bias ? in.bias[ch] : 0.f);
                u[k] = to_f32<T>(in.u[w.b * s.u_batch + t * s.u_node + ch]);
                if (in.z) z[k] = to_f32<T>(in.z[w.b * s.z_batch + t * s.z_node + ch]);
                v.x = step_of(raw, s.softplus);
                v.y = v.x * u[k];
            }
            sd[r][lc] = v;
        }
        for (int e = tid; e < TILE * NP; e += THREADS) {
            const int r = e / NP, n = e % NP;
            const bool there = r < here && n < s.states;
            sb[r][n] = there ? to_f32<T>(in.B[w.b * s.B_batch + (t0 + r) * s.B_node + n]) : 0.f;
            sc[r][n] = there ? to_f32<T>(in.C[w.b * s.C_batch + (t0 + r) * s.C_node + n]) : 0.f;
        }
        __syncthreads();
        for (int k0 = 0; k0 < TILE; k0 += 4) {       // nodes past the end have dt = 0: the state stays
            if (kept != nullptr && k0 % KEEP == 0 && k0 < here && c < s.channels) {
                float* dst = kept + ((w.b * s.kept_nodes + (t0 + k0) / KEEP) * s.channels + c) * s.states + q * NS;
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    if (q * NS + i < s.states) dst[i] = h[i];
            }
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 d = sd[k0 + k][cl];
                const float4 b4 = *reinterpret_cast<const float4*>(&sb[k0 + k][q * NS]);
                const float4 c4 = *reinterpret_cast<const float4*>(&sc[k0 + k][q * NS]);
                const float bb[NS] = {b4.x, b4.y, b4.z, b4.w}, cc[NS] = {c4.x, c4.y, c4.z, c4.w};
                y[k] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    h[i] = fmaf(exp2_f32(d.x * a2[i]), h[i], d.y * bb[i]);
                    y[k] = fmaf(cc[i], h[i], y[k]);
                }
            }
            sum_lanes<S>(y, q);
            put_sums<S, CT>(sy, y, k0, cl, q);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int e = tid + k * THREADS, r = e / CT, lc = e % CT, ch = c0 + lc;
            if (r < here && ch < s.channels) {
                float y = sy[r][lc];
                if (in.D) y = fmaf(in.D[ch], u[k], y);
                if (in.z) y *= z[k] * sigmoid_f32(z[k]);
                out[(w.b * s.length + t0 + r) * s.channels + ch] = from_f32<T>(y);
            }
        }
        // no barrier: the next tile writes sy only after its own first barrier, and sd, sb, sc were
        // last read before the barrier above
    }
    if (state_out != nullptr && w.chunk == s.chunks - 1 && c < s.channels) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (q * NS + i < s.states) state_out[w.b * per + (int64_t)c * s.states + q * NS + i] = h[i];
    }
}

// ----------------------------------------------------------------------------------------- backward
// part_bc[tile][b][t][2 NP]: this block's share of gB and gC; part_a[b][chunk][channel][states + 2]:
// this chunk's share of gA, gD and gdelta_bias.
template <typename T, int S>
__global__ void __launch_bounds__(THREADS) scan_bwd_kernel(ScanIn<T> in, const float* __restrict__ kept, const float* __restrict__ enter,
                                                           const float* __restrict__ gstate_out, T* __restrict__ gu, T* __restrict__ gdelta,
                                                           T* __restrict__ gz, float* __restrict__ gstate, float* __restrict__ part_bc,
                                                           float* __restrict__ part_a, int64_t rows, ScanShape s) {
    pdl_wait_then_trigger();
    constexpr int CT = THREADS / S, NP = S * NS, PER = KEEP * CT / THREADS;
    constexpr int CW = 32 / S;                     // channels of a warp
    __shared__ float2 sd[KEEP][CT];                // dt, dt u
    __shared__ float sg[KEEP][CT];                 // gy
    __shared__ float sb[KEEP][NP], sc[KEEP][NP];
    __shared__ float sy[KEEP][CT], st[KEEP][CT], sq[KEEP][CT];   // C.h, p.B, sum p a h A
    __shared__ float red[WARPS][KEEP][2 * NP];
    const Where w = where(s);
    const int tid = threadIdx.x, q = tid % S, cl = tid / S, warp = tid / 32, lane = tid % 32;
    const int c0 = w.tile * CT, c = c0 + cl;
    const int64_t first = (int64_t)w.chunk * s.chunk;
    const int64_t end = first + s.chunk < s.length ? first + s.chunk : s.length;
    const int64_t per = (int64_t)s.channels * s.states;
    float a2[NS], p[NS], ga[NS];                   // p: what the adjoint state brings from behind
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int n = q * NS + i;
        const bool there = c < s.channels && n < s.states;
        a2[i] = there ? in.A[(int64_t)c * s.states + n] * LOG2_E : 0.f;
        ga[i] = 0.f;
        p[i] = !there       ? 0.f
               : enter      ? enter[(w.b * s.chunks + w.chunk) * per + (int64_t)c * s.states + n]
               : gstate_out ? gstate_out[w.b * per + (int64_t)c * s.states + n]
                            : 0.f;
    }
    float gd = 0.f, gbias = 0.f;                   // of channel c0 + tid % CT
    const int ntiles = (int)((end - first + KEEP - 1) / KEEP);
    for (int k = ntiles - 1; k >= 0; --k) {
        const int64_t t0 = first + (int64_t)k * KEEP;
        const int here = (int)(end - t0 < KEEP ? end - t0 : KEEP);
        float u[PER], z[PER], go[PER], raw[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = tid + j * THREADS, r = e / CT, lc = e % CT, ch = c0 + lc;
            float2 v = make_float2(0.f, 0.f);
            float g = 0.f;
            u[j] = z[j] = go[j] = raw[j] = 0.f;
            if (r < here && ch < s.channels) {
                const int64_t t = t0 + r;
                raw[j] = to_f32<T>(in.delta[w.b * s.delta_batch + t * s.delta_node + ch]) + (in.bias ? in.bias[ch] : 0.f);
                u[j] = to_f32<T>(in.u[w.b * s.u_batch + t * s.u_node + ch]);
                go[j] = to_f32<T>(in.gout[w.b * s.g_batch + t * s.g_node + ch]);
                g = go[j];
                if (in.z) {
                    z[j] = to_f32<T>(in.z[w.b * s.z_batch + t * s.z_node + ch]);
                    g *= z[j] * sigmoid_f32(z[j]);
                }
                v.x = step_of(raw[j], s.softplus);
                v.y = v.x * u[j];
            }
            sd[r][lc] = v;
            sg[r][lc] = g;
        }
        for (int e = tid; e < KEEP * NP; e += THREADS) {
            const int r = e / NP, n = e % NP;
            const bool there = r < here && n < s.states;
            sb[r][n] = there ? to_f32<T>(in.B[w.b * s.B_batch + (t0 + r) * s.B_node + n]) : 0.f;
            sc[r][n] = there ? to_f32<T>(in.C[w.b * s.C_batch + (t0 + r) * s.C_node + n]) : 0.f;
        }
        __syncthreads();
        // forward through the tile: hs[r] is the state BEFORE node r
        float hs[KEEP + 1][NS];
#pragma unroll
        for (int i = 0; i < NS; ++i)
            hs[0][i] = c < s.channels && q * NS + i < s.states
                           ? kept[((w.b * s.kept_nodes + t0 / KEEP) * s.channels + c) * s.states + q * NS + i]
                           : 0.f;
#pragma unroll
        for (int k0 = 0; k0 < KEEP; k0 += 4) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = k0 + j;
                const float2 d = sd[r][cl];
                const float4 b4 = *reinterpret_cast<const float4*>(&sb[r][q * NS]);
                const float4 c4 = *reinterpret_cast<const float4*>(&sc[r][q * NS]);
                const float bb[NS] = {b4.x, b4.y, b4.z, b4.w}, cc[NS] = {c4.x, c4.y, c4.z, c4.w};
                y[j] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    hs[r + 1][i] = fmaf(exp2_f32(d.x * a2[i]), hs[r][i], d.y * bb[i]);
                    y[j] = fmaf(cc[i], hs[r + 1][i], y[j]);
                }
            }
            sum_lanes<S>(y, q);
            put_sums<S, CT>(sy, y, k0, cl, q);
        }
        // and backwards
#pragma unroll
        for (int k0 = KEEP - 4; k0 >= 0; k0 -= 4) {
            float tb[4], ta[4];
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                const int r = k0 + j;
                const float2 d = sd[r][cl];
                const float g = sg[r][cl];
                const float4 b4 = *reinterpret_cast<const float4*>(&sb[r][q * NS]);
                const float4 c4 = *reinterpret_cast<const float4*>(&sc[r][q * NS]);
                const float bb[NS] = {b4.x, b4.y, b4.z, b4.w}, cc[NS] = {c4.x, c4.y, c4.z, c4.w};
                float v[2 * NS];                   // shares of gB and gC of this node
                tb[j] = ta[j] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    p[i] = fmaf(cc[i], g, p[i]);
                    v[i] = p[i] * d.y;
                    v[NS + i] = hs[r + 1][i] * g;
                    tb[j] = fmaf(p[i], bb[i], tb[j]);
                    p[i] *= exp2_f32(d.x * a2[i]);
                    const float ph = p[i] * hs[r][i];
                    ta[j] = fmaf(ph, a2[i], ta[j]);
                    ga[i] = fmaf(ph, d.x, ga[i]);
                }
                // sum over the warp's channels: halve the values while halving the lanes, then add
                constexpr int TOP = 16;
                int at = 0;                        // first value this lane still holds
#pragma unroll
                for (int m = TOP, n = 2 * NS; m >= S; m /= 2) {
                    if (n > 1) {
                        n /= 2;
                        const bool up = lane & m;
#pragma unroll
                        for (int i = 0; i < n; ++i) {
                            const float send = up ? v[i] : v[n + i];
                            v[i] = (up ? v[n + i] : v[i]) + __shfl_xor_sync(~0u, send, m);
                        }
                        at += up ? n : 0;
                    } else {
                        v[0] += __shfl_xor_sync(~0u, v[0], m);
                    }
                }
                constexpr int LEFT = CW >= 2 * NS ? 1 : 2 * NS / CW;   // values left in a lane
#pragma unroll
                for (int i = 0; i < LEFT; ++i) {
                    const int n = at + i;
                    red[warp][r][(n / NS) * NP + q * NS + n % NS] = v[i];
                }
            }
            sum_lanes<S>(tb, q);
            put_sums<S, CT>(st, tb, k0, cl, q);
            sum_lanes<S>(ta, q);
            put_sums<S, CT>(sq, ta, k0, cl, q);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = tid + j * THREADS, r = e / CT, lc = e % CT, ch = c0 + lc;
            if (r < here && ch < s.channels) {
                const float dt = sd[r][lc].x, gy = sg[r][lc], through = st[r][lc];
                const float dd = in.D ? in.D[ch] : 0.f;
                const int64_t at = (w.b * s.length + t0 + r) * s.channels + ch;
                gu[at] = from_f32<T>(fmaf(dt, through, dd * gy));
                float gr = fmaf(u[j], through, sq[r][lc] * (1.f / LOG2_E));
                if (s.softplus) gr *= sigmoid_f32(raw[j]);
                gdelta[at] = from_f32<T>(gr);
                if (in.z) {
                    const float y = fmaf(dd, u[j], sy[r][lc]), sig = sigmoid_f32(z[j]);
                    gz[at] = from_f32<T>(go[j] * y * sig * fmaf(z[j], 1.f - sig, 1.f));
                }
                gd = fmaf(gy, u[j], gd);
                gbias += gr;
            }
        }
        for (int e = tid; e < here * 2 * NP; e += THREADS) {
            const int r = e / (2 * NP), n = e % (2 * NP);
            float v = 0.f;
#pragma unroll
            for (int k2 = 0; k2 < WARPS; ++k2) v += red[k2][r][n];
            part_bc[(((int64_t)w.tile * rows + w.b) * s.length + t0 + r) * (2 * NP) + n] = v;
        }
        __syncthreads();
    }
    // this chunk's share of the parameters' gradients
    float* pa = part_a + ((w.b * s.chunks + w.chunk) * s.channels) * (int64_t)(s.states + 2);
    if (c < s.channels) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (q * NS + i < s.states) {
                pa[(int64_t)c * (s.states + 2) + q * NS + i] = ga[i];
                if (gstate != nullptr && w.chunk == 0) gstate[w.b * per + (int64_t)c * s.states + q * NS + i] = p[i];
            }
    }
    // threads tid, tid + CT, ... hold the same channel's sums
    static_assert(KEEP * CT >= THREADS, "room for two sums of every thread");
    float* fin = &sd[0][0].x;
    fin[tid] = gd;
    fin[THREADS + tid] = gbias;
    __syncthreads();
    if (tid < CT && c0 + tid < s.channels) {
        float v0 = 0.f, v1 = 0.f;
        for (int e = tid; e < THREADS; e += CT) { v0 += fin[e]; v1 += fin[THREADS + e]; }
        pa[(int64_t)(c0 + tid) * (s.states + 2) + s.states] = v0;
        pa[(int64_t)(c0 + tid) * (s.states + 2) + s.states + 1] = v1;
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
// S lanes share a channel, four states each; state_out may be state.
template <typename T, int S>
__global__ void __launch_bounds__(THREADS) scan_step_kernel(ScanIn<T> in, const float* state, T* __restrict__ out, float* state_out,
                                                            int64_t rows, ScanShape s) {
    pdl_wait_then_trigger();
    const int64_t e = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / S;
    const int q = threadIdx.x % S;
    const bool there = e < rows * s.channels;
    const int64_t b = there ? e / s.channels : 0;
    const int c = there ? (int)(e % s.channels) : 0;
    float y = 0.f, u = 0.f;
    if (there) {
        const float dt = step_of(to_f32<T>(in.delta[b * s.delta_batch + c]) + (in.bias ? in.bias[c] : 0.f), s.softplus);
        u = to_f32<T>(in.u[b * s.u_batch + c]);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int n = q * NS + i;
            if (n < s.states) {
                const float h0 = state ? state[e * s.states + n] : 0.f;
                const float h = fmaf(exp2_f32(dt * (in.A[(int64_t)c * s.states + n] * LOG2_E)), h0,
                                     dt * u * to_f32<T>(in.B[b * s.B_batch + n]));
                y = fmaf(to_f32<T>(in.C[b * s.C_batch + n]), h, y);
                if (state_out != nullptr) state_out[e * s.states + n] = h;
            }
        }
    }
#pragma unroll
    for (int m = 1; m < S; m *= 2) y += __shfl_xor_sync(~0u, y, m);
    if (there && q == 0) {
        if (in.D) y = fmaf(in.D[c], u, y);
        if (in.z) {
            const float z = to_f32<T>(in.z[b * s.z_batch + c]);
            y *= z * sigmoid_f32(z);
        }
        out[e] = from_f32<T>(y);
    }
}

// --------------------------------------------------------------------------------------------- host
int lanes_of(int states) {
    int s = 2;
    while (s * NS < states) s *= 2;
    return s;
}

// The plan depends on sizes only, so that the forward and the backward call agree on it.
ScanShape plan(const fpde_scan_args* a, bool backward) {
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
    s.tiles = (int)ceil_div(a->channels, THREADS / lanes_of(a->states));
    s.kept_nodes = ceil_div(a->length, KEEP);
    // Splitting a row costs a second pass over its exponentials: done while it still fills idle SMs.
    const int64_t blocks = a->batch * s.tiles;
    const int64_t want = 148 * (backward ? 3 : 6);
    int64_t chunks = 1;
    if (blocks * 2 <= want) chunks = want / (blocks > 0 ? blocks : 1);
    int64_t chunk = ceil_div(ceil_div(a->length > 0 ? a->length : 1, chunks), TILE) * TILE;
    if (chunk < 2 * TILE) chunk = 2 * TILE;
    if (chunk > (1 << 30)) chunk = 1 << 30;
    s.chunk = (int)chunk;
    s.chunks = (int)ceil_div(a->length > 0 ? a->length : 1, chunk);
    return s;
}

int check_scan(const fpde_scan_args* a, bool step) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->states < 1 || a->states > FPDE_SCAN_MAX_STATES) return FPDE_ERR_PARAM;
    if (a->batch < 0 || a->channels < 0 || a->length < 0 || a->channels > (1 << 24) || a->length > (1ll << 36) || a->batch > (1ll << 36))
        return FPDE_ERR_SHAPE;
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

template <typename T, int S>
cudaError_t run_fwd(const fpde_scan_args* a, cudaStream_t st) {
    const ScanShape s = plan(a, false);
    const ScanSpace w = space(a, s, false);
    const ScanIn<T> in = inputs<T>(a);
    const int64_t blocks = a->batch * s.tiles * s.chunks;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    float* local = nullptr;
    if (s.chunks > 1) {
        local = (float*)((char*)a->workspace + w.local);
        float* sums = (float*)((char*)a->workspace + w.sums);
        FPDE_TRY(launch_kernel(scan_local_kernel<T, S, false>, dim3((unsigned)blocks), dim3(THREADS), st, in, local, sums, s));
        FPDE_TRY(launch_kernel(scan_join_kernel<false>, dim3((unsigned)ceil_div(a->batch * s.channels * s.states, 256)), dim3(256), st,
                               local, (const float*)sums, a->A, a->state, a->batch, s));
    }
    return launch_kernel(scan_fwd_kernel<T, S>, dim3((unsigned)blocks), dim3(THREADS), st, in, a->state, (const float*)local, (T*)a->out,
                         a->state_out, (float*)a->kept, s);
}

template <typename T, int S>
cudaError_t run_bwd(const fpde_scan_args* a, cudaStream_t st) {
    const ScanShape s = plan(a, true);
    const ScanSpace w = space(a, s, true);
    const ScanIn<T> in = inputs<T>(a);
    const int64_t blocks = a->batch * s.tiles * s.chunks;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    char* ws = (char*)a->workspace;
    float *local = nullptr, *part_bc = (float*)(ws + w.part_bc), *part_a = (float*)(ws + w.part_a);
    if (s.chunks > 1) {
        local = (float*)(ws + w.local);
        float* sums = (float*)(ws + w.sums);
        FPDE_TRY(launch_kernel(scan_local_kernel<T, S, true>, dim3((unsigned)blocks), dim3(THREADS), st, in, local, sums, s));
        FPDE_TRY(launch_kernel(scan_join_kernel<true>, dim3((unsigned)ceil_div(a->batch * s.channels * s.states, 256)), dim3(256), st,
                               local, (const float*)sums, a->A, a->gstate_out, a->batch, s));
    }
    FPDE_TRY(launch_kernel(scan_bwd_kernel<T, S>, dim3((unsigned)blocks), dim3(THREADS), st, in, (const float*)a->kept, (const float*)local,
                           a->gstate_out, (T*)a->gu, (T*)a->gdelta, (T*)a->gz, a->gstate, part_bc, part_a, a->batch, s));
    if (a->batch * a->length > 0)
        FPDE_TRY(launch_kernel(scan_sum_bc_kernel<T>, dim3((unsigned)ceil_div(a->batch * a->length * 2 * S * NS, 256)), dim3(256), st,
                               (const float*)part_bc, s.tiles, a->batch * a->length, S * NS, s.states, (T*)a->gB, (T*)a->gC));
    return launch_kernel(scan_sum_a_kernel, dim3((unsigned)ceil_div((int64_t)s.channels * (s.states + 2), 32)), dim3(32, 8), st,
                         (const float*)part_a, a->batch * s.chunks, s.channels, s.states, a->gA, a->gD, a->gdelta_bias);
}

template <typename T, int S>
cudaError_t run_step(const fpde_scan_args* a, cudaStream_t st) {
    const ScanShape s = plan(a, false);
    const int64_t blocks = ceil_div(a->batch * s.channels * S, THREADS);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(scan_step_kernel<T, S>, dim3((unsigned)blocks), dim3(THREADS), st, inputs<T>(a), a->state, (T*)a->out, a->state_out,
                         a->batch, s);
}

enum Call { CALL_FWD, CALL_BWD, CALL_STEP };

template <typename T, int S>
cudaError_t run(const fpde_scan_args* a, Call call, cudaStream_t st) {
    if (call == CALL_FWD) return run_fwd<T, S>(a, st);
    if (call == CALL_BWD) return run_bwd<T, S>(a, st);
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
    if (check_scan(a, false) != FPDE_OK) return 0;
    return (size_t)(a->batch * ceil_div(a->length, KEEP) * a->channels * a->states) * 4;
}

size_t fpde_selective_scan_workspace_bytes(const fpde_scan_args* a, int backward) {
    if (check_scan(a, false) != FPDE_OK) return 0;
    return space(a, plan(a, backward != 0), backward != 0).total;
}

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
