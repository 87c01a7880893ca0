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

template <int DA, int DC>
struct Sizes {
    static constexpr int PA = DA + 4, PC = DC + 4, PP = C + 4;
    static constexpr size_t BYTES = sizeof(float) * (2 * C * PA + C * PC + DA * PC + C * PP);
};

template <typename T, int W, int P>
__device__ __forceinline__ void load_rows(float* to, const T* from, int64_t stride, int rows, int cols) {
    for (int i = threadIdx.x; i < C * W; i += THREADS) {
        const int r = i / W, c = i % W;
        to[r * P + c] = r < rows && c < cols ? to_f32<T>(from[r * stride + c]) : 0.f;
    }
}

// One piece of a row and head and DC features of c.  ENDS: only the state that the piece leaves, from zero.
template <typename T, int DA, int DC, bool ENDS>
__global__ void __launch_bounds__(THREADS) march_kernel(March m) {
    using Z = Sizes<DA, DC>;
    extern __shared__ __align__(16) float smem[];
    float *sa = smem, *sb = sa + C * Z::PA, *sc = sb + C * Z::PA, *ss = sc + C * Z::PC, *sp = ss + DA * Z::PC;
    __shared__ float powers[C + 2];
    __shared__ float whole[2];
    pdl_wait_then_trigger();
    const int tid = threadIdx.x;
    const int across = (m.dc + DC - 1) / DC;
    int64_t id = blockIdx.x;
    const int c0 = (int)(id % across) * DC;
    id /= across;
    const int p = (int)(id % m.pieces);
    id /= m.pieces;
    const int64_t h = id % m.heads, bt = id / m.heads;
    const int cols = min(DC, m.dc - c0);
    const float ld = m.log_decay[h];
    if (tid < C + 2) powers[tid] = (float)power(ld, tid);
    const int64_t first = p * m.piece, last = min(m.length, first + m.piece);
    const int64_t st = (bt * m.heads + h) * m.da * m.dc;
    float* local = m.local + ((bt * m.heads + h) * m.pieces + p) * m.da * m.dc;
    for (int i = tid; i < DA * DC; i += THREADS) {
        const int r = i / DC, c = i % DC;
        float v = 0.f;
        if (!ENDS && r < m.da && c < cols) {
            if (m.pieces > 1) v = local[r * m.dc + c0 + c];
            else if (m.start != nullptr) v = m.start_turned ? m.start[st + (int64_t)(c0 + c) * m.da + r] : m.start[st + r * m.dc + c0 + c];
        }
        ss[r * Z::PC + c] = v;
    }
    const T* a = (const T*)m.a.p + bt * m.a.batch + h * m.a.head;
    const T* b = (const T*)m.b.p + bt * m.b.batch + h * m.b.head;
    const T* cc = (const T*)m.c.p + bt * m.c.batch + h * m.c.head + c0;
    constexpr int GC = DC / 4, GR = THREADS / GC;          // threads along the columns and the rows of a result
    constexpr int RO = C / GR, RS = DA / GR;               // rows of a thread
    const int tc = tid % GC * 4, tr = tid / GC;
    for (int64_t t = first; t < last; t += C) {
        const int n = (int)min((int64_t)C, last - t);
        const int64_t node = m.reversed ? m.length - 1 - t : t;
        const int64_t dir = m.reversed ? -1 : 1;
        __syncthreads();
        if (!ENDS) load_rows<T, DA, Z::PA>(sa, a + node * m.a.node, dir * m.a.node, n, m.da);
        load_rows<T, DA, Z::PA>(sb, b + node * m.b.node, dir * m.b.node, n, m.da);
        load_rows<T, DC, Z::PC>(sc, cc + node * m.c.node, dir * m.c.node, n, cols);
        if (tid == 0) {
            const double g = power(ld, n);
            whole[0] = (float)g;
            whole[1] = (float)(g - (float)g);
        }
        __syncthreads();
        if (!ENDS) {
            // (a_i . b_j), 2 x 4 a thread, with the decay between the nodes
            const int j0 = tid % 8, i0 = tid / 8 * 2;
            float s[2][4] = {};
            for (int d = 0; d < DA; d += 4) {
                float4 x[2], y[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) x[i] = *reinterpret_cast<const float4*>(sa + (i0 + i) * Z::PA + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(sb + (j0 + 8 * j) * Z::PA + d);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, s[i][j]))));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int back = i0 + i - (j0 + 8 * j);
                    sp[(i0 + i) * Z::PP + j0 + 8 * j] = back < 0 ? 0.f : m.near * powers[back] * s[i][j];
                }
            __syncthreads();
            float o[RO][4] = {};
            for (int d = 0; d < DA; d += 4) {
                float4 y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = *reinterpret_cast<const float4*>(ss + (d + e) * Z::PC + tc);
#pragma unroll
                for (int i = 0; i < RO; ++i) {
                    const float4 x = *reinterpret_cast<const float4*>(sa + (tr * RO + i) * Z::PA + d);
                    const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[i][0] = fmaf(xs[e], y[e].x, o[i][0]);
                        o[i][1] = fmaf(xs[e], y[e].y, o[i][1]);
                        o[i][2] = fmaf(xs[e], y[e].z, o[i][2]);
                        o[i][3] = fmaf(xs[e], y[e].w, o[i][3]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RO; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] *= m.far * powers[tr * RO + i + 1 - m.shift];
            for (int j = 0; j < (tr + 1) * RO; ++j) {      // rows behind a node are not looked at: they may hold anything
                const float4 y = *reinterpret_cast<const float4*>(sc + j * Z::PC + tc);
#pragma unroll
                for (int i = 0; i < RO; ++i) {
                    if (j > tr * RO + i) continue;
                    const float x = sp[(tr * RO + i) * Z::PP + j];
                    o[i][0] = fmaf(x, y.x, o[i][0]);
                    o[i][1] = fmaf(x, y.y, o[i][1]);
                    o[i][2] = fmaf(x, y.z, o[i][2]);
                    o[i][3] = fmaf(x, y.w, o[i][3]);
                }
            }
#pragma unroll
            for (int i = 0; i < RO; ++i) {
                const int r = tr * RO + i;
                if (r >= n) continue;
                T* to = (T*)m.out + ((bt * m.length + node + dir * r) * m.heads + h) * m.dc + c0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (tc + e < cols) to[tc + e] = from_f32<T>(o[i][e]);
            }
            __syncthreads();
        }
        float u[RS][4] = {};
        for (int j = 0; j < n; ++j) {
            const float w = m.gain * powers[n - 1 - j + m.shift];
            float4 y = *reinterpret_cast<const float4*>(sc + j * Z::PC + tc);
#pragma unroll
            for (int i = 0; i < RS; ++i) {
                const float x = sb[j * Z::PA + tr * RS + i] * w;
                u[i][0] = fmaf(x, y.x, u[i][0]);
                u[i][1] = fmaf(x, y.y, u[i][1]);
                u[i][2] = fmaf(x, y.z, u[i][2]);
                u[i][3] = fmaf(x, y.w, u[i][3]);
            }
        }
#pragma unroll
        for (int i = 0; i < RS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float& v = ss[(tr * RS + i) * Z::PC + tc + e];
                v = fmaf(whole[0], v, fmaf(whole[1], v, u[i][e]));
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

// Eight pieces at a time, so that their loads are on their way together.
__global__ void __launch_bounds__(256) join_kernel(March m) {
    pdl_wait_then_trigger();
    const int64_t size = (int64_t)m.da * m.dc, across = (size + 255) / 256;
    const int64_t i = blockIdx.x % across * 256 + threadIdx.x, row = blockIdx.x / across;
    if (i >= size) return;
    const double g = power(m.log_decay[row % m.heads], (double)m.piece);
    const float hi = (float)g, lo = (float)(g - hi);
    float s = 0.f;
    if (m.start != nullptr) s = m.start[row * size + (m.start_turned ? i % m.dc * m.da + i / m.dc : i)];
    float* at = m.local + row * m.pieces * size + i;
    for (int p = 0; p < m.pieces; p += 8, at += 8 * size) {
        float u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = p + e < m.pieces ? at[e * size] : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p + e < m.pieces) at[e * size] = s;
            s = fmaf(hi, s, fmaf(lo, s, u[e]));
        }
    }
}

// One node of every row and head.  A block takes one head's state: LX lanes of V columns each, the rows over the
// rest of its threads, whose shares of the output are summed in shared memory.
constexpr int STEP_THREADS = 256;
template <typename T, int V>
__global__ void __launch_bounds__(STEP_THREADS) linear_step_kernel(LinearView q, LinearView k, LinearView v, const float* __restrict__ log_decay,
                                                                   const float* state, float* state_out, T* __restrict__ o, int heads, int dk, int dv,
                                                                   int lx, float scale) {
    __shared__ float sq[FPDE_LINEAR_MAX_DIM], sk[FPDE_LINEAR_MAX_DIM], part[STEP_THREADS * V];
    pdl_wait_then_trigger();
    const int64_t row = blockIdx.x, b = row / heads;
    const int h = (int)(row - b * heads), tid = threadIdx.x;
    if (tid < dk) {
        sq[tid] = to_f32<T>(((const T*)q.p)[b * q.batch + h * q.head + tid]) * scale;
        sk[tid] = to_f32<T>(((const T*)k.p)[b * k.batch + h * k.head + tid]);
    }
    const float g = expf(log_decay[h]);
    const int x = tid % lx, y = tid / lx, rows = STEP_THREADS / lx, c = x * V;
    const bool in = c < dv;
    float val[V];
    if (in)
        for (int e = 0; e < V; ++e) val[e] = to_f32<T>(((const T*)v.p)[b * v.batch + h * v.head + c + e]);
    __syncthreads();
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
                s[e] = fmaf(g, s[e], sk[d] * val[e]);
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

// Rows of up to 64 nodes fill less than half of a chunk there.
bool on_tensor_cores(const fpde_linear_args* a) { return a->dtype == FPDE_BF16 && a->length > 64; }

// Pieces of a row.  With more than one every piece is marched through twice, the first time for its end alone (ENDS of the
// time); a block's start costs as much as START chunks.  The number that takes the fewest waves of chunks is taken.
void cut(const fpde_linear_args* a, March& m) {
    const bool mma = on_tensor_cores(a);
    const int chunk = mma ? MMA_CHUNK : C;
    const double ends = 0.5, start = 1.;
    const int64_t rows = m.batch * m.heads * (mma ? 1 : ceil_div(m.dc, 64)), slots = mma ? march_mma_blocks() : 148 * 4, chunks = ceil_div(m.length, chunk);
    int64_t best = 1;
    double least = 1e300;
    for (int64_t p = 1; p <= chunks && p <= 1024 && rows * (p - 1) < 8 * slots; ++p) {
        const int64_t each = ceil_div(chunks, p);
        if (ceil_div(chunks, each) != p) continue;
        const double waves = (double)ceil_div(rows * p, slots), time = waves * (p > 1 ? (start + each) * (1. + ends) + 2. : start + each);
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
    cut(a, m);
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
    cut(a, m);
    return m;
}
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
    m.start_turned = 1;
    m.out = a->gk;
    cut(a, m);
    return m;
}
March march_gv(const fpde_linear_args* a) {
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
    cut(a, m);
    return m;
}

#define FPDE_TRY(x)                           \
    do {                                      \
        const cudaError_t e_ = (x);           \
        if (e_ != cudaSuccess) return e_;     \
    } while (0)

template <typename T, int DA, int DC>
cudaError_t march_launch(const March& m, cudaStream_t st) {
    const size_t bytes = Sizes<DA, DC>::BYTES;
    const int64_t blocks = m.batch * m.heads * m.pieces * ceil_div(m.dc, DC);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    if (m.pieces > 1) {
        static std::atomic<uint64_t> done{0};
        FPDE_TRY(allow_smem(march_kernel<T, DA, DC, true>, bytes, done));
        FPDE_TRY(launch_kernel_smem(march_kernel<T, DA, DC, true>, dim3((unsigned)blocks), dim3(THREADS), bytes, st, m));
        FPDE_TRY(march_join(m, st));
    }
    static std::atomic<uint64_t> done{0};
    FPDE_TRY(allow_smem(march_kernel<T, DA, DC, false>, bytes, done));
    return launch_kernel_smem(march_kernel<T, DA, DC, false>, dim3((unsigned)blocks), dim3(THREADS), bytes, st, m);
}

template <typename T>
cudaError_t march_run(const March& m, cudaStream_t st) {
    if (m.dc <= 32) return m.da <= 32 ? march_launch<T, 32, 32>(m, st) : m.da <= 64 ? march_launch<T, 64, 32>(m, st) : march_launch<T, 128, 32>(m, st);
    return m.da <= 32 ? march_launch<T, 32, 64>(m, st) : m.da <= 64 ? march_launch<T, 64, 64>(m, st) : march_launch<T, 128, 64>(m, st);
}

cudaError_t march_by_type(const fpde_linear_args* a, const March& m, cudaStream_t st) {
    cudaError_t e;
    if (on_tensor_cores(a) && march_mma(m, st, &e)) return e;
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
    const int64_t blocks = m.batch * m.heads * ceil_div((int64_t)m.da * m.dc, 256);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(join_kernel, dim3((unsigned)blocks), dim3(256), st, m);
}

}  // namespace fpde

using namespace fpde;

extern "C" {

size_t fpde_linear_attention_workspace_bytes(const fpde_linear_args* a, int backward) {
    if (check_linear_sizes(a) != FPDE_OK) return 0;
    if (!backward) return local_bytes(march_o(a));
    const size_t q = local_bytes(march_gq(a)), k = local_bytes(march_gk(a)), v = local_bytes(march_gv(a));
    return q > k ? (q > v ? q : v) : (k > v ? k : v);
}

static int check_workspace(const fpde_linear_args* a, int backward) {
    const size_t need = fpde_linear_attention_workspace_bytes(a, backward);
    return need > 0 && (a->workspace == nullptr || !aligned(a->workspace, 16) || a->workspace_bytes < need) ? FPDE_ERR_WORKSPACE : FPDE_OK;
}

int fpde_linear_attention_fwd(const fpde_linear_args* a, void* stream) {
    int st = check_linear(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->heads == 0) return FPDE_OK;
    if (a->o == nullptr && a->length > 0) return FPDE_ERR_NULL;
    if (a->state != nullptr && a->state == a->state_out) return FPDE_ERR_PARAM;      // blocks still read it
    if ((st = check_workspace(a, 0)) != FPDE_OK) return st;
    return as_status(march_by_type(a, march_o(a), (cudaStream_t)stream));
}

int fpde_linear_attention_bwd(const fpde_linear_args* a, void* stream) {
    int st = check_linear(a, false);
    if (st != FPDE_OK) return st;
    if (a->batch * a->heads == 0) return FPDE_OK;
    if (a->length > 0 && (a->go == nullptr || a->gq == nullptr || a->gk == nullptr || a->gv == nullptr)) return FPDE_ERR_NULL;
    if (a->gstate != nullptr && a->gstate == a->gstate_out) return FPDE_ERR_PARAM;
    if ((st = check_workspace(a, 1)) != FPDE_OK) return st;
    const cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = march_by_type(a, march_gq(a), s);
    if (e == cudaSuccess) e = march_by_type(a, march_gk(a), s);
    if (e == cudaSuccess) e = march_by_type(a, march_gv(a), s);
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

unsigned int fpde_diag_linear_timeouts(void) { return march_mma_timeouts(); }

}  // extern "C"
