// Orthogonalised update of a stack of matrices by Newton-Schulz products, and the optimiser's whole
// step around it.
//
//   X = U / (|U| + eps);  `steps` times:  S = X X^T,  P = b S + c S S,  X <- a X + P X
// on the shorter side (taller matrices are turned on the way in and back on the way out).
//
// Per step m^2 (m + 3 n) multiplications and additions are needed with the symmetry of S and S S, m <= n.
// 4096^2 bf16, 5 steps: 1.37e12, 831 us at the measured bf16 rate, measured 1.22 ms in short runs and 1.44 to 1.48 at the clock of
// a loaded GPU (a step 231 us; its products 66, 65 and 113 under a profiler, the last, which has no symmetry, at 1216
// TFLOP/s; the passes around them 68 us).  Four fp32 1000 x 333 steps of the optimiser: 172 us, small products that are
// bound by latency.  Eight fp32 128 x 128 matrices: 37 us, 9 around the steps and 5.5 a step.
#include <type_traits>

#include "mma_common.cuh"
#include "seq_common.cuh"

namespace fpde {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.775f, NS_C = 2.0315f;
constexpr float SCALE = 16384.f;    // 2^14: matrices are stored times this, see the products
constexpr int MOST_SUMS = 256;      // blocks that sum the squares of one matrix, at most

// What the matrices are read from and written to.
struct OrthoIo {
    const void* grad;
    int64_t grad_matrix, grad_row;
    void* out;          // orthogonalize: result;  muon: weight
    float* momentum;    // muon only
    int rows, cols, m, n, mp, np;   // m <= n: the sides of X; mp, np padded
    bool turned, nesterov, wide;   // wide: eight neighbours of a row can be moved together
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

template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T* p) {
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        const Pack<T, N> k = load_pack<T, N>(p + i);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i + j] = to_f32<T>(k.v[j]);
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        Pack<T, N> k;
#pragma unroll
        for (int j = 0; j < N; ++j) k.v[j] = from_f32<T>(v[i + j]);
        *reinterpret_cast<Pack<T, N>*>(p + i) = k;
    }
}
// Eight neighbours of update_at (io.wide).
template <typename T>
__device__ __forceinline__ void update8(float (&v)[8], const OrthoIo& io, int64_t k, int64_t r, int64_t c) {
    load8<T>(v, (const T*)io.grad + k * io.grad_matrix + r * io.grad_row + c);
    if (io.momentum == nullptr) return;
    float m[8];
    load8<float>(m, io.momentum + (k * io.rows + r) * io.cols + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = io.nesterov ? fmaf(io.decay, m[i], v[i]) : m[i];
}

// Moves the momentum on (muon) and leaves each block's sum of squares of the update, in 64 bits: the
// squares of gradients of any scale fit.  A warp takes whole rows, `blocks` blocks share a matrix.
template <typename T>
__global__ void __launch_bounds__(256) ortho_square_kernel(OrthoIo io, double* __restrict__ sums, int blocks, unsigned int* lost) {
    pdl_wait_then_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *lost = 0;
    __shared__ double part[8];
    const int k = blockIdx.x / blocks, lane = threadIdx.x % 32;
    const float decay = io.decay;
    double v = 0.0;
    for (int r = (blockIdx.x % blocks) * 8 + threadIdx.x / 32; r < io.rows; r += blocks * 8) {
        const T* g = (const T*)io.grad + k * io.grad_matrix + r * io.grad_row;
        float* mom = io.momentum ? io.momentum + ((int64_t)k * io.rows + r) * io.cols : nullptr;
        if (io.wide) {
#pragma unroll 4
            for (int c = lane * 8; c < io.cols; c += 256) {
                float u[8];
                load8<T>(u, g + c);
                if (mom != nullptr) {
                    float next[8];
                    load8<float>(next, mom + c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        next[i] = fmaf(decay, next[i], u[i]);
                        u[i] = io.nesterov ? fmaf(decay, next[i], u[i]) : next[i];
                    }
                    store8<float>(mom + c, next);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v += (double)u[i] * u[i];
            }
            continue;
        }
#pragma unroll 8
        for (int c = lane; c < io.cols; c += 32) {
            float u = to_f32<T>(g[c]);
            if (mom != nullptr) {
                const float next = fmaf(decay, mom[c], u);
                mom[c] = next;
                u = io.nesterov ? fmaf(decay, next, u) : next;
            }
            v += (double)u * u;
        }
    }
#pragma unroll
    for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(~0u, v, m);
    if (lane == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += part[i];
        sums[blockIdx.x] = v;
    }
}

// What makes the first X of U: 2^14 / (|U| + eps), in two factors.  The first is a power of two, and 1 unless the whole
// nears the ends of fp32's range (norms below 1.3e-26 or above 2.1e34, which fp32 and bf16 gradients can have: with eps = 0
// the single factor overflowed below 5e-35, and lost digits above 1.4e42).
struct Fit {
    float first, second;
    Fit() = default;
    __device__ __forceinline__ Fit(double norm, double eps) {
        const double whole = (double)SCALE / (norm + eps);
        const int side = whole > 0x1p100 ? 1 : whole < 0x1p-100 ? -1 : 0;
        first = side > 0 ? 0x1p100f : side < 0 ? 0x1p-100f : 1.f;
        second = (float)(side > 0 ? whole * 0x1p-100 : side < 0 ? whole * 0x1p100 : whole);
    }
    __device__ __forceinline__ float operator()(float v) const { return v * first * second; }
};

// The same from the blocks' sums of squares (at most 256), added in the same order by every block that asks.
__device__ __forceinline__ Fit fit_of(const double* sums, int blocks, double eps, double (&part)[8]) {
    double v = threadIdx.x < blocks ? sums[threadIdx.x] : 0.0;
#pragma unroll
    for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(~0u, v, m);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += part[i];
    return Fit(sqrt(v), eps);
}

// Eight values of a row, already scaled, as hi and lo halves.
__device__ __forceinline__ void split8(const float (&v)[8], Pack<__half, 8>& hi, Pack<__half, 8>& lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi.v[i] = __float2half_rn(v[i]);
        lo.v[i] = __float2half_rn(v[i] - __half2float(hi.v[i]));
    }
}

// The first X (m x n, padded to mp x np) of every matrix, turned where the matrix is taller than wide.
// A block moves 64 x 64 elements through shared memory: read along the matrix's rows, written along X's.
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(OrthoIo io, const double* __restrict__ sums, int blocks, __half* __restrict__ x) {
    pdl_wait_then_trigger();
    __shared__ float tile[64][65];
    __shared__ double part[8];
    const int across = io.np / 64, down = io.mp / 64;
    const int k = blockIdx.x / (across * down), t = blockIdx.x % (across * down), i0 = t / across * 64, j0 = t % across * 64;
    const int r0 = io.turned ? j0 : i0, c0 = io.turned ? i0 : j0;
    // the elements are on their way while the norm is added up
    Fit fit;
    if (io.wide) {
        float in[2][8];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int r = threadIdx.x / 8 + q * 32, c = threadIdx.x % 8 * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) in[q][i] = 0.f;
            if (r0 + r < io.rows && c0 + c < io.cols) update8<T>(in[q], io, k, r0 + r, c0 + c);
        }
        fit = fit_of(sums + (int64_t)k * blocks, blocks, io.eps, part);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) tile[threadIdx.x / 8 + q * 32][threadIdx.x % 8 * 8 + i] = in[q][i];
    } else {
        float in[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int r = threadIdx.x / 64 + q * 4, c = threadIdx.x % 64;
            in[q] = r0 + r < io.rows && c0 + c < io.cols ? update_at<T>(io, k, r0 + r, c0 + c) : 0.f;
        }
        fit = fit_of(sums + (int64_t)k * blocks, blocks, io.eps, part);
#pragma unroll
        for (int q = 0; q < 16; ++q) tile[threadIdx.x / 64 + q * 4][threadIdx.x % 64] = in[q];
    }
    __syncthreads();
    const int64_t plane = (int64_t)io.mp * io.np;
#pragma unroll
    for (int e = threadIdx.x; e < 64 * 8; e += 256) {
        const int i = e / 8, j = e % 8 * 8;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {       // padding stays zero, whatever the norm is
            const bool there = i0 + i < io.m && j0 + j + q < io.n;
            v[q] = there ? fit(io.turned ? tile[j + q][i] : tile[i][j + q]) : 0.f;
        }
        Pack<__half, 8> hi, lo;
        split8(v, hi, lo);
        Pack<__half, 8>* p = reinterpret_cast<Pack<__half, 8>*>(x + 2 * k * plane + (int64_t)(i0 + i) * io.np + j0 + j);
        p[0] = hi;
        p[plane / 8] = lo;
    }
}

// ------------------------------------------------------------------------------------------ products
// One product of the iteration over all matrices of the stack, on the tensor cores:
//   GRAM    S  = X X^T              SQUARE  P = b S + c S S             APPLY  X' = a X + P X
//
// Every matrix is held as two fp16 planes, hi and lo, of the value times 2^14: hi is the value rounded to
// 11 bits, lo the next 11 bits of what is left.  The entries are at most 1.21 (X), 1.45 (S) or 2.81 (P) in size
// (the quintic takes no singular value past 1.2025),
// so the scaled hi stays below 65504, and 2^14 keeps lo above fp16's smallest numbers for entries down to
// 2^-16.  With PAIR three products (hi hi, hi lo, lo hi) go into one fp32 accumulator: 22-bit factors.
// Without it only hi hi is formed, and lo serves the terms a X and b S that are added in the epilogue.
//
// The cross products have an accumulator of their own: every product rounds the running sum towards zero,
// and the large sum then sees a third of the roundings; with 64-column tiles, where TMEM has the room, it
// is split in two as well (40 x 900 fp32, S over 57 products: error 6.3e-6 before, 2.7e-6 after; plain fp32
// 2.7e-6).  And with PAIR the sums leave the accumulators every SEGMENT slices, to be added up in fp32 with
// ordinary rounding: 33 x 70001 fp32 was 1.2e-4 off in one run of products.
//
// S and P are symmetric: where their tiles fill the GPU, only those on and below the diagonal are
// computed, and stored twice; where they do not, computing all of them is faster than storing twice.
//
// A block is persistent and has one warp that loads (TMA into a ring of 64-deep slices, 128-byte
// swizzle), one that issues tcgen05.mma (accumulators in TMEM, two sets, so that a tile's epilogue runs
// under the next tile's products) and eight that turn the sums into the next operand.  X enters APPLY as
// it is stored, rows along k: its slices are MN-major operands.  The planes are padded to multiples of
// 64 with zeros.
//
// Large products run on pairs of SMs (CG = 2, cta_group::2): a tile has 256 rows, each block of the pair
// loads its 128 rows of the left factor and half of the right one, and the first block issues for both.
// What a block has to load per product is what bounds the one-block form (an SM takes 64 bytes a clock
// from L2; 128 x 256 tiles need 96).  Pairs bring 8.6, 9.3 and 10.1e12 bytes a second out of L2 in the three products of
// 4096 x 4096, with the tensor pipe 68, 69 and 79 % busy.
enum Kind { GRAM, SQUARE, APPLY };

// Every wait is bounded: it gives up after WAIT_NS, or WAIT_TRIES tries (of 20 ns at the very least).  The longest that is
// due, an epilogue's for all the products of a tile 2^20 deep, takes some 9 ms when nothing else uses the GPU.  A
// thread that gives up tells the others of its block, which then stop too, and the call (`lost`): its result is NaN.
constexpr uint64_t WAIT_NS = 2000000000, LANDING_NS = 20000000, LOSE_NS = 1000000;
constexpr int WAIT_TRIES = 1 << 28;
// On one SM a wait is for one product, a microsecond: tries alone (20 ms at the very least) do, and cost less code.
constexpr int SMALL_TRIES = 1 << 20;
// Seconds that a pair of blocks takes longer to start (four fp32 333 x 1000: 14.4 us a product, 13.1 without pairs).  Other sizes at
// which the two meet, us a call with pairs against single blocks: 1024 x 1024 fp32 +23 (X X^T), 4 x 512 x 1024 +5 (P X), 2 x 1024 x 2048 +4
// (X X^T, taken), 1536 x 1536 +7 (X X^T, taken), 2048 x 2048 +9 (X X^T, taken): more would do no harm.
constexpr double PAIRS_START = 2e-6;
constexpr int SEGMENT = 16;                 // slices of 64: 1024 of depth

constexpr int BM = 128, BK = 64;
constexpr int EPILOGUE_WARPS = 8;
constexpr int PRODUCT_THREADS = 64 + 32 * EPILOGUE_WARPS;

template <bool PAIR, int CG, int BN>
struct Ring {
    static constexpr int PLANES = PAIR ? 2 : 1;
    static constexpr int A_BYTES = BM * BK * 2, B_COLS = BN / CG, B_BYTES = B_COLS * BK * 2;    // of one block and plane
    static constexpr int STAGE = PLANES * (A_BYTES + B_BYTES);
    static constexpr int STAGES = 196608 / STAGE > 6 ? 6 : 196608 / STAGE;      // 229376 and 7 measured the same
    static constexpr int BYTES = STAGES * STAGE + 1024 + 256;    // slack to start on 1024 bytes, barriers
    static constexpr int MAINS = PAIR && BN == 64 ? 2 : 1;       // accumulators of the products of hi parts
    static constexpr int SET = (MAINS + PLANES - 1) * BN <= 64 ? 64 : (MAINS + PLANES - 1) * BN <= 128 ? 128 : 256;     // TMEM columns of one set
    static_assert((MAINS + PLANES - 1) * BN <= SET && 2 * SET <= 512 && STAGES >= 2, "accumulators fit TMEM, the ring shared memory");
};

struct ProductShape {
    int mp, np;                 // padded extents of X; S and P are mp x mp
    int depth;                  // np (GRAM) or mp
    int tiles, per_matrix, across;   // tiles in all, of one matrix, of one row of tiles
    int cols;                   // columns of the result: mp or np
    float alpha, beta;          // stored = alpha acc + beta (hi + lo of the added term)
};

// A 64-column slice to this block's shared memory; CG = 2: its bytes count on the first block's barrier.
template <int CG>
__device__ __forceinline__ void load_slice(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    if constexpr (CG == 1)
        tma_load_3d(dst, map, c0, c1, c2, bar);
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
            : "memory");
}
__device__ __forceinline__ uint32_t in_first_block(uint32_t addr) {      // the same place in the pair's first block
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same summed over `SETS` accumulators, `apart` columns from one another.
template <int SETS>
__device__ __forceinline__ void load_sums(float (&v)[32], uint32_t addr, int apart) {
    tmem_load32(addr, v);
#pragma unroll
    for (int s = 1; s < SETS; ++s) {
        float x[32];
        tmem_load32(addr + s * apart, x);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += x[i];
    }
}

__device__ unsigned int g_ortho_timeouts;

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Waits for the phase of `bar`, or gives up: `gave_up` then, and from then on.  `broken`: a word of shared memory, not 0
// once a thread of the block has given up (none: nobody else waits for this one, and it is not counted).
__device__ __forceinline__ void wait_for(uint32_t bar, uint32_t parity, bool& gave_up, volatile uint32_t* broken, unsigned int* lost, uint64_t limit = WAIT_NS) {
    if (gave_up) return;
    uint64_t start = 0;                   // the clock is slow to read: only once a wait has become a long one
    for (int i = 0; i < WAIT_TRIES; ++i) {
        if (mbar_try(bar, parity)) return;
        if (i % 64 != 63) continue;
        if (broken != nullptr && *broken != 0) break;
        const uint64_t t = now_ns();
        if (start == 0) start = t;
        if (t - start > limit) break;
    }
    gave_up = true;
    if (lost != nullptr) atomicExch(lost, 1u);
    if (broken == nullptr) return;
    *broken = 1;
    atomicAdd(&g_ortho_timeouts, 1u);
}

// Tile number t of one matrix -> first row and column of the tile (CG * 128 rows, BN columns).
template <bool LOWER, int CG, int BN>
__device__ __forceinline__ void tile_at(int t, int across, int& i0, int& j0) {
    if (!LOWER) {
        i0 = t / across * (CG * BM);
        j0 = t % across * BN;
    } else {                    // the tiles that touch the lower triangle, row by row: R (i + 1) in row i
        constexpr int R = CG * BM / BN;
        const int u = t / R;
        int i = (int)((sqrtf(8.f * u + 1.f) - 1.f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= u) ++i;
        while (i * (i + 1) / 2 > u) --i;
        i0 = i * (CG * BM);
        j0 = (t - R * (i * (i + 1) / 2)) * BN;
    }
}

// left: K-major map of X (GRAM), S (SQUARE) or P (APPLY), also the right operand of GRAM and SQUARE;
// right: map of X in 64 x 64 boxes (APPLY).  added: planes of the term in the epilogue (S or X).
template <bool PAIR, int CG, int BN, int KIND, bool LOWER, int KS>
__global__ void __launch_bounds__(PRODUCT_THREADS, 1) product_kernel(const __grid_constant__ CUtensorMap left, const __grid_constant__ CUtensorMap right,
                                                                      const __half* __restrict__ added, __half* __restrict__ out, unsigned int* lost, ProductShape s) {
    using R = Ring<PAIR, CG, BN>;
    static_assert(!LOWER || CG * BM % BN == 0, "columns of tiles end where rows do");
    static_assert(KS == 1 || (CG == 1 && BN == 64 && !LOWER), "the depth is split where tiles are few and narrow");
    extern __shared__ uint8_t raw[];
    uint8_t* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + R::STAGES * R::STAGE);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * R::STAGES + 5);
    volatile uint32_t* broken = tmem_slot + 1;
    const uint32_t full = smem_u32(bars), empty = full + 8 * R::STAGES, done = empty + 8 * R::STAGES, freed = done + 16, ended = freed + 16;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = CG == 2 ? (int)(blockIdx.x & 1) : 0, workers = gridDim.x / (CG * KS), worker = blockIdx.x / (CG * KS);
    const int slice = KS > 1 ? (int)(blockIdx.x % KS) : 0;      // which part of the depth
    if (threadIdx.x == 0) {
        for (int i = 0; i < R::STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(done + 8 * i, 1); mbar_init(freed + 8 * i, CG * EPILOGUE_WARPS); }
        mbar_init(ended, 1);
        *broken = 0;
        mbar_fence_init();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&left) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&right) : "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(2 * R::SET) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(2 * R::SET) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if constexpr (CG == 2) cluster_sync();       // the other block's barriers are there
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    pdl_wait_then_trigger();
    const int steps = s.depth / BK, step0 = steps * slice / KS, step1 = steps * (slice + 1) / KS;
    bool gave_up = false;

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t full_first = CG == 2 ? in_first_block(full) : full;
            int stage = 0, phase = 0;
            for (int tile = worker; tile < s.tiles && !gave_up; tile += workers) {
                const int k = tile / s.per_matrix;
                int i0, j0;
                tile_at<LOWER, CG, BN>(tile % s.per_matrix, s.across, i0, j0);
                i0 += rank * BM;
                j0 += rank * R::B_COLS;
                for (int step = step0; step < step1; ++step) {
                    wait_for(empty + 8 * stage, phase ^ 1, gave_up, broken, lost);
                    if (gave_up) break;
                    if (rank == 0) mbar_expect_tx(full + 8 * stage, CG * R::STAGE);
                    const uint32_t base = smem_u32(ring + stage * R::STAGE);
                    const uint32_t bar = full_first + 8 * stage;
#pragma unroll
                    for (int p = 0; p < R::PLANES; ++p) {
                        load_slice<CG>(base + p * R::A_BYTES, &left, step * BK, i0, 2 * k + p, bar);
                        const uint32_t b = base + R::PLANES * R::A_BYTES + p * R::B_BYTES;
                        if (KIND == APPLY) {
#pragma unroll
                            for (int q = 0; q < R::B_COLS / 64; ++q) load_slice<CG>(b + q * 8192, &right, j0 + 64 * q, step * BK, 2 * k + p, bar);
                        } else {
                            load_slice<CG>(b, &right, step * BK, j0, 2 * k + p, bar);
                        }
                    }
                    if (++stage == R::STAGES) { stage = 0; phase ^= 1; }
                }
            }
            // the last copies have to land before the block may end: wait until they have been used
            const int issued = stage, pass = phase;
            for (int i = 0; i < R::STAGES && !gave_up; ++i) {
                wait_for(empty + 8 * stage, phase ^ 1, gave_up, broken, lost);
                if (++stage == R::STAGES) { stage = 0; phase ^= 1; }
            }
            if (gave_up)      // nobody uses them any more: until they have landed (the second block of a pair, whose bytes
                              // count on the first one's barriers: until they must have)
                for (int i = 0; i < R::STAGES; ++i) {
                    bool late = false;
                    wait_for(full + 8 * i, i < issued ? pass : pass ^ 1, late, nullptr, nullptr, LANDING_NS);
                }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t IDESC = (1u << 4) | (KIND == APPLY ? 1u << 16 : 0u) | ((uint32_t)(BN / 8) << 17) | ((uint32_t)(CG * BM / 16) << 24);
            constexpr int KB = KIND == APPLY ? 2048 : 32;      // bytes from one 16-deep piece of B to the next
            // one thread issues everything: what it computes per product has to stay short
            const uint64_t a0 = slice_desc(smem_u32(ring), false), b0 = slice_desc(smem_u32(ring) + R::PLANES * R::A_BYTES, KIND == APPLY);
            int stage = 0, phase = 0, acc = 0, acc_phase = 0;
            for (int tile = worker; tile < s.tiles && !gave_up; tile += workers) {
                for (int begin = step0; begin < step1 && !gave_up;) {
                    const int stop = PAIR && begin + SEGMENT < step1 ? begin + SEGMENT : step1;
                    wait_for(freed + 8 * acc, acc_phase ^ 1, gave_up, broken, lost);
                    if (gave_up) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + acc * R::SET;
                    for (int step = begin; step < stop; ++step) {
                        wait_for(full + 8 * stage, phase, gave_up, broken, lost);
                        if (gave_up) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = desc_at(a0, stage * R::STAGE), b = desc_at(b0, stage * R::STAGE);
#pragma unroll
                        for (int kk = 0; kk < BK / 16; ++kk) {
                            const uint64_t ah = desc_at(a, kk * 32), bh = desc_at(b, kk * KB);
                            mma_f16<CG>(d + kk % R::MAINS * BN, ah, bh, IDESC, step > begin || kk >= R::MAINS);
                            if (PAIR) {
                                constexpr int CROSS = R::MAINS * BN;
                                mma_f16<CG>(d + CROSS, ah, desc_at(b, R::B_BYTES + kk * KB), IDESC, step > begin || kk > 0);
                                mma_f16<CG>(d + CROSS, desc_at(a, R::A_BYTES + kk * 32), bh, IDESC, true);
                            }
                        }
                        mma_commit<CG>(empty + 8 * stage);
                        if (++stage == R::STAGES) { stage = 0; phase ^= 1; }
                    }
                    if (gave_up) break;
                    mma_commit<CG>(done + 8 * acc);
                    if (acc == 1) acc_phase ^= 1;
                    acc ^= 1;
                    begin = stop;
                }
            }
            if (gave_up) {       // the products issued so far have to end before their accumulators are given back
                bool late = false;
                mma_commit<CG>(ended);
                wait_for(ended, 0, late, nullptr, nullptr);
            }
        }
    } else if constexpr (KS == 1) {
        const int quarter = warp % 4, half = (warp - 2) / 4;          // TMEM lanes this warp may read; its half of the columns
        const uint32_t freed_first = CG == 2 ? in_first_block(freed) : freed;
        int acc = 0, acc_phase = 0;
        const int64_t out_plane = (int64_t)s.mp * s.cols;
        for (int tile = worker; tile < s.tiles && !gave_up; tile += workers) {
            const int k = tile / s.per_matrix;
            int i0, j0;
            tile_at<LOWER, CG, BN>(tile % s.per_matrix, s.across, i0, j0);
            const bool mirror = LOWER && j0 < i0;      // tiles of the diagonal block hold both halves
            const int row = i0 + rank * BM + quarter * 32 + lane;
            __half* hi = out + 2 * k * out_plane;
            __half* lo = hi + out_plane;
            const __half* add = KIND == GRAM ? nullptr : added + 2 * k * out_plane + (int64_t)row * s.cols;
            Pack<__half, 8> ph[4] = {}, pl[4] = {};
            auto fetch = [&](int c) {                      // the added term of 32 columns: on its way while the sums are formed
                if constexpr (KIND != GRAM) {
                    const int col = j0 + c;
                    if (row >= s.mp || col >= s.cols) return;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        ph[g] = load_pack<__half, 8>(add + col + 8 * g);
                        pl[g] = load_pack<__half, 8>(add + out_plane + col + 8 * g);
                    }
                }
            };
            fetch(half * 32);
            auto wait_done = [&]() {
                wait_for(done + 8 * acc, acc_phase, gave_up, broken, lost);
                gave_up = __any_sync(~0u, gave_up);        // the reads of TMEM are the whole warp's
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            };
            auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 2) arrive_cluster(freed_first + 8 * acc);
                    else mbar_arrive(freed + 8 * acc);
                }
                if (acc == 1) acc_phase ^= 1;
                acc ^= 1;
            };
            float run[PAIR ? BN / 64 : 1][32];             // the segments before the last
            if constexpr (PAIR) {
#pragma unroll
                for (int g = 0; g < BN / 64; ++g)
#pragma unroll
                    for (int i = 0; i < 32; ++i) run[g][i] = 0.f;
                for (int begin = step0 + SEGMENT; begin < step1; begin += SEGMENT) {
                    wait_done();
                    if (gave_up) break;
#pragma unroll
                    for (int g = 0; g < BN / 64; ++g) {
                        float v[32];
                        load_sums<R::MAINS + R::PLANES - 1>(v, tmem + acc * R::SET + half * 32 + 64 * g + ((uint32_t)(quarter * 32) << 16), BN);
#pragma unroll
                        for (int i = 0; i < 32; ++i) run[g][i] += v[i];
                    }
                    release();
                }
            }
            wait_done();
            if (gave_up) break;
#pragma unroll(PAIR ? BN / 64 : 1)
            for (int part = 0; part < BN / 64; ++part) {
                const int c = half * 32 + 64 * part, col = j0 + c;
                const bool there = row < s.mp && col < s.cols;       // the same for the whole warp: extents are multiples of 64
                if (part > 0) fetch(c);
                float v[32];
                load_sums<R::MAINS + R::PLANES - 1>(v, tmem + acc * R::SET + c + ((uint32_t)(quarter * 32) << 16), BN);
                if constexpr (PAIR) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] += run[part][i];
                }
                if (!there) continue;
                const bool both = PAIR || KIND != SQUARE;        // P is only ever a factor
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        w[i] = s.alpha * v[8 * g + i];
                        if (KIND != GRAM) w[i] = fmaf(s.beta, __half2float(ph[g].v[i]) + __half2float(pl[g].v[i]), w[i]);
                    }
                    split8(w, ph[g], pl[g]);
                    *reinterpret_cast<Pack<__half, 8>*>(hi + (int64_t)row * s.cols + col + 8 * g) = ph[g];
                    if (both) *reinterpret_cast<Pack<__half, 8>*>(lo + (int64_t)row * s.cols + col + 8 * g) = pl[g];
                }
                if (mirror) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        hi[(int64_t)(col + i) * s.cols + row] = ph[i / 8].v[i % 8];
                        if (both) lo[(int64_t)(col + i) * s.cols + row] = pl[i / 8].v[i % 8];
                    }
                }
            }
            release();
        }
    }
    if constexpr (KS > 1) {
        // Every block of the cluster has its part of the depth: it leaves its sums in shared memory (the ring is
        // free by now), and then each adds up BN / KS of the tile's columns, in the same order everywhere.
        const int quarter = warp % 4, half = (warp - 2) / 4;
        float* mine = reinterpret_cast<float*>(ring);                 // [BN][128]
        if (warp >= 2) {
            float run[32] = {};
            int acc = 0, acc_phase = 0;
            for (int begin = step0; begin < step1; begin = PAIR ? begin + SEGMENT : step1) {
                wait_for(done + 8 * acc, acc_phase, gave_up, broken, lost);
                gave_up = __any_sync(~0u, gave_up);
                if (gave_up) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                float v[32];
                load_sums<R::MAINS + R::PLANES - 1>(v, tmem + acc * R::SET + half * 32 + ((uint32_t)(quarter * 32) << 16), BN);
#pragma unroll
                for (int i = 0; i < 32; ++i) run[i] += v[i];
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(freed + 8 * acc);
                if (acc == 1) acc_phase ^= 1;
                acc ^= 1;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) mine[(half * 32 + i) * BM + quarter * 32 + lane] = run[i];
        }
        __syncwarp();
        cluster_sync();
        if (warp >= 2) {
            constexpr int COLS = BN / KS / 2;                         // of a warp
            int i0, j0;
            tile_at<LOWER, CG, BN>(worker % s.per_matrix, s.across, i0, j0);
            const int k = worker / s.per_matrix, row = i0 + quarter * 32 + lane, c = slice * (BN / KS) + half * COLS, col = j0 + c;
            const int64_t out_plane = (int64_t)s.mp * s.cols;
            if (row < s.mp && col < s.cols) {
                __half* hi = out + 2 * k * out_plane + (int64_t)row * s.cols + col;
                const __half* add = KIND == GRAM ? nullptr : added + 2 * k * out_plane + (int64_t)row * s.cols + col;
                const uint32_t here = smem_u32(mine) + (uint32_t)(c * BM + quarter * 32 + lane) * 4;
                uint32_t from[KS];
#pragma unroll
                for (int r = 0; r < KS; ++r) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from[r]) : "r"(here), "r"(r));
#pragma unroll
                for (int g = 0; g < COLS; g += 8) {
                    Pack<__half, 8> ph = {}, pl = {};
                    if constexpr (KIND != GRAM) {
                        ph = load_pack<__half, 8>(add + g);
                        pl = load_pack<__half, 8>(add + out_plane + g);
                    }
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float v = 0.f;
#pragma unroll
                        for (int r = 0; r < KS; ++r) {
                            float x;
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(from[r] + (uint32_t)((g + i) * BM * 4)) : "memory");
                            v += x;
                        }
                        w[i] = s.alpha * v;
                        if (KIND != GRAM) w[i] = fmaf(s.beta, __half2float(ph.v[i]) + __half2float(pl.v[i]), w[i]);
                    }
                    split8(w, ph, pl);
                    *reinterpret_cast<Pack<__half, 8>*>(hi + g) = ph;
                    if (PAIR || KIND != SQUARE) *reinterpret_cast<Pack<__half, 8>*>(hi + out_plane + g) = pl;
                }
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if constexpr (CG == 2 || KS > 1) cluster_sync();       // nobody's barriers or sums are needed any more
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) {
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * R::SET) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * R::SET) : "memory");
    }
}

// Planes of a stack of r x c matrices as a 3-D tensor (columns, rows, 2 count) read in boxes of 64 columns
// by `box_rows` rows; what lies outside reads as zero.
bool encode_planes(CUtensorMap* m, const __half* p, int64_t count, int r, int c, int box_rows) {
    EncodeTiledFn fn = tma_encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)c, (cuuint64_t)r, (cuuint64_t)(2 * count)};
    const cuuint64_t strides[2] = {(cuuint64_t)c * 2u, (cuuint64_t)c * r * 2u};
    const cuuint32_t box[3] = {64u, (cuuint32_t)box_rows, 1u}, one[3] = {1u, 1u, 1u};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The maps of one operand: boxes of 128 rows, of 64 rows, and of 64 rows for MN-major slices (the same).
struct Maps {
    CUtensorMap tall, low;
    bool encode(const __half* p, int64_t count, int r, int c) {
        return encode_planes(&tall, p, count, r, c, BM) && encode_planes(&low, p, count, r, c, 64);
    }
};

template <bool PAIR, int CG, int BN, int KIND, bool LOWER, int KS = 1>
cudaError_t launch_product(const Maps& left, const Maps& right, const __half* added, __half* out, unsigned int* lost, ProductShape s,
                           int64_t count, int sms, cudaStream_t st) {
    using R = Ring<PAIR, CG, BN>;
    const int64_t down = ceil_div(s.mp, CG * BM);
    s.across = (int)ceil_div(s.cols, BN);
    s.depth = KIND == GRAM ? s.np : s.mp;
    const int64_t per = LOWER ? down * (down + 1) / 2 * (CG * BM / BN) : down * s.across;
    if (per * count > 0x3fffffff) return cudaErrorInvalidConfiguration;
    s.per_matrix = (int)per;
    s.tiles = (int)(per * count);
    auto kernel = product_kernel<PAIR, CG, BN, KIND, LOWER, KS>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_smem(kernel, R::BYTES, allowed);
    if (e != cudaSuccess) return e;
    const int workers = KS > 1 || s.tiles < sms / CG ? s.tiles : sms / CG;      // KS > 1: one tile each
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(workers * CG * KS));
    cfg.blockDim = dim3(PRODUCT_THREADS);
    cfg.dynamicSmemBytes = R::BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (CG * KS > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = CG * KS;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (pdl_enabled()) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const bool boxes64 = KIND == APPLY || R::B_COLS == 64;
    return cudaLaunchKernelEx(&cfg, kernel, left.tall, boxes64 ? right.low : right.tall, added, out, lost, s);
}

// Seconds that a form of a product takes, for comparing the forms.  A block brings `STAGE` bytes per 64 of
// depth; all of them together are reckoned to get 9e12 bytes a second out of L2 (8.6 to 10.1e12 in
// products of 4096 x 4096), one alone some 76e9 (0.63 us for 48 KB), and its tensor core needs its time;
// the last tile's epilogue is not hidden, and joining a split depth takes two barriers of the cluster.
// Each product was forced through every other form it could take, for 14 sizes from 40 x 900 to 2048 x 2048, stacks of up
// to 16, fp32 and bf16: what is chosen is within 5 % of the best call, but for sixteen 300 x 300 (8 and 6 %
// slower with the square in 128 columns a tile than in 64).
template <bool PAIR, int CG, int BN, int KIND, bool LOWER, int KS = 1>
double product_seconds(const ProductShape& s, int64_t count, int sms) {
    using R = Ring<PAIR, CG, BN>;
    const int64_t down = ceil_div(s.mp, CG * BM), across = ceil_div(s.cols, BN), workers = sms / (CG * KS);
    const int64_t tiles = count * (LOWER ? down * (down + 1) / 2 * (CG * BM / BN) : down * across), steps = (KIND == GRAM ? s.np : s.mp) / BK;
    if (KS > 1 && (tiles > workers || steps < KS)) return 1e9;      // one tile a cluster, all of them at once
    const int64_t waves = ceil_div(tiles, workers), blocks = (tiles < workers ? tiles : workers) * CG * KS;
    const double shared = R::STAGE * (double)blocks / 9e12, alone = R::STAGE / 76e9, math = (PAIR ? 3 : 1) * 2.0 * BM * BN * BK * 1.0 / 14e12;
    const double step = shared > alone ? (shared > math ? shared : math) : (alone > math ? alone : math);
    return waves * ceil_div(steps, KS) * step + 3e-6 * BN / 128 + (LOWER ? 2e-6 : 0) + (KS > 1 ? 1.5e-6 : 0) + (CG > 1 ? PAIRS_START : 0);
}

// Pairs of SMs, or single blocks with tiles of 128 or 64 columns, the latter with the depth split over 2 or 4
// blocks where there are few: whichever is reckoned fastest.
// The forms with 64 columns a tile are for few tiles.  S S of single factors is formed from 1088 rows on and has 153 of
// them, against 45 of 128 columns.
template <bool PAIR, int KIND>
constexpr bool has_narrow() { return PAIR || KIND != SQUARE; }

template <bool PAIR, int KIND>
int best_form(const ProductShape& s, int64_t count, int sms) {
    constexpr int WIDE = PAIR ? 128 : 256;      // PAIR: two accumulators a set
    constexpr bool LOWER = KIND != APPLY;
    const double t[5] = {product_seconds<PAIR, 2, WIDE, KIND, LOWER>(s, count, sms), product_seconds<PAIR, 1, 128, KIND, LOWER>(s, count, sms),
                         product_seconds<PAIR, 1, 64, KIND, false>(s, count, sms), product_seconds<PAIR, 1, 64, KIND, false, 2>(s, count, sms),
                         product_seconds<PAIR, 1, 64, KIND, false, 4>(s, count, sms)};
    int best = 0;
    for (int i = 1; i < (has_narrow<PAIR, KIND>() ? 5 : 2); ++i)
        if (t[i] < t[best]) best = i;
    return best;
}

template <bool PAIR, int KIND>
cudaError_t run_product(const Maps& left, const Maps& right, const __half* added, __half* out, unsigned int* lost, ProductShape s, int64_t count,
                        int sms, cudaStream_t st) {
    constexpr int WIDE = PAIR ? 128 : 256;
    constexpr bool LOWER = KIND != APPLY;
    const int form = best_form<PAIR, KIND>(s, count, sms);
    if constexpr (has_narrow<PAIR, KIND>()) {
        if (form == 2) return launch_product<PAIR, 1, 64, KIND, false>(left, right, added, out, lost, s, count, sms, st);
        if (form == 3) return launch_product<PAIR, 1, 64, KIND, false, 2>(left, right, added, out, lost, s, count, sms, st);
        if (form == 4) return launch_product<PAIR, 1, 64, KIND, false, 4>(left, right, added, out, lost, s, count, sms, st);
    }
    if (form == 1) return launch_product<PAIR, 1, 128, KIND, LOWER>(left, right, added, out, lost, s, count, sms, st);
    return launch_product<PAIR, 2, WIDE, KIND, LOWER>(left, right, added, out, lost, s, count, sms, st);
}

// --------------------------------------------------------------------------------- small matrices
// A matrix whose shorter side is at most 128 and whose longer side is at most 256 stays on one SM for the
// whole call: X and S (then P) as swizzled hi and lo planes in shared memory, the products' sums in TMEM,
// cross products apart.  One launch instead of three per step and three
// around them; what bounds it is the chain of 3 x steps products, each of which waits for the one before.
// The planes of X, rows of 64-column blocks, serve as K-major factor of S and as MN-major factor of P X.
//
// With 16-bit types X enters X X^T and P X as a single factor; S S and P are pairs whatever the type, which costs a product
// each where three wait for one another anyway.  Error of bf16 results, of which 1.66e-3 is their own rounding: 64 x 200 3.8e-3 with
// single factors throughout, 2.5e-3 with S as a pair, 2.1e-3 with P as one too (fp16: 3.5e-3, 1.9e-3, 1.3e-3, own 2.1e-4); P
// takes eight 128 x 128 from 32 to 34 us, 400 128 x 256 from 150 to 165.
//
// 16-bit matrices of up to SMALL_PAIRS on their shorter side are multiplied as pairs too.  A direction in which such a matrix
// is almost singular is a large part of it, and single factors' rounding grows in it at every step.  The worst of 4096 to 16384
// matrices, single factors, against 3e-3 (bf16) or 4e-4 (fp16) of the result's own rounding, which is all that pairs leave: 2 x 2
// 1.5e-2, 3 x 5 1.2e-2, 3 x 20 1.1e-2, 6 x 6 9.9e-3, 8 x 8 5.8e-3, 16 x 16 3.6e-3, 24 x 24 3.3e-3, 128 x 128 2.4e-3: from 8 on the
// rest dilutes it below the 8.3e-3 that single factors are allowed, and they are faster (eight 16 x 256 27 against 35 us, 64 x 256
// 37 against 45, 128 x 128 34 against 39).
constexpr int SMALL_PAIRS = 8;
constexpr int SMALL_M = 128, SMALL_N = 256, SMALL_THREADS = 512;
constexpr int SMALL_BLOCK = SMALL_M * 128;              // bytes of a 64-column block of a plane
constexpr int SMALL_S = 4 * SMALL_BLOCK;                // S: two blocks, hi and lo
inline size_t small_bytes(int np) { return 2 * (size_t)(np / 64) * SMALL_BLOCK + SMALL_S + 1024; }

// The 16 bytes of row r that hold columns c .. c+7 (c % 8 == 0), in a plane of swizzled blocks.
__device__ __forceinline__ uint8_t* chunk_at(uint8_t* plane, int r, int c) {
    return plane + (c / 64) * SMALL_BLOCK + r * 128 + (((c % 64 / 8) ^ (r & 7)) * 16);
}
__device__ __forceinline__ void put8(uint8_t* hi_plane, uint8_t* lo_plane, int r, int c, const float (&v)[8]) {
    Pack<__half, 8> hi, lo;
    split8(v, hi, lo);
    *reinterpret_cast<Pack<__half, 8>*>(chunk_at(hi_plane, r, c)) = hi;
    *reinterpret_cast<Pack<__half, 8>*>(chunk_at(lo_plane, r, c)) = lo;
}
__device__ __forceinline__ float value_at(uint8_t* hi_plane, uint8_t* lo_plane, int r, int c) {
    return __half2float(*reinterpret_cast<const __half*>(chunk_at(hi_plane, r, c & ~7) + 2 * (c & 7))) +
           __half2float(*reinterpret_cast<const __half*>(chunk_at(lo_plane, r, c & ~7) + 2 * (c & 7)));
}

template <typename T, bool PAIR>
__global__ void __launch_bounds__(SMALL_THREADS, 1) ortho_small_kernel(OrthoIo io, int steps, bool lose) {
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bar, ended;
    __shared__ uint32_t tmem_slot;
    __shared__ float part[SMALL_THREADS / 32];
    uint8_t* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const int xplane = io.np / 64 * SMALL_BLOCK;
    uint8_t *xh = base, *xl = base + xplane, *sh = base + 2 * xplane, *sl = sh + 2 * SMALL_BLOCK;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    if (tid == 0) {
        mbar_init(smem_u32(&bar), 1);
        mbar_init(smem_u32(&ended), 1);
        mbar_fence_init();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait_then_trigger();
    const int64_t k = blockIdx.x;
    // The update (muon: after moving the momentum on), read once: a thread holds its elements, 32 columns
    // apart in the rows of its warp, until the norm is known.
    const T* g = (const T*)io.grad + k * io.grad_matrix;
    float* mom = io.momentum ? io.momentum + k * io.rows * io.cols : nullptr;
    constexpr int WARPS = SMALL_THREADS / 32, MOST = SMALL_M * SMALL_N / SMALL_THREADS;
    float u[MOST], top = 0.f;
    auto read = [&](auto segments) {            // 32-column segments of a row
        constexpr int SEG = decltype(segments)::value, ROWS = 16 * SEG <= MOST ? 16 : MOST / SEG;
        const T* gr = g + warp * io.grad_row + lane;
        float* mr = mom ? mom + warp * io.cols + lane : nullptr;
#pragma unroll
        for (int e = 0; e < MOST; ++e) u[e] = 0.f;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (warp + WARPS * i >= io.rows) break;
#pragma unroll
            for (int q = 0; q < SEG; ++q) {
                if (lane + 32 * q >= io.cols) continue;
                float v = to_f32<T>(gr[32 * q]);
                if (mom != nullptr) {
                    const float next = fmaf(io.decay, mr[32 * q], v);
                    mr[32 * q] = next;
                    v = io.nesterov ? fmaf(io.decay, next, v) : next;
                }
                u[i * SEG + q] = v;
            }
            gr += WARPS * io.grad_row;
            if (mom != nullptr) mr += WARPS * io.cols;
        }
#pragma unroll
        for (int e = 0; e < ROWS * SEG; ++e) top = max_nan(top, fabsf(u[e]));
    };
    if (io.cols > 128) read(std::integral_constant<int, 8>{});
    else if (io.cols > 64) read(std::integral_constant<int, 4>{});
    else if (io.cols > 32) read(std::integral_constant<int, 2>{});
    else read(std::integral_constant<int, 1>{});
    if (io.m < SMALL_M || io.n < io.np)                    // zeros around X
        for (int i = tid; i < 2 * xplane / 16; i += SMALL_THREADS) reinterpret_cast<uint4*>(xh)[i] = make_uint4(0, 0, 0, 0);
    // the largest element first: squares of u 2^-e of a matrix of any scale fit in 32 bits
#pragma unroll
    for (int m = 16; m > 0; m /= 2) top = max_nan(top, __shfl_xor_sync(~0u, top, m));
    if (lane == 0) part[warp] = top;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) top = max_nan(top, part[i]);
    const int e2 = top > 0.f && top < INFINITY ? max(ilogbf(top), -100) : 0;
    const float fit = ldexpf(1.f, -e2);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < MOST; ++e) sum = fmaf(u[e] * fit, u[e] * fit, sum);
#pragma unroll
    for (int m = 16; m > 0; m /= 2) sum += __shfl_xor_sync(~0u, sum, m);
    __syncthreads();
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) sum += part[i];
    const Fit to_x(ldexp((double)sqrtf(sum), e2), io.eps);
    auto place = [&](auto segments) {                      // the first X
        constexpr int SEG = decltype(segments)::value, ROWS = 16 * SEG <= MOST ? 16 : MOST / SEG;
#pragma unroll
        for (int n = 0; n < ROWS; ++n) {
            const int r = warp + WARPS * n;
            if (r >= io.rows) break;
#pragma unroll
            for (int q = 0; q < SEG; ++q) {
                const int c = lane + 32 * q, i = io.turned ? c : r, j = io.turned ? r : c;
                if (c >= io.cols) continue;
                const float v = to_x(u[n * SEG + q]);
                const __half h = __float2half_rn(v);
                const uint32_t at = (uint32_t)(chunk_at(xh, i, j & ~7) - xh) + 2 * (j & 7);
                *reinterpret_cast<__half*>(xh + at) = h;
                *reinterpret_cast<__half*>(xl + at) = __float2half_rn(v - __half2float(h));
            }
        }
    };
    if (io.cols > 128) place(std::integral_constant<int, 8>{});
    else if (io.cols > 64) place(std::integral_constant<int, 4>{});
    else if (io.cols > 32) place(std::integral_constant<int, 2>{});
    else place(std::integral_constant<int, 1>{});
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();

    const uint32_t axh = smem_u32(xh), axl = smem_u32(xl), ash = smem_u32(sh), asl = smem_u32(sl);
    const int deep_m = (io.m + 15) / 16, deep_n = (io.n + 15) / 16;      // 16-deep pieces that are not all zeros
    const int quarter = warp % 4, part_of = warp / 4, row = quarter * 32 + lane;      // TMEM lanes; which columns
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    uint32_t phase = 0;
    bool gave_up = false;
    // D = L R^T over `deep` pieces, K-major factors as hi and lo planes
    auto k_major = [](uint64_t plane, int piece) { return desc_at(plane, piece / 4 * SMALL_BLOCK + piece % 4 * 32); };
    const uint64_t dxh = slice_desc(axh, false), dxl = slice_desc(axl, false), dsh = slice_desc(ash, false), dsl = slice_desc(asl, false);
    const uint64_t rxh = slice_desc(axh, true, SMALL_BLOCK), rxl = slice_desc(axl, true, SMALL_BLOCK);
    auto finish = [&]() {               // the products are done, and every thread may read their sums
        mbar_wait<SMALL_TRIES>(smem_u32(&bar), phase, gave_up, &g_ortho_timeouts);
        phase ^= 1;
        __syncwarp();                   // the reads of TMEM are the whole warp's
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    auto written = [&]() {              // planes are written and sums are read: the next products may start
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(SMALL_M / 16) << 24), SQUARE_IDESC = IDESC | (uint32_t)(128 / 8) << 17;
    for (int step = 0; step < steps; ++step) {
        if (tid == 0) {                                                   // S = X X^T: columns 0-127, cross products 128-255
#pragma unroll
            for (int p = 0; p < SMALL_N / 16; ++p) {
                if (p >= deep_n) break;
                const uint64_t h = k_major(dxh, p);
                mma_f16(tmem, h, h, SQUARE_IDESC, p > 0);
                if (PAIR) {
                    const uint64_t l = k_major(dxl, p);
                    mma_f16(tmem + 128, h, l, SQUARE_IDESC, p > 0);
                    mma_f16(tmem + 128, l, h, SQUARE_IDESC, true);
                }
            }
            mma_commit(smem_u32(&bar));
        }
        finish();
        float kept[32];                                                   // this thread's part of S, times 2^14
        {
            const int c = part_of * 32;
            load_sums<PAIR ? 2 : 1>(kept, tmem + lanes + c, 128);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = kept[8 * q + i] *= 1.f / SCALE;
                put8(sh, sl, row, c + 8 * q, w);
            }
        }
        written();
        if (tid == 0) {                                                   // S S: columns 256-383, cross products 384-511
#pragma unroll
            for (int p = 0; p < SMALL_M / 16; ++p) {
                if (p >= deep_m) break;
                const uint64_t h = k_major(dsh, p), l = k_major(dsl, p);
                mma_f16(tmem + 256, h, h, SQUARE_IDESC, p > 0);
                mma_f16(tmem + 384, h, l, SQUARE_IDESC, p > 0);
                mma_f16(tmem + 384, l, h, SQUARE_IDESC, true);
            }
            mma_commit(smem_u32(&bar));
        }
        finish();
        {                                                                 // P over S, which has been read
            const int c = part_of * 32;
            float v[32];
            load_sums<2>(v, tmem + lanes + 256 + c, 128);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = fmaf(NS_C / SCALE, v[8 * q + i], NS_B * kept[8 * q + i]);
                put8(sh, sl, row, c + 8 * q, w);
            }
        }
        written();
        if (tid == 0) {                                                   // P X: columns 0-255, cross products 256-511
            const uint32_t idesc = IDESC | 1u << 16 | (uint32_t)(io.np / 8) << 17;
#pragma unroll
            for (int p = 0; p < SMALL_M / 16; ++p) {
                if (p >= deep_m) break;
                const uint64_t h = k_major(dsh, p), r = desc_at(rxh, p * 2048);
                mma_f16(tmem, h, r, idesc, p > 0);
                mma_f16(tmem + 256, k_major(dsl, p), r, idesc, p > 0);
                if (PAIR) mma_f16(tmem + 256, h, desc_at(rxl, p * 2048), idesc, true);
            }
            mma_commit(smem_u32(&bar));
        }
        finish();
#pragma unroll 1
        for (int c = part_of * 32; c < io.np; c += 128) {
            float v[32];
            load_sums<2>(v, tmem + lanes + c, 256);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const Pack<__half, 8> h = *reinterpret_cast<const Pack<__half, 8>*>(chunk_at(xh, row, c + 8 * q));
                const Pack<__half, 8> l = *reinterpret_cast<const Pack<__half, 8>*>(chunk_at(xl, row, c + 8 * q));
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = fmaf(NS_A, __half2float(h.v[i]) + __half2float(l.v[i]), v[8 * q + i] * (1.f / SCALE));
                put8(xh, xl, row, c + 8 * q, w);
            }
        }
        written();
    }
    if (lose) wait_for(smem_u32(&bar), phase, gave_up, nullptr, nullptr, LOSE_NS);      // nothing arrives any more
    const bool lost = __syncthreads_or(gave_up);
    if (lost) {                         // what has been issued has to end before the accumulators are given back
        bool late = false;
        if (tid == 0) mma_commit(smem_u32(&ended));
        wait_for(smem_u32(&ended), 0, late, nullptr, nullptr);
        __syncthreads();
    }
    const float unit = lost ? NAN : 1.f / SCALE;     // as in ortho_finish_kernel
    // out, along the matrix's rows
    T* out = (T*)io.out + k * io.rows * io.cols;
#pragma unroll 2
    for (int r = warp; r < io.rows; r += SMALL_THREADS / 32)
#pragma unroll 4
        for (int c = lane; c < io.cols; c += 32) {
            const float v = (io.turned ? value_at(xh, xl, c, r) : value_at(xh, xl, r, c)) * unit;
            T* o = out + r * io.cols + c;
            *o = from_f32<T>(mom == nullptr ? v : fmaf(-io.rate, v, io.keep * to_f32<T>(*o)));
        }
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// X back in the shape of the matrices: written out, or applied to the weights.  64 x 64 elements a block:
// read in 16-byte packs along X's rows, written along the matrix's rows, through shared memory where those
// are not the same.
template <typename T>
__global__ void __launch_bounds__(256) ortho_finish_kernel(OrthoIo io, const __half* __restrict__ x, const unsigned int* __restrict__ lost) {
    pdl_wait_then_trigger();
    __shared__ float tile[64][65];
    const float unit = *lost != 0 ? NAN : 1.f / SCALE;      // products that were not waited for: nobody may take X for a result
    const int across = io.np / 64, down = io.mp / 64;
    const int k = blockIdx.x / (across * down), t = blockIdx.x % (across * down), i0 = t / across * 64, j0 = t % across * 64;
    const int64_t plane = (int64_t)io.mp * io.np;
    const int r0 = io.turned ? j0 : i0, c0 = io.turned ? i0 : j0, a = threadIdx.x / 64, b = threadIdx.x % 64;
    T* out = (T*)io.out + ((int64_t)k * io.rows + r0 + a) * io.cols + c0 + b;
    float w[16];                         // the weights, on their way while X is turned
    if (io.momentum != nullptr && !io.wide) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            w[q] = r0 + a + q * 4 < io.rows && c0 + b < io.cols ? to_f32<T>(out[(int64_t)q * 4 * io.cols]) : 0.f;
    }
#pragma unroll
    for (int e = threadIdx.x; e < 64 * 8; e += 256) {
        const int i = e / 8, j = e % 8 * 8;
        const Pack<__half, 8>* p = reinterpret_cast<const Pack<__half, 8>*>(x + 2 * k * plane + (int64_t)(i0 + i) * io.np + j0 + j);
        const Pack<__half, 8> hi = p[0], lo = p[plane / 8];
#pragma unroll
        for (int q = 0; q < 8; ++q) tile[i][j + q] = (__half2float(hi.v[q]) + __half2float(lo.v[q])) * unit;
    }
    __syncthreads();
    if (io.wide) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int r = threadIdx.x / 8 + q * 32, c = threadIdx.x % 8 * 8;
            if (r0 + r >= io.rows || c0 + c >= io.cols) continue;
            T* o = (T*)io.out + ((int64_t)k * io.rows + r0 + r) * io.cols + c0 + c;
            float v[8], old[8];
            if (io.momentum != nullptr) load8<T>(old, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = io.turned ? tile[c + i][r] : tile[r][c + i];
                if (io.momentum != nullptr) v[i] = fmaf(-io.rate, v[i], io.keep * old[i]);
            }
            store8<T>(o, v);
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const int r = a + q * 4;
        if (r0 + r >= io.rows || c0 + b >= io.cols) continue;
        const float v = io.turned ? tile[b][r] : tile[r][b];
        out[(int64_t)q * 4 * io.cols] = from_f32<T>(io.momentum == nullptr ? v : fmaf(-io.rate, v, io.keep * w[q]));
    }
}

// For tests: a wait that nothing ends.
__global__ void ortho_lose_kernel(unsigned int* lost) {
    pdl_wait_then_trigger();
    __shared__ __align__(8) uint64_t bar;
    bool gave_up = false;
    mbar_init(smem_u32(&bar), 1);
    mbar_fence_init();
    wait_for(smem_u32(&bar), 0, gave_up, nullptr, lost, LOSE_NS);
}

struct OrthoSpace {
    size_t sums, lost, x[2], s, p, total;
};
int64_t padded(int64_t n) { return ceil_div(n, 64) * 64; }
bool is_small(int64_t m, int64_t n) { return m <= SMALL_M && n <= SMALL_N; }
OrthoSpace space(int64_t count, int64_t m, int64_t n) {
    OrthoSpace w = {};
    if (is_small(m, n)) return w;
    const int64_t mp = padded(m), np = padded(n);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    w.sums = take(count * MOST_SUMS * 8);
    w.lost = take(4);
    w.x[0] = take(count * mp * np * 4);
    w.x[1] = take(count * mp * np * 4);
    w.s = take(count * mp * mp * 4);
    w.p = take(count * mp * mp * 4);
    w.total = at;
    return w;
}

int check(const fpde_ortho_args* a) {
    if (a == nullptr) return FPDE_ERR_NULL;
    if (!dtype_ok(a->dtype)) return FPDE_ERR_DTYPE;
    if (a->steps < 0 || a->steps > 100 || !(a->eps >= 0)) return FPDE_ERR_PARAM;
    if (a->count < 0 || a->rows < 0 || a->cols < 0 || a->rows > (1 << 20) || a->cols > (1 << 20) || a->count > (1 << 20) ||
        !product_fits(a->count, padded(a->rows), padded(a->cols)))
        return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

#define FPDE_TRY(x)                           \
    do {                                      \
        const cudaError_t e_ = (x);           \
        if (e_ != cudaSuccess) return e_;     \
    } while (0)

ProductShape shape_of(int kind, int mp, int np) {
    if (kind == GRAM) return {mp, np, 0, 0, 0, 0, mp, 1.f / SCALE, 0.f};
    if (kind == SQUARE) return {mp, np, 0, 0, 0, 0, mp, NS_C / SCALE, NS_B};
    return {mp, np, 0, 0, 0, 0, np, 1.f / SCALE, NS_A};
}
// 16-bit matrices: up to which padded shorter side S S and P X are formed from pairs.  While S is small its square is a small
// part of the time and its factors' rounding a large part of the error (bf16, own rounding 1.66e-3): 40 x 900 5.1e-3 without and
// 2.9e-3 with pairs there, 576 x 576 2.48e-3 and 2.19e-3, 1000 x 1000 2.35e-3 and 2.08e-3; at 1100 it is 2.33e-3 without.  Time: 640 x 640 and
// 1024 x 1024 alike to 3 %, four 768 x 1536 279 -> 301 us.  P X of up to 128 rows: 32 x 300 2.9e-3 and 1.76e-3, 64 x 900 2.5e-3 and 1.67e-3;
// two 40 x 900 85 -> 87 us.
bool square_of_pairs(int mp) { return mp <= 1024; }
bool apply_of_pairs(int mp) { return mp <= 128; }

template <typename T>
cudaError_t run(const fpde_ortho_args* a, bool muon, bool lose, cudaStream_t st) {
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
    io.mp = (int)padded(io.m); io.np = (int)padded(io.n);
    io.wide = io.cols % 8 == 0 && packs(io.grad, io.grad_matrix, io.grad_row, sizeof(T), 16 / sizeof(T)) && aligned(io.out, 16) && aligned(io.momentum, 16);
    if (is_small(io.m, io.n)) {
        auto launch = [&](auto* kernel, std::atomic<uint64_t>& allowed) {
            FPDE_TRY(allow_smem(kernel, small_bytes(SMALL_N), allowed));
            return launch_kernel_smem(kernel, dim3((unsigned)a->count), dim3(SMALL_THREADS), small_bytes(io.np), st, io, a->steps, lose);
        };
        static std::atomic<uint64_t> pairs{0}, single{0};
        if (sizeof(T) == 4 || io.m <= SMALL_PAIRS) return launch(ortho_small_kernel<T, true>, pairs);
        if constexpr (sizeof(T) == 2) return launch(ortho_small_kernel<T, false>, single);
    }
    const OrthoSpace w = space(a->count, io.m, io.n);
    char* ws = (char*)a->workspace;
    double* sums = (double*)(ws + w.sums);
    __half* x[2] = {(__half*)(ws + w.x[0]), (__half*)(ws + w.x[1])};
    __half *s = (__half*)(ws + w.s), *p = (__half*)(ws + w.p);
    unsigned int* lost = (unsigned int*)(ws + w.lost);
    // enough blocks for two per SM over the stack, at least 8 rows (one per warp) each
    const int sms = sm_count_or_default();
    int64_t blocks = ceil_div(io.rows, 8);
    if (blocks > ceil_div(4 * sms, a->count)) blocks = ceil_div(4 * sms, a->count);
    if (blocks > MOST_SUMS) blocks = MOST_SUMS;
    const int64_t pieces = (int64_t)(io.mp / 64) * (io.np / 64) * a->count;
    if (pieces > 0x7fffffff || a->count * blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    Maps xm[2], sm, pm;
    if (a->steps > 0 && !(sm.encode(s, a->count, io.mp, io.mp) && pm.encode(p, a->count, io.mp, io.mp) && xm[0].encode(x[0], a->count, io.mp, io.np) &&
                          xm[1].encode(x[1], a->count, io.mp, io.np)))
        return cudaErrorNotSupported;
    FPDE_TRY(launch_kernel(ortho_square_kernel<T>, dim3((unsigned)(a->count * blocks)), dim3(256), st, io, sums, (int)blocks, lost));
    FPDE_TRY(launch_kernel(ortho_start_kernel<T>, dim3((unsigned)pieces), dim3(256), st, io, (const double*)sums, (int)blocks, x[0]));
    if (lose) FPDE_TRY(launch_kernel(ortho_lose_kernel, dim3(1), dim3(1), st, lost));
    int at = 0;
    for (int i = 0; i < a->steps; ++i, at ^= 1) {
        constexpr bool PAIR = sizeof(T) == 4;
        const ProductShape gram = shape_of(GRAM, io.mp, io.np), square = shape_of(SQUARE, io.mp, io.np), apply = shape_of(APPLY, io.mp, io.np);
        FPDE_TRY((run_product<PAIR, GRAM>(xm[at], xm[at], s, s, lost, gram, a->count, sms, st)));
        if (PAIR || square_of_pairs(io.mp)) FPDE_TRY((run_product<true, SQUARE>(sm, sm, s, p, lost, square, a->count, sms, st)));
        else FPDE_TRY((run_product<false, SQUARE>(sm, sm, s, p, lost, square, a->count, sms, st)));
        if (PAIR || apply_of_pairs(io.mp)) FPDE_TRY((run_product<true, APPLY>(pm, xm[at], x[at], x[at ^ 1], lost, apply, a->count, sms, st)));
        else FPDE_TRY((run_product<PAIR, APPLY>(pm, xm[at], x[at], x[at ^ 1], lost, apply, a->count, sms, st)));
    }
    return launch_kernel(ortho_finish_kernel<T>, dim3((unsigned)pieces), dim3(256), st, io, (const __half*)x[at], (const unsigned int*)lost);
}

int call(const fpde_ortho_args* a, bool muon, void* stream, bool lose = false) {
    const int st = check(a);
    if (st != FPDE_OK) return st;
    if (a->count * a->rows * a->cols == 0) return FPDE_OK;
    const size_t e = dtype_bytes(a->dtype);
    if (a->grad == nullptr || (muon ? a->weight == nullptr || a->momentum == nullptr : a->out == nullptr)) return FPDE_ERR_NULL;
    if (!aligned(a->grad, e) || !aligned(a->out, e) || !aligned(a->weight, e) || !aligned(a->momentum, 4)) return FPDE_ERR_ALIGN;
    const size_t need = fpde_orthogonalize_workspace_bytes(a);
    if (need > 0 && (a->workspace == nullptr || !aligned(a->workspace, 256) || a->workspace_bytes < need))
        return FPDE_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t err = a->dtype == FPDE_F32 ? run<float>(a, muon, lose, s) : a->dtype == FPDE_BF16 ? run<__nv_bfloat16>(a, muon, lose, s) : run<__half>(a, muon, lose, s);
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

int fpde_diag_ortho_form(const fpde_ortho_args* a, int product) {
    if (check(a) != FPDE_OK || product < GRAM || product > APPLY) return -1;
    const int64_t m = a->rows < a->cols ? a->rows : a->cols, n = a->rows < a->cols ? a->cols : a->rows;
    if (m == 0 || a->count == 0 || is_small(m, n)) return -1;
    const int mp = (int)padded(m), np = (int)padded(n), sms = sm_count_or_default();
    const ProductShape s = shape_of(product, mp, np);
    const bool pair = a->dtype == FPDE_F32 || (product == SQUARE && square_of_pairs(mp)) || (product == APPLY && apply_of_pairs(mp));
    if (product == GRAM) return pair ? best_form<true, GRAM>(s, a->count, sms) : best_form<false, GRAM>(s, a->count, sms);
    if (product == SQUARE) return pair ? best_form<true, SQUARE>(s, a->count, sms) : best_form<false, SQUARE>(s, a->count, sms);
    return pair ? best_form<true, APPLY>(s, a->count, sms) : best_form<false, APPLY>(s, a->count, sms);
}

int fpde_orthogonalize(const fpde_ortho_args* a, void* stream) { return call(a, false, stream); }
int fpde_muon_step(const fpde_ortho_args* a, void* stream) { return call(a, true, stream); }
int fpde_diag_orthogonalize_lost(const fpde_ortho_args* a, void* stream) { return call(a, false, stream, true); }
unsigned int fpde_diag_ortho_timeouts(void) {
    unsigned int n = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&n, g_ortho_timeouts, sizeof n) != cudaSuccess) {
        (void)cudaGetLastError();
        return ~0u;
    }
    return n;
}

}  // extern "C"
