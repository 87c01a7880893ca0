// Linear attention's march on the tensor cores, for bf16 arrays with up to 128 features.
//
// A block marches one row and head, or a piece of it, in chunks of 128 nodes.  The chunk's a, b and c lie in shared memory as
// they come (rows of nodes, 64-feature blocks, 128-byte swizzle), zeros where there is no node or feature.  Products of a chunk:
//   G = a b^T        128 x 128, both factors K-major
//   far = a S        S, the state before the chunk, in shared memory, MN-major
//   U = bw^T c       what the chunk adds to the state; bw = b with the decays to the chunk's end, MN-major
//   near = P c       P = G with the decays between the nodes, as left factor in TMEM; c MN-major
// Sums are fp32 in TMEM.  out = near + g^(i+1-shift) far, S <- g^128 S + U in fp32 registers.  A march from the last node to the
// first takes the same tiles with their rows in the arrays' order: the masks and the decays are turned round instead.
//
// Roundings to fewer bits.  P and the S that `far` reads are single bf16 factors: each moves a bf16 result by about as much as
// its own rounding, and nothing else.  The state itself stays fp32: bw is three bf16 parts that hold all 24 bits of b times its
// decay, c is exact, U is formed of three products and the state is added up with ordinary rounding.  In a march whose last
// state nobody takes (gq and gk) bw is two parts of 8 bits, a hundredth of the rounding that the state sees in `far`.
//
// Threads.  One block an SM; its warps have tasks of their own, so that a chunk's steps run beside one another and beside those of
// the chunks before and after: eight turn G into P, eight turn b into bw, eight write the output and move the state on (two
// threads for each lane of TMEM), one issues the products and one loads (TMA).  A tile's place takes the next chunk's as soon as
// the products that read it are done.  (With all warps at the same step, one after the other, they wait for one another's
// latencies: 11 800 cycles a chunk of 128 x 128 features at a quarter of the issue slots.)  A chunk of 128 x 128 features takes 7 700 to
// 8 500 clocks, 3 072 of them products; no task bounds it alone.  A call of 8 x 2048 nodes of 32 heads of 128 takes 183 to 187 us, memory's
// floor 87; 16384 nodes of 16 heads of 64, with their pieces' ends, 71 of 20.
#include "mma_common.cuh"
#include "seq_linear.cuh"

namespace fpde {
namespace {

constexpr int N = MMA_CHUNK;
constexpr int BLOCK = N * 128;                 // bytes of 64 features of a chunk
// A wait (for microseconds, in a healthy run) gives up after TRIES tries of a microsecond each, or less where the hardware holds a
// try for less: 0.26 s at most, 5 ms at the very least.
constexpr int TRIES = 1 << 18, TRY_NS = 1000;

__device__ unsigned int g_linear_timeouts;

// A loop of its own in a few instructions: a block's tasks share an instruction cache, and there are some thirty waits.
__device__ __forceinline__ void wait_for(uint32_t bar, uint32_t parity, bool& gave_up) {
    if (gave_up) return;
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .u32 n;\n\t"
        "mov.u32 n, %4;\n\t"
        "AGAIN:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\t"
        "setp.ne.u32 p, n, 0;\n\t"
        "@p bra AGAIN;\n\t"
        "DONE:\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(TRY_NS), "n"(TRIES) : "memory");
    gave_up = done == 0;
}

template <int DA, int DC, int PARTS>
struct Room {
    static constexpr int STATE = (DA * (DC + 1) * 4 + 1023) / 1024 * 1024, PLANES = PARTS * (DA / 64) * BLOCK;      // fp32 state and bw share a place
    static constexpr int TILES = (2 * DA + DC) / 64 * BLOCK, REST = (PLANES > STATE ? PLANES : STATE) + DC / 64 * DA * 128 + 1024;
    static constexpr int STAGES = 2 * TILES + REST <= 226 * 1024 ? 2 : 1;       // places of each tile: 16 x 2048 x 16 x 64 102 us with one, 98 with two
    static constexpr int A = 0, B = A + STAGES * (DA / 64) * BLOCK, V = B + STAGES * (DA / 64) * BLOCK, BW = V + STAGES * (DC / 64) * BLOCK;
    static constexpr int S = BW + (PLANES > STATE ? PLANES : STATE);
    static constexpr int BYTES = S + DC / 64 * DA * 128 + 1024;      // slack to start on 1024 bytes
    static constexpr int G = 0, NEAR = 128, FAR = NEAR + DC, U = FAR + DC;      // columns of TMEM; P lies over G
};
// Groups of eight warps (2 is OUT), the last of four, and their registers: 896 threads start with 72 each.
constexpr int GROUP_P = 0, GROUP_BW = 1, GROUP_CONTROL = 3, CONTROL = 24, THREADS = 28 * 32;
constexpr int OUT_REGS = 128, P_REGS = 64, OTHER_REGS = 40;
static_assert(256 * (OUT_REGS + P_REGS) + 384 * OTHER_REGS <= THREADS * 72, "the groups share what the block starts with");
// P lies over G, each 32 columns' 16 over their own: the column of 16 nodes' products.
__host__ __device__ constexpr int p_column(int k) { return 32 * (k / 2) + 8 * (k % 2); }

// Barriers.  FULL: a tile has arrived; DONE: the products up to these are done; READY: warps have written what products read;
// FREE: warps have read what products write.  AGAIN: rows with an infinity or NaN behind them have been summed again; its phases are those
// of such chunks.
enum Bar { FULL_A, FULL_B, FULL_C, DONE_G, DONE_FAR, DONE_NEAR, DONE_U, READY_P, READY_BW, READY_S, SCANNED, FREE_OUT, AGAIN, ENDED, BARS };

__device__ __forceinline__ void sts16(uint32_t to, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t from) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
    return v;
}
// Where row r's 8 features from 8 * q on lie in an array of `rows` rows.
__device__ __forceinline__ uint32_t chunk_at(uint32_t base, int r, int q, int rows = N) { return base + (q / 8) * rows * 128 + r * 128 + ((q % 8) ^ (r & 7)) * 16; }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// D += A B, by the one lane of a warp that asks for it; all come here, so that operands are the warp's.  An instruction's operands
// are moved one by one otherwise: 100 clocks a product in a loop of one thread, against the 64 that it takes.
__device__ __forceinline__ void product(bool leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)leader)
        : "memory");
}
// The same with A in TMEM: 16 bf16 of each row, two a column.
__device__ __forceinline__ void product_tmem(bool leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add),
        "r"((uint32_t)leader)
        : "memory");
}
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tmem_store8(uint32_t addr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_ask16(uint32_t addr, uint32_t (&r)[16]) {          // there after tmem_asked()
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_asked() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    tmem_ask16(addr, r);
    tmem_asked();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load_both(uint32_t addr, float (&v)[16], uint32_t other, float (&w)[16]) {
    uint32_t r[16], q[16];
    tmem_ask16(addr, r);
    tmem_ask16(other, q);
    tmem_asked();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = __uint_as_float(r[i]);
        w[i] = __uint_as_float(q[i]);
    }
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t tmem_load1(uint32_t addr) {
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    return r;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 64 features of a tile's 128 nodes; what the map does not hold becomes zeros.
__device__ __forceinline__ void load_tile(uint32_t to, const CUtensorMap* map, int feature, int head, int node, int batch, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to), "l"(map),
                 "r"(feature), "r"(head), "r"(node), "r"(batch), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void store32(void* to, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7])
                 : "memory");
}

__device__ __forceinline__ float top_part(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ uint32_t tops(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }

// Eight features of b times their node's weight, as PARTS bf16 each.
template <int PARTS>
__device__ __forceinline__ void weigh(uint32_t (&out)[PARTS][4], uint4 v, float w, __nv_bfloat162 w1, __nv_bfloat162 w2) {
    const uint32_t in[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (PARTS == 3) {                            // 8 bits at a time, exactly
            uint64_t x = mul2(pair(__uint_as_float(in[k] << 16), __uint_as_float(in[k] & 0xffff0000u)), both(w));
#pragma unroll
            for (int s = 0; s < PARTS; ++s) {
                float lo, hi;
                unpair(x, lo, hi);
                out[s][k] = tops(lo, hi);
                if (s < PARTS - 1) x = add2(x, pair(-top_part(lo), -top_part(hi)));
            }
        } else {                                               // b w1 and what its rounding left, exactly, plus b w2
            const __nv_bfloat162 y = reinterpret_cast<const __nv_bfloat162&>(in[k]), first_part = __hmul2(y, w1);
            const __nv_bfloat162 second = __hfma2(y, w2, __hfma2(y, w1, __hneg2(first_part)));
            out[0][k] = reinterpret_cast<const uint32_t&>(first_part);
            out[1][k] = reinterpret_cast<const uint32_t&>(second);
        }
    }
}

struct Tiles {
    CUtensorMap a, b, c;                       // (features, heads, nodes, batch)
    int head_a, head_b, head_c, batch_a, batch_b, batch_c;      // 0: one for all
};

// A row's output where c holds an infinity or NaN.  The product with a node behind is 0 times what c holds there, which is none of
// this row's: those sums are formed once more, over the nodes up to the row's own, from the same P.
template <int DC>
__device__ __forceinline__ void sum_again(const March& m, const __nv_bfloat16* c, int64_t node, __nv_bfloat16* to, int n, int r, uint32_t lanes, int col0, float w) {
    using R = Room<64, DC, 2>;                 // the columns of TMEM are those of every DA
    for (int e = 0; e < DC / 2 && col0 + e < m.dc; e += 16) {
        const int left = m.dc - col0 - e;
        float o[16], f[16], again[16] = {};
        tmem_load_both(R::NEAR + lanes + col0 + e, o, R::FAR + lanes + col0 + e, f);
        uint32_t bad = 0;                      // features of which a row is none, until a node up to j has made them so
#pragma unroll
        for (int k = 0; k < 16; ++k) bad |= (o[k] - o[k] != 0.f) << k;
        bad = __reduce_or_sync(~0u, bad);
#pragma unroll 1
        for (int j = 0; j < n && bad != 0; ++j) {
            const int at = m.reversed ? N - 1 - j : j;
            const uint32_t two = tmem_load1(R::G + lanes + p_column(at / 16) + at % 16 / 2);
            const float x = at % 2 ? __uint_as_float(two & 0xffff0000u) : __uint_as_float(two << 16);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const float y = k < left ? __bfloat162float(c[j * node + col0 + e + k]) : 0.f;
                if (j <= r) again[k] = fmaf(x, y, again[k]);
                if (y - y != 0.f) bad &= ~(1u << k);
            }
        }
        // a row before j has its sum; in the others an infinity or NaN is their own
        if (r < n)
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k < left && o[k] - o[k] != 0.f) to[col0 + e + k] = __float2bfloat16_rn(fmaf(again[k], m.near, w * f[k]));
    }
}

template <int DA, int DC, int PARTS>
__global__ void __launch_bounds__(THREADS, 1) march_mma_kernel(const __grid_constant__ March m, const __grid_constant__ Tiles tiles) {
    using R = Room<DA, DC, PARTS>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) float powers[N + 2];
    __shared__ int odd_chunk[2];                                 // the last chunk of either parity with an infinity or NaN in c, counted from 1
    __shared__ float whole[4];                                   // g^128 and that of the last chunk, each in two parts
    const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, group = warp / 8, half = warp / 4 % 2, quarter = warp % 4;
    auto bar = [&](int i, int c) { return smem_u32(&bars[2 * i + (c & 1)]); };
    if (tid == 0) {
        odd_chunk[0] = odd_chunk[1] = 0;
        for (int i = 0; i < 2 * BARS; ++i) mbar_init(bar(i / 2, i), i / 2 >= READY_P && i / 2 <= AGAIN ? 8 : 1);
        mbar_fence_init();
    }
    if (warp == CONTROL) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait_then_trigger();

    const unsigned rest = blockIdx.x / (unsigned)m.pieces;
    const int p = (int)(blockIdx.x - rest * (unsigned)m.pieces);
    const int64_t bt = rest / (unsigned)m.heads, h = rest - (unsigned)bt * (unsigned)m.heads;
    const int64_t first = p * m.piece, last = min(m.length, first + m.piece);
    const int chunks = (int)((last - first + N - 1) / N), tail = (int)(last - first) - (chunks - 1) * N;
    const float ld = m.log_decay[h];
    {
        if (tid < N + 4) {
            const double g = power(ld, tid < N + 2 ? tid : tid == N + 2 ? N : max(tail, 0));
            if (tid < N + 2) {
                powers[tid] = (float)g;
            } else {
                whole[2 * (tid - N - 2)] = (float)g;
                whole[2 * (tid - N - 2) + 1] = (float)(g - (float)g);
            }
        }
    }
    // The state comes and goes through bw's place, along its rows or, turned, its columns.
    constexpr int PITCH = DC + 1;
    float* stage = reinterpret_cast<float*>(raw + (base - smem_u32(raw)) + R::BW);
    const int64_t st = (bt * m.heads + h) * m.da * m.dc;
    {
        const float* local = m.local + ((bt * m.heads + h) * m.pieces + p) * m.da * m.dc;
        const float* from = m.pieces > 1 ? local : m.start != nullptr ? m.start + st : nullptr;
        const bool turned = m.pieces > 1 ? m.local_turned : m.start_turned;
        const int across = turned ? m.da : m.dc;
        if (from == nullptr || m.da < DA || m.dc < DC) {
            for (int i = tid; i < DA * PITCH; i += THREADS) stage[i] = 0.f;
            __syncthreads();
        }
        if (from != nullptr)
#pragma unroll 4
            for (int i = tid; i < m.da * m.dc; i += THREADS) {
                const int a = i / across, b = i - a * across;
                stage[turned ? b * PITCH + a : a * PITCH + b] = from[i];
            }
    }
    fence_before();
    __syncthreads();
    fence_after();
    constexpr uint32_t tmem = 0;               // all 512 columns: they start there
    uint32_t odd_phase = 0;
    bool gave_up = false;
    int asked_a = 0, asked_b = 0, asked_c = 0; // tiles that this thread has asked for
    auto wait = [&](int i, int c) { wait_for(bar(i, c), (c >> 1) & 1, gave_up); };
    auto wait_warp = [&](int i, int c) {
        wait(i, c);
        gave_up = __any_sync(~0u, gave_up);
        fence_after();
    };
    auto signal = [&](int i, int c) {
        fence_async();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(i, c));
    };
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const int row = quarter * 32 + lane, r = m.reversed ? N - 1 - row : row;      // of the tile, and in the march's order

    if (group == GROUP_CONTROL) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
        constexpr uint32_t IDESC = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(128 / 16) << 24;      // fp32 sums of bf16 factors, 128 rows
        constexpr uint32_t IDESC_G = IDESC | (uint32_t)(N / 8) << 17, IDESC_OUT = IDESC | 1u << 16 | (uint32_t)(DC / 8) << 17;
        constexpr uint32_t IDESC_U = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(DC / 8) << 17 | (uint32_t)(DA / 16) << 24;
        if (__shfl_sync(~0u, quarter, 0) == 0) {               // products
            const uint64_t da = slice_desc(base + R::A, false), db = slice_desc(base + R::B, false), dc = slice_desc(base + R::V, true, BLOCK),
                           ds = slice_desc(base + R::S, true, DA * 128), dw = slice_desc(base + R::BW, true, BLOCK);
            const bool leader = elected();
            auto commit = [&](int i, int c) {
                if (leader) mma_commit(bar(i, c));
            };
            auto all_wait = [&]() {
                __syncwarp();
                gave_up = __any_sync(~0u, gave_up);
                fence_after();
            };
            for (int c = 0; c < chunks; ++c) {
                wait(FULL_A, c);
                wait(FULL_B, c);
                if (c > 0) wait(DONE_NEAR, c - 1);           // G is written over P: products run in the order of their issue only where they share a sum
                if (c > 0 && *(volatile int*)&odd_chunk[(c - 1) & 1] == c) {         // P, near and far are still read
                    wait_for(bar(AGAIN, 0), odd_phase, gave_up);
                    odd_phase ^= 1;
                }
                all_wait();
                if (gave_up) break;
                const uint32_t at_a = c % R::STAGES * (DA / 64 * BLOCK), at_c = c % R::STAGES * (DC / 64 * BLOCK);
#pragma unroll
                for (int k = 0; k < DA / 16; ++k)
                    product(leader, tmem + R::G, desc_at(da, at_a + k / 4 * BLOCK + k % 4 * 32), desc_at(db, at_a + k / 4 * BLOCK + k % 4 * 32), IDESC_G, k > 0);
                commit(DONE_G, c);
                wait(READY_BW, c);
                wait(READY_S, c);                 // U before this one has been added, and S is the state before this chunk
                wait(FULL_C, c);
                all_wait();
                if (gave_up) break;
#pragma unroll
                for (int s = PARTS - 1; s >= 0; --s)           // the small parts first: the sum is rounded towards zero at every product
#pragma unroll
                    for (int k = 0; k < N / 16; ++k)
                        product(leader, tmem + R::U, desc_at(dw, s * (DA / 64) * BLOCK + k * 2048), desc_at(dc, at_c + k * 2048), IDESC_U, s < PARTS - 1 || k > 0);
                commit(DONE_U, c);
                if (c > 0) wait(FREE_OUT, c - 1);
                all_wait();
                if (gave_up) break;
#pragma unroll
                for (int k = 0; k < DA / 16; ++k)
                    product(leader, tmem + R::FAR, desc_at(da, at_a + k / 4 * BLOCK + k % 4 * 32), desc_at(ds, k * 2048), IDESC_OUT, k > 0);
                commit(DONE_FAR, c);
                wait(READY_P, c);
                all_wait();
                if (gave_up) break;
#pragma unroll
                for (int k = 0; k < N / 16; ++k) product_tmem(leader, tmem + R::NEAR, tmem + R::G + p_column(k), desc_at(dc, at_c + k * 2048), IDESC_OUT, k > 0);
                commit(DONE_NEAR, c);
            }
        } else if (quarter == 1 && lane == 0) {                // tiles
            auto load = [&](int full, int at, int blocks, const CUtensorMap* map, int head, int batch, int c) {
                const uint32_t to = base + at + c % R::STAGES * (blocks * BLOCK);
                mbar_expect_tx(bar(full, c), blocks * BLOCK);
                const int node = (int)(m.reversed ? m.length - first - N : first) + (m.reversed ? -N : N) * c;
                for (int f = 0; f < blocks; ++f) load_tile(to + f * BLOCK, map, 64 * f, head * (int)h, node, batch * (int)bt, bar(full, c));
            };
            // the places are an earlier chunk's: b is read by G and for bw, a by G and far, c by U, near and the scan
            for (int c = 0; c < chunks; ++c) {
                const int before = c - R::STAGES;
                if (before >= 0) {
                    wait(READY_BW, before);
                    wait(DONE_G, before);
                }
                if (gave_up) break;
                load(FULL_B, R::B, DA / 64, &tiles.b, tiles.head_b, tiles.batch_b, c);
                ++asked_b;
                if (before >= 0) wait(DONE_FAR, before);
                if (gave_up) break;
                load(FULL_A, R::A, DA / 64, &tiles.a, tiles.head_a, tiles.batch_a, c);
                ++asked_a;
                if (before >= 0) wait(DONE_NEAR, before);
                if (gave_up) break;
                load(FULL_C, R::V, DC / 64, &tiles.c, tiles.head_c, tiles.batch_c, c);
                ++asked_c;
            }
        }
    } else if (group == GROUP_BW) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
        for (int c = 0; c < chunks; ++c) {
            const int n = c < chunks - 1 ? N : tail;
            wait_warp(FULL_B, c);
            // bw's place is the last chunk's until U is done, the state's before that
            if (c > 0) wait(DONE_U, c - 1);
            else wait(READY_S, 0);
            gave_up = __any_sync(~0u, gave_up);
            if (gave_up) break;
            const float w = r < n ? m.gain * powers[n - 1 - r + m.shift] : 0.f;
            const __nv_bfloat162 w1 = __float2bfloat162_rn(w), w2 = __float2bfloat162_rn(w - __low2float(w1));
#pragma unroll 1
            for (int q = half * (DA / 16); q < (half + 1) * (DA / 16); ++q) {
                uint32_t out[PARTS][4];
                weigh<PARTS>(out, lds16(chunk_at(base + R::B + c % R::STAGES * (DA / 64 * BLOCK), row, q)), w, w1, w2);
#pragma unroll
                for (int s = 0; s < PARTS; ++s)
                    sts16(chunk_at(base + R::BW + s * (DA / 64) * BLOCK, row, q), make_uint4(out[s][0], out[s][1], out[s][2], out[s][3]));
            }
            signal(READY_BW, c);
        }
    } else if (group == GROUP_P) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P_REGS));
        // g^n as 2^(n log2 g), good to 2^-22 or, far back, to n log2 g 2^-24 of itself; the least finite number stands for log 0,
        // of which 2^(0 x) has to be 1
        const float l2 = fmaxf(ld * LOG2_E, -3e38f);
        uint64_t steps[8];                     // of 16 columns: whole blocks take these times the power of their nearest column
        auto make_steps = [&]() {
            float l = l2;
            asm volatile("" : "+f"(l));        // made anew each time
#pragma unroll
            for (int k = 0; k < 8; ++k)
                steps[k] = m.reversed ? pair(exp2_f32(2 * k * l), exp2_f32((2 * k + 1) * l)) : pair(exp2_f32((15 - 2 * k) * l), exp2_f32((14 - 2 * k) * l));
        };
        make_steps();
        if (m.lose == 1) wait_for(bar(ENDED, 0), 0, gave_up);
        for (int c = 0; c < chunks; ++c) {
            wait_warp(DONE_G, c);
            if (gave_up) break;
            // 32 columns at a time, a thread every other: those of this quarter's own nodes are cut along the diagonal, those of the
            // nodes before them are whole, the others zeros.  Column k of the 32 is the product times g^(32 before + lane - k), or + k - lane.
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                const int part = e / 2 * 2 + half, col = e % 2 * 16, before = m.reversed ? part - quarter : quarter - part;
                uint32_t packed[8] = {};
                if (before >= 0) {
                    float v[16];
                    tmem_load(tmem + R::G + lanes + part * 32 + col, v);
                    const float from = 32 * before + (m.reversed ? col - lane : lane - col), step = m.reversed ? 1.f : -1.f;
                    if (before > 0) {
                        const uint64_t w = both(exp2_f32((m.reversed ? from : from - 15.f) * l2));
#pragma unroll
                        for (int k = 0; k < 16; k += 2) unpair(mul2(pair(v[k], v[k + 1]), mul2(w, steps[k / 2])), v[k], v[k + 1]);
                    } else {
                        const uint32_t there = (m.reversed ? ~0u << lane : (2u << lane) - 1u) >> col;
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = (there >> k & 1u) != 0 ? v[k] * exp2_f32(fmaf(k, step, from) * l2) : 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) packed[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
                }
                tmem_store8(tmem + R::G + p_column(2 * part) + col / 2 + lanes, packed);
            }
            tmem_stored();
            wait_warp(SCANNED, c);                // before READY_P: the next chunk's cannot be over yet
            if (gave_up) break;
            signal(READY_P, c);
            if (*(volatile int*)&odd_chunk[c & 1] == c + 1) {
                wait_warp(FREE_OUT, c);           // and the rows are stored
                if (gave_up) break;
                const int64_t dir = m.reversed ? -1 : 1, node = (m.reversed ? m.length - 1 - first : first) + dir * (c * N);
                sum_again<DC>(m, (const __nv_bfloat16*)m.c.p + bt * m.c.batch + h * m.c.head + node * m.c.node, dir * m.c.node,
                              (__nv_bfloat16*)m.out + ((bt * m.length + node + dir * r) * m.heads + h) * m.dc, c < chunks - 1 ? N : tail, r, lanes, half * (DC / 2),
                              m.far * powers[r + 1 - m.shift]);
                signal(AGAIN, 0);
                make_steps();                  // rather than kept meanwhile
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(OUT_REGS));
        // The state: row d, half of the columns.  With 64 rows the products use 16 lanes of each quarter.
        constexpr int COLS = DC / 2;
        const bool holds = DA == 128 || lane < 16;
        const int d = DA == 128 ? quarter * 32 + lane : quarter * 16 + lane, col0 = half * COLS;
        float S[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) S[c] = stage[min(d, DA - 1) * PITCH + col0 + c];
        auto put_state = [&]() {               // the factor of `far`
            if (holds) {
#pragma unroll
                for (int q = 0; q < COLS / 8; ++q)
                    sts16(chunk_at(base + R::S, d, col0 / 8 + q, DA),
                          make_uint4(pack_bf16(S[8 * q], S[8 * q + 1]), pack_bf16(S[8 * q + 2], S[8 * q + 3]), pack_bf16(S[8 * q + 4], S[8 * q + 5]),
                                     pack_bf16(S[8 * q + 6], S[8 * q + 7])));
            }
        };
        put_state();
        signal(READY_S, 0);
        const int64_t dir = m.reversed ? -1 : 1, origin = m.reversed ? m.length - 1 - first : first;
        __nv_bfloat16* out = (__nv_bfloat16*)m.out + (bt * m.length * m.heads + h) * m.dc + col0;
        for (int c = 0; c < chunks; ++c) {
            const int n = c < chunks - 1 ? N : tail;
            // an infinity or NaN in c makes NaN of P's zeros for the nodes before it: their rows are summed again
            wait_warp(FULL_C, c);
            if (gave_up) break;
            __nv_bfloat162 sum = {}, zero = {};
#pragma unroll 2
            for (int q = half * (DC / 16); q < (half + 1) * (DC / 16); ++q) {
                const uint4 v = lds16(chunk_at(base + R::V + c % R::STAGES * (DC / 64 * BLOCK), row, q));
                sum = __hfma2(reinterpret_cast<const __nv_bfloat162&>(v.x), zero, sum);
                sum = __hfma2(reinterpret_cast<const __nv_bfloat162&>(v.y), zero, sum);
                sum = __hfma2(reinterpret_cast<const __nv_bfloat162&>(v.z), zero, sum);
                sum = __hfma2(reinterpret_cast<const __nv_bfloat162&>(v.w), zero, sum);
            }
            if ((reinterpret_cast<const uint32_t&>(sum) & 0x7fff7fffu) != 0) odd_chunk[c & 1] = c + 1;
            signal(SCANNED, c);
            wait_warp(DONE_U, c);
            wait_warp(DONE_FAR, c);                   // S is written over
            if (gave_up) break;
            const float hi = whole[n == N ? 0 : 2], lo = whole[n == N ? 1 : 3];
#pragma unroll
            for (int e = 0; e < COLS; e += 32) {
                float u[32];
                tmem_load32(tmem + R::U + lanes + col0 + e, u);
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    const uint64_t x = pair(S[e + k], S[e + k + 1]);
                    unpair(fma2(both(hi), x, fma2(both(lo), x, pair(u[k], u[k + 1]))), S[e + k], S[e + k + 1]);
                }
            }
            put_state();
            signal(READY_S, c + 1);
            wait_warp(DONE_NEAR, c);
            if (gave_up) break;
            const float w = m.far * powers[r + 1 - m.shift];
            __nv_bfloat16* to = out + (origin + dir * (c * N + r)) * m.heads * m.dc;
#pragma unroll 1
            for (int e = 0; e < COLS; e += 16) {
                const int left = m.dc - col0 - e;
                if (left <= 0) break;
                float o[16], f[16];
                tmem_load_both(tmem + R::NEAR + lanes + col0 + e, o, tmem + R::FAR + lanes + col0 + e, f);
#pragma unroll
                for (int k = 0; k < 16; k += 2) unpair(fma2(pair(o[k], o[k + 1]), both(m.near), mul2(pair(f[k], f[k + 1]), both(w))), o[k], o[k + 1]);
                if (r < n) {
                    if (left >= 16 && m.out_packed) {
                        uint32_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = pack_bf16(o[2 * k], o[2 * k + 1]);
                        store32(to + e, v);
                    } else {
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (k < left) to[e + k] = __float2bfloat16_rn(o[k]);
                    }
                }
            }
            signal(FREE_OUT, c);
        }
        if (holds)
#pragma unroll
            for (int c = 0; c < COLS; ++c) stage[d * PITCH + col0 + c] = S[c];      // U is done, and with it all that read bw
    }
    const bool lost = __syncthreads_or(gave_up);
    if (lost) {                 // what has been issued has to end before the block does; the results are NaN
        if (tid == 0) atomicAdd(&g_linear_timeouts, 1u);
        bool late = false;
        // a commit stands for the products of its own thread: the one that issued them, as a whole warp always elects the same
        if (warp == CONTROL && elected()) {
            mma_commit(bar(ENDED, 0));
            wait_for(bar(ENDED, 0), 0, late);
        }
        for (int s = 0; s < 2; ++s) {
            if (asked_a > s) wait_for(bar(FULL_A, s), ((asked_a - 1 - s) >> 1) & 1, late);
            if (asked_b > s) wait_for(bar(FULL_B, s), ((asked_b - 1 - s) >> 1) & 1, late);
            if (asked_c > s) wait_for(bar(FULL_C, s), ((asked_c - 1 - s) >> 1) & 1, late);
        }
        for (int64_t i = first * m.dc + tid; i < last * m.dc; i += THREADS) {
            const int64_t node = m.reversed ? m.length - 1 - i / m.dc : i / m.dc;
            ((__nv_bfloat16*)m.out)[((bt * m.length + node) * m.heads + h) * m.dc + i % m.dc] = __float2bfloat16_rn(NAN);
        }
    }
    float* to = p == m.pieces - 1 && m.end != nullptr ? m.end + st : nullptr;
    if (to != nullptr)
#pragma unroll 4
        for (int i = tid; i < m.da * m.dc; i += THREADS) to[i] = lost ? NAN : stage[i / m.dc * PITCH + i % m.dc];
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == CONTROL) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// The state that each piece but the last leaves, from zero: U alone.  Nothing but bw's products is there to wait for, so tiles and U have
// two places each: the tiles' way from memory, bw, its products and the sum of their results overlap.  bw has two places too: of
// a whole chunk with 64 features of b; of half a chunk's nodes with 128, where eight warps make the one half and eight the other
// (one place of a whole chunk: half of the nodes of 4 x 4096 x 16 x 128 47 us, 38 so).
template <int DA, int DC, int PARTS>
struct EndsRoom {
    static constexpr int TILE_B = DA / 64 * BLOCK, TILE_C = DC / 64 * BLOCK, FACTORS = PARTS * TILE_B, ROUNDS = DA == 64 ? 2 : 1;      // places of whole chunks
    static constexpr int B = 0, V = B + 2 * TILE_B, BW = V + 2 * TILE_C, BYTES = BW + ROUNDS * FACTORS + 1024;
    static_assert(DA * (DC + 1) * 4 <= BW, "the state leaves through the tiles' places");
};
enum EndsBar { E_FULL_B, E_FULL_C = E_FULL_B + 2, E_READY_BW = E_FULL_C + 2, E_DONE_U = E_READY_BW + 2, E_READ_U = E_DONE_U + 2, E_DONE_HALF = E_READ_U + 2, E_ENDED = E_DONE_HALF + 2, E_BARS };
constexpr int E_BW_WARPS = 16, E_SUM = 16, E_CONTROL = 24, E_BW_REGS = 48, E_SUM_REGS = 128, E_CONTROL_REGS = 40;
static_assert(512 * E_BW_REGS + 256 * E_SUM_REGS + 128 * E_CONTROL_REGS <= THREADS * 72, "the groups share what the block starts with");

template <int DA, int DC, int PARTS>
__global__ void __launch_bounds__(THREADS, 1) march_mma_ends_kernel(const __grid_constant__ March m, const __grid_constant__ Tiles tiles) {
    using R = EndsRoom<DA, DC, PARTS>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[E_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ float powers[N + 1];
    const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, quarter = warp % 4;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid == 0) {
        for (int i = 0; i < E_BARS; ++i)
            mbar_init(bar(i), i >= E_READY_BW && i < E_DONE_U ? E_BW_WARPS * R::ROUNDS / 2 : i >= E_READ_U && i < E_DONE_HALF ? E_CONTROL - E_SUM : 1);
        mbar_fence_init();
    }
    if (warp == E_CONTROL) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait_then_trigger();

    const unsigned pieces = m.pieces - 1, rest = blockIdx.x / pieces;      // nobody starts from the last one's end
    const int p = (int)(blockIdx.x - rest * pieces);
    const int64_t bt = rest / (unsigned)m.heads, h = rest - (unsigned)bt * (unsigned)m.heads, first = p * m.piece;
    const int chunks = (int)(m.piece / N);     // all of them whole
    if (tid < N + 1) powers[tid] = (float)power(m.log_decay[h], tid);
    fence_before();
    __syncthreads();
    fence_after();
    constexpr uint32_t tmem = 0;               // all 512 columns: they start there
    bool gave_up = false;
    int asked_b = 0, asked_c = 0;              // tiles that this thread has asked for
    // for chunk c's phase of the one of two barriers that even or odd chunks use
    auto wait = [&](int i, int c) { wait_for(bar(i + (c & 1)), (c >> 1) & 1, gave_up); };
    auto wait_warp = [&](int i, int c) {
        wait(i, c);
        gave_up = __any_sync(~0u, gave_up);
        fence_after();
    };
    auto signal = [&](int i, int c) {
        fence_async();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(i + (c & 1)));
    };
    constexpr int PITCH = DC + 1;
    float* stage = reinterpret_cast<float*>(raw + (base - smem_u32(raw)));

    float S[DC / 2];
    const bool holds = DA == 128 || lane < 16;               // with 64 rows the products use 16 lanes of each quarter
    const int d = DA == 128 ? quarter * 32 + lane : quarter * 16 + lane, col0 = warp / 4 % 2 * (DC / 2);
    if (warp >= E_CONTROL) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(E_CONTROL_REGS));
        constexpr uint32_t IDESC_U = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(DC / 8) << 17 | (uint32_t)(DA / 16) << 24;
        if (__shfl_sync(~0u, quarter, 0) == 0) {
            const bool leader = elected();
            for (int c = 0; c < chunks; ++c) {
                wait(E_FULL_C, c);
                if (c >= 2) wait(E_READ_U, c - 2);
                const uint64_t dc = slice_desc(base + R::V + (c & 1) * R::TILE_C, true, BLOCK),
                               dw = slice_desc(base + R::BW + (R::ROUNDS == 2 ? c & 1 : 0) * R::FACTORS, true, BLOCK);
#pragma unroll 1
                for (int half = 0; half < 3 - R::ROUNDS; ++half) {
                    if (R::ROUNDS == 2) wait(E_READY_BW, c);
                    else wait_for(bar(E_READY_BW + half), c & 1, gave_up);
                    __syncwarp();
                    gave_up = __any_sync(~0u, gave_up);
                    fence_after();
                    if (gave_up) break;
                    constexpr int K = N / 16 * R::ROUNDS / 2;
#pragma unroll
                    for (int s = PARTS - 1; s >= 0; --s)       // the small parts first: the sum is rounded towards zero at every product
#pragma unroll
                        for (int k = 0; k < K; ++k)
                            product(leader, tmem + (c & 1) * DC, desc_at(dw, s * R::TILE_B + (half * K + k) * 2048), desc_at(dc, (half * K + k) * 2048), IDESC_U,
                                    half > 0 || s < PARTS - 1 || k > 0);
                    if (R::ROUNDS == 1 && leader) mma_commit(bar(E_DONE_HALF + half));
                }
                if (gave_up) break;
                if (leader) mma_commit(bar(E_DONE_U + (c & 1)));
            }
        } else if (quarter == 1 && lane == 0) {
            for (int c = 0; c < chunks; ++c) {
                const int node = (int)(m.reversed ? m.length - first - N : first) + (m.reversed ? -N : N) * c;
                if (c >= 2) wait(R::ROUNDS == 2 ? E_READY_BW : E_DONE_U, c - 2);      // b has been read
                if (gave_up) break;
                mbar_expect_tx(bar(E_FULL_B + (c & 1)), R::TILE_B);
                for (int f = 0; f < DA / 64; ++f)
                    load_tile(base + R::B + (c & 1) * R::TILE_B + f * BLOCK, &tiles.b, 64 * f, tiles.head_b * (int)h, node, tiles.batch_b * (int)bt, bar(E_FULL_B + (c & 1)));
                ++asked_b;
                if (c >= 2) wait(E_DONE_U, c - 2);
                if (gave_up) break;
                mbar_expect_tx(bar(E_FULL_C + (c & 1)), R::TILE_C);
                for (int f = 0; f < DC / 64; ++f)
                    load_tile(base + R::V + (c & 1) * R::TILE_C + f * BLOCK, &tiles.c, 64 * f, tiles.head_c * (int)h, node, tiles.batch_c * (int)bt, bar(E_FULL_C + (c & 1)));
                ++asked_c;
            }
        }
    } else if (warp < E_SUM) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(E_BW_REGS));
        const int row = quarter * 32 + lane, r = m.reversed ? N - 1 - row : row, share = warp / 4;
        const float w = m.gain * powers[N - 1 - r + m.shift];
        const __nv_bfloat162 w1 = __float2bfloat162_rn(w), w2 = __float2bfloat162_rn(w - __low2float(w1));
        if (m.lose == 2) wait_for(bar(E_ENDED), 0, gave_up);
        for (int c = 0; c < chunks; ++c) {
            wait(E_FULL_B, c);
            // its place is free
            if (R::ROUNDS == 2 && c >= 2) wait(E_DONE_U, c - 2);
            if (R::ROUNDS == 1 && c >= 1) wait_for(bar(E_DONE_HALF + quarter / 2), (c - 1) & 1, gave_up);
            gave_up = __any_sync(~0u, gave_up);
            if (gave_up) break;
            fence_after();
            const uint32_t from = base + R::B + (c & 1) * R::TILE_B, to = base + R::BW + (R::ROUNDS == 2 ? c & 1 : 0) * R::FACTORS;
#pragma unroll 1
            for (int q = share * (DA / 32); q < (share + 1) * (DA / 32); ++q) {
                uint32_t out[PARTS][4];
                weigh<PARTS>(out, lds16(chunk_at(from, row, q)), w, w1, w2);
#pragma unroll
                for (int s = 0; s < PARTS; ++s) sts16(chunk_at(to + s * R::TILE_B, row, q), make_uint4(out[s][0], out[s][1], out[s][2], out[s][3]));
            }
            signal(E_READY_BW, R::ROUNDS == 2 ? c : quarter / 2);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(E_SUM_REGS));
        const double g = power(m.log_decay[h], N);
        const float hi = (float)g, lo = (float)(g - hi);
#pragma unroll
        for (int c = 0; c < DC / 2; ++c) S[c] = 0.f;
        for (int c = 0; c < chunks; ++c) {
            wait_warp(E_DONE_U, c);
            if (gave_up) break;
#pragma unroll
            for (int e = 0; e < DC / 2; e += 32) {
                float u[32];
                tmem_load32(tmem + (c & 1) * DC + ((uint32_t)(quarter * 32) << 16) + col0 + e, u);
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    const uint64_t x = pair(S[e + k], S[e + k + 1]);
                    unpair(fma2(both(hi), x, fma2(both(lo), x, pair(u[k], u[k + 1]))), S[e + k], S[e + k + 1]);
                }
            }
            signal(E_READ_U, c);
        }
        // U is done, and with it all that read the tiles
        if (holds)
#pragma unroll
            for (int c = 0; c < DC / 2; ++c) stage[d * PITCH + col0 + c] = S[c];
    }
    const bool lost = __syncthreads_or(gave_up);
    if (lost) {                 // as above
        if (tid == 0) atomicAdd(&g_linear_timeouts, 1u);
        bool late = false;
        if (warp == E_CONTROL && elected()) {
            mma_commit(bar(E_ENDED));
            wait_for(bar(E_ENDED), 0, late);
        }
        for (int s = 0; s < 2; ++s) {
            if (asked_b > s) wait_for(bar(E_FULL_B + s), ((asked_b - 1 - s) >> 1) & 1, late);
            if (asked_c > s) wait_for(bar(E_FULL_C + s), ((asked_c - 1 - s) >> 1) & 1, late);
        }
    }
    float* to = m.local + ((bt * m.heads + h) * m.pieces + p) * m.da * m.dc;
#pragma unroll 4
    for (int i = tid; i < m.da * m.dc; i += THREADS) to[i] = lost ? NAN : stage[i / m.dc * PITCH + i % m.dc];
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == E_CONTROL) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------------------------------- host
// The map of one array, (features, heads, nodes, batch).  An axis of stride zero has one entry for all.
bool tile_map(const LinearView& x, int width, int64_t heads, int64_t length, int64_t batch, CUtensorMap* map, int* head, int* row) {
    const EncodeTiledFn fn = tma_encode_fn();
    const int64_t strides[3] = {x.head, x.node, x.batch}, extents[3] = {heads, length, batch};
    if (fn == nullptr || !aligned(x.p, 16) || !tile_steps(x, heads, length, batch)) return false;
    cuuint64_t dims[4] = {(cuuint64_t)width}, bytes[3];
    for (int i = 0; i < 3; ++i) {
        const bool one = extents[i] == 1 || strides[i] == 0;
        dims[i + 1] = one ? 1 : (cuuint64_t)extents[i];
        bytes[i] = one ? 16 : (cuuint64_t)strides[i] * 2;
    }
    *head = dims[1] > 1;
    *row = dims[3] > 1;
    const cuuint32_t box[4] = {64, 1, N, 1}, step[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(x.p), dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Kernel>
cudaError_t launch(Kernel kernel, size_t bytes, int pieces, std::atomic<uint64_t>& done, const March& m, const Tiles& tiles, cudaStream_t st) {
    const cudaError_t e = allow_smem(kernel, bytes, done);
    if (e != cudaSuccess) return e;
    const int64_t blocks = m.batch * m.heads * pieces;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel_smem(kernel, dim3((unsigned)blocks), dim3(THREADS), bytes, st, m, tiles);
}

template <int DA, int DC, int PARTS>
cudaError_t run_parts(const March& m, const Tiles& tiles, cudaStream_t st) {
    if (m.pieces > 1 && !m.local_there) {
        static std::atomic<uint64_t> done{0};
        cudaError_t e = launch(march_mma_ends_kernel<DA, DC, PARTS>, EndsRoom<DA, DC, PARTS>::BYTES, m.pieces - 1, done, m, tiles, st);
        if (e == cudaSuccess) e = march_join(m, st);
        if (e != cudaSuccess) return e;
    }
    static std::atomic<uint64_t> done{0};
    return launch(march_mma_kernel<DA, DC, PARTS>, Room<DA, DC, PARTS>::BYTES, m.pieces, done, m, tiles, st);
}
// A state that leaves the march is fp32's; one that only `far` reads is rounded to bf16 there, and two parts of bw are enough.
template <int DA, int DC>
cudaError_t run(const March& m, const Tiles& tiles, cudaStream_t st) {
    return m.end != nullptr ? run_parts<DA, DC, 3>(m, tiles, st) : run_parts<DA, DC, 2>(m, tiles, st);
}

}  // namespace

bool tile_steps(const LinearView& x, int64_t heads, int64_t length, int64_t batch) {
    const int64_t strides[3] = {x.head, x.node, x.batch}, extents[3] = {heads, length, batch};
    for (int i = 0; i < 3; ++i) {
        if (extents[i] > 0x7fffffff - 2 * N) return false;
        if (extents[i] == 1) continue;
        if (i == 1 && strides[i] == 0) return false;
        if (strides[i] < 0 || strides[i] % 8 != 0 || strides[i] >= (1ll << 38)) return false;
    }
    return true;
}

bool march_mma(const March& given, cudaStream_t st, cudaError_t* e) {
    March m = given;
    Tiles tiles;
    if (!tile_map(m.a, m.da, m.heads, m.length, m.batch, &tiles.a, &tiles.head_a, &tiles.batch_a) ||
        !tile_map(m.b, m.da, m.heads, m.length, m.batch, &tiles.b, &tiles.head_b, &tiles.batch_b) ||
        !tile_map(m.c, m.dc, m.heads, m.length, m.batch, &tiles.c, &tiles.head_c, &tiles.batch_c))
        return false;
    m.out_packed = m.dc % 16 == 0 && aligned(m.out, 32);
    if (m.dc <= 64) *e = m.da <= 64 ? run<64, 64>(m, tiles, st) : run<128, 64>(m, tiles, st);
    else *e = m.da <= 64 ? run<64, 128>(m, tiles, st) : run<128, 128>(m, tiles, st);
    return true;
}

unsigned int march_mma_timeouts() {
    unsigned int n = 0;
    return cudaMemcpyFromSymbol(&n, g_linear_timeouts, sizeof n) == cudaSuccess ? n : 0xffffffffu;
}

}  // namespace fpde
