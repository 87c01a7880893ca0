// The march that linear attention and its gradients are made of, as its two kernels see it.
#pragma once
#include "seq_common.cuh"

namespace fpde {

struct LinearView {
    const void* p;
    int64_t batch, node, head;
};

// A march over all rows and heads.
struct March {
    LinearView a, b, c;
    int64_t batch, length, heads;
    int da, dc;                    // features of a and b, and of c
    bool mma;                      // on the tensor cores
    int reversed;                  // from the last node to the first
    int shift;
    float near, far, gain;
    const float* log_decay;
    const float* start;            // (batch, heads, da, dc), or turned: (batch, heads, dc, da); NULL: zeros
    int start_turned;
    void* out;                     // (batch, length, heads, dc) dense
    float* end;                    // (batch, heads, da, dc), or NULL
    // pieces of a row: states at their starts in `local` (batch, heads, pieces, da, dc), or turned
    int pieces;
    int64_t piece;                 // nodes of a piece
    float* local;
    int local_turned;
    bool local_there;              // another march's, which has been joined
    bool out_packed;               // rows of out start on 32 bytes
    int lose;                      // a wait that nothing ends, in the march 1 or in the pass for the pieces' ends 2; 0 but in a test
};

// g^n for n >= 0, from 64 bits: rounded once, so that it stays exact enough when it is applied chunk after chunk.
__device__ __forceinline__ double power(float log_decay, double n) { return n == 0. ? 1. : exp((double)log_decay * n); }

// What each piece leaves becomes the state that each starts from.
cudaError_t march_join(const March& m, cudaStream_t st);

// The march of bf16 arrays on the tensor cores (seq_linear_mma.cu).  Its pieces are multiples of MMA_CHUNK nodes.  False, with
// nothing launched: the copy engine cannot read one of the arrays (steps as below, or a start on no multiple of 16 bytes).
constexpr int MMA_CHUNK = 128;
constexpr int MMA_BLOCKS = 148;                      // resident on the GPU
bool march_mma(const March& m, cudaStream_t st, cudaError_t* e);
// Can the copy engine step through a bf16 array: strides of whole 16 bytes, or zero, but for the nodes', which a tile needs one by one.
bool tile_steps(const LinearView& x, int64_t heads, int64_t length, int64_t batch);
unsigned int march_mma_timeouts();

}  // namespace fpde
