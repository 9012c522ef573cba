// Sums of row losses, shared by the objectives.
#pragma once

#include "sat_internal.h"

// Loss kernels.  The rows go round-robin over the lane groups of at most LOSS_MAX_BLOCKS blocks (one resident wave).  Row losses
// are summed in double per thread, then per warp, the warps of a block in fixed order, and the last block to finish adds the block
// partials in fixed order: which rows a thread owns depends on the row count alone, so the total does not depend on scheduling.
#define LOSS_MAX_BLOCKS(ctx) ((ctx)->sms * 6)

#ifdef __CUDACC__
// NT: threads of the block, a power of two
template <int NT = 256>
__device__ __forceinline__ void loss_finish(double thread_sum, double *__restrict__ block_partial, int *__restrict__ ticket, double *total, int overwrite)
{
    __shared__ double red[NT];
    __shared__ int last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int o = 16; o > 0; o >>= 1) thread_sum += __shfl_xor_sync(0xffffffffu, thread_sum, o);
    if (lane == 0) red[warp] = thread_sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int w = 0; w < NT / 32; ++w) s += red[w];
        block_partial[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += NT) s += __ldcg(block_partial + i);
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = NT / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *ticket = 0;   // the next launch on this stream starts from zero again
        if (total) *total = overwrite ? red[0] : *total + red[0];
    }
}

// The same where the sums are one thread's of each block, `who`: any number of whole warps, little shared memory.
template <int who>
__device__ __forceinline__ void loss_finish_first(double sum, double *__restrict__ block_partial, int *__restrict__ ticket, double *total)
{
    __shared__ int last;
    if (threadIdx.x == who) {
        block_partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last || threadIdx.x >= 32) return;
    __threadfence();
    double s = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += 32) s += __ldcg(block_partial + i);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) {
        *ticket = 0;
        *total += s;
    }
}
#endif
