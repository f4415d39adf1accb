// Every model's gradient norm over a range of tensors: norm_n = sqrt(sum_i g_n,i^2), squares and sums in binary64 (a square of a binary32
// value is exact there and neither overflows nor underflows), added in an order that depends on the launch's shape only.
//
// One pass: a resident grid walks the chunks, a thread adds up its octets' squares, a block leaves one partial sum a model, and the block that reports last
// adds the blocks' partials and takes the root.
#include "wash_octet.cuh"

namespace wash {

__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

// The block that reports last sums the partials, a warp a model, and leaves the ticket at 0.
__device__ __forceinline__ void finish_norms(const NormArgs &a)
{
    __shared__ bool last;
    __syncthreads();   // the block's partials are stored
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicInc(a.ticket, gridDim.x - 1u) == gridDim.x - 1u;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    const uint32_t lane = threadIdx.x & 31u;
    for (int n = static_cast<int>(threadIdx.x >> 5); n < a.pop.N; n += kChunkThreads / 32) {
        double s = 0.0;
        for (uint32_t b = lane; b < a.per_model; b += 32) s += __ldcg(a.partial + static_cast<size_t>(n) * a.per_model + b);
        s = warp_sum(s);
        if (lane == 0) a.out[n] = sqrt(s);
    }
}

template <class T>
__global__ void __launch_bounds__(kChunkThreads) norm_np_kernel(const __grid_constant__ NormArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t n = blockIdx.x / a.per_model, b = blockIdx.x - n * a.per_model;
    const char *row = static_cast<const char *>(a.grads) + static_cast<size_t>(n) * a.pop.padded_P * T::kBytes;
    double sum = 0.0;
    for (uint32_t c = b; c < a.n_chunks; c += a.per_model) {
        const uint32_t unit = a.unit_lo + c * kChunkThreads + threadIdx.x;
        if (unit >= a.unit_hi) break;
        Octet<T> g;
        g.load(row + static_cast<size_t>(unit) * 8 * T::kBytes);
        float decay;
        const uint32_t mask = existing_np(a.pop, 8ll * unit, a.status, &decay);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const double x = (mask >> q) & 1u ? static_cast<double>(g.get(q)) : 0.0;
            sum = fma(x, x, sum);
        }
    }
    __shared__ double part[kChunkThreads / 32];
    sum = warp_sum(sum);
    if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < kChunkThreads / 32; ++w) s += part[w];
        a.partial[static_cast<size_t>(n) * a.per_model + b] = s;
    }
    finish_norms(a);
}

template <class T>
__global__ void __launch_bounds__(kChunkThreads) norm_pn_kernel(const __grid_constant__ NormArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t N = static_cast<uint32_t>(a.pop.N), units = chunk_units(kLayoutPN, a.pop.N), octets = units * N;
    const uint32_t e0 = 8u * threadIdx.x / N, n0 = 8u * threadIdx.x - e0 * N;
    double sum[8];   // of model (n0 + q) mod N
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.0;
    for (uint32_t c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
        const uint32_t first = a.unit_lo + c * units, here = min(units, a.unit_hi - first) * N;
        if (threadIdx.x >= here) break;
        Octet<T> g;
        g.load(static_cast<const char *>(a.grads) + (static_cast<size_t>(first) * N + threadIdx.x) * 8 * T::kBytes);
        float decay[8];
        const uint32_t mask = existing_pn(a.pop, 8ll * first + e0, n0, a.status, decay);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const double x = (mask >> q) & 1u ? static_cast<double>(g.get(q)) : 0.0;
            sum[q] = fma(x, x, sum[q]);
        }
    }
    __shared__ double part[8 * kChunkThreads];   // value f of the chunk's 8 * octets: model f mod N
#pragma unroll
    for (int q = 0; q < 8; ++q) part[8u * threadIdx.x + q] = sum[q];
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31u;
    for (uint32_t n = threadIdx.x >> 5; n < N; n += kChunkThreads / 32) {   // 8 * units values a model
        double s = 0.0;
        for (uint32_t i = lane; i < 8u * units; i += 32) s += part[i * N + n];
        s = warp_sum(s);
        if (lane == 0) a.partial[static_cast<size_t>(n) * a.per_model + blockIdx.x] = s;
    }
    finish_norms(a);
}

template <class T>
static cudaError_t launch_typed(const NormArgs &args, uint32_t grid, cudaStream_t stream)
{
    if (args.pop.layout == kLayoutNP) return launch_chained(norm_np_kernel<T>, grid, kChunkThreads, 0, stream, args);
    return launch_chained(norm_pn_kernel<T>, grid, kChunkThreads, 0, stream, args);
}

cudaError_t launch_grad_norm(NormArgs args, int dtype, int sm_count, cudaStream_t stream)
{
    const uint32_t units = args.unit_hi - args.unit_lo, per_chunk = chunk_units(args.pop.layout, args.pop.N);
    const uint32_t sm = static_cast<uint32_t>(sm_count), N = static_cast<uint32_t>(args.pop.N);
    args.n_chunks = (units + per_chunk - 1) / per_chunk;
    uint32_t most = args.pop.layout == kLayoutNP ? kNormBlocksNP * sm / N : kNormBlocksPN * sm;
    if (most < 1) most = 1;
    args.per_model = args.n_chunks < most ? args.n_chunks : most;
    if (args.per_model < 1) args.per_model = 1;   // an empty range: one block finds nothing
    const uint32_t grid = args.pop.layout == kLayoutNP ? args.per_model * N : args.per_model;
    return dtype == kDtypeF32 ? launch_typed<F32>(args, grid, stream) : launch_typed<BF16>(args, grid, stream);
}

}  // namespace wash
