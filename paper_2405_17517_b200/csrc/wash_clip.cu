// Clipping: the gradients of the models whose factor is below 1 are multiplied by it, in place; the other models' bits stay as they are.
#include "wash_octet.cuh"

namespace wash {

template <class T>
__global__ void __launch_bounds__(kChunkThreads) clip_np_kernel(const __grid_constant__ ClipArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t N = static_cast<uint32_t>(a.pop.N), c = blockIdx.x / N, n = blockIdx.x - c * N;
    const float factor = clip_factor(a.norm[n], a.max_norm);
    if (factor == 1.f) return;
    const uint32_t unit = c * kChunkThreads + threadIdx.x;
    if (unit >= a.pop.n_groups / 2) return;
    char *at = static_cast<char *>(a.grads) + (static_cast<size_t>(n) * a.pop.padded_P + 8ull * unit) * T::kBytes;
    Octet<T> g;
    g.load(at);
    float decay, r[8];
    const uint32_t mask = existing_np(a.pop, 8ll * unit, a.status, &decay);
#pragma unroll
    for (int q = 0; q < 8; ++q) r[q] = __fmul_rn(factor, g.get(q));
    g.put(r, 0xFFu);
    if (mask == 0xFFu) g.store(at);
    else g.store_some(at, mask);
}

template <class T>
__global__ void __launch_bounds__(kChunkThreads) clip_pn_kernel(const __grid_constant__ ClipArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t N = static_cast<uint32_t>(a.pop.N), units = chunk_units(kLayoutPN, a.pop.N);
    __shared__ float factor[kMaxN];
    if (threadIdx.x < N) factor[threadIdx.x] = clip_factor(a.norm[threadIdx.x], a.max_norm);
    if (!__syncthreads_or(threadIdx.x < N && factor[threadIdx.x] != 1.f)) return;
    const uint32_t e0 = 8u * threadIdx.x / N, n0 = 8u * threadIdx.x - e0 * N;
    const uint32_t first = blockIdx.x * units, here = min(units, a.pop.n_groups / 2 - first) * N;
    if (threadIdx.x >= here) return;
    char *at = static_cast<char *>(a.grads) + (static_cast<size_t>(first) * N + threadIdx.x) * 8 * T::kBytes;
    Octet<T> g;
    g.load(at);
    float decay[8], r[8];
    const uint32_t mask = existing_pn(a.pop, 8ll * first + e0, n0, a.status, decay);
    uint32_t active = 0, n = n0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float c = factor[n];
        if (c != 1.f) active |= 1u << q;
        r[q] = __fmul_rn(c, g.get(q));
        if (++n == N) n = 0;
    }
    if (!active) return;
    g.put(r, active);
    if (mask == 0xFFu) g.store(at);
    else g.store_some(at, mask & active);
}

template <class T>
static cudaError_t launch_typed(const ClipArgs &args, cudaStream_t stream)
{
    const uint32_t units = args.pop.n_groups / 2, per_chunk = chunk_units(args.pop.layout, args.pop.N);
    const uint64_t chunks = (units + per_chunk - 1) / per_chunk, grid = args.pop.layout == kLayoutNP ? chunks * args.pop.N : chunks;
    if (grid > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    if (args.pop.layout == kLayoutNP) return launch_chained(clip_np_kernel<T>, static_cast<unsigned>(grid), kChunkThreads, 0, stream, args);
    return launch_chained(clip_pn_kernel<T>, static_cast<unsigned>(grid), kChunkThreads, 0, stream, args);
}

cudaError_t launch_clip(const ClipArgs &args, int dtype, int, cudaStream_t stream)
{
    return dtype == kDtypeF32 ? launch_typed<F32>(args, stream) : launch_typed<BF16>(args, stream);
}

}  // namespace wash
