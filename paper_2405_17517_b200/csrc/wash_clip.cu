// Clipping: the gradients of the models whose factor is below 1 are multiplied by it, in place; the other models' bits stay as they are (in [P][N] those that share an octet
// with a clipped model's are written back as they were read: an octet's store is one or two 16-byte pieces).
// Bound by HBM: the clipped models' gradients are read and written once.  The grid walks the chunks from the last to the first: wash_grad_norm, which ran
// before, went from the first to the last and left the last in the L2.
//
// The number of blocks: a resident grid (one wave) reads and writes in step and loses a quarter of the bandwidth (fp32 [N][P], ResNet-50 N = 10: 1 wave 425 us, 4 365, 8 337,
// 16 326, a trip a block 311 = 6.58 TB/s), but blocks that find nothing to clip cost, too (1 wave 3.5 us, 16 9.4, a trip a block 46).  [P][N], whose threads look up eight factors
// first: fp32 N = 8 8 waves 250 us, 16 245, a trip a block 253; bf16 134 and 133.  bf16 [N][P] N = 8 129 us (6.35 TB/s), half of the models 65, none 10.
#include "wash_octet.cuh"

namespace wash {

// Octets a thread has in flight: 64 bytes.
template <class T>
constexpr int kTogether = 64 / (8 * T::kBytes);
constexpr int kClipBlocksNP = 4, kClipBlocksPN = 3;   // an SM; bf16 [P][N] of which three quarters are clipped 140 us with three, 146 with four
constexpr uint32_t kWavesNP = 16, kWavesPN = 8;

template <class T>
__device__ __forceinline__ void scale_octet(Octet<T> &g, const float (&c)[8], uint32_t active)
{
    float r[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) r[q] = __fmul_rn(c[q], g.get(q));
    g.put(r, active);
}

// [N][P]: the blocks share the chunks of the clipped models, of which each block makes itself a list; none clipped, and they end.
template <class T>
__global__ void __launch_bounds__(kChunkThreads, kClipBlocksNP) clip_np_kernel(const __grid_constant__ ClipArgs a, uint32_t trips)
{
    await_previous();
    let_next_start();
    constexpr int K = kTogether<T>;
    __shared__ float factors[kMaxN];
    __shared__ uint32_t models[kMaxN], count_shared;
    const uint32_t N = static_cast<uint32_t>(a.pop.N);
    if (threadIdx.x < 32) {
        uint32_t before = 0;
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half) {
            const uint32_t n = threadIdx.x + 32u * half;
            const float c = n < N ? clip_factor(a.norm[n], a.max_norm) : 1.f;
            const uint32_t votes = __ballot_sync(0xFFFFFFFFu, c != 1.f);
            if (c != 1.f) {
                const uint32_t at = before + __popc(votes & ((1u << threadIdx.x) - 1u));
                factors[at] = c;
                models[at] = n;
            }
            before += __popc(votes);
        }
        if (threadIdx.x == 0) count_shared = before;
    }
    __syncthreads();
    const uint32_t count = count_shared, unit_hi = a.pop.n_groups / 2;
    FullUnits full;
    for (uint32_t w = blockIdx.x; w < trips * count; w += gridDim.x) {
        const uint32_t trip = w / count, j = w - trip * count, first = (trips - 1u - trip) * K * kChunkThreads, unit = first + threadIdx.x;
        char *row = static_cast<char *>(a.grads) + (static_cast<size_t>(models[j]) * a.pop.padded_P + 8ull * unit) * T::kBytes;
        const float factor = factors[j];
        const float c[8] = {factor, factor, factor, factor, factor, factor, factor, factor};
        Octet<T> g[K];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (unit + k * kChunkThreads < unit_hi) g[k].load(row + static_cast<size_t>(k * kChunkThreads) * 8 * T::kBytes);
        const bool whole = one_tensor(a.pop, full, first, K * kChunkThreads, a.status);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            char *out = row + static_cast<size_t>(k * kChunkThreads) * 8 * T::kBytes;
            float decay;
            const uint32_t mask = whole ? 0xFFu : existing_np(a.pop, min(unit + k * kChunkThreads, unit_hi - 1u), a.status, &decay);
            if (unit + k * kChunkThreads >= unit_hi) continue;
            scale_octet(g[k], c, 0xFFu);
            if (mask == 0xFFu) g[k].store(out);
            else g[k].store_some(out, mask);
        }
    }
}

// [P][N]: a thread's octets hold the same models in every chunk, so it looks their factors up once.
template <class T>
__global__ void __launch_bounds__(kChunkThreads, kClipBlocksPN) clip_pn_kernel(const __grid_constant__ ClipArgs a, uint32_t trips)
{
    await_previous();
    let_next_start();
    constexpr int K = kTogether<T>;
    const uint32_t N = static_cast<uint32_t>(a.pop.N), units = chunk_units(kLayoutPN, a.pop.N), octets = units * N, unit_hi = a.pop.n_groups / 2;
    __shared__ float factors[kMaxN];
    if (threadIdx.x < N) factors[threadIdx.x] = clip_factor(a.norm[threadIdx.x], a.max_norm);
    __syncthreads();
    const uint32_t e0 = 8u * threadIdx.x / N, n0 = 8u * threadIdx.x - e0 * N;
    uint32_t active = 0, n = n0;
    float c[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        c[q] = factors[n];
        if (c[q] != 1.f) active |= 1u << q;
        if (++n == N) n = 0;
    }
    if (!__syncthreads_or(threadIdx.x < octets && active)) return;
    FullUnits full;
    for (uint32_t trip = blockIdx.x; trip < trips; trip += gridDim.x) {
        const uint32_t first = (trips - 1u - trip) * K * units;
        const uint64_t left = static_cast<uint64_t>(unit_hi - first) * N;   // octets from here on
        char *src = static_cast<char *>(a.grads) + (static_cast<size_t>(first) * N + threadIdx.x) * 8 * T::kBytes;
        Octet<T> g[K];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (threadIdx.x < octets && k * octets + threadIdx.x < left && active) g[k].load(src + static_cast<size_t>(k * octets) * 8 * T::kBytes);
        const bool whole = one_tensor(a.pop, full, first, K * units, a.status);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            char *out = src + static_cast<size_t>(k * octets) * 8 * T::kBytes;
            float decay[8];
            const uint32_t mask = whole ? 0xFFu : existing_pn(a.pop, first + k * units, e0, n0, unit_hi, a.status, decay);
            if (threadIdx.x >= octets || k * octets + threadIdx.x >= left || !active) continue;
            scale_octet(g[k], c, active);
            if (mask == 0xFFu) g[k].store(out);
            else g[k].store_some(out, mask & active);
        }
    }
}

cudaError_t launch_clip(const ClipArgs &args, int dtype, int sm_count, cudaStream_t stream)
{
    const bool np = args.pop.layout == kLayoutNP, f32 = dtype == kDtypeF32;
    const uint32_t per_trip = chunk_units(args.pop.layout, args.pop.N) * (f32 ? kTogether<F32> : kTogether<BF16>);
    const uint32_t trips = (args.pop.n_groups / 2 + per_trip - 1) / per_trip, most = (np ? kWavesNP * kClipBlocksNP : kWavesPN * kClipBlocksPN) * static_cast<uint32_t>(sm_count);
    const uint64_t work = np ? static_cast<uint64_t>(trips) * args.pop.N : trips;   // trips of at least 512 units: below 2^27 with N = 64
    const uint32_t grid = work < most ? static_cast<uint32_t>(work) : most;
    if (np) return launch_chained(f32 ? clip_np_kernel<F32> : clip_np_kernel<BF16>, grid, kChunkThreads, 0, stream, args, trips);
    return launch_chained(f32 ? clip_pn_kernel<F32> : clip_pn_kernel<BF16>, grid, kChunkThreads, 0, stream, args, trips);
}

}  // namespace wash
