// Every model's gradient norm over a range of tensors: norm_n = sqrt(sum_i g_n,i^2), squares and sums in binary64 (a square of a binary32
// value is exact there and neither overflows nor underflows), added in an order that depends on the launch's shape only.
//
// One pass: a resident grid walks the chunks, a thread adds up its octets' squares, a block leaves one partial sum a model, and the block that reports last
// adds the blocks' partials and takes the root.  [N][P]: a block has one model, five of 256 threads an SM (four for bf16).  [P][N]: a block has them all; there are 1024 threads an SM, in
// four blocks or two.
// Bound by HBM in fp32 (ResNet-50 N = 10, norm behind norm, 147 us = 6.97 TB/s, [P][N] N = 8 120 us = 6.8), nearly so in bf16: a trip of as many bytes
// holds twice the values and keeps half of the issue slots busy, during which its warp has no loads in flight (N = 8 67 us = 6.1 TB/s, [P][N] 67).
#include "wash_octet.cuh"

namespace wash {

__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

// A square is added up in binary64 in one of two ways, turn about, since they load different pipes: by converting the number (one instruction, at a fraction of the
// others' rate), or by the shifts that make a binary64 number of its pattern -- without its sign, moved left by 29, it is the number times 2^-896, denormals
// included -- and a multiplication.  bf16, ResNet-50 N = 8: conversions alone 74.7 us, shifts alone 71.6, half and half 67.9 ([P][N] 74.3, 75.1, 70.7); fp32 147 all three.
// Infinities and NaNs come out of the shifts as numbers of 2^128 and more: a sum below 2^256 has none (kSuspect).
__device__ __forceinline__ double add_square(uint32_t hi, uint32_t lo, double sum)
{
    const double x = __hiloint2double(static_cast<int>(hi), static_cast<int>(lo)) * 0x1p896;
    return fma(x, x, sum);
}
constexpr double kSuspect = 0x1p256;

// value q of the octet
template <class T>
__device__ __forceinline__ double add_value(const Octet<T> &g, int q, double sum)
{
    if (q & 1) {
        const double x = static_cast<double>(g.get(q));
        return fma(x, x, sum);
    }
    const uint32_t w = T::kBytes == 4 ? g.word(q) : g.word(q / 2);
    if constexpr (T::kBytes == 4) return add_square((w >> 3) & 0x0FFFFFFFu, w << 29, sum);
    else return add_square((w << 13) & 0x0FFFE000u, 0u, sum);
}

// Clears the values of an octet that do not exist.
template <class T>
__device__ __forceinline__ void keep_existing(Octet<T> &g, uint32_t mask)
{
    Octet<T> zero;
#pragma unroll
    for (int i = 0; i < Octet<T>::kVecs; ++i) zero.v[i] = make_uint4(0u, 0u, 0u, 0u);
    g.merge(zero, mask);
}

// A sum that is not below kSuspect: are there infinities or NaNs among the octet's values?  bit 0, bit 1 of value q's two bits.
template <class T>
__device__ __forceinline__ uint32_t specials(const Octet<T> &g)
{
    uint32_t found = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const uint32_t magnitude = __float_as_uint(g.get(q)) & 0x7FFFFFFFu;
        found |= (magnitude > 0x7F800000u ? 2u : magnitude == 0x7F800000u ? 1u : 0u) << (2 * q);
    }
    return found;
}
__device__ __forceinline__ double with_specials(double sum, uint32_t found)
{
    return found & 2u ? __longlong_as_double(0x7FF8000000000000ll) : found & 1u ? __longlong_as_double(0x7FF0000000000000ll) : sum;
}

// Adds up `count` values of each of N models, value i of model n being value(i, n), and gives the totals to store(n, total): a group of 32, 16, 8 or 4 lanes a model, so that
// all models are summed at the same time (N = 64: 1.5 us less than a warp a model, one after the other; several groups a model need two barriers more and lose .3 us).
template <int THREADS, class V, class S>
__device__ __forceinline__ void sum_models(uint32_t N, uint32_t count, V value, S store)
{
    static_assert(THREADS / 4 >= kMaxN, "a group a model");
    const uint32_t lanes = N <= THREADS / 32 ? 32u : N <= THREADS / 16 ? 16u : N <= THREADS / 8 ? 8u : 4u;
    const uint32_t n = threadIdx.x / lanes;
    double s = 0.0;
    if (n < N)
        for (uint32_t i = threadIdx.x % lanes; i < count; i += lanes) s += value(i, n);
    for (uint32_t d = lanes / 2; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (threadIdx.x % lanes == 0 && n < N) store(n, s);
}

// The blocks' partial sums lie one block after the other, N to a block.  The block that reports last adds them up and leaves the ticket at 0: thread t takes
// every (THREADS / N * N)-th from t on, all of model t mod N, then the threads of a model are added up.
template <int THREADS>
__device__ __forceinline__ void finish_norms(const NormArgs &a, double *part)
{
    __shared__ bool last;
    __syncthreads();   // the block's partials are stored, `part` is free
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicInc(a.ticket, gridDim.x - 1u) == gridDim.x - 1u;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    const uint32_t N = static_cast<uint32_t>(a.pop.N), shares = THREADS / N, stride = shares * N, count = a.per_model * N;
    double s = 0.0;
    if (threadIdx.x < stride) {
        constexpr int kBatch = 16;   // loads in flight: a trip to the L2 is most of this kernel's end
        for (uint32_t i = threadIdx.x; i < count; i += kBatch * stride) {
            double v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) v[k] = i + k * stride < count ? __ldcg(a.partial + i + k * stride) : 0.0;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) s += v[k];
        }
    }
    part[threadIdx.x] = s;   // of model threadIdx.x mod N
    __syncthreads();
    sum_models<THREADS>(N, shares, [&](uint32_t i, uint32_t n) { return part[i * N + n]; }, [&](uint32_t n, double total) { a.out[n] = sqrt(total); });
}

// Where a block's value f lies in shared memory: eight neighbours trade places, so that neither the threads' writes (8 values apart) nor the reads of a model's
// values (N apart) fall into one bank (N = 64, 10408 coordinates: 12 -> 9.4 us).
__device__ __forceinline__ uint32_t spread(uint32_t f) { return (f & ~7u) | ((f ^ (f >> 3) ^ (f >> 6)) & 7u); }

// K: octets a thread has in flight
template <class T, int THREADS, int K>
__global__ void __launch_bounds__(THREADS, THREADS == kNormThreads ? norm_blocks_np(T::kBytes) : 1) norm_np_kernel(const __grid_constant__ NormArgs a)
{
    await_previous();
    let_next_start();
    __shared__ double part[THREADS];
    const uint32_t N = static_cast<uint32_t>(a.pop.N), b = blockIdx.x / N, n = blockIdx.x - b * N, lane = threadIdx.x & 31u;
    const char *row = static_cast<const char *>(a.grads) + static_cast<size_t>(n) * a.pop.padded_P * T::kBytes;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    FullUnits full;
    constexpr size_t kStride = static_cast<size_t>(THREADS) * 8 * T::kBytes;   // from a thread's octet to its next one
    for (uint32_t c = b * K; c < a.n_chunks; c += a.per_model * K) {
        const uint32_t first = a.unit_lo + c * THREADS, unit = first + threadIdx.x;
        const char *src = row + static_cast<size_t>(unit) * 8 * T::kBytes;
        Octet<T> g[K];
        if (first + K * THREADS <= a.unit_hi) {
#pragma unroll
            for (int k = 0; k < K; ++k) g[k].load(src + k * kStride);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (unit + k * THREADS < a.unit_hi) g[k].load(src + k * kStride);
                else keep_existing(g[k], 0u);
            }
        }
        if (!one_tensor(a.pop, full, first, K * THREADS, a.status)) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float decay;   // (values behind unit_hi are zeros)
                keep_existing(g[k], existing_np(a.pop, min(unit + k * THREADS, a.unit_hi - 1u), a.status, &decay));
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q % 4] = add_value(g[k], q, sum[q % 4]);
    }
    double total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if (!(total < kSuspect)) {   // large, or not numbers: look again
        uint32_t found = 0;
        for (uint32_t c = b * K; c < a.n_chunks; c += a.per_model * K)
            for (int k = 0; k < K; ++k) {
                const uint32_t unit = a.unit_lo + (c + k) * THREADS + threadIdx.x;
                if (unit >= a.unit_hi) continue;
                Octet<T> g;
                g.load(row + static_cast<size_t>(unit) * 8 * T::kBytes);
                keep_existing(g, existing(find_place(a.pop, unit, a.status), unit));
                found |= specials(g);
            }
        found |= found >> 8;
        found |= found >> 4;
        total = with_specials(total, found | found >> 2);
    }
    total = warp_sum(total);
    if (lane == 0) part[threadIdx.x >> 5] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) s += part[w];
        if (a.per_model == 1) a.out[n] = sqrt(s);
        else a.partial[blockIdx.x] = s;
    }
    if (a.per_model != 1) finish_norms<THREADS>(a, part);
}

template <class T, int THREADS, int K>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) norm_pn_kernel(const __grid_constant__ NormArgs a)
{
    await_previous();
    let_next_start();
    __shared__ double part[8 * THREADS];
    const uint32_t N = static_cast<uint32_t>(a.pop.N), units = THREADS / N, octets = units * N;
    const uint32_t octet = min(threadIdx.x, octets - 1u);   // the last threads repeat the chunk's last octet; nobody reads their sums
    const uint32_t e0 = 8u * octet / N, n0 = 8u * octet - e0 * N;
    double sum[8];   // of model (n0 + q) mod N
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.0;
    FullUnits full;
    // of the chunk whose first unit is `first`
    const auto there = [&](uint32_t first) { return first < a.unit_hi && (units <= a.unit_hi - first || octet < (a.unit_hi - first) * N); };
    const size_t stride = static_cast<size_t>(octets) * 8 * T::kBytes;   // from a thread's octet to its next one
    const auto at = [&](uint32_t first) { return static_cast<const char *>(a.grads) + (static_cast<size_t>(first) * N + octet) * 8 * T::kBytes; };
    for (uint32_t c = blockIdx.x * K; c < a.n_chunks; c += gridDim.x * K) {
        const uint32_t first = a.unit_lo + c * units;
        const char *src = at(first);
        Octet<T> g[K];
        if (first + K * units <= a.unit_hi) {
#pragma unroll
            for (int k = 0; k < K; ++k) g[k].load(src + k * stride);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (there(first + k * units)) g[k].load(src + k * stride);
                else keep_existing(g[k], 0u);
            }
        }
        if (!one_tensor(a.pop, full, first, K * units, a.status)) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float decay[8];
                keep_existing(g[k], existing_pn(a.pop, first + k * units, e0, n0, a.unit_hi, a.status, decay));
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] = add_value(g[k], q, sum[q]);
    }
    bool suspect = false;
#pragma unroll
    for (int q = 0; q < 8; ++q) suspect = suspect || !(sum[q] < kSuspect);
    if (suspect) {
        uint32_t found = 0;
        for (uint32_t c = blockIdx.x * K; c < a.n_chunks; c += gridDim.x * K)
            for (int k = 0; k < K; ++k) {
                const uint32_t first = a.unit_lo + (c + k) * units;
                if (!there(first)) continue;
                Octet<T> g;
                float decay[8];
                g.load(at(first));
                keep_existing(g, existing_pn<false>(a.pop, first, e0, n0, a.unit_hi, a.status, decay));
                found |= specials(g);
            }
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[q] = with_specials(sum[q], found >> (2 * q));
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) part[spread(8u * threadIdx.x + q)] = sum[q];   // value f of the chunk's 8 * octets: model f mod N
    __syncthreads();
    sum_models<THREADS>(N, 8u * units, [&](uint32_t i, uint32_t n) { return part[spread(i * N + n)]; },
        [&](uint32_t n, double total) {
            if (gridDim.x == 1) a.out[n] = sqrt(total);
            else a.partial[static_cast<size_t>(blockIdx.x) * N + n] = total;
        });
    if (gridDim.x != 1) finish_norms<THREADS>(a, part);
}

// BYTES of gradients a thread has in flight, THREADS of a block, `blocks` at most for a model ([N][P]) or for all.
template <class T, int THREADS, int BYTES>
static cudaError_t launch_norm(NormArgs args, uint32_t blocks, cudaStream_t stream)
{
    constexpr int K = BYTES / (8 * T::kBytes);
    const uint32_t N = static_cast<uint32_t>(args.pop.N);
    const bool np = args.pop.layout == kLayoutNP;
    const NormGrid grid = norm_grid(args.pop.layout, args.pop.N, args.unit_hi - args.unit_lo, THREADS, K, blocks);
    args.n_chunks = grid.n_chunks;
    args.per_model = grid.per_model;
    if constexpr (THREADS != kNormThreadsMany)   // (the sizes that the other layout has to itself)
        if (np) return launch_chained(norm_np_kernel<T, THREADS, K>, args.per_model * N, THREADS, 0, stream, args);
    if constexpr (THREADS != kNormThreadsAlone)
        if (!np) return launch_chained(norm_pn_kernel<T, THREADS, K>, args.per_model, THREADS, 0, stream, args);
    return cudaErrorInvalidValue;
}

template <class T>
static cudaError_t launch_typed(const NormArgs &args, int sm_count, cudaStream_t stream)
{
    const NormPlan plan = norm_plan(args.pop.layout, args.pop.N, args.unit_hi - args.unit_lo, T::kBytes, sm_count);
    if (plan.threads == kNormThreadsAlone) return launch_norm<T, kNormThreadsAlone, 64>(args, plan.blocks, stream);
    if (plan.threads == kNormThreadsMany)
        return plan.bytes == 32 ? launch_norm<T, kNormThreadsMany, 32>(args, plan.blocks, stream) : launch_norm<T, kNormThreadsMany, 64>(args, plan.blocks, stream);
    return plan.bytes == 32 ? launch_norm<T, kNormThreads, 32>(args, plan.blocks, stream) : launch_norm<T, kNormThreads, 64>(args, plan.blocks, stream);
}

cudaError_t launch_grad_norm(NormArgs args, int dtype, int sm_count, cudaStream_t stream)
{
    return dtype == kDtypeF32 ? launch_typed<F32>(args, sm_count, stream) : launch_typed<BF16>(args, sm_count, stream);
}

}  // namespace wash
