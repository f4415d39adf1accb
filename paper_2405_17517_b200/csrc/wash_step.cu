// The optimizer's step for all models in one pass, with the clipping's factor folded into the read of the gradients:
//   SGD    d = c g + wd_t p;  m <- mu m + d;  p <- p - lr u,  u = m, with Nesterov d + mu m, without momentum d
//   AdamW  g' = c g;  m <- b1 m + (1 - b1) g';  v <- b2 v + (1 - b2) g'^2;
//          p <- p - lr (s1 m / (s2 sqrt(v) + eps) + wd_t p),  s1 = 1 / (1 - b1^t), s2 = 1 / sqrt(1 - b2^t)
// in binary32, products fused with the additions behind them (explicit _rn intrinsics), bf16 weights rounded to nearest even at the store: large steps cost the bytes they
// move, so nothing is approximated (quotient and root as the hardware's approximations: AdamW of ResNet-50 N = 8 bf16 [P][N] 664 -> 649 us, [N][P] and fp32 the same).
//
// Bound by HBM: one trip a thread, an octet of every stack, all loads in flight before anything else (a lookup of the tensor in front of the barrier costs a
// tenth).  Blocks of 256 threads go from the last chunk to the first, as wash_clip.cu has it; the norm's pass leaves little in the L2 that lasts until the step
// has come to it (ResNet-18 N = 5 norm and step: 214 us in the norm's order, 210 in this; loads and stores marked as used once, or with an evict-first policy: the same or slower).
// ResNet-50, us and share of the measured copy rate: SGD with momentum N = 10 fp32 755 (103 %), N = 8 bf16 434 (101 %), [P][N] N = 8 583 (107 %) and 416 (105 %);
// AdamW N = 10 fp32 1086 (101 %), N = 8 bf16 678 (101 %), [P][N] N = 8 831 (105 %) and 666 (103 %).
#include "wash_octet.cuh"

namespace wash {

template <int RULE>
__device__ __forceinline__ void update(const StepArgs &a, float c, float wd, float g, float &p, float &m, float &v)
{
    g = __fmul_rn(c, g);
    float u;
    if constexpr (RULE == kRuleAdamW) {
        m = __fmaf_rn(a.beta1, m, __fmul_rn(a.one_minus_beta1, g));
        v = __fmaf_rn(a.beta2, v, __fmul_rn(__fmul_rn(a.one_minus_beta2, g), g));
        u = __fdiv_rn(__fmul_rn(a.first_scale, m), __fmaf_rn(a.second_scale, __fsqrt_rn(v), a.eps));
        u = __fmaf_rn(wd, p, u);
    } else {
        u = __fmaf_rn(wd, p, g);
        if constexpr (RULE != kRuleSgd) {
            m = __fmaf_rn(a.beta1, m, u);
            u = RULE == kRuleNesterov ? __fmaf_rn(a.beta1, m, u) : m;
        }
    }
    p = __fmaf_rn(-a.lr, u, p);
}

// A model's factor for a step: -1 (no factor is negative) where the model is to keep everything.
__device__ __forceinline__ float step_factor(const StepArgs &a, uint32_t n)
{
    if (!a.norm) return 1.f;
    const double norm = a.norm[n];
    if (a.skip_nonfinite && !(norm <= 1.7976931348623157e308)) return -1.f;
    return clip_factor(norm, a.max_norm);
}

template <class TW, class TG, int RULE>
struct StepOctet {
    Octet<TW> p;
    Octet<TG> g;
    Octet<F32> m, v;
    __device__ __forceinline__ void load(const StepArgs &a, size_t element)
    {
        p.load(static_cast<const char *>(a.params) + element * TW::kBytes);
        g.load(static_cast<const char *>(a.grads) + element * TG::kBytes);
        if constexpr (RULE != kRuleSgd) m.load(static_cast<const char *>(a.m) + element * 4);
        if constexpr (RULE == kRuleAdamW) v.load(static_cast<const char *>(a.v) + element * 4);
    }
    // c(q), wd(q): factor and decay of value q; mask: values that exist; active: values whose model is updated
    template <class C, class D>
    __device__ __forceinline__ void finish(const StepArgs &a, size_t element, C c, D wd, uint32_t mask, uint32_t active)
    {
        float rp[8], rm[8], rv[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            rp[q] = p.get(q);
            rm[q] = RULE != kRuleSgd ? m.get(q) : 0.f;
            rv[q] = RULE == kRuleAdamW ? v.get(q) : 0.f;
            update<RULE>(a, c(q), wd(q), g.get(q), rp[q], rm[q], rv[q]);
        }
        p.put(rp, active);
        if constexpr (RULE != kRuleSgd) m.put(rm, active);
        if constexpr (RULE == kRuleAdamW) v.put(rv, active);
        char *pp = static_cast<char *>(a.params) + element * TW::kBytes, *pm = static_cast<char *>(a.m) + element * 4, *pv = static_cast<char *>(a.v) + element * 4;
        if (mask == 0xFFu) {
            p.store(pp);
            if constexpr (RULE != kRuleSgd) m.store(pm);
            if constexpr (RULE == kRuleAdamW) v.store(pv);
        } else {
            mask &= active;
            p.store_some(pp, mask);
            if constexpr (RULE != kRuleSgd) m.store_some(pm, mask);
            if constexpr (RULE == kRuleAdamW) v.store_some(pv, mask);
        }
    }
};

// Blocks an SM holds at least, by the registers that are left to a thread then ([P][N] AdamW fp32: 4 spill 48 bytes a thread, and are faster for it).  us with 1 / 4 / 5 / 6:
//   [N][P], 1 / 5 / 6 / 7  ResNet-50 N = 10 fp32 without momentum 467 / 463 / 464 / 446, with 760 / 757 / 767 / 938, AdamW 1082 / 1087 / 1186 / 1618;
//           N = 8 bf16 243 / 243 / 255 / 220, 438 / 461 / 437 / 439 (fp32 gradients 522 / 494 / 479 / 538), 699 / 678 / 710 / 852
//   [P][N]  ResNet-50 N = 8  momentum fp32 582 / 583 / 591 / 661, bf16 439 / 443 / 410 / 415, bf16 and fp32 474 / 470 / 466 / 525;  without fp32 370 / 371 / 348 / 349, bf16
//           250 / 251 / 250 / 227;  AdamW fp32 933 / 849 / 1463 (spills), bf16 689 / 692 / 1025
template <class TW, class TG, int RULE>
constexpr int step_blocks(int layout)
{
    constexpr int halves = (TW::kBytes == 2) + (TG::kBytes == 2);
    if (layout == kLayoutNP) return RULE == kRuleAdamW ? 5 : RULE == kRuleSgd ? 7 : halves ? 6 : 5;
    return RULE == kRuleAdamW ? 4 : RULE == kRuleSgd ? (halves == 2 ? 6 : 5) : halves ? 5 : 4;
}

template <class TW, class TG, int RULE>
__global__ void __launch_bounds__(kChunkThreads, step_blocks<TW, TG, RULE>(kLayoutNP)) step_np_kernel(const __grid_constant__ StepArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t N = static_cast<uint32_t>(a.pop.N), back = gridDim.x - 1u - blockIdx.x, chunk = back / N, n = back - chunk * N;
    const uint32_t unit = chunk * kChunkThreads + threadIdx.x;
    const uint32_t unit_hi = a.pop.n_groups / 2;
    const size_t element = static_cast<size_t>(n) * a.pop.padded_P + 8ull * unit;
    StepOctet<TW, TG, RULE> o;
    if (unit < unit_hi) o.load(a, element);
    float decay;
    const uint32_t mask = existing_np(a.pop, min(unit, unit_hi - 1u), a.status, &decay);
    const float factor = step_factor(a, n);
    if (factor < 0.f || unit >= unit_hi) return;
    decay = __fmul_rn(a.decay, decay);
    o.finish(a, element, [&](int) { return factor; }, [&](int) { return decay; }, mask, 0xFFu);
}

template <class TW, class TG, int RULE>
__global__ void __launch_bounds__(kChunkThreads, step_blocks<TW, TG, RULE>(kLayoutPN)) step_pn_kernel(const __grid_constant__ StepArgs a)
{
    await_previous();
    let_next_start();
    const uint32_t N = static_cast<uint32_t>(a.pop.N), units = chunk_units(kLayoutPN, a.pop.N);
    const uint32_t first = (gridDim.x - 1u - blockIdx.x) * units, here = min(units, a.pop.n_groups / 2 - first) * N;
    const size_t element = (static_cast<size_t>(first) * N + threadIdx.x) * 8;
    StepOctet<TW, TG, RULE> o;
    if (threadIdx.x < here) o.load(a, element);
    __shared__ float factors[kMaxN + 8];   // model after model, and once more the first ones, so that an octet's are neighbours
    if (threadIdx.x < N) {
        const float c = step_factor(a, threadIdx.x);
        for (uint32_t i = threadIdx.x; i < N + 8u; i += N) factors[i] = c;
    }
    __syncthreads();
    const Place at = warp_place(a.pop, first, a.status);   // (before the barrier it holds up the block)
    const uint32_t e0 = 8u * threadIdx.x / N, n0 = 8u * threadIdx.x - e0 * N;
    uint32_t active = 0xFFu;
    if (a.skip_nonfinite) {
        active = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) active |= factors[n0 + q] < 0.f ? 0u : 1u << q;
    }
    const auto c = [&](int q) { return factors[n0 + q]; };
    if (first + units <= at.full_end) {   // the chunk lies in one tensor
        const float decay = __fmul_rn(a.decay, at.decay);
        if (threadIdx.x >= here) return;
        o.finish(a, element, c, [&](int) { return decay; }, 0xFFu, active);
    } else {
        float wd[8];
        const uint32_t mask = existing_pn(a.pop, first, e0, n0, a.pop.n_groups / 2, a.status, wd);
        if (threadIdx.x >= here) return;
        o.finish(a, element, c, [&](int q) { return __fmul_rn(a.decay, wd[q]); }, mask, active);
    }
}

template <class TW, class TG, int RULE>
static cudaError_t launch_rule(const StepArgs &args, cudaStream_t stream)
{
    const uint32_t units = args.pop.n_groups / 2, per_chunk = chunk_units(args.pop.layout, args.pop.N);
    const uint64_t chunks = (units + per_chunk - 1) / per_chunk, grid = args.pop.layout == kLayoutNP ? chunks * args.pop.N : chunks;
    if (grid > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    if (args.pop.layout == kLayoutNP) return launch_chained(step_np_kernel<TW, TG, RULE>, static_cast<unsigned>(grid), kChunkThreads, 0, stream, args);
    return launch_chained(step_pn_kernel<TW, TG, RULE>, static_cast<unsigned>(grid), kChunkThreads, 0, stream, args);
}

template <class TW, class TG>
static cudaError_t launch_typed(const StepArgs &args, int rule, cudaStream_t stream)
{
    switch (rule) {
    case kRuleSgd: return launch_rule<TW, TG, kRuleSgd>(args, stream);
    case kRuleMomentum: return launch_rule<TW, TG, kRuleMomentum>(args, stream);
    case kRuleNesterov: return launch_rule<TW, TG, kRuleNesterov>(args, stream);
    default: return launch_rule<TW, TG, kRuleAdamW>(args, stream);
    }
}

cudaError_t launch_step(const StepArgs &args, int rule, int params_dtype, int grads_dtype, cudaStream_t stream)
{
    if (params_dtype == kDtypeF32) return grads_dtype == kDtypeF32 ? launch_typed<F32, F32>(args, rule, stream) : launch_typed<F32, BF16>(args, rule, stream);
    return grads_dtype == kDtypeF32 ? launch_typed<BF16, F32>(args, rule, stream) : launch_typed<BF16, BF16>(args, rule, stream);
}

}  // namespace wash
