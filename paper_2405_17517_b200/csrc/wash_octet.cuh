// What the kernels on the optimizer's side of a training step share: octets of a stack's values, the place of an octet among the tensors,
// and a model's clipping factor.
#pragma once
#include "wash_device.cuh"
#include "wash_launch.cuh"

namespace wash {

// Eight consecutive elements, as raw words: two 16-byte vectors of fp32, one of bf16.
template <class T>
struct Octet {
    static constexpr int kVecs = T::kBytes / 2;
    uint4 v[kVecs];

    __device__ __forceinline__ void load(const char *p)
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = F32::load_group(p + 16 * i);
    }
    __device__ __forceinline__ void store(char *p) const
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) *reinterpret_cast<uint4 *>(p + 16 * i) = v[i];
    }
    __device__ __forceinline__ uint32_t word(int i) const
    {
        const uint4 &x = v[i / 4];
        return i % 4 == 0 ? x.x : i % 4 == 1 ? x.y : i % 4 == 2 ? x.z : x.w;
    }
    __device__ __forceinline__ float get(int q) const
    {
        if constexpr (T::kBytes == 4) return __uint_as_float(word(q));
        else return __uint_as_float((q & 1) ? word(q / 2) & 0xFFFF0000u : word(q / 2) << 16);
    }
    __device__ __forceinline__ uint32_t raw(int q) const
    {
        if constexpr (T::kBytes == 4) return word(q);
        else return (q & 1) ? word(q / 2) >> 16 : word(q / 2) & 0xFFFFu;
    }
    // The values of `r`, which are results of arithmetic: a NaN among them has the one pattern that the conversion to bf16 gives it, too.
    __device__ __forceinline__ void put(const float (&r)[8])
    {
        uint32_t w[4 * kVecs];
#pragma unroll
        for (int i = 0; i < 4 * kVecs; ++i) {
            if constexpr (T::kBytes == 4) w[i] = __float_as_uint(r[i]);
            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(r[2 * i + 1]), "f"(r[2 * i]));
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
    // the values whose bit is set in `mask` stay, the others become `other`'s
    __device__ __forceinline__ void merge(const Octet &other, uint32_t mask)
    {
        uint32_t w[4 * kVecs];
#pragma unroll
        for (int i = 0; i < 4 * kVecs; ++i) {
            if constexpr (T::kBytes == 4) w[i] = (mask >> i) & 1u ? word(i) : other.word(i);
            else {
                const uint32_t two = (mask >> (2 * i)) & 3u, keep = (two & 1u ? 0xFFFFu : 0u) | (two & 2u ? 0xFFFF0000u : 0u);
                w[i] = (word(i) & keep) | (other.word(i) & ~keep);
            }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
    // the values of `r` whose bit is set in `active`, the others' bits as they are
    __device__ __forceinline__ void put(const float (&r)[8], uint32_t active)
    {
        if (active == 0xFFu) {
            put(r);
            return;
        }
        const Octet before = *this;
        put(r);
        merge(before, active);
    }
    __device__ __forceinline__ void store_some(char *p, uint32_t mask) const
    {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if ((mask >> q) & 1u) T::store_elem(p, q, raw(q));
    }
};

// The tensor of a unit of 8 coordinates of a row.  Units are counted in 32 bits (a row has less than 2^30).
struct Place {
    uint32_t seg;
    uint32_t begin, full_end, end;   // units: the tensor's, and how far its units are full; behind its coordinates comes padding
    uint32_t rest;                   // coordinates of unit full_end (0 to 7)
    float decay;
};
__device__ __forceinline__ Place place_entry(const PopView &pop, uint32_t s)
{
    const uint2 lo = __ldg(reinterpret_cast<const uint2 *>(pop.seg + s));       // group_begin, group_end
    const uint2 hi = __ldg(reinterpret_cast<const uint2 *>(pop.seg + s) + 2);   // numel, decay
    Place at;
    at.seg = s;
    at.begin = lo.x / 2;
    at.end = lo.y / 2;
    at.full_end = at.begin + hi.x / 8;
    at.rest = hi.x % 8;
    at.decay = __uint_as_float(hi.y);
    return at;
}
__device__ __forceinline__ Place find_place(const PopView &pop, uint32_t unit, uint32_t *status)
{
    const uint32_t g = 2 * unit;
    uint32_t s = __ldg(pop.tile_first + (g >> kTileShift));
    const uint32_t last = static_cast<uint32_t>(pop.n_seg) - 1u;
    while (s < last && g >= __ldg(&pop.seg[s].group_end)) ++s;
    Place at = place_entry(pop, s);
    if (unit < at.begin || unit >= at.end) {   // table inconsistent with the row: report, touch nothing
        if (status) atomicOr(status, 1u);
        at.full_end = at.begin;
        at.rest = 0;
    }
    return at;
}
// The same for every lane of a warp, all lanes calling, their units ascending: the lanes fetch the entries of 32 tensors at once, from the first lane's tile on, and
// pick theirs by shuffles -- two trips to the L2 instead of one a tensor (the SGD step of five models with 12 small tensors 3.3 -> 2.3 us in a graph).
__device__ __forceinline__ Place warp_place(const PopView &pop, uint32_t unit, uint32_t *status)
{
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x & 31u, lowest = __shfl_sync(kAll, unit, 0), highest = __shfl_sync(kAll, unit, 31);
    const uint32_t first = __ldg(pop.tile_first + (2u * lowest >> kTileShift));
    const Place mine = place_entry(pop, min(first + lane, static_cast<uint32_t>(pop.n_seg) - 1u));
    uint32_t k = min(static_cast<uint32_t>(__popc(__ballot_sync(kAll, mine.end <= lowest))), 31u);   // entries that end at or before the first lane's unit
    if (highest >= __shfl_sync(kAll, mine.end, k))   // the others' are further on
        for (bool later = true; __any_sync(kAll, later); k += later) {
            const uint32_t end = __shfl_sync(kAll, mine.end, k);   // by all lanes, those that have found theirs, too
            later = k < 31u && unit >= end;
        }
    Place at;
    at.seg = min(first + k, static_cast<uint32_t>(pop.n_seg) - 1u);
    at.begin = __shfl_sync(kAll, mine.begin, k);
    at.full_end = __shfl_sync(kAll, mine.full_end, k);
    at.end = __shfl_sync(kAll, mine.end, k);
    at.rest = __shfl_sync(kAll, mine.rest, k);
    at.decay = __shfl_sync(kAll, mine.decay, k);
    return unit >= at.begin && unit < at.end ? at : find_place(pop, unit, status);   // more than 32 tensors away
}

// Whether units [unit, unit + count) exist in full and belong to one tensor, the same for all lanes; `full` is where the tensor looked up last does.
struct FullUnits {
    uint32_t begin = 0, end = 0;
};
__device__ __forceinline__ bool one_tensor(const PopView &pop, FullUnits &full, uint32_t unit, uint32_t count, uint32_t *status)
{
    if (unit < full.begin || unit + count > full.end) {
        const Place at = warp_place(pop, unit, status);
        full.begin = at.begin;
        full.end = at.full_end;
    }
    return unit + count <= full.end;
}

// which of a unit's 8 coordinates exist
__device__ __forceinline__ uint32_t existing(const Place &at, uint32_t unit)
{
    return unit < at.full_end ? 0xFFu : unit == at.full_end ? (1u << at.rest) - 1u : 0u;
}

// [N][P]: which of the unit's 8 coordinates exist, and their tensor's decay.  All lanes call; lanes beyond the row's end give any unit of it.
__device__ __forceinline__ uint32_t existing_np(const PopView &pop, uint32_t unit, uint32_t *status, float *decay)
{
    const Place at = warp_place(pop, unit, status);
    *decay = at.decay;
    return existing(at, unit);
}

// [P][N]: the same for the octet whose first value is model `n`'s of coordinate `c` (0 and up) from the unit's first on.  Its values may belong to more than
// one unit and tensor.  WARP: all lanes call (units from `unit_hi` on, the end of the row, are none).
template <bool WARP = true>
__device__ __forceinline__ uint32_t existing_pn(const PopView &pop, uint32_t unit, uint32_t c, uint32_t n, uint32_t unit_hi, uint32_t *status, float (&decay)[8])
{
    unit = min(unit + c / 8u, unit_hi - 1u);
    c %= 8u;
    Place at = WARP ? warp_place(pop, unit, status) : find_place(pop, unit, status);
#pragma unroll
    for (int q = 0; q < 8; ++q) decay[q] = at.decay;
    if (unit + (c + (n + 7u) / static_cast<uint32_t>(pop.N)) / 8u < at.full_end) return 0xFFu;
    uint32_t mask = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (unit >= at.end && at.seg + 1u < static_cast<uint32_t>(pop.n_seg)) at = place_entry(pop, at.seg + 1u);
        decay[q] = at.decay;
        mask |= ((existing(at, unit) >> c) & 1u) << q;
        if (++n == static_cast<uint32_t>(pop.N)) {
            n = 0;
            if (++c == 8u) {
                c = 0;
                ++unit;
            }
        }
    }
    return mask;
}

// A model's clipping factor: max_norm / (norm + 1e-6) in binary64, at most 1, rounded to binary32.  A norm that is NaN gives NaN, an infinite one 0.
__device__ __forceinline__ float clip_factor(double norm, double max_norm)
{
    const double c = max_norm / (norm + 1e-6);
    return c >= 1.0 ? 1.f : static_cast<float>(c);
}

}  // namespace wash
