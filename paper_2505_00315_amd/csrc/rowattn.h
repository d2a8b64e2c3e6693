// Attention one row at a time, by one wave, straight from the definition: keys
// that the query does not see are not read, so whatever they hold stays out of
// the result.  The tiled kernels multiply the rows of whole tiles, where a
// weight of 0 meets every value; they call these for the rows of a wave whose
// result is not finite.
#pragma once

#include "cache4.h"

namespace mosa {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// LDS written by lanes of this wave is seen by its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ float wave_sum_f32(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

// Columns of a row of DH held by a lane: lane, lane + 64 (none past DH).
template <int DH>
struct RowLanes {
    static constexpr int N = DH > 64 ? DH / 64 : 1;
    static __device__ __forceinline__ bool has(int lane) { return DH >= 64 || lane < DH; }
};

template <typename ST, int DH>
__device__ __forceinline__ void row_load(const ST* p, int lane, float (&x)[RowLanes<DH>::N]) {
#pragma unroll
    for (int i = 0; i < RowLanes<DH>::N; ++i) x[i] = RowLanes<DH>::has(lane) ? ld1<ST>(p + lane + 64 * i) : 0.f;
}
template <int DH>
__device__ __forceinline__ float row_dot(const float (&x)[RowLanes<DH>::N], const float (&y)[RowLanes<DH>::N]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < RowLanes<DH>::N; ++i) s += x[i] * y[i];
    return wave_sum_f32(s);
}

// The keys and values of one sequence and key head.
template <int DH>
struct CacheKeys {
    const CacheArgs& c;
    UDiv page;
    int b, h;
    __device__ __forceinline__ bool load(int j, int lane, float (&k)[RowLanes<DH>::N], float (&v)[RowLanes<DH>::N]) const {
        CacheBlock blk;
        int tl;
        if (!cache_find(c, page, b, h, j, blk, tl)) return false;
#pragma unroll
        for (int i = 0; i < RowLanes<DH>::N; ++i) {
            k[i] = RowLanes<DH>::has(lane) ? cache_k(c, blk, tl, lane + 64 * i) : 0.f;
            v[i] = RowLanes<DH>::has(lane) ? cache_v(c, blk, tl, lane + 64 * i) : 0.f;
        }
        return true;
    }
};

// One query row at position p over entries e0 .. e1 - 1 of a key list: running
// maximum m (log2 units), sum l and unnormalised o of this lane's columns.
template <int DH, class KEYS, class LIST>
__device__ __forceinline__ void row_attend(const AttnArgs& a, const KEYS& keys, const LIST& key_at, int e0, int e1,
                                           int p, int kn, const float (&q)[RowLanes<DH>::N], int lane, float& m,
                                           float& l, float (&o)[RowLanes<DH>::N]) {
    constexpr int N = RowLanes<DH>::N;
    const float c2 = a.scale * kLog2e;
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
        const int j = key_at(e);
        if (j < 0 || j >= kn || !sees(a, p, j)) continue;
        float k[N], v[N];
        if (!keys.load(j, lane, k, v)) continue;
        const float s = row_dot<DH>(q, k) * c2;
        const float mn = fmaxf(m, s), mu = mn == -__builtin_inff() ? 0.f : mn;
        const float al = __builtin_amdgcn_exp2f(m - mu), w = __builtin_amdgcn_exp2f(s - mu);
        m = mn;
        l = l * al + w;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * al + w * v[i];
    }
}

}  // namespace mosa
