// Operators of the dense heads (norm and rotation, windowed attention, the
// 4-bit cache): arguments shared by their kernels and the host layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.h"
#include "kernels.h"

namespace mosa {

// Rows of one head: d_head contiguous values every `row` elements; the strides
// of axes of one entry are 0 here.
struct Rows {
    char* p;
    int64_t batch, head, row;
};
template <typename ST>
__device__ __forceinline__ ST* row_ptr(const Rows& r, int b, int h, int64_t t) {
    return reinterpret_cast<ST*>(r.p) + b * r.batch + h * r.head + t * r.row;
}

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// LDS written by lanes of this wave is seen by its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f(storage value, integral constant d_head) for the type and head size of a call.
template <typename F>
inline int heads_by_type(int dtype, int dh, F f) {
    if (dtype == kBF16) {
        if (dh == 32) return f(uint16_t{}, std::integral_constant<int, 32>{});
        if (dh == 64) return f(uint16_t{}, std::integral_constant<int, 64>{});
        return f(uint16_t{}, std::integral_constant<int, 128>{});
    }
    if (dh == 32) return f(float{}, std::integral_constant<int, 32>{});
    if (dh == 64) return f(float{}, std::integral_constant<int, 64>{});
    return f(float{}, std::integral_constant<int, 128>{});
}

// ---------------------------------------------------------------------------
// norm and rotation
// ---------------------------------------------------------------------------
constexpr int kMaxTurns = 64;  // pairs of a row of 128
struct Turns {                 // theta_j / (2 pi): the turns of pair j per position
    double t[kMaxTurns];
};
struct NormArgs {
    int B, T, Hq, Hkv, dh, rope, halves;
    float eps;
    Rows q, k, qo, ko, dq, dk;  // forward: q, k -> qo, ko; backward: q, k and the gradients qo, ko -> dq, dk
    const void *wq, *wk;
    const int32_t* pos;
    Turns turns;
};
size_t norm_partial_bytes(int dtype, int64_t tokens, int dh);
int launch_qk_norm(int dtype, const NormArgs& a, hipStream_t stream);
int launch_qk_norm_bwd(int dtype, const NormArgs& a, void* dwq, void* dwk, void* scratch, hipStream_t stream);

// ---------------------------------------------------------------------------
// windowed attention
// ---------------------------------------------------------------------------
// Division of x < 2^31 by n: the product with the reciprocal, rounded up, is at
// most one too large.
struct UDiv {
    uint32_t n, m;
    __device__ __forceinline__ int div(int x) const {
        const uint32_t q = m ? (uint32_t)(((uint64_t)(uint32_t)x * m) >> 32) : (uint32_t)x;
        return (int)(q * n > (uint32_t)x ? q - 1 : q);
    }
};
inline UDiv make_udiv(uint32_t n) { return {n, n == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + n - 1) / n)}; }

// The query rows of a key head are taken as one list, the G heads of a query
// next to each other: row r is query r / G of head r % G of the group.  A block
// of rows then spans few positions, so the keys that it walks are close to those
// that each of its rows sees, and the group's heads share every key that is read.
struct AttnArgs {
    int B, Hq, Hkv, G, Tq, N, W, S;  // W: 0 or a window below N; S: sinks, at most N
    UDiv gd;                         // by G
    float scale;
    Rows q, k, v, out, dout, dq, dk, dv;
    const int32_t *ql, *kl;
    float* lse;  // [B, Hq, Tq] (forward: may be nullptr)
    float2* ld;  // backward: of every query row, lse in log2 units (+inf where it sees nothing) and -sum(out dout)
};

// Lengths of sequence b, taken into the tensors.
__device__ __forceinline__ int seq_len_of(const int32_t* lens, int b, int most) {
    return lens ? min(max(lens[b], 0), most) : most;
}

// The visibility rule (positions p, j of the query and the key).
__device__ __forceinline__ bool sees(const AttnArgs& a, int p, int j) {
    return (j <= p) & ((a.W == 0) | (p - j < a.W) | (j < a.S));  // (without branches)
}

// Keys that some query of positions p0 .. p1 sees: 0 .. s - 1 and lo .. hi - 1
// (s <= lo), as one list of `count` keys: entry e is key e below s, lo + e - s above.
struct KeyList {
    int s, lo, count;
    __device__ __forceinline__ int key(int e) const { return e < s ? e : e - s + lo; }
};
__device__ __forceinline__ KeyList keys_of(const AttnArgs& a, int p0, int p1, int kn) {
    KeyList l;
    const int hi = min(p1 + 1, kn);
    l.lo = a.W ? min(max(p0 - a.W + 1, 0), max(hi, 0)) : 0;
    l.s = min(a.S, l.lo);
    l.count = hi <= 0 ? 0 : l.s + hi - l.lo;
    return l;
}

// Row r of the list of (b, key head hk): its query index, and its address in a
// tensor of query rows.
template <typename ST>
__device__ __forceinline__ ST* qrow_ptr(const AttnArgs& a, const Rows& t, int b, int hk, int r, int i) {
    return row_ptr<ST>(t, b, hk * a.G + (r - i * a.G), i);
}
// The same row among [B, Hq, Tq].
__device__ __forceinline__ int64_t qrow_index(const AttnArgs& a, int b, int hk, int r, int i) {
    return ((int64_t)b * a.Hq + hk * a.G + (r - i * a.G)) * a.Tq + i;
}

// Results over a part of a row's keys, for every row of [B, Hq, Tq]: the
// unnormalised sum o, the running maximum m (log2 units) and the sum l of the
// weights 2^(score - m); merge_parts joins them in the order of the parts.
struct Parts {
    float *o, *ml;  // [parts][rows][DH], [parts][rows][2]
};
inline size_t parts_bytes(int parts, int64_t rows, int dh) {
    return parts > 1 ? (size_t)parts * (size_t)rows * (size_t)(dh + 2) * sizeof(float) : 0;
}
inline Parts make_parts(float* buf, int parts, int64_t rows, int dh) {
    return {buf, buf + (size_t)parts * (size_t)rows * (size_t)dh};
}
int launch_merge_parts(int dtype, int dh, const AttnArgs& a, int parts, const Parts& p, hipStream_t stream);

size_t attn_fwd_scratch(int dtype, int dh, const AttnArgs& a);
size_t attn_bwd_scratch(int dtype, int dh, const AttnArgs& a);
int launch_window_attn(int dtype, int dh, const AttnArgs& a, float* part, hipStream_t stream);
int launch_window_attn_bwd(int dtype, int dh, AttnArgs a, void* scratch, hipStream_t stream);

// ---------------------------------------------------------------------------
// the 4-bit cache
// ---------------------------------------------------------------------------
struct CacheArgs {
    int B, H, dh, pages, ps, per;  // ps: positions per page, per: table entries per sequence
    unsigned char* cache;
    const int32_t *table, *start, *lens;
    int rows;
    Rows k, v;
};
int launch_cache4_append(int dtype, const CacheArgs& a, hipStream_t stream);
int launch_cache4_read(int dtype, const CacheArgs& a, hipStream_t stream);
size_t cache4_attn_scratch(int dtype, int dh, const AttnArgs& a);
int launch_cache4_attn(int dtype, const AttnArgs& a, const CacheArgs& c, float* part, hipStream_t stream);

}  // namespace mosa
