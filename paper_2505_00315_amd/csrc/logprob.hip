// Log probabilities of tokens out of rows of logits, forward and backward.
//
//   M = max_j x_j,  L = log sum_j exp(scale (x_j - M)),  lse = scale M + L,
//   logp = scale (x_t - M) - L,
//   entropy = L - sum_j e_j scale (x_j - M) / sum_j e_j,  e_j = exp(scale (x_j - M))
//   dx_j = scale [ dlogp (1[j = t] - p_j) + dlse p_j - dentropy p_j (log p_j + entropy) ]
//
// The forward reads the logits once, the backward reads and writes them once:
// memory bounds both where rows are many.  M and L are kept apart: differences
// to M are exact where their sum lse would have rounded them away (rows far from
// 0, rows of the type's lowest value alone).
//
// Forward: a workgroup takes a row or a part of one; every lane keeps a running
// maximum and sum over its units of 16 bytes and they are joined at the end, the
// parts of a row by a second kernel.  Measured (4096 rows of 131072 bf16): with entropy
// 235 us for 1.07 GB, 4.6 TB/s, where the 10 vector instructions per value (an exponential
// takes the time of 4) bound it; backward 388 us for 2.15 GB, 5.5 TB/s.  One row of
// 32000 with 20 alternatives: 9.6 us, a chain of loads, sums, threshold and ranks.
//
// Alternatives (the `top` largest, equal ones by index): every lane also keeps the
// first of its units that holds its maximum.  The lanes form 64 groups; the top-th
// of the groups' greatest (maximum, unit) is a threshold: at least `top` values are at
// or above it, all of them in the units of the lanes that reach it (few more than
// `top`), which are read once more, from L2.  What is at or above the threshold is
// ranked by counting.  Where that is more than the list in LDS holds (rows of equal
// values), the values are taken one by one instead.
#include <math.h>

#include "block.h"

namespace mosa {

namespace {

constexpr int kThreads = 256;
constexpr int kList = 1024;  // values that are ranked at once

// Maxima in one instruction: the compiler quiets NaN of fmaxf's arguments before each (2
// instructions of 11 per value).  Quiet NaN are left out, as by fmaxf; a signaling one
// becomes the result, so that what is found by maxima is found again in rows with NaN.
__device__ __forceinline__ float max2(float x, float y) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
    return r;
}
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}

// Order of two values as unsigned numbers: larger first counts as larger; NaN as
// -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }

// A row in units of 16 bytes, counted from the aligned address at or before its
// first value: the first and the last unit may hold fewer of its values.
template <typename ST>
struct Row {
    static constexpr int E = Unit<ST>::E;
    const ST* p;  // aligned
    int lead, V, units, begin, end;  // begin .. end - 1: the units that are the row's throughout
    __device__ __forceinline__ Row(const char* base, int64_t stride, int64_t r, int V) : V(V) {
        const ST* at = reinterpret_cast<const ST*>(base) + r * stride;
        lead = (int)(((uintptr_t)at & 15) / sizeof(ST));
        p = at - lead;
        units = (int)(((int64_t)lead + V + E - 1) / E);
        begin = lead > 0;
        end = (int)(((int64_t)lead + V) / E);
    }
    __device__ __forceinline__ int first(int u) const { return u * E - lead; }  // index of a unit's first value
    __device__ __forceinline__ bool whole(int u) const { return u >= begin && u < end; }
    // Unit u, -inf in the place of values that are not the row's: its load where it is a whole one, and after
    // the loads of others the rest.
    __device__ __forceinline__ void load(Unit<ST>& v, int u) const {
        constexpr uint32_t none = sizeof(ST) == 2 ? 0xff80ff80u : 0xff800000u;
        v.u = make_uint4(none, none, none, none);
        if (whole(u)) v.load(p + (int64_t)u * E);
    }
    __device__ __forceinline__ void get(const Unit<ST>& v, int u, float (&x)[E]) const {
        v.get(x);
        if (u >= 0 && u < units && !whole(u)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int64_t j = (int64_t)first(u) + e;
                if (j >= 0 && j < V) x[e] = ld1<ST>(p + (int64_t)u * E + e);
            }
        }
    }
};

// Running maximum m and sums over the values, in log2 units: l of w = 2^(x c - b)
// and s of w (x c - b), c = scale log2(e).  b is m c rounded, one instruction per
// value with its product exact; what the rounding adds is common to the row and is
// taken out at the end.  Far from 0, where it would not be small, and before the
// first value b stands for m c itself, and the exponent is (x - m) c.
struct Run {
    float m, l, s;
};
constexpr float kNear = 1048576.f;  // of m c: its rounding is at most 2^-5
constexpr float kNoWeight = -1000.f;  // an exponent of weight 0 that times 0 gives 0
__device__ __forceinline__ bool near_base(float m, float c) { return fabsf(m * c) < kNear; }

// From the base of m0 to that of m1, both near: the difference of the rounded products that values were and are
// taken against.  (One of them unrounded, as in a fused product and difference, would leave its rounding, up to
// 2^-5, in the exponents.)
__device__ __forceinline__ float base_step(float m0, float m1, float c) {
#pragma clang fp contract(off)
    return m0 * c - m1 * c;
}

// Sums of a maximum r.m in terms of a maximum m >= r.m.
template <bool ENT>
__device__ __forceinline__ void rebase(Run& r, float m, float c) {
    const bool from = near_base(r.m, c), to = near_base(m, c);
    float d = from ? (to ? base_step(r.m, m, c) : fmaf(-m, c, r.m * c)) : to ? fmaf(r.m, c, -(m * c)) : (r.m - m) * c;
    d = r.m == m ? 0.f : fmaxf(d, kNoWeight);
    const float f = __builtin_amdgcn_exp2f(d);
    if constexpr (ENT) r.s = f * (r.s + d * r.l);
    r.l *= f;
    r.m = m;
}
template <bool ENT, int N>
__device__ __forceinline__ void add_values(Run& r, const float (&x)[N], float c) {
    if (near_base(r.m, c)) {
        const float b = r.m * c;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = fmaf(x[e], c, -b), w = __builtin_amdgcn_exp2f(d);
            r.l += w;
            if constexpr (ENT) r.s += w * max2(d, kNoWeight);
        }
    } else {
        const float m = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = (x[e] - m) * c, w = __builtin_amdgcn_exp2f(d);
            r.l += w;
            if constexpr (ENT) r.s += w * max2(d, kNoWeight);
        }
    }
}
// Over the 16 lanes of a row of the wave, then its four rows, in every lane.
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp_f32<0xB1, 0xf>(x));
    x = fmaxf(x, dpp_f32<0x4E, 0xf>(x));
    x = fmaxf(x, dpp_f32<0x141, 0xf>(x));
    x = fmaxf(x, dpp_f32<0x140, 0xf>(x));
    return rows4_max(x);
}
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp_f32<0xB1, 0xf>(x);
    x += dpp_f32<0x4E, 0xf>(x);
    x += dpp_f32<0x141, 0xf>(x);
    x += dpp_f32<0x140, 0xf>(x);
    return rows4_sum(x);
}
template <bool ENT>
__device__ __forceinline__ Run wave_join(Run r, float c) {
    rebase<ENT>(r, wave_max(r.m), c);
    r.l = wave_sum(r.l);
    if constexpr (ENT) r.s = wave_sum(r.s);
    return r;
}
template <bool ENT>
__device__ __forceinline__ Run join_all(const Run* r, int n, float c) {
    Run t{-INFINITY, 0.f, 0.f};
    for (int i = 0; i < n; ++i) t.m = fmaxf(t.m, r[i].m);
    for (int i = 0; i < n; ++i) {
        Run q = r[i];
        rebase<ENT>(q, t.m, c);
        t.l += q.l, t.s += q.s;
    }
    return t;
}
// log sum exp(scale (x - m)): with b for m c, 2^(m c - b) too much.
__device__ __forceinline__ float log_sum(const Run& t, float c) {
    return logf(t.l) + (near_base(t.m, c) ? kLn2 * fmaf(-t.m, c, t.m * c) : 0.f);
}

// Scratch of a row's parts: their Runs, then their lists of keys.
struct PartBuf {
    Run* run;        // [R][P]
    uint64_t* keys;  // [R][P][top]
};

// The outputs of a row, by one lane.
template <typename ST>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int r, const Run& t, float c) {
    // nothing but -inf: every weight is 0
    const bool none = t.m == -INFINITY && t.l == 0.f;
    const float L = none ? -INFINITY : log_sum(t, c);
    if (a.stats) a.stats[2 * (int64_t)r] = t.m, a.stats[2 * (int64_t)r + 1] = L;
    if (a.lse) a.lse[r] = none ? -INFINITY : a.scale * t.m + L;
    if (a.entropy) a.entropy[r] = none ? 0.f : logf(t.l) - kLn2 * t.s / t.l;
    if (a.logp) {
        const int j = a.target[r];
        float v = 0.f;
        if (j >= 0 && j < a.V) {
            const float x = ld1<ST>(reinterpret_cast<const ST*>(a.x) + (int64_t)r * a.row + j);
            v = none ? -INFINITY : a.scale * (x - t.m) - L;
        }
        a.logp[r] = v;
    }
}

// The `top` largest of n distinct keys, in order, with their log p.  (t.l is NaN in a row
// with NaN or +inf.)  put(rank, key, log p).
template <int T, typename F>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int top, F put) {
    for (int i = threadIdx.x; i < n; i += T) {
        const uint64_t k = keys[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += keys[j] > k;
        if (rank < top && k) put(rank, k);
    }
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int r, int at, uint64_t key, const Run& t, float L) {
    const float x = value_of((uint32_t)(key >> 32));
    a.top_logp[(int64_t)r * a.top + at] = t.l != t.l ? t.l : x == -INFINITY ? x : a.scale * (x - t.m) - L;
    a.top_index[(int64_t)r * a.top + at] = (int)~(uint32_t)key;
}

// The top-th largest of 64 keys, one per lane (equal keys, 0, in the order of the lanes).
__device__ __forceinline__ uint64_t wave_kth(uint64_t key, int top) {
    const int lane = threadIdx.x & 63;
    int rank = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) {
        const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), j) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)key, j);
        rank += k > key || (k == key && j < lane);
    }
    const int at = __builtin_ctzll(__ballot(rank == top - 1));
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), at) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)key, at);
}

template <typename ST, bool ENT, bool TOP, int T>
__global__ __launch_bounds__(T) void logprob_kernel(LogprobArgs a, int P, int per, PartBuf buf) {
    constexpr int E = Unit<ST>::E, U = 4, W = T / 64;
    __shared__ Run runs[W];
    __shared__ uint64_t keys[TOP ? kList : 1];
    __shared__ uint64_t threshold;
    __shared__ int lanes[TOP ? T : 1], count[2];
    const int r = blockIdx.x / P, part = blockIdx.x % P, tid = threadIdx.x;
    const Row<ST> row(a.x, a.row, r, a.V);
    const int u0 = part * per, u1 = min(row.units, u0 + per);  // (the last part may be empty)
    const float c = a.scale * kLog2e;
    Run t{-INFINITY, 0.f, 0.f};
    float best = -INFINITY;
    int unit = -1;  // the first unit that holds the lane's maximum
    for (int u = u0 + tid; u < u1; u += U * T) {
        Unit<ST> v[U];
        float x[U][E];
#pragma unroll
        for (int i = 0; i < U; ++i) row.load(v[i], u + i * T < u1 ? u + i * T : -1);
#pragma unroll
        for (int i = 0; i < U; ++i) row.get(v[i], u + i * T < u1 ? u + i * T : -1, x[i]);
        float m = t.m;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float w = -INFINITY;  // (NaN are left out)
#pragma unroll
            for (int e = 0; e < E; e += 2) w = max3(w, x[i][e], x[i][e + 1]);
            if constexpr (TOP) {
                if ((w > best || unit < 0) && u + i * T < u1) best = w, unit = u + i * T;
            }
            m = fmaxf(m, w);
        }
        if (m > t.m) rebase<ENT>(t, m, c);
#pragma unroll
        for (int i = 0; i < U; ++i) add_values<ENT>(t, x[i], c);
    }
    t = wave_join<ENT>(t, c);
    if ((tid & 63) == 0) runs[tid >> 6] = t;
    uint64_t mine = unit < 0 ? 0 : key_of(best, unit);  // (a lane without units: below every key)
    if constexpr (TOP) {
        keys[tid] = mine;
        if (tid < 2) count[tid] = 0;
    }
    __syncthreads();
    if (TOP || tid < 64) t = join_all<ENT>(runs, W, c);
    if (tid == 0) {
        if (P > 1) buf.run[(int64_t)r * P + part] = t;
        else write_row<ST>(a, r, t, c);
    }
    if constexpr (TOP) {
        if (t.l != t.l) {  // NaN (or +inf) in some lane's units: every lane's maximum without them
            best = -INFINITY, unit = -1;
            for (int u = u0 + tid; u < u1; u += T) {
                Unit<ST> v;
                float x[E], w = -INFINITY;
                row.load(v, u);
                row.get(v, u, x);
#pragma unroll
                for (int e = 0; e < E; ++e) w = x[e] > w ? x[e] : w;
                if (w > best || unit < 0) best = w, unit = u;
            }
            keys[tid] = mine = unit < 0 ? 0 : key_of(best, unit);
            __syncthreads();
        }
        const float L = P > 1 ? 0.f : log_sum(t, c);
        auto put = [&](int rank, uint64_t key) {
            if (P > 1) buf.keys[((int64_t)r * P + part) * a.top + rank] = key;
            else write_top(a, r, rank, key, t, L);
        };
        if (tid < 64) {
            uint64_t group = keys[tid];
#pragma unroll
            for (int w = 1; w < W; ++w) {
                const uint64_t k = keys[tid + 64 * w];
                group = k > group ? k : group;
            }
            const uint64_t k = wave_kth(group, a.top);
            if (tid == 0) threshold = k;
        }
        __syncthreads();
        const uint64_t least = threshold;  // 0: every value
        if (mine >= least && mine) lanes[atomicAdd(&count[0], 1)] = tid;
        __syncthreads();  // (keys are read until here)
        const int each = (u1 - u0 + T - 1) / T, total = count[0] * each;
        // the units of those lanes: f(index, value) for what is at or above the threshold
        auto visit = [&](auto f) {
            for (int i = tid; i < total; i += T) {
                const int u = u0 + lanes[i / each] + (i % each) * T;
                if (u >= u1) continue;
                Unit<ST> v;
                float x[E];
                row.load(v, u);
                row.get(v, u, x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int j = row.first(u) + e;
                    if (j >= 0 && j < a.V && key_of(x[e], u) >= least) f(j, x[e]);
                }
            }
        };
        visit([&](int j, float x) {
            const int n = atomicAdd(&count[1], 1);
            if (n < kList) keys[n] = key_of(x, j);
        });
        __syncthreads();
        const int n = count[1];
        if (n <= kList) {
            rank_keys<T>(keys, n, a.top, put);
        } else {
            uint64_t last = ~(uint64_t)0;
            for (int k = 0; k < a.top; ++k) {
                uint64_t next = 0;
                visit([&](int j, float x) {
                    const uint64_t key = key_of(x, j);
                    if (key < last && key > next) next = key;
                });
                keys[tid] = next;
                __syncthreads();
                for (int o = T / 2; o > 0; o >>= 1) {
                    if (tid < o && keys[tid + o] > keys[tid]) keys[tid] = keys[tid + o];
                    __syncthreads();
                }
                last = keys[0];
                __syncthreads();
                if (tid == 0) put(k, last);
            }
        }
        if (P > 1) {  // a part of fewer values
            for (int k = n + tid; k < a.top; k += T) put(k, 0);
        }
    }
}

// The parts of a row joined.
template <typename ST, bool ENT, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobArgs a, int P, PartBuf buf) {
    __shared__ uint64_t keys[TOP ? kList : 1];
    const int r = blockIdx.x;
    const float c = a.scale * kLog2e;
    const Run t = join_all<ENT>(buf.run + (int64_t)r * P, P, c);
    if (threadIdx.x == 0) write_row<ST>(a, r, t, c);
    if constexpr (TOP) {
        const int n = P * a.top;  // (at most kList / 2: see parts_of)
        const float L = log_sum(t, c);
        for (int i = threadIdx.x; i < n; i += kThreads) keys[i] = buf.keys[(int64_t)r * n + i];
        __syncthreads();
        rank_keys<kThreads>(keys, n, a.top, [&](int rank, uint64_t key) { write_top(a, r, rank, key, t, L); });
    }
}

// A wave takes `per` units of a row.
template <typename ST>
__global__ __launch_bounds__(kThreads) void logprob_bwd_kernel(LogprobArgs a, int P, int per, int64_t waves) {
    constexpr int E = Unit<ST>::E;
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); w < waves;
         w += (int64_t)gridDim.x * (kThreads / 64)) {
        const int r = (int)(w / P), part = (int)(w % P);
        const Row<ST> row(a.x, a.row, r, a.V);
        ST* out = reinterpret_cast<ST*>(a.dx) + (int64_t)r * a.drow - row.lead;
        const bool even = ((uintptr_t)out & 15) == 0;
        const int u0 = part * per, u1 = min(row.units, u0 + per);
        const float M = a.stats[2 * (int64_t)r], L = a.stats[2 * (int64_t)r + 1], c = a.scale * kLog2e;
        const bool none = M == -INFINITY && L == -INFINITY;
        const int t = a.target ? a.target[r] : -1;
        const bool has = a.dlogp && t >= 0 && t < a.V && !none;
        const float g = has ? a.scale * a.dlogp[r] : 0.f, gl = a.dlse ? a.scale * a.dlse[r] : 0.f;
        const float ge = a.dent ? a.scale * a.dent[r] : 0.f, H = a.dent ? a.entropy[r] : 0.f;
        // dx = p (A - ge log p) + g at the target
        const float A = gl - g - ge * H, M0 = M == -INFINITY ? 0.f : M, L0 = none ? 0.f : L;
        const float l2 = L0 * kLog2e, gk = ge * kLn2;
        for (int u = u0 + lane; u < u1; u += 64) {
            Unit<ST> v;
            float x[E];
            row.load(v, u);
            row.get(v, u, x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = (x[e] - M0) * c - l2, p = __builtin_amdgcn_exp2f(d);
                x[e] = p * (A - gk * max2(d, kNoWeight));
            }
            const int j = t - row.first(u);
            if (has && j >= 0 && j < E) {
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] += e == j ? g : 0.f;
            }
            if (even && row.whole(u)) {
                Unit<ST> o;
                o.set(x);
                o.store(out + (int64_t)u * E);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int64_t i = (int64_t)row.first(u) + e;
                    if (i >= 0 && i < a.V) st1<ST>(out + (int64_t)u * E + e, x[e]);
                }
            }
        }
    }
}

// Lanes of a workgroup, parts of a row and units of each; parts take a second kernel (4 us and the gap before it).
// Measured (us, logits not in a cache): up to a row per CU 1024 lanes take a row at once (128 rows of 50001 fp32: 12.8
// against 16.3 with parts for 256 lanes; 1 of 32000 bf16 with 20 alternatives: 10 against 12), in parts only very long
// ones of a few (1 of 200000 fp32: 10.7 in 4 parts against 17.2).  More rows: 256 lanes (700 of 100000 bf16: 34 against 46),
// and two parts where long rows are few for the chip (300 of 50001 fp32: 21.5 against 23.7; 512 of 32000 bf16: 11.4
// without parts against 13.4).  Many short rows: a wave each (8192 of 1000 bf16: 8 against 14, with 5 alternatives 19
// against 35; of 8000: 23 against 22 and 39 against 40).
struct Split {
    int T, P, per;
};
Split parts_of(int dtype, int R, int V, int top) {
    const int E = dtype == kBF16 ? 8 : 4;
    const int64_t units = ((int64_t)V + 2 * E - 2) / E;  // (a row that does not start at a unit)
    int T = R > 4 * kCus && units <= (top ? 1024 : 512) ? 64 : kThreads;
    int64_t P = R > kCus && R < 2 * kCus && units >= 8192 ? 2 : 1;
    if (R <= kCus && units > 4 * kThreads) {
        T = 1024;
        if (units >= 16 * 1024) P = kCus / R < units / 4096 ? kCus / R : units / 4096;
    }
    if (top && P > kList / 2 / top) P = kList / 2 / top;
    if (P < 1) P = 1;
    const int64_t per = (units + P - 1) / P;
    return {T, (int)((units + per - 1) / per), (int)per};
}

template <typename ST, bool ENT, bool TOP>
int forward_t(const LogprobArgs& a, const Split& s, const PartBuf& buf, hipStream_t stream) {
    auto kern = s.T == 1024 ? logprob_kernel<ST, ENT, TOP, 1024>
                : s.T == 64 ? logprob_kernel<ST, ENT, TOP, 64> : logprob_kernel<ST, ENT, TOP, kThreads>;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.R * s.P)), dim3(s.T), 0, stream, a, s.P, s.per, buf);
    if (hipGetLastError() != hipSuccess) return -1;
    if (s.P > 1) {
        hipLaunchKernelGGL((logprob_join_kernel<ST, ENT, TOP>), dim3(a.R), dim3(kThreads), 0, stream, a, s.P, buf);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}

}  // namespace

size_t logprob_scratch_bytes(int dtype, int R, int V, int top) {
    const Split s = parts_of(dtype, R, V, top);
    if (s.P == 1) return 0;
    const size_t runs = ((size_t)R * s.P * sizeof(Run) + 255) / 256 * 256;
    return runs + (size_t)R * s.P * top * sizeof(uint64_t);
}

int launch_logprobs(int dtype, const LogprobArgs& a, void* scratch, hipStream_t stream) {
    const Split s = parts_of(dtype, a.R, a.V, a.top);
    const bool top = a.top > 0 && a.top_logp;
    PartBuf buf{};
    if (s.P > 1) {
        buf.run = static_cast<Run*>(scratch);
        buf.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(scratch) +
                                               ((size_t)a.R * s.P * sizeof(Run) + 255) / 256 * 256);
    }
    auto go = [&](auto st) {
        using ST = decltype(st);
        if (top) return a.entropy ? forward_t<ST, true, true>(a, s, buf, stream) : forward_t<ST, false, true>(a, s, buf, stream);
        return a.entropy ? forward_t<ST, true, false>(a, s, buf, stream) : forward_t<ST, false, false>(a, s, buf, stream);
    };
    return dtype == kBF16 ? go(uint16_t{}) : go(float{});
}

int launch_logprobs_bwd(int dtype, const LogprobArgs& a, hipStream_t stream) {
    const int E = dtype == kBF16 ? 8 : 4;
    const int per = 256;  // units of a wave: 4 per lane
    const int64_t units = ((int64_t)a.V + 2 * E - 2) / E, P = (units + per - 1) / per, waves = P * a.R;
    const int64_t need = (waves + kThreads / 64 - 1) / (kThreads / 64), most = 1 << 22, blocks = need < most ? need : most;
    if (dtype == kBF16)
        hipLaunchKernelGGL((logprob_bwd_kernel<uint16_t>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, (int)P, per, waves);
    else
        hipLaunchKernelGGL((logprob_bwd_kernel<float>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, (int)P, per, waves);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace mosa
