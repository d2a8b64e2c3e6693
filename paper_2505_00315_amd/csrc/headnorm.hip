// Norm and rotation of the query and key rows of every head, forward and
// backward, in one pass over the rows.
//
//   y = R(p) n,  n = w z,  z = x s,  s = 1 / sqrt(mean(x^2) + eps)
//   dn = R(p)^T dy,  dw = sum over rows of dn z,
//   dx = s (g - z mean(g z)),  g = dn w
//
// Both passes move each row once (forward 2, backward 3 row transfers) and do
// about 10 to 30 operations per value, so memory bounds them: a row lies across
// the 4 to 32 lanes that read 16 bytes of it each, and its mean is a sum over
// those lanes by register moves.  The backward recomputes s from x, which it
// has to read anyway, so the forward keeps nothing.
//
// A workgroup takes a group of tokens with all their heads.  The (cos, sin)
// pairs of a token are the same for all its heads: they are computed once per
// group into LDS (a table in memory would add its rows to the traffic).  The
// angle is reduced in 64 bits, p theta / 2 pi less its nearest integer, so that
// far positions lose nothing; the remaining fraction of a turn goes through
// the accurate fp32 sine and cosine.
//
// Measured (bf16, 4 x 4096 tokens, 32 query and 8 key heads of 128, all columns
// turned): forward 73 us for 336 MB, 4.6 TB/s; backward 104 us for 505 MB, 4.8
// TB/s, and 5 us for the sum of the 1024 partials of dwq and dwk (a large copy on
// the same card: 5.2 TB/s).  One token of 8 + 2 heads of 64: 4.4 us, a launch and
// two memory latencies.
#include <math.h>

#include "heads.h"

namespace mosa {

namespace {

constexpr int kGroupTokens = 8;  // most tokens of a group (LDS: 8 * 64 pairs = 4 KB)
// Workgroups of the backward: each leaves one partial of dwq and dwk.
// Four per CU keep 64 KB of loads per CU in flight (256 lanes, x and dy of 2 rows).
constexpr int kBwdBlocks = 1024;
constexpr int kFwdBlocks = 2048;

// Sums of dwq and dwk.  With fp32 storage they are taken in 64 bits, so that the
// result is rounded once, whatever the number of rows (in 32 bits the error was
// three times that).  bf16 storage rounds the result to 2^-9, far above the
// error of a lane's few dozen terms in fp32; only the partials' sum is in 64 bits.
template <typename ST>
using DwSum = std::conditional_t<sizeof(ST) == 4, double, float>;

template <typename ST, int DH>
struct NormGeom {
    static constexpr int E = 16 / (int)sizeof(ST);  // values per lane
    static constexpr int LPR = DH / E;              // lanes per row
    static constexpr int RP = 256 / LPR;            // rows per pass of a workgroup
};

// Sum over the LPR = 4, 8, 16 or 32 lanes of a row, in every one of them.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float x) {
    x += dpp_f32<0xB1, 0xf>(x);   // lane ^ 1
    x += dpp_f32<0x4E, 0xf>(x);   // lane ^ 2
    if constexpr (LPR >= 8) x += dpp_f32<0x141, 0xf>(x);   // the other half of 8
    if constexpr (LPR >= 16) x += dpp_f32<0x140, 0xf>(x);  // the other half of 16
    if constexpr (LPR >= 32) x += __shfl_xor(x, 16, 64);
    return x;
}

template <typename ST> struct Chunk;  // the 16 bytes of a lane
template <> struct Chunk<uint16_t> {
    uint4 u;
    __device__ __forceinline__ void get(float (&x)[8]) const {
        Frag8<uint16_t> f;
        f.v = __builtin_bit_cast(bf16x8, u);
        frag8_to_f32<uint16_t>(f, x);
    }
    __device__ __forceinline__ void set(const float (&x)[8]) { u = __builtin_bit_cast(uint4, frag8_from<uint16_t>(x).v); }
};
template <> struct Chunk<float> {
    uint4 u;
    __device__ __forceinline__ void get(float (&x)[4]) const {
        x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    }
    __device__ __forceinline__ void set(const float (&x)[4]) {
        u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// What a lane does to its columns when a row is turned: the same for every row.
template <typename ST, int DH>
struct Turn {
    static constexpr int E = NormGeom<ST, DH>::E;
    int c0, partner, pair;  // first column, lane with the other columns of the pairs (halves), first pair
    bool on, second;
    __device__ __forceinline__ Turn(const NormArgs& a, int lane) {
        const int li = lane % NormGeom<ST, DH>::LPR, half = a.rope / 2;
        c0 = li * E;
        on = c0 < a.rope;
        second = a.halves && c0 >= half;
        partner = lane;
        pair = c0 / 2;
        if (a.halves && on) {
            partner = second ? lane - half / E : lane + half / E;
            pair = second ? c0 - half : c0;
        }
    }
};

// x turned by the token's angles (sign 1) or back (sign -1).  other: the
// partner lane's columns (halves).  cs: the token's (cos, sin) pairs.
template <typename ST, int DH>
__device__ __forceinline__ void turn_row(const NormArgs& a, const Turn<ST, DH>& t, float (&x)[Turn<ST, DH>::E],
                                         const float (&other)[Turn<ST, DH>::E], const float2* cs, float sign) {
    constexpr int E = Turn<ST, DH>::E;
    if (!t.on) return;
    if (a.halves) {
        const float sg = t.second ? sign : -sign;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float2 c = cs[t.pair + e];
            x[e] = x[e] * c.x + other[e] * (sg * c.y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            if (t.c0 + e >= a.rope) break;
            const float2 c = cs[t.pair + e / 2];
            const float u = x[e], v = x[e + 1], s = sign * c.y;
            x[e] = u * c.x - v * s;
            x[e + 1] = u * s + v * c.x;
        }
    }
}

template <typename ST, int DH>
__device__ __forceinline__ Chunk<ST> partner_chunk(const Chunk<ST>& x, const Turn<ST, DH>& t) {
    Chunk<ST> y;
    y.u.x = __shfl(x.u.x, t.partner, 64);
    y.u.y = __shfl(x.u.y, t.partner, 64);
    y.u.z = __shfl(x.u.z, t.partner, 64);
    y.u.w = __shfl(x.u.w, t.partner, 64);
    return y;
}

// Columns c0 .. c0 + E - 1 of a weight vector (NULL: ones).
template <typename ST, int E>
__device__ __forceinline__ void load_weight(const void* w, int c0, float (&x)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 1.f;
    if (w) {
        Chunk<ST> c;
        c.u = *reinterpret_cast<const uint4*>(static_cast<const ST*>(w) + c0);
        c.get(x);
    }
}

struct GroupLds {
    float2 cs[kGroupTokens * kMaxTurns];
    int b[kGroupTokens], t[kGroupTokens];
};

// Tokens tok0 .. tok0 + n - 1 (flattened b T + t): where they are and their pairs.
__device__ __forceinline__ void load_group(const NormArgs& a, GroupLds& g, int64_t tok0, int n) {
    const int half = a.rope / 2;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int tok = (int)(tok0 + i);
        g.b[i] = tok / a.T;
        g.t[i] = tok % a.T;
    }
    for (int i = threadIdx.x; i < n * half; i += 256) {
        const int tl = i / half, j = i % half, tok = (int)(tok0 + tl);
        const int p = a.pos ? a.pos[tok] : tok % a.T;
        const double turns = (double)p * a.turns.t[j];
        const float f = (float)(turns - rint(turns));
        float s, c;
        sincospif(2.f * f, &s, &c);
        g.cs[tl * half + j] = make_float2(c, s);
    }
}

template <typename ST, int DH>
__global__ __launch_bounds__(256) void qk_norm_kernel(NormArgs a, int TB, FastDiv hq, FastDiv hk) {
    using G = NormGeom<ST, DH>;
    constexpr int E = G::E, U = 2;
    __shared__ GroupLds lds;
    const int lane = threadIdx.x & 63, slot = threadIdx.x / G::LPR;
    const Turn<ST, DH> turn(a, lane);
    const int cp = turn.c0 + (turn.partner - lane) * E;  // the partner's columns
    const int64_t total = (int64_t)a.B * a.T;
    for (int64_t tok0 = (int64_t)blockIdx.x * TB; tok0 < total; tok0 += (int64_t)gridDim.x * TB) {
        const int nt = (int)min((int64_t)TB, total - tok0);
        __syncthreads();
        load_group(a, lds, tok0, nt);
        __syncthreads();
        static_for<0, 2>([&](auto kc) {
            constexpr int K = decltype(kc)::value;
            const Rows &in = K ? a.k : a.q, &out = K ? a.ko : a.qo;
            const FastDiv& heads = K ? hk : hq;
            const int R = nt * heads.n;
            float w[E], wp[E];
            load_weight<ST, E>(K ? a.wk : a.wq, turn.c0, w);
            load_weight<ST, E>(K ? a.wk : a.wq, cp, wp);
            for (int r0 = slot; r0 < R; r0 += U * G::RP) {
                Chunk<ST> x[U];
                ST* to[U];
                int tl[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    int h;
                    fast_divmod(heads, min(r0 + u * G::RP, R - 1), tl[u], h);
                    const int b = lds.b[tl[u]], t = lds.t[tl[u]];
                    x[u].u = *reinterpret_cast<const uint4*>(row_ptr<ST>(in, b, h, t) + turn.c0);
                    to[u] = row_ptr<ST>(out, b, h, t) + turn.c0;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float v[E], o[E];
                    x[u].get(v);
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) ss += v[e] * v[e];
                    const float s = rsqrtf(lanes_sum<G::LPR>(ss) * (1.f / DH) + a.eps);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = v[e] * s * w[e];
                    if (a.halves) {
                        partner_chunk<ST, DH>(x[u], turn).get(o);
#pragma unroll
                        for (int e = 0; e < E; ++e) o[e] = o[e] * s * wp[e];
                    }
                    turn_row<ST, DH>(a, turn, v, o, lds.cs + tl[u] * (a.rope / 2), 1.f);
                    Chunk<ST> y;
                    y.set(v);
                    if (r0 + u * G::RP < R) *reinterpret_cast<uint4*>(to[u]) = y.u;
                }
            }
        });
    }
}

template <typename ST, int DH, bool DW>
__global__ __launch_bounds__(256) void qk_norm_bwd_kernel(NormArgs a, int TB, FastDiv hq, FastDiv hk,
                                                          DwSum<ST>* __restrict__ partial) {
    using G = NormGeom<ST, DH>;
    constexpr int E = G::E, U = 2;
    __shared__ GroupLds lds;
    __shared__ DwSum<ST> red[DW ? 256 * E : 1];
    const int lane = threadIdx.x & 63, slot = threadIdx.x / G::LPR;
    const Turn<ST, DH> turn(a, lane);
    DwSum<ST> acc[2][E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[0][e] = acc[1][e] = 0;
    const int64_t total = (int64_t)a.B * a.T;
    for (int64_t tok0 = (int64_t)blockIdx.x * TB; tok0 < total; tok0 += (int64_t)gridDim.x * TB) {
        const int nt = (int)min((int64_t)TB, total - tok0);
        __syncthreads();
        load_group(a, lds, tok0, nt);
        __syncthreads();
        static_for<0, 2>([&](auto kc) {
            constexpr int K = decltype(kc)::value;
            const Rows &in = K ? a.k : a.q, &gr = K ? a.ko : a.qo, &out = K ? a.dk : a.dq;
            const FastDiv& heads = K ? hk : hq;
            const int R = nt * heads.n;
            float w[E];
            load_weight<ST, E>(K ? a.wk : a.wq, turn.c0, w);
            for (int r0 = slot; r0 < R; r0 += U * G::RP) {
                Chunk<ST> x[U], dy[U];
                ST* to[U];
                int tl[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    int h;
                    fast_divmod(heads, min(r0 + u * G::RP, R - 1), tl[u], h);
                    const int b = lds.b[tl[u]], t = lds.t[tl[u]];
                    x[u].u = *reinterpret_cast<const uint4*>(row_ptr<ST>(in, b, h, t) + turn.c0);
                    dy[u].u = *reinterpret_cast<const uint4*>(row_ptr<ST>(gr, b, h, t) + turn.c0);
                    to[u] = row_ptr<ST>(out, b, h, t) + turn.c0;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool live = r0 + u * G::RP < R;
                    float v[E], g[E], o[E];
                    x[u].get(v);
                    dy[u].get(g);
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) ss += v[e] * v[e];
                    const float s = rsqrtf(lanes_sum<G::LPR>(ss) * (1.f / DH) + a.eps);
                    if (a.halves) partner_chunk<ST, DH>(dy[u], turn).get(o);
                    turn_row<ST, DH>(a, turn, g, o, lds.cs + tl[u] * (a.rope / 2), -1.f);
                    float c = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        v[e] *= s;  // z
                        if constexpr (DW) acc[K][e] += live ? g[e] * v[e] : 0.f;
                        g[e] *= w[e];
                        c += g[e] * v[e];
                    }
                    c = lanes_sum<G::LPR>(c) * (1.f / DH);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = s * (g[e] - v[e] * c);
                    Chunk<ST> dx;
                    dx.set(v);
                    if (live) *reinterpret_cast<uint4*>(to[u]) = dx.u;
                }
            }
        });
    }
    if constexpr (DW) {  // partial[block][q, k][DH]: the rows of a pass, added in order
#pragma unroll
        for (int K = 0; K < 2; ++K) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) red[slot * DH + turn.c0 + e] = acc[K][e];
            __syncthreads();
            for (int d = threadIdx.x; d < DH; d += 256) {
                DwSum<ST> s = 0;
                for (int r = 0; r < G::RP; ++r) s += red[r * DH + d];
                partial[((size_t)blockIdx.x * 2 + K) * DH + d] = s;
            }
        }
    }
}

// dw = sum of the partials, 16 columns per workgroup: 64 strands of rows, then
// the strands in order.
template <typename ST>
__global__ __launch_bounds__(1024) void qk_norm_dw_kernel(const DwSum<ST>* __restrict__ partial, int blocks, int dh,
                                                          ST* __restrict__ dwq, ST* __restrict__ dwk) {
    __shared__ double red[64][17];
    const int c = threadIdx.x & 15, strand = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    double s = 0.0;
#pragma unroll 4
    for (int i = strand; i < blocks; i += 64) s += partial[(size_t)i * 2 * dh + col];
    red[strand][c] = s;
    __syncthreads();
    if (threadIdx.x < 16) {
        double t = 0.0;
        for (int i = 0; i < 64; ++i) t += red[i][c];
        ST* to = col < dh ? dwq : dwk;
        if (to) st1<ST>(to + (col < dh ? col : col - dh), (float)t);
    }
}

// Tokens per group: enough rows for the unrolled passes, but groups for every CU.
int group_tokens(int64_t total, int heads, int rows_per_pass, int unroll) {
    const int64_t want = ((int64_t)unroll * rows_per_pass + heads - 1) / heads, spread = total / 1024;
    const int64_t tb = want < spread ? want : spread;
    return tb < 1 ? 1 : tb > kGroupTokens ? kGroupTokens : (int)tb;
}

template <typename ST, int DH>
int norm_t(const NormArgs& a, hipStream_t stream) {
    const int64_t total = (int64_t)a.B * a.T;
    const int tb = group_tokens(total, a.Hkv, NormGeom<ST, DH>::RP, 2);
    const int64_t groups = (total + tb - 1) / tb;
    hipLaunchKernelGGL((qk_norm_kernel<ST, DH>), dim3((unsigned)(groups < kFwdBlocks ? groups : kFwdBlocks)), dim3(256),
                       0, stream, a, tb, make_fastdiv(a.Hq), make_fastdiv(a.Hkv));
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <typename ST, int DH>
int norm_bwd_t(const NormArgs& a, void* dwq, void* dwk, void* scratch, hipStream_t stream) {
    DwSum<ST>* partial = static_cast<DwSum<ST>*>(scratch);
    const int64_t total = (int64_t)a.B * a.T;
    const int tb = group_tokens(total, a.Hkv, NormGeom<ST, DH>::RP, 2);
    const int64_t groups = (total + tb - 1) / tb;
    const int blocks = (int)(groups < kBwdBlocks ? groups : kBwdBlocks);
    const bool dw = dwq || dwk;
    auto kern = dw ? qk_norm_bwd_kernel<ST, DH, true> : qk_norm_bwd_kernel<ST, DH, false>;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, stream, a, tb, make_fastdiv(a.Hq), make_fastdiv(a.Hkv), partial);
    if (hipGetLastError() != hipSuccess) return -1;
    if (dw) {
        hipLaunchKernelGGL((qk_norm_dw_kernel<ST>), dim3(2 * DH / 16), dim3(1024), 0, stream, partial, blocks, DH,
                           (ST*)dwq, (ST*)dwk);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}

}  // namespace

size_t norm_partial_bytes(int dtype, int64_t tokens, int dh) {
    return (size_t)(tokens < kBwdBlocks ? tokens : kBwdBlocks) * 2 * dh * (dtype == kBF16 ? sizeof(float) : sizeof(double));
}

int launch_qk_norm(int dtype, const NormArgs& a, hipStream_t stream) {
    return heads_by_type(dtype, a.dh, [&](auto st, auto dh) { return norm_t<decltype(st), decltype(dh)::value>(a, stream); });
}

int launch_qk_norm_bwd(int dtype, const NormArgs& a, void* dwq, void* dwk, void* scratch, hipStream_t stream) {
    return heads_by_type(dtype, a.dh, [&](auto st, auto dh) {
        return norm_bwd_t<decltype(st), decltype(dh)::value>(a, dwq, dwk, scratch, stream);
    });
}

}  // namespace mosa
