// The residual stream between two blocks: the block's output normed, gated,
// scaled and added to the stream, and the stream normed for the next block.
//
//   u = wp zy,  zy = y sy,  sy = 1 / sqrt(mean(y^2) + eps)      (or u = y)
//   h = ra x + rb g u
//   n = wn zh,  zh = h sh,  sh = 1 / sqrt(mean(h^2) + eps)
// backward, with dh and dn of the outputs:
//   dwn = sum dn zh,   D = dh + sh (e - zh mean(e zh)),  e = dn wn
//   dx = ra D,  dg = rb D u (summed as the gate is shared),  du = rb g D
//   dwp = sum du zy,   dy = sy (e - zy mean(e zy)),  e = du wp
//
// Every value is read and written once (forward 2 rows in, 2 out; backward 4 in,
// 2 out, and a token's own gate in and out), with 10 to 40 operations per value:
// memory bounds it.  A row lies across a team of lanes that keep their columns in
// registers from the loads to the stores: a quarter of a wave for short rows, up
// to a workgroup of 1024 lanes; the means are sums over the team.  The backward
// recomputes h from x and y, which it reads anyway, so that the forward keeps
// nothing and h is not rounded in between.
//
// Sums over tokens (dwp, dwn, dg of a shared gate): a lane adds up its columns
// over the rows of its team, the teams of a workgroup are added in order, and the
// workgroups' partials in a second kernel; a workgroup takes a run of rows, so a
// sequence's gate has a partial per workgroup that its rows lie in.
//
// Measured (bf16, 4 x 4096 tokens of 4096, both norms, one gate): forward 105 us for
// 537 MB, 5.1 TB/s; backward 183 us for 831 MB, 4.5 TB/s, and 7 us for the partials'
// sum (a large copy on the same card: 5.05 TB/s).  The backward waits for its
// three sums over the team one after the other; loads of the next row issued before them
// took the registers of a wave in four and were no faster.  One token of 1024: 2.4 us.
#include "block.h"

namespace mosa {

namespace {

template <typename ST, int LPR, int C>
struct TeamGeom {
    static constexpr int E = Unit<ST>::E, THREADS = LPR < 128 ? 256 : LPR, TEAMS = THREADS / LPR, WAVES = THREADS / 64;
};

// Sum over the LPR lanes of a team, in every one of them.
template <int LPR>
__device__ __forceinline__ float team_sum(float x, float (&red)[2][16], int& phase) {
    x += dpp_f32<0xB1, 0xf>(x);   // lane ^ 1
    x += dpp_f32<0x4E, 0xf>(x);   // lane ^ 2
    x += dpp_f32<0x141, 0xf>(x);  // the other half of 8
    if constexpr (LPR >= 16) x += dpp_f32<0x140, 0xf>(x);  // the other half of 16
    if constexpr (LPR == 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if constexpr (LPR >= 64) x = rows4_sum(x);
    if constexpr (LPR > 64) {  // (two buffers: a wave that writes one again has met a barrier since it was read)
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[phase][wave] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int w = 0; w < LPR / 64; ++w) x += red[phase][w];
        phase ^= 1;
    }
    return x;
}

// The columns of a lane: units li, li + LPR, ... of a row of n units.
template <typename ST, int LPR, int C>
struct Cols {
    int li, n;
    __device__ __forceinline__ bool has(int c) const { return c * LPR + li < n; }
    __device__ __forceinline__ int at(int c) const { return (c * LPR + li) * Unit<ST>::E; }
    __device__ __forceinline__ void load(Unit<ST> (&u)[C], const ST* row) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            u[c].u = make_uint4(0, 0, 0, 0);
            if (has(c)) u[c].load(row + at(c));
        }
    }
    // a weight vector (NULL: ones)
    __device__ __forceinline__ void weight(Unit<ST> (&u)[C], const void* w) const {
        constexpr uint32_t one = sizeof(ST) == 2 ? 0x3f803f80u : 0x3f800000u;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            u[c].u = make_uint4(one, one, one, one);
            if (w && has(c)) u[c].load(static_cast<const ST*>(w) + at(c));
        }
    }
};

template <typename ST, int LPR, int C>
__global__ __launch_bounds__((TeamGeom<ST, LPR, C>::THREADS)) void residual_norm_kernel(ResidualArgs a, int64_t rows) {
    using G = TeamGeom<ST, LPR, C>;
    constexpr int E = G::E;
    __shared__ float red[2][16];
    int phase = 0;
    const Cols<ST, LPR, C> cols{(int)(threadIdx.x % LPR), a.d / E};
    const float inv = 1.f / (float)a.d;
    Unit<ST> wp[C], wn[C], g[C];
    cols.weight(wp, a.wpost);
    cols.weight(wn, a.wpre);
    cols.weight(g, a.gate == kGateVector ? a.g.p : nullptr);
    for (int64_t r = (int64_t)blockIdx.x * G::TEAMS + threadIdx.x / LPR; r < rows; r += (int64_t)gridDim.x * G::TEAMS) {
        const int b = (int)(r / a.T), t = (int)(r % a.T);
        Unit<ST> x[C], y[C];
        cols.load(x, row_ptr<ST>(a.x, b, 0, t));
        if (a.has_y) cols.load(y, row_ptr<ST>(a.y, b, 0, t));
        if (a.gate >= kGateSequence) cols.load(g, row_ptr<ST>(a.g, b, 0, t));
        float h[C][E];
#pragma unroll
        for (int c = 0; c < C; ++c) x[c].get(h[c]);
        if (a.has_y) {
            float s = a.rb;
            if (a.post) {
                float ss = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[E];
                    y[c].get(v);
#pragma unroll
                    for (int e = 0; e < E; ++e) ss += v[e] * v[e];
                }
                s *= rsqrtf(team_sum<LPR>(ss, red, phase) * inv + a.eps);
            }
            ST* to = row_ptr<ST>(a.h, b, 0, t);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[E], w[E], q[E];
                y[c].get(v), wp[c].get(w), g[c].get(q);
#pragma unroll
                for (int e = 0; e < E; ++e) h[c][e] = a.ra * h[c][e] + s * v[e] * w[e] * q[e];
                Unit<ST> o;
                o.set(h[c]);
                if (cols.has(c)) o.store(to + cols.at(c));
            }
        }
        if (a.pre) {
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) ss += h[c][e] * h[c][e];
            const float s = rsqrtf(team_sum<LPR>(ss, red, phase) * inv + a.eps);
            ST* to = row_ptr<ST>(a.n, b, 0, t);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float w[E];
                wn[c].get(w);
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] *= h[c][e] * s;
                Unit<ST> o;
                o.set(w);
                if (cols.has(c)) o.store(to + cols.at(c));
            }
        }
    }
}

// The lanes' sums of the teams, added in order: f(column, total) by one lane per column.
// Called by the whole workgroup.
template <typename ST, int LPR, int C, typename F>
__device__ __forceinline__ void add_teams(const Cols<ST, LPR, C>& cols, const WideSum<ST> (&acc)[C][Unit<ST>::E],
                                          WideSum<ST>* lds, F f) {
    constexpr int E = Unit<ST>::E, TEAMS = TeamGeom<ST, LPR, C>::TEAMS;
    if constexpr (TEAMS == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (cols.has(c)) {
#pragma unroll
                for (int e = 0; e < E; ++e) f(cols.at(c) + e, acc[c][e]);
            }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) lds[threadIdx.x * E + e] = acc[c][e];
            __syncthreads();
            for (int i = threadIdx.x; i < LPR * E; i += TeamGeom<ST, LPR, C>::THREADS) {
                const int col = c * LPR * E + i;
                if (col < cols.n * E) {
                    WideSum<ST> s = 0;
                    for (int t = 0; t < TEAMS; ++t) s += lds[t * LPR * E + i];
                    f(col, s);
                }
            }
        }
        __syncthreads();
    }
}

// Workgroup k takes rows k per .. (k + 1) per - 1.  part [workgroup][3][d]: its sums
// for dwp, dwn and a vector's dg; slots [workgroup][2][d]: for a gate per sequence,
// those of the first sequence in its rows and of the last, where these have rows in
// other workgroups too.
template <typename ST, int LPR, int C>
__global__ __launch_bounds__((TeamGeom<ST, LPR, C>::THREADS)) void residual_norm_bwd_kernel(
    ResidualArgs a, int rows, int per, int sums, WideSum<ST>* __restrict__ part, WideSum<ST>* __restrict__ slots) {
    using G = TeamGeom<ST, LPR, C>;
    using W = WideSum<ST>;
    constexpr int E = G::E;
    __shared__ float red[2][16];
    __shared__ W lds[G::TEAMS > 1 ? 256 * E : 1];
    int phase = 0;
    const Cols<ST, LPR, C> cols{(int)(threadIdx.x % LPR), a.d / E};
    const int team = threadIdx.x / LPR;
    const float inv = 1.f / (float)a.d;
    const bool seq = a.gate == kGateSequence;
    Unit<ST> wp[C], wn[C], g[C];
    cols.weight(wp, a.wpost);
    cols.weight(wn, a.wpre);
    cols.weight(g, a.gate == kGateVector ? a.g.p : nullptr);
    W swp[C][E], swn[C][E], sg[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) swp[c][e] = swn[c][e] = sg[c][e] = 0;
    const int r0 = blockIdx.x * per, r1 = min(rows, r0 + per), first = r0 / a.T;
    for (int s0 = r0; s0 < r1;) {
        const int b = s0 / a.T;
        const int s1 = seq ? (int)min((int64_t)r1, (int64_t)(b + 1) * a.T) : r1;
        if (seq) cols.load(g, row_ptr<ST>(a.g, b, 0, 0));
        for (int r = s0 + team; r < s1; r += G::TEAMS) {
            const int rb = r / a.T, t = r % a.T;
            Unit<ST> x[C], y[C], dn[C], dh[C];
            cols.load(x, row_ptr<ST>(a.x, rb, 0, t));
            if (a.has_y) cols.load(y, row_ptr<ST>(a.y, rb, 0, t));
            if (a.pre) cols.load(dn, row_ptr<ST>(a.n, rb, 0, t));
            if (a.has_dh) cols.load(dh, row_ptr<ST>(a.h, rb, 0, t));
            if (a.gate == kGateToken) cols.load(g, row_ptr<ST>(a.g, rb, 0, t));
            float sy = 1.f;
            if (a.post) {
                float ss = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[E];
                    y[c].get(v);
#pragma unroll
                    for (int e = 0; e < E; ++e) ss += v[e] * v[e];
                }
                sy = rsqrtf(team_sum<LPR>(ss, red, phase) * inv + a.eps);
            }
            float D[C][E];  // gradient of h
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (a.has_dh) {
                    dh[c].get(D[c]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) D[c][e] = 0.f;
                }
            }
            if (a.pre) {
                float h[C][E], ss = 0.f, eh = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float w[E], q[E];
                    x[c].get(h[c]);
                    if (a.has_y) {
                        float v[E];
                        y[c].get(v), wp[c].get(w), g[c].get(q);
#pragma unroll
                        for (int e = 0; e < E; ++e) h[c][e] = a.ra * h[c][e] + a.rb * sy * v[e] * w[e] * q[e];
                    }
                    dn[c].get(q), wn[c].get(w);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        ss += h[c][e] * h[c][e];
                        eh += q[e] * w[e] * h[c][e];
                    }
                }
                ss = team_sum<LPR>(ss, red, phase);
                eh = team_sum<LPR>(eh, red, phase);
                const float s = rsqrtf(ss * inv + a.eps), m = eh * s * inv;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float w[E], q[E];
                    dn[c].get(q), wn[c].get(w);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float z = h[c][e] * s;
                        swn[c][e] += q[e] * z;
                        D[c][e] += s * (q[e] * w[e] - z * m);
                    }
                }
            }
            {
                const float ra = a.has_y ? a.ra : 1.f;
                ST* to = row_ptr<ST>(a.dx, rb, 0, t);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = ra * D[c][e];
                    Unit<ST> o;
                    o.set(v);
                    if (cols.has(c)) o.store(to + cols.at(c));
                }
            }
            if (a.has_y) {
                float ey = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[E], w[E], q[E], dg[E];
                    y[c].get(v), wp[c].get(w), g[c].get(q);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float du = a.rb * D[c][e], z = v[e] * sy;
                        dg[e] = du * z * w[e];
                        sg[c][e] += dg[e];
                        const float k = du * q[e];
                        swp[c][e] += k * z;
                        D[c][e] = k * w[e];  // gradient of zy (of y where it is not normed)
                        ey += D[c][e] * z;
                    }
                    if (a.dg.p && a.gate == kGateToken && cols.has(c)) {
                        Unit<ST> o;
                        o.set(dg);
                        o.store(row_ptr<ST>(a.dg, rb, 0, t) + cols.at(c));
                    }
                }
                const float m = a.post ? team_sum<LPR>(ey, red, phase) * inv : 0.f;
                ST* to = row_ptr<ST>(a.dy, rb, 0, t);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[E];
                    y[c].get(v);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = sy * (D[c][e] - v[e] * sy * m);
                    Unit<ST> o;
                    o.set(v);
                    if (cols.has(c)) o.store(to + cols.at(c));
                }
            }
        }
        if (seq && slots) {
            const bool whole = s0 == b * a.T && s1 - s0 == a.T;
            ST* to = row_ptr<ST>(a.dg, b, 0, 0);
            W* slot = slots + ((size_t)blockIdx.x * 2 + (b != first)) * a.d;
            add_teams<ST, LPR, C>(cols, sg, lds, [&](int col, W v) {
                if (whole) st1<ST>(to + col, (float)v);
                else slot[col] = v;
            });
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) sg[c][e] = 0;
        }
        s0 = s1;
    }
    W* p = part + (size_t)blockIdx.x * 3 * a.d;
    if (sums & 1) add_teams<ST, LPR, C>(cols, swp, lds, [&](int col, W v) { p[col] = v; });
    if (sums & 2) add_teams<ST, LPR, C>(cols, swn, lds, [&](int col, W v) { p[a.d + col] = v; });
    if (sums & 4) add_teams<ST, LPR, C>(cols, sg, lds, [&](int col, W v) { p[2 * a.d + col] = v; });
}

// dg of the sequences whose rows lie in several workgroups: their slots in order, by a lane per column; or, where
// sequences are long, 32 columns by 32 strands of slots, then the strands in order.  (A sequence may have as many slots
// as there are workgroups.  Backward of 1 x 4096 tokens of 1024, 2048 slots: 684 us with a lane per column, a memory's
// latency per slot or so, 40 with strands; of 32 x 512 of 2048, 32 slots: 114 and 108; of 64 x 256, 16 slots: 104 and
// 112; of 2048 x 4 of 8192, where sequences have 1 or none: 231 and 720.)
constexpr int kManySlots = 24;
template <typename ST, int STRANDS>
__global__ __launch_bounds__((STRANDS == 1 ? 256 : 32 * STRANDS)) void sequence_gate_kernel(
    ResidualArgs a, int per, const WideSum<ST>* __restrict__ slots) {
    constexpr int COLS = STRANDS == 1 ? 256 : 32;
    __shared__ double red[COLS * STRANDS];
    const int c = threadIdx.x % COLS, strand = threadIdx.x / COLS, col = blockIdx.x * COLS + c;
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        const int k0 = b * a.T / per, k1 = (b * a.T + a.T - 1) / per;
        if (k0 == k1) continue;
        // the rows of the first workgroup may begin with another sequence, those of the rest begin with this one
        const int behind = k0 * per / a.T != b;
        double s = 0.0;
        if (col < a.d) {
#pragma unroll 8
            for (int k = k0 + strand; k <= k1; k += STRANDS) s += slots[((size_t)k * 2 + (k == k0 ? behind : 0)) * a.d + col];
        }
        if constexpr (STRANDS > 1) {
            red[threadIdx.x] = s;
            __syncthreads();
            s = 0.0;
            if (strand == 0) {
                for (int i = 0; i < STRANDS; ++i) s += red[COLS * i + c];
            }
            __syncthreads();
        }
        if (strand == 0 && col < a.d) st1<ST>(row_ptr<ST>(a.dg, b, 0, 0) + col, (float)s);
    }
}
template <typename ST, int STRANDS>
void launch_sequence_gate(const ResidualArgs& a, int per, const WideSum<ST>* slots, hipStream_t stream) {
    // (a grid's second axis is bounded, and most sequences may have no slots: workgroups stride over them)
    constexpr int COLS = STRANDS == 1 ? 256 : 32, MOST = STRANDS == 1 ? 4096 : kCus;
    hipLaunchKernelGGL((sequence_gate_kernel<ST, STRANDS>), dim3((a.d + COLS - 1) / COLS, a.B < MOST ? a.B : MOST),
                       dim3(COLS * STRANDS), 0, stream, a, per, slots);
}

// 32 columns per workgroup (128 bytes of the partials at once): 32 strands of parts, then the strands in order.
template <typename ST>
__global__ __launch_bounds__(1024) void sum_parts_kernel(SumParts s) {
    __shared__ double red[1024];
    sum_parts_columns<ST, 1024>(s, blockIdx.y, blockIdx.x, red);
}

// f(LPR, C) for the team of a row of d values.  One unit per lane keeps the backward's
// sums within 128 registers, 4 waves per SIMD (with fp32 storage 93, 5 waves).  Rows of
// more than 1024 units (fp32, above 4096 values) take two per lane: a workgroup of 1024
// lanes has 128 registers for each, and 89 lie in memory (2 x 2048 tokens of 8192: backward
// 300 us for 805 MB, 2.7 TB/s; the forward 100 us for 537 MB, 5.4).
template <typename ST, typename F>
int team_for(int d, F f) {
    const int units = d / Unit<ST>::E;
    constexpr std::integral_constant<int, 1> one{};
    if (units <= 8) return f(std::integral_constant<int, 8>{}, one);
    if (units <= 16) return f(std::integral_constant<int, 16>{}, one);
    if (units <= 32) return f(std::integral_constant<int, 32>{}, one);
    if (units <= 64) return f(std::integral_constant<int, 64>{}, one);
    if (units <= 128) return f(std::integral_constant<int, 128>{}, one);
    if (units <= 256) return f(std::integral_constant<int, 256>{}, one);
    if (units <= 512) return f(std::integral_constant<int, 512>{}, one);
    if constexpr (sizeof(ST) == 4)
        if (units > 1024) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1024>{}, one);
}

// Workgroups of the backward and rows of each: as many workgroups as the chip holds at
// once, however few rows are left for each.  Each leaves partial sums, 3 vectors at most,
// so that one row per workgroup (2048 rows of 1024 bf16) writes about as many bytes of
// them as its rows have.
struct BwdSplit {
    int blocks, per;
};
template <typename ST>
BwdSplit bwd_split(const ResidualArgs& a) {
    const int64_t rows = (int64_t)a.B * a.T;
    BwdSplit s{};
    team_for<ST>(a.d, [&](auto lpr, auto c) {
        using G = TeamGeom<ST, decltype(lpr)::value, decltype(c)::value>;
        constexpr int MOST = 1024 * 256 / G::THREADS;
        int64_t per = (rows + MOST - 1) / MOST;
        per = (per + G::TEAMS - 1) / G::TEAMS * G::TEAMS;
        s.per = (int)per;
        s.blocks = (int)((rows + per - 1) / per);
        return 0;
    });
    return s;
}

template <typename ST>
int residual_bwd_t(const ResidualArgs& a, int dtype, void* dwpost, bool dgate, void* dwpre, void* scratch,
                   hipStream_t stream) {
    using W = WideSum<ST>;
    const BwdSplit s = bwd_split<ST>(a);
    W* part = static_cast<W*>(scratch);
    W* slots = dgate && a.gate == kGateSequence ? part + (size_t)s.blocks * 3 * a.d : nullptr;
    const bool gv = dgate && a.gate == kGateVector;
    const int sums = (dwpost ? 1 : 0) | (dwpre ? 2 : 0) | (gv ? 4 : 0);
    const int rows = a.B * a.T;
    team_for<ST>(a.d, [&](auto lpr, auto c) {
        constexpr int L = decltype(lpr)::value, C = decltype(c)::value;
        hipLaunchKernelGGL((residual_norm_bwd_kernel<ST, L, C>), dim3(s.blocks), dim3(TeamGeom<ST, L, C>::THREADS), 0,
                           stream, a, rows, s.per, sums, part, slots);
        return 0;
    });
    if (hipGetLastError() != hipSuccess) return -1;
    if (slots && s.blocks > 1) {
        if (a.T / s.per >= kManySlots) launch_sequence_gate<ST, 32>(a, s.per, slots, stream);
        else launch_sequence_gate<ST, 1>(a, s.per, slots, stream);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    if (sums) {
        const SumParts sp{part, s.blocks, 3, a.d, {dwpost, dwpre, gv ? a.dg.p : nullptr}};
        if (launch_sum_parts(dtype, sp, stream)) return -1;
    }
    return 0;
}

}  // namespace

int launch_sum_parts(int dtype, const SumParts& s, hipStream_t stream) {
    const dim3 grid((s.cols + 31) / 32, s.n);
    if (dtype == kBF16) hipLaunchKernelGGL((sum_parts_kernel<uint16_t>), grid, dim3(1024), 0, stream, s);
    else hipLaunchKernelGGL((sum_parts_kernel<float>), grid, dim3(1024), 0, stream, s);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

size_t residual_scratch_bytes(int dtype, const ResidualArgs& a) {
    const BwdSplit s = dtype == kBF16 ? bwd_split<uint16_t>(a) : bwd_split<float>(a);
    return (size_t)s.blocks * (3 + (a.gate == kGateSequence ? 2 : 0)) * a.d * wide_sum_bytes(dtype);
}

int launch_residual_norm(int dtype, const ResidualArgs& a, hipStream_t stream) {
    auto go = [&](auto st) {
        using ST = decltype(st);
        return team_for<ST>(a.d, [&](auto lpr, auto c) {
            constexpr int L = decltype(lpr)::value, C = decltype(c)::value;
            using G = TeamGeom<ST, L, C>;
            const int64_t rows = (int64_t)a.B * a.T, groups = (rows + G::TEAMS - 1) / G::TEAMS;
            const int64_t most = 2048 * 256 / G::THREADS;
            hipLaunchKernelGGL((residual_norm_kernel<ST, L, C>), dim3((unsigned)(groups < most ? groups : most)),
                               dim3(G::THREADS), 0, stream, a, rows);
            return hipGetLastError() == hipSuccess ? 0 : -1;
        });
    };
    return dtype == kBF16 ? go(uint16_t{}) : go(float{});
}

int launch_residual_norm_bwd(int dtype, const ResidualArgs& a, void* dwpost, bool dgate, void* dwpre, void* scratch,
                             hipStream_t stream) {
    return dtype == kBF16 ? residual_bwd_t<uint16_t>(a, dtype, dwpost, dgate, dwpre, scratch, stream)
                          : residual_bwd_t<float>(a, dtype, dwpost, dgate, dwpre, scratch, stream);
}

}  // namespace mosa
