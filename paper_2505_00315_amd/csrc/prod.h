// Products of the linear operator on the matrix cores:
//
//   C[M x N] = sum_k Q[M x K] P[K x N]     (fp32 accumulation), C^T = P^T Q^T by tile
//
// An operand lies in memory with k along its rows ("k-contiguous": x, and w^T for dx)
// or with its own axis along them (w, and both operands of dw).  A workgroup
// computes NT columns by MT rows of C; its waves own WTN x WTM of them.  Chunks of
// 128 bytes of k (64 bf16, 32 fp32) go from global memory straight into LDS, STG
// chunks in flight, one barrier per chunk; a wave's fragments of the next 32 k are
// read while the current ones are multiplied.
//
// The columns are the matrix instruction's rows, so that a lane ends up with 4
// consecutive columns of one row of C; with bf16 the two 16-column blocks of a pair
// interleave by 4 columns, so that a lane holds 8 consecutive ones and stores 16
// bytes.
//
// In LDS a k-contiguous tile is [rows][8 units of 16 bytes], unit u of row r at u ^
// f(r), f chosen so that the 8 lanes that are served at once read 8 different unit
// places.  The other tiles are [k][columns] as in memory; bf16 fragments are read from
// them transposed (ds_read_b64_tr_b16), fp32 ones value by value, with units
// permuted by k.
#pragma once

#include "block.h"
#include "gemm2.h"
#include "wattn_dma.h"

namespace mosa {

struct ProdArgs {
    const char *p, *q;    // operands: n side (P), m side (Q)
    int64_t prow, qrow;   // bytes from one row in memory to the next
    int M, N, K;
    int tm, tn;           // tiles
    int splits, kper;     // parts of K, k of each (a multiple of the chunk)
    float* part;          // splits > 1: [splits][M][N]
    // epilogue: c + bias, activation, + r
    const void* bias;
    int act;
    Matrix r, y, z;
};

// The normal distribution's tail Phi(-x) = erfc(x / sqrt 2) / 2, x >= 0.  fp32 storage: the library's erfc, to a few
// units of the result.  bf16: 2 to a polynomial of degree 8, fitted to log2 Phi(-x) over 0 .. 5.5 and falling beyond: within
// 9e-8 everywhere and 6e-5 of the result up to 5.5, where it is below 2e-8.
template <typename ST>
__device__ __forceinline__ float normal_tail(float x) {
    if constexpr (sizeof(ST) == 4) {
        return 0.5f * erfcf(x * 0.70710678118654752f);
    } else {
        float p = -8.168329941327102e-07f;
        p = fmaf(p, x, 1.4119014849711675e-05f);
        p = fmaf(p, x, -6.255447078729048e-05f);
        p = fmaf(p, x, -0.0004383266787044704f);
        p = fmaf(p, x, 0.007451288867741823f);
        p = fmaf(p, x, -0.052753835916519165f);
        p = fmaf(p, x, -0.45912837982177734f);
        p = fmaf(p, x, -1.1511142253875732f);
        p = fmaf(p, x, -0.9999998211860657f);
        return __builtin_amdgcn_exp2f(p);
    }
}
template <typename ST>
__device__ __forceinline__ float sigmoid(float z) {
    if constexpr (sizeof(ST) == 4) return 1.f / (1.f + expf(-z));
    else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
}
// The activation (not kActNone) of N values, and a gradient times its slope.  The choice is made once for all of them:
// made value by value it keeps the values' chains of instructions apart (gelu behind 8192 x 1024 by 4096 columns: 94
// us, as here 80, without an activation 70).
constexpr float kFar = 1e30f;  // infinities are taken as this where a factor of 0 meets them
template <typename ST, int N>
__device__ __forceinline__ void activate(float (&z)[N], int act) {
    if (act == kActGelu) {  // z Phi(z)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = fabsf(z[e]) > kFar ? kFar : fabsf(z[e]);
            z[e] = fmaxf(z[e], 0.f) - x * normal_tail<ST>(x);
        }
    } else if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = (z[e] < -kFar ? -kFar : z[e]) * sigmoid<ST>(z[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = z[e] > 0.f ? z[e] : z[e] != z[e] ? z[e] : 0.f;
    }
}
template <typename ST, int N>
__device__ __forceinline__ void times_slope(float (&d)[N], float (&z)[N], int act) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = z[e] > kFar ? kFar : z[e] < -kFar ? -kFar : z[e];
    if (act == kActGelu) {  // Phi(z) + z phi(z)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float q = normal_tail<ST>(fabsf(z[e]));
            const float g = sizeof(ST) == 4 ? expf(-0.5f * z[e] * z[e]) : __builtin_amdgcn_exp2f(z[e] * z[e] * (-0.5f * kLog2e));
            d[e] *= (z[e] > 0.f ? 1.f - q : q) + z[e] * g * 0.39894228040143268f;
        }
    } else if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float s = sigmoid<ST>(z[e]);
            d[e] *= s * (1.f + z[e] * (1.f - s));
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] *= z[e] > 0.f ? 1.f : z[e] != z[e] ? z[e] : 0.f;
    }
}

// The epilogue of Unit<ST>::E values from column n on in R rows m[i] (those below M): bias, activation, residual,
// stores.  Loads come first, so that they are in flight together.
template <typename ST, int R>
__device__ __forceinline__ void finish_units(const ProdArgs& a, const int (&m)[R], int n, float (&x)[R][Unit<ST>::E]) {
    constexpr int E = Unit<ST>::E;
    Unit<ST> b, r[R];
    if (a.bias) b.load(static_cast<const ST*>(a.bias) + n);
    if (a.r.p) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (m[i] < a.M) r[i].load(reinterpret_cast<const ST*>(a.r.p) + (int64_t)m[i] * a.r.row + n);
    }
    if (a.bias) {
        float v[E];
        b.get(v);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] += v[e];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (m[i] >= a.M) continue;
        Unit<ST> u;
        if (a.z.p) {
            u.set(x[i]);
            u.store(reinterpret_cast<ST*>(a.z.p) + (int64_t)m[i] * a.z.row + n);
        }
        if (a.act) activate<ST>(x[i], a.act);
        if (a.r.p) {
            float v[E];
            r[i].get(v);
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] += v[e];
        }
        u.set(x[i]);
        u.store(reinterpret_cast<ST*>(a.y.p) + (int64_t)m[i] * a.y.row + n);
    }
}

template <typename ST_, bool PKC_, bool QKC_, int NT_, int MT_, int WN_, int WM_, int STG_, int NH_ = 1>
struct ProdShape {
    using ST = ST_;
    static constexpr bool PKC = PKC_, QKC = QKC_;
    static constexpr int NT = NT_, MT = MT_, WN = WN_, WM = WM_, STG = STG_, NH = NH_, T = 64 * WN * WM;
    static constexpr int ES = (int)sizeof(ST), E = 16 / ES, KC = 128 / ES, KS = KC / 32;
    static constexpr int WTN = NT / WN, WTM = MT / WM, FN = WTN / 16, FM = WTM / 16;
    static constexpr int PU = NT * ES / 16, QU = MT * ES / 16;  // units of a [k][columns] row
    static constexpr int P_BYTES = NT * 128, Q_BYTES = MT * 128, STAGE = P_BYTES + Q_BYTES, LDS = STG * STAGE;
    static constexpr int IP = P_BYTES / 16 / T, IQ = Q_BYTES / 16 / T, L = IP + IQ;  // loads per lane and chunk
    static_assert(P_BYTES % (16 * T) == 0 && Q_BYTES % (16 * T) == 0, "whole instructions per wave");
    static constexpr bool PAIR = ES == 2 && FN > 1;  // column blocks in interleaved pairs
    static_assert(FN % NH == 0 && (!PAIR || FN / NH % 2 == 0), "pairs of column blocks");
    static_assert(LDS <= 160 * 1024 && (STG - 1) * L <= 63 && STG >= 2, "stages");
};

// Unit places of a k-contiguous tile's row; the rows of interleaved pairs are read
// as two runs of 4.
template <bool PAIR>
__device__ __forceinline__ int prod_swz(int r) {
    return PAIR ? (r & 3) | ((r >> 3) & 1) << 2 : r & 7;
}
// Unit places of a [k][columns] tile of U units a row.
template <typename ST, int U>
__device__ __forceinline__ int prod_kswz(int k, int u) {
    if constexpr (sizeof(ST) == 2) return mswz<U>(k, u);
    else return u ^ ((4 * ((k >> 3) & 3)) & (U - 1));
}

// One operand: where a lane's units come from, and its fragments.
template <class S, bool PSIDE>
struct ProdSide {
    using ST = typename S::ST;
    static constexpr bool KCON = PSIDE ? S::PKC : S::QKC, PAIR = PSIDE && S::PAIR;
    static constexpr int E = S::E, U = PSIDE ? S::PU : S::QU, I = PSIDE ? S::IP : S::IQ, T = S::T;
    static constexpr int BYTES = PSIDE ? S::P_BYTES : S::Q_BYTES;
    const char* base;  // of the tile and the split's first k
    int64_t row, step;
    int left;  // columns (or rows of C) of the tile that exist, at least one unit's
    int tid;   // of the S::T lanes that copy a tile
    uint32_t off[I];

    // unit i of the tile -> (row in memory, unit in the row) of its source
    static __device__ __forceinline__ void place(int i, int& r, int& u) {
        if constexpr (KCON) {
            r = i / 8;
            u = (i % 8) ^ prod_swz<PAIR>(r);
        } else {
            r = i / U;
            u = prod_kswz<ST, U>(r, i % U);
        }
    }
    __device__ __forceinline__ ProdSide(const ProdArgs& a, int o0, int k0, int tid) : tid(tid) {
        const int size = PSIDE ? a.N : a.M;
        row = PSIDE ? a.prow : a.qrow;
        const char* p = PSIDE ? a.p : a.q;
        base = KCON ? p + (int64_t)o0 * row + (int64_t)k0 * S::ES : p + (int64_t)k0 * row + (int64_t)o0 * S::ES;
        step = KCON ? 128 : S::KC * row;
        left = size - o0;
#pragma unroll
        for (int j = 0; j < I; ++j) {
            int r, u;
            place(tid + j * T, r, u);
            if constexpr (KCON) r = min(r, left - 1);
            else u = min(u, left / E - 1);
            off[j] = (uint32_t)(r * row) + 16 * u;
        }
    }
    // Chunk c of the split into the stage at `lds` (this wave's first block); v: k of it that exist.
    __device__ __forceinline__ void issue(int c, uint32_t lds, int v) const {
        const char* at = uniform_ptr(base + c * step);
        if (v >= S::KC) {
#pragma unroll
            for (int j = 0; j < I; ++j) lds_load16s(off[j], at, lds + 16 * T * j);
        } else {  // what lies past the last k is another valid place's, and cleared after it has landed
#pragma unroll
            for (int j = 0; j < I; ++j) {
                int r, u;
                place(tid + j * T, r, u);
                if constexpr (KCON) r = min(r, left - 1), u = min(u, v / E - 1);
                else r = min(r, v - 1), u = min(u, left / E - 1);
                lds_load16s((uint32_t)(r * row) + 16 * u, at, lds + 16 * T * j);
            }
        }
    }
    __device__ __forceinline__ void clear(unsigned char* tile, int v) const {
#pragma unroll 1
        for (int i = tid; i < BYTES / 16; i += T) {
            int r, u;
            place(i, r, u);
            if (KCON ? u * E >= v : r >= v) *reinterpret_cast<uint4*>(tile + 16 * i) = make_uint4(0, 0, 0, 0);
        }
    }
    // 16 rows (of the matrix instruction) from `o` on, 32 k from ks on.  odd: block of an interleaved pair at o.
    static __device__ __forceinline__ Frag8<ST> frag(const unsigned char* t, int o, int odd, int ks, int g, int c16) {
        Frag8<ST> f;
        if constexpr (KCON) {
            const int r = o + (PAIR ? 8 * (c16 >> 2) + (c16 & 3) + 4 * odd : c16), s = prod_swz<PAIR>(r);
            if constexpr (sizeof(ST) == 2) {
                f.v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(t + r * 128 + (((ks >> 3) + g) ^ s) * 16));
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 x = *reinterpret_cast<const float4*>(t + r * 128 + ((2 * g + h) ^ s) * 16);
                    f.v[4 * h] = x.x, f.v[4 * h + 1] = x.y, f.v[4 * h + 2] = x.z, f.v[4 * h + 3] = x.w;
                }
            }
        } else if constexpr (sizeof(ST) == 2) {
            const int col = o + (PAIR ? 8 : 4) * (c16 & 3) + 4 * odd, k = ks + 8 * g + (c16 >> 2);
            const int u = col >> 3, half = 8 * ((col >> 2) & 1);
            const u32x2 lo = lds_tr16(t + (k * U + prod_kswz<ST, U>(k, u)) * 16 + half);
            const u32x2 hi = lds_tr16(t + ((k + 4) * U + prod_kswz<ST, U>(k + 4, u)) * 16 + half);
            f.v = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
        } else {
            const int col = o + c16;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = ks + 8 * g + e;
                f.v[e] = *reinterpret_cast<const float*>(t + (k * U + prod_kswz<ST, U>(k, col >> 2)) * 16 + 4 * (col & 3));
            }
        }
        return f;
    }
};

// Tile (and part of K) `id` of a product, by the whole workgroup.
template <class S>
__device__ __forceinline__ void prod_tile(const ProdArgs& a, int id, unsigned char* smem) {
    using ST = typename S::ST;
    constexpr int STG = S::STG, KS = S::KS, L = S::L, E = S::E;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
    const int wn = wave % S::WN, wm = wave / S::WN;
    // consecutive ids: tiles of 8 row blocks side by side, so that they share operands in an XCD's L2
    const int tiles = a.tm * a.tn, split = id / tiles;
    id -= split * tiles;
    const int band = id / (8 * a.tn), bm = min(8, a.tm - 8 * band), in = id - band * 8 * a.tn;
    const int m0 = (8 * band + in % bm) * S::MT, n0 = (in / bm) * S::NT;
    const int k0 = split * a.kper, klen = min(a.kper, a.K - k0), chunks = (klen + S::KC - 1) / S::KC;

    const ProdSide<S, true> P(a, n0, k0, tid);
    const ProdSide<S, false> Q(a, m0, k0, tid);
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(smem) + 1024 * wave);
    auto issue = [&](int c, int buf) {
        const int v = klen - c * S::KC;
        P.issue(c, lds + buf * S::STAGE, v);
        Q.issue(c, lds + buf * S::STAGE + S::P_BYTES, v);
    };
    // chunk c has landed in buffer buf; k past the end are cleared
    auto clear_tail = [&](int c, int buf) {
        const int v = klen - c * S::KC;
        if (v >= S::KC || v <= 0) return;
        P.clear(smem + buf * S::STAGE, v);
        Q.clear(smem + buf * S::STAGE + S::P_BYTES, v);
        __syncthreads();
    };

    f32x4 acc[S::FN][S::FM];
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
        for (int i = 0; i < S::FM; ++i) acc[j][i] = zero4();
    // One step: HN column blocks by all row blocks over 32 k.  The fragments of the next step are read while this one
    // is multiplied; the Q fragments last for the steps of their 32 k.
    constexpr int NH = S::NH, HN = S::FN / NH, STEPS = KS * NH;  // steps of a chunk
    Frag8<ST> fp[2][HN], fq[2][S::FM];
    auto load_p = [&](Frag8<ST> (&f)[HN], int buf, int ks, int h) {
        const unsigned char* t = smem + buf * S::STAGE;
#pragma unroll
        for (int jj = 0; jj < HN; ++jj) {
            const int j = h * HN + jj, o = wn * S::WTN + (sizeof(ST) == 2 ? 32 * (j >> 1) : 16 * j);
            f[jj] = ProdSide<S, true>::frag(t, o, sizeof(ST) == 2 ? j & 1 : 0, 32 * ks, g, c16);
        }
    };
    auto load_q = [&](Frag8<ST> (&f)[S::FM], int buf, int ks) {
        const unsigned char* t = smem + buf * S::STAGE + S::P_BYTES;
#pragma unroll
        for (int i = 0; i < S::FM; ++i) f[i] = ProdSide<S, false>::frag(t, wm * S::WTM + 16 * i, 0, 32 * ks, g, c16);
    };
    constexpr int READS_P = (S::PKC ? (S::ES == 2 ? 1 : 2) : (S::ES == 2 ? 2 : 8)) * HN;
    constexpr int READS_Q = (S::QKC ? (S::ES == 2 ? 1 : 2) : (S::ES == 2 ? 2 : 8)) * S::FM;
    constexpr int MFMAS = HN * S::FM * (S::ES == 2 ? 1 : 8);

#pragma unroll
    for (int s = 0; s < STG; ++s)
        if (s < chunks) issue(s, s);
    if (chunks >= STG) wait_vmcnt<(STG - 1) * L>();
    else wait_vmcnt<0>();
    __syncthreads();
    clear_tail(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_p(fp[0], 0, 0, 0);
    load_q(fq[0], 0, 0);
    constexpr int UNROLL = STG * KS % 2 == 0 ? STG : 2 * STG;  // (the register sets' names are constants)
    for (int c0 = 0;; c0 += UNROLL) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int c = c0 + u;
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const int h = st % NH, cp = (u * STEPS + st) & 1, cq = (u * KS + st / NH) & 1;
                if (st + 1 < STEPS) {
                    load_p(fp[cp ^ 1], u % STG, (st + 1) / NH, (st + 1) % NH);
                    if (h + 1 == NH) load_q(fq[cq ^ 1], u % STG, (st + 1) / NH);
                } else {
                    // chunk c + 1 has landed and every wave has read chunk c: its buffer takes chunk c + STG.  The
                    // fragments read past the last chunk are never used.
                    if (c + STG <= chunks) wait_vmcnt<(STG - 2) * L>();
                    else wait_vmcnt<0>();
                    __syncthreads();
                    if (c + STG < chunks) issue(c + STG, u % STG);
                    clear_tail(c + 1, (u + 1) % STG);
                    __builtin_amdgcn_sched_barrier(0);
                    load_p(fp[cp ^ 1], (u + 1) % STG, 0, 0);
                    load_q(fq[cq ^ 1], (u + 1) % STG, 0);
                }
#pragma unroll
                for (int jj = 0; jj < HN; ++jj)
#pragma unroll
                    for (int i = 0; i < S::FM; ++i) mma8(acc[h * HN + jj][i], fp[cp][jj], fq[cq][i]);
                if (h + 1 == NH) sched_mix<MFMAS, READS_P + READS_Q>();
                else sched_mix<MFMAS, READS_P>();
                __builtin_amdgcn_sched_barrier(0);
            }
            if (c + 1 == chunks) goto multiplied;
        }
    }
multiplied:
    mfma_drain();
    int m[S::FM];
#pragma unroll
    for (int i = 0; i < S::FM; ++i) m[i] = m0 + wm * S::WTM + 16 * i + c16;
    constexpr int B = S::PAIR ? 2 : 1;  // column blocks that hold a lane's consecutive columns
#pragma unroll
    for (int j = 0; j < S::FN; j += B) {
        const int n = n0 + wn * S::WTN + 16 * j + 4 * B * g;
        if (n >= a.N) continue;
        float x[S::FM][E];
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = acc[j + e / 4][i][e % 4];
        if (a.splits > 1) {
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                if (m[i] >= a.M) continue;
                float* to = a.part + ((int64_t)split * a.M + m[i]) * a.N + n;
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    *reinterpret_cast<float4*>(to + e) = make_float4(x[i][e], x[i][e + 1], x[i][e + 2], x[i][e + 3]);
            }
        } else {
            finish_units<ST>(a, m, n, x);
        }
    }
}

template <class S>
__global__ __launch_bounds__((S::T)) void prod_kernel(const ProdArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    prod_tile<S>(a, xcd_logical_id(blockIdx.x, gridDim.x), smem);
}

// Two products and the sum of partials beside them in one launch: n1 and n2 workgroups (padded to multiples of 8, the
// XCDs) for the tiles of each, the rest for 32 columns of the sums each.  The product with the longer workgroups goes
// first (8192 x 4096 by 1024 beside 1024 x 8192 by 4096: 139 us, 175 with the others first, 160 one after the other).
struct ProdPair {
    ProdArgs a, b;
    SumParts sums;
    int n1, n2;
    bool second_first;
};
template <class S1, class S2>
__global__ __launch_bounds__((S1::T)) void prod_pair_kernel(const ProdPair p) {
    static_assert(S1::T == S2::T, "one workgroup size");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lead = p.second_first ? p.n2 : p.n1, b = blockIdx.x;
    if (b >= p.n1 + p.n2) {
        sum_parts_columns<typename S1::ST, S1::T>(p.sums, 0, b - p.n1 - p.n2, reinterpret_cast<double*>(smem));
    } else if ((b < lead) != p.second_first) {
        const int id = xcd_logical_id(p.second_first ? b - lead : b, p.n1);
        if (id < p.a.tm * p.a.tn * p.a.splits) prod_tile<S1>(p.a, id, smem);
    } else {
        const int id = xcd_logical_id(p.second_first ? b : b - lead, p.n2);
        if (id < p.b.tm * p.b.tn * p.b.splits) prod_tile<S2>(p.b, id, smem);
    }
}

// Few rows: W waves share the k of NT columns by 16 FM rows, each with a ring of chunks of its own (no barriers until
// the end), and their sums are added in order in LDS.  The weight's bytes bound it.  k-contiguous: 16 columns give every
// CU a part of narrow weights too, in one launch, and a CU has up to 64 KB of them in flight (weights not in a cache: 1 x
// 4096 by 4096 8.4 us, 12.5 with tiles, parts of K and their sum; 1 x 16384 by 4096 25.5 us, 5.3 TB/s).  A weight with
// the columns along its rows: a CU gets some 260 of its rows per us, however wide a piece of each it takes (16, 32 and 64
// columns, 2 to 4 chunks of each wave in flight and the strips of an XCD side by side or apart were alike), so that
// the k of a strip bound it: 32 columns of 512 rows 3.0 us (tiles of 64 columns 4.4), of 1024 6.4 (7.3), of 4096 17
// (14 with parts of K).
template <typename ST, bool PKC, int NT, int FM, int STG>
struct ProdRows : ProdShape<ST, PKC, true, NT, 16 * FM, 1, 1, STG> {};

template <class S, int W>
__global__ __launch_bounds__(64 * W) void prod_rows_kernel(const ProdArgs a) {
    using ST = typename S::ST;
    constexpr int STG = S::STG, KS = S::KS, L = S::L, E = S::E, FN = S::FN, FM = S::FM, NT = S::NT, LDC = NT + 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c16 = lane & 15;
    const int n0 = xcd_logical_id(blockIdx.x, gridDim.x) * NT;
    const ProdSide<S, true> P(a, n0, 0, lane);
    const ProdSide<S, false> Q(a, 0, 0, lane);
    unsigned char* ring = smem + wave * S::LDS;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(ring));
    const int chunks = (a.K + S::KC - 1) / S::KC, mine = (chunks - wave + W - 1) / W;
    auto issue = [&](int i, int buf) {
        const int c = wave + i * W, v = a.K - c * S::KC;
        P.issue(c, lds + buf * S::STAGE, v);
        Q.issue(c, lds + buf * S::STAGE + S::P_BYTES, v);
    };
    f32x4 acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[j][m] = zero4();
#pragma unroll
    for (int s = 0; s < STG; ++s)
        if (s < mine) issue(s, s);
    for (int i0 = 0; i0 < mine; i0 += STG) {
#pragma unroll
        for (int u = 0; u < STG; ++u) {
            const int i = i0 + u;
            if (i < mine) {
                if (i + STG <= mine) wait_vmcnt<(STG - 1) * L>();
                else wait_vmcnt<0>();
                unsigned char *tp = ring + u * S::STAGE, *tq = tp + S::P_BYTES;
                const int v = a.K - (wave + i * W) * S::KC;
                if (v < S::KC) {
                    P.clear(tp, v);
                    Q.clear(tq, v);
                    wave_sync();
                }
                __builtin_amdgcn_sched_barrier(0);
                Frag8<ST> p[KS][FN], q[KS][FM];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        p[ks][j] = ProdSide<S, true>::frag(tp, S::PAIR ? 32 * (j >> 1) : 16 * j, S::PAIR ? j & 1 : 0, 32 * ks, g, c16);
#pragma unroll
                    for (int m = 0; m < FM; ++m) q[ks][m] = ProdSide<S, false>::frag(tq, 16 * m, 0, 32 * ks, g, c16);
                }
                lds_wait();  // read before another chunk takes their place
                __builtin_amdgcn_sched_barrier(0);
                if (i + STG < mine) issue(i + STG, u);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int m = 0; m < FM; ++m) mma8(acc[j][m], p[ks][j], q[ks][m]);
            }
        }
    }
    mfma_drain();
    __syncthreads();  // every wave has read its ring
    float* sums = reinterpret_cast<float*>(smem);  // [wave][row][LDC]
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int n = S::PAIR ? 32 * (j >> 1) + 8 * g + 4 * (j & 1) : 16 * j + 4 * g;  // a lane's 4 columns of block j
#pragma unroll
        for (int m = 0; m < FM; ++m) *reinterpret_cast<f32x4*>(sums + ((wave * FM + m) * 16 + c16) * LDC + n) = acc[j][m];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * FM * (NT / E); i += 64 * W) {
        const int m = i / (NT / E), n = i % (NT / E) * E;
        if (m >= a.M || n0 + n >= a.N) continue;
        float x[1][E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[0][e] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int e = 0; e < E; ++e) x[0][e] += sums[(w * 16 * FM + m) * LDC + n + e];
        const int at[1] = {m};
        finish_units<ST>(a, at, n0 + n, x);
    }
}

template <class S, int W>
int launch_prod_rows(const ProdArgs& a, hipStream_t stream) {
    constexpr int lds = W * S::LDS;
    static_assert(lds <= 160 * 1024 && lds >= W * S::MT * (S::NT + 4) * 4, "rings, and the waves' sums in their place");
    if (allow_lds((const void*)prod_rows_kernel<S, W>, lds)) return -1;
    hipLaunchKernelGGL((prod_rows_kernel<S, W>), dim3((a.N + S::NT - 1) / S::NT), dim3(64 * W), lds, stream, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

// Parts of K added in order, and the epilogue, of one product or two.
template <typename ST>
__global__ __launch_bounds__(256) void prod_join_kernel(const ProdArgs first, const ProdArgs second) {
    constexpr int E = Unit<ST>::E;
    const ProdArgs& a = blockIdx.y ? second : first;
    const int64_t units = (int64_t)a.M * a.N / E;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (int64_t)gridDim.x * 256) {
        const int m = (int)(i * E / a.N), n = (int)(i * E - (int64_t)m * a.N);
        float x[1][E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[0][e] = 0.f;
        const float* p = a.part + i * E;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)s * a.M * a.N + e);
                x[0][e] += v.x, x[0][e + 1] += v.y, x[0][e + 2] += v.z, x[0][e + 3] += v.w;
            }
        }
        const int at[1] = {m};
        finish_units<ST>(a, at, n, x);
    }
}

template <typename ST>
int launch_prod_join(const ProdArgs& a, const ProdArgs& b, int count, hipStream_t stream) {
    int64_t units = (int64_t)a.M * a.N;
    if (count > 1 && (int64_t)b.M * b.N > units) units = (int64_t)b.M * b.N;
    const int64_t need = (units / Unit<ST>::E + 255) / 256;
    hipLaunchKernelGGL((prod_join_kernel<ST>), dim3((unsigned)(need < 4096 ? need : 4096), count), dim3(256), 0, stream, a, b);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <class S>
int launch_prod(const ProdArgs& a, hipStream_t stream) {
    if (allow_lds((const void*)prod_kernel<S>, S::LDS)) return -1;
    const int64_t blocks = (int64_t)a.tm * a.tn * a.splits;
    hipLaunchKernelGGL((prod_kernel<S>), dim3((unsigned)blocks), dim3(S::T), S::LDS, stream, a);
    if (hipGetLastError() != hipSuccess) return -1;
    return a.splits > 1 ? launch_prod_join<typename S::ST>(a, a, 1, stream) : 0;
}

// Both products with tiles of one size, their parts joined in one more launch.
template <class S1, class S2>
int launch_prod_pair(ProdPair p, hipStream_t stream) {
    constexpr int lds = S1::LDS > S2::LDS ? S1::LDS : S2::LDS;
    static_assert(lds >= S1::T * (int)sizeof(double), "the sums' place");
    if (allow_lds((const void*)prod_pair_kernel<S1, S2>, lds)) return -1;
    p.n1 = (p.a.tm * p.a.tn * p.a.splits + 7) / 8 * 8, p.n2 = (p.b.tm * p.b.tn * p.b.splits + 7) / 8 * 8;
    p.second_first = p.b.kper > p.a.kper;
    const int sums = p.sums.n ? (p.sums.cols + 31) / 32 : 0;
    hipLaunchKernelGGL((prod_pair_kernel<S1, S2>), dim3(p.n1 + p.n2 + sums), dim3(S1::T), lds, stream, p);
    if (hipGetLastError() != hipSuccess) return -1;
    if (p.a.splits > 1 && p.b.splits > 1) return launch_prod_join<typename S1::ST>(p.a, p.b, 2, stream);
    if (p.a.splits > 1) return launch_prod_join<typename S1::ST>(p.a, p.a, 1, stream);
    if (p.b.splits > 1) return launch_prod_join<typename S1::ST>(p.b, p.b, 1, stream);
    return 0;
}

}  // namespace mosa
