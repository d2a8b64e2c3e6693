// Causal attention with a sliding window and first tokens that stay visible:
// the forward over rows.
//
// One pass over the keys with the running maximum and sum of the softmax.  A
// workgroup of 4 waves owns 64 QN rows of a key head's row list (16 QN per
// wave) and walks the keys that some row of the block sees, sinks first, in
// tiles of 64 (fp32: 32) through an LDS ring filled by direct global-to-LDS loads:
//   S^T = K Q^T  (query in the lane),  p = 2^(s c - m),  O^T += V^T P^T
// with P^T as it lies in the registers of S^T and V^T read transposed from the
// row-major tile.  The products cost 4 d_head operations per pair and the
// exponential about as much issue time as a quarter of them; a wave of 32 rows
// reads each K and V fragment once per 2 matrix instructions, which is what the
// LDS can deliver at their full rate.
//
// Measured (heads of 128, bf16): 16384 tokens, 32 / 8 heads, window 4096, 4 sinks: 967
// us, 995 TFLOP/s over the pairs that are seen (an 8192^3 matrix product of the
// library on the same card: 1113); one token for each of 32 sequences of up to 8192
// keys, window 4096: 101 us, the keys and values at 5.4 TB/s.  Heads of 64, 8192
// tokens, 4 heads, window 512: 17 us, a chain of 10 tiles whose loads and
// exponentials wait for each other.  fp32: 67 to 78 TFLOP/s over a prompt of 4096
// (a library product 151), matrix instructions busy 72% of the time; one token for
// each of 32 sequences 369 us, as the products of a block's 60 rows that are none
// (61% busy) take longer than the bytes.
#include "launch_parts.h"
#include "wattn_dma.h"

namespace mosa {

namespace {

constexpr int kStages = 2;  // ring of at most 64 KB: two workgroups and more per CU (4 stages of the narrower heads: no faster)

// Launch geometry: blocks of QB rows, nb per (b, key head), each cut into parts.
struct FwdGeom {
    int nb, parts;
};

struct FwdCall {
    AttnArgs a;
    FwdGeom G;
    Parts part;
    uint32_t first;
};

// A part of a block of QB rows, by its number: 64 QN of its rows, from row `from` on.
// True (only without `again`): to be done again.
template <typename ST, int DH, int QN, int QB, bool again>
__device__ __forceinline__ bool fwd_body(unsigned char* smem, const AttnArgs& a, const FwdGeom& G, const Parts& part,
                                         uint32_t id, int from, int tid) {
    using TL = TileLoad<ST, DH>;
    constexpr int KB = TL::TB, NB = KB / 16, STG = kStages, NS = DH / 32, ND = DH / 16;
    constexpr int TILE = TL::BYTES, STAGE = 2 * TILE, LD = TL::LD;
    const int lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
    const uint32_t per = (uint32_t)G.nb * G.parts;
    const int bh = (int)(id / per), b = bh / a.Hkv, hk = bh % a.Hkv;
    id %= per;
    const int pt = (int)(id % G.parts), blk = a.W ? (int)(id / G.parts) : G.nb - 1 - (int)(id / G.parts);
    const int R = a.Tq * a.G, r0 = blk * QB, wr0 = r0 + from + 16 * QN * wave;
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn;
    const int rn = qn * a.G;  // rows of this sequence

    // keys of the block's rows, and this part's tiles of them
    KeyList list{0, 0, 0};
    if (r0 < rn) list = keys_of(a, off + a.gd.div(r0), off + a.gd.div(min(r0 + QB, rn) - 1), kn);
    const int all = (list.count + KB - 1) / KB, share = (all + G.parts - 1) / G.parts;
    const int tbeg = min(pt * share, all), ntile = min(all, tbeg + share) - tbeg;

    // this wave's rows: query index and position of row wr0 + 16 qs + c16
    int qi[QN], pos[QN];
#pragma unroll
    for (int qs = 0; qs < QN; ++qs) {
        qi[qs] = a.gd.div(min(wr0 + 16 * qs + c16, R - 1));
        pos[qs] = off + qi[qs];
    }
    float m_run[QN], l_run[QN];
    f32x4 o[QN][ND];
#pragma unroll
    for (int qs = 0; qs < QN; ++qs) {
        m_run[qs] = -__builtin_inff();
        l_run[qs] = 0.f;
#pragma unroll
        for (int db = 0; db < ND; ++db) o[qs][db] = zero4();
    }

    if (ntile > 0) {
        // positions of the wave's first and last row, for the tests of whole tiles
        const int pw0 = off + a.gd.div(min(wr0, rn - 1)), pw1 = off + a.gd.div(min(wr0 + 16 * QN, rn) - 1);
        const TL tl(wave, lane);
        const TileReads<ST, DH> rd(g, c16);
        const KeyTiles<ST, DH> kt(a.k, b, hk, tl), vt(a.v, b, hk, tl);
        const uint32_t lbase = __builtin_amdgcn_readfirstlane(lds_addr(smem));
        // tile t of this part (past the end: the last one again, into a buffer
        // that nobody reads); entries past the list are masked
        auto issue = [&](int t, int buf) __attribute__((always_inline)) {
            const int e0 = KB * (tbeg + min(t, ntile - 1));
            kt.issue(tl, list, e0, lbase + buf * STAGE);
            vt.issue(tl, list, e0, lbase + buf * STAGE + TILE);
        };
        // (the first tiles are on their way while the rows are loaded)
#pragma unroll
        for (int s = 0; s < STG - 1; ++s) issue(s, s);
        // query fragments (B operand): columns 32 st + 8 g .. + 7 (rows past the
        // sequence are clamped to its last one; they are not written)
        Frag8<ST> qf[QN][NS];
#pragma unroll
        for (int qs = 0; qs < QN; ++qs) {
            const int r = min(wr0 + 16 * qs + c16, rn - 1);
            const ST* qp = qrow_ptr<ST>(a, a.q, b, hk, r, a.gd.div(r));
#pragma unroll
            for (int st = 0; st < NS; ++st) qf[qs][st] = frag8_load<ST>(qp + 32 * st + 8 * g);
        }
#pragma unroll
        for (int qs = 0; qs < QN; ++qs)
#pragma unroll
            for (int st = 0; st < NS; ++st) take(qf[qs][st]);

        const float c2 = a.scale * kLog2e;  // scores in log2 units
        // whether the block's rows see tile e0 in part
        const int pb0 = off + a.gd.div(r0), pb1 = off + a.gd.div(min(r0 + QB, rn) - 1);
        auto in_part = [&](int e0) __attribute__((always_inline)) {
            return e0 + KB > list.count || list.key(e0 + KB - 1) > pb0 ||
                   (a.W && (e0 >= list.s ? list.key(e0) : list.lo) <= pb1 - a.W);
        };
        auto tile_step = [&](int it, auto bufc) __attribute__((always_inline)) {
            constexpr int BUF = decltype(bufc)::value;
            wait_vmcnt<(STG - 2) * 2 * LD>();  // tile it is in LDS
            __syncthreads();                   // for every wave; the buffer of tile it - 1 is free
            issue(it + STG - 1, (BUF + STG - 1) % STG);
            const unsigned char* Kb = smem + BUF * STAGE;
            const unsigned char* Vb = Kb + TILE;
            const int e0 = KB * (tbeg + it);
            // keys of the tile's window part: at least kmin, at most kmax
            const int kmax = list.key(min(e0 + KB, list.count) - 1), kmin = e0 >= list.s ? list.key(e0) : list.lo;
            if constexpr (again)
                if (in_part(e0)) {
                    keep_finite<ST, DH>(smem + BUF * STAGE + TILE, tid);
                    __syncthreads();
                }
            if (e0 >= list.s && (kmin > pw1 || (a.W && kmax <= pw0 - a.W && kmin >= a.S))) return;  // nothing for this wave

            f32x4 s[QN][NB];
#pragma unroll
            for (int sb = 0; sb < NB; ++sb) {
                Frag8<ST> kf[NS];
#pragma unroll
                for (int st = 0; st < NS; ++st) kf[st] = rd.rows(Kb, sb, st);
#pragma unroll
                for (int qs = 0; qs < QN; ++qs) s[qs][sb] = zero4();
#pragma unroll
                for (int st = 0; st < NS; ++st)
#pragma unroll
                    for (int qs = 0; qs < QN; ++qs) mma8(s[qs][sb], kf[st], qf[qs][st]);
            }
            // per-element mask only where the tile is not seen whole by the wave's rows
            if (e0 + KB > list.count || kmax > pw0 || (a.W && kmin <= pw1 - a.W)) {
                if (e0 >= list.s && (a.W == 0 || kmin >= a.S)) {
                    // keys kmin + 0 .. KB - 1, no sinks: those of the row are a run
                    // (entries past the list lie behind every row)
#pragma unroll
                    for (int qs = 0; qs < QN; ++qs) {
                        const int d = pos[qs] - kmin - 4 * g;
                        const Span run(a.W ? d - a.W + 1 : -4 * KB, d);
#pragma unroll
                        for (int sb = 0; sb < NB; ++sb)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                s[qs][sb][i] = run.has(16 * sb + i) ? s[qs][sb][i] : -__builtin_inff();
                    }
                } else {
#pragma unroll
                    for (int sb = 0; sb < NB; ++sb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int e = e0 + 16 * sb + 4 * g + i, key = list.key(e);
                            const bool in = e < list.count;
#pragma unroll
                            for (int qs = 0; qs < QN; ++qs)
                                s[qs][sb][i] = (in & sees(a, pos[qs], key)) ? s[qs][sb][i] : -__builtin_inff();
                        }
                }
            }
            // The reference maximum moves only when the tile's exceeds it by more
            // than 8 (log2 units): weights stay below 2^8, and O and l are rescaled
            // only in tiles where some row of the wave moved.
            // Again: it is a score, not in log2 units, so that differences are not
            // rounded at its size, and weights are 2^-16 of that, so that sums over
            // values of any size stay finite.
            float m_new[QN], m_use[QN];
            bool moved = false;
#pragma unroll
            for (int qs = 0; qs < QN; ++qs) {
                float mloc = -__builtin_inff();  // over the raw scores (the scale is positive)
#pragma unroll
                for (int sb = 0; sb < NB; ++sb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mloc = fmaxf(mloc, s[qs][sb][i]);
                mloc = rows4_max(mloc) * (again ? 1.f : c2);
                m_new[qs] = mloc > m_run[qs] + (again ? 8.f / c2 : 8.f) ? mloc : m_run[qs];
                m_use[qs] = m_new[qs] == -__builtin_inff() ? 0.f : m_new[qs];
                moved |= m_new[qs] != m_run[qs];
            }
            if (__builtin_amdgcn_ballot_w64(moved)) {
#pragma unroll
                for (int qs = 0; qs < QN; ++qs) {
                    const float alpha = __builtin_amdgcn_exp2f((m_run[qs] - m_use[qs]) * (again ? c2 : 1.f));
                    l_run[qs] *= alpha;
#pragma unroll
                    for (int db = 0; db < ND; ++db) o[qs][db] *= alpha;
                    m_run[qs] = m_new[qs];
                }
            }
#pragma unroll
            for (int qs = 0; qs < QN; ++qs) {
                float lsum[2] = {0.f, 0.f};
#pragma unroll
                for (int sb = 0; sb < NB; ++sb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (again) s[qs][sb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qs][sb][i] - m_use[qs], c2, -16.f));
                        else s[qs][sb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qs][sb][i], c2, -m_use[qs]));
                        lsum[i & 1] += s[qs][sb][i];
                    }
                l_run[qs] += lsum[0] + lsum[1];  // this lane's keys; the 4 lanes of a row are added at the end
            }
            // O^T += V^T P^T, 32 keys at a time: slots 0..3 are keys 4 g + i of
            // block 2 u, slots 4..7 those of block 2 u + 1.  With bf16 storage P is
            // rounded to it here, the type of the matrix operands (l sums it unrounded).
#pragma unroll
            for (int u = 0; u < NB / 2; ++u) {
                Frag8<ST> pf[QN];
#pragma unroll
                for (int qs = 0; qs < QN; ++qs) pf[qs] = pack_frag<ST>(s[qs][2 * u], s[qs][2 * u + 1]);
#pragma unroll
                for (int db = 0; db < ND; ++db) {
                    const Frag8<ST> vf = rd.cols(Vb, u, db);
#pragma unroll
                    for (int qs = 0; qs < QN; ++qs) mma8(o[qs][db], vf, pf[qs]);
                }
            }
        };
        for (int it0 = 0;; it0 += STG) {
            bool last = false;
            static_for<0, STG>([&](auto u) {
                if (last) return;
                const int it = it0 + decltype(u)::value;
                tile_step(it, u);
                last = it + 1 >= ntile;
            });
            if (last) break;
        }
        mfma_drain();     // the MFMA results are read below
        wait_vmcnt<0>();  // the trailing loads still write into the ring
        __syncthreads();
#pragma unroll
        for (int qs = 0; qs < QN; ++qs) l_run[qs] = rows4_sum(l_run[qs]);
        if constexpr (again) {
            TL ul = tl;  // (uniform, which the compiler does not see here)
            ul.lds = __builtin_amdgcn_readfirstlane(ul.lds);
#pragma unroll 1
            for (int e0 = KB * tbeg; e0 < KB * (tbeg + ntile); e0 += KB) {
                if (!in_part(e0)) continue;
                vt.issue(ul, list, e0, __builtin_amdgcn_readfirstlane(lbase));
                wait_vmcnt<0>();
                __syncthreads();
                add_not_finite<ST, DH, false>(rd, smem, g, o, [&](int r, int qs) __attribute__((always_inline)) {
                    return (e0 + r < list.count) & sees(a, pos[qs], list.key(e0 + r));
                });
                __syncthreads();
            }
#pragma unroll
            for (int qs = 0; qs < QN; ++qs) m_run[qs] = __builtin_fmaf(m_run[qs], c2, 16.f);
        } else {
            // A value of a key that the row does not see may have got in; or scores have
            // passed 2^30, where a product with the scale is rounded by more than 2^5 and
            // all weights of a row with it, out of the type's range at last.
            bool spoilt = false;
#pragma unroll
            for (int qs = 0; qs < QN; ++qs) {
                const bool sum = m_run[qs] == -__builtin_inff() || (l_run[qs] > 0x1p-32f && l_run[qs] < __builtin_inff());
                spoilt |= wr0 + 16 * qs + c16 < rn && !(sum && finite4(o[qs]));
            }
            if (any_of_workgroup(smem, wave, lane, spoilt)) return true;
        }
    }

    if (G.parts > 1) {
        const int64_t rows = (int64_t)a.B * a.Hq * a.Tq;
#pragma unroll
        for (int qs = 0; qs < QN; ++qs) {
            const int r = wr0 + 16 * qs + c16;
            if (r >= R) continue;
            const int64_t at = pt * rows + qrow_index(a, b, hk, r, qi[qs]);
            const bool live = r < rn;
#pragma unroll
            for (int db = 0; db < ND; ++db)
                *reinterpret_cast<float4*>(part.o + at * DH + 16 * db + 4 * g) =
                    live ? make_float4(o[qs][db][0], o[qs][db][1], o[qs][db][2], o[qs][db][3]) : make_float4(0, 0, 0, 0);
            if (g == 0) *reinterpret_cast<float2*>(part.ml + at * 2) = live ? make_float2(m_run[qs], l_run[qs]) : make_float2(-__builtin_inff(), 0.f);
        }
        return false;
    }
    // out = O / l, lse = m ln 2 + log l
    float inv[QN];
#pragma unroll
    for (int qs = 0; qs < QN; ++qs) {
        const int r = wr0 + 16 * qs + c16;
        const bool live = r < rn && l_run[qs] != 0.f;  // (a sum that is NaN is a result)
        inv[qs] = live ? 1.f / l_run[qs] : 0.f;
        if (!live)
#pragma unroll
            for (int db = 0; db < ND; ++db) o[qs][db] = zero4();
        if (a.lse && g == 0 && r < R)
            a.lse[qrow_index(a, b, hk, r, qi[qs])] = live ? m_run[qs] * kLn2 + logf(l_run[qs]) : -__builtin_inff();
    }
    store_rows<ST, DH, QN>(smem + wave * store_rows_bytes<ST, DH>(QN), o, inv, lane, [&](int lr) {
        const int r = wr0 + lr;
        return r < R ? qrow_ptr<ST>(a, a.out, b, hk, r, a.gd.div(r)) : nullptr;
    });
    return false;
}

// The second time, as a function of its own: what it takes of registers, and how its
// code is laid out, is no matter of the first walk.  c: the kernel's arguments, lds: its LDS.
template <typename ST, int DH, int QB>
__device__ __attribute__((noinline)) void fwd_again(const void* c, uint32_t lds, uint32_t id) {
    const FwdCall call = uniform_args<FwdCall>(c);
    unsigned char* smem = lds_at(__builtin_amdgcn_readfirstlane(lds));
    id = __builtin_amdgcn_readfirstlane(id);
#pragma unroll 1
    for (int from = 0; from < QB; from += 64) {
        __syncthreads();
        fwd_body<ST, DH, 1, QB, true>(smem, call.a, call.G, call.part, id, from, threadIdx.x);
    }
}

// Waves per SIMD that the first walk's registers allow.
template <typename ST, int DH, int QN>
constexpr int fwd_waves() {
    if (DH == 128) return 2;
    if (sizeof(ST) == 4) return DH == 64 ? 4 : 5;
    return DH == 64 ? (QN == 2 ? 3 : 4) : QN == 2 ? 4 : 6;
}

template <typename ST, int DH, int QN>
__global__ __launch_bounds__(256, (fwd_waves<ST, DH, QN>())) void wattn_fwd_kernel(FwdCall c) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    // Workgroups of one XCD take neighbouring blocks: the blocks of a key head
    // share its keys.  Without a window later blocks are longer and go first.
    const uint32_t id = c.first ? c.first + blockIdx.x : (uint32_t)xcd_logical_id(blockIdx.x, gridDim.x);
    if (fwd_body<ST, DH, QN, 64 * QN, false>(smem, c.a, c.G, c.part, id, 0, threadIdx.x))
        fwd_again<ST, DH, 64 * QN>((const void*)__builtin_amdgcn_kernarg_segment_ptr(), lds_addr(smem), id);
}

// Columns of a row of DH held by a lane: lane, lane + 64 (none past DH).
template <int DH>
struct RowLanes {
    static constexpr int N = DH > 64 ? DH / 64 : 1;
    static __device__ __forceinline__ bool has(int lane) { return DH >= 64 || lane < DH; }
};

// A row of the call: the parts in their order, M = max m_s, L = sum l_s 2^(m_s - M).
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_merge_kernel(AttnArgs a, int parts, Parts p, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.B * a.Hq * a.Tq, row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    float M = -__builtin_inff(), L = 0.f, o[RowLanes<DH>::N] = {};
    for (int s = lane; s < parts; s += 64) M = fmaxf(M, p.ml[(s * rows + row) * 2]);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
    const float mu = M == -__builtin_inff() ? 0.f : M;
#pragma unroll 4
    for (int s = 0; s < parts; ++s) {
        const float2 ml = *reinterpret_cast<const float2*>(p.ml + (s * rows + row) * 2);
        const float f = __builtin_amdgcn_exp2f(ml.x - mu);
        L += ml.y * f;
#pragma unroll
        for (int n = 0; n < RowLanes<DH>::N; ++n)
            if (RowLanes<DH>::has(lane)) {
                const float x = p.o[(s * rows + row) * DH + lane + 64 * n];
                o[n] += f == 0.f ? 0.f : x * f;
            }
    }
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    // L is 0 for a row that sees nothing (its out is 0), and NaN stays NaN
    const float f = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int n = 0; n < RowLanes<DH>::N; ++n)
        if (RowLanes<DH>::has(lane)) st1<ST>(row_ptr<ST>(a.out, b, h, i) + lane + 64 * n, o[n] * f);
    if (lane == 0 && a.lse) a.lse[row] = L == 0.f ? -__builtin_inff() : M * kLn2 + logf(L);
}

// Blocks of 128 rows share K and V fragments over two matrix instructions each
// (bf16); blocks of 64 where those of 128 leave CUs idle, and parts of a block's
// keys where even they do.
int blocks_of(const AttnArgs& a, int qn) { return (int)(((int64_t)a.Tq * a.G + 64 * qn - 1) / (64 * qn)); }

int fwd_qn(int dtype, const AttnArgs& a) {
    return dtype == kBF16 && (int64_t)blocks_of(a, 2) * a.B * a.Hkv >= 512 ? 2 : 1;
}

FwdGeom fwd_geom(int dtype, const AttnArgs& a) {
    FwdGeom G;
    G.nb = blocks_of(a, fwd_qn(dtype, a));
    const int64_t blocks = (int64_t)G.nb * a.B * a.Hkv, tb = dtype == kBF16 ? 64 : 32;
    // most keys of a block, in tiles; a part keeps at least 4 of them
    const int64_t span = a.W ? (int64_t)a.W + a.S + 64 / a.G + 1 : a.N;
    const int64_t tiles = ((span < a.N ? span : a.N) + tb - 1) / tb;
    int64_t parts = blocks >= 256 ? 1 : (512 + blocks - 1) / blocks;
    if (parts > tiles / 4) parts = tiles / 4;
    G.parts = parts < 1 ? 1 : (int)parts;
    return G;
}

template <typename ST, int DH, int QN>
int launch_fwd(const AttnArgs& a, const FwdGeom& G, float* buf, hipStream_t stream) {
    const size_t ring = (size_t)kStages * 2 * TileLoad<ST, DH>::BYTES, outs = 4 * (size_t)store_rows_bytes<ST, DH>(QN);
    const size_t lds = ring > outs ? ring : outs;
    const Parts part = make_parts(buf, G.parts, (int64_t)a.B * a.Hq * a.Tq, DH);
    auto kern = wattn_fwd_kernel<ST, DH, QN>;
    if (allow_lds((const void*)kern, lds)) return -1;
    return launch_parts((uint64_t)a.B * a.Hkv * G.nb * G.parts, 256, [&](uint32_t first, uint32_t blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), lds, stream, FwdCall{a, G, part, first});
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
}

}  // namespace

int launch_merge_parts(int dtype, int dh, const AttnArgs& a, int parts, const Parts& p, hipStream_t stream) {
    return heads_by_type(dtype, dh, [&](auto st, auto d) {
        return launch_parts(((uint64_t)a.B * a.Hq * a.Tq + 3) / 4, 256, [&](uint32_t first, uint32_t blocks) {
            hipLaunchKernelGGL((wattn_merge_kernel<decltype(st), decltype(d)::value>), dim3(blocks), dim3(256), 0,
                               stream, a, parts, p, first);
            return hipGetLastError() == hipSuccess ? 0 : -1;
        });
    });
}

size_t attn_fwd_scratch(int dtype, int dh, const AttnArgs& a) {
    return parts_bytes(fwd_geom(dtype, a).parts, (int64_t)a.B * a.Hq * a.Tq, dh);
}

int launch_window_attn(int dtype, int dh, const AttnArgs& a, float* buf, hipStream_t stream) {
    const FwdGeom G = fwd_geom(dtype, a);
    const int e = heads_by_type(dtype, dh, [&](auto st, auto d) {
        using ST = decltype(st);
        constexpr int DH = decltype(d)::value;
        if constexpr (sizeof(ST) == 2)
            if (fwd_qn(dtype, a) == 2) return launch_fwd<ST, DH, 2>(a, G, buf, stream);
        return launch_fwd<ST, DH, 1>(a, G, buf, stream);
    });
    if (e || G.parts == 1) return e;
    return launch_merge_parts(dtype, dh, a, G.parts, make_parts(buf, G.parts, (int64_t)a.B * a.Hq * a.Tq, dh), stream);
}

}  // namespace mosa
