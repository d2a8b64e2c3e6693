// Causal attention with a sliding window and first tokens that stay visible:
// the backward over rows.
//
//   p = 2^(s c - lse'),  dp = dout v,  ds = p (dp - D)
//   dv = sum p dout,  dk = scale sum ds q,  dq = scale sum ds k
//
// Two kinds of workgroups in one launch, neither with atomics: one owns 64 CB
// keys of a key head and walks the rows that see them (the group's heads are
// in the row list, so their sum is the loop's), one owns 64 QN rows and walks
// the keys that they see.  Both form s and dp again from tiles of 64 (fp32: 32) that come
// through an LDS ring: 7 products in place of the 5 that one pass with atomic
// sums would take, for results that do not depend on the order of workgroups.
// The other operand stays in registers, and p and ds are fed to the second
// products as they lie in them, against tiles read transposed.  bf16 storage rounds
// p and ds to bf16 there, the type of the matrix operands, to half a step each;
// the sums over them, lse and D are fp32.  (dq, dk and dv are 0.0026, 0.0024 and
// 0.0023 off, a result rounded once 0.0017; ds in two parts would make dq 0.0018
// for 5 to 6% of a training step.)  p comes from lse, which is rounded at its size:
// past scores of about 2^20 its error shows.
//
// Measured (bf16): 2 x 4096 tokens, 32 / 8 heads of 128, window 1024, 4 sinks: this
// kernel 617 us in a trace, 0.68 PFLOP/s over its 7 products, matrix instructions
// busy 37% and the LDS 46% of the time (beside it the forward 182, (lse, -D) 24,
// sums 6; a training step in a loop, at higher clocks, 679 in all); the LDS's time
// for the transposed reads bounds the key blocks.  8192 tokens, 4 heads of 64,
// window 512: 37 us, chains of 10 tiles.  fp32 (2 x 2048 tokens, 16 / 8 heads of 128):
// matrix instructions busy 73%.
//
// Sinks are seen by every later row.  So that their keys' workgroups do not
// walk the whole sequence while all others walk a window, the pairs beyond the
// window are a third kind of work: up to kSinkKeys first keys, the rows cut
// into chunks, fp32 sums of every chunk added in order by a last kernel.  The
// same kernel adds up the parts of all keys where there is no window and few key
// blocks, whose rows are then cut into parts (the first keys are seen by every
// row, the last by few).
#include "launch_parts.h"
#include "wattn_dma.h"

namespace mosa {

namespace {

constexpr int kSinkKeys = 256;   // most sinks whose far pairs go by chunks of rows
constexpr int kSinkChunks = 32;  // most chunks of a key head's rows
constexpr int kMaxParts = 16;    // most parts of a key block's rows

// Two: with 4 stages of the 64-wide heads' tiles a CU holds two workgroups in
// place of four (8192 tokens, 4 heads, window 512, training step: 81 -> 65 us).
constexpr int kStages = 2;

// Launch geometry: per (b, key head) nk blocks of keys, their rows cut into kp
// parts, and nq blocks of rows; nc chunks for each of ns blocks of 64 sinks (ns =
// 0: far pairs are the key blocks' own work).  Sums are kept of the first `keys`
// keys of a head (all of them where kp > 1, otherwise the sinks where ns > 0): of
// every part, and of every chunk those of the sinks.
struct BwdGeom {
    int nk, kp, nq, ns, nc, keys;
};

// Tiles of a key head's rows: q, dout and (lse, -D).  A tile is 64 / G queries of
// the group's G heads (its last 64 % G rows are none), or 64 rows where G is
// larger, so that the lanes' offsets are the same for every tile.
template <typename ST, int DH>
struct RowTiles {
    using TL = TileLoad<ST, DH>;
    static constexpr int TB = TL::TB, ES = (int)sizeof(ST), LL = TB / 32;  // loads of (lse, -D), a word per lane
    int b, hk, nr;  // nr: rows per tile
    bool near;
    uint32_t qoff[TL::LD], goff[TL::LD], loff[LL];
    __device__ __forceinline__ RowTiles(const AttnArgs& a, int b, int hk, const TL& tl, int lane) : b(b), hk(hk) {
        const int nq = TB / a.G;  // queries per tile
        nr = nq ? nq * a.G : TB;
        // a tile's rows of G heads within 2^31 bytes
        near = nq > 0 && fits(a, a.q) && fits(a, a.dout) && (int64_t)a.G * a.Tq < ((int64_t)1 << 27);
#pragma unroll
        for (int j = 0; j < TL::LD; ++j) {
            const int r = tl.row + TL::STEP * j, i = a.gd.div(r), g = r - i * a.G;
            qoff[j] = (uint32_t)((g * a.q.head + i * a.q.row + tl.col) * ES);
            goff[j] = (uint32_t)((g * a.dout.head + i * a.dout.row + tl.col) * ES);
        }
#pragma unroll
        for (int j = 0; j < LL; ++j) {
            const int r = 32 * j + (lane >> 1), i = a.gd.div(r), g = r - i * a.G;
            loff[j] = (uint32_t)(((int64_t)g * a.Tq + i) * 8 + 4 * (lane & 1));
        }
    }
    __device__ __forceinline__ bool fits(const AttnArgs& a, const Rows& t) const {
        return a.G * t.head + TB * t.row < ((int64_t)1 << 29);
    }
    // The tile from row r0 on (of rows below rhi; those past it are the last one), to LDS byte `at`:
    // q, dout, and for this wave alone (lse, -D) of every row.
    __device__ __forceinline__ void issue(const AttnArgs& a, const TL& tl, int r0, int rhi, uint32_t at, uint32_t ld_at, int lane) const {
        if (near && r0 + TB <= rhi) {
            const int i0 = a.gd.div(r0);
            const char* q = uniform_ptr(reinterpret_cast<const char*>(row_ptr<ST>(a.q, b, hk * a.G, i0)));
            const char* g = uniform_ptr(reinterpret_cast<const char*>(row_ptr<ST>(a.dout, b, hk * a.G, i0)));
            const char* l = uniform_ptr(reinterpret_cast<const char*>(a.ld + ((int64_t)b * a.Hq + hk * a.G) * a.Tq + i0));
#pragma unroll
            for (int j = 0; j < TL::LD; ++j) {
                lds_load16s(qoff[j], q, at + tl.lds + 4096 * j);
                lds_load16s(goff[j], g, at + TL::BYTES + tl.lds + 4096 * j);
            }
#pragma unroll
            for (int j = 0; j < LL; ++j) lds_load4s(loff[j], l, ld_at + 256 * j);
            return;
        }
#pragma unroll
        for (int j = 0; j < TL::LD; ++j) {
            const int r = min(r0 + tl.row + TL::STEP * j, rhi - 1), i = a.gd.div(r);
            lds_load16(qrow_ptr<ST>(a, a.q, b, hk, r, i) + tl.col, at + tl.lds + 4096 * j);
            lds_load16(qrow_ptr<ST>(a, a.dout, b, hk, r, i) + tl.col, at + TL::BYTES + tl.lds + 4096 * j);
        }
#pragma unroll
        for (int j = 0; j < LL; ++j) {
            const int r = min(r0 + 32 * j + (lane >> 1), rhi - 1), i = a.gd.div(r);
            lds_load4(reinterpret_cast<const float*>(a.ld + qrow_index(a, b, hk, r, i)) + (lane & 1), ld_at + 256 * j);
        }
    }
};

// The order in which a key block takes its tiles of rows, so that the walks of
// neighbouring blocks meet in L2: with a window each starts at the tile whose
// number in the sequence its length divides, and goes round; without one from
// the last tile down.  (2 x 4096 tokens, 32 / 8 heads of 128, window 1024: 0.54 GB
// come from HBM in place of 2.0.)
struct Walk {
    int cut, early, late, step, last;
    __device__ __forceinline__ Walk(int rlo, int nr, int tbeg, int n, bool down) {
        const int r0 = rlo + nr * tbeg, far_end = down ? nr * (n - 1) : 0;
        cut = down ? 0 : (rlo / nr + tbeg) % n;
        early = r0 + nr * (n - cut);
        late = r0 + far_end - nr * cut;
        step = down ? -nr : nr;
        last = n - 1;
    }
    // first row of tile t (past the end: the last one)
    __device__ __forceinline__ int row(int t) const { return (t < cut ? early : late) + step * min(t, last); }
};

// Keys k0 .. k0 + KEYS - 1 of (b, hk): part `chunk` of the rows that see them
// within the window, or, far, chunk `chunk` of those beyond the sinks' window.
// This call does 64 CB of the keys, from k0 + from on.  True (only without
// `again`): to be done again.
template <typename ST, int DH, int CB, int KEYS, bool far, bool again>
__device__ __forceinline__ bool dkv_body(unsigned char* smem, const AttnArgs a, const BwdGeom G, int b, int hk, int k0,
                                         int from, int chunk, float* sums) {
    using TL = TileLoad<ST, DH>;
    constexpr int TB = TL::TB, NS = DH / 32, ND = DH / 16, STG = kStages, LD = TL::LD;
    constexpr int TILE = TL::BYTES, LDB = 4 * TB * 8, STAGE = 2 * TILE + LDB;  // q, dout, a copy of (lse, -D) per wave
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
    const bool apart = G.ns > 0;  // apart: far pairs are done by chunks
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn;
    const int kend = min(far ? min(a.S, k0 + KEYS) : k0 + KEYS, kn);  // past the block's last key
    const int wk0 = k0 + from + 16 * CB * wave, wk1 = min(wk0 + 16 * CB, kend) - 1;  // this wave's keys (none: wk1 < wk0)

    // rows that may see the block's keys
    int i0 = 0, i1 = 0;
    if (k0 < kend && qn > 0) {
        i0 = max(0, (far ? k0 + a.W : k0) - off);
        i1 = far || a.W == 0 || (!apart && k0 < a.S) ? qn : min(qn, kend - 1 + a.W - off);
    }
    const int rlo = i0 * a.G, rhi = max(i1, i0) * a.G;
    const TL tl(wave, lane);
    const RowTiles<ST, DH> rows(a, b, hk, tl, lane);
    const int nr = rows.nr, all = (rhi - rlo + nr - 1) / nr, cuts = far ? G.nc : G.kp, share = (all + cuts - 1) / cuts;
    const int tbeg = min(chunk * share, all), ntile = min(all, tbeg + share) - tbeg;

    f32x4 dk[CB][ND], dv[CB][ND];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int db = 0; db < ND; ++db) dk[cb][db] = dv[cb][db] = zero4();

    if (ntile > 0) {
        const TileReads<ST, DH> rd(g, c16);
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(smem));
        const Walk walk(rlo, nr, tbeg, ntile, !far && a.W == 0);
        // tile t (past the end: the last one again, into a buffer that nobody reads)
        auto issue = [&](int t, int buf) __attribute__((always_inline)) {
            const uint32_t at = base + buf * STAGE;
            rows.issue(a, tl, walk.row(t), rhi, at, at + 2 * TILE + 8 * TB * (tl.lds / 1024), lane);
        };
        // (the first tiles are on their way while the keys are loaded)
#pragma unroll
        for (int s = 0; s < STG - 1; ++s) issue(s, s);
        int key[CB];
        Frag8<ST> kf[CB][NS], vf[CB][NS];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            key[cb] = min(wk0 + 16 * cb + c16, kend - 1);  // (past the block: its last key again, not written)
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                kf[cb][st] = frag8_load<ST>(row_ptr<ST>(a.k, b, hk, key[cb]) + 32 * st + 8 * g);
                vf[cb][st] = frag8_load<ST>(row_ptr<ST>(a.v, b, hk, key[cb]) + 32 * st + 8 * g);
            }
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int st = 0; st < NS; ++st) take(kf[cb][st]), take(vf[cb][st]);

        // Of the tile from row r0 on, the rows (less 4 g) that the lane's keys pair with:
        // positions from the key on and within its window, or, far, from there on.
        auto pairs = [&](int r0, Span (&run)[CB]) __attribute__((always_inline)) {
            const int n = min(r0 + nr, rhi) - r0, i = a.gd.div(r0), p = off + i;
            const int skip = r0 - i * a.G + 4 * g;  // rows of the first position before the tile
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const int j = key[cb];
                const bool all_later = far || a.W == 0 || (!apart && j < a.S);
                const int lo = min(max((far ? j + a.W : j) - p, -1), TB + 1);  // in positions of the tile's first
                const int hi = min(max(j + a.W - p, 0), TB + 1);
                run[cb] = Span(lo * a.G - skip, min(all_later ? n : hi * a.G - (skip - 4 * g), n) - 1 - 4 * g);
            }
        };
        // whether the block's keys pair with the rows of the tile from r0 on in part
        auto in_part = [&](int r0) __attribute__((always_inline)) {
            const int rt = min(r0 + nr, rhi), p0 = off + a.gd.div(r0), p1 = off + a.gd.div(rt - 1);
            return !(r0 + TB == rt && (far ? p0 - (kend - 1) >= a.W : p0 >= kend - 1 && (a.W == 0 || p1 - k0 < a.W)));
        };
        const float c2 = a.scale * kLog2e;
        auto tile_step = [&](int it, auto bufc) __attribute__((always_inline)) {
            constexpr int BUF = decltype(bufc)::value;
            wait_vmcnt<(STG - 2) * (2 * LD + RowTiles<ST, DH>::LL)>();
            __syncthreads();
            issue(it + STG - 1, (BUF + STG - 1) % STG);
            const unsigned char* Qt = smem + BUF * STAGE;
            const unsigned char* Gt = Qt + TILE;
            const unsigned char* Lt = Gt + TILE + 8 * TB * wave;
            const int r0 = walk.row(it), rt = min(r0 + nr, rhi);  // the tile's rows
            const int pt0 = off + a.gd.div(r0), pt1 = off + a.gd.div(rt - 1);  // and their positions
            if constexpr (again)
                if (in_part(r0)) {
                    keep_finite<ST, DH>(smem + BUF * STAGE, tid);
                    keep_finite<ST, DH>(smem + BUF * STAGE + TILE, tid);
                    __syncthreads();
                }
            // nothing for this wave: no keys, rows before the keys, or past their window
            if (wk1 < wk0) return;
            if (far ? wk0 >= a.S || pt1 - wk0 < a.W : pt1 < wk0 || (a.W && pt0 - wk1 >= a.W && (apart || wk0 >= a.S))) return;
            const bool whole = r0 + TB == rt &&
                               (far ? pt0 - wk1 >= a.W : pt0 >= wk1 && (a.W == 0 || pt1 - wk0 < a.W));
            Span run[CB];
            if (!whole) pairs(r0, run);
            // the whole tile without a branch, so that its reads, products and
            // exponentials overlap
            auto products = [&](auto mc) __attribute__((always_inline)) {
                constexpr bool masked = decltype(mc)::value;
#pragma unroll
                for (int u = 0; u < TB / 32; ++u) {  // 32 rows at a time
                    __builtin_amdgcn_sched_barrier(0);
                    f32x4 s[CB][2], dp[CB][2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int sb = 2 * u + x;
                        const float4 l0 = *reinterpret_cast<const float4*>(Lt + 8 * (16 * sb + 4 * g));
                        const float4 l1 = *reinterpret_cast<const float4*>(Lt + 8 * (16 * sb + 4 * g) + 16);
                        const float lse[4] = {l0.x, l0.z, l1.x, l1.z};
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) {
                            s[cb][x] = zero4();
                            dp[cb][x] = f32x4{l0.y, l0.w, l1.y, l1.w};  // the product adds to -D
                        }
#pragma unroll
                        for (int st = 0; st < NS; ++st) {
                            const Frag8<ST> qa = rd.rows(Qt, sb, st), ga = rd.rows(Gt, sb, st);
#pragma unroll
                            for (int cb = 0; cb < CB; ++cb) {
                                mma8(s[cb][x], qa, kf[cb][st]);
                                mma8(dp[cb][x], ga, vf[cb][st]);
                            }
                        }
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                s[cb][x][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[cb][x][i], c2, -lse[i]));
                                dp[cb][x][i] *= s[cb][x][i];
                            }
                        if constexpr (masked) {
#pragma unroll
                            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const bool in = run[cb].has(16 * sb + i);
                                    s[cb][x][i] = in ? s[cb][x][i] : 0.f;
                                    dp[cb][x][i] = in ? dp[cb][x][i] : 0.f;
                                }
                        }
                    }
                    // dv^T += dout^T p, dk^T += q^T ds: with bf16 storage p and ds are
                    // rounded to it, the type of the matrix operands
                    Frag8<ST> pf[CB], df[CB];
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        pf[cb] = pack_frag<ST>(s[cb][0], s[cb][1]);
                        df[cb] = pack_frag<ST>(dp[cb][0], dp[cb][1]);
                    }
#pragma unroll
                    for (int db = 0; db < ND; ++db) {
                        const Frag8<ST> gt = rd.cols(Gt, u, db), qt = rd.cols(Qt, u, db);
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) {
                            mma8(dv[cb][db], gt, pf[cb]);
                            mma8(dk[cb][db], qt, df[cb]);
                        }
                    }
                }
            };
            if (whole) products(std::false_type{});
            else products(std::true_type{});
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
        mfma_drain();
        wait_vmcnt<0>();
        __syncthreads();
        if constexpr (again) {
            const uint32_t at = __builtin_amdgcn_readfirstlane(base);
            TL ul = tl;  // (uniform, which the compiler does not see here)
            ul.lds = __builtin_amdgcn_readfirstlane(ul.lds);
#pragma unroll 1
            for (int t = 0; t < ntile; ++t) {
                const int r0 = walk.row(t);
                if (!in_part(r0)) continue;
                rows.issue(a, ul, r0, rhi, at, at + 2 * TILE + 8 * TB * (ul.lds / 1024), lane);
                Span run[CB];
                pairs(r0, run);
                wait_vmcnt<0>();
                __syncthreads();
                auto in = [&](int r, int cb) __attribute__((always_inline)) { return run[cb].has(r - 4 * g); };
                add_not_finite<ST, DH, true>(rd, smem, g, dk, in);
                add_not_finite<ST, DH, false>(rd, smem + TILE, g, dv, in);
                __syncthreads();
            }
        } else {
            bool spoilt = false;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                spoilt |= wk0 + 16 * cb + c16 <= wk1 && !(finite4(dk[cb]) && finite4(dv[cb]));
            if (any_of_workgroup(smem, wave, lane, spoilt)) return true;
        }
    }

    // keys past the sequence are zero (their lanes computed its last key again)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
        if (wk0 + 16 * cb + c16 > wk1)
#pragma unroll
            for (int db = 0; db < ND; ++db) dk[cb][db] = dv[cb][db] = zero4();
    // sums: of every part the first G.keys keys, then of every chunk the sinks
    const int top = far ? a.S : a.N, summed = far ? a.S : G.keys;  // keys of the output, those whose sums are kept
    const int64_t heads = (int64_t)a.B * a.Hkv, bh = (int64_t)b * a.Hkv + hk;
    float* sum = sums + ((far ? heads * G.kp * G.keys : 0) + (heads * chunk + bh) * summed) * 2 * DH;
    const float scale = a.scale;
    if (wk0 < summed) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int j = wk0 + 16 * cb + c16;
            if (j >= min(summed, top)) continue;
#pragma unroll
            for (int db = 0; db < ND; ++db) {
                float* to = sum + (int64_t)j * 2 * DH + 16 * db + 4 * g;
                const f32x4 x = dk[cb][db] * scale, y = dv[cb][db];
                *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(to + DH) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
    }
    if constexpr (far) return false;
    unsigned char* mine = smem + wave * store_rows_bytes<ST, DH>(CB);
    float fk[CB], fv[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        fk[cb] = scale;
        fv[cb] = 1.f;
    }
    const Rows to_k = a.dk, to_v = a.dv;
    store_rows<ST, DH, CB>(mine, dk, fk, lane, [&](int r) __attribute__((always_inline)) {
        const int j = wk0 + r;
        return j < a.N && j >= summed ? row_ptr<ST>(to_k, b, hk, j) : nullptr;
    });
    store_rows<ST, DH, CB>(mine, dv, fv, lane, [&](int r) __attribute__((always_inline)) {
        const int j = wk0 + r;
        return j < a.N && j >= summed ? row_ptr<ST>(to_v, b, hk, j) : nullptr;
    });
    return false;
}

// Rows r0 .. r0 + ROWS - 1 of (b, hk); this call does 64 QN of them, from r0 + from on.
// True (only without `again`): to be done again.
template <typename ST, int DH, int QN, int ROWS, bool again>
__device__ __forceinline__ bool dq_body(unsigned char* smem, const AttnArgs a, int b, int hk, int r0, int from) {
    using TL = TileLoad<ST, DH>;
    constexpr int TB = TL::TB, NS = DH / 32, ND = DH / 16, STG = kStages, LD = TL::LD;
    constexpr int TILE = TL::BYTES, STAGE = 2 * TILE;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn;
    const int R = a.Tq * a.G, rn = qn * a.G, wr0 = r0 + from + 16 * QN * wave;
    KeyList list{0, 0, 0};
    if (r0 < rn) list = keys_of(a, off + a.gd.div(r0), off + a.gd.div(min(r0 + ROWS, rn) - 1), kn);
    const int ntile = (list.count + TB - 1) / TB;

    f32x4 dq[QN][ND];
#pragma unroll
    for (int qs = 0; qs < QN; ++qs)
#pragma unroll
        for (int db = 0; db < ND; ++db) dq[qs][db] = zero4();

    if (ntile > 0) {
        const int pw0 = off + a.gd.div(min(wr0, rn - 1)), pw1 = off + a.gd.div(min(wr0 + 16 * QN, rn) - 1);
        const TL tl(wave, lane);
        const TileReads<ST, DH> rd(g, c16);
        const KeyTiles<ST, DH> kt(a.k, b, hk, tl), vt(a.v, b, hk, tl);
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(smem));
        auto issue = [&](int t, int buf) __attribute__((always_inline)) {
            const int e0 = TB * min(t, ntile - 1);
            kt.issue(tl, list, e0, base + buf * STAGE);
            vt.issue(tl, list, e0, base + buf * STAGE + TILE);
        };
        // (the first tiles are on their way while the rows are loaded)
#pragma unroll
        for (int s = 0; s < STG - 1; ++s) issue(s, s);
        int pos[QN];
        float2 ld[QN];
        Frag8<ST> qf[QN][NS], gf[QN][NS];
#pragma unroll
        for (int qs = 0; qs < QN; ++qs) {
            const int r = min(wr0 + 16 * qs + c16, rn - 1), i = a.gd.div(r);
            pos[qs] = off + i;
            ld[qs] = a.ld[qrow_index(a, b, hk, r, i)];
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                qf[qs][st] = frag8_load<ST>(qrow_ptr<ST>(a, a.q, b, hk, r, i) + 32 * st + 8 * g);
                gf[qs][st] = frag8_load<ST>(qrow_ptr<ST>(a, a.dout, b, hk, r, i) + 32 * st + 8 * g);
            }
        }
#pragma unroll
        for (int qs = 0; qs < QN; ++qs) {
            asm volatile("" : "+v"(ld[qs].x), "+v"(ld[qs].y));
#pragma unroll
            for (int st = 0; st < NS; ++st) take(qf[qs][st]), take(gf[qs][st]);
        }
        const float c2 = a.scale * kLog2e;
        // whether the block's rows see tile e0 in part
        const int pb0 = off + a.gd.div(r0), pb1 = off + a.gd.div(min(r0 + ROWS, rn) - 1);
        auto in_part = [&](int e0) __attribute__((always_inline)) {
            return e0 + TB > list.count || list.key(e0 + TB - 1) > pb0 ||
                   (a.W && (e0 >= list.s ? list.key(e0) : list.lo) <= pb1 - a.W);
        };
        auto tile_step = [&](int it, auto bufc) __attribute__((always_inline)) {
            constexpr int BUF = decltype(bufc)::value;
            wait_vmcnt<(STG - 2) * 2 * LD>();
            __syncthreads();
            issue(it + STG - 1, (BUF + STG - 1) % STG);
            const unsigned char* Kt = smem + BUF * STAGE;
            const unsigned char* Vt = Kt + TILE;
            const int e0 = TB * it;
            const int kmax = list.key(min(e0 + TB, list.count) - 1), kmin = e0 >= list.s ? list.key(e0) : list.lo;
            if constexpr (again)
                if (in_part(e0)) {
                    keep_finite<ST, DH>(smem + BUF * STAGE, tid);
                    __syncthreads();
                }
            if (e0 >= list.s && (kmin > pw1 || (a.W && kmax <= pw0 - a.W && kmin >= a.S))) return;
            const bool whole = e0 + TB <= list.count && kmax <= pw0 && (a.W == 0 || kmin > pw1 - a.W);
            // keys kmin + 0 .. TB - 1, no sinks: those of a row are a run (entries
            // past the list lie behind every row)
            const bool plain = e0 >= list.s && (a.W == 0 || kmin >= a.S);
            auto products = [&](auto mc) __attribute__((always_inline)) {
                constexpr bool masked = decltype(mc)::value;
#pragma unroll
                for (int u = 0; u < TB / 32; ++u) {  // 32 keys at a time
                    __builtin_amdgcn_sched_barrier(0);
                    f32x4 s[QN][2], dp[QN][2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int sb = 2 * u + x;
#pragma unroll
                        for (int qs = 0; qs < QN; ++qs) {
                            s[qs][x] = zero4();
                            dp[qs][x] = f32x4{ld[qs].y, ld[qs].y, ld[qs].y, ld[qs].y};  // the product adds to -D
                        }
#pragma unroll
                        for (int st = 0; st < NS; ++st) {
                            const Frag8<ST> ka = rd.rows(Kt, sb, st), va = rd.rows(Vt, sb, st);
#pragma unroll
                            for (int qs = 0; qs < QN; ++qs) {
                                mma8(s[qs][x], ka, qf[qs][st]);
                                mma8(dp[qs][x], va, gf[qs][st]);
                            }
                        }
#pragma unroll
                        for (int qs = 0; qs < QN; ++qs)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                dp[qs][x][i] *= __builtin_amdgcn_exp2f(__builtin_fmaf(s[qs][x][i], c2, -ld[qs].x));
                        if (masked && plain) {
#pragma unroll
                            for (int qs = 0; qs < QN; ++qs) {
                                const int d = pos[qs] - kmin - 4 * g;
                                const Span run(a.W ? d - a.W + 1 : -4 * TB, d);
#pragma unroll
                                for (int i = 0; i < 4; ++i) dp[qs][x][i] = run.has(16 * sb + i) ? dp[qs][x][i] : 0.f;
                            }
                        } else if (masked) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int e = e0 + 16 * sb + 4 * g + i, key = list.key(e);
#pragma unroll
                                for (int qs = 0; qs < QN; ++qs)
                                    dp[qs][x][i] = ((e < list.count) & sees(a, pos[qs], key)) ? dp[qs][x][i] : 0.f;
                            }
                        }
                    }
                    Frag8<ST> df[QN];
#pragma unroll
                    for (int qs = 0; qs < QN; ++qs) df[qs] = pack_frag<ST>(dp[qs][0], dp[qs][1]);
#pragma unroll
                    for (int db = 0; db < ND; ++db) {
                        const Frag8<ST> kf = rd.cols(Kt, u, db);
#pragma unroll
                        for (int qs = 0; qs < QN; ++qs) mma8(dq[qs][db], kf, df[qs]);
                    }
                }
            };
            if (whole) products(std::false_type{});
            else products(std::true_type{});
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
        mfma_drain();
        wait_vmcnt<0>();
        __syncthreads();
        if constexpr (again) {
            const uint32_t at = __builtin_amdgcn_readfirstlane(base);
            TL ul = tl;  // (uniform, which the compiler does not see here)
            ul.lds = __builtin_amdgcn_readfirstlane(ul.lds);
#pragma unroll 1
            for (int e0 = 0; e0 < list.count; e0 += TB) {
                if (!in_part(e0)) continue;
                kt.issue(ul, list, e0, at);
                wait_vmcnt<0>();
                __syncthreads();
                add_not_finite<ST, DH, true>(rd, smem, g, dq, [&](int r, int qs) __attribute__((always_inline)) {
                    return (e0 + r < list.count) & sees(a, pos[qs], list.key(e0 + r));
                });
                __syncthreads();
            }
        } else {
            bool spoilt = false;
#pragma unroll
            for (int qs = 0; qs < QN; ++qs) spoilt |= wr0 + 16 * qs + c16 < rn && !finite4(dq[qs]);
            if (any_of_workgroup(smem, wave, lane, spoilt)) return true;
        }
    }
#pragma unroll
    for (int qs = 0; qs < QN; ++qs)
        if (wr0 + 16 * qs + c16 >= rn)
#pragma unroll
            for (int db = 0; db < ND; ++db) dq[qs][db] = zero4();
    const float scale = a.scale;
    float fq[QN];
#pragma unroll
    for (int qs = 0; qs < QN; ++qs) fq[qs] = scale;
    store_rows<ST, DH, QN>(smem + wave * store_rows_bytes<ST, DH>(QN), dq, fq, lane, [&](int lr) -> ST* {
        const int r = wr0 + lr;
        return r < R ? qrow_ptr<ST>(a, a.dq, b, hk, r, a.gd.div(r)) : nullptr;
    });
    return false;
}

// Waves per SIMD that the first walk's registers allow.
template <typename ST, int DH, int CB>
constexpr int bwd_waves() {
    return DH == 128 || (DH == 64 && (CB == 2 || sizeof(ST) == 4)) ? 2 : DH == 32 && CB == 1 && sizeof(ST) == 2 ? 5 : 3;
}

// A workgroup's work: key blocks, then chunks of far rows, then row blocks; each kind in
// neighbouring order on an XCD (a key head's workgroups share its rows and keys).
struct BwdWork {
    int kind, bh, at, part;  // keys (0) or rows (2) from `at` on, part or chunk (1) of their rows
    __device__ __forceinline__ BwdWork(const AttnArgs& a, const BwdGeom& G, uint32_t first, uint32_t block, uint32_t blocks,
                                       int keys, int rows) {
        const uint32_t heads = (uint32_t)a.B * a.Hkv, n0 = heads * G.nk * G.kp, n1 = heads * G.ns * G.nc, n2 = heads * G.nq;
        uint32_t id = first + block;
        const bool one = first == 0 && blocks == n0 + n1 + n2;
        if (id < n0) {
            if (one) id = xcd_logical_id(id, n0);
            const int per = G.nk * G.kp, k = id % per;
            kind = 0, bh = id / per, at = k / G.kp * keys, part = k % G.kp;
        } else if (id < n0 + n1) {
            id -= n0;
            const int per = G.ns * G.nc, k = id % per;
            kind = 1, bh = id / per, at = k / G.nc * 64, part = k % G.nc;
        } else {
            id -= n0 + n1;
            if (one) id = xcd_logical_id(id, n2);
            const int q = id % G.nq;
            kind = 2, bh = id / G.nq, at = (a.W ? q : G.nq - 1 - q) * rows, part = 0;
        }
    }
};

struct BwdCall {
    AttnArgs a;
    BwdGeom G;
    float* sums;
    uint32_t first;
};

// The second time, as functions of their own: what they take of registers, and how their code
// is laid out, is no matter of the first walk.  c: the kernel's arguments, lds: its LDS.
template <typename ST, int DH, int KEYS, bool far>
__device__ __attribute__((noinline)) void dkv_again(const void* c, uint32_t lds, int bh, int k0, int chunk) {
    const BwdCall call = uniform_args<BwdCall>(c);
    unsigned char* smem = lds_at(__builtin_amdgcn_readfirstlane(lds));
    bh = __builtin_amdgcn_readfirstlane(bh), k0 = __builtin_amdgcn_readfirstlane(k0);
    chunk = __builtin_amdgcn_readfirstlane(chunk);
#pragma unroll 1
    for (int from = 0; from < KEYS; from += 64) {
        __syncthreads();
        dkv_body<ST, DH, 1, KEYS, far, true>(smem, call.a, call.G, bh / call.a.Hkv, bh % call.a.Hkv, k0, from, chunk, call.sums);
    }
}
template <typename ST, int DH, int ROWS>
__device__ __attribute__((noinline)) void dq_again(const void* c, uint32_t lds, int bh, int r0) {
    const BwdCall call = uniform_args<BwdCall>(c);
    unsigned char* smem = lds_at(__builtin_amdgcn_readfirstlane(lds));
    bh = __builtin_amdgcn_readfirstlane(bh), r0 = __builtin_amdgcn_readfirstlane(r0);
#pragma unroll 1
    for (int from = 0; from < ROWS; from += 64) {
        __syncthreads();
        dq_body<ST, DH, 1, ROWS, true>(smem, call.a, bh / call.a.Hkv, bh % call.a.Hkv, r0, from);
    }
}
// (one call at the kernel's end: what lives across a call would take registers)
template <typename ST, int DH, int CB, int QN>
__device__ __attribute__((noinline)) void bwd_again(const void* c, uint32_t lds, uint32_t block, uint32_t blocks) {
    const BwdCall call = uniform_args<BwdCall>(c);
    const BwdWork w(call.a, call.G, call.first, __builtin_amdgcn_readfirstlane(block), __builtin_amdgcn_readfirstlane(blocks),
                    64 * CB, 64 * QN);
    if (w.kind == 0) dkv_again<ST, DH, 64 * CB, false>(c, lds, w.bh, w.at, w.part);
    else if (w.kind == 1) dkv_again<ST, DH, 64, true>(c, lds, w.bh, w.at, w.part);
    else dq_again<ST, DH, 64 * QN>(c, lds, w.bh, w.at);
}

template <typename ST, int DH, int CB, int QN>
__global__ __launch_bounds__(256, (bwd_waves<ST, DH, CB>())) void wattn_bwd_kernel(BwdCall c) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const BwdWork w(c.a, c.G, c.first, blockIdx.x, gridDim.x, 64 * CB, 64 * QN);
    const int b = w.bh / c.a.Hkv, hk = w.bh % c.a.Hkv;
    bool redo;
    if (w.kind == 0) redo = dkv_body<ST, DH, CB, 64 * CB, false, false>(smem, c.a, c.G, b, hk, w.at, 0, w.part, c.sums);
    else if (w.kind == 1) redo = dkv_body<ST, DH, 1, 64, true, false>(smem, c.a, c.G, b, hk, w.at, 0, w.part, c.sums);
    else redo = dq_body<ST, DH, QN, 64 * QN, false>(smem, c.a, b, hk, w.at, 0);
    if (redo)
        bwd_again<ST, DH, CB, QN>((const void*)__builtin_amdgcn_kernarg_segment_ptr(), lds_addr(smem), blockIdx.x, gridDim.x);
}

// (lse in log2 units, -D), D = sum(out dout), of every query row, 8 columns per lane:
// what the backward's kernels read of a row beside q and dout.  Bound by the
// rows of out and dout, which it reads once.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_ld_kernel(AttnArgs a, uint32_t first) {
    constexpr int L = DH / 8;
    const int64_t row = ((int64_t)first + blockIdx.x) * (256 / L) + threadIdx.x / L;
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int li = threadIdx.x % L;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    float d = 0.f;
    const bool live = i < seq_len_of(a.ql, b, a.Tq);
    if (live) {
        float x[8], y[8];
        frag8_to_f32<ST>(frag8_load<ST>(row_ptr<ST>(a.out, b, h, i) + 8 * li), x);
        frag8_to_f32<ST>(frag8_load<ST>(row_ptr<ST>(a.dout, b, h, i) + 8 * li), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) d += x[e] * y[e];
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) d += __shfl_xor(d, o, 64);
    if (li == 0) {
        const float l = live ? a.lse[row] : -__builtin_inff();
        a.ld[row] = make_float2(l == -__builtin_inff() ? __builtin_inff() : l * kLog2e, -d);
    }
}

// dk and dv of the keys whose sums are kept: the slots in order, 4 values per thread.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_sums_kernel(AttnArgs a, BwdGeom G, const float* __restrict__ sums) {
    const int64_t heads = (int64_t)a.B * a.Hkv, all = heads * G.keys * 2 * DH, chunk = heads * a.S * 2 * DH;
    for (int64_t e = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); e < all; e += 1024 * (int64_t)gridDim.x) {
        const int c = (int)(e % DH), which = (int)(e / DH % 2);
        const int64_t row = e / (2 * DH), bh = row / G.keys;
        const int j = (int)(row % G.keys), hk = (int)(bh % a.Hkv), b = (int)(bh / a.Hkv);
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float* p) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        };
#pragma unroll 4
        for (int k = 0; k < G.kp; ++k) add(sums + k * all + e);
        if (j < a.S) {
            const float* far = sums + G.kp * all + (bh * a.S + j) * 2 * DH + which * DH + c;
#pragma unroll 4
            for (int k = 0; k < G.nc; ++k) add(far + k * chunk);
        }
        if (j >= seq_len_of(a.kl, b, a.N)) s = make_float4(0.f, 0.f, 0.f, 0.f);
        ST* to = row_ptr<ST>(which ? a.dv : a.dk, b, hk, j) + c;
        if constexpr (sizeof(ST) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
        else *reinterpret_cast<float4*>(to) = s;
    }
}

// Keys and rows per block.  Blocks of 128 halve the reads of the tiles per
// product; blocks of 64 where those leave CUs idle.  128-wide heads keep to 64
// keys (16 per wave): the sums of 32 keys and their operands are 192 registers
// of a lane, which leaves too few for the rest at 2 waves per SIMD.  There the
// transposed reads of the tiles take most of the LDS's time; workgroups of 8
// waves, four for dv and four for dk of 32 keys each, halve them for one more
// product, and measured slower (2 x 4096 tokens, 32 / 8 heads, window 1024,
// training step: 787 against 687 us; 8 waves of 16 keys each: 722).
bool wide_blocks(int dtype, const AttnArgs& a) {
    return dtype == kBF16 && (int64_t)a.B * a.Hkv * ((a.N + 127) / 128) >= 512;
}
constexpr int wide_keys(int dh) { return dh == 128 ? 1 : 2; }

BwdGeom bwd_geom(int dtype, int dh, const AttnArgs& a) {
    BwdGeom G;
    const bool wide = wide_blocks(dtype, a);
    const int kw = wide ? 64 * wide_keys(dh) : 64, qw = wide ? 128 : 64;
    const int64_t R = (int64_t)a.Tq * a.G;
    G.nk = (a.N + kw - 1) / kw;
    G.nq = (int)((R + qw - 1) / qw);
    G.ns = a.W && a.S && a.S <= kSinkKeys ? (a.S + 63) / 64 : 0;
    // A key block walks more rows than a row block walks keys (G heads of a window
    // of queries; without a window the first keys are seen by every row).  Where
    // the key blocks are fewer than the chip's places their walks alone would set
    // the time, so they are cut, into parts of at least 4 tiles: without a window
    // up to the 512 places (2 x 2048 tokens, 16 / 4 heads of 128, training step: 325
    // us with whole blocks, 232 with parts); with one up to half of them, as the
    // row blocks fill the rest (2048 tokens, 16 / 4 heads of 128, window 1024: 184
    // us whole, 165 with 512, 132 with 256; at 256 whole blocks parts lose, 199
    // against 204).  Row blocks are not cut: without a window and with one or two
    // heads the last of them, 8192 keys in one chain, sets the time (131 us of a step
    // of 169 with one head of 64, 8192 tokens).
    const int64_t nk = (int64_t)a.B * a.Hkv * G.nk, walk = (int64_t)(a.W + kw) * a.G;
    const int64_t tiles = (a.W && walk < R ? walk : R) / (dtype == kBF16 ? 64 : 32), places = a.W ? 256 : 512;
    int64_t kp = nk < places ? (places + nk - 1) / nk : 1;
    if (kp > tiles / 4) kp = tiles / 4;
    if (kp > kMaxParts) kp = kMaxParts;
    G.kp = kp < 1 ? 1 : (int)kp;
    G.keys = G.kp > 1 ? a.N : G.ns ? a.S : 0;
    // a chunk walks about as many rows as a key block does
    const int64_t c = (R + (int64_t)(a.W + kw) * a.G - 1) / ((int64_t)(a.W + kw) * a.G);
    G.nc = G.ns ? (int)(c < kSinkChunks ? c : kSinkChunks) : 0;
    return G;
}

template <typename ST, int DH, int CB, int QN>
int launch_bwd(const AttnArgs& a, const BwdGeom& G, float* sums, hipStream_t stream) {
    using TL = TileLoad<ST, DH>;
    auto kern = wattn_bwd_kernel<ST, DH, CB, QN>;
    const size_t ring = (size_t)kStages * (2 * TL::BYTES + 4 * TL::TB * 8);
    const size_t outs = 4 * (size_t)store_rows_bytes<ST, DH>(CB > QN ? CB : QN);
    const size_t lds = ring > outs ? ring : outs;
    if (allow_lds((const void*)kern, lds)) return -1;
    const uint64_t blocks = (uint64_t)a.B * a.Hkv * ((uint64_t)G.nk * G.kp + G.ns * G.nc + G.nq);
    const int e = launch_parts(blocks, 256, [&](uint32_t first, uint32_t n) {
        hipLaunchKernelGGL(kern, dim3(n), dim3(256), lds, stream, BwdCall{a, G, sums, first});
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
    if (e || !G.keys) return e;
    const int64_t n = ((int64_t)a.B * a.Hkv * G.keys * 2 * DH + 1023) / 1024;
    hipLaunchKernelGGL((wattn_sums_kernel<ST, DH>), dim3((unsigned)(n < 65536 ? n : 65536)), dim3(256), 0, stream, a, G, sums);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

size_t ld_bytes(const AttnArgs& a) { return ((size_t)a.B * a.Hq * a.Tq * sizeof(float2) + 255) / 256 * 256; }

}  // namespace

size_t attn_bwd_scratch(int dtype, int dh, const AttnArgs& a) {
    const BwdGeom G = bwd_geom(dtype, dh, a);
    return ld_bytes(a) + ((size_t)G.kp * G.keys + (size_t)G.nc * a.S) * a.B * a.Hkv * 2 * dh * sizeof(float);
}

int launch_window_attn_bwd(int dtype, int dh, AttnArgs a, void* scratch, hipStream_t stream) {
    a.ld = static_cast<float2*>(scratch);
    float* sums = reinterpret_cast<float*>(static_cast<char*>(scratch) + ld_bytes(a));
    const BwdGeom G = bwd_geom(dtype, dh, a);
    return heads_by_type(dtype, dh, [&](auto st, auto d) {
        using ST = decltype(st);
        constexpr int DH = decltype(d)::value, per = 256 / (DH / 8);
        const int e = launch_parts(((uint64_t)a.B * a.Hq * a.Tq + per - 1) / per, 256, [&](uint32_t first, uint32_t n) {
            hipLaunchKernelGGL((wattn_ld_kernel<ST, DH>), dim3(n), dim3(256), 0, stream, a, first);
            return hipGetLastError() == hipSuccess ? 0 : -1;
        });
        if (e) return e;
        if constexpr (sizeof(ST) == 2)
            if (wide_blocks(dtype, a)) return launch_bwd<ST, DH, wide_keys(DH), 2>(a, G, sums, stream);
        return launch_bwd<ST, DH, 1, 1>(a, G, sums, stream);
    });
}

}  // namespace mosa
