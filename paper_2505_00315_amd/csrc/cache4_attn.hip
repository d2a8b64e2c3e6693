// Attention over the 4-bit cache: a few query rows of a key head against its
// whole cache, so the cache's bytes bound it (dh + dh / 4 per position and head).
//
// What is read is multiplied as it is held.  A code n goes into a matrix
// operand as the bf16 number 16 + n, which is a shift and a mask for two of
// them, and the scales and minima come in around the products:
//   q k = sum_g s_g (q (16 + n))_g + sum_g (m_g - 16 s_g) sum(q)_g
// with one matrix instruction per group of 32 columns, and one for the whole
// second sum: the words (s, m) of a position, as they are held, times
// (-16 sum(q), sum(q)), split into three bf16 parts so that nothing is lost.
//   out_g = sum_j (p_j s_jg) (16 + n_j) - 24 sum_j (p_j s_jg) + sum_j p_j (m_jg + 8 s_jg)
// where the weights times the scales of a group are the matrix operand, rounded
// to bf16 once, and the second sum is taken over the same rounded numbers (a
// product with ones): the rounding meets n - 8, the distance from the middle of
// the group, and not n, which would double its share.  fp32 storage takes q and
// p s in three bf16 parts and the codes as n - 8, so that nothing large cancels.
//
// Every wave walks its own tiles of 32 positions with its own running maximum
// and sum, loads straight into registers one tile ahead and the page numbers
// two ahead; the waves of a workgroup are joined in LDS, parts of the keys by
// merge_parts.  Scores have the key in the lane, which so has the scales of its
// key at hand for both products; the weights change lanes through LDS.
//
// Beside the bytes it is vector instructions that count: two for every pair of
// codes, and, per tile and lane, those for RI score rows of two keys.  A lane of
// the 16 x 16 result has rows 4 g .. 4 g + 3, so up to 4 query rows are put in rows
// 0, 4, 8, 12 (RI = 1), up to 8 in rows 4 g and 4 g + 1, and no lane works on rows
// that are none.
//
// Measured (bf16, one token for each of 64 sequences of 8k to 16k positions, 32 / 8
// heads of 128): 185 us for 1.02 GB, 5.5 TB/s, and 5 us for the parts' sum; one
// short sequence (8 / 2 heads of 64, 1000 positions, window 512): 8.5 us, a launch
// and a chain of a table read, a tile's loads and four tiles.  Every 16 rows expand
// the codes again: many queries are better served from the rows (8 sequences of 8192,
// 32 / 8 heads of 128: 64 queries 232 us, 512 queries 1702; read and attention over
// the rows 222 and 584).
#include "cache4.h"
#include "launch_parts.h"

namespace mosa {

namespace {

constexpr int kWaves = 4;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// The keys that some row sees, in aligned octets: so octets of sinks, then
// those from w0 on.
struct OctetList {
    int so, w0, count;
    __device__ __forceinline__ int first_key(int e) const { return 8 * (e < so ? e : e - so + w0); }
};
__device__ __forceinline__ OctetList octets_of(const KeyList& l) {
    OctetList o;
    o.so = (l.s + 7) / 8;
    o.w0 = max(l.lo / 8, o.so);
    const int hi = l.lo + l.count - l.s;  // past the last key
    o.count = l.count <= 0 ? 0 : o.so + max((hi + 7) / 8 - o.w0, 0);
    return o;
}

template <int DH, int SPLIT>
struct AttnLds {
    static constexpr int NG = DH / 32;
    static constexpr int PROW = 32 * 2 + 16;             // weights of a row: 32 positions, padded
    static constexpr int PW = SPLIT * NG * 16 * PROW;    // of a wave and 16 rows
};

// Nibbles nib and nib + 4 of w as a pair of bf16: 16 + n (the constants are
// registers, so that the mask and the 16 are one instruction), or n - 8.
template <int SPLIT>
struct CodeBits {
    static constexpr float middle = SPLIT == 1 ? 24.f : 0.f, least = middle - 8.f;  // what 8 and 0 become
    uint32_t mask, sixteen;
    __device__ __forceinline__ CodeBits() : mask(0x00780078u), sixteen(0x41804180u) {
        asm volatile("" : "+v"(mask), "+v"(sixteen));
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t w, int nib) const {
        if constexpr (SPLIT > 1)
            return pack_bf16x2((float)(w >> (4 * nib) & 15) - 8.f, (float)(w >> (4 * nib + 16) & 15) - 8.f);
        const int sh = 4 * nib - 3;
        return ((sh < 0 ? w << 3 : w >> sh) & mask) | sixteen;
    }
};

template <int N>
__device__ __forceinline__ void load_words(const unsigned char* p, uint32_t (&w)[N]) {
    if constexpr (N == 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else if constexpr (N == 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x, w[1] = u.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// A lane's words of a tile.
template <int DH>
struct Tile {
    static constexpr int NG = DH / 32, NV = DH == 128 ? 4 : 2;
    uint32_t kc[2][NG], km[2][NG], vm[2][NG], vc[2][NV];
    int key;    // the lane's keys are key and key + 1 (negative: on no page)
};

__device__ __forceinline__ bf16x8 frag_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, u32x4_t{a, b, c, d});
}

// Row sums and maxima over the 16 lanes of a result's row.
__device__ __forceinline__ float lanes16_max(float x) {
    x = fmaxf(x, dpp_f32<0xB1, 0xf>(x));
    x = fmaxf(x, dpp_f32<0x4E, 0xf>(x));
    x = fmaxf(x, dpp_f32<0x141, 0xf>(x));
    return fmaxf(x, dpp_f32<0x140, 0xf>(x));
}
__device__ __forceinline__ float lanes16_sum(float x) {
    x += dpp_f32<0xB1, 0xf>(x);
    x += dpp_f32<0x4E, 0xf>(x);
    x += dpp_f32<0x141, 0xf>(x);
    return x + dpp_f32<0x140, 0xf>(x);
}

struct CacheGeom {
    int nb, parts;  // blocks of rows per (b, key head), parts of their keys
    UDiv page;      // by the page size
};

// SPLIT: bf16 parts of q and of the weights (1 for bf16 storage, 3 for fp32).
// A block has 4 RI NQ rows: row (4 q + g) RI + i is row 4 g + i of result q.
template <typename ST, int DH, int NQ, int RI>
__global__ __launch_bounds__(64 * kWaves, 2) void cache4_attn_kernel(AttnArgs a, CacheArgs c, CacheGeom G, Parts part,
                                                                    uint32_t first) {
    constexpr int SPLIT = sizeof(ST) == 2 ? 1 : 3, NG = DH / 32, ND = DH / 16, RB = 4 * RI * NQ;
    using L = AttnLds<DH, SPLIT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c16 = lane & 15;
    uint32_t id = first + blockIdx.x;
    const int pt = (int)(id % G.parts);
    id /= G.parts;
    const int blk = (int)(id % G.nb), bh = (int)(id / G.nb), b = bh / a.Hkv, hk = bh % a.Hkv;
    const int R = a.Tq * a.G, r0 = blk * RB;
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn, rn = qn * a.G;

    KeyList keys{0, 0, 0};
    int p0 = 0, p1 = 0;  // positions of the block's first and last row
    if (r0 < rn) {
        p0 = off + a.gd.div(r0);
        p1 = off + a.gd.div(min(r0 + RB, rn) - 1);
        keys = keys_of(a, p0, p1, kn);
    }
    const OctetList list = octets_of(keys);
    const int all = (list.count + 3) / 4, share = (all + G.parts - 1) / G.parts;
    const int tbeg = min(pt * share, all), tend = min(all, tbeg + share);  // this part's tiles; a wave takes every fourth

    float m_run[NQ][RI], l_run[NQ][RI], pm[NQ][NG][RI];
    f32x4 o[NQ][ND], ones[NQ][NG];
    int pos[NQ][RI];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            m_run[q][i] = -__builtin_inff();
            l_run[q][i] = 0.f;
            pos[q][i] = off + a.gd.div(min(r0 + (4 * q + g) * RI + i, max(rn, 1) - 1));
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) pm[q][gr][i] = 0.f;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) o[q][d] = zero4();
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) ones[q][gr] = zero4();
    }

    if (tbeg + wave < tend) {
        const size_t block = cache_block_bytes(c.ps, DH);
        const int32_t* table = c.table + (size_t)b * c.per;
        // Where the octets of tile t are that this lane reads, that of its two
        // keys and that of V: page, place in the page, and the keys.
        struct Spots { int k, v, tk, tv, key; };
        auto octet = [&](int t, int x) __attribute__((always_inline)) { return list.first_key(min(4 * t + x, list.count - 1)); };
        auto spots = [&](int t) __attribute__((always_inline)) {
            t = min(t, tend - 1);
            const int ek = octet(t, c16 >> 2), ev = octet(t, g), pk = G.page.div(ek), pv = G.page.div(ev);
            return Spots{table[pk], table[pv], ek - pk * c.ps + 2 * (c16 & 3), ev - pv * c.ps,
                         4 * t + (c16 >> 2) < list.count ? ek + 2 * (c16 & 3) : -2};
        };
        auto load = [&](const Spots& sp, Tile<DH>& x) __attribute__((always_inline)) {
            const bool kin = sp.k >= 0 && sp.k < c.pages, vin = sp.v >= 0 && sp.v < c.pages;
            x.key = kin ? sp.key : -2;
            // (a page that does not exist: page 0 is read and masked)
            const unsigned char* kb = c.cache + ((size_t)(kin ? sp.k : 0) * c.H + hk) * block;
            const unsigned char* vb = c.cache + ((size_t)(vin ? sp.v : 0) * c.H + hk) * block;
            const unsigned char* kc = kb + sp.tk * (DH / 2) + g * (DH / 8);
            const unsigned char* km = kb + c.ps * DH + sp.tk * (DH / 8);
            const unsigned char* vm = km + c.ps * (DH / 8);
            const unsigned char* vc = vb + c.ps * (DH / 2) + sp.tv * (DH / 2) + (DH == 32 ? c16 / 2 * 8 : c16 * (DH / 8));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                load_words<NG>(kc + y * (DH / 2), x.kc[y]);
                load_words<NG>(km + y * (DH / 8), x.km[y]);
                load_words<NG>(vm + y * (DH / 8), x.vm[y]);
                load_words<Tile<DH>::NV>(vc + y * (2 * DH), x.vc[y]);
            }
        };
        // the first tile is on its way while q is prepared
        Tile<DH> even, odd;
        Spots sp = spots(tbeg + wave);
        load(sp, even);
        sp = spots(tbeg + wave + kWaves);

        // q / 8 (16 + n and the minima make terms of up to 8 times a score, which is to
        // stay finite where the score is) as A operand: columns 32 gr + 8 g .. + 7 of the
        // row, in SPLIT parts;
        // its sums over a group, times (-16, 1) (of codes n - 8: (8, 1)), as the operand of the words (s, m):
        // lane group 0 holds the upper bf16 part, 1 and 2 what that leaves
        bf16x8 qf[NQ][SPLIT][NG], qs[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int r = min(r0 + (4 * q + (c16 >> 2)) * RI + min(c16 & 3, RI - 1), rn - 1);
            const ST* qp = qrow_ptr<ST>(a, a.q, b, hk, r, a.gd.div(r));
            uint32_t sums[4] = {0, 0, 0, 0};
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float x[8], s = 0.f;
                frag8_to_f32<ST>(frag8_load<ST>(qp + 32 * gr + 8 * g), x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= 0.125f;
                    s += x[e];
                }
                s = rows4_sum(s);
#pragma unroll
                for (int sp2 = 0; sp2 < SPLIT; ++sp2) {
                    qf[q][sp2][gr] = frag8_from<uint16_t>(x).v;
                    float y[8];
                    Frag8<uint16_t> f;
                    f.v = qf[q][sp2][gr];
                    frag8_to_f32<uint16_t>(f, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] -= y[e];
                }
                const float hi = bf16_to_f32(f32_to_bf16(s)), mid = bf16_to_f32(f32_to_bf16(s - hi)), lo = s - hi - mid;
                const float mine = g == 0 ? hi : g == 1 ? mid : g == 2 ? lo : 0.f;
                sums[gr] = pack_bf16x2(-CodeBits<SPLIT>::least * mine, mine);
            }
            qs[q] = frag_of(sums[0], sums[1], sums[2], sums[3]);
        }
        const float c2 = a.scale * (8.f * kLog2e), step = 8.f / c2;
        unsigned char* pw = smem + wave * NQ * L::PW;  // this wave's weights
        const bf16x8 one8 = frag_of(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
        const CodeBits<SPLIT> codes;

        auto tile_step = [&](int t, Tile<DH>& cur, Tile<DH>& nxt) __attribute__((always_inline)) {
            load(sp, nxt);
            sp = spots(t + 2 * kWaves);

            // scores of rows 4 g + i and keys cur.key + y
            float s[NQ][2][RI];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                bf16x8 meta;
                if constexpr (NG == 4) meta = frag_of(cur.km[y][0], cur.km[y][1], cur.km[y][2], cur.km[y][3]);
                else if constexpr (NG == 2) meta = frag_of(cur.km[y][0], cur.km[y][1], 0, 0);
                else meta = frag_of(cur.km[y][0], 0, 0, 0);
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qs[q], meta, zero4(), 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < RI; ++i) s[q][y][i] = x[i];
                }
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    const uint32_t w = cur.kc[y][gr];
                    const bf16x8 kf = frag_of(codes(w, 0), codes(w, 1), codes(w, 2), codes(w, 3));
                    const float sc = __uint_as_float(cur.km[y][gr] << 16);
#pragma unroll
                    for (int q = 0; q < NQ; ++q) {
                        f32x4 x = zero4();
#pragma unroll
                        for (int p = SPLIT - 1; p >= 0; --p)
                            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[q][p][gr], kf, x, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < RI; ++i) s[q][y][i] = __builtin_fmaf(x[i], sc, s[q][y][i]);
                    }
                }
            }
            // masks only where some row does not see some key of the tile
            const int lastkey = octet(t, 3) + 7, firstkey = octet(t, 0);
            const bool whole = 4 * t >= list.so && 4 * t + 4 <= list.count && lastkey <= p0 &&
                               (a.W == 0 || firstkey > p1 - a.W) && __builtin_amdgcn_ballot_w64(cur.key < 0) == 0;
            if (!whole) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int key = cur.key + y;
                    const bool in = key >= 0 && key < kn;
                    bool any = false;
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int i = 0; i < RI; ++i) {
                            const bool ok = in & sees(a, pos[q][i], key);
                            s[q][y][i] = ok ? s[q][y][i] : -__builtin_inff();
                            any |= ok;
                        }
                    // what no row sees may be anything: its scale and minimum are taken as 0;
                    // what is not finite leaves the products, and joins the sums of the rows
                    // that see it here
                    const uint64_t bal = __builtin_amdgcn_ballot_w64(any);
                    const bool seen = (bal >> c16 | bal >> (c16 + 16) | bal >> (c16 + 32) | bal >> (c16 + 48)) & 1;
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        const bool bad = ((cur.vm[y][gr] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
                        cur.vm[y][gr] = (seen & !bad) ? cur.vm[y][gr] : 0u;
#pragma unroll
                        for (int q = 0; q < NQ; ++q)
#pragma unroll
                            for (int i = 0; i < RI; ++i)
                                pm[q][gr][i] += (bad & (s[q][y][i] != -__builtin_inff())) ? __builtin_nanf("") : 0.f;
                    }
                }
            }
            // Weights are 2^((s - m) c - 16): differences of scores, which are not rounded
            // at the scores' size; below 2^-8, so that their products with the largest
            // scales are finite.  m, a score, moves only when exceeded by 8 in log2 units.
            bool up = false;
#pragma unroll
            for (int q = 0; q < NQ; ++q)
#pragma unroll
                for (int i = 0; i < RI; ++i) up |= fmaxf(s[q][0][i], s[q][1][i]) > m_run[q][i] + step;
            if (__builtin_amdgcn_ballot_w64(up)) {
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int i = 0; i < RI; ++i) {
                        const float top = lanes16_max(fmaxf(s[q][0][i], s[q][1][i]));
                        const float mn = fmaxf(m_run[q][i], top);
                        const float al = mn == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m_run[q][i] - mn) * c2);
                        m_run[q][i] = mn;
                        l_run[q][i] *= al;
#pragma unroll
                        for (int d = 0; d < ND; ++d) o[q][d][i] *= al;
#pragma unroll
                        for (int gr = 0; gr < NG; ++gr) {
                            pm[q][gr][i] *= al;
                            ones[q][gr][i] *= al;
                        }
                    }
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q)
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    const float mu = m_run[q][i] == -__builtin_inff() ? 0.f : m_run[q][i];
                    const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][0][i] - mu, c2, -16.f));
                    const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][1][i] - mu, c2, -16.f));
                    l_run[q][i] += w0 + w1;
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        const float s0 = __uint_as_float(cur.vm[0][gr] << 16), s1 = __uint_as_float(cur.vm[1][gr] << 16);
                        const float mid0 = __builtin_fmaf(8.f, s0, __uint_as_float(cur.vm[0][gr] & 0xffff0000u));
                        const float mid1 = __builtin_fmaf(8.f, s1, __uint_as_float(cur.vm[1][gr] & 0xffff0000u));
                        pm[q][gr][i] = __builtin_fmaf(w1, mid1, __builtin_fmaf(w0, mid0, pm[q][gr][i]));
                        float x0 = w0 * s0, x1 = w1 * s1;
#pragma unroll
                        for (int p = 0; p < SPLIT; ++p) {
                            const uint32_t u = pack_bf16x2(x0, x1);
                            *reinterpret_cast<uint32_t*>(pw + ((((q * SPLIT + p) * NG + gr) * 16) + 4 * g + i) * L::PROW + 4 * c16) = u;
                            if constexpr (SPLIT > 1) {
                                x0 -= __uint_as_float(u << 16);
                                x1 -= __uint_as_float(u & 0xffff0000u);
                            }
                        }
                    }
                }
            wave_sync();
            // out += (p s) (16 + n), or (p s) (n - 8): column c16 of result (gr, e) is 32 gr + 2 c16 + e
            // (rows 4 g + RI .. hold what an earlier call left; nothing reads their results)
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                bf16x8 wf[NQ][SPLIT];
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p) {
                        wf[q][p] = __builtin_bit_cast(
                            bf16x8, *reinterpret_cast<const u32x4_t*>(pw + ((((q * SPLIT + p) * NG + gr) * 16) + c16) * L::PROW + 16 * g));
                        if constexpr (CodeBits<SPLIT>::middle != 0.f)
                            ones[q][gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[q][p], one8, ones[q][gr], 0, 0, 0);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    constexpr int H = DH == 128 ? 2 : 0;  // words of a second unit
                    const int u = H * (gr / 2), nib = DH == 128 ? 2 * (gr % 2) + e : 2 * gr + e;
                    uint32_t w[4] = {cur.vc[0][u], cur.vc[0][u + 1], cur.vc[1][u], cur.vc[1][u + 1]};
                    if constexpr (DH == 32)
#pragma unroll
                        for (int x = 0; x < 4; ++x) w[x] >>= 8 * (c16 & 1);
                    const bf16x8 vf = frag_of(codes(w[0], nib), codes(w[1], nib), codes(w[2], nib), codes(w[3], nib));
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int p = SPLIT - 1; p >= 0; --p)
                            o[q][2 * gr + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[q][p], vf, o[q][2 * gr + e], 0, 0, 0);
                }
            }
            wave_sync();  // the weights' place is written again by the next tile
        };
        // (by twos, so that the tile in hand and the next one keep their
        // registers; the forms with the most sums have none left for that)
        for (int t = tbeg + wave;;) {
            tile_step(t, even, odd);
            if ((t += kWaves) >= tend) break;
            if constexpr (RI < 4) {
                tile_step(t, odd, even);
                if ((t += kWaves) >= tend) break;
            } else {
                even = odd;
            }
        }
        mfma_drain();
    }

    // This wave's rows to LDS: [RB][DH] sums, then m and l of every row.
    __syncthreads();
    float* wo = reinterpret_cast<float*>(smem) + wave * RB * (DH + 2);
    float* wml = wo + RB * DH;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const int lr = (4 * q + g) * RI + i;
            l_run[q][i] = lanes16_sum(l_run[q][i]);
            m_run[q][i] = __builtin_fmaf(m_run[q][i], a.scale * (8.f * kLog2e), 16.f);  // in log2 units, with the weights' 2^-16
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                const float add = lanes16_sum(pm[q][gr][i]) - CodeBits<SPLIT>::middle * ones[q][gr][i];
                const float x = o[q][2 * gr][i] + add, y = o[q][2 * gr + 1][i] + add;
                *reinterpret_cast<float2*>(wo + lr * DH + 32 * gr + 2 * c16) = make_float2(x, y);
            }
            if (c16 == 0) *reinterpret_cast<float2*>(wml + 2 * lr) = make_float2(m_run[q][i], l_run[q][i]);
        }
    __syncthreads();
    // The waves in order: M = max m_w, L = sum l_w 2^(m_w - M); 8 columns per thread.
    const float* base = reinterpret_cast<const float*>(smem);
    const int64_t rows = (int64_t)a.B * a.Hq * a.Tq;
    for (int e = tid; e < RB * (DH / 8); e += 64 * kWaves) {
        const int lr = e / (DH / 8), d0 = e % (DH / 8) * 8, r = r0 + lr;
        if (r >= R) continue;
        const int i = a.gd.div(r);
        const int64_t row = qrow_index(a, b, hk, r, i);
        float M = -__builtin_inff(), S = 0.f, x[8] = {};
        if (r < rn) {
            float ml[kWaves][2];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float* p = base + w * RB * (DH + 2) + RB * DH + 2 * lr;
                ml[w][0] = p[0], ml[w][1] = p[1];
                M = fmaxf(M, ml[w][0]);
            }
            const float mu = M == -__builtin_inff() ? 0.f : M;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[w][0] - mu);
                S += ml[w][1] * f;
                const float* p = base + w * RB * (DH + 2) + lr * DH + d0;
#pragma unroll
                for (int n = 0; n < 8; ++n) x[n] += f == 0.f ? 0.f : p[n] * f;
            }
        }
        if (G.parts > 1) {
            float* to = part.o + (pt * rows + row) * DH + d0;
            reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
            if (d0 == 0) *reinterpret_cast<float2*>(part.ml + (pt * rows + row) * 2) = make_float2(M, S);
        } else {
            const float f = S > 0.f ? 1.f / S : S == 0.f ? 0.f : S;
#pragma unroll
            for (int n = 0; n < 8; ++n) x[n] *= f;
            ST* to = qrow_ptr<ST>(a, a.out, b, hk, r, i) + d0;
            if constexpr (SPLIT == 1) {
                *reinterpret_cast<uint4*>(to) = __builtin_bit_cast(uint4, frag8_from<uint16_t>(x).v);
            } else {
                reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
                reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
            }
            if (a.lse && d0 == 0) a.lse[row] = S == 0.f ? -__builtin_inff() : M * kLn2 + logf(S);
        }
    }
}

// Rows per block: 4, 8 or 16 by the rows there are; 32 share what is expanded of
// a tile, where there are more than 16 and the registers hold them (bf16 heads of
// 32 columns).
int rows_per_block(int dtype, int dh, const AttnArgs& a) {
    const int64_t R = (int64_t)a.Tq * a.G;
    return R <= 4 ? 4 : R <= 8 ? 8 : R <= 16 || dtype != kBF16 || dh > 32 ? 16 : 32;
}

CacheGeom cache_geom(int dtype, int dh, const AttnArgs& a) {
    CacheGeom G{};
    const int rb = rows_per_block(dtype, dh, a);
    const int64_t R = (int64_t)a.Tq * a.G;
    G.nb = (int)((R + rb - 1) / rb);
    // Parts as the chip's 512 places have room for (4 sequences of 16000, 8 key
    // heads: 512 workgroups 27 us, 768 33, 1024 and 2048 34), and two where the
    // blocks alone fill them, so that sequences of different lengths even out (64
    // of 8k to 16k positions, 8 key heads: 512 workgroups 203 us, 1024 196, 2048
    // 203); a part keeps at least 512 positions, 4 tiles per wave (8 sequences of
    // 4000: parts of 128 positions 36 us, of 256 26, of 512 22, of 1024 22).
    const int64_t blocks = (int64_t)G.nb * a.B * a.Hkv;
    const int64_t span = a.W ? (int64_t)a.W + a.S + rb / a.G + 16 : a.N;
    const int64_t tiles = ((span < a.N ? span : a.N) + 31) / 32;
    int64_t parts = blocks >= 1024 ? 1 : blocks > 256 ? 2 : 512 / blocks;
    if (parts > tiles / 16) parts = tiles / 16;
    G.parts = parts < 1 ? 1 : (int)parts;
    return G;
}

template <typename ST, int DH, int NQ, int RI>
int launch_attn(const AttnArgs& a, const CacheArgs& c, const CacheGeom& G, float* buf, hipStream_t stream) {
    constexpr int SPLIT = sizeof(ST) == 2 ? 1 : 3;
    const size_t w = (size_t)kWaves * NQ * AttnLds<DH, SPLIT>::PW, o = (size_t)kWaves * 4 * RI * NQ * (DH + 2) * 4;
    const size_t lds = w > o ? w : o;
    auto kern = cache4_attn_kernel<ST, DH, NQ, RI>;
    if (allow_lds((const void*)kern, lds)) return -1;
    const Parts part = make_parts(buf, G.parts, (int64_t)a.B * a.Hq * a.Tq, DH);
    return launch_parts((uint64_t)G.nb * a.B * a.Hkv * G.parts, 64 * kWaves, [&](uint32_t first, uint32_t blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * kWaves), lds, stream, a, c, G, part, first);
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
}

}  // namespace

size_t cache4_attn_scratch(int dtype, int dh, const AttnArgs& a) {
    return parts_bytes(cache_geom(dtype, dh, a).parts, (int64_t)a.B * a.Hq * a.Tq, dh);
}

int launch_cache4_attn(int dtype, const AttnArgs& a, const CacheArgs& c, float* buf, hipStream_t stream) {
    CacheGeom G = cache_geom(dtype, c.dh, a);
    G.page = make_udiv((uint32_t)c.ps);
    const int e = heads_by_type(dtype, c.dh, [&](auto st, auto d) {
        using ST = decltype(st);
        constexpr int DH = decltype(d)::value;
        const int rb = rows_per_block(dtype, DH, a);
        if constexpr (sizeof(ST) == 2 && DH == 32)
            if (rb == 32) return launch_attn<ST, DH, 2, 4>(a, c, G, buf, stream);
        if (rb == 4) return launch_attn<ST, DH, 1, 1>(a, c, G, buf, stream);
        if (rb == 8) return launch_attn<ST, DH, 1, 2>(a, c, G, buf, stream);
        return launch_attn<ST, DH, 1, 4>(a, c, G, buf, stream);
    });
    if (e || G.parts == 1) return e;
    return launch_merge_parts(dtype, c.dh, a, G.parts, make_parts(buf, G.parts, (int64_t)a.B * a.Hq * a.Tq, c.dh), stream);
}

}  // namespace mosa
