// The 4-bit cache: rows written and read back (attention over it: cache4_attn.hip).
//
// Both copies move each byte once.  Measured (bf16, 4 x 4096 positions, 8 heads of
// 128, 88 MB each): read 17 us, 5.3 TB/s, what memory gives; write 25 us, 3.5 TB/s,
// bound by the vector instructions of the codes, more than 20 per value.
#include "cache4.h"
#include "launch_parts.h"

namespace mosa {

namespace {

// Both copies work on aligned groups of 4 positions ("quads", the unit in which
// V is laid out) of one sequence and head: DH / 8 lanes per position, 8 columns
// each, K and V together.
template <int DH>
struct Quad {
    static constexpr int LPP = DH / 8;      // lanes per position
    static constexpr int LPQ = 4 * LPP;     // lanes per quad
    static constexpr int QPB = 256 / LPQ;   // quads per workgroup
};

template <typename ST>
__device__ __forceinline__ void load8(const ST* p, float (&x)[8]) {
    frag8_to_f32<ST>(frag8_load<ST>(p), x);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = __builtin_bit_cast(uint4, frag8_from<uint16_t>(x).v);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Meta word and codes (a nibble each) of a lane's 8 columns of a group of 32 (its
// 4 lanes).
//
// The code is the integer nearest to d / s, ties to even, for d = x - m in
// fp32.  c, d (1 / s) rounded to an integer, may be off by one next to a
// midpoint, and the remainder d - c s decides exactly: the product has 13 bits
// and the fused sum is rounded once, which keeps its order against s / 2.  An odd
// c is left at the midpoint too, an even one only past it.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t& word) {
    // (maximum and minimum hand on NaN)
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = __builtin_elementwise_minimum(lo, x[i]);
        hi = __builtin_elementwise_maximum(hi, x[i]);
    }
    lo = __builtin_elementwise_minimum(lo, dpp_f32<0xB1, 0xf>(lo));
    hi = __builtin_elementwise_maximum(hi, dpp_f32<0xB1, 0xf>(hi));
    lo = __builtin_elementwise_minimum(lo, dpp_f32<0x4E, 0xf>(lo));
    hi = __builtin_elementwise_maximum(hi, dpp_f32<0x4E, 0xf>(hi));
    const uint32_t mb = f32_to_bf16(lo);
    const float m = __uint_as_float(mb << 16);
    uint32_t sb = f32_to_bf16((hi - m) * (1.f / 15.f));
    float s = __uint_as_float(sb << 16);
    // an infinity among the values makes m or s infinite or NaN, a NaN both
    const bool ok = fabsf(m) < __builtin_inff() && fabsf(s) < __builtin_inff();
    if (!(s >= 1.17549435e-38f)) s = 0.f, sb = 0;
    const float inv = s > 0.f && ok ? 1.f / s : 0.f, half = 0.5f * s;
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // (a sum with 1.5 2^23 is rounded to an integer, its lowest bit in the last place)
        const float d = x[i] - m, t = __builtin_fmaf(d, inv, 12582912.f), n = t - 12582912.f, r = __builtin_fmaf(-n, s, d);
        const uint32_t odd = __float_as_uint(t) & 1;
        const float limit = __uint_as_float(__float_as_uint(half) - odd);  // the number next below half
        c[i] = __builtin_amdgcn_fmed3f(n + (fabsf(r) > limit ? __builtin_copysignf(1.f, r) : 0.f), 0.f, 15.f);
    }
    const float a = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[3], 16.f, c[2]), 16.f, c[1]), 16.f, c[0]);
    const float b = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[7], 16.f, c[6]), 16.f, c[5]), 16.f, c[4]);
    word = inv > 0.f ? (uint32_t)a | (uint32_t)b << 16 : 0u;
    return ok ? sb | (mb << 16) : 0x7fc00000u;
}

// The K word of 8 codes: column 2 i in nibble i, column 2 i + 1 in nibble i + 4.
__device__ __forceinline__ uint32_t k_order(uint32_t w) {
    uint32_t e = w & 0x0f0f0f0fu, o = w >> 4 & 0x0f0f0f0fu;  // the even columns' nibbles, the odd ones'
    e = (e | e >> 4) & 0x00ff00ffu, o = (o | o >> 4) & 0x00ff00ffu;
    return (e & 0xffu) | (e >> 8 & 0xff00u) | (o & 0xffu) << 16 | (o >> 16) << 24;
}

// V's column order: a lane's 8 columns 8 li .. + 7 are the pairs c = 4 (li % 4) +
// 0 .. 3 of group g = li / 4, a byte each; the lanes of the other groups hold the
// same pairs of theirs.  They trade bytes so that lane g ends with the bytes of
// all groups of some of the pairs: the pieces `unit` (low half) and unit + 1 of
// the row.  untrade undoes it.
template <int DH>
__device__ __forceinline__ int v_unit(int li) {
    if constexpr (DH == 128) return 2 * (4 * (li & 3) + (li >> 2));
    else if constexpr (DH == 64) return 4 * (li & 3) + 2 * (li >> 2);
    else return 2 * li;
}
template <int DH>
__device__ __forceinline__ uint32_t v_trade(uint32_t w, int li) {
    const int lane = threadIdx.x & 63, g = li >> 2;
    if constexpr (DH == 128) {  // byte k of the result: byte g of group k's lane
        uint32_t r = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) r |= (__shfl(w, lane + 4 * (k - g), 64) >> (8 * g) & 0xffu) << (8 * k);
        return r;
    } else if constexpr (DH == 64) {
        const uint32_t o = __shfl_xor(w, 4, 64), a = g ? o : w, b = g ? w : o;  // groups 0 and 1
        const uint32_t x = a >> (16 * g), y = b >> (16 * g);
        return (x & 0xffu) | (y & 0xffu) << 8 | (x & 0xff00u) << 8 | (y & 0xff00u) << 16;
    } else {
        return w;
    }
}
template <int DH>
__device__ __forceinline__ uint32_t v_untrade(uint32_t w, int li) {
    if constexpr (DH == 128) return v_trade<DH>(w, li);
    else if constexpr (DH == 64) {
        const int g = li >> 2;
        const uint32_t o = __shfl_xor(w, 4, 64), a = (g ? o : w) >> (8 * g), b = (g ? w : o) >> (8 * g);
        return (a & 0xffu) | (a >> 8 & 0xff00u) | (b & 0xffu) << 16 | (b >> 16 & 0xffu) << 24;
    } else {
        return w;
    }
}

// Workgroups of a (sequence, head): each takes `span` quads of it, QPB at a time.
struct QuadGeom {
    UDiv per, heads, page;  // by the workgroups of a head, the heads, the page size
    int span;
};

// What a workgroup's quads have in common.
template <int DH>
struct QuadRun {
    int b, h, q0, len;
    int64_t start;
    __device__ __forceinline__ QuadRun(const CacheArgs& c, const QuadGeom& G, uint32_t id) {
        const int bh = G.per.div((int)id);
        q0 = ((int)id - bh * (int)G.per.n) * G.span;
        b = G.heads.div(bh);
        h = bh - b * (int)G.heads.n;
        start = c.start ? c.start[b] : 0;
        len = seq_len_of(c.lens, b, c.rows);
    }
};

// Where a quad's lane works: the row t that it takes or fills, and its place in the cache.
struct QuadSpot {
    int64_t t, pos;
    int tl;
    bool live, mine, held;  // a row of the call; within its length; on a page
    CacheBlock blk;
};
template <int DH>
__device__ __forceinline__ QuadSpot quad_row(const CacheArgs& c, const QuadRun<DH>& r, int quad, int lane) {
    QuadSpot s;
    // positions (start & ~3) + 4 quad + 0 .. 3
    s.pos = (r.start & ~(int64_t)3) + 4 * (int64_t)quad + lane / Quad<DH>::LPP;
    s.t = s.pos - r.start;
    s.live = s.t >= 0 && s.t < c.rows;
    s.mine = s.t >= 0 && s.t < r.len && s.pos >= 0 && s.pos <= 0x7fffffff;
    return s;
}
template <int DH>
__device__ __forceinline__ void quad_place(const CacheArgs& c, const QuadGeom& G, const QuadRun<DH>& r, QuadSpot& s) {
    s.held = s.mine && cache_find(c, G.page, r.b, r.h, (int)s.pos, s.blk, s.tl);
}

template <typename ST, int DH>
__global__ __launch_bounds__(256) void cache4_append_kernel(CacheArgs c, QuadGeom G, uint32_t first) {
    using Q = Quad<DH>;
    const int lane = threadIdx.x % Q::LPQ, li = lane % Q::LPP;
    const QuadRun<DH> run(c, G, first + blockIdx.x);
    for (int quad = threadIdx.x / Q::LPQ; quad < G.span; quad += Q::QPB) {
        QuadSpot s = quad_row<DH>(c, run, run.q0 + quad, lane);
        float x[8] = {}, y[8] = {};
        if (s.mine) {
            load8<ST>(row_ptr<ST>(c.k, run.b, run.h, s.t) + 8 * li, x);
            load8<ST>(row_ptr<ST>(c.v, run.b, run.h, s.t) + 8 * li, y);
        }
        quad_place<DH>(c, G, run, s);
        uint32_t kw, vw;
        const uint32_t km = quantise8(x, kw), vm = quantise8(y, vw);
        // V: a word takes the pieces of two neighbouring positions, the even
        // one's lane the first of its two pieces, the odd one's the second
        vw = v_trade<DH>(vw, li);
        const uint32_t v0 = vw & 0xffffu, v1 = vw >> 16;
        const int unit = v_unit<DH>(li);
        const int other = (threadIdx.x & 63) ^ Q::LPP;  // the neighbour's lane with the same columns
        const uint32_t theirs = __shfl(vw, other, 64);
        const int both = __shfl((int)s.held, other, 64);
        if (!s.held) continue;
        const int g = li >> 2, kg = li & 3;
        *reinterpret_cast<uint32_t*>(c.cache + s.blk.kword(s.tl, kg * (DH / 32) + g)) = k_order(kw);
        if (both) {
            const bool odd = s.tl & 1;
            const uint32_t word = odd ? (theirs >> 16 | v1 << 16) : (v0 | theirs << 16);
            *reinterpret_cast<uint32_t*>(c.cache + s.blk.vpiece(s.tl & ~1, unit + odd)) = word;
        } else {
            *reinterpret_cast<uint16_t*>(c.cache + s.blk.vpiece(s.tl, unit)) = (uint16_t)v0;
            *reinterpret_cast<uint16_t*>(c.cache + s.blk.vpiece(s.tl, unit + 1)) = (uint16_t)v1;
        }
        if (kg == 0) {
            *reinterpret_cast<uint32_t*>(c.cache + s.blk.kmeta(s.tl, g)) = km;
            *reinterpret_cast<uint32_t*>(c.cache + s.blk.vmeta(s.tl, g)) = vm;
        }
    }
}

template <typename ST, int DH>
__global__ __launch_bounds__(256) void cache4_read_kernel(CacheArgs c, QuadGeom G, uint32_t first) {
    using Q = Quad<DH>;
    const int lane = threadIdx.x % Q::LPQ, li = lane % Q::LPP, g = li >> 2, kg = li & 3;
    const QuadRun<DH> run(c, G, first + blockIdx.x);
    for (int quad = threadIdx.x / Q::LPQ; quad < G.span; quad += Q::QPB) {
        QuadSpot s = quad_row<DH>(c, run, run.q0 + quad, lane);
        quad_place<DH>(c, G, run, s);
        float x[8] = {}, y[8] = {};
        uint32_t w = 0, v = 0, km = 0, vm = 0;
        if (s.held) {
            const int unit = v_unit<DH>(li);
            w = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.kword(s.tl, kg * (DH / 32) + g));
            v = *reinterpret_cast<const uint16_t*>(c.cache + s.blk.vpiece(s.tl, unit));
            v |= (uint32_t)*reinterpret_cast<const uint16_t*>(c.cache + s.blk.vpiece(s.tl, unit + 1)) << 16;
            km = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.kmeta(s.tl, g));
            vm = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.vmeta(s.tl, g));
        }
        v = v_untrade<DH>(v, li);
        if (!s.live) continue;
        if (s.held) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = cache_value(km, (w >> (4 * ((i >> 1) + 4 * (i & 1)))) & 15);
                y[i] = cache_value(vm, (v >> (4 * i)) & 15);
            }
        }
        store8(row_ptr<ST>(c.k, run.b, run.h, s.t) + 8 * li, x);
        store8(row_ptr<ST>(c.v, run.b, run.h, s.t) + 8 * li, y);
    }
}

template <class K>
int launch_quads(K kern, const CacheArgs& c, int per_pass, hipStream_t stream) {
    const int quads = c.rows / 4 + 2;  // of a sequence and head: a start inside a quad adds one
    // up to 16 passes per workgroup, where that leaves 16 workgroups to a CU
    const int64_t passes = (int64_t)c.B * c.H * ((quads + per_pass - 1) / per_pass);
    const int64_t each = passes / 4096 < 1 ? 1 : passes / 4096 > 16 ? 16 : passes / 4096;
    QuadGeom G;
    G.span = (int)each * per_pass;
    const int per = (quads + G.span - 1) / G.span;
    G.per = make_udiv((uint32_t)per), G.heads = make_udiv((uint32_t)c.H), G.page = make_udiv((uint32_t)c.ps);
    return launch_parts((uint64_t)c.B * c.H * per, 256, [&](uint32_t first, uint32_t blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, stream, c, G, first);
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
}

}  // namespace

int launch_cache4_append(int dtype, const CacheArgs& c, hipStream_t stream) {
    return heads_by_type(dtype, c.dh, [&](auto st, auto d) {
        constexpr int DH = decltype(d)::value;
        return launch_quads(cache4_append_kernel<decltype(st), DH>, c, Quad<DH>::QPB, stream);
    });
}

int launch_cache4_read(int dtype, const CacheArgs& c, hipStream_t stream) {
    return heads_by_type(dtype, c.dh, [&](auto st, auto d) {
        constexpr int DH = decltype(d)::value;
        return launch_quads(cache4_read_kernel<decltype(st), DH>, c, Quad<DH>::QPB, stream);
    });
}

}  // namespace mosa
