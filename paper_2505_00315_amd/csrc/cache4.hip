// The 4-bit cache: rows written and read back (attention over it: cache4_attn.hip).
#include "cache4.h"

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

// Meta word and codes of a lane's 8 columns of a group of 32 (its 4 lanes).
//
// The code is the integer nearest to d / s, ties to even, for d = x - m in
// fp32.  With n the integer part of d (1 / s), which may be off by one near an
// integer, the sign of d - (n + 1/2) s decides between n and n + 1 exactly: the
// product has 13 bits and the fused sum is rounded once, which keeps its sign.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t (&code)[8]) {
    float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        bad += x[i] * 0.f;  // NaN for infinities and NaN
    }
    lo = fminf(lo, dpp_f32<0xB1, 0xf>(lo));
    hi = fmaxf(hi, dpp_f32<0xB1, 0xf>(hi));
    bad += dpp_f32<0xB1, 0xf>(bad);
    lo = fminf(lo, dpp_f32<0x4E, 0xf>(lo));
    hi = fmaxf(hi, dpp_f32<0x4E, 0xf>(hi));
    bad += dpp_f32<0x4E, 0xf>(bad);
    const uint32_t mb = f32_to_bf16(lo);
    const float m = __uint_as_float(mb << 16);
    const float range = hi - m;
    uint32_t sb = f32_to_bf16(range * (1.f / 15.f));
    float s = __uint_as_float(sb << 16);
    if (!(s >= 1.17549435e-38f)) s = 0.f, sb = 0;
    const bool ok = bad == 0.f && s < __builtin_inff() && fabsf(m) < __builtin_inff();
    const float inv = s > 0.f && ok ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = x[i] - m;
        const float n = fminf(fmaxf(floorf(d * inv), 0.f), 15.f);
        const float over = __builtin_fmaf(-(n + 0.5f), s, d);
        const bool up = over > 0.f || (over == 0.f && ((int)n & 1));
        const int c = min((int)n + (up ? 1 : 0), 15);
        code[i] = inv > 0.f ? c : 0;
    }
    return ok ? sb | (mb << 16) : 0x7fc00000u;
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

// Where a quad's lane works: its position, the row it comes from or goes to,
// and its block of the cache.
struct QuadSpot {
    int b, h, t, pos, tl;
    bool live, held;  // a row of the call; a position of the cache
    CacheBlock blk;
};
template <int DH>
__device__ __forceinline__ bool quad_spot(const CacheArgs& c, int64_t quad, int quads, int lane, QuadSpot& s) {
    if (quad >= (int64_t)c.B * c.H * quads) return false;
    const int qi = (int)(quad % quads);
    s.h = (int)(quad / quads % c.H);
    s.b = (int)(quad / quads / c.H);
    const int64_t start = c.start ? c.start[s.b] : 0;
    // positions (start & ~3) + 4 qi + 0 .. 3
    const int64_t pos = (start & ~(int64_t)3) + 4 * (int64_t)qi + lane / Quad<DH>::LPP, t = pos - start;
    s.t = (int)t;
    s.live = t >= 0 && t < c.rows;
    s.pos = (int)pos;
    s.held = s.live && t < seq_len_of(c.lens, s.b, c.rows) && pos <= 0x7fffffff && cache_find(c, s.b, s.h, s.pos, s.blk, s.tl);
    return true;
}

template <typename ST, int DH>
__global__ __launch_bounds__(256) void cache4_append_kernel(CacheArgs c, int quads) {
    using Q = Quad<DH>;
    const int lane = threadIdx.x % Q::LPQ, li = lane % Q::LPP;
    for (int64_t quad = (int64_t)blockIdx.x * Q::QPB + threadIdx.x / Q::LPQ;; quad += (int64_t)gridDim.x * Q::QPB) {
        QuadSpot s;
        if (!quad_spot<DH>(c, quad, quads, lane, s)) break;
        float x[8] = {}, y[8] = {};
        if (s.held) {
            load8<ST>(row_ptr<ST>(c.k, s.b, s.h, s.t) + 8 * li, x);
            load8<ST>(row_ptr<ST>(c.v, s.b, s.h, s.t) + 8 * li, y);
        }
        uint32_t kc[8], vc[8];
        const uint32_t km = quantise8(x, kc), vm = quantise8(y, vc);
        // V: a word takes the pieces of two neighbouring positions, the even
        // one's lane the first of its two pieces, the odd one's the second
        uint32_t vw = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) vw |= vc[i] << (4 * i);
        vw = v_trade<DH>(vw, li);
        const uint32_t v0 = vw & 0xffffu, v1 = vw >> 16;
        const int unit = v_unit<DH>(li);
        const int other = (threadIdx.x & 63) ^ Q::LPP;  // the neighbour's lane with the same columns
        const uint32_t theirs = __shfl(vw, other, 64);
        const int both = __shfl((int)s.held, other, 64);
        if (!s.held) continue;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= kc[2 * i] << (4 * i) | kc[2 * i + 1] << (4 * i + 16);
        const int g = li >> 2, kg = li & 3;
        *reinterpret_cast<uint32_t*>(c.cache + s.blk.kword(s.tl, kg * (DH / 32) + g)) = w;
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
__global__ __launch_bounds__(256) void cache4_read_kernel(CacheArgs c, int quads) {
    using Q = Quad<DH>;
    const int lane = threadIdx.x % Q::LPQ, li = lane % Q::LPP, g = li >> 2, kg = li & 3;
    for (int64_t quad = (int64_t)blockIdx.x * Q::QPB + threadIdx.x / Q::LPQ;; quad += (int64_t)gridDim.x * Q::QPB) {
        QuadSpot s;
        if (!quad_spot<DH>(c, quad, quads, lane, s)) break;
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
        store8(row_ptr<ST>(c.k, s.b, s.h, s.t) + 8 * li, x);
        store8(row_ptr<ST>(c.v, s.b, s.h, s.t) + 8 * li, y);
    }
}

template <class K>
int launch_quads(K kern, const CacheArgs& c, int per_block, hipStream_t stream) {
    const int quads = c.rows / 4 + 2;  // of a sequence and head: a start inside a quad adds one
    const int64_t all = (int64_t)c.B * c.H * quads, blocks = (all + per_block - 1) / per_block;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, stream, c, quads);
    return hipGetLastError() == hipSuccess ? 0 : -1;
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
