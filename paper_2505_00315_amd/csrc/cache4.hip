// The 4-bit cache: rows written, rows read back, attention over it.
#include "cache4.h"
#include "launch_parts.h"
#include "rowattn.h"

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
        // V: the pieces of columns 0..3 and 4..7; a word takes those of two
        // neighbouring positions, the even one's lane the first piece, the odd one's the second
        const uint32_t v0 = vc[0] | vc[1] << 4 | vc[2] << 8 | vc[3] << 12, v1 = vc[4] | vc[5] << 4 | vc[6] << 8 | vc[7] << 12;
        const int other = (threadIdx.x & 63) ^ Q::LPP;  // the neighbour's lane with the same columns
        const uint32_t theirs = __shfl(v0 | v1 << 16, other, 64);
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
            *reinterpret_cast<uint32_t*>(c.cache + s.blk.vpiece(s.tl & ~1, 2 * li + odd)) = word;
        } else {
            *reinterpret_cast<uint16_t*>(c.cache + s.blk.vpiece(s.tl, 2 * li)) = (uint16_t)v0;
            *reinterpret_cast<uint16_t*>(c.cache + s.blk.vpiece(s.tl, 2 * li + 1)) = (uint16_t)v1;
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
        if (!s.live) continue;
        float x[8] = {}, y[8] = {};
        if (s.held) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.kword(s.tl, kg * (DH / 32) + g));
            const uint32_t v0 = *reinterpret_cast<const uint16_t*>(c.cache + s.blk.vpiece(s.tl, 2 * li));
            const uint32_t v1 = *reinterpret_cast<const uint16_t*>(c.cache + s.blk.vpiece(s.tl, 2 * li + 1));
            const uint32_t km = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.kmeta(s.tl, g));
            const uint32_t vm = *reinterpret_cast<const uint32_t*>(c.cache + s.blk.vmeta(s.tl, g));
            const uint32_t v = v0 | v1 << 16;
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

// One wave per query row.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void cache4_rows_kernel(AttnArgs a, CacheArgs c, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), p = kn - qn + i;
    float q[RowLanes<DH>::N], o[RowLanes<DH>::N] = {}, m = -__builtin_inff(), l = 0.f;
    if (i < qn) {
        row_load<ST, DH>(row_ptr<ST>(a.q, b, h, i), lane, q);
        const KeyList list = keys_of(a, p, p, kn);
        row_attend<DH>(a, CacheKeys<DH>{c, b, h / a.G}, [&](int e) { return list.key(e); }, 0, list.count, p, kn, q, lane,
                       m, l, o);
    }
    row_finish<ST, DH>(a, b, h, i, row, lane, m, l, o, nullptr, nullptr);
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

size_t cache4_attn_scratch(int, int, const AttnArgs&) { return 0; }

int launch_cache4_attn(int dtype, const AttnArgs& a, const CacheArgs& c, float*, hipStream_t stream) {
    return heads_by_type(dtype, c.dh, [&](auto st, auto d) {
        return launch_parts(((uint64_t)a.B * a.Hq * a.Tq + 3) / 4, 256, [&](uint32_t first, uint32_t blocks) {
            hipLaunchKernelGGL((cache4_rows_kernel<decltype(st), decltype(d)::value>), dim3(blocks), dim3(256), 0,
                               stream, a, c, first);
            return hipGetLastError() == hipSuccess ? 0 : -1;
        });
    });
}

}  // namespace mosa
