// Tiles of 64 rows of bf16 or 32 rows of fp32 copied from global memory straight
// into LDS by the 4 waves of a workgroup, for the windowed attention's kernels.
//
// One instruction of a wave fills 1 KB, lane l the bytes 16 l .. 16 l + 15: unit
// p = 64 (wave + 4 j) + lane of a tile is row p / U, stored unit p % U (U units
// of 16 bytes per row), and holds the row's unit (p % U) ^ swizzle(row).  The
// swizzles depend on a row's low 4 bits (3 for rows of 512 bytes), and the rows of
// a lane's loads are 16 (8) or more apart, so all its loads take the same unit.
//
// A load's address is a uniform base in scalar registers and a lane offset of
// 32 bits that does not change from tile to tile: the copies cost no vector
// instructions beside the matrix products.  Tiles at the ends of a list, and
// tensors whose rows are further apart than that reaches, go by 64-bit
// addresses instead.
#pragma once

#include "attn_lds.h"
#include "heads.h"

namespace mosa {

__device__ __forceinline__ void lds_load16s(uint32_t off, const void* base, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
// 4 bytes per lane (256 bytes per wave).
__device__ __forceinline__ void lds_load4(const void* g, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" : : "v"(g), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4s(uint32_t off, const void* base, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dword %0, %1" : : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ const char* uniform_ptr(const char* p) {
    const uint64_t u = (uint64_t)p;
    return (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 |
                         (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}

// A kernel's arguments by the address of their segment, in scalar registers.
template <typename T>
__device__ __forceinline__ T uniform_args(const void* segment) {
    T t;
    __builtin_memcpy(&t, (const __attribute__((address_space(4))) void*)(uintptr_t)uniform_ptr(static_cast<const char*>(segment)), sizeof(T));
    return t;
}
// LDS by its byte address.
__device__ __forceinline__ unsigned char* lds_at(uint32_t at) {
    return (unsigned char*)(__attribute__((address_space(3))) unsigned char*)(uintptr_t)at;
}

template <typename ST>
constexpr int kTileRows = sizeof(ST) == 2 ? 64 : 32;

// Unit permutation of a tile's rows.  bf16: with 16-byte reads of one unit of 16
// rows and transposed 8-byte reads of unit pairs of 4 x 4 rows, both as fast as
// reads of consecutive bytes (4.5 and 5.4 cycles of a CU's LDS per wave read;
// other permutations of the 128-byte rows measured 8.2 and 5.4, none 16 and 8.3).
// fp32: the columns' reads take 4 bytes of rows 4 apart.
template <typename ST, int DH>
__device__ __forceinline__ int tile_swz(int r) {
    if constexpr (sizeof(ST) == 4) return (r & 3) + 4 * ((r >> 2) & (DH == 64 ? 3 : 1));
    else if constexpr (DH == 128) return r & 15;
    else if constexpr (DH == 64) return r & 7;
    else return (r >> 1) & 3;
}

template <typename ST, int DH>
struct TileLoad {
    static constexpr int TB = kTileRows<ST>, E = 16 / (int)sizeof(ST), U = DH / E;  // values per unit, units per row
    static constexpr int BYTES = TB * DH * (int)sizeof(ST), LD = BYTES / 4096, STEP = 256 / U;  // loads per wave, rows between them
    int row, col;     // this lane's row of load 0, and its first column
    uint32_t lds;     // byte offset of the wave's first block within a tile
    __device__ __forceinline__ TileLoad(int wave, int lane)
        : row((64 * wave + lane) / U), lds(1024 * (uint32_t)__builtin_amdgcn_readfirstlane(wave)) {
        col = E * ((64 * wave + lane) % U ^ tile_swz<ST, DH>(row));
    }
};

// Keys e0 .. e0 + TB - 1 of a list.
template <typename ST, int DH>
struct KeyTiles {
    using TL = TileLoad<ST, DH>;
    const ST* base;
    int64_t stride;
    uint32_t off;
    bool near;
    __device__ __forceinline__ KeyTiles(const Rows& t, int b, int hk, const TL& tl)
        : base(row_ptr<ST>(t, b, hk, 0)), stride(t.row) {
        near = stride < ((int64_t)1 << 24);  // a tile's rows within 2^31 bytes
        off = (uint32_t)((tl.row * stride + tl.col) * (int)sizeof(ST));
    }
    __device__ __forceinline__ void issue(const TL& tl, const KeyList& l, int e0, uint32_t at) const {
        if (near && e0 >= l.s && e0 + TL::TB <= l.count) {
            const char* p = uniform_ptr(reinterpret_cast<const char*>(base + (int64_t)(e0 - l.s + l.lo) * stride));
#pragma unroll
            for (int j = 0; j < TL::LD; ++j)
                lds_load16s(off, p + (int64_t)((int)sizeof(ST) * TL::STEP * j) * stride, at + tl.lds + 4096 * j);
        } else {  // entries past the list are its last one
#pragma unroll
            for (int j = 0; j < TL::LD; ++j)
                lds_load16(base + (int64_t)l.key(min(e0 + tl.row + TL::STEP * j, l.count - 1)) * stride + tl.col,
                           at + tl.lds + 4096 * j);
        }
    }
};

// Fragment reads of a tile: 16 rows by 32 columns as they lie, and, transposed,
// 16 columns by 32 rows in the slot order of two 16-row result blocks (slots
// 0 .. 3 rows 4 g + i of block 2 u, slots 4 .. 7 the same of block 2 u + 1).
template <typename ST, int DH>
struct TileReads;
template <int DH>
struct TileReads<uint16_t, DH> {
    static constexpr int U = DH / 8, NS = DH / 32, ND = DH / 16;
    int row[NS], tr[ND];
    __device__ __forceinline__ TileReads(int g, int c16) {
#pragma unroll
        for (int st = 0; st < NS; ++st) row[st] = (c16 * U + ((4 * st + g) ^ tile_swz<uint16_t, DH>(c16))) * 16;
        const int r = 4 * g + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < ND; ++db) {
            const int col = 16 * db + 4 * (c16 & 3);
            tr[db] = (r * U + ((col >> 3) ^ tile_swz<uint16_t, DH>(r))) * 16 + 8 * ((col >> 2) & 1);
        }
    }
    __device__ __forceinline__ Frag8<uint16_t> rows(const unsigned char* t, int sb, int st) const {
        Frag8<uint16_t> f;
        f.v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(t + row[st] + 16 * U * 16 * sb));
        return f;
    }
    __device__ __forceinline__ Frag8<uint16_t> cols(const unsigned char* t, int u, int db) const {
        const u32x2 lo = lds_tr16(t + tr[db] + 32 * u * U * 16);
        const u32x2 hi = lds_tr16(t + tr[db] + (32 * u + 16) * U * 16);
        Frag8<uint16_t> f;
        f.v = __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
        return f;
    }
};
template <int DH>
struct TileReads<float, DH> {
    static constexpr int U = DH / 4, NS = DH / 32, ND = DH / 16;
    int g, c16;
    __device__ __forceinline__ TileReads(int g, int c16) : g(g), c16(c16) {}
    static __device__ __forceinline__ int at(int r, int unit) { return (r * U + (unit ^ tile_swz<float, DH>(r))) * 16; }
    __device__ __forceinline__ Frag8<float> rows(const unsigned char* t, int sb, int st) const {
        Frag8<float> f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 x = *reinterpret_cast<const float4*>(t + at(16 * sb + c16, 8 * st + 2 * g + h));
            f.v[4 * h] = x.x, f.v[4 * h + 1] = x.y, f.v[4 * h + 2] = x.z, f.v[4 * h + 3] = x.w;
        }
        return f;
    }
    __device__ __forceinline__ Frag8<float> cols(const unsigned char* t, int u, int db) const {
        Frag8<float> f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r = 32 * u + 16 * (e >> 2) + 4 * g + (e & 3), col = 16 * db + c16;
            f.v[e] = *reinterpret_cast<const float*>(t + at(r, col >> 2) + 4 * (col & 3));
        }
        return f;
    }
};

// Numbers lo .. hi of a run: which rows (keys) of a tile a lane's key (row) pairs with.
struct Span {
    int lo = 1 << 30;  // (an empty run lies past every tile)
    uint32_t n = 0;    // hi - lo
    __device__ __forceinline__ Span() {}
    __device__ __forceinline__ Span(int lo, int hi) : lo(hi < lo ? 1 << 30 : lo), n(hi < lo ? 0u : (uint32_t)(hi - lo)) {}
    __device__ __forceinline__ bool has(int c) const { return (uint32_t)(c - lo) <= n; }
};

// A fragment's loads are waited for here: a first use inside a pipeline would
// wait there for every load in flight, the next tiles' included.
__device__ __forceinline__ void take(Frag8<uint16_t>& f) { asm volatile("" : "+v"(f.v)); }
__device__ __forceinline__ void take(Frag8<float>& f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(f.v[e]));
}

// Two 16-row result blocks as an operand (bf16: rounded here).
template <typename ST>
__device__ __forceinline__ Frag8<ST> pack_frag(const f32x4& x, const f32x4& y) {
    const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    return frag8_from<ST>(v);
}

// What a row does not see has a weight of 0 in the products of a tile, which is
// not enough where it holds infinities or NaN: 0 times those is NaN.  Only tiles
// that some of the workgroup's rows (keys) pair with in part can do that harm.
// A workgroup whose results are not finite walks its tiles a second time.  Before
// such a tile is multiplied its infinities then become the largest numbers of
// their sign, NaN too (keep_finite): scores keep their meaning, and a weight of 0
// gives 0.  At the end these tiles are visited once more, and what was not finite
// joins the results that it belongs to (add_not_finite).

// One call by the whole workgroup; a barrier follows.
template <typename ST, int DH>
__device__ __forceinline__ void keep_finite(unsigned char* t, int tid) {
    constexpr uint32_t body = sizeof(ST) == 2 ? 0x7fff7fffu : 0x7fffffffu, one = sizeof(ST) == 2 ? 0x00800080u : 0x00800000u;
    constexpr uint32_t sign = ~body;  // where an exponent of all ones overflows to
#pragma unroll 1
    for (int i = 4 * tid; i < TileLoad<ST, DH>::BYTES; i += 1024) {
        uint32_t* p = reinterpret_cast<uint32_t*>(t + i);
        const uint32_t x = *p, bad = ((x & body) + one) & sign;
        if constexpr (sizeof(ST) == 2) {
            const uint32_t lo = bad & 0x8000u ? (x & 0x8000u) | 0x7f7fu : x & 0xffffu;
            const uint32_t hi = bad >> 31 ? (x & 0x80000000u) | 0x7f7f0000u : x & 0xffff0000u;
            *p = lo | hi;
        } else {
            *p = bad ? (x & sign) | 0x7f7fffffu : x;
        }
    }
}

// 1 where a value is infinite with this sign or NaN (any: not finite), otherwise 0.
template <bool any>
__device__ __forceinline__ Frag8<uint16_t> not_finite(const Frag8<uint16_t>& f, uint32_t sign) {
    u32x4 w = __builtin_bit_cast(u32x4, f.v);
    auto is = [&](uint32_t h) __attribute__((always_inline)) {
        const uint32_t m = h & 0x7fffu;
        return any ? m >= 0x7f80u : (m > 0x7f80u) | (h == (0x7f80u | sign << 15));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = (is(w[i] & 0xffffu) ? 0x3f80u : 0u) | (is(w[i] >> 16) ? 0x3f800000u : 0u);
    Frag8<uint16_t> x;
    x.v = __builtin_bit_cast(bf16x8, w);
    return x;
}
template <bool any>
__device__ __forceinline__ Frag8<float> not_finite(const Frag8<float>& f, uint32_t sign) {
    const float inf = sign ? -__builtin_inff() : __builtin_inff();
    Frag8<float> x;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x.v[e] = (any ? !(fabsf(f.v[e]) < __builtin_inff()) : (f.v[e] == inf) | (f.v[e] != f.v[e])) ? 1.f : 0.f;
    return x;
}

// What is not finite in a tile joins the sums x (value i of x[n][db] is column
// 16 db + 4 g + i of the lane's n-th row or key, which pairs with tile row r iff
// in(r, n)): products of ones count it, by sign, as NaN where both signs count.
// nan: NaN for either, for sums whose other factor may have any sign or be 0.
template <typename ST, int DH, bool nan, int N, class IN>
__device__ __forceinline__ void add_not_finite(const TileReads<ST, DH>& rd, const unsigned char* t, int g,
                                               f32x4 (&x)[N][DH / 16], const IN& in) {
    constexpr int M = kTileRows<ST> / 32;
    Frag8<ST> pairs[N][M];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int u = 0; u < M; ++u) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = in(32 * u + 16 * (e >> 2) + 4 * g + (e & 3), n) ? 1.f : 0.f;
            pairs[n][u] = frag8_from<ST>(v);
        }
#pragma unroll
    for (int db = 0; db < DH / 16; ++db) {
        __builtin_amdgcn_sched_barrier(0);  // (a rare path: few registers)
        f32x4 up[N], down[N];
#pragma unroll
        for (int n = 0; n < N; ++n) up[n] = down[n] = zero4();
#pragma unroll
        for (int u = 0; u < M; ++u) {
            const Frag8<ST> f = rd.cols(t, u, db), p = not_finite<nan>(f, 0), m = not_finite<nan>(f, 1);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                mma8(up[n], p, pairs[n][u]);
                if constexpr (!nan) mma8(down[n], m, pairs[n][u]);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[n][db][i] += up[n][i] > 0.f ? (nan ? __builtin_nanf("") : __builtin_inff()) : 0.f;
                if constexpr (!nan) x[n][db][i] += down[n][i] > 0.f ? -__builtin_inff() : 0.f;
            }
    }
}

template <int N>
__device__ __forceinline__ bool finite4(const f32x4 (&x)[N]) {
    float t = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __builtin_fmaf(x[n][i], 0.f, t);
    return t == 0.f;
}

// Whether x holds in some lane of the workgroup's 4 waves (lds: 16 bytes that are free).
__device__ __forceinline__ bool any_of_workgroup(unsigned char* lds, int wave, int lane, bool x) {
    uint32_t* f = reinterpret_cast<uint32_t*>(lds);
    const bool mine = __builtin_amdgcn_ballot_w64(x) != 0;
    if (lane == 0) f[wave] = mine;
    __syncthreads();
    const uint32_t any = __builtin_amdgcn_readfirstlane((int)(f[0] | f[1] | f[2] | f[3]));
    __syncthreads();
    return any != 0;
}

// Rows of 16 N results (column c16 of block n, values 4 g + i of every 16, times
// f[n]) through this wave's part of LDS to 16-byte stores: to(row) is the row's
// address or nullptr.
template <typename ST, int DH>
constexpr int store_rows_bytes(int n) { return 16 * n * (DH * (int)sizeof(ST) + 16); }
template <typename ST, int DH, int N, class TO>
__device__ __forceinline__ void store_rows(unsigned char* lds, const f32x4 (&x)[N][DH / 16], const float (&f)[N], int lane,
                                           const TO& to) {
    constexpr int E = 16 / (int)sizeof(ST), LDO = DH + E, U = DH / E;
    ST* o = reinterpret_cast<ST*>(lds);
    const int g = lane >> 4, c16 = lane & 15;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int db = 0; db < DH / 16; ++db) {
            ST* p = o + (16 * n + c16) * LDO + 16 * db + 4 * g;
            const f32x4 v = x[n][db] * f[n];
            if constexpr (sizeof(ST) == 2)
                *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            else
                *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        }
    wave_sync();
#pragma unroll
    for (int e = lane; e < 16 * N * U; e += 64) {
        const int r = e / U, dc = (e % U) * E;
        if (ST* p = to(r)) *reinterpret_cast<uint4*>(p + dc) = *reinterpret_cast<const uint4*>(o + r * LDO + dc);
    }
    wave_sync();
}

}  // namespace mosa
