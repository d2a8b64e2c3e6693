// Tiles of 64 rows of bf16 copied from global memory straight into LDS by the 4
// waves of a workgroup, for the windowed attention's kernels.
//
// One instruction of a wave fills 1 KB, lane l the bytes 16 l .. 16 l + 15: unit
// p = 64 (wave + 4 j) + lane of a tile is row p / U, stored unit p % U (U units
// of 16 bytes per row), and holds the row's unit (p % U) ^ swizzle(row).  The
// swizzles depend on a row's low 4 bits, and the rows of a lane's loads are 16
// or more apart, so all its loads take the same unit.
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

constexpr int kTB = 64;  // rows per tile

// Unit permutation of a tile's rows.  With 16-byte reads of one unit of 16 rows
// and transposed 8-byte reads of unit pairs of 4 x 4 rows, both as fast as reads
// of consecutive bytes (4.5 and 5.4 cycles of a CU's LDS per wave read; other
// permutations of the 128-byte rows measured 8.2 and 5.4, none 16 and 8.3).
template <int DH>
__device__ __forceinline__ int tile_swz(int r) {
    if constexpr (DH == 128) return r & 15;
    else if constexpr (DH == 64) return r & 7;
    else return (r >> 1) & 3;
}

template <int DH>
struct TileLoad {
    static constexpr int U = DH / 8, LD = kTB * DH * 2 / 4096, STEP = 256 / U;  // loads per wave, rows between them
    static constexpr int BYTES = kTB * DH * 2;
    int row, col;     // this lane's row of load 0, and its first column
    uint32_t lds;     // byte offset of the wave's first block within a tile
    __device__ __forceinline__ TileLoad(int wave, int lane)
        : row((64 * wave + lane) / U), lds(1024 * (uint32_t)__builtin_amdgcn_readfirstlane(wave)) {
        col = 8 * ((64 * wave + lane) % U ^ tile_swz<DH>(row));
    }
};

// Keys e0 .. e0 + 63 of a list.
template <int DH>
struct KeyTiles {
    using TL = TileLoad<DH>;
    const uint16_t* base;
    int64_t stride;
    uint32_t off;
    bool near;
    __device__ __forceinline__ KeyTiles(const Rows& t, int b, int hk, const TL& tl)
        : base(row_ptr<uint16_t>(t, b, hk, 0)), stride(t.row) {
        near = stride < ((int64_t)1 << 24);  // 64 rows within 2^31 bytes
        off = (uint32_t)(((int64_t)tl.row * stride + tl.col) * 2);
    }
    __device__ __forceinline__ void issue(const TL& tl, const KeyList& l, int e0, uint32_t at) const {
        if (near && e0 >= l.s && e0 + kTB <= l.count) {
            const char* p = uniform_ptr(reinterpret_cast<const char*>(base + (int64_t)(e0 - l.s + l.lo) * stride));
#pragma unroll
            for (int j = 0; j < TL::LD; ++j) lds_load16s(off, p + (int64_t)(2 * TL::STEP * j) * stride, at + tl.lds + 4096 * j);
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
template <int DH>
struct TileReads {
    static constexpr int U = DH / 8, NS = DH / 32, ND = DH / 16;
    int row[NS], tr[ND];
    __device__ __forceinline__ TileReads(int g, int c16) {
#pragma unroll
        for (int st = 0; st < NS; ++st) row[st] = (c16 * U + ((4 * st + g) ^ tile_swz<DH>(c16))) * 16;
        const int r = 4 * g + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < ND; ++db) {
            const int col = 16 * db + 4 * (c16 & 3);
            tr[db] = (r * U + ((col >> 3) ^ tile_swz<DH>(r))) * 16 + 8 * ((col >> 2) & 1);
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

__device__ __forceinline__ Frag8<uint16_t> pack_frag(const f32x4& x, const f32x4& y) {
    const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    return frag8_from<uint16_t>(v);
}

}  // namespace mosa
