// Layout of the 4-bit cache.
//
// A page holds, for every key head, a block of page_size positions:
//   codes of K   page_size rows of dh / 2 bytes
//   codes of V   page_size / 4 groups of 4 positions, 2 dh bytes each
//   meta of K    page_size rows of dh / 32 words, s in the low and m in the high half (bf16)
//   meta of V    the same
// A K row is dh / 8 words; word kg dh / 32 + g holds columns 32 g + 8 kg .. + 7,
// column 2 i in nibble i and column 2 i + 1 in nibble i + 4: lane group kg of a
// matrix instruction over the 32 columns of a group reads its words of all
// groups with one load, and a shift and a mask give a pair of neighbours.
// For V the instruction runs over positions, and its 16 columns have to be of one
// group, whose scale goes with the weights: column 32 g + 2 c + e is number
// c dh / 16 + 2 g + e of its row, so that the columns 2 c and 2 c + 1 of all
// groups, lane c's share, lie together.  In that order a row is kept in 16-bit
// pieces of 4 columns, the pieces of 4 neighbouring positions next to each other:
// a word holds the same columns of two positions.
#pragma once

#include "heads.h"

namespace mosa {

struct CacheBlock {
    size_t at;  // byte offset of the block
    int ps, dh;
    __device__ __forceinline__ size_t kword(int t, int w) const { return at + (size_t)t * (dh / 2) + 4 * w; }
    __device__ __forceinline__ size_t vpiece(int t, int u) const {
        return at + (size_t)ps * (dh / 2) + 2 * (((t >> 2) * (dh / 4) + u) * 4 + (t & 3));
    }
    __device__ __forceinline__ size_t kmeta(int t, int g) const { return at + (size_t)ps * dh + 4 * (t * (dh / 32) + g); }
    __device__ __forceinline__ size_t vmeta(int t, int g) const {
        return kmeta(t, g) + (size_t)ps * (dh / 32) * 4;
    }
};
__host__ __device__ inline size_t cache_block_bytes(int ps, int dh) { return (size_t)ps * (dh + dh / 32 * 8); }

// The block and the place in it of position t of sequence b, head h; false
// where the table ends or names no page.  page_div: by the page size.
__device__ __forceinline__ bool cache_find(const CacheArgs& c, const UDiv& page_div, int b, int h, int t, CacheBlock& blk,
                                           int& tl) {
    if (t < 0) return false;
    const int e = page_div.div(t);
    if (e >= c.per) return false;
    const int page = c.table[(size_t)b * c.per + e];
    if (page < 0 || page >= c.pages) return false;
    blk.at = ((size_t)page * c.H + h) * cache_block_bytes(c.ps, c.dh);
    blk.ps = c.ps;
    blk.dh = c.dh;
    tl = t - e * c.ps;
    return true;
}

// m + s code: the product is exact in fp32 (8 and 4 bits), so there is one rounding.
__device__ __forceinline__ float cache_value(uint32_t meta, uint32_t code) {
    return __builtin_fmaf((float)code, __uint_as_float(meta << 16), __uint_as_float(meta & 0xffff0000u));
}
}  // namespace mosa
