// Layout of a paged cache of keys and values in mx4, and what its kernels share.
//
// A pool u8 [pages][heads][page / 32][34 D]: page positions (a power of two, 32 or more) of each key-value head in records of 32
// positions.  D = 64, 128 or 256 is what a head is filled up to with zeros.  A record:
//   keys    codes [32 positions][D / 2], then behind the values' codes scales [32][D / 32]
//   values  codes [4][16][8][D / 32], scales [4][D / 32][8]
// in the order  key codes (16 D bytes), value codes (16 D), key scales (D), value scales (D).
//
// The order of the values is that of the matrix instructions (v_mfma_f32_16x16x32): the transposed scores S^T = K Q^T of 16 positions
// leave position 4 g + i of a query in register i of lane quarter g, and as the right operand of O^T = V^T P^T a lane of quarter
// g holds 8 positions: two such tiles of scores, 4 g + i and 16 + 4 g + i, are that operand as they stand, if V^T brings the same
// positions.  So the lane of row m and quarter g of the left operand finds its 8 positions' codes of the elements m D / 16 .. (one for each of
// the D / 16 instructions along D) side by side: one load of D / 4 bytes, and one of 8 for the scales.  No value is turned
// round through LDS, and a position's own bytes belong to no other, so that appending one needs no read.
//
// Scales are held to 2^-23 .. 2^13, where fp16 has every value of a block.  A position whose key or value is not finite has key scales of 255
// (NaN: whoever sees it gets NaN) and is zeros otherwise: a NaN among the values would reach rows that do not see it (0 x NaN).
#pragma once

#include "mx4.h"

namespace mx4 {

constexpr int RECORD = 32;                        // positions
constexpr uint32_t CACHE_LEAST = 104, CACHE_MOST = 140;      // scale bytes of 2^-23, 2^13

inline int filled_head(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

template <int D>
struct Record {
    static constexpr int BYTES = 34 * D, VALUES = 16 * D, KEY_SCALES = 32 * D, VALUE_SCALES = 33 * D;
    static constexpr int UNIT = D / 32;           // bytes of a position's value codes that lie together
    // position t of a record among the values: quarter and place
    static __host__ __device__ constexpr int quarter(int t) { return (t & 15) >> 2; }
    static __host__ __device__ constexpr int place(int t) { return (t & 3) + ((t >> 4) << 2); }
};

// Where slot (page * positions + position) of a head begins; LOG: log2 of the page's positions.
__device__ __forceinline__ int64_t record_of(int64_t page, int heads, int head, int log_page, int at, int bytes) {
    return (((page * heads + head) << (log_page - 5)) + (at >> 5)) * bytes;
}

struct Attention {
    const void* Q;
    int64_t tokens, ldq;
    const uint8_t* cache;
    int64_t pages;
    int log_page, heads, group, dim;              // key-value heads, query heads to each
    const int32_t* table;
    int64_t width;                                // pages that a sequence may have
    int sequences;
    const int32_t* offsets;
    const int32_t* lengths;
    void* Y;
    int y_type;
    int64_t ldy;
    float scale;
    int causal;
    int64_t window;                               // 0: none
    int64_t max_new, max_length;                  // what a launch is laid out for; results do not depend on them
};

}  // namespace mx4
