// What the product kernels of microscaled 4-bit weights are given, and how they read it.
//     Y[r, o] = sum_k W[o, k] X[src(r), k],   W in mx4; X in fp16, bf16 or mx4; sums in fp32, rounded once
// One weight for all rows, or one per expert with the rows in groups: rows offsets[e] .. offsets[e + 1] belong to expert
// e.  src(r) = r, or rows[r].
#pragma once

#include "mx4.h"

namespace mx4 {

struct Product {
    const void* X;
    const uint32_t* x_scales;      // mx4 only
    int64_t tokens, ldx;           // rows of X that rows[] may name, their pitch in elements (mx4: the codes are contiguous)
    int64_t x_rows;                // words of a piece of x_scales
    const int32_t* rows;           // or null
    bool gather;                   // row r of Y is that of row rows[r] of X (otherwise X has been brought into that order)
    const int32_t* offsets;        // or null: one group of all rows
    int64_t n_rows;
    int experts;
    const uint8_t* codes;
    const uint32_t* scales;
    int64_t out, in;
    void* Y;
    int y_type;
    int64_t ldy;
};

// The same as a kernel's argument: up to 112 bytes a launch costs the host 2.7 us, beyond 3.4.  (The host has checked that the sizes fit.)
struct ProductArgs {
    const void* X;
    const uint32_t* x_scales;
    const int32_t *rows, *offsets;
    const uint8_t* codes;
    const uint32_t* scales;
    void* Y;
    int32_t tokens, ldx, x_rows, n_rows, out, in, ldy;
    uint16_t experts;
    uint8_t y_type, gather;

    explicit ProductArgs(const Product& a)
        : X(a.X), x_scales(a.x_scales), rows(a.rows), offsets(a.offsets), codes(a.codes), scales(a.scales), Y(a.Y),
          tokens(static_cast<int32_t>(a.tokens)), ldx(static_cast<int32_t>(a.ldx)), x_rows(static_cast<int32_t>(a.x_rows)),
          n_rows(static_cast<int32_t>(a.n_rows)), out(static_cast<int32_t>(a.out)), in(static_cast<int32_t>(a.in)),
          ldy(static_cast<int32_t>(a.ldy)), experts(static_cast<uint16_t>(a.experts)), y_type(static_cast<uint8_t>(a.y_type)), gather(a.gather) {}
    __device__ __forceinline__ Product open() const {
        return Product{X, x_scales, tokens, ldx, x_rows, rows, gather != 0, offsets, n_rows, experts, codes, scales, out, in, Y, y_type, ldy};
    }
};
static_assert(sizeof(ProductArgs) <= 104, "a pointer more");

// Where the workgroups that share a contraction leave their sums: a counter for each output tile, zero between launches, then the sums.
constexpr int SHARE_TICKETS = 1024;
__device__ __forceinline__ unsigned* tickets_of(void* shared) { return static_cast<unsigned*>(shared); }
__device__ __forceinline__ float* parts_of(void* shared) { return static_cast<float*>(shared) + SHARE_TICKETS; }

struct Group {
    int64_t lo, hi;
    const uint8_t* codes;
    const uint32_t* scales;
};

// Expert e's rows, held inside [0, n_rows] whatever the offsets say, and its weight.
__device__ __forceinline__ Group group_of(const Product& a, int e) {
    Group g{0, a.n_rows, a.codes, a.scales};
    if (a.offsets) {
        g.lo = min(int64_t(max(a.offsets[e], 0)), a.n_rows);
        g.hi = min(int64_t(max(a.offsets[e + 1], 0)), a.n_rows);
        g.codes += int64_t(e) * a.out * pieces(a.in) * PIECE_BYTES;
        g.scales += int64_t(e) * a.out * pieces(a.in);
    }
    return g;
}

// The row of X behind row r of Y; -1 behind the group's end or where rows[] names none (that row of Y is zeros).
__device__ __forceinline__ int64_t source_row(const Product& a, int64_t r, int64_t hi) {
    if (r >= hi) return -1;
    if (!a.rows) return r;
    const int64_t s = a.rows[r];
    return s >= 0 && s < a.tokens ? (a.gather ? s : r) : -1;
}

__device__ __forceinline__ void store_y(const Product& a, int64_t row, int64_t col, float v) {
    const int64_t at = row * a.ldy + col;
    if (a.y_type == ADADIM_TYPE_F16) static_cast<_Float16*>(a.Y)[at] = static_cast<_Float16>(v);
    else if (a.y_type == ADADIM_TYPE_BF16) static_cast<__bf16*>(a.Y)[at] = static_cast<__bf16>(v);
    else static_cast<float*>(a.Y)[at] = v;
}

}  // namespace mx4
