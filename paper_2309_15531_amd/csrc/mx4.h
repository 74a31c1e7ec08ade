// Microscaled 4-bit storage ("mx4") and the device helpers its kernels share.
//
// A row is held in pieces of 128 values: 64 bytes of codes (value 2i in the low half of byte i) and one 32-bit word
// with the scale bytes of the piece's four blocks of 32.  codes u8 [rows][64 * pieces]; scales u32 [pieces][rows]: the
// words that the matrix kernels fetch for one step along the contraction, one per row, lie side by side.  The last
// piece is filled up with codes of 0 and scale bytes of 127 (2^0).
//
// Everything the hardware does here is exact: v_cvt_scalef32_pk_{f32,f16,bf16}_fp4 multiply the value of a code by the
// power of two in the exponent field of their scale operand (a field of 0 is 2^-127, 255 is NaN),
// v_cvt_scalef32_pk_fp4_f32 divides by it, rounds to nearest with ties to even and saturates at 6.
#pragma once

#include "common.h"

namespace mx4 {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

constexpr int PIECE = 128;                        // values that share a word of scales
constexpr int PIECE_BYTES = 64;
constexpr uint32_t ONE_WORD = 0x7f7f7f7fu;        // four scales of 1

__host__ __device__ inline int64_t pieces(int64_t cols) { return (cols + PIECE - 1) / PIECE; }

// Loads and stores of what need not be aligned to more than its element: the compiler's own choice of instructions.
template <class V>
__device__ __forceinline__ V load_any(const void* p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V>
__device__ __forceinline__ void store_any(void* p, const V& v) {
    __builtin_memcpy(p, &v, sizeof(V));
}

// N consecutive elements of a row of which the first `have` exist (the rest reads as zero).
template <class T, int N>
struct Chunk {
    typedef T vec __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ vec load(const T* p, int have) {
        if (have >= N) return load_any<vec>(p);
        vec v = {};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) v[i] = p[i];
        return v;
    }
    static __device__ __forceinline__ void store(T* p, int have, const vec& v) {
        if (have >= N) {
            store_any(p, v);
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) p[i] = v[i];
    }
};

// The scale operand of a conversion: the scale byte in the exponent field.
__device__ __forceinline__ float scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// The eight values of a word of codes, times the scale.
__device__ __forceinline__ void values8(uint32_t w, float scale, float (&v)[8]) {
    const float2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
                  c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
}
__device__ __forceinline__ half8v values8_f16(uint32_t w, float scale) {
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
    return half8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ bf8v values8_bf16(uint32_t w, float scale) {
    const bf2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// fp16 holds the values of a block exactly for scales 2^-23 (half of it is fp16's smallest subnormal) to 2^13 (6 times it
// is 49152).  Whether a scale byte lies outside 104 .. 140, as NaN's does.
__device__ __forceinline__ bool beyond_f16(uint32_t byte) { return byte - 104u > 36u; }

// x = hi + lo with both in bf16: the first 8 of fp16's 11 bits and the rest.  Cut, not rounded: 65504 would become 65536, and its product
// with a weight pass fp32's range where the exact one does not.  What is not finite goes whole into hi.
__device__ __forceinline__ void split_f16(const half8v& x, bf8v& hi, bf8v& lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = static_cast<float>(x[i]);
        const bool finite = f - f == 0.0f;
        const float first = finite ? __uint_as_float(__float_as_uint(f) & 0xffff0000u) : f;
        hi[i] = static_cast<__bf16>(first);
        lo[i] = static_cast<__bf16>(finite ? f - first : 0.0f);
    }
}

}  // namespace mx4
