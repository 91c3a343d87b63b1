// Pieces of 16 bytes: products on the matrix cores, roundings, and exchanges between lanes, for the attention kernels.
#pragma once

#include "attend_row.h"

namespace approxifer {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kMfma = 0x8, kDsRead = 0x100;                   // of sched_group_barrier
constexpr int kNoVmem = 0x0f70;                               // of s_waitcnt: until no load from memory is on its way

// D += A B of 16-byte pieces: A [32 x 2 pieces], B [2 pieces x 32]; lane l has row (column) l % 32 and piece l / 32.
template <class E>
__device__ __forceinline__ v16f multiply(v4i a, v4i b, v16f d);
template <>
__device__ __forceinline__ v16f multiply<BF16>(v4i a, v4i b, v16f d) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), d, 0, 0, 0);
}
template <>
__device__ __forceinline__ v16f multiply<F16>(v4i a, v4i b, v16f d) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), d, 0, 0, 0);
}
template <>
__device__ __forceinline__ v16f multiply<F32>(v4i a, v4i b, v16f d) {
    const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) d = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k], y[k], d, 0, 0, 0);
    return d;
}

// Weights relative to a running maximum are kept as 2^kLift times themselves, below 2^15: their sum is, too, and what is small against
// the largest keeps the bits that half precision loses below 2^-14 (many such weights together count).
template <class E>
constexpr float kLift = std::is_same<E, F16>::value ? 7.0f : 0.0f;

// Eight floats rounded to 16 bits.
template <class E>
__device__ __forceinline__ v4i rounded8(const float *p) {
    typedef typename E::Value V8 __attribute__((ext_vector_type(8)));
    V8 x;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = E::store(p[k]);
    return __builtin_bit_cast(v4i, x);
}

// Whether any of a piece's values is an infinity or NaN: its exponent has all ones.
template <class E>
__device__ __forceinline__ bool not_finite(v4i x) {
    constexpr bool kWide = sizeof(typename E::Value) == 4;
    constexpr unsigned kMask = kWide ? 0x7f800000u : std::is_same<E, F16>::value ? 0x7c007c00u : 0x7f807f80u;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned u = static_cast<unsigned>(x[k]) & kMask;
        if (kWide) bad |= u == kMask;
        else bad |= (u & 0xffffu) == (kMask & 0xffffu) || (u >> 16) == (kMask >> 16);
    }
    return bad;
}

// D += A B of 16-byte pieces: A [16 x 4 pieces], B [4 pieces x 16]; lane l has row (column) l % 16 and piece l / 16.
template <class E>
__device__ __forceinline__ v4f multiply16(v4i a, v4i b, v4f d);
template <>
__device__ __forceinline__ v4f multiply16<BF16>(v4i a, v4i b, v4f d) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), d, 0, 0, 0);
}
template <>
__device__ __forceinline__ v4f multiply16<F16>(v4i a, v4i b, v4f d) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), d, 0, 0, 0);
}
template <>
__device__ __forceinline__ v4f multiply16<F32>(v4i a, v4i b, v4f d) {
    const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) d = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k], y[k], d, 0, 0, 0);
    return d;
}

// A row's piece d..d+kPerPiece-1 of a head, whatever its alignment; zeros behind the head.  flip: sign bits to turn.
template <class E>
__device__ __forceinline__ v4i query_piece(const typename E::Value *x, int d, int Dh, bool whole, unsigned flip) {
    typedef typename E::Value V;
    typedef V VP __attribute__((ext_vector_type(16 / sizeof(V))));
    v4i y = {0, 0, 0, 0};
    if (d < Dh) {
        if (whole) {
            y = *reinterpret_cast<const v4i *>(x + d);
        } else {
            VP z;
#pragma unroll
            for (int k = 0; k < static_cast<int>(16 / sizeof(V)); ++k) z[k] = x[d + k];
            y = __builtin_bit_cast(v4i, z);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] ^= flip;
    return y;
}

// Four values, at a multiple of four elements.
template <class E>
__device__ __forceinline__ void store4(typename E::Value *y, float a, float b, float c, float d) {
    typedef typename E::Value V4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<V4 *>(y) = V4{E::store(a), E::store(b), E::store(c), E::store(d)};
}

// The transposing load: lanes 16 g .. 16 g + 15 give the addresses of a 4 x 16 block of 16-bit values, lane i that of row i / 4 and columns
// 4 (i % 4) ..+3, and get column i.
__device__ __forceinline__ v4s load_transposed(const char *a) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(a));
}

// The other half's value as well as this one's: lanes l and l ^ 32 combined.
__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return __int_as_float(r[0]) + __int_as_float(r[1]);
}

// Lanes l, l ^ 16, l ^ 32 and l ^ 48 combined.
__device__ __forceinline__ float quarters_max(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    return half_max(fmaxf(__int_as_float(r[0]), __int_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    return half_sum(__int_as_float(r[0]) + __int_as_float(r[1]));
}

constexpr int pow2_at_least(int n, int p = 1) { return p >= n ? p : pow2_at_least(n, 2 * p); }

// Permutation of the pieces of a row of kStride pieces in LDS: reads of one piece by 16 rows, and of neighbouring pieces by rows next to
// each other, meet all banks.
template <int kStride>
__device__ __forceinline__ int permuted(int row) {
    return kStride == 8 ? ((row >> 1 & 1) << 2 | (row >> 2 & 3)) : ((row & 3) << 2 | (row >> 2 & 3));
}
template <int kStride>
__device__ __forceinline__ int piece_at(int row, int piece) {
    return row * kStride * 16 + ((piece ^ permuted<kStride>(row)) << 4);
}

}  // namespace approxifer
