// Pages that hold keys and values in 4 bits: where things lie in a tile, and what codes stand for.  Not part of the C ABI, and
// not exported.
#ifndef HPS_SEQ_PACKED_H
#define HPS_SEQ_PACKED_H

#include "hps_seq_common.h"

// Scales up to this byte are numbers.  Above it, 6 times the scale is beyond what the type holds.
template <typename T> constexpr uint32_t kPackedMost = 252;
template <> constexpr inline uint32_t kPackedMost<_Float16> = 140;
// Scales that are written: 2^-126 .. 2^125; for f16 the least, 2^-23, is half of the largest code's distance to f16's least number.
template <typename T> constexpr int kPackedLeast = 1;
template <> constexpr inline int kPackedLeast<_Float16> = 104;

inline bool seq_packed_dim(uint32_t d) { return d == 32 || d == 64 || d == 96 || d == 128 || d == 256; }
inline bool seq_packed_block(uint32_t b) { return seq_block_size(b) && b >= 16; }

// What all calls with packed pages ask of them.
SEQ_HIDDEN hps_status_t seq_check_packed(const hps_seq_packed_t &pages, uint32_t head_dim);

// A scale byte as a factor; what is above the type's becomes NaN in the conversions (as 255 does by itself).
template <typename T> __device__ __forceinline__ float packed_scale(uint32_t b) { return __uint_as_float((b > kPackedMost<T> ? 255u : b) << 23); }

// Two codes, byte kByte of x, as numbers.
template <typename T> struct Packed;
template <> struct Packed<float> {
    typedef float pair __attribute__((ext_vector_type(2)));
    template <int kByte> static __device__ __forceinline__ pair values(uint32_t x, float s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, s, kByte); }
};
template <> struct Packed<_Float16> {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    template <int kByte> static __device__ __forceinline__ pair values(uint32_t x, float s) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, s, kByte); }
};
template <> struct Packed<__bf16> {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    template <int kByte> static __device__ __forceinline__ pair values(uint32_t x, float s) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, kByte); }
};

#endif  // HPS_SEQ_PACKED_H
