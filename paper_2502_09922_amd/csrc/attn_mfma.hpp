// What the matrix-core kernels of attention over a cache share: tiles' layout in LDS, bf16 operands in two parts.
#pragma once
#include "device_util.hpp"

namespace ls {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16-byte chunks of a row of a tile are permuted by its key, so that 16 rows' equal chunks (keys) and 4 rows' 32 bytes (values,
// transposing) lie in different banks.
template <class T, int HD> __device__ __forceinline__ int key_swizzle(int key) { return HD == 128 || sizeof(T) == 4 ? key & 15 : ((key & 3) << 1) | ((key >> 2) & 1); }
template <class T, int HD> __device__ __forceinline__ int value_swizzle(int key) {
  return sizeof(T) == 4 ? 0 : HD == 128 ? (key & 7) << 1 : ((key & 3) << 1) | ((key >> 2) & 1);
}

// v as a sum of two bf16: the first is v cut off, the second the rest, rounded, at least 2^-23 of v and of its sign.  Off by 2^-15 of v at
// most; infinite factors take part with their sign alone (inf + 0 inf or inf - inf would be no number).  0 stays 0.
__device__ __forceinline__ void two_parts(float v, bf16& first, bf16& second) {
  const unsigned bits = __builtin_bit_cast(unsigned, v);
  first = __builtin_bit_cast(bf16, (unsigned short)(bits >> 16));
  second = (bf16)fmaf(v, 0x1.000002p0f, -__builtin_bit_cast(float, bits & 0xFFFF0000u));
}

// v as a sum of three bf16, exactly: v cut off, the rest cut off, what is left of its 24 bits.  None of them is zero unless v is, and all have
// its sign: where nothing is left a part is halved.
__device__ __forceinline__ void three_parts(float v, bf16* part) {
  auto cut = [](float w) { return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, w) & 0xFFFF0000u); };
  float a = cut(v), rest = v - a;
  if (rest == 0.f) rest = a *= 0.5f;
  float b = cut(rest), c = rest - b;
  if (c == 0.f) c = b *= 0.5f;
  part[0] = (bf16)a;
  part[1] = (bf16)b;
  part[2] = (bf16)c;
}

}  // namespace ls
