// kept.hpp — keys and values held in 8 or 4 bits: where the bytes of a page lie, and
// how they become bf16.
//
// 32 dims of a token's head share a scale 2^e, kept as the byte e + 127 (255: all 32
// are NaN); a value is a multiple of it with 8 bits (E4M3) or 4 (E2M1, the even dim
// in the low half of a byte).  A page of one head is the codes of its tokens, then their
// scales.  Keys lie token by token.  Values lie in fours of tokens, of which
// each sixteenth of a head's dims, or each scale, comes in turn: what a lane of the
// attention multiplies, four tokens at D / 16 dims, is then consecutive bytes, and
// what a wave loads of 16 tokens, keys or values, is one stretch in lane order.
#pragma once

#include "wise_device.hpp"

namespace wise {

template <int D, int B>
struct Kept {
  static constexpr int kRow = D * B / 8;              // bytes of a token's codes
  static constexpr int kScales = D / 32;              // and scales
  static constexpr int kPiece = kRow / 4;             // bytes of a lane: a quarter of a key, or four tokens' sixteenths
  static constexpr int kWords = kPiece / 4;
  static constexpr int kPairs = D / 32;               // pairs of dims of a token's sixteenth

  // Byte of dim d of token t's codes, and of its scale of dims 32 g ..., behind the page's codes.
  __device__ static int v_code(int t, int d) {
    const int j = d * B / 8, piece = kRow / 16;
    return (t >> 2) * 4 * kRow + j / piece * kPiece + (t & 3) * piece + j % piece;
  }
  __device__ static int v_scale(int t, int g) { return ((t >> 2) * kScales + g) * 4 + (t & 3); }
};

inline int kept_key_bytes(int d, int bits) { return 2 * (d * bits / 8 + d / 32); }   // of K and V, a key and key-value head

// Two values of a word as bf16 (or kHalf: as fp16): number i of its bytes (B = 4) or half words (B = 8).  Only
// the exponent of `scale` counts, whatever its other bits; 255 makes NaN of any code.
template <int B, bool kHalf = false>
__device__ __forceinline__ uint32_t widen_pair(uint32_t w, float scale, int i) {
  if constexpr (B == 4 && !kHalf) {
    return __builtin_bit_cast(uint32_t, i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
                                        : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
                                        : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  } else if constexpr (B == 4) {
    return __builtin_bit_cast(uint32_t, i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)
                                        : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)
                                        : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3));
  } else if constexpr (!kHalf) {
    return __builtin_bit_cast(uint32_t, i == 0 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  } else {
    return __builtin_bit_cast(uint32_t, i == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false)
                                               : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
  }
}
// Pair i of consecutive words.
template <int B, bool kHalf = false>
__device__ __forceinline__ uint32_t widen_at(const uint32_t* w, float scale, int i) {
  constexpr int kPer = B == 4 ? 4 : 2;
  return widen_pair<B, kHalf>(w[i / kPer], scale, i % kPer);
}

// Nonzero bits where one of a word's scales makes products that fp16 does not hold exactly: it does
// with e from -23 to 8 for 4 bits (0.5 to 6 times 2^e, and would to 13), from -15 to 7 for 8 (2^-9 to 448).  A byte
// carries into the next one only where it is itself past a border.
template <int B>
__device__ __forceinline__ uint32_t past_half(uint32_t w) {
  return B == 4 ? ((w + 0x18181818u) ^ 0x80808080u) & 0xe0e0e0e0u : ~((w + 0x10101010u) & (w + 0x79797979u)) & 0x80808080u;
}

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {   // of two 16-bit numbers each
  typedef uint16_t U2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(U2, a), __builtin_bit_cast(U2, b)));
}

// Scale byte i of a word, as widen_pair takes it.
__device__ __forceinline__ float scale_of(uint32_t w, int i) {
  return __builtin_bit_cast(float, i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1);
}

// A word whose first n bytes are 255 (none for n < 0, all for n > 4).
__device__ __forceinline__ uint32_t low_bytes(int n) { return n <= 0 ? 0u : ~0u >> (32 - 8 * min(n, 4)); }

// The bytes of w that are 255, and (kCode) those whose lower seven bits are set, as 255.
template <bool kCode>
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t t = ((w & 0x7f7f7f7fu) + 0x01010101u) & (kCode ? 0x80808080u : 0x80808080u & w);
  return (t >> 7) * 255u;
}

// N words at p, which is aligned as a lane's bytes are.  kOnce: they are not read again soon, and need not stay in the L2.
template <int N, bool kOnce = false>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  typedef uint32_t W2 __attribute__((ext_vector_type(2), aligned(8)));
  typedef uint32_t W3 __attribute__((ext_vector_type(3), aligned(4)));
  typedef uint32_t W4 __attribute__((ext_vector_type(4), aligned(8)));
  static_assert(N == 2 || N == 3 || N == 4 || N == 6 || N == 8, "words of a lane");
  if constexpr (N >= 4) {
    const W4 x = kOnce ? __builtin_nontemporal_load((const W4*)p) : *(const W4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
    if constexpr (N > 4) load_words<N - 4, kOnce>(p + 16, w + 4);
  } else if constexpr (N == 3) {
    const W3 x = kOnce ? __builtin_nontemporal_load((const W3*)p) : *(const W3*)p;
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = x[i];
  } else {
    const W2 x = kOnce ? __builtin_nontemporal_load((const W2*)p) : *(const W2*)p;
    w[0] = x[0], w[1] = x[1];
  }
}

}  // namespace wise
