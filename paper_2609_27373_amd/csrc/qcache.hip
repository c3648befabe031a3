// qcache.hip — tokens' keys and values into and out of a paged cache that holds them in 8
// or 4 bits (kept.hpp).
//
// A scale is the least power of two 2^e under which the largest magnitude a of its 32 dims
// is off by at most half a step: a <= T 2^e with T = 7 for 4 bits, whose largest code is 6 and
// whose last step is 2, and T = 464 for 8 (448 and 32).  Values go to the nearest
// code, ties to even, which the conversions of the hardware do.  a, T and e come from the bits of
// the bf16 values, so that nothing is rounded twice.
#include <type_traits>

#include "kept.hpp"
#include "plan.hpp"
#include "wise_kernels.hpp"

namespace wise {
namespace {

__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {   // of two 16-bit numbers each
  typedef uint16_t U2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(U2, a), __builtin_bit_cast(U2, b)));
}
template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max_pair(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kCtrl, 0xF, 0xF, true));
}

// Scale byte for a largest magnitude of the given bits: e from a <= T 2^e, within the exponents that
// leave every product of a code and the scale normal in bf16; 255 if the bits are of an infinite value or NaN.  Zeros
// take 2^0: the least scale would send the attention that reads them the longer way.
template <int B>
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  const int e = B == 4 ? (((int)a + 31) >> 7) - 2 : (((int)a + 23) >> 7) - 8;
  return a >= 0x7f80 ? 255 : a == 0 ? 127 : B == 4 ? min(max(e, 2), 252) : min(max(e, 10), 246);
}

// A lane's share of a token: D / 16 consecutive dims.
template <int D>
struct Dims {
  uint32_t w[D / 32];
  __device__ __forceinline__ void load(const uint16_t* p) {
    if constexpr (D == 128) {
      const u32x4_t x = *(const u32x4_t*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else if constexpr (D == 96) {
      typedef uint32_t W3 __attribute__((ext_vector_type(3), aligned(4)));
      const W3 x = *(const W3*)p;
#pragma unroll
      for (int i = 0; i < 3; ++i) w[i] = x[i];
    } else {
      const u32x2_t x = *(const u32x2_t*)p;
      w[0] = x[0], w[1] = x[1];
    }
  }
  __device__ __forceinline__ void store(uint16_t* p) const {
    if constexpr (D == 128) {
      __builtin_nontemporal_store(u32x4_t{w[0], w[1], w[2], w[3]}, (u32x4_t*)p);
    } else if constexpr (D == 96) {
      typedef uint32_t W3 __attribute__((ext_vector_type(3), aligned(4)));
      __builtin_nontemporal_store(W3{w[0], w[1], w[2]}, (W3*)p);
    } else {
      __builtin_nontemporal_store(u32x2_t{w[0], w[1]}, (u32x2_t*)p);
    }
  }
};

// The bytes of a lane's share of one token: kPiece / 4 of them, in words.
template <int D, int B>
struct Share {
  static constexpr int kBytes = D * B / 128, kWords = (kBytes + 3) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void store(uint8_t* p) const {
    if constexpr (kBytes == 8) {
      *(u32x2_t*)p = u32x2_t{w[0], w[1]};
    } else if constexpr (kBytes == 4) {
      *(uint32_t*)p = w[0];
    } else {                                        // 2, 3 or 6 bytes
      if constexpr (kBytes == 3) {
        p[0] = (uint8_t)w[0], p[1] = (uint8_t)(w[0] >> 8), p[2] = (uint8_t)(w[0] >> 16);
      } else {
#pragma unroll
        for (int i = 0; i < kBytes / 2; ++i) *(uint16_t*)(p + 2 * i) = (uint16_t)(w[i / 2] >> 16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kBytes == 8) {
      const u32x2_t x = *(const u32x2_t*)p;
      w[0] = x[0], w[1] = x[1];
    } else if constexpr (kBytes == 4) {
      w[0] = *(const uint32_t*)p;
    } else if constexpr (kBytes == 3) {
      w[0] = p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16;
    } else {
      const uint16_t* h = (const uint16_t*)p;
      w[0] = h[0];
      if constexpr (kBytes == 6) w[0] |= (uint32_t)h[1] << 16, w[1] = h[2];
    }
  }
};

// Quantises the shares that the 16 lanes of a row hold of one token: codes and, per pair of
// dims, the byte of the scale that it lies in.  sub: the lane's place in the row.
template <int D, int B>
__device__ __forceinline__ void quantise(const Dims<D>& x, int sub, Share<D, B>& out, uint32_t scale[D / 32]) {
  constexpr int kPairs = D / 32;
  uint32_t a[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) a[i] = x.w[i] & 0x7fff7fffu;
  if constexpr (D == 96) {
    // Pair i of lane n lies in scale (6 n + 2 i) / 32: three maxima over the row.
    uint32_t m[3];
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      m[s] = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if ((6 * sub + 2 * i) / 32 == s) m[s] = max_pair(m[s], a[i]);
      m[s] = max_dpp<0xB1>(m[s]);
      m[s] = max_dpp<0x4E>(m[s]);
      m[s] = max_dpp<0x141>(m[s]);
      m[s] = max_dpp<0x140>(m[s]);
      m[s] = scale_byte<B>(max(m[s] & 0xffff, m[s] >> 16));
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int s = (6 * sub + 2 * i) / 32;
      scale[i] = s == 0 ? m[0] : s == 1 ? m[1] : m[2];
    }
  } else {
    uint32_t m = max_pair(a[0], a[1]);
    if constexpr (D == 128) m = max_pair(m, max_pair(a[2], a[3]));
    m = max_dpp<0xB1>(m);                           // quad_perm [1,0,3,2], [2,3,0,1]: four lanes
    m = max_dpp<0x4E>(m);
    if constexpr (D == 64) m = max_dpp<0x141>(m);   // row_half_mirror: eight
    m = scale_byte<B>(max(m & 0xffff, m >> 16));
#pragma unroll
    for (int i = 0; i < kPairs; ++i) scale[i] = m;
  }
#pragma unroll
  for (int i = 0; i < Share<D, B>::kWords; ++i) out.w[i] = 0;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    uint32_t v = x.w[i];
    // Past 448 * 2^119 the conversion to 8 bits has no number, and what is NaN has code 0.
    if constexpr (B == 8) v = (v & 0x80008000u) | min_pair(v & 0x7fff7fffu, 0x7f607f60u);
    if (scale[i] == 255) v = 0;
    const float s = scale_of(scale[i] == 255 ? 127 : scale[i], 0);
    const float lo = __builtin_bit_cast(float, v << 16), hi = __builtin_bit_cast(float, v & 0xffff0000u);
    if constexpr (B == 4) {
      const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, lo, hi, s, 0) & 255;
      out.w[i / 4] |= c << 8 * (i % 4);
    } else {
      typedef short S2 __attribute__((ext_vector_type(2)));
      const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(S2{}, lo, hi, s, false)) & 0xffff;
      out.w[i / 2] |= c << 16 * (i % 2);
    }
  }
}

// Bytes before a head's page in a plane, for position pos of sequence s; -1: nowhere.
__device__ __forceinline__ int64_t page_of(const Cache& c, const int32_t* tables, int s, int64_t pos, int h, int page_bytes) {
  if (pos < 0 || pos >= (int64_t)c.max_pages * c.page) return -1;
  const int p = tables[(size_t)s * c.max_pages + (uint32_t)pos / (uint32_t)c.page];
  return in_range(p, c.pages) ? ((int64_t)p * c.kv_heads + h) * page_bytes : -1;
}

// ---------------------------------------------------------------------------
// Append, and the way back.  16 lanes take the tokens of one entry and head that lie in one four of
// positions, K and V: the unit in which values are laid out, so a store of four tokens' values, as of each key, is
// consecutive in the lanes, and a lane has up to eight loads of 16 bytes in flight.  A maximum over 32 dims is two or
// three steps over the lanes.  Bound by HBM: 8 prompts of up to 4K tokens, 6 layers of 8 heads of 128 in 4 bits, 1285 MB
// written and read back in 274 us (4.7 TB/s, the rate of a large copy); 32 histories of up to 8K read, 670 MB in
// 133 us (5.0 TB/s).  Few tokens: 3.3 us on the device, 8 from Python.
// ---------------------------------------------------------------------------
struct Four {                          // the lanes' share of the work
  uint32_t entry, head;
  int64_t at;                          // first position of the four
  int sub;
};

__device__ __forceinline__ bool my_four(const Cache& c, int n, int fours, Four& f, uint32_t& which) {
  const uint32_t x = blockIdx.x * 16 + (threadIdx.x >> 4);
  const uint32_t eh = x / (uint32_t)fours;
  which = x - eh * fours;
  f.entry = eh / (uint32_t)c.kv_heads;
  f.head = eh - f.entry * c.kv_heads;
  f.sub = threadIdx.x & 15;
  return f.entry < (uint32_t)n;
}

template <int D, int B>
__global__ void __launch_bounds__(256)
qappend_kernel(Cache c, int n, int tokens, int fours, const int32_t* __restrict__ ids, const int32_t* __restrict__ counts,
               const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, const int32_t* __restrict__ tables,
               const int32_t* __restrict__ lens, uint8_t* kp, uint8_t* vp) {
  using L = Kept<D, B>;
  using S = Share<D, B>;
  Four f;
  uint32_t which;
  if (!my_four(c, n, fours, f, which)) return;
  const int s = ids[f.entry], count = min(max(counts[f.entry], 0), tokens);
  if (!in_range(s, c.seqs)) return;
  const int64_t first = (int64_t)lens[s] - count;   // may lie below 0
  f.at = (first & ~(int64_t)3) + 4 * (int64_t)which;
  const int64_t t0 = f.at - first;                  // the four's first token, -3 .. count
  if (t0 >= count) return;
  const int page_bytes = c.page * (L::kRow + L::kScales);
  const int64_t page = page_of(c, tables, s, f.at, f.head, page_bytes);
  if (page < 0) return;
  const size_t from = ((size_t)(f.entry * (size_t)c.kv_heads + f.head) * tokens) * D + D / 16 * f.sub;
  Dims<D> x[2][4];
  bool live[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    live[e] = t0 + e >= 0 && t0 + e < count;
    if (live[e]) {
      x[0][e].load(k + from + (t0 + e) * D);
      x[1][e].load(v + from + (t0 + e) * D);
    } else {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) x[0][e].w[i] = x[1][e].w[i] = 0;
    }
  }
  const int t = (int)f.at & (c.page - 1);
  // The first lane of those that a scale covers writes it.
  const int mine = (D / 16 * f.sub + D / 16 - 2) / 32;
  const bool writes = D == 96 ? f.sub == 0 || f.sub == 5 || f.sub == 10 : D / 16 * f.sub % 32 == 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    S codes[2];
    uint32_t scale[2][D / 32];
    quantise<D, B>(x[0][e], f.sub, codes[0], scale[0]);
    quantise<D, B>(x[1][e], f.sub, codes[1], scale[1]);
    if (!live[e]) continue;
    uint8_t *kb = kp + page, *vb = vp + page;
    codes[0].store(kb + (t + e) * L::kRow + f.sub * S::kBytes);
    codes[1].store(vb + t * L::kRow + f.sub * L::kPiece + e * S::kBytes);
    if (writes) {
      kb[c.page * L::kRow + (t + e) * L::kScales + mine] = (uint8_t)scale[0][D / 32 - 1];
      vb[c.page * L::kRow + L::v_scale(t + e, mine)] = (uint8_t)scale[1][D / 32 - 1];
    }
  }
}

template <int D, int B>
__global__ void __launch_bounds__(256)
qread_kernel(Cache c, int n, int tokens, int fours, const int32_t* __restrict__ ids, const int32_t* __restrict__ counts,
             const int32_t* __restrict__ starts, const uint8_t* __restrict__ kp, const uint8_t* __restrict__ vp,
             const int32_t* __restrict__ tables, const int32_t* __restrict__ lens, uint16_t* k, uint16_t* v) {
  using L = Kept<D, B>;
  using S = Share<D, B>;
  Four f;
  uint32_t which;
  if (!my_four(c, n, fours, f, which)) return;
  const int s = ids[f.entry], count = min(max(counts[f.entry], 0), tokens);
  if (!in_range(s, c.seqs)) return;
  const int64_t first = starts ? starts[f.entry] : 0, len = lens[s];
  f.at = (first & ~(int64_t)3) + 4 * (int64_t)which;
  const int64_t t0 = f.at - first, end = min((int64_t)count, len - first);
  if (t0 >= end) return;
  const int page_bytes = c.page * (L::kRow + L::kScales);
  const int64_t page = page_of(c, tables, s, f.at, f.head, page_bytes);
  if (page < 0) return;
  const int t = (int)f.at & (c.page - 1);
  const uint8_t *kb = kp + page, *vb = vp + page;
  S codes[2][4];
  uint32_t ks[4][D == 96 ? 2 : 1], vs[D == 96 ? 2 : 1];
  const int g0 = D / 16 * f.sub / 32, g1 = (D / 16 * f.sub + D / 16 - 2) / 32;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    codes[0][e].load(kb + (t + e) * L::kRow + f.sub * S::kBytes);
    codes[1][e].load(vb + t * L::kRow + f.sub * L::kPiece + e * S::kBytes);
    ks[e][0] = kb[c.page * L::kRow + (t + e) * L::kScales + g0];
    if constexpr (D == 96) ks[e][1] = kb[c.page * L::kRow + (t + e) * L::kScales + g1];
  }
  vs[0] = *(const uint32_t*)(vb + c.page * L::kRow + L::v_scale(t, g0));
  if constexpr (D == 96) vs[1] = *(const uint32_t*)(vb + c.page * L::kRow + L::v_scale(t, g1));
  const size_t to = ((size_t)(f.entry * (size_t)c.kv_heads + f.head) * tokens) * D + D / 16 * f.sub;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (t0 + e < 0 || t0 + e >= end) continue;
    Dims<D> x[2];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      uint32_t kw = ks[e][0], vw = vs[0];
      if constexpr (D == 96) {
        if ((6 * f.sub + 2 * i) / 32 == g1) kw = ks[e][1], vw = vs[1];
      }
      x[0].w[i] = widen_at<B>(codes[0][e].w, scale_of(kw, 0), i);
      x[1].w[i] = widen_at<B>(codes[1][e].w, scale_of(vw, e), i);
    }
    x[0].store(k + to + (t0 + e) * D);
    x[1].store(v + to + (t0 + e) * D);
  }
}

template <class Run>
hipError_t by_kind(int d, int bits, Run run) {
  using I4 = std::integral_constant<int, 4>;
  using I8 = std::integral_constant<int, 8>;
  const auto of = [&](auto dim) { return bits == 4 ? run(dim, I4{}) : run(dim, I8{}); };
  return d == 64   ? of(std::integral_constant<int, 64>{})
         : d == 96 ? of(std::integral_constant<int, 96>{})
                   : of(std::integral_constant<int, 128>{});
}

// Fours that `tokens` consecutive positions reach into, and the groups of all entries and heads.
int fours_of(int tokens) { return (int)(((int64_t)tokens + 6) / 4); }
unsigned four_groups(const Cache& c, int n, int fours) { return (unsigned)(((int64_t)n * c.kv_heads * fours + 15) / 16); }

}  // namespace

hipError_t launch_qcache_append(const Cache& c, int bits, int n, int tokens, const int32_t* ids, const int32_t* counts, const void* k,
                                const void* v, const int32_t* tables, const int32_t* lens, void* kp, void* vp, hipStream_t st) {
  const int fours = fours_of(tokens);
  return by_kind(c.head_dim, bits, [&](auto d, auto b) {
    qappend_kernel<decltype(d)::value, decltype(b)::value><<<four_groups(c, n, fours), 256, 0, st>>>(
        c, n, tokens, fours, ids, counts, (const uint16_t*)k, (const uint16_t*)v, tables, lens, (uint8_t*)kp, (uint8_t*)vp);
    return hipGetLastError();
  });
}

hipError_t launch_qcache_read(const Cache& c, int bits, int n, int tokens, const int32_t* ids, const int32_t* counts, const int32_t* starts,
                              const void* kp, const void* vp, const int32_t* tables, const int32_t* lens, void* k, void* v, hipStream_t st) {
  const int fours = fours_of(tokens);
  return by_kind(c.head_dim, bits, [&](auto d, auto b) {
    qread_kernel<decltype(d)::value, decltype(b)::value><<<four_groups(c, n, fours), 256, 0, st>>>(
        c, n, tokens, fours, ids, counts, starts, (const uint8_t*)kp, (const uint8_t*)vp, tables, lens, (uint16_t*)k, (uint16_t*)v);
    return hipGetLastError();
  });
}

}  // namespace wise
