// qprefix.hip — attention of a batch's newest tokens over a paged cache whose keys and
// values are held in 8 or 4 bits (the causal attention of the paper's Section 3, eq.
// recurrent_attention, over what is kept of them).  The plan, the pieces and their
// join are those of the cache in bf16 (prefix_plan.hpp); here is a piece of work.
//
// What is kept is exact in bf16 (a code has at most 4 significant bits, the scale is a
// power of two), so each key is widened to bf16 in a register, two values an instruction, right before
// the matrix cores take it, and a score is as exact as with keys in bf16.  Values are widened to fp16 where that
// is exact too, which their scales tell (past_half), and meet probabilities of 11 bits in one MFMA: o is off by
// 2^-12 of sum p |v| at most beside its own rounding of 2^-8, and measures 0.16 to 0.17% rms from its definition as
// with exact probabilities.  Else, and where a row's reference is past kHalfReach, both are bf16 and a probability is two numbers
// (split_bf16x2), an MFMA more.  Two everywhere would take 32 sequences of up to 8K tokens from 42 to 43 us, 128 over a 32K document from
// 150 to 190 in 4 bits and from 183 to 277 in 8.
#include "kept.hpp"
#include "prefix_plan.hpp"

namespace wise {
namespace {

// Whether every sequence is one piece, which saves the plan and the join, 7 to 10 us, and reads shared pages once for each.
// By the tokens of a table (what a sequence can hold) and the groups G that this gives, us a call cut and whole,
// 8 heads of 128 in 4 bits:
//   nothing shared: up to 2048 always.  1 x 640 12.8 and 8.7, 32 x 1536 23.5 and 15.4, 48 x 2048 27.5 and 22.1, 1 x 2048 15.5
//     and 16.0; up to 2560 with G of 192 to 1024, which fill the chip without ending one by one
//   shared: up to 2048 while whole tables are at most 2^20 keys of a head, and 144 MB: 64 over 576 21.0 and 11.3, 32 over 1984
//     22.2 and 16.6, 64 over 1984 24.1 and 22.0; not 128 over 1472, 28.0 and 32.4, nor 256 over 960, 36 and 47, nor 76 over 576 with
//     15 heads in 8 bits, 183 MB, 24.5 and 28.9
constexpr int kWholeMore = 2048, kWholeMost = 2560, kWholeFew = 192, kWholeMany = 1024;
constexpr int64_t kWholeShared = 1 << 20, kWholeBytes = 144 << 20;

bool never_cut(const Cache& c, const Queries& a, bool shared, int64_t tiles, int key_bytes) {
  const int64_t keys = (int64_t)c.max_pages * c.page, groups = a.batch * tiles * c.kv_heads;
  if (shared) return keys <= kWholeMore && groups * keys <= kWholeShared && groups * keys * key_bytes <= kWholeBytes;
  return keys <= kWholeMore || (keys <= kWholeMost && groups >= kWholeFew && groups <= kWholeMany);
}

// ---------------------------------------------------------------------------
// A piece of up to R rows (8, 16, 32).  A wave takes every fourth tile of 32 keys (S^T = K Q^T and
// O^T = V^T P^T in 16x16x32 MFMAs, queries in columns).  The sums may run in
// any order, which the layout uses twice:
//   K  lane (n, g), g = lane / 16, loads the quarter g of key n's dims, D / 4 of
//      them; eight at a time are its slice of the A operand, and of Q it holds the same dims
//   V  the scores end up as keys 4 g .. 4 g + 3 of each 16-key half at one query, which is
//      a slice of the B operand as it stands; the lane loads the same four tokens at dims
//      (D / 16) n .., widens a pair of dims of all eight keys, and two permutes a register make the A
//      operands of two MFMAs, row m of the t-th being dim (D / 16) m + t
// Of up to 8 rows the 16 columns hold each twice, and the second half of the columns does the softmax of the second 16
// keys: half the exponentials (1%).  kTilesAhead tiles are in flight in registers; more did no
// better (one of 128K tokens: 44 us with two, 45 with three, 46 with four), nor did three waves a SIMD instead of two (45).
// Bound by HBM while tiles run, 1.05 us a tile of 32 keys of 128 in 4 bits with 2048 waves at work (8.5 TB/s, part of it from
// the last-level cache).  A call has 10 to 15 us beside that: launch, plan (2 to 4), a piece's page ids and first
// tiles (3.5), its join (1), the join of pieces (5).
// Keys in 4 bits are loaded past the L2 (32 x 8K 39.8 -> 37.4 us, 128 x up to 4K 68.7 -> 65.2); in 8 bits a lane's bytes take
// two loads that meet a line twice (128 x up to 4K 111 -> 120), and values past it lose where the last-level cache holds
// a call's (8 samples of 4K 27 -> 29).
// ---------------------------------------------------------------------------
template <int D, int B, int NT>
constexpr int kTilesAhead = NT == 2 && D * B > 384 ? 1 : 2;   // registers hold no more in tiles of 32 rows

template <int D, int B>
struct Raw {                           // a lane's share of a tile of 32 keys
  uint32_t k[2][Kept<D, B>::kWords], v[2][Kept<D, B>::kWords];
  uint32_t ks[2][D == 96 ? 2 : 1], vs[2][D == 96 ? 2 : 1];
  int64_t at[2];                       // bytes of a plane before the half's codes
  int apart[2];                        // and from there to its scales
  bool ok[2];                          // the half has a page
};

// Puts NaN into dims d .. d + 3 of a row's values where a key that it sees has NaN.
template <int D, int B>
__device__ __forceinline__ void put_nan(const Args& x, const int32_t* table, int kh, int k0, int end, int d, f32x4_t& o) {
  using L = Kept<D, B>;
  const int page = x.c.page;
#pragma unroll 1
  for (int key = k0; key < end; ++key) {
    const int id = table[key >> x.page_bits], t = key & (page - 1);
    if (!in_range(id, x.c.pages)) continue;
    const uint8_t* v = (const uint8_t*)x.vp + ((size_t)id * x.c.kv_heads + kh) * (page * (L::kRow + L::kScales));
    const bool all = v[page * L::kRow + L::v_scale(t, d / 32)] == 255;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (all || (B == 8 && (v[L::v_code(t, d + i)] & 127) == 127)) o[i] = __builtin_nanf("");
  }
}

// What a row's exponents are taken against when its largest score becomes mx: `low` below it, or, from 2^24 on, where fp32's
// steps are too large for that, the number at or next below it: mx has then a probability from 1 up to 2^(a step).  From 2^30 on that
// may be infinite, and is taken as kFarMost: what is less than a step apart there has equal weights.
constexpr float kFarMost = 0x1p64f;
__device__ __forceinline__ float reference(float mx, float sc, float low) {
  const float s = mx * sc;
  if (__builtin_fabsf(s) < 0x1p24f) return s - low;
  const int bits = __builtin_bit_cast(int, s);
  return __builtin_fmaf(mx, sc, -s) < 0.f ? __builtin_bit_cast(float, s > 0.f ? bits - 1 : bits + 1) : s;
}

// threadIdx.x, unknown to the compiler, which would else keep what a piece computes from it
// over the loop over pieces.
__device__ __forceinline__ int fresh_tid() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

// A constant in a scalar register, unknown to the compiler, which would else keep it in vector registers over the loop over
// pieces (infinities among 16 of them, spilled, and read back for each tile with a mask).
__device__ __forceinline__ float scalar(float c) {
  asm volatile("" : "+s"(c));
  return c;
}

// The kernel's argument where the hardware has put it, unknown to the compiler, which would else keep what it has read of it,
// for every kind of piece at once, and spill scalars inside their loops.
__device__ __forceinline__ const Args& fresh_args() {
  auto p = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Args*)p;
}

template <int D, int B, int R, bool kAlone>
__device__ __forceinline__ void stream_piece(const Args& x, const Piece& p, float* lds) {
  using L = Kept<D, B>;
  constexpr int NT = (R + 15) / 16;
  constexpr bool kPack = R == 8;
  constexpr int kC = D / 32, kT = D / 16, kStride = D + 4, kRows = 16 * NT, kS = kPack ? 4 : 8, kWords = L::kWords, kAhead = kTilesAhead<D, B, NT>;
  const int tid = fresh_tid(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int rows = x.rows, page = x.c.page;
  // The four waves share the piece, or (kAlone) each has its own, of the next head.
  constexpr int stride = kAlone ? 32 : 128;
  const int begin = p.k0 + (kAlone ? 0 : 32 * wave);
  const int my_head = kAlone ? 4 * p.head + wave : p.head, kh = min(my_head, x.c.kv_heads - 1);
  const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
  u32x4_t qf[NT][kC];
  int see[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const int r = p.row0 + min(kPack ? n & 7 : 16 * u + n, p.rows - 1);
    const int b = p.first + r / rows, w = r % rows;
    see[u] = min(p.see + w % x.a.q_len, p.k1);
    const uint16_t* row = x.q + (((size_t)b * x.c.kv_heads + kh) * rows + w) * D + D / 4 * g;
#pragma unroll
    for (int i = 0; i < kC; ++i) qf[u][i] = *(const u32x4_t*)(row + 8 * i);
  }
  const int least = min(p.see, p.k1);              // every row sees the keys below
  f32x4_t o[NT][kT];
  float m[NT], l[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    m[u] = scalar(-INFINITY);
    l[u] = 0.f;
#pragma unroll
    for (int t = 0; t < kT; ++t) o[u][t] = f32x4_t{};
  }
  // Where the halves of this wave's tiles lie in a plane: lane 2 i + s has the bytes before half s of tile i (mod 32), -1
  // for no page.
  const int tiles = my_head < x.c.kv_heads ? (p.k1 - begin + stride - 1) / stride : 0;
  const int page_bytes = page * (L::kRow + L::kScales);
  int64_t halves = -1;
  auto load_ids = [&](int i0) {
    const int key = begin + stride * (i0 + (lane >> 1)) + 16 * (lane & 1);
    const int id = key < p.k1 ? table[key >> x.page_bits] : -1;
    halves = in_range(id, x.c.pages) ? ((int64_t)id * x.c.kv_heads + kh) * page_bytes + (key & (page - 1)) * L::kRow : -1;
  };
  const int k_code = (4 * n + g) * L::kPiece, v_code = lane * L::kPiece;
  const int k_scale = n * L::kScales + D / 4 * g / 32, k_last = n * L::kScales + (D / 4 * g + D / 4 - 8) / 32;
  const int v_scale = 4 * (g * L::kScales + D / 16 * n / 32), v_last = 4 * (g * L::kScales + (D / 16 * n + D / 16 - 2) / 32);
  const char *kp = (const char*)x.kp, *vp = (const char*)x.vp;
  Raw<D, B> raw[kAhead];
  auto load_k = [&](int i, Raw<D, B>& w) {
    if ((i & 31) == 0) load_ids(i);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int lo = __builtin_amdgcn_readlane((int)halves, 2 * (i & 31) + s), hi = __builtin_amdgcn_readlane((int)(halves >> 32), 2 * (i & 31) + s);
      w.ok[s] = hi >= 0;
      w.at[s] = w.ok[s] ? (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo) : 0;
      // Of the page's scales, those of token t are (kRow - kScales) t bytes nearer than its codes.
      w.apart[s] = page * L::kRow - ((begin + stride * i + 16 * s) & (page - 1)) * (L::kRow - L::kScales);
      const char* codes = kp + w.at[s];
      uint32_t at = k_code;                           // NT = 2: its 64 bits anew, which the compiler would else spill
      if constexpr (NT == 2) asm volatile("" : "+v"(at));
      load_words<kWords, B == 4>(codes + at, w.k[s]);
      w.ks[s][0] = *(const uint8_t*)(codes + (uint32_t)(w.apart[s] + k_scale));
      if constexpr (D == 96) w.ks[s][1] = *(const uint8_t*)(codes + (uint32_t)(w.apart[s] + k_last));
    }
  };
  auto load_v = [&](Raw<D, B>& w) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const char* codes = vp + w.at[s];
      uint32_t at = v_code;
      if constexpr (NT == 2) asm volatile("" : "+v"(at));
      load_words<kWords>(codes + at, w.v[s]);
      w.vs[s][0] = *(const uint32_t*)(codes + (uint32_t)(w.apart[s] + v_scale));
      if constexpr (D == 96) w.vs[s][1] = *(const uint32_t*)(codes + (uint32_t)(w.apart[s] + v_last));
    }
  };
  // Past its last tile a wave loads what page 0 holds, which nothing uses.
  if (tiles > 0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      load_k(i, raw[i]);
      load_v(raw[i]);
    }
  }
  int poisoned = 0x7fffffff;                        // first key of the first tile that had NaN values set aside
  auto tile = [&](int i, Raw<D, B>& w) {
    const int key0 = begin + stride * i;
    const bool ok0 = w.ok[0], ok1 = w.ok[1];
    const bool masked = key0 + 32 > least || !ok0 || !ok1;
    f32x4_t s[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int u = 0; u < NT; ++u) s[u][h] = f32x4_t{};
#pragma unroll
      for (int e = 0; e < kC; ++e) {
        // At D = 96 quarter 1 begins in the scale before that of its other dims, quarter 2 ends in the one behind.
        const uint32_t byte = D != 96 || e == 0 ? w.ks[h][0] : e == 2 || g == 1 ? w.ks[h][D == 96] : w.ks[h][0];
        const float scale = scale_of(byte, 0);
        u32x4_t f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = widen_at<B>(w.k[h], scale, 4 * e + j);
#pragma unroll
        for (int u = 0; u < NT; ++u) s[u][h] = mfma16x16x32(f, qf[u][e], s[u][h]);
      }
    }
    load_k(i + kAhead, w);
    // kPack: the half of the columns that repeats the queries takes the scores of the second 16 keys.
    float y[NT][kS];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int r = 0; r < kS; ++r) y[u][r] = kPack ? (n < 8 ? s[u][0][r] : s[u][1][r]) : s[u][r >> 2][r & 3];
    if (masked) {
      const float none = scalar(-INFINITY);
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int r = 0; r < kS; ++r) {
          const bool second = kPack ? n >= 8 : r >= 4;
          if (key0 + (second ? 16 : 0) + 4 * g + (r & 3) >= see[u] || !(second ? ok1 : ok0)) y[u][r] = none;
        }
      // Values that no row sees may be anything, and NaN must not reach the rows that don't see
      // it (0 * NaN is NaN): they count as 0 or as some number, and the rows that see NaN get it at the end.
      uint32_t poison = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = (h ? ok1 : ok0) ? min(max(p.k1 - (key0 + 16 * h + 4 * g), 0), 4) : 0;
        const uint32_t keep = low_bytes(left);
#pragma unroll
        for (int j = 0; j < (D == 96 ? 2 : 1); ++j) {
          const uint32_t bad = nan_bytes<false>(w.vs[h][j] & keep);
          poison |= bad;
          w.vs[h][j] = (w.vs[h][j] & keep & ~bad) | (0x7f7f7f7fu & (~keep | bad));
        }
        if constexpr (B == 8) {
#pragma unroll
          for (int j = 0; j < kWords; ++j) {
            const uint32_t bad = nan_bytes<true>(w.v[h][j]);
            poison |= bad & low_bytes(left * (D / 16) - 4 * j);   // those of tokens behind the last one are nobody's
            w.v[h][j] &= ~bad;
          }
        }
      }
      if (__builtin_amdgcn_ballot_w64(poison != 0)) poisoned = min(poisoned, key0);
    }
    uint32_t far = 0;                                 // a scale is past what fp16 holds
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < (D == 96 ? 2 : 1); ++j) far |= past_half<B>(w.vs[h][j]);
    bool half = __builtin_amdgcn_ballot_w64(far != 0) == 0, past = false;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      float mx = y[u][0];
#pragma unroll
      for (int r = 1; r < kS; ++r) mx = fmaxf(mx, y[u][r]);
      // The reference of the exponents is raised as kProbHalf says, not for each new maximum; where values are not in fp16 for
      // each, since a weight above 1 could take their sum out of fp32's range.
      if (!half || __builtin_amdgcn_ballot_w64(mx * x.sc > m[u] + kHalfTop)) {
        const float top = half ? kHalfTop : 0.f, low = half ? kHalfLow : 0.f;
        if constexpr (kPack) mx = fmaxf(mx, dpp_mov<0x128>(mx));   // row_ror 8
        mx = quad_max(mx);
        const bool grow = mx * x.sc > m[u] + top;
        const float mn = grow ? reference(mx, x.sc, low) : m[u];
        const float alpha = grow ? fast_exp2(m[u] - mn) : 1.f;
        l[u] *= alpha;
#pragma unroll
        for (int t = 0; t < kT; ++t)                 // in place, as in WaveRows::softmax
#pragma unroll
          for (int r = 0; r < 4; ++r) asm volatile("v_mul_f32 %0, %0, %1" : "+v"(o[u][t][r]) : "v"(alpha));
        m[u] = mn;
      }
      const float mb = m[u] == -INFINITY ? 0.f : m[u];
      past |= __builtin_fabsf(mb) >= kHalfReach;
#pragma unroll
      for (int r = 0; r < kS; ++r) y[u][r] = fast_exp2(__builtin_fmaf(y[u][r], x.sc, -mb));
    }
    if (__builtin_amdgcn_ballot_w64(past)) {
      half = false;
      const float most = scalar(kFarMost);
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int r = 0; r < kS; ++r) y[u][r] = y[u][r] > most ? most : y[u][r];
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      float ts = 0.f;
#pragma unroll
      for (int r = 0; r < kS; ++r) ts += y[u][r];
      l[u] += ts;
    }
    // Values in fp16 and probabilities with 11 bits where that is exact for the values, else both in bf16 and the
    // probabilities as two numbers.
    auto weigh = [&](auto in_half) {
      constexpr bool kHalf = decltype(in_half)::value;
      u32x4_t pb[NT], pr[NT];
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int j = 0; j < kS / 2; ++j) {
          if constexpr (kHalf) {
            pb[u][j] = pack_f16x2(y[u][2 * j], y[u][2 * j + 1]);
          } else {
            uint32_t rest;
            pb[u][j] = split_bf16x2(y[u][2 * j], y[u][2 * j + 1], rest);
            pr[u][j] = rest;
            if constexpr (kPack) pr[u][2 + j] = (uint32_t)__builtin_amdgcn_mov_dpp((int)rest, 0x128, 0xF, 0xF, true);
          }
          if constexpr (kPack) pb[u][2 + j] = (uint32_t)__builtin_amdgcn_mov_dpp((int)pb[u][j], 0x128, 0xF, 0xF, true);
        }
#pragma unroll
      for (int b = 0; b < L::kPairs; ++b) {
        uint32_t v[8];                              // the pair of dims of all keys
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t sw = w.vs[e >> 2][0];
          if constexpr (D == 96) sw = b == 2 || (b == 1 && n == 5) ? w.vs[e >> 2][1] : sw;   // pair 1 of piece 5 lies in the next scale
          v[e] = widen_at<B, kHalf>(w.v[e >> 2], scale_of(sw, e & 3), (e & 3) * L::kPairs + b);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32x4_t f;
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], c ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            f32x4_t& to = o[u][2 * b + c];
            if constexpr (kHalf) to = mfma16x16x32_f16(f, pb[u], to);
            else to = mfma16x16x32(f, pr[u], mfma16x16x32(f, pb[u], to));
          }
        }
      }
    };
    if (half) weigh(std::true_type{});
    else weigh(std::false_type{});
    load_v(w);
  };
  for (int i = 0; i < tiles; i += kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= tiles) break;
      tile(i + j, raw[j]);
    }
  }
  // Join the waves.
  float* mls = lds + 4 * kRows * kStride;
  int32_t* first = (int32_t*)(mls + 8 * kRows);     // the waves' `poisoned`
  __syncthreads();
  if (lane == 0) first[wave] = poisoned;
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    float lt = quad_sum(l[u]);
    if constexpr (kPack) lt += dpp_mov<0x128>(lt);
    const int r = wave * kRows + 16 * u + n;
    if (g == 0) {
      mls[2 * r] = m[u];
      mls[2 * r + 1] = lt;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < kT; t += 2) *(f32x2_t*)(lds + r * kStride + kT * (4 * g + i) + t) = f32x2_t{o[u][t][i], o[u][t + 1][i]};
  }
  __syncthreads();
  poisoned = __builtin_amdgcn_readfirstlane(min(min(first[0], first[1]), min(first[2], first[3])));
  if (my_head >= x.c.kv_heads) return;
  for (int j = kAlone ? lane : tid; j < p.rows * (D / 4); j += kAlone ? 64 : 256) {
    const int r = j / (D / 4), d = j % (D / 4) * 4;
    const float none = scalar(-INFINITY);
    float mw[4], mx = none, lt = 0.f;
    f32x4_t sum{};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mw[w] = kAlone && w != wave ? none : mls[2 * (w * kRows + r)];
      mx = fmaxf(mx, mw[w]);
    }
    const float mb = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (kAlone && w != wave) continue;
      const float f = fast_exp2(mw[w] - mb);
      lt += f * mls[2 * (w * kRows + r) + 1];
      sum += f * *(const f32x4_t*)(lds + (w * kRows + r) * kStride + d);
    }
    if (poisoned < p.k1) put_nan<D, B>(x, table, kh, poisoned, min(p.see + (p.row0 + r) % rows % x.a.q_len, p.k1), d, sum);
    if (p.slot >= 0) {
      const size_t at = (size_t)p.slot + (size_t)kh * p.seg_rows + p.row0 + r;
      *(f32x4_t*)(x.part + at * D + d) = sum;
      if (d == 0) x.ml[at] = float2{mx, lt};
    } else {
      const size_t at = ((size_t)p.first * x.c.kv_heads + kh) * rows + p.row0 + r;
      const float inv = lt == 0.f ? 0.f : 1.f / lt;
      *(u32x2_t*)(x.o + at * D + d) = u32x2_t{pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
      if (d == 0 && x.lse != nullptr) x.lse[at] = lt == 0.f ? none : (mx + __builtin_log2f(lt)) * kLn2;
    }
  }
}

// This lane's half of its row of Q in a piece of many rows.
template <int D>
__device__ __forceinline__ const uint16_t* tile_query(const Args& x, const Piece& p, int wave, int lane) {
  const int r = p.row0 + min(32 * wave + (lane & 31), p.rows - 1);
  const int b = p.first + r / x.rows;
  return x.q + (((size_t)b * x.c.kv_heads + p.head) * x.rows + r % x.rows) * D + 8 * (lane >> 5);
}

// Whether tile_piece can do a piece: all page ids name pages, fp16 holds its values by their scales, and no score
// is past kHalfReach by the largest scale of its keys and the largest number of Q.  A thread looks at four tokens at a time.
// Beside tile_piece, not in it, where the compiler kept what the two share in registers over the loop.  most: 4 words of LDS
// that tile_piece leaves alone.
template <int D, int B>
__device__ __forceinline__ bool tile_ready(const Args& x, const Piece& p, int32_t* most) {
  using L = Kept<D, B>;
  const int tid = fresh_tid(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int page = x.c.page;
  const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
  const uint16_t* row = tile_query<D>(x, p, wave, lane);
  u32x4_t q[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) q[i] = *(const u32x4_t*)(row + 16 * i);
  uint32_t bad = 0, k_most = 0, q_most = 0;         // q_most: bits of two numbers without their signs
  for (int t = p.k0 + 4 * tid; t < p.k1; t += 1024) {
    const int id = table[t >> x.page_bits], at = t & (page - 1);
    if (!in_range(id, x.c.pages)) {
      bad = 1;
      break;
    }
    const size_t scales = ((size_t)id * x.c.kv_heads + p.head) * (page * (L::kRow + L::kScales)) + page * L::kRow;
    const char *ks = (const char*)x.kp + scales + at * L::kScales, *vs = (const char*)x.vp + scales;
#pragma unroll
    for (int i = 0; i < L::kScales; ++i) {
      bad |= past_half<B>(*(const uint32_t*)(vs + L::v_scale(at, i)));
      const uint32_t k = *(const uint32_t*)(ks + 4 * i);
      k_most = max_pair(k_most, max_pair(k & 0xff00ff, k >> 8 & 0xff00ff));
    }
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) q_most = max_pair(q_most, q[i][j] & 0x7fff7fff);
  const auto larger = [](int x, int y) { return (int)max_pair((uint32_t)x, (uint32_t)y); };
  const int w = wave_scan((int)(max(q_most & 0xffff, q_most >> 16) | max(k_most & 0xffff, k_most >> 16) << 16), 0, larger);
  if (lane == 63) most[wave] = w;
  const int refused = __syncthreads_or(bad != 0);
  const uint32_t all = max_pair(max_pair(most[0], most[1]), max_pair(most[2], most[3]));
  const float top = x.sc * (D * (B == 4 ? 6.f : 448.f)) * __builtin_bit_cast(float, all << 16) * scale_of(all >> 16, 0);
  return __builtin_amdgcn_readfirstlane(!refused && top < kHalfReach);   // the same in every lane
}

// ---------------------------------------------------------------------------
// A piece of up to 128 rows, all of which see all its keys (whole tiles of 64): the
// pipeline of the dense kernel (WaveRows::step), four waves of 32 rows over rings of two K
// and two V tiles in LDS, in bf16: a wave widens 16 consecutive keys of a tile, which lie in one page, for
// all four, a tile ahead of their use, from registers that were loaded a step before.  Only where tile_ready says so.  Bound
// by the latency of two waves a SIMD and by VALU work: of some 600 instructions of two tiles of 64 keys of 128, 96 widen, 66 are exponentials
// and 128 rescale at need.  1.5 us a tile alone on a CU, 2.1 beside a group of few rows (512 rows over 32K tokens 108 us, 147 when
// 32 rows at a time were streamed).  Its loop takes all 256 registers at D = 128: the compiler spills 13 to 36 in these kernels, most of
// them at a piece's ends, one or two reads of them in the last slots of a step.
// ---------------------------------------------------------------------------
template <int D, int B>
__device__ __forceinline__ void tile_piece(const Args& x, const Piece& p, char* smem) {
  using L = Kept<D, B>;
  using G = Geo<D>;
  using S = Swizzle<D>;
  constexpr int kT = S::kTile, kC = D / 32, kWords = L::kWords;
  const int tid = fresh_tid(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int page = x.c.page;
  int kh = p.head;
  asm volatile("" : "+s"(kh));                      // in a scalar register: addresses computed with it are then scalars too
  const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
  const int tiles = (p.k1 - p.k0) / kKeyTile;
  // Page ids of this wave's keys: lane i has the one of tile 64 u + i, of stretch u and the next one.
  auto load_ids = [&](int u) {
    const int key = p.k0 + (64 * u + lane) * kKeyTile + 16 * wave;
    return key < p.k1 ? table[key >> x.page_bits] : 0;
  };
  int stretch = 0, ids = load_ids(0), next_ids = load_ids(1);
  WaveRows<D> w;
  w.reset();
  w.m = scalar(-INFINITY);
  {
    const uint16_t* row = tile_query<D>(x, p, wave, lane);
#pragma unroll
    for (int i = 0; i < G::kDChunks; ++i) w.qf[i] = *(const u32x4_t*)(row + 16 * i);
  }
  ReadAddr<D> ra;
  ra.init(lane);
  const int page_bytes = page * (L::kRow + L::kScales);
  const int k_code = (4 * n + g) * L::kPiece, v_code = lane * L::kPiece;
  const int k_scale = n * L::kScales + D / 4 * g / 32, k_last = n * L::kScales + (D / 4 * g + D / 4 - 8) / 32;
  const int v_scale = 4 * (g * L::kScales + D / 16 * n / 32), v_last = 4 * (g * L::kScales + (D / 16 * n + D / 16 - 2) / 32);
  uint32_t kw[kWords], vw[kWords], ks[2], vs[2];    // this wave's share of the tiles to be widened next
  auto source = [&](const uint16_t* pool, int it, const char*& scales) {
    const int id = __builtin_amdgcn_readlane(it >> 6 == stretch ? ids : next_ids, it & 63);
    const int t = (p.k0 + it * kKeyTile + 16 * wave) & (page - 1);
    const char* head = (const char*)pool + ((size_t)id * x.c.kv_heads + kh) * page_bytes;
    scales = head + page * L::kRow + t * L::kScales;
    return head + t * L::kRow;
  };
  auto load_k = [&](int it) {
    const char* scales;
    load_words<kWords>(source(x.kp, min(it, tiles - 1), scales) + k_code, kw);
    ks[0] = *(const uint8_t*)(scales + k_scale);
    if constexpr (D == 96) ks[1] = *(const uint8_t*)(scales + k_last);
  };
  auto load_v = [&](int it) {
    const char* scales;
    load_words<kWords>(source(x.vp, min(it, tiles - 1), scales) + v_code, vw);
    vs[0] = *(const uint32_t*)(scales + v_scale);
    if constexpr (D == 96) vs[1] = *(const uint32_t*)(scales + v_last);
  };
  // Eight dims of key n into the K tile; a token's dims into the V tile.
  const int k_row = k_lds_row(16 * wave + n);
  auto put_k = [&](char* tile, int e) {
    const uint32_t byte = D != 96 || e == 0 ? ks[0] : e == 2 || g == 1 ? ks[D == 96] : ks[0];
    u32x4_t f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = widen_at<B>(kw, scale_of(byte, 0), 4 * e + j);
    *(u32x4_t*)(tile + k_row * S::kRow + S::k_chunk(k_row, kC * g + e) * 16) = f;
  };
  auto put_v = [&](char* tile, int e) {
    const int row = 16 * wave + 4 * g + e, at = D / 8 * n;
    uint32_t f[D / 32];
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
      uint32_t sw = vs[0];
      if constexpr (D == 96) sw = b == 2 || (b == 1 && n == 5) ? vs[1] : vs[0];
      f[b] = widen_at<B, true>(vw, scale_of(sw, e), e * L::kPairs + b);
    }
    char* to = tile + row * S::kRow + S::v_block(row, at / 64) * 64 + at % 64;
    if constexpr (D == 128) *(u32x4_t*)to = u32x4_t{f[0], f[1], f[2], f[3]};
    else if constexpr (D == 64) *(u32x2_t*)to = u32x2_t{f[0], f[1]};
    else
#pragma unroll
      for (int b = 0; b < 3; ++b) *(uint32_t*)(to + 4 * b) = f[b];
  };
  char *sk = smem, *sv = smem + 2 * kT;
  auto put_all_k = [&](int it) {
#pragma unroll
    for (int e = 0; e < kC; ++e) put_k(sk + (it & 1) * kT, e);
  };
  load_k(0);
  load_v(0);
  put_all_k(0);
  if (tiles > 1) {
    load_k(1);
    put_all_k(1);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) put_v(sv, e);
  load_v(1);
  load_k(2);
  __syncthreads();
  const bool active = 32 * wave < p.rows;
  f32x16_t s0[2], s1[2];
  float mx = 0.f;
  if (active) w.template step<2, true, false, 0, kProbHalf>(sk, sv, ra, lane, x.sc, s1, s0, mx, [](auto, int) {}, [](f32x16_t*) {});
  __syncthreads();                                  // K(0) read by every wave: K(2) may take its place
  // Step `it`: S^T of tile it + 1, softmax and PV of tile it; V(it + 1) and K(it + 2)
  // go where V(it - 1) and K(it) were, and the words of the ones after them are loaded.
  auto fused = [&](int it, f32x16_t sc[2], f32x16_t sn[2]) {
    const int b = it & 1;
    if (it >> 6 != stretch) {
      stretch = it >> 6;
      ids = next_ids;
      next_ids = load_ids(stretch + 1);
    }
    const bool more = it + 2 < tiles;
    auto part = [&](int i) {                        // 4 + kC parts
      if (i < 4) put_v(sv + (b ^ 1) * kT, i);
      if (i == 3) load_v(it + 2);
      if (i >= 4 && more) put_k(sk + b * kT, i - 4);
      if (i == 3 + kC) load_k(it + 3);
    };
    if (active) {
      w.template step<2, true, true, 0, kProbHalf>(sk + (b ^ 1) * kT, sv + b * kT, ra, lane, x.sc, sc, sn, mx,
                                              [&](auto n, int j) {
                                                constexpr int kGap = (decltype(n)::value - 2) / (4 + kC);
                                                if (j >= 2 && (j - 2) % kGap == 0 && (j - 2) / kGap < 4 + kC) part((j - 2) / kGap);
                                              },
                                              [](f32x16_t*) {});
    } else {
#pragma unroll
      for (int i = 0; i < 4 + kC; ++i) part(i);
    }
    __syncthreads();
  };
  int it = 0;
  for (; it + 2 < tiles; it += 2) {
    fused(it, s0, s1);
    fused(it + 1, s1, s0);
  }
  if (it + 1 < tiles) {
    fused(it, s0, s1);
    s0[0] = s1[0];
    s0[1] = s1[1];
    ++it;
  }
  if (!active) return;
  w.template step<2, false, true, 0, kProbHalf>(sk, sv + (it & 1) * kT, ra, lane, x.sc, s0, s1, mx, [](auto, int) {}, [](f32x16_t*) {});
  const float lt = pair_sum(w.l);
  const int q = 32 * wave + (lane & 31), h = lane >> 5;
  if (q >= p.rows) return;
  const size_t at = (size_t)p.slot + (size_t)kh * p.seg_rows + p.row0 + q;
#pragma unroll
  for (int t = 0; t < G::kDTiles; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4_t*)(x.part + at * D + 32 * t + 8 * j + 4 * h) =
          f32x4_t{w.o[t][4 * j], w.o[t][4 * j + 1], w.o[t][4 * j + 2], w.o[t][4 * j + 3]};
  if (h == 0) x.ml[at] = float2{w.m, lt};
}

// Pieces of a group, at most: with 8 some calls had more groups than the chip holds at once, which planned in a second turn (64
// samples at 4 layers of 55 heads: 283 us a step, 260).
constexpr int kMine = 16;

template <int D, int B, int R, bool kShared>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
qpiece_kernel(Args x) {
  constexpr int kJoin = 4 * 16 * (kShared || R == 32 ? 2 : 1) * (D + 6) * 4 + 16, kRing = kShared ? 4 * Swizzle<D>::kTile + 16 : 0;
  __shared__ __attribute__((aligned(1024))) char smem[kJoin > kRing ? kJoin : kRing];
  static_assert(sizeof(Plan<256>) <= sizeof(smem), "the plan fits");
  __shared__ Piece todo[kMine];
  __shared__ int listed;
  __shared__ Shares shares;
  int count = my_pieces<kMine>(x, todo, &listed, smem, &shares);
  const bool even = x.mode == kOwnPlan && __builtin_amdgcn_readfirstlane(shares.used) > 0;
  for (;;) {
    if (even) {
      if (!share_pieces<kMine>(x, shares, todo)) return;
      count = kMine;
    }
    for (int i = 0; i < count; ++i) {
      Piece p = todo[i];
      int32_t* w = (int32_t*)&p;                   // the same in every lane
#pragma unroll
      for (int j = 0; j < 11; ++j) w[j] = __builtin_amdgcn_readfirstlane(w[j]);
      if (p.rows == 0) continue;
      if (i > 0) __syncthreads();                   // the piece before has left the LDS
      if (kShared && p.kind == kManyRows && tile_ready<D, B>(fresh_args(), p, (int32_t*)(smem + 4 * Swizzle<D>::kTile))) {
        tile_piece<D, B>(fresh_args(), p, smem);
        continue;
      }
      if (p.kind == kNarrow) {
        stream_piece<D, B, R, true>(fresh_args(), p, (float*)smem);
        continue;
      }
      Piece s = p;                                  // of shared pages it may have more rows: 32 at a time
      for (int r = 0; r < p.rows; r += 32) {
        if (r > 0) __syncthreads();
        s.row0 = p.row0 + r;
        s.rows = min(32, p.rows - r);
        if (R == 32 || (kShared && s.rows > R)) stream_piece<D, B, 32, false>(fresh_args(), s, (float*)smem);
        else stream_piece<D, B, R == 8 ? 8 : 16, false>(fresh_args(), s, (float*)smem);
      }
    }
    if (!even) return;
  }
}

template <int D, int B, int R>
hipError_t launch(const Args& x, hipStream_t st) {
  const int64_t rows = (int64_t)x.a.batch * x.a.heads * x.a.q_len;
  if (x.mode == kPlanned) {
    plan_kernel<<<1, kPlan, 0, st>>>(x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t pieces = (int64_t)x.most * x.c.kv_heads, hold = kHold;
  const unsigned grid = (unsigned)std::min(pieces, std::max(hold, (pieces + kMine - 1) / kMine));
  if (x.shared != nullptr) qpiece_kernel<D, B, R, true><<<grid, 256, 0, st>>>(x);
  else qpiece_kernel<D, B, R, false><<<grid, 256, 0, st>>>(x);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || x.mode == kWhole) return e;
  if (rows <= kFewJoins) join_kernel<D, 4><<<(unsigned)rows, 256, 0, st>>>(x, rows);
  else join_kernel<D, 1><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(x, rows);
  return hipGetLastError();
}

}  // namespace

size_t qprefix_workspace_bytes(const Cache& c, const Queries& a) { return space_bytes(c, a, nullptr, nullptr); }

hipError_t launch_qprefix(const Cache& c, int bits, const Queries& a, const void* q, const void* kp, const void* vp,
                          const int32_t* tables, const int32_t* lens, const int32_t* ids, const int32_t* shared, void* o, float* lse,
                          void* ws, hipStream_t st) {
  Args x = make_args(c, a, kept_key_bytes(c.head_dim, bits), never_cut, q, kp, vp, tables, lens, ids, shared, o, lse, ws);
  // Pieces are shorter work than in bf16, those of many rows the least so: a key to 128 rows takes three times one to few (128
  // over a 32K document 170 us dealt as equal, 159 as once, 145 as twice or more often), pieces of few rows may be longer, those of
  // many shorter (document 143 -> 137, 16 x 5 drafts 26.2 -> 25.7).
  x.wide_cost = 3;
  x.mid_keys = 1024, x.fill_all = 1, x.wide_keys = 512;
  // As many shares a head as give each group one, or two where that comes out evener.
  if (x.tiles == 1 && x.mode == kOwnPlan) {
    double best = 1e9;
    for (int turns = 1; turns <= 2; ++turns) {
      const int n = std::max(1, kHold * turns / c.kv_heads);
      const double cost = (double)((n * (int64_t)c.kv_heads + kHold - 1) / kHold) / n * (1 + 0.1 * turns);
      if (cost < best) best = cost, x.shares = n;
    }
  }
  const auto run = [&](auto d, auto b) {
    constexpr int D = decltype(d)::value, B = decltype(b)::value;
    return x.rows <= 8 ? launch<D, B, 8>(x, st) : x.tile == 16 ? launch<D, B, 16>(x, st) : launch<D, B, 32>(x, st);
  };
  const auto by_dim = [&](auto b) {
    return c.head_dim == 64   ? run(std::integral_constant<int, 64>{}, b)
           : c.head_dim == 96 ? run(std::integral_constant<int, 96>{}, b)
                              : run(std::integral_constant<int, 128>{}, b);
  };
  return bits == 4 ? by_dim(std::integral_constant<int, 4>{}) : by_dim(std::integral_constant<int, 8>{});
}

}  // namespace wise
