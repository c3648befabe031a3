// prefix.hip — attention of a batch's newest tokens over a paged key-value
// cache (the causal attention of the paper's Section 3, eq.
// recurrent_attention, with the keys and values of earlier positions kept),
// reading pages that sequences share once for all of them.
//
// A segment is a set of query rows that attend one range of keys: the shared
// pages of a run of sequences (all their rows), or the rest of one sequence (its own
// rows).  A row's result over a range of keys is (m, l, O): the running max and sum of its
// softmax, in base 2, and the sum of its values weighted with 2^(s - m).
// Results over disjoint ranges join as
//   m = max m_i,  l = sum l_i 2^(m_i - m),  O = sum O_i 2^(m_i - m),
// so segments are cut along the keys into as many pieces as fill the chip:
//   piece_kernel  finds the runs, cuts the segments, and does a few pieces a
//                 work-group: (m, l, O) in fp32
//   join_kernel   joins the pieces of every row, divides by l
//   plan_kernel   the runs and pieces of more than 256 sequences
// Rounded to fewer bits than 32: o, and the probabilities, to 16 bits: the matrix
// cores take them as V is, in bf16, so each goes in as two (split_bf16x2), with an MFMA
// more.  o then is as far from its definition as its own rounding puts it, 0.17% rms
// (0.20 to 0.23% with 8 bits), for 0.2 us in pieces of few rows, whose matrix cores
// are mostly idle, and up to a sixth of a call that pieces of many rows bound (87
// us instead of 75 at 28 x 5 drafts of 24 heads of 96 over 27K).
#include "prefix_plan.hpp"

namespace wise {
namespace {

// Whether every sequence is one piece, shared pages or not, which saves the plan and the
// join.  By the tokens of a table (what a sequence can hold) and the groups G that this gives:
//   up to 512: always, nothing shared.  1 x 301 tokens, 8 heads of 64: 12 -> 7.5 us; 1024 sequences of
//     512 tokens, 8 heads of 128: 194 -> 161.  Where they share 448 tokens, while the whole tables
//     are 256 MB of K and V: 64 x 8 heads of 128 17.2 -> 15.3, 256 x 8 of 64 28.2 -> 27.4; at the limit 128 x 8
//     of 128 21.0 -> 24.5 but 30.2 -> 25.4 at 256 x 8, 256 tokens; not 512 x 8 of 64: 36 -> 50, 1024 x 8 of 128: 66 -> 160
//   up to 1024, nothing shared, from 128 groups: 16 x 8 heads 21.4 -> 16.5, 32 x 8 24.7 -> 18.3 (10 x 55
//     32.9 -> 33.8); not 8 x 8: 15.1 -> 16.3, 1 x 8: 11.7 -> 14.2; shared, from 128 to 256
//     groups: 32 x 8 21.2 -> 16.2, 24 x 8 20.2 -> 15.6; not 64 x 8: 25.0 -> 25.4, 128 x 8: 34.0 -> 43.1
//   up to 2048, nothing shared, where G >= 512 fills its turns of 512 groups within 1.3 times: 250 x 8 117
//     -> 100, 200 x 8 181 -> 152, 24 x 55 114 -> 101; past 1.3 either may win: 20 x 55 92 -> 83, 131 x 8 105
//     -> 118; 10 x 55, 1.86: 59 -> 65
// Longer ones would leave one long sequence among short ones to one group.
constexpr int kWholeKeys = 512, kWholeMore = 1024, kWholeMost = 2048, kWholeGroups = 128, kWholeShared = 256;
constexpr int64_t kWholeBytes = 256 << 20;

bool never_cut(const Cache& c, const Queries& a, bool shared, int64_t tiles, int key_bytes) {
  const int64_t keys = (int64_t)c.max_pages * c.page, groups = a.batch * tiles * c.kv_heads;
  if (keys <= kWholeKeys) return !shared || groups * keys * key_bytes <= kWholeBytes;
  if (keys > (shared ? kWholeMore : kWholeMost)) return false;
  if (keys <= kWholeMore) return groups >= kWholeGroups && (!shared || groups <= kWholeShared);
  return groups >= kHold && (groups + kHold - 1) / kHold * kHold * 10 <= groups * 13;
}

// ---------------------------------------------------------------------------
// A piece of up to 16 NT rows.  Its keys go through registers only: a wave
// takes every fourth tile of 32 keys, loads K rows as the A operand of
// S^T = K Q^T (16x16x32 MFMAs, queries in columns), and ends up with 8 scores
// a lane of one query, at keys 4 g .. 4 g + 3 of both 16-key halves (g = lane / 16).
// The sum over keys in O^T = V^T P^T may run in any order, so these 8 are the
// lane's slice of the B operand as they are, and its slice of V^T, the
// same 8 keys at one dim, comes from loading D / 16 consecutive dims of each of the 8
// keys (a row of V per 16 lanes, whole lines that are read once and need not stay in
// the L2) and transposing within the lane: row m of the t-th MFMA is dim
// (D / 16) m + t.  No LDS, no barrier until the four waves join.  Bound by
// HBM: 32 sequences of up to 4K tokens, 8 heads of 128, 281 MB in 58 us (4.9 TB/s).
// ---------------------------------------------------------------------------
template <int D>
struct VRow;
template <>
struct VRow<64> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(8))); };
template <>
struct VRow<96> { typedef uint32_t type __attribute__((ext_vector_type(3), aligned(4))); };
template <>
struct VRow<128> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(16))); };

// Puts into o, dims d .. d + 3 of a row's values, the sum of the infinite and NaN values
// of keys k0 .. end - 1 where there are any: what a row that sees them gets, whatever
// their weights.  The product makes NaN of an infinite value whose weight, or the second
// part of it, is 0 or of the other sign, and leaves out those of tiles with a mask.
template <int D>
__device__ __forceinline__ void put_unbounded(const Args& x, const int32_t* table, int kh, int k0, int end, int d, f32x4_t& o) {
  f32x4_t sum{};
#pragma unroll 1
  for (int key = k0; key < end; ++key) {
    const int id = table[key >> x.page_bits];
    if (!in_range(id, x.c.pages)) continue;
    const uint16_t* v = x.vp + (((size_t)id * x.c.kv_heads + kh) * x.c.page + (key & (x.c.page - 1))) * D + d;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((v[i] & 0x7f80) == 0x7f80) sum[i] += __builtin_bit_cast(float, (uint32_t)v[i] << 16);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (sum[i] != 0.f) o[i] = sum[i];
}
__device__ __forceinline__ bool any_nan(const f32x4_t& o) { return o[0] != o[0] || o[1] != o[1] || o[2] != o[2] || o[3] != o[3]; }

// threadIdx.x, unknown to the compiler: what a piece computes from it would else be
// kept in registers over the loop over pieces, for every kind of piece at once
// (registers spilled at D = 128, 60 us instead of 53 at 64 sequences over 8K).
__device__ __forceinline__ int fresh_tid() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

template <int D, int NT, bool kAlone>
__device__ __forceinline__ void stream_piece(const Args& x, const Piece& p, float* lds) {
  constexpr int kC = D / 32, kT = D / 16, kStride = D + 4, kRows = 16 * NT;
  constexpr bool kAhead = D * NT <= 128;            // registers for a second V tile
  typedef typename VRow<D>::type VWords;
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
    const int r = p.row0 + min(16 * u + n, p.rows - 1);
    const int b = p.first + r / rows, w = r % rows;
    see[u] = min(p.see + w % x.a.q_len, p.k1);
    const uint16_t* row = x.q + (((size_t)b * x.c.kv_heads + kh) * rows + w) * D + 8 * g;
#pragma unroll
    for (int i = 0; i < kC; ++i) qf[u][i] = *(const u32x4_t*)(row + 32 * i);
  }
  const int least = min(p.see, p.k1);              // every row sees the keys below
  f32x4_t o[NT][kT];
  float m[NT], l[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    m[u] = -INFINITY;
    l[u] = 0.f;
#pragma unroll
    for (int t = 0; t < kT; ++t) o[u][t] = f32x4_t{};
  }
  // Page ids of this wave's tiles: lane 2 i + s has the one of half s of tile i (mod 32), -1 for none.
  const int tiles = my_head < x.c.kv_heads ? (p.k1 - begin + stride - 1) / stride : 0;
  int ids = -1;
  auto load_ids = [&](int i0) {
    const int key = begin + stride * (i0 + (lane >> 1)) + 16 * (lane & 1);
    ids = key < p.k1 ? table[key >> x.page_bits] : -1;
    if (!in_range(ids, x.c.pages)) ids = -1;
  };
  u32x4_t kf[2][kC];
  VWords va[8], vb[8];
  uint32_t poison = 0;                              // infinite or NaN values set aside
  auto half_at = [&](int i, int s, bool& ok) {      // element offset of half s of tile i
    const int id = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + s);
    const int key = begin + stride * i + 16 * s;
    ok = id >= 0;
    return (((size_t)(ok ? id : 0) * x.c.kv_heads + kh) * page + (key & (page - 1))) * D;
  };
  auto load_k = [&](int i) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bool ok;
      const uint16_t* base = x.kp + half_at(i, s, ok);
#pragma unroll
      for (int e = 0; e < kC; ++e) kf[s][e] = *(const u32x4_t*)(base + n * D + 8 * g + 32 * e);
    }
  };
  auto load_v = [&](int i, VWords (&vr)[8]) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bool ok;
      const uint16_t* base = x.vp + half_at(i, s, ok);
#pragma unroll
      for (int e = 0; e < 4; ++e) vr[4 * s + e] = __builtin_nontemporal_load((const VWords*)(base + (4 * g + e) * D + kT * n));
    }
  };
  if (tiles > 0) {
    load_ids(0);
    load_k(0);
    load_v(0, va);
  }
  // Tile i, its V in vr; the next tile's K and V (into vn) are loaded meanwhile.
  auto tile = [&](int i, VWords (&vr)[8], VWords (&vn)[8]) {
    const int key0 = begin + stride * i;
    bool ok0, ok1;
    half_at(i, 0, ok0);
    half_at(i, 1, ok1);
    const bool masked = key0 + 32 > least || !ok0 || !ok1;
    f32x4_t s[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[u][h] = f32x4_t{};
#pragma unroll
        for (int e = 0; e < kC; ++e) s[u][h] = mfma16x16x32(kf[h][e], qf[u][e], s[u][h]);
      }
    const bool more = i + 1 < tiles;
    if (more) {
      if (((i + 1) & 31) == 0) load_ids(i + 1);
      load_k(i + 1);
      if constexpr (kAhead) load_v(i + 1, vn);
    }
    if (masked) {
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key0 + 16 * h + 4 * g + r >= see[u] || !(h ? ok1 : ok0)) s[u][h][r] = -INFINITY;
    }
    u32x4_t pb[NT], pr[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      float mx = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[u][h][r]);
      mx = quad_max(mx) * x.sc;
      const bool grow = mx > m[u];
      if (__builtin_amdgcn_ballot_w64(grow)) {
        const float mn = grow ? mx : m[u];
        const float alpha = mn == m[u] ? 1.f : fast_exp2(m[u] - mn);
        l[u] *= alpha;
#pragma unroll
        for (int t = 0; t < kT; ++t)                 // in place, as in WaveRows::softmax
#pragma unroll
          for (int r = 0; r < 4; ++r) asm volatile("v_mul_f32 %0, %0, %1" : "+v"(o[u][t][r]) : "v"(alpha));
        m[u] = mn;
      }
      const float mb = m[u] == -INFINITY ? 0.f : m[u];
      float ts = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          y[r] = fast_exp2(__builtin_fmaf(s[u][h][r], x.sc, -mb));
          ts += y[r];
        }
        uint32_t rest[2];
        pb[u][2 * h] = split_bf16x2(y[0], y[1], rest[0]);
        pb[u][2 * h + 1] = split_bf16x2(y[2], y[3], rest[1]);
        pr[u][2 * h] = rest[0];
        pr[u][2 * h + 1] = rest[1];
      }
      l[u] += ts;
    }
    // V^T fragment of MFMA t: the keys e of this lane at dim (D / 16) n + t.
    auto frag = [&](int t) {
      u32x4_t f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = __builtin_amdgcn_perm(vr[2 * j + 1][t >> 1], vr[2 * j][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
      return f;
    };
    if (masked) {
      // Slots that no row sees may hold anything: they count as 0 (0 * NaN is NaN).
      // So do infinite and NaN values, which must not reach the rows that don't
      // see them; the others get them at the end.
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool any = key0 + 16 * (e >> 2) + 4 * g + (e & 3) < p.k1 && (e >= 4 ? ok1 : ok0);
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const uint32_t v = any ? vr[e][w] : 0;
          const uint32_t bad = ((v & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
          vr[e][w] = v & ~bad;
          poison |= bad;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      const u32x4_t f = frag(t);
#pragma unroll
      for (int u = 0; u < NT; ++u) o[u][t] = mfma16x16x32(f, pr[u], mfma16x16x32(f, pb[u], o[u][t]));
    }
    if (!kAhead && more) load_v(i + 1, vn);
  };
  if constexpr (kAhead) {
    int i = 0;
    for (; i + 1 < tiles; i += 2) {
      tile(i, va, vb);
      tile(i + 1, vb, va);
    }
    if (i < tiles) tile(i, va, vb);
  } else {
    for (int i = 0; i < tiles; ++i) tile(i, va, va);
  }
  // Join the waves.
  float* mls = lds + 4 * kRows * kStride;
  const bool poisoned = __syncthreads_or(poison != 0);
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const float lt = quad_sum(l[u]);
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
  if (my_head >= x.c.kv_heads) return;
  for (int j = kAlone ? lane : tid; j < p.rows * (D / 4); j += kAlone ? 64 : 256) {
    const int r = j / (D / 4), d = j % (D / 4) * 4;
    float mw[4], mx = -INFINITY, lt = 0.f;
    f32x4_t sum{};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mw[w] = kAlone && w != wave ? -INFINITY : mls[2 * (w * kRows + r)];
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
    if (poisoned || (lt == lt && any_nan(sum)))
      put_unbounded<D>(x, table, kh, p.k0, min(p.see + (p.row0 + r) % rows % x.a.q_len, p.k1), d, sum);
    if (p.slot >= 0) {
      const size_t at = (size_t)p.slot + (size_t)kh * p.seg_rows + p.row0 + r;
      *(f32x4_t*)(x.part + at * D + d) = sum;
      if (d == 0) x.ml[at] = float2{mx, lt};
    } else {
      const size_t at = ((size_t)p.first * x.c.kv_heads + kh) * rows + p.row0 + r;
      const float inv = lt == 0.f ? 0.f : 1.f / lt;
      *(u32x2_t*)(x.o + at * D + d) = u32x2_t{pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
      if (d == 0 && x.lse != nullptr) x.lse[at] = lt == 0.f ? -INFINITY : (mx + __builtin_log2f(lt)) * kLn2;
    }
  }
}

// ---------------------------------------------------------------------------
// A piece of up to 128 rows, all of which see all its keys (whole tiles of
// 64): the software pipeline of the dense kernel (WaveRows::step), four waves
// of 32 rows over rings of two K and two V tiles in LDS.  A wave copies 16
// consecutive keys of a tile, which lie in one page.  Bound by the matrix
// cores and the exponentials, 1.5 us a tile of 64 keys of 128 beside a group of few
// rows.  False, with nothing done, if some page id of the piece names no page.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ bool tile_piece(const Args& x, const Piece& p, char* smem) {
  using G = Geo<D>;
  constexpr int kT = Swizzle<D>::kTile, kC = TileCopy<D, 4>::kPer;
  const int tid = fresh_tid(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = x.rows, page = x.c.page, kh = p.head;
  const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
  const int tiles = (p.k1 - p.k0) / kKeyTile;
  // Page ids of this wave's keys: lane i has the one of tile 64 u + i, of stretch u and the next one.
  auto load_ids = [&](int u) {
    const int key = p.k0 + (64 * u + lane) * kKeyTile + 16 * wave;
    return key < p.k1 ? table[key >> x.page_bits] : 0;
  };
  int stretch = 0, ids = load_ids(0), next_ids = load_ids(1);
  bool bad = false;
  for (int j = (p.k0 >> x.page_bits) + tid; j <= (p.k1 - 1) >> x.page_bits; j += 256) bad |= !in_range(table[j], x.c.pages);
  if (__syncthreads_or(bad)) return false;
  WaveRows<D> w;
  w.reset();
  {
    const int r = p.row0 + min(32 * wave + (lane & 31), p.rows - 1);
    const int b = p.first + r / rows;
    const uint16_t* row = x.q + (((size_t)b * x.c.kv_heads + kh) * rows + r % rows) * D + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < G::kDChunks; ++i) w.qf[i] = *(const u32x4_t*)(row + 16 * i);
  }
  TileCopy<D, 4> cp;
  ReadAddr<D> ra;
  cp.init(wave, lane);
  ra.init(lane);
#pragma unroll
  for (int i = 0; i < kC; ++i) {                    // offsets from the wave's first key
    cp.ko[i] -= 16 * wave * Swizzle<D>::kRow;
    cp.vo[i] -= 16 * wave * Swizzle<D>::kRow;
  }
  const uint32_t lk = lds_address(smem), lv = lk + 2 * kT;
  const char* sk = smem;
  const char* sv = smem + 2 * kT;
  auto source = [&](const uint16_t* pool, int it) { // this wave's keys of tile it
    const int id = __builtin_amdgcn_readlane(it >> 6 == stretch ? ids : next_ids, it & 63);
    const int key = p.k0 + it * kKeyTile + 16 * wave;
    return buffer_words(pool + (((size_t)id * x.c.kv_heads + kh) * page + (key & (page - 1))) * D);
  };
  auto copy_k = [&](u32x4_t from, int it, int i) { cp.k1(from, 0, lk + (it & 1) * kT, wave, i); };
  auto copy_v = [&](u32x4_t from, int it, int i) { cp.v1(from, 0, lv + (it & 1) * kT, wave, i); };
  {
    const u32x4_t k0 = source(x.kp, 0), v0 = source(x.vp, 0);
#pragma unroll
    for (int i = 0; i < kC; ++i) copy_k(k0, 0, i);
#pragma unroll
    for (int i = 0; i < kC; ++i) copy_v(v0, 0, i);
    if (tiles > 1) {
      const u32x4_t k1 = source(x.kp, 1);
#pragma unroll
      for (int i = 0; i < kC; ++i) copy_k(k1, 1, i);
    }
  }
#pragma unroll
  for (int i = 0; i < G::kDChunks; ++i) asm volatile("" : "+v"(w.qf[i]));
  wait_copies<0>();
  __syncthreads();
  const bool active = 32 * wave < p.rows;
  f32x16_t s0[2], s1[2];
  float mx = 0.f;
  if (active) w.template step<2, true, false, 0>(sk, sv, ra, lane, x.sc, s1, s0, mx, [](auto, int) {}, [](f32x16_t*) {});
  __syncthreads();                                  // K(0) read by every wave: K(2) may take its place
  // Step `it`: S^T of tile it + 1, softmax and PV of tile it; V(it + 1) and K(it + 2)
  // go where V(it - 1) and K(it) were.  At its end both have landed.
  auto fused = [&](int it, f32x16_t sc[2], f32x16_t sn[2]) {
    const int b = it & 1;
    if (it >> 6 != stretch) {
      stretch = it >> 6;
      ids = next_ids;
      next_ids = load_ids(stretch + 1);
    }
    const u32x4_t fv = source(x.vp, it + 1), fk = source(x.kp, min(it + 2, tiles - 1));
    const bool more = it + 2 < tiles;
    auto copy = [&](int i) {
      if (i < kC) copy_v(fv, it + 1, i);
      else if (more) copy_k(fk, it + 2, i - kC);
    };
    if (active) {
      w.template step<2, true, true, 0, kProbSplit>(sk + (b ^ 1) * kT, sv + b * kT, ra, lane, x.sc, sc, sn, mx,
                                        [&](auto n, int j) {
                                          constexpr int kGap = std::max(1, (decltype(n)::value * 5 / 8 - 2) / (2 * kC));
                                          if (j >= 2 && (j - 2) % kGap == 0 && (j - 2) / kGap < 2 * kC) copy((j - 2) / kGap);
                                        },
                                        [](f32x16_t*) {});
    } else {
#pragma unroll
      for (int i = 0; i < 2 * kC; ++i) copy(i);
    }
    wait_copies<0>();
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
  if (!active) return true;
  w.template step<2, false, true, 0, kProbSplit>(sk, sv + (it & 1) * kT, ra, lane, x.sc, s0, s1, mx, [](auto, int) {}, [](f32x16_t*) {});
  const float lt = pair_sum(w.l);
  const int q = 32 * wave + (lane & 31), h = lane >> 5;
  if (q >= p.rows) return true;
  const size_t at = (size_t)p.slot + (size_t)kh * p.seg_rows + p.row0 + q;
#pragma unroll
  for (int t = 0; t < G::kDTiles; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4_t*)(x.part + at * D + 32 * t + 8 * j + 4 * h) =
          f32x4_t{w.o[t][4 * j], w.o[t][4 * j + 1], w.o[t][4 * j + 2], w.o[t][4 * j + 3]};
  if (h == 0) x.ml[at] = float2{w.m, lt};
  float all = 0.f;
#pragma unroll
  for (int t = 0; t < G::kDTiles; ++t)
#pragma unroll
    for (int j = 0; j < 16; ++j) all += w.o[t][j];
  if (lt == lt && all != all) {                     // of infinite values
#pragma unroll 1
    for (int d = 4 * h; d < D; d += 8) {
      f32x4_t o = *(const f32x4_t*)(x.part + at * D + d);
      if (!any_nan(o)) continue;
      put_unbounded<D>(x, table, kh, p.k0, p.k1, d, o);
      *(f32x4_t*)(x.part + at * D + d) = o;
    }
  }
  return true;
}

template <int D, int NT, bool kShared>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
piece_kernel(Args x) {
  constexpr int kJoin = 4 * 16 * (kShared ? 2 : NT) * (D + 6) * 4, kRing = kShared ? 4 * Swizzle<D>::kTile : 0;
  __shared__ __attribute__((aligned(1024))) char smem[kJoin > kRing ? kJoin : kRing];
  static_assert(sizeof(Plan<256>) <= sizeof(smem), "the plan fits");
  __shared__ Piece todo[kTodo];
  __shared__ int listed;
  const int count = my_pieces<kTodo>(x, todo, &listed, smem);
  for (int i = 0; i < count; ++i) {
    Piece p = todo[i];
    int32_t* w = (int32_t*)&p;                     // the same in every lane
#pragma unroll
    for (int j = 0; j < 11; ++j) w[j] = __builtin_amdgcn_readfirstlane(w[j]);
    if (i > 0) __syncthreads();                     // the piece before has left the LDS
    if constexpr (kShared) {
      if (p.kind == kManyRows && tile_piece<D>(x, p, smem)) continue;
      if (p.see != kSeeAll) {
        if (p.kind == kNarrow) stream_piece<D, NT, true>(x, p, (float*)smem);
        else stream_piece<D, NT, false>(x, p, (float*)smem);
        continue;
      }
      // A few rows, or, where a page is missing, many a few at a time.
      Piece s = p;
      for (int r = 0; r < p.rows; r += 32) {
        s.row0 = p.row0 + r;
        s.rows = min(32, p.rows - r);
        stream_piece<D, 2, false>(x, s, (float*)smem);
      }
    } else {
      if (p.kind == kNarrow) stream_piece<D, NT, true>(x, p, (float*)smem);
      else stream_piece<D, NT, false>(x, p, (float*)smem);
    }
  }
}

template <int D, int NT>
hipError_t launch(const Args& x, hipStream_t st) {
  const int64_t rows = (int64_t)x.a.batch * x.a.heads * x.a.q_len;
  if (x.mode == kPlanned) {
    plan_kernel<<<1, kPlan, 0, st>>>(x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // Two groups a CU (registers allow few kinds more, and three or four do worse where
  // they do: 62 and 64 us instead of 58 at 32 sequences of up to 4K), or as many as do
  // all the pieces kTodo at a time.
  const int64_t pieces = (int64_t)x.most * x.c.kv_heads, hold = kHold;
  const unsigned grid = (unsigned)std::min(pieces, std::max(hold, (pieces + kTodo - 1) / kTodo));
  if (x.shared != nullptr) piece_kernel<D, NT, true><<<grid, 256, 0, st>>>(x);
  else piece_kernel<D, NT, false><<<grid, 256, 0, st>>>(x);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || x.mode == kWhole) return e;
  if (rows <= kFewJoins) join_kernel<D, 4><<<(unsigned)rows, 256, 0, st>>>(x, rows);
  else join_kernel<D, 1><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(x, rows);
  return hipGetLastError();
}

}  // namespace

size_t prefix_workspace_bytes(const Cache& c, const Queries& a) { return space_bytes(c, a, nullptr, nullptr); }

hipError_t launch_prefix(const Cache& c, const Queries& a, const void* q, const void* kp, const void* vp, const int32_t* tables,
                         const int32_t* lens, const int32_t* ids, const int32_t* shared, void* o, float* lse, void* ws,
                         hipStream_t st) {
  const Args x = make_args(c, a, 4 * c.head_dim, never_cut, q, kp, vp, tables, lens, ids, shared, o, lse, ws);
  switch (c.head_dim + x.tile) {
    case 64 + 16: return launch<64, 1>(x, st);
    case 96 + 16: return launch<96, 1>(x, st);
    case 128 + 16: return launch<128, 1>(x, st);
    case 64 + 32: return launch<64, 2>(x, st);
    case 96 + 32: return launch<96, 2>(x, st);
    default: return launch<128, 2>(x, st);
  }
}

}  // namespace wise
