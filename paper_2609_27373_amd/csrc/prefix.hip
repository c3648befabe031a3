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
//   plan_kernel   finds the runs, cuts the segments, lists the pieces
//   piece_kernel  one piece a work-group and key-value head: (m, l, O) in fp32
//   join_kernel   joins the pieces of every row, divides by l
#include <algorithm>

#include "plan.hpp"
#include "wise_kernels.hpp"
#include "wise_tiles.hpp"

namespace wise {
namespace {

// One piece: rows row0 .. row0 + rows - 1 of a segment against keys k0 .. k1 - 1.
struct Piece {
  int32_t first, seg_rows;             // first sequence of the batch, rows of the segment per key-value head
  int32_t row0, rows, k0, k1;
  int32_t table;                       // table row with the segment's pages
  int32_t see;                         // positions that a sequence's first query sees
  int32_t slot;                        // row of the piece's results, key-value head 0, segment row 0; -1: the whole result, written to o
  int32_t wide;                        // up to kWide rows, for tile_piece
  int32_t pad[2];
};

// Where the pieces of a sequence's rows lie: results of row r over piece i of the
// shared pages at pre_slot + (i * kv_heads + kh) * pre_rows + pre_row0 + r, over piece i of
// its own at own_slot + (i * kv_heads + kh) * rows + r.
struct Joint {
  int32_t pre_slot, pre_pieces, pre_rows, pre_row0;
  int32_t own_slot, own_pieces, done, pad;   // done: a single piece wrote o
};

// Target numbers of work-groups, and the fewest keys of a piece.
constexpr int kGroups = 2048, kFewKeys = 64;
constexpr int kWide = 128, kWideGroups = 512, kWideKeys = 256;   // the same for pieces of many rows

struct Space {                         // the workspace
  int32_t* count;
  Joint* joint;
  Piece* piece;
  float2* ml;
  float* part;
};

struct Limits {
  int64_t pieces, rows;                // most pieces per key-value head, most result rows
};

int row_tile(const Cache& c, const Queries& a) { return a.heads / c.kv_heads * a.q_len > 16 ? 32 : 16; }

// A segment of t row tiles and K keys is cut into at most K / C + 1 pieces, and C is
// at least sum(t K) * kv_heads / groups and the fewest keys of a piece.
Limits limits(const Cache& c, const Queries& a) {
  const int64_t rows = (int64_t)a.heads / c.kv_heads * a.q_len, tile = row_tile(c, a), b = a.batch, kv = c.kv_heads;
  const int64_t cap = (int64_t)c.max_pages * c.page;
  const int64_t tiles = b * ((rows + tile - 1) / tile) + b / 2;                       // own rows, shared ones of one tile
  const int64_t most = (cap + kFewKeys - 1) / kFewKeys;                               // pieces of a segment
  const int64_t wide_tiles = std::min<int64_t>(b / 2, b * rows / tile) + b * rows / kWide;
  const int64_t wide_most = (cap + kWideKeys - 1) / kWideKeys;
  const int64_t few = std::min<int64_t>(kGroups / kv + 1 + tiles, tiles * most);
  const int64_t wide = std::min<int64_t>(kWideGroups / kv + 1 + wide_tiles, wide_tiles * wide_most);
  return Limits{few + wide, std::min<int64_t>(tile * (kGroups + kv) + 2 * kv * b * rows, 2 * kv * b * rows * most) +
                                std::min<int64_t>(kWide * (kWideGroups + kv) + kv * b * rows, kv * b * rows * wide_most)};
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t space_bytes(const Cache& c, const Queries& a, void* ws, Space* s) {
  const Limits l = limits(c, a);
  char* p = (char*)ws;
  size_t at = 256;
  auto take = [&](size_t bytes) {
    char* q = p + at;
    at += up256(bytes);
    return q;
  };
  char* joint = take(a.batch * sizeof(Joint));
  char* piece = take(l.pieces * sizeof(Piece));
  char* ml = take(l.rows * sizeof(float2));
  char* part = take(l.rows * c.head_dim * sizeof(float));
  if (s != nullptr) *s = Space{(int32_t*)p, (Joint*)joint, (Piece*)piece, (float2*)ml, (float*)part};
  return at;
}

// ---------------------------------------------------------------------------
// Plan: a thread a sequence.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int up_to(int64_t x, int y) { return (int)((x + y - 1) / y); }

// Pieces of K keys when a piece should hold about `chunk`, and their even length.
__device__ __forceinline__ void cut_keys(int keys, int chunk, int unit, int& pieces, int& len) {
  pieces = 0;
  len = unit;
  if (keys <= 0) return;
  len = up_to(up_to(keys, up_to(keys, chunk)), unit) * unit;
  pieces = up_to(keys, len);
}

__global__ void __launch_bounds__(kPlan)
plan_kernel(Cache c, Queries a, int tile, int64_t most, const int32_t* __restrict__ tables_ids, const int32_t* __restrict__ lens,
            const int32_t* __restrict__ shared, int32_t* __restrict__ count, Joint* __restrict__ joint, Piece* __restrict__ piece) {
  __shared__ int32_t members[kPlan], min_pages[kPlan], min_see[kPlan];
  __shared__ int32_t first_[kPlan], wide_first_[kPlan], id_[kPlan], len_[kPlan], own_len[kPlan], own_slot[kPlan], pre_slot[kPlan], pre_pieces[kPlan],
      pre_len[kPlan];
  __shared__ int64_t waves[kPlanWaves];
  __shared__ int32_t wave_start[kPlanWaves];
  const int b = threadIdx.x, lane = b & 63, wave = b >> 6;
  const bool live = b < a.batch;
  const int rows = a.heads / c.kv_heads * a.q_len;
  const int id = !live ? -1 : tables_ids ? tables_ids[b] : b;
  const bool known = in_range(id, c.seqs);
  const int cap = c.max_pages * c.page;
  const int len = known ? min(max(lens[id], 0), cap) : 0;
  const int see = len - a.q_len + 1;
  const int sh = live && b > 0 && shared ? shared[b] : 0;
  // Runs: a sequence belongs to the last start at or before it.
  int start = sh <= 0 ? b : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(start, o, 64);
    if (lane >= o) start = max(start, y);
  }
  if (lane == 63) wave_start[wave] = start;
  members[b] = 0;
  min_pages[b] = min_see[b] = 0x7fffffff;
  __syncthreads();
  for (int w = 0; w < wave; ++w) start = max(start, wave_start[w]);
  if (live) {
    atomicAdd(&members[start], 1);
    atomicMin(&min_see[start], see);
    if (b != start) atomicMin(&min_pages[start], sh);
  }
  __syncthreads();
  // What the run reads once: whole pages that every query sees, in whole
  // tiles of 64 keys (so that no piece of them needs a mask).
  const int n = members[start];
  int pre = 0;
  if (n > 1) pre = (min(min_pages[start], max(min_see[start], 0) / c.page) * c.page) & ~63;
  const int own = len - pre;
  const int own_tiles = up_to(rows, tile);
  const bool leads = live && b == start && pre > 0;
  const int pre_rows = leads ? n * rows : 0;
  const bool wide = pre_rows > tile;
  const int pre_tiles = up_to(pre_rows, wide ? kWide : tile);
  int64_t keys, wide_keys;
  plan_scan((int64_t)own_tiles * own + (wide ? 0 : (int64_t)pre_tiles * pre), &keys, waves);
  plan_scan(wide ? (int64_t)pre_tiles * pre : 0, &wide_keys, waves);
  auto even = [&](int64_t sum, int groups, int least) {
    return (int)min(max((sum * c.kv_heads + groups - 1) / groups, (int64_t)least), (int64_t)1 << 30);
  };
  const int chunk = even(keys, kGroups, kFewKeys);
  int own_n, own_l, pre_n, pre_l;
  cut_keys(live ? own : 0, chunk, 32, own_n, own_l);
  cut_keys(leads ? pre : 0, wide ? even(wide_keys, kWideGroups, kWideKeys) : chunk, 64, pre_n, pre_l);
  const bool done = live && pre == 0 && own_n == 1;
  int64_t few, wides, slots;
  const int64_t first = plan_scan((int64_t)own_n * own_tiles + (wide ? 0 : (int64_t)pre_n * pre_tiles), &few, waves);
  const int64_t wide_first = plan_scan(wide ? (int64_t)pre_n * pre_tiles : 0, &wides, waves);
  const int64_t slot = plan_scan((done ? 0 : (int64_t)own_n * c.kv_heads * rows) + (int64_t)pre_n * c.kv_heads * pre_rows, &slots, waves);
  first_[b] = (int)first;
  wide_first_[b] = (int)wide_first;
  id_[b] = id;
  len_[b] = len;
  own_len[b] = own_l;
  pre_slot[b] = (int)slot;
  own_slot[b] = done ? -1 : (int)(slot + (int64_t)pre_n * c.kv_heads * pre_rows);
  pre_pieces[b] = pre_n;
  pre_len[b] = pre_l;
  // From here on: keys of the run's shared pages.
  min_pages[b] = pre;
  __syncthreads();
  if (live)
    joint[b] = Joint{pre_slot[start], pre > 0 ? pre_pieces[start] : 0, n * rows, (b - start) * rows, own_slot[b], own_n, done, 0};
  const int all = (int)min(few + wides, most);
  if (b == 0) *count = all;
  // Pieces of few rows wait for memory, those of many for the matrix cores: the
  // two kinds alternate, so that a CU holds both.
  const int both = 2 * (int)min(few, wides);
  for (int k = b; k < all; k += kPlan) {
    const bool is_wide = k < both ? k % 2 == 0 : wides > few;
    const int in_kind = k < both ? k / 2 : k - both / 2;
    const int e = plan_entry(is_wide ? wide_first_ : first_, in_kind);
    int j = in_kind - (is_wide ? wide_first_ : first_)[e];
    const int p_rows = pre_pieces[e] > 0 ? members[e] * rows : 0;
    const int p_tile = is_wide ? kWide : tile, p_tiles = up_to(p_rows, p_tile), p_all = is_wide || p_rows <= tile ? pre_pieces[e] * p_tiles : 0;
    Piece p;
    p.first = e;
    p.wide = is_wide;
    if (j < p_all) {
      const int i = j / p_tiles, t = j % p_tiles;
      p.seg_rows = p_rows;
      p.row0 = t * p_tile;
      p.k0 = i * pre_len[e];
      p.k1 = min(p.k0 + pre_len[e], min_pages[e]);
      p.see = 0x7fffffff - a.q_len;
      p.slot = pre_slot[e] + i * c.kv_heads * p_rows;
    } else {
      j -= p_all;
      const int i = j / own_tiles, t = j % own_tiles;
      p.seg_rows = rows;
      p.row0 = t * tile;
      p.k0 = min_pages[e] + i * own_len[e];
      p.k1 = min(p.k0 + own_len[e], len_[e]);
      p.see = len_[e] - a.q_len + 1;
      p.slot = own_slot[e] < 0 ? -1 : own_slot[e] + i * c.kv_heads * rows;
    }
    p.rows = min(is_wide ? kWide : tile, p.seg_rows - p.row0);
    p.table = id_[e];
    p.pad[0] = p.pad[1] = 0;
    piece[k] = p;
  }
}

// ---------------------------------------------------------------------------
// A piece of up to 16 NT rows.  Its keys go through registers only: a wave
// takes every fourth tile of 32 keys, loads K rows as the A operand of
// S^T = K Q^T (16x16x32 MFMAs, queries in columns), and ends up with 8 scores
// a lane of one query, at keys 4 g .. 4 g + 3 of both 16-key halves (g = lane / 16).
// The sum over keys in O^T = V^T P^T may run in any order, so these 8 are the
// lane's slice of the B operand as they are, and its slice of V^T, the
// same 8 keys at one dim, comes from loading D / 16 consecutive dims of each of the 8 keys
// (a row of V per 16 lanes) and transposing within the lane: row m of the
// t-th MFMA is dim (D / 16) m + t.  No LDS, no barrier until the four waves join.
// ---------------------------------------------------------------------------
template <int D>
struct VRow;
template <>
struct VRow<64> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(8))); };
template <>
struct VRow<96> { typedef uint32_t type __attribute__((ext_vector_type(3), aligned(4))); };
template <>
struct VRow<128> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(16))); };

struct Args {
  Cache c;
  Queries a;
  float sc;                            // scale * log2(e)
  const uint16_t *q, *kp, *vp;
  const int32_t* tables;
  const int32_t* count;
  const Piece* piece;
  float2* ml;
  float* part;
  uint16_t* o;
  float* lse;
};

template <int D, int NT>
__device__ __forceinline__ void stream_piece(const Args& x, const Piece& p, int kh, float* lds) {
  constexpr int kC = D / 32, kT = D / 16, kStride = D + 4, kRows = 16 * NT;
  typedef typename VRow<D>::type VWords;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, n = lane & 15;
  const int rows = x.a.heads / x.c.kv_heads * x.a.q_len, page = x.c.page;
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
  const int tiles = (p.k1 - p.k0 - 32 * wave + 127) / 128;
  int ids = -1;
  auto load_ids = [&](int i0) {
    const int key = p.k0 + 32 * wave + 128 * (i0 + (lane >> 1)) + 16 * (lane & 1);
    ids = key < p.k1 ? table[key / page] : -1;
    if (!in_range(ids, x.c.pages)) ids = -1;
  };
  u32x4_t kf[2][kC];
  VWords vr[8];
  auto half_at = [&](int i, int s, bool& ok) {      // element offset of half s of tile i
    const int id = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + s);
    const int key = p.k0 + 32 * wave + 128 * i + 16 * s;
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
  auto load_v = [&](int i) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bool ok;
      const uint16_t* base = x.vp + half_at(i, s, ok);
#pragma unroll
      for (int e = 0; e < 4; ++e) vr[4 * s + e] = *(const VWords*)(base + (4 * g + e) * D + kT * n);
    }
  };
  if (tiles > 0) {
    load_ids(0);
    load_k(0);
    load_v(0);
  }
  for (int i = 0; i < tiles; ++i) {
    const int key0 = p.k0 + 32 * wave + 128 * i;
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
    u32x4_t pb[NT];
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
        for (int t = 0; t < kT; ++t) o[u][t] *= alpha;
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
        pb[u][2 * h] = pack_bf16x2(y[0], y[1]);
        pb[u][2 * h + 1] = pack_bf16x2(y[2], y[3]);
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
    bool plain = true;
    if (masked) {
      // Slots that no row sees may hold anything: they count as 0 (0 * NaN is NaN).
      // A value that some rows see and others don't must reach the former only.
      uint32_t bad = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool any = key0 + 16 * (e >> 2) + 4 * g + (e & 3) < p.k1 && (e >= 4 ? ok1 : ok0);
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          vr[e][w] = any ? vr[e][w] : 0;
          bad |= (vr[e][w] & 0x7f80u) == 0x7f80u || (vr[e][w] & 0x7f800000u) == 0x7f800000u;
        }
      }
      plain = !__builtin_amdgcn_ballot_w64(bad != 0);
    }
    if (plain) {
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        const u32x4_t f = frag(t);
#pragma unroll
        for (int u = 0; u < NT; ++u) o[u][t] = mfma16x16x32(f, pb[u], o[u][t]);
      }
    } else {
      // Token by token of the queries: the keys its rows see, added to their columns.
      for (int w = 0, last = p.k0; w < x.a.q_len; ++w) {
        const int end = min(p.see + w, p.k1);
        if (end <= last) continue;
        last = end;
        uint32_t keep[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = key0 + 16 * (j >> 1) + 4 * g + 2 * (j & 1);
          keep[j] = (key < end ? 0xffffu : 0u) | (key + 1 < end ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          u32x4_t f = frag(t);
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] &= keep[j];
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const f32x4_t y = mfma16x16x32(f, pb[u], f32x4_t{});
#pragma unroll
            for (int r = 0; r < 4; ++r) o[u][t][r] += see[u] == end ? y[r] : 0.f;
          }
        }
      }
    }
    if (more) load_v(i + 1);
  }
  // Join the waves.
  float* mls = lds + 4 * kRows * kStride;
  __syncthreads();
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
      for (int t = 0; t < kT; ++t) lds[r * kStride + kT * (4 * g + i) + t] = o[u][t][i];
  }
  __syncthreads();
  for (int j = tid; j < p.rows * (D / 4); j += 256) {
    const int r = j / (D / 4), d = j % (D / 4) * 4;
    float mw[4], mx = -INFINITY, lt = 0.f;
    f32x4_t sum{};
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, mw[w] = mls[2 * (w * kRows + r)]);
    const float mb = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(mw[w] - mb);
      lt += f * mls[2 * (w * kRows + r) + 1];
      sum += f * *(const f32x4_t*)(lds + (w * kRows + r) * kStride + d);
    }
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
// consecutive keys of a tile, which lie in one page.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void tile_piece(const Args& x, const Piece& p, int kh, char* smem) {
  using G = Geo<D>;
  constexpr int kT = Swizzle<D>::kTile, kC = TileCopy<D, 4>::kPer;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = x.a.heads / x.c.kv_heads * x.a.q_len, page = x.c.page;
  const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
  const int tiles = (p.k1 - p.k0) / kKeyTile;
  // Page ids of this wave's keys: lane i has the one of tile 64 u + i, of stretch u and the next one.
  auto load_ids = [&](int u) {
    const int key = p.k0 + (64 * u + lane) * kKeyTile + 16 * wave;
    return key < p.k1 ? table[key / page] : 0;
  };
  int stretch = 0, ids = load_ids(0), next_ids = load_ids(1);
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
      w.template step<2, true, true, 0>(sk + (b ^ 1) * kT, sv + b * kT, ra, lane, x.sc, sc, sn, mx,
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
  if (!active) return;
  w.template step<2, false, true, 0>(sk, sv + (it & 1) * kT, ra, lane, x.sc, s0, s1, mx, [](auto, int) {}, [](f32x16_t*) {});
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

template <int D, int NT, bool kShared>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
piece_kernel(Args x) {
  constexpr int kJoin = 4 * 16 * NT * (D + 6) * 4, kRing = kShared ? 4 * Swizzle<D>::kTile : 0;
  __shared__ __attribute__((aligned(1024))) char smem[kJoin > kRing ? kJoin : kRing];
  const int i = blockIdx.x / x.c.kv_heads, kh = blockIdx.x % x.c.kv_heads;
  if (i >= *x.count) return;
  const Piece p = x.piece[i];
  if constexpr (kShared) {
    bool whole = false;
    if (p.wide) {                                   // every page id of the piece names a page
      const int32_t* table = x.tables + (size_t)p.table * x.c.max_pages;
      bool bad = false;
      for (int j = p.k0 / x.c.page + threadIdx.x; j <= (p.k1 - 1) / x.c.page; j += 256) bad |= !in_range(table[j], x.c.pages);
      whole = !__syncthreads_or(bad);
      if (whole) tile_piece<D>(x, p, kh, smem);
    }
    if (whole) return;
    // A few rows, or, where a page is missing, many a few at a time.
    Piece s = p;
    for (int r = 0; r < p.rows; r += 16 * NT) {
      s.row0 = p.row0 + r;
      s.rows = min(16 * NT, p.rows - r);
      stream_piece<D, NT>(x, s, kh, (float*)smem);
    }
  } else {
    stream_piece<D, NT>(x, p, kh, (float*)smem);
  }
}

// ---------------------------------------------------------------------------
// Join: a wave a row.
// ---------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(256)
join_kernel(Args x, const Joint* __restrict__ joint, int64_t all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= all) return;
  const int rows = x.a.heads / x.c.kv_heads * x.a.q_len, kv = x.c.kv_heads;
  const int r = (int)(row % rows), kh = (int)(row / rows % kv), b = (int)(row / rows / kv);
  const Joint j = joint[b];
  if (j.done) return;
  const int pieces = j.pre_pieces + j.own_pieces;
  auto slot = [&](int i) {
    return i < j.pre_pieces ? (size_t)j.pre_slot + ((size_t)i * kv + kh) * j.pre_rows + j.pre_row0 + r
                            : (size_t)j.own_slot + ((size_t)(i - j.pre_pieces) * kv + kh) * rows + r;
  };
  float m = -INFINITY;
  for (int i = lane; i < pieces; i += 64) m = fmaxf(m, x.ml[slot(i)].x);
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor(m, w, 64));
  const float mb = m == -INFINITY ? 0.f : m;
  float l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += 64) {
    float f = 0.f;
    if (i0 + lane < pieces) {
      const float2 y = x.ml[slot(i0 + lane)];
      f = fast_exp2(y.x - mb);
      l += f * y.y;
    }
    const int end = min(64, pieces - i0);
    for (int i = 0; i < end; i += 8) {               // eight loads in flight
      float2 y[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        y[w] = float2{0.f, 0.f};
        if (i + w < end && lane < D / 2) y[w] = *(const float2*)(x.part + slot(i0 + i + w) * D + 2 * lane);
      }
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float fi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (i + w) & 63));
        if (i + w < end) {
          o0 += fi * y[w].x;
          o1 += fi * y[w].y;
        }
      }
    }
  }
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w, 64);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < D / 2) *(uint32_t*)(x.o + (size_t)row * D + 2 * lane) = pack_bf16x2(o0 * inv, o1 * inv);
  if (lane == 0 && x.lse != nullptr) x.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
}

template <int D, int NT>
hipError_t launch(const Args& x, const Joint* joint, bool shared, int64_t pieces, hipStream_t st) {
  const unsigned grid = (unsigned)(pieces * x.c.kv_heads);
  if (shared) piece_kernel<D, NT, true><<<grid, 256, 0, st>>>(x);
  else piece_kernel<D, NT, false><<<grid, 256, 0, st>>>(x);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)x.a.batch * x.a.heads * x.a.q_len;
  join_kernel<D><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(x, joint, rows);
  return hipGetLastError();
}

}  // namespace

size_t prefix_workspace_bytes(const Cache& c, const Queries& a) { return space_bytes(c, a, nullptr, nullptr); }

hipError_t launch_prefix(const Cache& c, const Queries& a, const void* q, const void* kp, const void* vp, const int32_t* tables,
                         const int32_t* lens, const int32_t* ids, const int32_t* shared, void* o, float* lse, void* ws,
                         hipStream_t st) {
  Space s;
  space_bytes(c, a, ws, &s);
  const Limits l = limits(c, a);
  const int tile = row_tile(c, a);
  plan_kernel<<<1, kPlan, 0, st>>>(c, a, tile, l.pieces, ids, lens, shared, s.count, s.joint, s.piece);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const Args x{c, a, a.scale * kLog2e, (const uint16_t*)q, (const uint16_t*)kp, (const uint16_t*)vp, tables, s.count, s.piece, s.ml,
               s.part, (uint16_t*)o, lse};
  switch (c.head_dim + tile) {
    case 64 + 16: return launch<64, 1>(x, s.joint, shared != nullptr, l.pieces, st);
    case 96 + 16: return launch<96, 1>(x, s.joint, shared != nullptr, l.pieces, st);
    case 128 + 16: return launch<128, 1>(x, s.joint, shared != nullptr, l.pieces, st);
    case 64 + 32: return launch<64, 2>(x, s.joint, shared != nullptr, l.pieces, st);
    case 96 + 32: return launch<96, 2>(x, s.joint, shared != nullptr, l.pieces, st);
    default: return launch<128, 2>(x, s.joint, shared != nullptr, l.pieces, st);
  }
}

}  // namespace wise
