// prefix_plan.hpp — what the kernels of attention over a paged cache share,
// whatever its pages hold: segments and their pieces, the plan of a call, the pieces of
// a work-group, the join of the pieces' results.
#pragma once

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
  int32_t kind, head;                  // head: key-value head, or group of four of them (kNarrow)
  int32_t pad;
};

// Pieces of up to kWide rows; of few rows; of few rows and keys, a wave each.
enum { kManyRows, kFewRows, kNarrow };

// Where the pieces of a sequence's rows lie: results of row r over piece i of the
// shared pages at pre_slot + (i * kv_heads + kh) * pre_rows + pre_row0 + r, over piece i of
// its own at own_slot + (i * kv_heads + kh) * rows + r.
struct Joint {
  int32_t pre_slot, pre_pieces, pre_rows, pre_row0;
  int32_t own_slot, own_pieces, done, pad;   // done: a single piece wrote o
};

// Sizes of the pieces.  Pieces of few rows: so many that there are kGroups / 2
// (the work-groups that the chip holds at once), of at least kFewKeys keys; where
// that makes them longer than kMidKeys, so many that there are kGroups.  us a call by the
// number of pieces, 512 / 1024 / 2048: 8 samples of 4K, 55 heads of 96, 31.9 / 32.1 /
// 36.3; 128 over a 32K prefix, 8 heads of 128, 289 / 256 / 303.
constexpr int kGroups = 1024, kFewKeys = 128, kMidKeys = 512;
// Pieces of up to 128 rows: at most kWideGroups, one a CU beside one of few rows (two, where
// those are few, are as often worse as better: 57 instead of 53 us at 128 over 32K with tails of 16, but 75
// instead of 80 over 30K under 4 heads of 64), and of at most kWideKeys keys where that leaves kWideFill, since each leaves 128 rows
// of results to join; of at least kWideLeast keys.  64 / 128 / 256 / 512 of them over the 32K prefix: 482 / 320
// / 256 / 331 us; at most 256 / 512 / 768 / 1024 keys: 58.0 / 58.3 / 53.1 / 53.3 us at 64
// sequences over 8K; filled up to 192 of them, not left at 768 keys each: 23.3 instead of 31.2 us
// at 40 over 2K, 32.5 instead of 34.9 at 16 x 5 drafts over 4K.
constexpr int kWide = 128, kWideGroups = 256, kWideFill = 192, kWideKeys = 768, kWideLeast = 256;
// Shared pages: rows of a piece of few rows, and rows of a segment up to which it has few
// (3 x 12 requests' 48 rows over 8K in a piece of 128: 43.8 us instead of 41.1; 120 rows over 16K in
// pieces of 32: 50 instead of 36).
constexpr int kPreTile = 32, kWideRows = 64;
// Where there are more (sequence, head)s than groups: keys of a sequence's own up to
// which a wave takes them alone, four heads a group, since the latency of a piece is most of
// its time (128 sequences of up to 64 tokens over a 16K prefix, 64 heads of 64 on 16: 92 us
// instead of 103).
constexpr int kNarrowKeys = 128, kNarrowTable = 512, kHold = 512;   // kNarrowTable: of uncut ones, those of tables of so many

constexpr int kSeeAll = 0x7fffffff - kMaxQueryRows;   // Piece::see of shared pages

// Who plans: nobody (every sequence is one piece), every work-group, a launch before.
enum { kWhole, kOwnPlan, kPlanned };

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
  const int64_t tiles = b * ((rows + tile - 1) / tile) + b * rows / kPreTile + b / 2;   // own rows, shared ones
  const int64_t most = (cap + kFewKeys - 1) / kFewKeys;                               // pieces of a segment
  const int64_t wide_tiles = std::min<int64_t>(b / 2, b * rows / kWideRows) + b * rows / kWide;
  const int64_t wide_most = (cap + kWideLeast - 1) / kWideLeast;
  const int64_t few = std::min<int64_t>(kGroups / kv + 1 + tiles, tiles * most);
  const int64_t wide = std::min<int64_t>(kWideGroups / kv + 1 + wide_tiles, wide_tiles * wide_most);
  return Limits{few + wide, std::min<int64_t>(kPreTile * (kGroups + kv) + 2 * kv * b * rows, 2 * kv * b * rows * most) +
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

struct Args {
  Cache c;
  Queries a;
  float sc;                            // scale * log2(e)
  int rows;                            // query rows of a sequence per key-value head
  int tile, tiles;                     // rows of a piece of few rows, such pieces of a sequence's rows
  int page_bits;
  int key_bytes;                       // of K and V, a key and key-value head
  int mode;                            // kWhole, kOwnPlan or kPlanned
  int most;                            // pieces that the workspace holds
  int narrow;                          // there may be pieces of a wave
  int mid_keys, fill_all, wide_keys;   // kMidKeys, kWideGroups instead of kWideFill, kWideKeys, or what does better
  int shares;                          // even shares per key-value head; 0: none
  int wide_cost;                       // time of a key to 128 rows, in times of one to few rows; 0: dealt as equal
  const uint16_t *q, *kp, *vp;
  const int32_t *tables, *lens, *ids, *shared;
  int32_t* count;
  Joint* joint;
  Piece* piece;
  float2* ml;
  float* part;
  uint16_t* o;
  float* lse;
};

// ---------------------------------------------------------------------------
// Plan: a thread a sequence.  Up to 256 sequences every work-group plans for
// itself, once for its few pieces (2 to 3 us, most of it the loads of ids and
// lengths; a launch before it took 8 to 10), up to 64 in one wave without barriers;
// more are planned by one group of 1024 threads.
// ---------------------------------------------------------------------------
template <int kN>
struct Plan {                          // LDS
  int32_t members[kN], pre_keys[kN], first[3][kN], id[kN], len[kN], own_len[kN], own_slot[kN], pre_slot[kN],
      pre_pieces[kN], pre_len[kN];
  int64_t wave_keys[kN / 64][2];
  int32_t wave_sum[kN / 64][4], wave_start[kN / 64];
  int32_t start[kN], size[kN];         // split_runs
  unsigned long long saved[kN];
};

struct Cuts {
  int pieces[3];                       // of each kind, per key-value head (kNarrow: per four)
  int worth;                           // pieces of few rows that take a group as long as one of many
};

__device__ __forceinline__ int up_to(int x, int y) { return (int)(((uint32_t)x + y - 1) / (uint32_t)y); }

// Pieces of `keys` keys when a piece should hold about `chunk`, and their even length
// (pieces of `chunk` and a rest: 263 us instead of 256 at 128 sequences over 32K).
__device__ __forceinline__ void cut_keys(int keys, int chunk, int unit, int& pieces, int& len) {
  pieces = 0;
  len = unit;
  if (keys <= 0) return;
  len = (up_to(keys, up_to(keys, chunk)) + unit - 1) & -unit;
  pieces = up_to(keys, len);
}

__device__ __forceinline__ int known_len(const Args& x, int id) {
  return in_range(id, x.c.seqs) ? min(max(x.lens[id], 0), x.c.max_pages * x.c.page) : 0;
}

// The planning threads are together: one wave needs no barrier for it.
template <int kN>
__device__ __forceinline__ void plan_sync() {
  if constexpr (kN > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Maximum (minimum, or) of v over the planning threads; `none` changes nothing.
template <int kN, class Op>
__device__ __forceinline__ int plan_all(int v, int none, Op op, int32_t* waves) {
  v = __builtin_amdgcn_readlane(wave_scan(v, none, op), 63);
  if constexpr (kN > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = none;
    for (int w = 0; w < kN / 64; ++w) v = op(v, waves[w]);
  }
  return v;
}

// Even shares, instead of pieces of about the same length.  Per key-value head, the segments of a batch are laid one behind
// another, each kPieceKeys longer than its keys (what a piece costs beside them), and cut into x.shares equal stretches, one a
// work-group: it does what lies in its stretch, and all end together (32 sequences of up to 8K in 4 bits, 1144 pieces over 512
// groups, ended 19 to 41 us after the start, 32 on average: 41.8 us a call, 39.0 with shares; 2 x 69K tokens 84 and 70; 128 of
// up to 4K 72.8 and 68.6).  A cut inside a segment is moved to a multiple of 128 keys.  Where sequences have fewer than
// kShareLeast keys on average, the pieces of a stretch are too many (64 samples over 16 prompts of 1K: 283 and 347 us a step).
constexpr int kPieceKeys = 256, kShareSeqs = 256, kShareLeast = 1024;

struct Shares {                        // LDS
  int32_t at[kShareSeqs], pre[kShareSeqs], len[kShareSeqs], id[kShareSeqs], members[kShareSeqs], pre_slot[kShareSeqs], own_slot[kShareSeqs];
  int32_t size, used;                  // of a stretch; how many there are, 0: pieces are made in the other way
  int32_t stretch, first;              // where the group is: of the stretches of all heads, and the sequence in it, -1 for the start
};

// Keys of a segment of `keys` keys at `at` that lie before stretch j.
__device__ __forceinline__ int share_cut(int at, int keys, int j, int size) {
  const int64_t y = (int64_t)j * size - at - kPieceKeys;
  return y >= keys ? keys : y <= 0 ? 0 : min(keys, ((int)y + 64) & ~127);
}
// The first stretch that has keys of it, and how many have.
__device__ __forceinline__ int share_first(int at, int keys, int size) {
  const int j = (int)((uint32_t)(at + kPieceKeys) / (uint32_t)size);
  return j + (share_cut(at, keys, j + 1, size) == 0);
}
__device__ __forceinline__ int share_count(int at, int keys, int size) {
  if (keys <= 0) return 0;
  const int last = (int)((uint32_t)(at + kPieceKeys + keys - 1) / (uint32_t)size);
  return last - (share_cut(at, keys, last, size) >= keys) - share_first(at, keys, size) + 1;
}

// Cuts runs where neighbours differ in what they share: `keys` are the keys that
// a sequence could read together with the one before it (0: none).  A run of n that
// reads m keys once saves (n - 1) m reads, and m is the least `keys` inside it, so one
// pair that shares little would take the sharing from all (64 users over 8192 keys with one
// short request among them read all 64 prompts).  From single sequences, the pairs are gone
// through from the most keys to the fewest, an eighth at a time: runs that lie side by
// side across pairs of at least L keys become one if each saves no less with L keys
// a member than alone, and all together no less than apart.  On random pairs that
// saves 99% of what the best cuts do (73% at the worst of 4000).  Pairs left after
// kRounds go into one round.  In: s.start, s.members, s.pre_keys of single sequences.  Out:
// the start of this sequence's run, and at a start s.members and s.pre_keys, the least `keys`.
constexpr int kRounds = 8;
// Bytes of K and V that cuts have to promise, up to 64 sequences and beyond, where a round has
// barriers: the search takes 1 to 5 us, and more runs are more pieces.  us a call, uncut and
// cut: 6 x 8 tasks of 2K with a common header, 170 MB, 35.1 and 23.8; 64 over 8K with
// a short request among them, 220 and 48; 2 x 8 over 576, 33 MB, 18.8 and 15.7; not 8 x 5, 26 MB,
// 18.7 and 21.6.  Beyond 64 sequences: 16 x 16 over 448, 110 MB, 34.9 and 26.8; not 16 x 5, 47 MB, 24.2
// and 28.9, nor 40 x 2, 84 MB, 72 and 76.
constexpr int64_t kCutBytes = 32 << 20, kCutMore = 96 << 20;

template <int kN>
__device__ __forceinline__ int split_runs(Plan<kN>& s, bool live, int keys) {
  const int b = threadIdx.x;
  const auto larger = [](int x, int y) { return x > y ? x : y; };
  const auto smaller = [](int x, int y) { return x < y ? x : y; };
  int start = b;
  bool left = live && keys > 0;        // not gone through yet
  for (int round = 1;; ++round) {
    const int top = plan_all<kN>(left ? keys : 0, 0, larger, s.wave_start);
    if (top == 0) return start;
    const bool now = left && (round == kRounds || keys >= top - top / 8);
    const int64_t least = plan_all<kN>(now ? keys : 0x7fffffff, 0x7fffffff, smaller, s.wave_start);
    left = left && !now;
    plan_sync<kN>();
    auto joins = [&](int g) {
      const int64_t n = s.members[g];
      return n * least >= (n - 1) * s.pre_keys[g];
    };
    const bool open = now && joins(b) && joins(s.start[b - 1]);
    int chain = wave_scan_max(start == b && !open ? b : 0);
    if constexpr (kN > 64) {
      if ((b & 63) == 63) s.wave_start[b >> 6] = chain;
    }
    s.size[b] = 0;
    s.saved[b] = 0;
    plan_sync<kN>();
    for (int w = 0; w < (kN > 64 ? b >> 6 : 0); ++w) chain = max(chain, s.wave_start[w]);
    if (live && start == b) {
      const int n = s.members[b];
      atomicAdd(&s.size[chain], n);
      atomicAdd(&s.saved[chain], (unsigned long long)(n - 1) * s.pre_keys[b]);
    }
    plan_sync<kN>();
    const int n = s.size[chain];
    if ((n - 1) * least >= (int64_t)s.saved[chain]) {
      start = chain;
      if (b == chain) s.members[b] = n;
      if (open) atomicMin(&s.pre_keys[chain], keys);
    }
    s.start[b] = start;
    plan_sync<kN>();
  }
}

// Runs and pieces of all sequences, or (shares, where there is a place for them and they do better) even shares.
// Writes x.joint if `write`.
template <int kN>
__device__ void make_plan(const Args& x, Plan<kN>& s, bool write, Cuts& cut, Shares* shares = nullptr) {
  const int b = threadIdx.x, lane = b & 63, wave = kN > 64 ? b >> 6 : 0;
  const Cache& c = x.c;
  const Queries& a = x.a;
  const bool live = b < a.batch;
  const int rows = x.rows;
  const int id = !live ? -1 : x.ids ? x.ids[b] : b;
  const int len = known_len(x, id), see = len - a.q_len + 1;
  int start = b, n = 1, pre = 0;
  if (x.shared != nullptr) {
    // What a sequence could read together with the one before it: whole pages
    // that every query of the two sees, in whole tiles of 64 keys (so that
    // no piece of them needs a mask).
    int keys = 0;
    if (live && b > 0) {
      const int see0 = known_len(x, x.ids ? x.ids[b - 1] : b - 1) - a.q_len + 1;
      keys = (min(max(x.shared[b], 0), max(min(see0, see), 0) >> x.page_bits) << x.page_bits) & ~63;
    }
    // Runs: a sequence belongs to the last start at or before it.
    start = wave_scan_max(keys == 0 ? b : 0);
    if (kN > 64 && lane == 63) s.wave_start[wave] = start;
    s.members[b] = 0;
    s.pre_keys[b] = 0x7fffffff;
    plan_sync<kN>();
    for (int w = 0; w < wave; ++w) start = max(start, s.wave_start[w]);
    if (live) {
      atomicAdd(&s.members[start], 1);
      if (b != start) atomicMin(&s.pre_keys[start], keys);
    }
    plan_sync<kN>();
    n = s.members[start];
    if (n > 1) pre = s.pre_keys[start];
    // No cuts save more than the sum of `keys`: they are sought where that is an eighth more than
    // the runs save, and kCutBytes or kCutMore of K and V more.
    const bool inside = live && b != start;
    int uneven = inside && keys != pre;
    uneven = kN > 64 ? __syncthreads_or(uneven) : __builtin_amdgcn_ballot_w64(uneven) != 0;
    if (uneven) {
      int64_t more = wave_total(inside ? keys - pre : 0), now = wave_total(inside ? pre : 0);
      if constexpr (kN > 64) {
        if (lane == 0) {
          s.wave_keys[wave][0] = more;
          s.wave_keys[wave][1] = now;
        }
        __syncthreads();
        more = now = 0;
        for (int w = 0; w < kN / 64; ++w) {
          more += s.wave_keys[w][0];
          now += s.wave_keys[w][1];
        }
        __syncthreads();
      }
      if (more * 8 > now && more * c.kv_heads * x.key_bytes >= (kN > 64 ? kCutMore : kCutBytes)) {
        s.start[b] = b;
        s.members[b] = 1;
        s.pre_keys[b] = 0x7fffffff;
        start = split_runs<kN>(s, live, keys);
        n = s.members[start];
        pre = n > 1 ? s.pre_keys[start] : 0;
      }
    }
  }
  const int own = len - pre, own_tiles = x.tiles;
  const bool leads = live && b == start && pre > 0;
  const int pre_rows = leads ? n * rows : 0;
  const bool wide = pre_rows > kWideRows;
  const int pre_tiles = wide ? (pre_rows + kWide - 1) / kWide : (pre_rows + kPreTile - 1) / kPreTile;
  int64_t k0 = (int64_t)own_tiles * own + (wide ? 0 : (int64_t)pre_tiles * pre), k1 = wide ? (int64_t)pre_tiles * pre : 0;
  k0 = wave_total(k0);
  k1 = x.shared != nullptr ? wave_total(k1) : 0;
  if constexpr (kN > 64) {
    if (lane == 0) {
      s.wave_keys[wave][0] = k0;
      s.wave_keys[wave][1] = k1;
    }
    __syncthreads();
    k0 = k1 = 0;
    for (int w = 0; w < kN / 64; ++w) {
      k0 += s.wave_keys[w][0];
      k1 += s.wave_keys[w][1];
    }
  }
  if (shares != nullptr) {
    // Where sequences are long, and segments one row tile each.
    bool place = x.shares > 0 && k1 == 0 && k0 < (int64_t)1 << 29 && k0 >= (int64_t)a.batch * kShareLeast;
    if (place) {
      const bool odd = leads && pre_tiles > 1;
      place = !(kN > 64 ? __syncthreads_or(odd) : __builtin_amdgcn_ballot_w64(odd) != 0);
    }
    if (place) {
      const int mine = (leads ? pre + kPieceKeys : 0) + (live && own > 0 ? own + kPieceKeys : 0);
      int end = wave_scan_add(mine), total = __builtin_amdgcn_readlane(end, 63);
      if constexpr (kN > 64) {
        if (lane == 63) s.wave_sum[wave][0] = end;
        __syncthreads();
        total = 0;
        for (int w = 0; w < kN / 64; ++w) {
          const int y = s.wave_sum[w][0];
          end += w < wave ? y : 0;
          total += y;
        }
        __syncthreads();
      }
      const int size = max(up_to(total, x.shares), kPieceKeys + kFewKeys), at = end - mine;
      const int pre_n = leads ? share_count(at, pre, size) : 0, own_n = live ? share_count(end - own - kPieceKeys, own, size) : 0;
      const bool done = live && pre == 0 && own_n == 1;
      const int slots = (done ? 0 : own_n * c.kv_heads * rows) + pre_n * c.kv_heads * pre_rows;
      int slot = wave_scan_add(slots);
      if constexpr (kN > 64) {
        if (lane == 63) s.wave_sum[wave][1] = slot;
        __syncthreads();
        for (int w = 0; w < wave; ++w) slot += s.wave_sum[w][1];
      }
      slot -= slots;
      shares->at[b] = at;
      for (int i = b + kN; i < kShareSeqs; i += kN) shares->at[i] = 0x7fffffff;
      shares->pre[b] = pre;
      shares->len[b] = len;
      shares->id[b] = id;
      shares->members[b] = leads ? n : 0;
      shares->pre_slot[b] = slot;
      shares->own_slot[b] = done ? -1 : slot + pre_n * c.kv_heads * pre_rows;
      s.pre_slot[b] = slot;
      s.pre_pieces[b] = pre_n;
      if (b == 0) {
        shares->size = size;
        shares->used = up_to(total, size);
        shares->stretch = blockIdx.x;
        shares->first = -1;
      }
      plan_sync<kN>();
      if (write && live)
        x.joint[b] = Joint{s.pre_slot[start], pre > 0 ? s.pre_pieces[start] : 0, n * rows, (b - start) * rows, shares->own_slot[b], own_n, done, 0};
      return;
    }
    if (b == 0) shares->used = 0;
  }
  auto even = [&](int64_t sum, int groups, int least) {
    return (int)min(max((sum * c.kv_heads + groups - 1) / groups, (int64_t)least), (int64_t)1 << 30);
  };
  const int chunk = max(even(k0, kGroups, kFewKeys), min(even(k0, kGroups / 2, kFewKeys), x.mid_keys));
  int wide_chunk = kWideLeast;
  cut.worth = 1;
  if (k1 > 0) {
    wide_chunk = max(even(k1, kWideGroups, kWideLeast), min(x.fill_all ? even(k1, kWideGroups, kWideLeast) : even(k1, kWideFill, kWideLeast), x.wide_keys));
    cut.worth = max(1, (int)((float)wide_chunk * (float)x.wide_cost / (float)chunk + 0.5f));
  }
  const bool narrow = x.narrow && own <= kNarrowKeys;
  int own_n, own_l, pre_n, pre_l;
  cut_keys(live ? own : 0, chunk, 32, own_n, own_l);
  cut_keys(leads ? pre : 0, wide ? wide_chunk : chunk, 64, pre_n, pre_l);
  const bool done = live && pre == 0 && own_n == 1;
  // Prefix sums: pieces of each kind, rows of results.
  const int own_all = own_n * own_tiles, pre_all = pre_n * pre_tiles;
  const int mine[4] = {wide ? pre_all : 0, (narrow ? 0 : own_all) + (wide ? 0 : pre_all), narrow ? own_all : 0,
                       (done ? 0 : own_n * c.kv_heads * rows) + pre_n * c.kv_heads * pre_rows};
  int sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = wave_scan_add(mine[i]);
  if constexpr (kN > 64) {
    if (lane == 63)
#pragma unroll
      for (int i = 0; i < 4; ++i) s.wave_sum[wave][i] = sum[i];
    __syncthreads();
    int all[4] = {0, 0, 0, 0};
    for (int w = 0; w < kN / 64; ++w) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int y = s.wave_sum[w][i];
        sum[i] += w < wave ? y : 0;
        all[i] += y;
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) cut.pieces[i] = all[i];
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) cut.pieces[i] = __builtin_amdgcn_readlane(sum[i], 63);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) s.first[i][b] = sum[i] - mine[i];
  s.pre_slot[b] = sum[3] - mine[3];
  s.own_slot[b] = done ? -1 : sum[3] - mine[3] + pre_n * c.kv_heads * pre_rows;
  s.id[b] = id;
  s.len[b] = len;
  s.own_len[b] = own_l;
  s.pre_pieces[b] = pre_n;
  s.pre_len[b] = pre_l;
  if (x.shared == nullptr) s.members[b] = 1;
  s.pre_keys[b] = pre;
  plan_sync<kN>();
  if (write && live)
    x.joint[b] = Joint{s.pre_slot[start], pre > 0 ? s.pre_pieces[start] : 0, n * rows, (b - start) * rows, s.own_slot[b], own_n, done, 0};
}

// Piece j of a kind.
template <int kN>
__device__ Piece piece_at(const Args& x, const Plan<kN>& s, int kind, int j) {
  const int rows = x.rows, kv = x.c.kv_heads;
  const int e = plan_entry<kN>(s.first[kind], j);
  j -= s.first[kind][e];
  Piece p;
  p.kind = kind;
  p.first = e;
  p.table = s.id[e];
  const int pre_rows = s.pre_pieces[e] > 0 ? s.members[e] * rows : 0;
  const bool pre_wide = pre_rows > kWideRows;
  const int pre_tiles = pre_wide ? (pre_rows + kWide - 1) / kWide : (pre_rows + kPreTile - 1) / kPreTile;
  const int pre_all = kind == kManyRows || (kind == kFewRows && !pre_wide) ? s.pre_pieces[e] * pre_tiles : 0;
  int tile;
  if (j < pre_all) {
    const int i = (uint32_t)j / (uint32_t)pre_tiles, len = s.pre_len[e];
    tile = pre_wide ? kWide : kPreTile;
    p.seg_rows = pre_rows;
    p.row0 = (j - i * pre_tiles) * tile;
    p.k0 = i * len;
    p.k1 = min(p.k0 + len, s.pre_keys[e]);
    p.see = kSeeAll;
    p.slot = s.pre_slot[e] + i * kv * pre_rows;
  } else {
    j -= pre_all;
    tile = x.tile;
    const int i = x.tiles == 1 ? j : (uint32_t)j / (uint32_t)x.tiles;
    p.seg_rows = rows;
    p.row0 = (j - i * x.tiles) * tile;
    p.k0 = s.pre_keys[e] + i * s.own_len[e];
    p.k1 = min(p.k0 + s.own_len[e], s.len[e]);
    p.see = s.len[e] - x.a.q_len + 1;
    p.slot = s.own_slot[e] < 0 ? -1 : s.own_slot[e] + i * kv * rows;
  }
  p.rows = min(tile, p.seg_rows - p.row0);
  p.pad = 0;
  return p;
}

// Kind of piece k of all, in the order of the kinds; k becomes its number in the kind.
__device__ __forceinline__ int kind_of(const Cuts& cut, int& k) {
  int kind = kManyRows;
  if (k >= cut.pieces[kManyRows]) {
    k -= cut.pieces[kManyRows];
    kind = kFewRows;
    if (k >= cut.pieces[kFewRows]) {
      k -= cut.pieces[kFewRows];
      kind = kNarrow;
    }
  }
  return kind;
}

__global__ void __launch_bounds__(kPlan)
plan_kernel(Args x) {
  __shared__ Plan<kPlan> s;
  Cuts cut;
  make_plan<kPlan>(x, s, true, cut);
  const int all = min(cut.pieces[0] + cut.pieces[1] + cut.pieces[2], x.most);
  if (threadIdx.x < 3) x.count[threadIdx.x] = cut.pieces[threadIdx.x];
  if (threadIdx.x == 3) x.count[3] = cut.worth;
  for (int k = threadIdx.x; k < all; k += kPlan) {
    int j = k;
    const int kind = kind_of(cut, j);
    x.piece[k] = piece_at<kPlan>(x, s, kind, j);
  }
}

// The pieces that this work-group is to do, in todo[0 .. count - 1]; returns the
// count.  The (piece, head)s are dealt to the groups in turn, there and back, those of
// many rows first: a group plans once and does a few, and the last ones go to the
// groups that began with the lightest.
constexpr int kTodo = 8;

template <int kTodo>
__device__ __forceinline__ int my_pieces(const Args& x, Piece* todo, int* listed, char* smem, Shares* shares = nullptr) {
  const int kv = x.c.kv_heads, fours = (kv + 3) / 4;
  Cuts cut{};
  const bool one_wave = x.a.batch <= 64;
  if (x.mode == kOwnPlan) {
    if (!one_wave) make_plan<256>(x, *(Plan<256>*)smem, blockIdx.x == 0, cut, shares);
    else if (threadIdx.x < 64) make_plan<64>(x, *(Plan<64>*)smem, blockIdx.x == 0, cut, shares);
    if (shares != nullptr) {
      __syncthreads();
      if (shares->used > 0) return 0;
    }
  } else if (x.mode == kPlanned) {
#pragma unroll
    for (int i = 0; i < 3; ++i) cut.pieces[i] = x.count[i];
    cut.worth = x.count[3];
  } else {
    cut.pieces[x.narrow ? kNarrow : kFewRows] = x.most;
  }
  const int64_t whole = (int64_t)(cut.pieces[kManyRows] + cut.pieces[kFewRows]) * kv, all = whole + (int64_t)cut.pieces[kNarrow] * fours;
  // Row r of the deal: the r-th piece of every group, but that a group which begins with a piece of many
  // rows sits out the rows that this one is worth (as many as leave room for all pieces).
  const int64_t groups = gridDim.x, many = (int64_t)cut.pieces[kManyRows] * kv;
  const int worth = many == 0 || many >= groups ? 1 : min(max(cut.worth, 1), max(1, (int)min((float)(kTodo * groups - (all - many)) / (float)many * 0.9999f, 1e6f)));
  const bool busy = blockIdx.x < many;
  const int r = (int)threadIdx.x + (busy && threadIdx.x > 0 ? worth - 1 : 0);
  const bool part = r > 0 && r < worth;             // only the other groups take part
  const int64_t seat = part ? blockIdx.x - many : blockIdx.x, seats = part ? groups - many : groups;
  const int64_t before = r == 0 ? 0 : r < worth ? groups + (r - 1) * (groups - many) : groups + (worth - 1) * (groups - many) + (r - worth) * groups;
  const int64_t f = before + (r % 2 ? seats - 1 - seat : seat);
  if (threadIdx.x < kTodo && f < all) {
    const uint32_t at = (uint32_t)(f < whole ? f : f - whole), heads = f < whole ? kv : fours;
    int k = (int)(at / heads);
    const int head = (int)(at - k * heads);
    if (f >= whole) k += cut.pieces[kManyRows] + cut.pieces[kFewRows];
    Piece p;
    if (x.mode == kPlanned) {
      p = x.piece[k];
    } else {
      const int kind = kind_of(cut, k);
      if (x.mode == kOwnPlan) {
        p = one_wave ? piece_at<64>(x, *(Plan<64>*)smem, kind, k) : piece_at<256>(x, *(Plan<256>*)smem, kind, k);
      } else {                                      // kWhole: a sequence's rows against all its keys
        p.first = x.tiles == 1 ? k : (int)((uint32_t)k / (uint32_t)x.tiles);
        p.seg_rows = x.rows;
        p.row0 = (k - p.first * x.tiles) * x.tile;
        p.rows = min(x.tile, x.rows - p.row0);
        const int id = x.ids ? x.ids[p.first] : p.first;
        p.k0 = 0;
        p.k1 = known_len(x, id);
        p.table = in_range(id, x.c.seqs) ? id : 0;
        p.see = p.k1 - x.a.q_len + 1;
        p.slot = -1;
        p.kind = kind;
      }
    }
    p.head = head;
    todo[threadIdx.x] = p;
  }
  // The first wave has them all.
  if (threadIdx.x < 64) {
    const int mine = __popcll(__builtin_amdgcn_ballot_w64(threadIdx.x < kTodo && f < all));
    if (threadIdx.x == 0) *listed = mine;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*listed);
}

// The next pieces of this group's stretches: two (of shared pages, of its own) for each of kTodo / 2 sequences, those
// without keys of 0 rows.  False if there are none left.
template <int kTodo>
__device__ __forceinline__ bool share_pieces(const Args& x, Shares& s, Piece* todo) {
  __syncthreads();                                  // the list before is done with
  const int size = s.size, kv = x.c.kv_heads, j = s.stretch / kv, head = s.stretch - j * kv;
  if (j >= s.used) return false;
  const int first = s.first >= 0 ? s.first : plan_entry<kShareSeqs>(s.at, j * size), next = first + kTodo / 2;
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool inside = next < x.a.batch && s.at[next] < (int64_t)(j + 1) * size;
    s.first = inside ? next : -1;
    s.stretch += inside ? 0 : gridDim.x;
  }
  if (threadIdx.x < kTodo) {
    const int e = first + (int)threadIdx.x / 2;
    Piece p;
    p.rows = 0;
    if (e < x.a.batch && s.at[e] < (int64_t)(j + 1) * size) {
      const bool shared = threadIdx.x % 2 == 0;
      const int lead = s.members[e] > 0 ? s.pre[e] + kPieceKeys : 0;
      const int at = s.at[e] + (shared ? 0 : lead), keys = shared ? (lead > 0 ? s.pre[e] : 0) : s.len[e] - s.pre[e];
      const int k0 = share_cut(at, keys, j, size), k1 = share_cut(at, keys, j + 1, size);
      if (k0 < k1) {
        const int i = j - share_first(at, keys, size);
        p.first = e;
        p.table = s.id[e];
        p.row0 = 0;
        p.rows = p.seg_rows = shared ? s.members[e] * x.rows : x.rows;
        p.k0 = shared ? k0 : s.pre[e] + k0;
        p.k1 = shared ? k1 : s.pre[e] + k1;
        p.see = shared ? kSeeAll : s.len[e] - x.a.q_len + 1;
        p.slot = shared ? s.pre_slot[e] + i * kv * p.rows : s.own_slot[e] < 0 ? -1 : s.own_slot[e] + i * kv * p.rows;
        p.kind = kFewRows;
        p.head = head;
        p.pad = 0;
      }
    }
    todo[threadIdx.x] = p;
  }
  __syncthreads();
  return true;
}

// ---------------------------------------------------------------------------
// Join: W waves a row, each its share of the pieces, eight in flight.  Four up to
// kFewJoins rows, whose pieces are many: 7 queries of two sequences of 26K tokens, one
// key-value head, 40 -> 21 us a call; from 1500 rows on they cost (47.5 instead of 45.3).
// ---------------------------------------------------------------------------
constexpr int kFewJoins = 512;

template <int D, int W>
__global__ void __launch_bounds__(256)
join_kernel(Args x, int64_t all) {
  __shared__ float mls[4][2], part[4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = W == 4 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (row >= all) return;
  const int rows = x.rows, kv = x.c.kv_heads, w0 = W == 4 ? wave : 0;
  const int r = (int)(row % rows), kh = (int)(row / rows % kv), b = (int)(row / rows / kv);
  const Joint j = x.joint[b];
  if (j.done) return;
  const int pieces = (j.pre_pieces + j.own_pieces + W - 1 - w0) / W;   // this wave's: w0, w0 + W, ...
  auto slot = [&](int k) {
    const int i = w0 + W * k;
    return i < j.pre_pieces ? (size_t)j.pre_slot + ((size_t)i * kv + kh) * j.pre_rows + j.pre_row0 + r
                            : (size_t)j.own_slot + ((size_t)(i - j.pre_pieces) * kv + kh) * rows + r;
  };
  float2 y[8];
  auto load = [&](int i0) {
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      y[w] = float2{0.f, 0.f};
      if (i0 + w < pieces && lane < D / 2) y[w] = *(const float2*)(x.part + slot(i0 + w) * D + 2 * lane);
    }
  };
  load(0);
  float2 ml = lane < pieces ? x.ml[slot(lane)] : float2{-INFINITY, 0.f};
  float m = ml.x;
  for (int i = lane + 64; i < pieces; i += 64) m = fmaxf(m, x.ml[slot(i)].x);
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor(m, w, 64));
  float mb = m == -INFINITY ? 0.f : m;
  float l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += 64) {
    if (i0 > 0) ml = i0 + lane < pieces ? x.ml[slot(i0 + lane)] : float2{-INFINITY, 0.f};
    const float f = fast_exp2(ml.x - mb);
    l += f * ml.y;
    const int end = min(64, pieces - i0);
    for (int i = 0; i < end; i += 8) {
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float fi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), i + w));
        if (i + w < end) {
          o0 += fi * y[w].x;
          o1 += fi * y[w].y;
        }
      }
      load(i0 + i + 8);
    }
  }
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w, 64);
  // An infinite part counts whatever its weight, and 0 times it is NaN.
  auto unbounded = [](float& u, float y) { u += __builtin_isfinite(y) ? 0.f : y; };
  if (l == l && (o0 != o0 || o1 != o1)) {
    float u0 = 0.f, u1 = 0.f;
#pragma unroll 1
    for (int i = 0; i < pieces; ++i) {
      const float2 z = *(const float2*)(x.part + slot(i) * D + 2 * lane);
      unbounded(u0, z.x);
      unbounded(u1, z.y);
    }
    if (u0 != 0.f) o0 = u0;
    if (u1 != 0.f) o1 = u1;
  }
  if constexpr (W == 4) {
    if (lane < D / 2) *(float2*)(part[wave] + 2 * lane) = float2{o0, o1};
    if (lane == 0) {
      mls[wave][0] = m;
      mls[wave][1] = l;
    }
    __syncthreads();
    if (wave > 0) return;
    m = fmaxf(fmaxf(mls[0][0], mls[1][0]), fmaxf(mls[2][0], mls[3][0]));
    mb = m == -INFINITY ? 0.f : m;
    l = o0 = o1 = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(mls[w][0] - mb);
      l += f * mls[w][1];
      if (lane < D / 2) {
        o0 += f * part[w][2 * lane];
        o1 += f * part[w][2 * lane + 1];
      }
    }
    if (l == l && (o0 != o0 || o1 != o1)) {
      float u0 = 0.f, u1 = 0.f;
#pragma unroll 1
      for (int w = 0; w < 4; ++w) {
        unbounded(u0, part[w][2 * lane]);
        unbounded(u1, part[w][2 * lane + 1]);
      }
      if (u0 != 0.f) o0 = u0;
      if (u1 != 0.f) o1 = u1;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < D / 2) *(uint32_t*)(x.o + (size_t)row * D + 2 * lane) = pack_bf16x2(o0 * inv, o1 * inv);
  if (lane == 0 && x.lse != nullptr) x.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
}

// The arguments of the kernels of one call.  whole: whether every sequence is one piece (never_cut).
inline Args make_args(const Cache& c, const Queries& a, int key_bytes, bool (*whole)(const Cache&, const Queries&, bool, int64_t, int),
                      const void* q, const void* kp, const void* vp, const int32_t* tables,
                      const int32_t* lens, const int32_t* ids, const int32_t* shared, void* o, float* lse, void* ws) {
  Space s;
  space_bytes(c, a, ws, &s);
  Args x;
  x.c = c;
  x.a = a;
  x.sc = a.scale * kLog2e;
  x.tile = row_tile(c, a);
  x.rows = a.heads / c.kv_heads * a.q_len;
  x.tiles = (x.rows + x.tile - 1) / x.tile;
  x.key_bytes = key_bytes;
  x.mode = whole(c, a, shared != nullptr, x.tiles, key_bytes) ? kWhole : a.batch <= 256 ? kOwnPlan : kPlanned;
  if (x.mode == kWhole) shared = nullptr;
  x.wide_cost = x.shares = 0;
  x.mid_keys = kMidKeys, x.fill_all = 0, x.wide_keys = kWideKeys;
  x.page_bits = __builtin_ctz(c.page);
  x.narrow = (int64_t)a.batch * c.kv_heads > kHold && (x.mode != kWhole || c.max_pages * c.page <= kNarrowTable);
  x.most = x.mode == kWhole ? a.batch * x.tiles : (int)limits(c, a).pieces;
  x.q = (const uint16_t*)q, x.kp = (const uint16_t*)kp, x.vp = (const uint16_t*)vp;
  x.tables = tables, x.lens = lens, x.ids = ids, x.shared = shared;
  x.count = s.count, x.joint = s.joint, x.piece = s.piece, x.ml = s.ml, x.part = s.part;
  x.o = (uint16_t*)o, x.lse = lse;
  return x;
}

}  // namespace
}  // namespace wise
