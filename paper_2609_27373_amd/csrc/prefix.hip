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
constexpr int kNarrowKeys = 128, kHold = 512;

constexpr int kSeeAll = 0x7fffffff - kMaxQueryRows;   // Piece::see of shared pages

// Who plans: nobody (every sequence is one piece), every work-group, a launch before.
enum { kWhole, kOwnPlan, kPlanned };
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

bool never_cut(const Cache& c, const Queries& a, bool shared, int64_t tiles) {
  const int64_t keys = (int64_t)c.max_pages * c.page, groups = a.batch * tiles * c.kv_heads;
  if (keys <= kWholeKeys) return !shared || groups * keys * c.head_dim * 4 <= kWholeBytes;
  if (keys > (shared ? kWholeMore : kWholeMost)) return false;
  if (keys <= kWholeMore) return groups >= kWholeGroups && (!shared || groups <= kWholeShared);
  return groups >= kHold && (groups + kHold - 1) / kHold * kHold * 10 <= groups * 13;
}

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
  int mode;                            // kWhole, kOwnPlan or kPlanned
  int most;                            // pieces that the workspace holds
  int narrow;                          // there may be pieces of a wave
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

// Runs and pieces of all sequences.  Writes x.joint if `write`.
template <int kN>
__device__ void make_plan(const Args& x, Plan<kN>& s, bool write, Cuts& cut) {
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
      if (more * 8 > now && more * c.kv_heads * c.head_dim * 4 >= (kN > 64 ? kCutMore : kCutBytes)) {
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
  auto even = [&](int64_t sum, int groups, int least) {
    return (int)min(max((sum * c.kv_heads + groups - 1) / groups, (int64_t)least), (int64_t)1 << 30);
  };
  const int chunk = max(even(k0, kGroups, kFewKeys), min(even(k0, kGroups / 2, kFewKeys), kMidKeys));
  const bool narrow = x.narrow && own <= kNarrowKeys;
  int own_n, own_l, pre_n, pre_l;
  cut_keys(live ? own : 0, chunk, 32, own_n, own_l);
  cut_keys(leads ? pre : 0, wide ? max(even(k1, kWideGroups, kWideLeast), min(even(k1, kWideFill, kWideLeast), kWideKeys)) : chunk, 64, pre_n, pre_l);
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

__device__ __forceinline__ int my_pieces(const Args& x, Piece* todo, char* smem) {
  const int kv = x.c.kv_heads, fours = (kv + 3) / 4;
  Cuts cut{};
  const bool one_wave = x.a.batch <= 64;
  if (x.mode == kOwnPlan) {
    if (!one_wave) make_plan<256>(x, *(Plan<256>*)smem, blockIdx.x == 0, cut);
    else if (threadIdx.x < 64) make_plan<64>(x, *(Plan<64>*)smem, blockIdx.x == 0, cut);
  } else if (x.mode == kPlanned) {
#pragma unroll
    for (int i = 0; i < 3; ++i) cut.pieces[i] = x.count[i];
  } else {
    cut.pieces[x.narrow ? kNarrow : kFewRows] = x.most;
  }
  const int64_t whole = (int64_t)(cut.pieces[kManyRows] + cut.pieces[kFewRows]) * kv, all = whole + (int64_t)cut.pieces[kNarrow] * fours;
  const int64_t f = (int64_t)threadIdx.x * gridDim.x + (threadIdx.x % 2 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
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
  return __syncthreads_count(threadIdx.x < kTodo && f < all);
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
      w.template step<2, true, true, 0, true>(sk + (b ^ 1) * kT, sv + b * kT, ra, lane, x.sc, sc, sn, mx,
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
  w.template step<2, false, true, 0, true>(sk, sv + (it & 1) * kT, ra, lane, x.sc, s0, s1, mx, [](auto, int) {}, [](f32x16_t*) {});
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
  const int count = my_pieces(x, todo, smem);
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
  Space s;
  space_bytes(c, a, ws, &s);
  Args x;
  x.c = c;
  x.a = a;
  x.sc = a.scale * kLog2e;
  x.tile = row_tile(c, a);
  x.rows = a.heads / c.kv_heads * a.q_len;
  x.tiles = (x.rows + x.tile - 1) / x.tile;
  x.mode = never_cut(c, a, shared != nullptr, x.tiles) ? kWhole : a.batch <= 256 ? kOwnPlan : kPlanned;
  if (x.mode == kWhole) shared = nullptr;
  x.page_bits = __builtin_ctz(c.page);
  x.narrow = (int64_t)a.batch * c.kv_heads > kHold && (x.mode != kWhole || c.max_pages * c.page <= kWholeKeys);
  x.most = x.mode == kWhole ? a.batch * x.tiles : (int)limits(c, a).pieces;
  x.q = (const uint16_t*)q, x.kp = (const uint16_t*)kp, x.vp = (const uint16_t*)vp;
  x.tables = tables, x.lens = lens, x.ids = ids, x.shared = shared;
  x.count = s.count, x.joint = s.joint, x.piece = s.piece, x.ml = s.ml, x.part = s.part;
  x.o = (uint16_t*)o, x.lse = lse;
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
