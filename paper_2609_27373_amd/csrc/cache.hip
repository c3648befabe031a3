// cache.hip — the pages of a key-value cache on gfx950: forks, trims, room for
// new tokens (with the copy of a shared last page), their keys and values,
// compaction, and the pages that neighbours of a batch share.
//
// The bookkeeping is small integer work whose order fixes the result (the
// lowest free page goes to the first entry that needs one), so one work-group
// plans it from ballots and prefix sums, and a second launch moves the bytes.
// Reference counts change by integer atomics: any order gives the same count.
#include "plan.hpp"
#include "wise_device.hpp"
#include "wise_kernels.hpp"

namespace wise {
namespace {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int clamp_len(int len, const Cache& c) {
  const int cap = c.max_pages * c.page;
  return len < 0 ? 0 : len > cap ? cap : len;
}

// Whether some ids[j], j < n, equals x: by the whole work-group (uniform x).
__device__ __forceinline__ bool any_equal(const int32_t* ids, int n, int x) {
  bool hit = false;
  for (int j = threadIdx.x; j < n; j += blockDim.x) hit |= ids[j] == x;
  return __syncthreads_or(hit);
}

// The pages of [lo, hi) that are free (kFree) or in use, ascending: page number r
// goes to put(r, page); returns how many there are.  Each wave walks a stretch
// of its own twice, counting first, so the order needs no step per page.
template <bool kFree, class Put>
__device__ int list_pages(const int32_t* refs, int lo, int hi, int64_t* waves, Put put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int span = ((hi - lo + kPlan - 1) / kPlan) * 64;
  const int64_t w0 = (int64_t)lo + (int64_t)wave * span;
  const int b0 = (int)(w0 < hi ? w0 : hi), b1 = (int)(w0 + span < hi ? w0 + span : hi);
  auto takes = [&](int p) { return p < b1 && ((refs[p] <= 0) == kFree); };
  int count = 0;
  for (int p = b0; p < b1; p += 512) {
#pragma unroll
    for (int u = 0; u < 8; ++u) count += __popcll(__ballot(takes(p + 64 * u + lane)));
  }
  int64_t total;
  int at = (int)plan_scan(lane == 0 ? count : 0, &total, waves);
  at = __builtin_amdgcn_readfirstlane(at);
  for (int p = b0; p < b1; p += 512) {
    bool t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = takes(p + 64 * u + lane);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint64_t m = __ballot(t[u]);
      if (t[u]) put(at + __popcll(m & ((1ull << lane) - 1)), p + 64 * u + lane);
      at += __popcll(m);
    }
  }
  return (int)total;
}

// ---------------------------------------------------------------------------
// Forks and trims: a work-group an entry.  An entry only writes its own
// sequence's row, which no other entry of the call reads: a source that is
// also a destination is refused, and of equal ids the first one acts.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
fork_kernel(Cache c, int n, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int32_t* tables, int32_t* lens,
            int32_t* refs, int32_t* done) {
  const int i = blockIdx.x, a = src[i], b = dst[i];
  bool ok = in_range(a, c.seqs) && in_range(b, c.seqs);
  ok = !any_equal(dst, n, a) && ok;
  ok = !any_equal(dst, i, b) && ok;
  if (ok) ok = lens[b] <= 0;
  __syncthreads();                     // lens[b] read by every thread
  if (ok) {
    const int len = clamp_len(lens[a], c), used = (len + c.page - 1) / c.page;
    const int32_t* from = tables + (size_t)a * c.max_pages;
    int32_t* to = tables + (size_t)b * c.max_pages;
    for (int j = threadIdx.x; j < used; j += blockDim.x) {
      const int p = from[j];
      to[j] = p;
      if (in_range(p, c.pages)) atomicAdd(refs + p, 1);
    }
    if (threadIdx.x == 0) lens[b] = len;
  }
  if (done != nullptr && threadIdx.x == 0) done[i] = ok;
}

__global__ void __launch_bounds__(256)
trim_kernel(Cache c, const int32_t* __restrict__ ids, const int32_t* __restrict__ new_lens, int32_t* tables, int32_t* lens,
            int32_t* refs) {
  const int i = blockIdx.x, s = ids[i];
  if (any_equal(ids, i, s) || !in_range(s, c.seqs)) return;
  const int old = clamp_len(lens[s], c);
  int now = new_lens ? new_lens[i] : 0;
  now = now < 0 ? 0 : now;
  if (now >= old) return;
  __syncthreads();                     // lens[s] read by every thread
  int32_t* row = tables + (size_t)s * c.max_pages;
  const int end = (old + c.page - 1) / c.page;
  for (int j = (now + c.page - 1) / c.page + threadIdx.x; j < end; j += blockDim.x) {
    const int p = row[j];
    if (in_range(p, c.pages)) atomicSub(refs + p, 1);
    row[j] = -1;
  }
  if (threadIdx.x == 0) lens[s] = now;
}

// ---------------------------------------------------------------------------
// Room for new tokens.  An entry is one thread of the planning group: it says how many
// pages it needs, a prefix sum gives each its place in the list of free
// pages, and the places are filled by all threads.
// ---------------------------------------------------------------------------
struct ReserveCopy {
  int32_t src, dst, rows, pad;         // rows 0: nothing to copy
};

__global__ void __launch_bounds__(kPlan)
reserve_plan_kernel(Cache c, int n, const int32_t* __restrict__ ids, const int32_t* __restrict__ counts, int32_t* tables,
                    int32_t* lens, int32_t* refs, int32_t* granted, int32_t* list, ReserveCopy* copies) {
  __shared__ __attribute__((aligned(16))) int32_t id_[kPlan];
  __shared__ int32_t begin_[kPlan], row_[kPlan], first_[kPlan];
  __shared__ int64_t waves[kPlanWaves];
  const int i = threadIdx.x;
  const int s = i < n ? ids[i] : -1, count = i < n ? counts[i] : 0;
  id_[i] = s;
  __syncthreads();
  bool again = false;                  // by the waves that have entries, against those before them
  const int before = i < n ? (i | 63) + 1 : 0;
#pragma unroll 4
  for (int j = 0; j < before; j += 4) {
    const i32x4_t y = *(const i32x4_t*)(id_ + j);
#pragma unroll
    for (int u = 0; u < 4; ++u) again |= j + u < i && y[u] == s;
  }
  bool ok = in_range(s, c.seqs) && count > 0 && !again;
  int len = 0, begin = 0, last = -1;
  int64_t need = 0;
  bool copy = false;
  if (ok) {
    len = clamp_len(lens[s], c);
    ok = (int64_t)len + count <= (int64_t)c.max_pages * c.page;
  }
  if (ok) {
    begin = (len + c.page - 1) / c.page;
    if (len % c.page != 0) {
      last = tables[(size_t)s * c.max_pages + begin - 1];
      copy = in_range(last, c.pages) && refs[last] > 1;
    }
    begin -= copy;
    need = (len + count + c.page - 1) / c.page - begin;
  }
  int64_t total;
  const int64_t first = plan_scan(need, &total, waves);
  const int free_pages = list_pages<true>(refs, 0, c.pages, waves, [&](int r, int p) { list[r] = p; });
  ok = ok && (need == 0 || first + need <= free_pages);
  first_[i] = (int32_t)(first < free_pages ? first : (int64_t)free_pages);   // past them: no place is its
  row_[i] = ok ? s : -1;
  begin_[i] = begin;
  __syncthreads();                     // the list, too, is written
  const int places = (int)(total < free_pages ? total : (int64_t)free_pages);
  for (int k = i; k < places; k += kPlan) {
    const int e = plan_entry<kPlan>(first_, k);
    if (row_[e] < 0) continue;
    const int p = list[k];
    refs[p] = 1;
    tables[(size_t)row_[e] * c.max_pages + begin_[e] + (k - first_[e])] = p;
  }
  if (i < n) {
    ReserveCopy r{0, 0, 0, 0};
    if (ok) {
      lens[s] = len + count;
      if (copy) {
        r = ReserveCopy{last, list[first], len % c.page, 0};
        atomicSub(refs + last, 1);
      }
    }
    copies[i] = r;
    granted[i] = ok ? count : 0;
  }
}

// Copies what an entry's last page holds of its tokens, in every plane and head: their
// rows, or (kept.hpp) the codes and scales of their fours.  kCopyHeads of them a work-group, as many side by side as its threads reach, four passes in flight.
// The stores, here and below, pass the L2 by: nothing reads them before other kernels do.
constexpr int kCopyHeads = 16;

// 16-byte chunks of one head's page.
__host__ __device__ __forceinline__ int page_chunks(const Cache& c, int bits) {
  return c.page / 16 * (c.head_dim * bits / 8 + (bits == 16 ? 0 : c.head_dim / 32));
}

template <bool kBf16>
__global__ void __launch_bounds__(256)
reserve_copy_kernel(Cache c, int bits, const ReserveCopy* __restrict__ copies, uint16_t* pool) {
  const ReserveCopy r = copies[blockIdx.y];
  if (r.rows == 0) return;
  const size_t head = kBf16 ? (size_t)c.page * c.head_dim / 8 : (size_t)page_chunks(c, bits), page = head * c.kv_heads;   // 16-byte chunks
  const int fours = (r.rows + 3) / 4, codes = fours * c.head_dim * bits / 32;      // codes of the fours, 16 bytes each
  const int apart = c.page * c.head_dim * bits / 128 - codes;                      // chunks between these and their scales
  const int chunks = kBf16 ? r.rows * c.head_dim / 8 : codes + (fours * c.head_dim / 8 + 15) / 16, per = chunks < 256 ? 256 / chunks : 1;
  const int mine = chunks < 256 ? threadIdx.x / chunks : 0;
  if (mine >= per) return;
  const uint32_t x0 = blockIdx.x * kCopyHeads, all = (uint32_t)(c.planes * c.kv_heads), x1 = min(x0 + kCopyHeads, all);
  for (int ch = threadIdx.x - mine * chunks; ch < chunks; ch += 256) {
    for (uint32_t x = x0 + mine; x < x1; x += 4 * per) {
      u32x4_t w[4];
      u32x4_t* to[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t y = x + u * per, plane = y / (uint32_t)c.kv_heads, h = y - plane * c.kv_heads;
        if (y < x1) {
          u32x4_t* base = (u32x4_t*)pool + (size_t)plane * c.pages * page + h * head + (kBf16 || ch < codes ? ch : ch + apart);
          to[u] = base + (size_t)r.dst * page;
          w[u] = base[(size_t)r.src * page];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (x + u * per < x1) __builtin_nontemporal_store(w[u], to[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// Append.  A few tokens an entry: a 16-byte chunk of a token row a thread, K and
// V.  Many: a work-group takes some of one entry and head, whose sequence and
// length are then scalars, a few chunks a thread in flight.
// ---------------------------------------------------------------------------
constexpr int kManyTokens = 64;
constexpr int append_tile(int d) { return d == 96 ? 64 : 32; }   // tokens a work-group

// Element offset in a plane of position pos of sequence s, head h; -1: nowhere.
__device__ __forceinline__ int64_t slot_of(const Cache& c, const int32_t* tables, int s, int64_t pos, int h) {
  if (pos < 0 || pos >= (int64_t)c.max_pages * c.page) return -1;
  const int p = tables[(size_t)s * c.max_pages + (uint32_t)pos / (uint32_t)c.page];
  return in_range(p, c.pages) ? (((int64_t)p * c.kv_heads + h) * c.page + (pos & (c.page - 1))) * c.head_dim : -1;
}

__global__ void __launch_bounds__(256)
append_kernel(Cache c, int rows, int tokens, const int32_t* __restrict__ ids, const int32_t* __restrict__ counts,
              const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, const int32_t* __restrict__ tables,
              const int32_t* __restrict__ lens, uint16_t* kp, uint16_t* vp) {
  const int chunks = c.head_dim / 8, per = 256 / chunks;
  const int mine = threadIdx.x / chunks, ch = threadIdx.x % chunks;
  const int64_t at = (int64_t)blockIdx.x * per + mine;
  if (mine >= per || at >= rows) return;
  const uint32_t row = (uint32_t)at, t = row % (uint32_t)tokens, eh = row / (uint32_t)tokens;
  const uint32_t h = eh % (uint32_t)c.kv_heads, e = eh / (uint32_t)c.kv_heads;
  const size_t from = (size_t)row * c.head_dim + 8 * ch;
  const int s = ids[e];
  const int count = min(counts[e], tokens);
  if (!in_range(s, c.seqs) || (int)t >= count) return;
  const u32x4_t kw = *(const u32x4_t*)(k + from), vw = *(const u32x4_t*)(v + from);
  const int64_t to = slot_of(c, tables, s, (int64_t)lens[s] - count + (int)t, h);
  if (to < 0) return;
  *(u32x4_t*)(kp + to + 8 * ch) = kw;
  *(u32x4_t*)(vp + to + 8 * ch) = vw;
}

template <int D>
__global__ void __launch_bounds__(256)
append_tile_kernel(Cache c, int tokens, int tiles, const int32_t* __restrict__ ids, const int32_t* __restrict__ counts,
                   const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, const int32_t* __restrict__ tables,
                   const int32_t* __restrict__ lens, uint16_t* kp, uint16_t* vp) {
  constexpr int kTile = append_tile(D), kChunks = D / 8, kPer = kTile * kChunks / 256;
  static_assert(kTile * kChunks % 256 == 0, "whole chunks a thread");
  const uint32_t tile = blockIdx.x % (uint32_t)tiles, eh = blockIdx.x / (uint32_t)tiles;
  const uint32_t h = eh % (uint32_t)c.kv_heads, e = eh / (uint32_t)c.kv_heads;
  const int s = ids[e], t0 = tile * kTile;
  const int count = min(counts[e], tokens);
  if (!in_range(s, c.seqs) || t0 >= count) return;
  const int64_t first = (int64_t)lens[s] - count;
  const size_t from = (size_t)eh * tokens * D;
  u32x4_t kw[kPer], vw[kPer];
  int64_t to[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int x = threadIdx.x + 256 * u, t = t0 + x / kChunks, ch = x % kChunks;
    to[u] = -1;
    if (t < count) {
      kw[u] = __builtin_nontemporal_load((const u32x4_t*)(k + from + (size_t)t * D + 8 * ch));
      vw[u] = __builtin_nontemporal_load((const u32x4_t*)(v + from + (size_t)t * D + 8 * ch));
      to[u] = slot_of(c, tables, s, first + t, h);
    }
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int ch = (threadIdx.x + 256 * u) % kChunks;
    if (to[u] >= 0) {
      __builtin_nontemporal_store(kw[u], (u32x4_t*)(kp + to[u] + 8 * ch));
      __builtin_nontemporal_store(vw[u], (u32x4_t*)(vp + to[u] + 8 * ch));
    }
  }
}

// ---------------------------------------------------------------------------
// Compaction.  plan[0] = live pages, plan[1] = moves.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(kPlan)
compact_plan_kernel(Cache c, int32_t* refs, int32_t* live, int32_t* plan, int32_t* src, int32_t* dst, int32_t* renamed) {
  __shared__ int64_t waves[kPlanWaves];
  const int used = list_pages<false>(refs, 0, c.pages, waves, [](int, int) {});
  for (int p = used + threadIdx.x; p < c.pages; p += kPlan) renamed[p] = p;
  __syncthreads();
  const int moves = list_pages<true>(refs, 0, used, waves, [&](int r, int p) { dst[r] = p; });
  list_pages<false>(refs, used, c.pages, waves, [&](int r, int p) { src[r] = p; });
  __syncthreads();
  for (int r = threadIdx.x; r < moves; r += kPlan) {
    const int from = src[r], to = dst[r];
    renamed[from] = to;
    refs[to] = refs[from];
    refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    plan[0] = used;
    plan[1] = moves;
    if (live != nullptr) *live = used;
  }
}

__global__ void __launch_bounds__(256)
compact_move_kernel(Cache c, const int32_t* __restrict__ plan, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                    const int32_t* __restrict__ renamed, int32_t* tables, u32x4_t* pool, int64_t page) {
  const int used = plan[0], moves = plan[1];
  if (moves == 0) return;
  const size_t entries = (size_t)c.seqs * c.max_pages;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (size_t)gridDim.x * 256) {
    const int p = tables[e];
    if (p >= used && p < c.pages) tables[e] = renamed[p];
  }
  // page: 16-byte chunks of a page in one plane
  const int64_t pieces = (page + 1023) / 1024, items = moves * (int64_t)c.planes * pieces;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int64_t piece = x % pieces, y = x / pieces, plane = y % c.planes, m = y / c.planes;
    const u32x4_t* from = pool + (plane * c.pages + src[m]) * page;
    u32x4_t* to = pool + (plane * c.pages + dst[m]) * page;
    const int64_t j0 = piece * 1024 + threadIdx.x;
    u32x4_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j0 + 256 * u < page) w[u] = __builtin_nontemporal_load(from + j0 + 256 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j0 + 256 * u < page) __builtin_nontemporal_store(w[u], to + j0 + 256 * u);
  }
}

// Leading pages that sequence b and the one before it both name and fill.
__global__ void __launch_bounds__(64)
shared_kernel(Cache c, int min_pages, const int32_t* __restrict__ ids, const int32_t* __restrict__ tables,
              const int32_t* __restrict__ lens, int32_t* __restrict__ shared) {
  const int b = blockIdx.x, lane = threadIdx.x;
  int same = 0;
  if (b > 0) {
    const int s0 = ids ? ids[b - 1] : b - 1, s1 = ids ? ids[b] : b;
    if (in_range(s0, c.seqs) && in_range(s1, c.seqs)) {
      const int full = min(clamp_len(lens[s0], c), clamp_len(lens[s1], c)) / c.page;
      const int32_t *t0 = tables + (size_t)s0 * c.max_pages, *t1 = tables + (size_t)s1 * c.max_pages;
      for (; same < full; same += 64) {
        const int j = same + lane;
        const uint64_t differ = __ballot(j >= full || t0[j] != t1[j] || !in_range(t0[j], c.pages));
        if (differ) {
          same += __ffsll((unsigned long long)differ) - 1;
          break;
        }
      }
    }
  }
  if (lane == 0) shared[b] = same < min_pages ? 0 : same;
}

struct CacheSpace {                    // the workspace of reserve and compact
  int32_t *plan, *src, *dst, *renamed;
  ReserveCopy* copies;
};

CacheSpace cache_space(const Cache& c, void* ws) {
  int32_t* p = (int32_t*)ws;
  const size_t n = ((size_t)c.pages + 63) & ~(size_t)63;
  return CacheSpace{p, p + 64, p + 64 + n, p + 64 + 2 * n, (ReserveCopy*)(p + 64 + 3 * n)};
}

}  // namespace

size_t cache_workspace_bytes(const Cache& c) {
  const size_t n = ((size_t)c.pages + 63) & ~(size_t)63;
  return (64 + 3 * n) * sizeof(int32_t) + kPlan * sizeof(ReserveCopy);
}

hipError_t launch_cache_fork(const Cache& c, int n, const int32_t* src, const int32_t* dst, int32_t* tables, int32_t* lens,
                             int32_t* refs, int32_t* done, hipStream_t st) {
  fork_kernel<<<n, 256, 0, st>>>(c, n, src, dst, tables, lens, refs, done);
  return hipGetLastError();
}

hipError_t launch_cache_trim(const Cache& c, int n, const int32_t* ids, const int32_t* new_lens, int32_t* tables, int32_t* lens,
                             int32_t* refs, hipStream_t st) {
  trim_kernel<<<n, 256, 0, st>>>(c, ids, new_lens, tables, lens, refs);
  return hipGetLastError();
}

hipError_t launch_cache_reserve(const Cache& c, int bits, int n, const int32_t* ids, const int32_t* counts, int32_t* tables, int32_t* lens,
                                int32_t* refs, int32_t* granted, void* pool, void* ws, hipStream_t st) {
  const CacheSpace w = cache_space(c, ws);
  reserve_plan_kernel<<<1, kPlan, 0, st>>>(c, n, ids, counts, tables, lens, refs, granted, w.src, w.copies);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((c.planes * c.kv_heads + kCopyHeads - 1) / kCopyHeads), n);
  if (bits == 16) reserve_copy_kernel<true><<<grid, 256, 0, st>>>(c, bits, w.copies, (uint16_t*)pool);
  else reserve_copy_kernel<false><<<grid, 256, 0, st>>>(c, bits, w.copies, (uint16_t*)pool);
  return hipGetLastError();
}

hipError_t launch_cache_append(const Cache& c, int n, int tokens, const int32_t* ids, const int32_t* counts, const void* k,
                               const void* v, const int32_t* tables, const int32_t* lens, void* kp, void* vp, hipStream_t st) {
  const uint16_t *kk = (const uint16_t*)k, *vv = (const uint16_t*)v;
  uint16_t *ko = (uint16_t*)kp, *vo = (uint16_t*)vp;
  if (tokens < kManyTokens) {
    const int rows = n * c.kv_heads * tokens, per = 256 / (c.head_dim / 8);
    append_kernel<<<(unsigned)(((int64_t)rows + per - 1) / per), 256, 0, st>>>(c, rows, tokens, ids, counts, kk, vv, tables, lens, ko, vo);
    return hipGetLastError();
  }
  const int tile = append_tile(c.head_dim), tiles = (tokens + tile - 1) / tile;
  const auto run = [&](auto kernel) {
    kernel<<<(unsigned)(n * c.kv_heads * tiles), 256, 0, st>>>(c, tokens, tiles, ids, counts, kk, vv, tables, lens, ko, vo);
    return hipGetLastError();
  };
  return c.head_dim == 64 ? run(append_tile_kernel<64>) : c.head_dim == 96 ? run(append_tile_kernel<96>) : run(append_tile_kernel<128>);
}

hipError_t launch_cache_compact(const Cache& c, int bits, int32_t* tables, int32_t* refs, void* pool, int32_t* live, void* ws,
                                hipStream_t st) {
  const CacheSpace w = cache_space(c, ws);
  compact_plan_kernel<<<1, kPlan, 0, st>>>(c, refs, live, w.plan, w.src, w.dst, w.renamed);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_move_kernel<<<2048, 256, 0, st>>>(c, w.plan, w.src, w.dst, w.renamed, tables, (u32x4_t*)pool, (int64_t)c.kv_heads * page_chunks(c, bits));
  return hipGetLastError();
}

hipError_t launch_cache_shared(const Cache& c, int batch, int min_pages, const int32_t* ids, const int32_t* tables,
                               const int32_t* lens, int32_t* shared, hipStream_t st) {
  shared_kernel<<<batch, 64, 0, st>>>(c, min_pages, ids, tables, lens, shared);
  return hipGetLastError();
}

}  // namespace wise
