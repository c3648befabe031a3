// qprefix.hip — attention of a batch's newest tokens over a paged cache whose keys and
// values are held in 8 or 4 bits (the causal attention of the paper's Section 3, eq.
// recurrent_attention, over what is kept of them).  The plan, the pieces and their
// join are those of the cache in bf16 (prefix_plan.hpp); here is a piece of work.
//
// What is kept is exact in bf16 (a code has at most 4 significant bits, the scale is a
// power of two), so each value is widened to bf16 in a register, two an instruction, right before
// the matrix cores take it, and nothing else is rounded that the cache in bf16 does
// not round: o, and the probabilities, which enter the product with V with 16 bits.
#include "kept.hpp"
#include "prefix_plan.hpp"

namespace wise {
namespace {

// ---------------------------------------------------------------------------
// A piece of up to 16 NT rows.  A wave takes every fourth tile of 32 keys (S^T = K Q^T and
// O^T = V^T P^T in 16x16x32 MFMAs, queries in columns).  The sums may run in
// any order, which the layout uses twice:
//   K  lane (n, g), g = lane / 16, loads the quarter g of key n's dims, D / 4 of
//      them; eight at a time are its slice of the A operand, and of Q it holds the same dims
//   V  the scores end up as keys 4 g .. 4 g + 3 of each 16-key half at one query, which is
//      a slice of the B operand as it stands; the lane loads the same four tokens at dims
//      (D / 16) n .., widens a pair of dims of all eight keys, and two permutes a register make the A
//      operands of two MFMAs, row m of the t-th being dim (D / 16) m + t
// kAhead tiles are in flight in registers.
// ---------------------------------------------------------------------------
constexpr int kAhead = 2;

template <int D, int B>
struct Raw {                           // a lane's share of a tile of 32 keys
  uint32_t k[2][Kept<D, B>::kWords], v[2][Kept<D, B>::kWords];
  uint32_t ks[2][D == 96 ? 2 : 1], vs[2][D == 96 ? 2 : 1];
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

// threadIdx.x, unknown to the compiler, which would else keep what a piece computes from it
// over the loop over pieces.
__device__ __forceinline__ int fresh_tid() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

template <int D, int B, int NT, bool kAlone>
__device__ __forceinline__ void stream_piece(const Args& x, const Piece& p, float* lds) {
  using L = Kept<D, B>;
  constexpr int kC = D / 32, kT = D / 16, kStride = D + 4, kRows = 16 * NT, kWords = L::kWords;
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
    const uint16_t* row = x.q + (((size_t)b * x.c.kv_heads + kh) * rows + w) * D + D / 4 * g;
#pragma unroll
    for (int i = 0; i < kC; ++i) qf[u][i] = *(const u32x4_t*)(row + 8 * i);
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
  const int page_bytes = page * (L::kRow + L::kScales);
  const int k_code = (4 * n + g) * L::kPiece, v_code = lane * L::kPiece;
  const int k_scale = n * L::kScales + D / 4 * g / 32, k_last = n * L::kScales + (D / 4 * g + D / 4 - 8) / 32;
  const int v_scale = 4 * (g * L::kScales + D / 16 * n / 32), v_last = 4 * (g * L::kScales + (D / 16 * n + D / 16 - 2) / 32);
  const char *kp = (const char*)x.kp, *vp = (const char*)x.vp;
  auto half = [&](int i, int s, bool& ok, size_t& scales) {   // bytes of a plane before the codes, the scales, of half s of tile i
    const int id = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + s);
    const int t = (begin + stride * i + 16 * s) & (page - 1);
    ok = id >= 0;
    const size_t head = ((size_t)(ok ? id : 0) * x.c.kv_heads + kh) * page_bytes;
    scales = head + page * L::kRow + t * L::kScales;
    return head + t * L::kRow;
  };
  Raw<D, B> raw[kAhead];
  auto load_k = [&](int i, Raw<D, B>& w) {
    if ((i & 31) == 0) load_ids(i);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      size_t scales;
      const size_t codes = half(i, s, w.ok[s], scales);
      load_words<kWords>(kp + codes + k_code, w.k[s]);
      w.ks[s][0] = *(const uint8_t*)(kp + scales + k_scale);
      if constexpr (D == 96) w.ks[s][1] = *(const uint8_t*)(kp + scales + k_last);
    }
  };
  auto load_v = [&](int i, Raw<D, B>& w) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bool ok;
      size_t scales;
      const size_t codes = half(i, s, ok, scales);
      load_words<kWords>(vp + codes + v_code, w.v[s]);
      w.vs[s][0] = *(const uint32_t*)(vp + scales + v_scale);
      if constexpr (D == 96) w.vs[s][1] = *(const uint32_t*)(vp + scales + v_last);
    }
  };
  // Past its last tile a wave loads what page 0 holds, which nothing uses.
  if (tiles > 0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      load_k(i, raw[i]);
      load_v(i, raw[i]);
    }
  }
  uint32_t poison = 0;                              // NaN values set aside
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
    if (masked) {
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key0 + 16 * h + 4 * g + r >= see[u] || !(h ? ok1 : ok0)) s[u][h][r] = -INFINITY;
      // Values that no row sees may be anything, and NaN must not reach the rows that don't see
      // it (0 * NaN is NaN): they count as 0 or as some number, and the rows that see NaN get it at the end.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = min(max(p.k1 - (key0 + 16 * h + 4 * g), 0), 4);
        const uint32_t keep = !(h ? ok1 : ok0) || left == 0 ? 0u : ~0u >> (32 - 8 * left);
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
            poison |= bad;
            w.v[h][j] &= ~bad;
          }
        }
      }
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
#pragma unroll
    for (int b = 0; b < L::kPairs; ++b) {
      uint32_t y[8];                                // the pair of dims of all keys
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t word = w.vs[e >> 2][0];
        uint32_t sw = word;
        if constexpr (D == 96) {                    // pair 1 of piece 5 lies in the next scale
          const uint32_t last = w.vs[e >> 2][1];
          sw = b == 0 ? word : b == 2 || n == 5 ? last : word;
        }
        y[e] = widen_at<B>(w.v[e >> 2], scale_of(sw, e & 3), (e & 3) * L::kPairs + b);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4_t f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], c ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int u = 0; u < NT; ++u) o[u][2 * b + c] = mfma16x16x32(f, pr[u], mfma16x16x32(f, pb[u], o[u][2 * b + c]));
      }
    }
    load_v(i + kAhead, w);
  };
  for (int i = 0; i < tiles; i += kAhead) {
    tile(i, raw[0]);
    if (i + 1 >= tiles) break;
    tile(i + 1, raw[1]);
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
    if (poisoned) put_nan<D, B>(x, table, kh, p.k0, min(p.see + (p.row0 + r) % rows % x.a.q_len, p.k1), d, sum);
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

template <int D, int B, int NT, bool kShared>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
qpiece_kernel(Args x) {
  constexpr int kJoin = 4 * 16 * (kShared ? 2 : NT) * (D + 6) * 4;
  __shared__ __attribute__((aligned(1024))) char smem[kJoin];
  static_assert(sizeof(Plan<256>) <= sizeof(smem), "the plan fits");
  __shared__ Piece todo[kTodo];
  const int count = my_pieces(x, todo, smem);
  for (int i = 0; i < count; ++i) {
    Piece p = todo[i];
    int32_t* w = (int32_t*)&p;                     // the same in every lane
#pragma unroll
    for (int j = 0; j < 11; ++j) w[j] = __builtin_amdgcn_readfirstlane(w[j]);
    if (i > 0) __syncthreads();                     // the piece before has left the LDS
    if (kShared && p.see == kSeeAll) {
      Piece s = p;
      for (int r = 0; r < p.rows; r += 32) {
        if (r > 0) __syncthreads();
        s.row0 = p.row0 + r;
        s.rows = min(32, p.rows - r);
        stream_piece<D, B, 2, false>(x, s, (float*)smem);
      }
    } else if (p.kind == kNarrow) {
      stream_piece<D, B, NT, true>(x, p, (float*)smem);
    } else {
      stream_piece<D, B, NT, false>(x, p, (float*)smem);
    }
  }
}

template <int D, int B, int NT>
hipError_t launch(const Args& x, hipStream_t st) {
  const int64_t rows = (int64_t)x.a.batch * x.a.heads * x.a.q_len;
  if (x.mode == kPlanned) {
    plan_kernel<<<1, kPlan, 0, st>>>(x);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t pieces = (int64_t)x.most * x.c.kv_heads, hold = kHold;
  const unsigned grid = (unsigned)std::min(pieces, std::max(hold, (pieces + kTodo - 1) / kTodo));
  if (x.shared != nullptr) qpiece_kernel<D, B, NT, true><<<grid, 256, 0, st>>>(x);
  else qpiece_kernel<D, B, NT, false><<<grid, 256, 0, st>>>(x);
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
  const Args x = make_args(c, a, kept_key_bytes(c.head_dim, bits), q, kp, vp, tables, lens, ids, shared, o, lse, ws);
  const auto run = [&](auto d, auto b) {
    constexpr int D = decltype(d)::value, B = decltype(b)::value;
    return x.tile == 16 ? launch<D, B, 1>(x, st) : launch<D, B, 2>(x, st);
  };
  const auto by_dim = [&](auto b) {
    return c.head_dim == 64   ? run(std::integral_constant<int, 64>{}, b)
           : c.head_dim == 96 ? run(std::integral_constant<int, 96>{}, b)
                              : run(std::integral_constant<int, 128>{}, b);
  };
  return bits == 4 ? by_dim(std::integral_constant<int, 4>{}) : by_dim(std::integral_constant<int, 8>{});
}

}  // namespace wise
