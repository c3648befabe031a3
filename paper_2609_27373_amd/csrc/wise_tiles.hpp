// wise_tiles.hpp — the tile engine of the attention kernels.
//
// A wave owns 32 consecutive queries.  For each tile of 64 keys (32 for 32-key
// blocks) it computes S^T = K Q^T with v_mfma_f32_32x32x16_bf16 (A = K from
// LDS, B = Q^T held in registers for the whole row), so every lane ends up
// holding 32 scores of ONE query.  The row max needs one cross-lane step
// (lanes l and l^32 share a query), the row sum none until the end, and the
// probabilities are already in the B-operand layout of O^T = V^T P^T: they are
// packed to bf16 in place and fed straight to the second MFMA chain.  V stays
// row-major in LDS and its A-operand fragments are read transposed with
// ds_read_b64_tr_b16; row pads (2-wave dense and grouped kernels, which stage
// tiles through registers) or permuted rows (Swizzle, the others) make those
// reads, like the 128-bit K reads, free of bank conflicts.  Softmax is
// online in base 2 with the exact running max (so the largest probability of
// a row is exactly 1 in bf16); the O rescale is skipped, wave-uniformly, on
// tiles that raise no row's max.
#pragma once

#include <type_traits>

#include "wise_device.hpp"

namespace wise {

// ---------------------------------------------------------------------------
// Global -> register -> LDS staging of one tile of 64 keys (K rows permuted so
// the S^T accumulator comes out in PV operand order; V rows in natural order).  Loads for the next tile are
// issued before the current one is computed, so the memory latency hides
// behind the MFMA work; stores go to an LDS tile no wave still reads: after
// the barrier that retires it, or, in the 8-wave grouped late step, into its
// second buffer.  Used by that kernel's groups and the 2-wave dense group.
// ---------------------------------------------------------------------------
template <int D, int NT>
struct TileStage {
  using G = Geo<D>;
  static constexpr int kRowChunks = D / 8;                    // 16-B chunks per key row
  static constexpr int kChunks = kKeyTile * kRowChunks;       // per tensor
  static constexpr int kPer = (kChunks + NT - 1) / NT;

  u32x4_t kr[kPer];
  u32x4_t vr[kPer];

  // Chunk i of this thread: key row ch / kRowChunks, column (ch % kRowChunks) * 8.
  __device__ __forceinline__ static int chunk(int tid, int i) { return tid + i * NT; }
  __device__ __forceinline__ static bool live(int tid, int i) {
    return kChunks % NT == 0 || chunk(tid, i) < kChunks;
  }

  // rk, rv: the head's K and V; key0: this tile's first key row (uniform,
  // a scalar byte offset), per-lane offsets constant across tiles.
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv,
                                       int key0, int tid) {
    const uint32_t soff = (uint32_t)key0 * (D * 2);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (live(tid, i)) {
        const int ch = chunk(tid, i);
        const uint32_t off = (uint32_t)((ch / kRowChunks) * D + (ch % kRowChunks) * 8) * 2;
        kr[i] = buffer_load16(rk, off, soff);
        vr[i] = buffer_load16(rv, off, soff);
      }
    }
  }

  __device__ __forceinline__ void store(uint16_t* ks, uint16_t* vs, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (live(tid, i)) {
        const int ch = chunk(tid, i);
        const int key = ch / kRowChunks, c8 = (ch % kRowChunks) * 8;
        *(u32x4_t*)(ks + k_lds_row(key) * G::kKStride + c8) = kr[i];
        *(u32x4_t*)(vs + key * G::kVStride + c8) = vr[i];
      }
    }
  }
};

// Global -> LDS copies of one 64-key tile by NW waves into the swizzled layout:
// copy i of wave w fills 1 KB at (w * kPer + i) * 1024.
template <int D, int NW>
struct TileCopy {
  using S = Swizzle<D>;
  static constexpr int kPer = S::kTile / 1024 / NW;
  static_assert(S::kTile % (1024 * NW) == 0, "whole copies per wave");
  uint32_t ko[kPer], vo[kPer];                        // this lane's source bytes in a tile

  __device__ __forceinline__ void init(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = (wave * kPer + i) * 1024 + lane * 16;
      const int row = at / S::kRow, slot = at % S::kRow / 16;
      ko[i] = k_lds_row(row) * S::kRow + S::k_chunk(row, slot) * 16;
      vo[i] = row * S::kRow + (S::v_block(row, slot >> 2) * 4 + (slot & 3)) * 16;
    }
  }
  // One copy of tile `tile`'s K (V) into the buffer at LDS address `lds`.
  __device__ __forceinline__ void k1(u32x4_t r, int tile, uint32_t lds, int wave, int i) const {
    copy16_to_lds(r, ko[i], (uint32_t)tile * S::kTile, lds + (uint32_t)(wave * kPer + i) * 1024);
  }
  __device__ __forceinline__ void v1(u32x4_t r, int tile, uint32_t lds, int wave, int i) const {
    copy16_to_lds(r, vo[i], (uint32_t)tile * S::kTile, lds + (uint32_t)(wave * kPer + i) * 1024);
  }
  __device__ __forceinline__ void k(u32x4_t r, int tile, uint32_t lds, int wave) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) k1(r, tile, lds, wave, i);
  }
  __device__ __forceinline__ void v(u32x4_t r, int tile, uint32_t lds, int wave) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v1(r, tile, lds, wave, i);
  }
};

// LDS byte offsets of a lane's operand reads in a swizzled tile: K fragment
// (chunk c, half u) at k[c] + u * 32 rows, V fragment (k-step, dims 32 t) at
// v[t] + 16 ks rows (and 4 rows further).
template <int D>
struct ReadAddr {
  using S = Swizzle<D>;
  uint32_t k[D / 16], v[D / 32];
  __device__ __forceinline__ void init(int lane) {
    const int m = lane & 31, h = lane >> 5, r = 8 * h + ((lane >> 2) & 3);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) k[c] = m * S::kRow + S::k_chunk(m, 2 * c + h) * 16;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
      v[t] = r * S::kRow + S::v_block(r, t) * 64 + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
  }
};

// Tile-local key held by register r of S^T tile t in a lane of half-wave h.
__device__ __forceinline__ int score_key(int t, int r, int h) {
  const int j = r >> 2, i = r & 3;
  return 32 * t + 16 * (j >> 1) + 8 * h + 4 * (j & 1) + i;
}

// ---------------------------------------------------------------------------
// Per-wave state and steps of the tile engine.
// ---------------------------------------------------------------------------
template <int D>
struct WaveRows {
  using G = Geo<D>;
  u32x4_t qf[G::kDChunks];   // Q^T B-operand fragments, one per 16-dim chunk
  f32x16_t o[G::kDTiles];    // O^T accumulator, 32 dims x 32 queries per tile
  float m;                   // running max of scale*log2(e)*s (per query)
  float l;                   // running sum over this lane's half of the keys
  float hs[4];               // last tile's per-part sums (softmax_pv<H, P>, P > 0)

  __device__ __forceinline__ void load_q(const uint16_t* qg, int q0, int lane) {
    const uint16_t* row = qg + (size_t)(q0 + (lane & 31)) * D + 8 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < G::kDChunks; ++c) qf[c] = *(const u32x4_t*)(row + 16 * c);
  }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int t = 0; t < G::kDTiles; ++t) o[t] = f32x16_t{};
    m = -INFINITY;
    l = 0.f;
  }

  // S^T of one LDS tile of 32*H keys: s[t] covers LDS rows 32t..32t+31.
  template <int H>
  __device__ __forceinline__ void scores(const uint16_t* ks, int lane, f32x16_t s[H]) const {
    const uint16_t* a0 = ks + (lane & 31) * G::kKStride + 8 * (lane >> 5);
    const uint16_t* a1 = a0 + 32 * G::kKStride;
    f32x16_t s0{}, s1{};
#pragma unroll
    for (int c = 0; c < G::kDChunks; ++c) {
      s0 = mfma32x32x16(*(const u32x4_t*)(a0 + 16 * c), qf[c], s0);
      if constexpr (H == 2) s1 = mfma32x32x16(*(const u32x4_t*)(a1 + 16 * c), qf[c], s1);
    }
    s[0] = s0;
    if constexpr (H == 2) s[1] = s1;
  }

  // Causal mask inside a tile: key0 + local key > query -> -inf.
  template <int H>
  __device__ __forceinline__ static void mask(f32x16_t s[H], int key0, int qi, int lane) {
    const int h = lane >> 5;
#pragma unroll
    for (int t = 0; t < H; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + score_key(t, r, h) > qi) s[t][r] = -INFINITY;
  }

  // Online softmax of one tile: the probabilities packed in pb, O and l
  // rescaled.  With kParts = 2 (4) the sums of this lane's probabilities over
  // each 32-key half (16-key quarter) of the tile are kept in hs[] (the row
  // sum then adds the parts).
  template <int H, int kParts = 0>
  __device__ __forceinline__ void softmax(f32x16_t s[H], u32x4_t pb[2 * H], float c) {
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < H; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    mx = pair_max(mx) * c;
    const bool grow = mx > m;
    if (__builtin_amdgcn_ballot_w64(grow)) {
      const float mn = grow ? mx : m;
      const float alpha = (mn == m) ? 1.f : fast_exp2(m - mn);
      l *= alpha;
      // In-place multiply: keeps O in the same registers on both sides of the
      // branch (a plain `*=` lets the allocator rename O and copy all of it
      // back on the path that skips the rescale).
#pragma unroll
      for (int t = 0; t < G::kDTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) asm volatile("v_mul_f32 %0, %0, %1" : "+v"(o[t][r]) : "v"(alpha));
      m = mn;
    }
    const float mb = (m == -INFINITY) ? 0.f : m;
    // The tile's probabilities are summed on their own and added to the row
    // sum once per tile: a long row (16K keys per lane at 32K) then carries
    // rounding error ~ tiles * eps instead of ~ keys * eps.
    float ts = 0.f;
#pragma unroll
    for (int t = 0; t < H; ++t) {
      float th = 0.f, tq[2] = {0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = fast_exp2(__builtin_fmaf(s[t][r], c, -mb));
        s[t][r] = p;
        if constexpr (kParts == 4) tq[r >> 3] += p;
        else if constexpr (kParts == 2) th += p;
        else ts += p;
      }
      if constexpr (kParts == 4) {
        hs[2 * t] = tq[0];
        hs[2 * t + 1] = tq[1];
        ts += tq[0] + tq[1];
      } else if constexpr (kParts == 2) {
        hs[t] = th;
        ts += th;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pb[2 * t + u][e] = pack_bf16x2(s[t][8 * u + 2 * e], s[t][8 * u + 2 * e + 1]);
    }
    l += ts;
  }

  // Softmax of one tile and O^T += V^T P^T.  A = V^T fragment: lane L needs
  // V[16ks + 8(L/32) + e][32t + L%32], e = 0..7, fetched as two transpose
  // reads of 4 keys each (see lds_read_tr16).
  template <int H, int kParts = 0>
  __device__ __forceinline__ void softmax_pv(f32x16_t s[H], const uint16_t* vt, int lane, float c) {
    u32x4_t pb[2 * H];
    softmax<H, kParts>(s, pb, c);
    const uint16_t* a = vt + (8 * (lane >> 5) + ((lane >> 2) & 3)) * G::kVStride +
                        16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int ks = 0; ks < 2 * H; ++ks)
#pragma unroll
      for (int t = 0; t < G::kDTiles; ++t) {
        const u32x2_t lo = lds_read_tr16(a + (16 * ks) * G::kVStride + 32 * t);
        const u32x2_t hi = lds_read_tr16(a + (16 * ks + 4) * G::kVStride + 32 * t);
        o[t] = mfma32x32x16(u32x4_t{lo[0], lo[1], hi[0], hi[1]}, pb[ks], o[t]);
      }
  }

  // One tile: S^T, the causal mask when the tile reaches past this wave's
  // first query (only ever on diagonal tiles, and only instantiated for
  // them), online softmax and PV.
  template <bool kMask, int H = 2, int kParts = 0>
  __device__ __forceinline__ void attend(const uint16_t* ks, const uint16_t* vt, int lane,
                                         float c, int key0, int q0) {
    f32x16_t s[H];
    scores<H>(ks, lane, s);
    if constexpr (kMask) {
      if (key0 + 32 * H - 1 > q0) mask<H>(s, key0, q0 + (lane & 31), lane);
    }
    softmax_pv<H, kParts>(s, vt, lane, c);
  }

  // S^T of a swizzled 64-key tile, and O^T += V^T P^T from one.
  __device__ __forceinline__ void scores_swizzled(const char* kt, const ReadAddr<D>& ra, f32x16_t s[2]) const {
#pragma unroll
    for (int i = 0; i < G::kDChunks; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = mfma32x32x16(*(const u32x4_t*)(kt + ra.k[i] + 32 * t * Swizzle<D>::kRow), qf[i], s[t]);
  }
  __device__ __forceinline__ void pv_swizzled(const char* vt, const ReadAddr<D>& ra, const u32x4_t pb[4]) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int t = 0; t < G::kDTiles; ++t) {
        const char* p = vt + ra.v[t] + 16 * ks * Swizzle<D>::kRow;
        const u32x2_t lo = lds_read_tr16((const uint16_t*)p);
        const u32x2_t hi = lds_read_tr16((const uint16_t*)(p + 4 * Swizzle<D>::kRow));
        o[t] = mfma32x32x16(u32x4_t{lo[0], lo[1], hi[0], hi[1]}, pb[ks], o[t]);
      }
  }

  // New running max from a tile's max mx; true (wave-uniform) when some
  // query's max grew: alpha then holds the factor of O, l is rescaled here.
  __device__ __forceinline__ bool raise_max(float mx, float& alpha) {
    const bool grow = mx > m;
    if (!__builtin_amdgcn_ballot_w64(grow)) return false;
    const float mn = grow ? mx : m;
    alpha = (mn == m) ? 1.f : fast_exp2(m - mn);
    l *= alpha;
    m = mn;
    return true;
  }

  static constexpr int kAhead = 4;               // LDS fragments in flight

  // One step of the software pipeline of the dense groups: S^T of the
  // next tile (kQk: into sn, from its K tile kn, masked by maskn) and online
  // softmax and PV of the current one (kPv: its masked scores s, their max mx,
  // its V tile vt).  The same operations in the same order as attend(), so the
  // same bits.  It is laid out in 2 kN slots of one MFMA each, the LDS reads
  // kAhead slots before their use and the exponentials, sums, packing and the
  // next tile's max spread between the MFMAs, because two waves per SIMD in
  // step leave nothing else to fill a wave's waits; mid(n, j) runs in slot j
  // (the copies).  The wave's priority falls through the step, so of the two
  // waves of a SIMD the one behind issues first and they reach the barrier
  // together.  VALU and matrix cores are then both close to full.  kSplit: PV with 16
  // bits of each probability, in two MFMAs a slot.
  template <int H, bool kQk, bool kPv, int kParts, bool kSplit = false, class Mid, class Mask>
  __device__ __forceinline__ void step(const char* kn, const char* vt, const ReadAddr<D>& ra, int lane, float c,
                                       f32x16_t s[H], f32x16_t sn[H], float& mx, Mid mid, Mask maskn) {
    constexpr int kN = G::kDChunks * H;          // MFMAs of S^T; PV has as many
    constexpr int kPairs = 8 * H;
    u32x4_t kf[kN], vf[kN], pb[2 * H], pr[2 * H];
    auto read_k = [&](int j) {
      kf[j] = *(const u32x4_t*)(kn + ra.k[j / H] + (j % H) * 32 * Swizzle<D>::kRow);
    };
    auto read_v = [&](int j) {
      const int ks = j / G::kDTiles, t = j % G::kDTiles;
      const char* p = vt + ra.v[t] + 16 * ks * Swizzle<D>::kRow;
      const u32x2_t lo = lds_read_tr16((const uint16_t*)p);
      const u32x2_t hi = lds_read_tr16((const uint16_t*)(p + 4 * Swizzle<D>::kRow));
      vf[j] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    };
    float mb = 0.f, ts = 0.f, tp[4] = {0.f, 0.f, 0.f, 0.f};
    // Pair k: probabilities 2k, 2k + 1 of this lane, exponentials first, sums
    // and packing a slot later.  The empty asm keeps each in its slot.
    float pv[2 * kPairs];
    auto pair_exp = [&](int k) {
      if (k >= kPairs) return;
      const int t = k / 8, r = 2 * (k % 8);
      float p0 = fast_exp2(__builtin_fmaf(s[t][r], c, -mb));
      float p1 = fast_exp2(__builtin_fmaf(s[t][r + 1], c, -mb));
      asm volatile("" : "+v"(p0), "+v"(p1));
      pv[2 * k] = p0;
      pv[2 * k + 1] = p1;
    };
    auto pair_fin = [&](int k) {
      if (k < 0 || k >= kPairs) return;
      const int t = k / 8, r = 2 * (k % 8);
      float& a = kParts == 0 ? ts : kParts == 4 ? tp[2 * t + (r >> 3)] : tp[t];
      a += pv[2 * k];
      a += pv[2 * k + 1];
      uint32_t w;
      if constexpr (kSplit) {
        uint32_t rest;
        w = split_bf16x2(pv[2 * k], pv[2 * k + 1], rest);
        asm volatile("" : "+v"(rest));
        pr[2 * t + (r >> 3)][(r & 7) >> 1] = rest;
      } else {
        w = pack_bf16x2(pv[2 * k], pv[2 * k + 1]);
      }
      asm volatile("" : "+v"(a), "+v"(w));
      pb[2 * t + (r >> 3)][(r & 7) >> 1] = w;
    };
    // Slot of the exponentials of pair k: slots 0 .. kN-1 hold the MFMAs of
    // S^T, kN .. 2 kN - 1 those of PV.
    constexpr int kS0 = 3;                        // S^T MFMAs issued before the new max is needed
    auto pairs_before = [](int slot) {           // pairs whose exponentials are done before it
      const int first = kS0, last = 2 * kN - kN / 4 - 1;   // first slot used, first slot past them
      const int x = slot <= first ? 0 : (slot - first) * kPairs / (last - first);
      return x > kPairs ? kPairs : x;
    };
    constexpr int kM0 = kN + 2;                  // first slot of the next tile's max
    auto maxes_before = [](int slot) {
      const int x = slot <= kM0 ? 0 : ((slot - kM0) * kPairs + 2 * kN - kM0 - 1) / (2 * kN - kM0);
      return x > kPairs ? kPairs : x;
    };
    if constexpr (kQk) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) read_k(j);
    }
    __builtin_amdgcn_s_setprio(3);
    float alpha = 1.f;
    bool grew = false;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      if constexpr (kQk) {
        if (j + kAhead < kN) read_k(j + kAhead);
        sn[j % H] = mfma32x32x16(kf[j], qf[j / H], j < H ? f32x16_t{} : sn[j % H]);
      }
      if constexpr (kPv) {
        if (j == kS0) {
          __builtin_amdgcn_sched_barrier(0);
          grew = raise_max(mx, alpha);
          mb = (m == -INFINITY) ? 0.f : m;
        }
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k >= pairs_before(j) && k < pairs_before(j + 1)) pair_exp(k);
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k >= pairs_before(j - 1) && k < pairs_before(j)) pair_fin(k);
        // O rescaled in place, a tile of 32 dims at a time between the MFMAs
        // (a plain `*=` lets the allocator rename O and copy all of it back on
        // the path that skips the rescale).
        constexpr int kGap = (kN - kS0) / G::kDTiles;
        if (j >= kS0 && (j - kS0) % kGap == 0 && (j - kS0) / kGap < G::kDTiles) {
          const int t = (j - kS0) / kGap;
          if (grew) {
#pragma unroll
            for (int r = 0; r < 16; ++r) asm volatile("v_mul_f32 %0, %0, %1" : "+v"(o[t][r]) : "v"(alpha));
          }
        }
        if (j + kAhead >= kN) read_v(j + kAhead - kN);
      }
      mid(std::integral_constant<int, 2 * kN>{}, j);
      if (j == kN / 2) __builtin_amdgcn_s_setprio(2);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(1);
    if constexpr (kQk) maskn(sn);
    __builtin_amdgcn_sched_barrier(0);
    float mn = -INFINITY;
#pragma unroll
    for (int j = kN; j < 2 * kN; ++j) {
      if constexpr (kPv) {
        const int i = j - kN;
        if (i + kAhead < kN) read_v(i + kAhead);
        o[i % G::kDTiles] = mfma32x32x16(vf[i], pb[i / G::kDTiles], o[i % G::kDTiles]);
        if constexpr (kSplit) o[i % G::kDTiles] = mfma32x32x16(vf[i], pr[i / G::kDTiles], o[i % G::kDTiles]);
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k >= pairs_before(j) && k < pairs_before(j + 1)) pair_exp(k);
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k >= pairs_before(j - 1) && k < pairs_before(j)) pair_fin(k);
      }
      if constexpr (kQk) {
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
          if (k >= maxes_before(j) && k < maxes_before(j + 1)) {
            mn = fmaxf(fmaxf(mn, sn[k / 8][2 * (k % 8)]), sn[k / 8][2 * (k % 8) + 1]);
            asm volatile("" : "+v"(mn));
          }
      }
      mid(std::integral_constant<int, 2 * kN>{}, j);
      if (j == kN + kN / 2) __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kPv) {
      if constexpr (kParts == 4) {
#pragma unroll
        for (int t = 0; t < H; ++t) {
          hs[2 * t] = tp[2 * t];
          hs[2 * t + 1] = tp[2 * t + 1];
          ts += tp[2 * t] + tp[2 * t + 1];
        }
      } else if constexpr (kParts == 2) {
#pragma unroll
        for (int t = 0; t < H; ++t) {
          hs[t] = tp[t];
          ts += tp[t];
        }
      }
      l += ts;
    }
    if constexpr (kQk) mx = pair_max(mn) * c;
  }

  // log2 of the last tile's probability mass per query, unnormalised (taken
  // against the running max m): entries 0..3 for the four 16-key quarters
  // (E = 16), 0 and 1 for the two 32-key halves (E = 32) or entry 0 for the
  // whole tile (E = 64).  -inf for no mass.
  template <int E>
  __device__ __forceinline__ void tile_log_mass(float out[4]) const {
    if constexpr (E == 16) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float x = pair_sum(hs[t]);
        out[t] = x > 0.f ? m + __builtin_log2f(x) : -INFINITY;
      }
    } else if constexpr (E == 32) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float x = pair_sum(hs[t]);
        out[t] = x > 0.f ? m + __builtin_log2f(x) : -INFINITY;
      }
    } else {
      const float x = pair_sum(hs[0] + hs[1]);
      out[0] = x > 0.f ? m + __builtin_log2f(x) : -INFINITY;
    }
  }

  // log2 of the row normaliser: lse / ln 2.
  __device__ __forceinline__ float lse2() const { return m + __builtin_log2f(pair_sum(l)); }

  // O = O^T / l written as bf16 rows; lse in natural log.  Only the first
  // nq of the wave's 32 query columns are written.
  __device__ __forceinline__ void finish(uint16_t* og, float* lse, int q0, int lane,
                                         int nq = 32) const {
    const float lt = pair_sum(l);
    const float inv = lt > 0.f ? 1.f / lt : 0.f;
    const int q = q0 + (lane & 31), h = lane >> 5;
    if ((lane & 31) >= nq) return;
    uint16_t* row = og + (size_t)q * D + 4 * h;
#pragma unroll
    for (int t = 0; t < G::kDTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x2_t w;
        w[0] = pack_bf16x2(o[t][4 * j] * inv, o[t][4 * j + 1] * inv);
        w[1] = pack_bf16x2(o[t][4 * j + 2] * inv, o[t][4 * j + 3] * inv);
        *(u32x2_t*)(row + 32 * t + 8 * j) = w;
      }
    if (lse != nullptr && h == 0) lse[q] = lt > 0.f ? (m + __builtin_log2f(lt)) * kLn2 : -INFINITY;
  }
};

}  // namespace wise
