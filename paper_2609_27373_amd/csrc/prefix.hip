// prefix.hip — attention of a batch's newest tokens over a paged key-value
// cache (the causal attention of the paper's Section 3, eq.
// recurrent_attention, with the keys and values of earlier positions kept).
//
// One wave per query row: lanes take keys for the scores and dims for the
// output, softmax online in base 2.
#include "wise_device.hpp"
#include "wise_kernels.hpp"

namespace wise {
namespace {

__device__ __forceinline__ float bf(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }

template <int D>
__global__ void __launch_bounds__(64)
row_attn_kernel(Cache c, Queries a, float sc, const uint16_t* __restrict__ q, const uint16_t* __restrict__ kp,
                const uint16_t* __restrict__ vp, const int32_t* __restrict__ tables, const int32_t* __restrict__ lens,
                const int32_t* __restrict__ ids, uint16_t* __restrict__ o, float* __restrict__ lse) {
  const int lane = threadIdx.x, t = blockIdx.x % a.q_len, bh = blockIdx.x / a.q_len;
  const int b = bh / a.heads, h = bh % a.heads, kh = h / (a.heads / c.kv_heads);
  const int s = ids ? ids[b] : b;
  int see = 0;
  if ((unsigned)s < (unsigned)c.seqs) see = min(lens[s], c.max_pages * c.page) - a.q_len + t + 1;
  const int32_t* row = tables + (size_t)(see > 0 ? s : 0) * c.max_pages;
  const uint16_t* qr = q + (size_t)blockIdx.x * D;
  float m = -INFINITY, l = 0.f, acc[(D + 63) / 64] = {};
  for (int j0 = 0; j0 < see; j0 += 64) {
    const int j = j0 + lane;
    const int p = j < see ? row[j / c.page] : -1;
    const bool live = (unsigned)p < (unsigned)c.pages;
    const size_t at = (((size_t)(live ? p : 0) * c.kv_heads + kh) * c.page + j % c.page) * D;
    float x = -INFINITY;
    if (live) {
      x = 0.f;
      for (int e = 0; e < D; ++e) x += bf(qr[e]) * bf(kp[at + e]);
      x *= sc;
    }
    float mx = x;
    for (int w = 32; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w, 64));
    const float mn = fmaxf(m, mx), mb = mn == -INFINITY ? 0.f : mn;
    const float alpha = fast_exp2(m - mb), pr = fast_exp2(x - mb);
    m = mn;
    l = l * alpha + pr;
    for (float& y : acc) y *= alpha;
    for (int i = 0; i < 64; ++i) {
      const float pi = __shfl(pr, i, 64);
      const uint64_t ai = __shfl((unsigned long long)at, i, 64);
      if (!__shfl((int)live, i, 64)) continue;
      for (int u = 0; u < (D + 63) / 64; ++u)
        if (lane + 64 * u < D) acc[u] += pi * bf(vp[ai + lane + 64 * u]);
    }
  }
  for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w, 64);
  for (int u = 0; u < (D + 63) / 64; ++u)
    if (lane + 64 * u < D) o[(size_t)blockIdx.x * D + lane + 64 * u] = (uint16_t)pack_bf16x2(l > 0.f ? acc[u] / l : 0.f, 0.f);
  if (lse != nullptr && lane == 0) lse[blockIdx.x] = l > 0.f ? (m + __builtin_log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace

size_t prefix_workspace_bytes(const Cache&, const Queries&) { return 256; }

hipError_t launch_prefix(const Cache& c, const Queries& a, const void* q, const void* kp, const void* vp, const int32_t* tables,
                         const int32_t* lens, const int32_t* ids, const int32_t*, void* o, float* lse, void*, hipStream_t st) {
  const unsigned rows = (unsigned)a.batch * a.heads * a.q_len;
  const auto run = [&](auto kernel) {
    kernel<<<rows, 64, 0, st>>>(c, a, a.scale * kLog2e, (const uint16_t*)q, (const uint16_t*)kp, (const uint16_t*)vp, tables, lens,
                                ids, (uint16_t*)o, lse);
    return hipGetLastError();
  };
  return c.head_dim == 64 ? run(row_attn_kernel<64>) : c.head_dim == 96 ? run(row_attn_kernel<96>) : run(row_attn_kernel<128>);
}

}  // namespace wise
