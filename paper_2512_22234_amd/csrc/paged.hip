// Decoding over a paged KV cache for gfx950: the S queries of each sequence
// attend to the first cache_lens[b] keys of its pages (row b of the page table)
// and, if given, to the block's own S keys.  A page outside the pool holds no
// keys; a row that sees no key at all gets O = 0 and LSE = -inf.
#include "device.hpp"
#include "kernels.hpp"

namespace bd {
namespace {

struct PagedParams {
  PagedArgs a;
  int B, S, Hq, Hkv, G;
  float c;  // scale * log2(e)
};

// One wave per query row: the keys one after another, a lane holds D / 64
// features, running maximum and sum of the softmax.
template <int D>
__global__ __launch_bounds__(64) void paged_row_kernel(PagedParams p) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x;
  const unsigned row = blockIdx.x;  // (b * Hq + h) * S + s
  const int bh = (int)(row / (unsigned)p.S), b = bh / p.Hq, h = bh - b * p.Hq, hkv = h / p.G;
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = (float)static_cast<const bf16*>(p.a.Q)[(size_t)row * D + lane * E + e];
    o[e] = 0.f;
  }
  auto key = [&](const bf16* k, const bf16* v) {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) x += q[e] * (float)k[lane * E + e];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    x *= p.c;
    const float mn = fmaxf(m, x), al = m == mn ? 1.f : fast_exp2(m - mn), w = fast_exp2(x - mn);
    l = l * al + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * al + w * (float)v[lane * E + e];
    m = mn;
  };
  const PageLayout& g = p.a.pages;
  const int len = imin(imax(p.a.cache_lens[b], 0), p.a.width << g.log_size);
  for (int j = 0; j < len; ++j) {
    const int id = p.a.table[b * p.a.table_stride + (j >> g.log_size)];
    if (id < 0 || id >= g.num) continue;
    const int64_t at = id * g.sp + hkv * g.sh + (j & ((1 << g.log_size) - 1)) * g.sr;
    key(static_cast<const bf16*>(p.a.Kp) + at, static_cast<const bf16*>(p.a.Vp) + at);
  }
  if (p.a.Kn)
    for (int j = 0; j < p.S; ++j) {
      const size_t at = (((size_t)b * p.Hkv + hkv) * p.S + j) * D;
      key(static_cast<const bf16*>(p.a.Kn) + at, static_cast<const bf16*>(p.a.Vn) + at);
    }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) static_cast<bf16*>(p.a.O)[(size_t)row * D + lane * E + e] = (bf16)(o[e] * inv);
  if (lane == 0) p.a.LSE[row] = l > 0.f ? (m + __log2f(l)) * LN2 : -INFINITY;
}

}  // namespace

hipError_t launch_paged_decode(const DecodeShape& s, const PagedArgs& a, void* ws, hipStream_t st) {
  (void)ws;
  const PagedParams p{a, s.B, s.S, s.Hq, s.Hkv, s.Hq / s.Hkv, s.scale * LOG2E};
  const dim3 grid((unsigned)((size_t)s.B * s.Hq * s.S));
  if (s.D == 128) hipLaunchKernelGGL((paged_row_kernel<128>), grid, dim3(64), 0, st, p);
  else hipLaunchKernelGGL((paged_row_kernel<64>), grid, dim3(64), 0, st, p);
  return hipGetLastError();
}

}  // namespace bd
