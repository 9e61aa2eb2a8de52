// Decoding over a paged KV cache for gfx950 where groups of consecutive sequences
// share a prefix, as the samples of one prompt do: the S queries of each sequence
// attend to the prefix_lens[g] keys of their group's prefix, to the cache_lens[b]
// keys of their own, and, if given, to the block's own S keys.
//
// The softmax splits over any partition of the keys: with (m, l, o) the maximum,
// sum and unnormalised output over a part,
//   M = max_i m_i,  O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.
// So the prefix is taken once for the n G S query rows that all members have for
// a KV head, and its K and V are read once a group instead of once a sequence
// (more than 32 TW rows: once for each TW waves, which run at about the same time).  One launch
// does the prefixes, one the sequences' own keys, both by the paged kernel
// (paged.hpp), and a third joins the partial results of both.
#include "paged.hpp"

namespace bd {
namespace {

struct MergeParams {
  DecParams own, pre;  // pre: desc, part and grows of the prefixes
  const SharedRef* refs;
  const int* members;  // sequences that are in a group
};

// A running (maximum, sum, output) of one query row and four features.
struct MergeState {
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ void add(float m2, float l2, const f32x4& o2) {
    const float mn = fmaxf(m, m2);
    const float a = m == mn ? 1.f : fast_exp2(m - mn), c = m2 == mn ? 1.f : fast_exp2(m2 - mn);
    l = l * a + l2 * c;
    o = o * a + o2 * c;
    m = mn;
  }
};

// Partial result of row r of a slot that starts at row `slot`, features 4 q4 ...: rows of
// D + 4 floats, or (COLS) for each 32 rows [D / 4][32] float4 and [32] pairs, as the kernels leave them.
template <int D, bool COLS>
__device__ inline void merge_part(MergeState& s, const float* part, size_t slot, int r, int q4) {
  constexpr int PST = D + 4;
  if constexpr (COLS) {
    const float* ps = part + (slot + (r & ~31)) * PST;
    const float2 ml = *reinterpret_cast<const float2*>(ps + 32 * D + 2 * (r & 31));
    s.add(ml.x, ml.y, *reinterpret_cast<const f32x4*>(ps + 4 * (32 * q4 + (r & 31))));
  } else {
    const float* ps = part + (slot + r) * PST;
    const f32x4 x = *reinterpret_cast<const f32x4*>(ps + D);
    s.add(x[0], x[1], *reinterpret_cast<const f32x4*>(ps + 4 * q4));
  }
}

// One thread per (query row, 4 features, part of the runs), as dec_combine_kernel:
// P threads take every P-th run of the row's own item and of its prefix's and meet
// in LDS in part order.
template <int D, int P, bool OWN_COLS, bool PRE_COLS>
__global__ __launch_bounds__(256) void shared_merge_kernel(MergeParams p) {
  constexpr int NT = 256, TPR = D / 4, RPW = NT / (TPR * P);
  static_assert(RPW >= 1, "a workgroup holds whole rows");
  constexpr bool COLS = (OWN_COLS || PRE_COLS) && RPW > 1;  // consecutive threads take consecutive rows
  constexpr int APART = COLS ? RPW * TPR : TPR;
  __shared__ f32x4 so[P > 1 ? NT : 1];
  __shared__ float2 sml[P > 1 ? NT : 1];
  const int tid = threadIdx.x;
  const int q4 = COLS ? tid / RPW % TPR : tid % TPR, part = COLS ? tid / APART : tid / TPR % P;
  const size_t qrow = (size_t)blockIdx.x * RPW + (COLS ? tid % RPW : tid / (TPR * P));
  const int GS = p.own.G * p.own.S;
  const bool live = qrow < (size_t)p.own.B * p.own.Hkv * GS;
  MergeState s;
  if (live) {
    const int R = (int)(qrow % GS);
    const size_t bh = qrow / GS;
    const int g = R / p.own.grows, b = (int)(bh / p.own.Hkv), h = (int)(bh - (size_t)b * p.own.Hkv);
    const DecRuns d = p.own.desc[bh * p.own.ng + g];
    DecRuns e = {0, -1};
    int r2 = 0, item = 0;
    if (b < *p.members) {
      const SharedRef ref = p.refs[b];
      const int G2 = (ref.row0 + R) / p.pre.grows;
      r2 = ref.row0 + R - G2 * p.pre.grows;
      item = ref.item0 + h * ref.ng + G2;
      e = p.pre.desc[item];
    }
#pragma unroll 4
    for (int gw = d.first + part; gw <= d.last; gw += P)
      merge_part<D, OWN_COLS>(s, p.own.part, dec_slot_row(p.own, gw, bh, g), R - g * p.own.grows, q4);
#pragma unroll 4
    for (int gw = e.first + part; gw <= e.last; gw += P)
      merge_part<D, PRE_COLS>(s, p.pre.part, (size_t)(gw + item) * p.pre.grows, r2, q4);
  }
  if constexpr (P > 1) {
    so[tid] = s.o;
    sml[tid] = float2{s.m, s.l};
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int u = 1; u < P; ++u) {
      const float2 ml = sml[tid + u * APART];
      s.add(ml.x, ml.y, so[tid + u * APART]);
    }
  }
  if (!live) return;
  const bool none = !(s.l > 0.f);
  const float inv = none ? 0.f : 1.f / s.l;
  st_bf16x4(p.own.O + qrow * D + 4 * q4, s.o[0] * inv, s.o[1] * inv, s.o[2] * inv, s.o[3] * inv);
  if (q4 == 0) p.own.LSE[qrow] = none ? -INFINITY : (s.m + __log2f(s.l)) * LN2;
}

template <int D, int P, bool OWN_COLS, bool PRE_COLS>
void launch_merge_as(const MergeParams& p, hipStream_t st) {
  constexpr int RPW = 256 / (D / 4 * P);
  const size_t rows = (size_t)p.own.B * p.own.Hq * p.own.S;
  hipLaunchKernelGGL((shared_merge_kernel<D, P, OWN_COLS, PRE_COLS>), dim3((unsigned)((rows + RPW - 1) / RPW)), dim3(256), 0,
                     st, p);
}
template <int D, int P>
void launch_merge(const MergeParams& p, bool own_cols, bool pre_cols, hipStream_t st) {
  if (own_cols) {
    if (pre_cols) launch_merge_as<D, P, true, true>(p, st);
    else launch_merge_as<D, P, true, false>(p, st);
  } else {
    if (pre_cols) launch_merge_as<D, P, false, true>(p, st);
    else launch_merge_as<D, P, false, false>(p, st);
  }
}

template <int D>
hipError_t launch_shared_d(const DecodeShape& s, const SharedArgs& a, void* ws, hipStream_t st) {
  char* const pre_ws = static_cast<char*>(ws) + shared_own_bytes(s);
  const DecodeGroups g = decode_groups(s);
  const PagedParams own = paged_params(s, g, a.own, ws);

  const int waves = shared_waves(s, a.groups);
  const DecodeGroups gp = {waves, 1, DEC_QT * waves, DEC_WAVES / waves};
  PagedArgs pa = a.own;
  pa.table = a.table;
  pa.width = a.width;
  pa.table_stride = a.table_stride;
  pa.cache_lens = a.lens;
  pa.Kn = pa.Vn = nullptr;
  PagedParams pre = paged_params(s, gp, pa, ws);
  const size_t items = shared_items(s, a.groups);
  pre.d.B = a.groups;
  pre.d.C = a.width << a.own.pages.log_size;
  pre.d.desc = reinterpret_cast<DecRuns*>(pre_ws);
  pre.d.part = reinterpret_cast<float*>(pre_ws + shared_desc_bytes(s, a.groups));
  pre.sizes = a.sizes;
  pre.seqs = s.B;
  pre.refs = reinterpret_cast<SharedRef*>(pre_ws) + items;
  pre.members = reinterpret_cast<int*>(pre.refs + s.B);

  hipError_t e = launch_paged_runs<D, PagedMode::Prefix>(gp, pre, st);
  if (e != hipSuccess) return e;
  e = launch_paged_runs<D, PagedMode::Own>(g, own, st);
  if (e != hipSuccess) return e;
  const MergeParams m = {own.d, pre.d, pre.refs, pre.members};
  // (as launch_dec_combine: eight runs or more an item)
  const bool many = decode_items(s) * 8 <= (size_t)g.runs || (size_t)s.Hkv * a.groups * 8 <= (size_t)gp.runs;
  if (many) launch_merge<D, 8>(m, g.waves > 1, waves > 1, st);
  else launch_merge<D, 1>(m, g.waves > 1, waves > 1, st);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_decode(const DecodeShape& s, const SharedArgs& a, void* ws, hipStream_t st) {
  return s.D == 128 ? launch_shared_d<128>(s, a, ws, st) : launch_shared_d<64>(s, a, ws, st);
}

}  // namespace bd
