// What the decode kernels over a dense and over a paged KV cache share: how the
// key tiles of all items are shared out over runs, where partial results lie,
// and the kernel that merges them.
#pragma once

#include "device.hpp"
#include "kernels.hpp"

namespace bd {
namespace {

// The runs that hold an item: first and last, or last = -1 where the decode
// kernel wrote the item directly.
struct alignas(16) DecRuns {
  int first, last;
};

struct DecParams {
  const bf16* Q;   // [B][Hq][S][D]
  const bf16* Kc;  // [B][Hkv][C][D]
  const bf16* Vc;
  const bf16* Kn;  // [B][Hkv][S][D]
  const bf16* Vn;
  const int* cache_lens;  // [B], device
  bf16* O;                // [B][Hq][S][D]
  float* LSE;             // [B][Hq][S]
  DecRuns* desc;          // [item]
  float* part;            // [row][D + 4]: unnormalised O, max (log2 units), sum
  int B, S, Hq, Hkv, G, C;
  int ng;     // row groups per (sequence, KV head)
  int grows;  // query rows of a group (a multiple of 32, at most 32 * TW)
  int hrows;  // partial rows of a (sequence, KV head): its G*S rows rounded up to 32
  int runs;   // teams of the grid
  float c;    // scale * log2(e)
};

// Cache length of sequence b, clamped to [0, C].  `lens` is p.cache_lens
// passed as a restrict kernel argument: the compiler may then read it through
// the scalar cache where the index is uniform.
__device__ inline int dec_len(const DecParams& p, const int* __restrict__ lens, int b) {
  return imin(imax(lens[b], 0), p.C);
}
// Key tiles of an item of a sequence with cache length len.
template <int KT>
__device__ inline int dec_tiles(const DecParams& p, int len) {
  return cdiv(len, KT) + cdiv(p.S, KT);
}
// Teams that take part in a call of T tiles on a grid of `runs` teams: at
// least about DEC_MIN_RUN tiles for each team of several waves, so that a short
// call is not cut into single tiles with as many partial results of its many
// rows to merge (30 sequences of 30 to 60 tokens, S = 32: 15.7 us, single tiles
// 23.0), and no run is empty (T >= 1).  One wave takes single tiles: the same
// time within 2% on one sequence of 1500 tokens, and the nearest to float64,
// since the largest P of a run is 1 exactly (relative error 2.28e-3, with two
// tiles a run 2.32e-3).
template <int TW>
__device__ inline int dec_runs(int runs, int T) {
  constexpr int DEC_MIN_RUN = TW == 1 ? 1 : 2;
  return imin(runs, cdiv(T, DEC_MIN_RUN));
}
// Keys and values of more than 288 MiB, beyond the 256 MiB of the last-level
// cache, are loaded nontemporal: nothing of them survives to the next call, and
// without their lines in L2 and the last-level cache the same bytes come faster
// (822 MB: 150 -> 132 us, 6.2 TB/s).  Smaller ones may still be there from the
// last call, as when a block is denoised step by step.  The line lies where both
// are the same (64 sequences, S = 4, default and nontemporal: 264 MiB 49.9 and
// 50.8 us, 288 MiB 52.4 and 53.9, 296 MiB 56.1 and 56.0, 312 MiB 59.9 and 58.1,
// 336 MiB 68.8 and 61.1).  It holds for rows that a call reads more than once as
// well, by the teams of a KV head's row groups: they run at about the same time
// (256 query rows per KV head: 271 MiB 125 and 131 us, 337 MiB 157 and 156, 412
// MiB 189 and 186, 768 MiB 334 and 324; 512 rows, 375 MiB, the other way round:
// 312 and 316).
constexpr size_t DEC_STREAM_BYTES = (size_t)288 << 20;
// First tile of run gw <= n (the runs cut T tiles into n near-equal pieces).
// RUNS, the teams of the grid, is a power of two, and T <= 2 n where fewer take
// part: no 64-bit division (three of them took 1 us of a call).
template <int RUNS>
__device__ inline int dec_run_start(int gw, int n, int T) {
  return n == RUNS ? (int)(((long long)gw * T) / RUNS) : (int)((unsigned)(gw * T) / (unsigned)n);
}
// First row of the partial slot of run gw for row group g of (sequence, KV head) bh.
__device__ inline size_t dec_slot_row(const DecParams& p, int gw, size_t bh, int g) {
  return (size_t)(gw + g) * p.grows + bh * p.hrows;
}

// The reference maximum of a row moves only when the row's scores exceed it
// by more than this (log2 units): P stays below 2^8, well inside bf16 and the
// float32 sums, and most tiles skip the rescale.
constexpr float DEC_SLACK = 8.0f;

// Merge the runs of each query row of an item held by several teams:
// O = sum_r 2^(m_r - M) O_r / sum_r 2^(m_r - M) l_r with M = max_r m_r, over
// the runs first..last, merged in one pass (the running maximum moves as runs
// are added, so every run's loads are independent of the others' results).
// One thread per (query row, 4 features, part of the runs): P threads take
// every P-th run each and meet in LDS, in part order.  Rows are those of Q, so
// no thread is spent on padding rows.  Bound by the latency of its dependent
// loads: where few items share the teams (eight runs or more each), P = 8
// (one sequence of 1500 tokens, 24 runs per item: 4 us, against 32 us for one
// thread over the 128 runs it had with empty ones); with more items one
// thread takes the few runs of each (64 sequences: 6.2 us either way).
// EMPTY: a run may hold no key of its item (m_r = -inf, l_r = 0), and so may all
// of them (O = 0, LSE = -inf).
// COLS: each 32 rows of a slot lie as [D / 4][32] float4, then [32] pairs (max,
// sum), in place of rows of D + 4 floats (paged_kernel's teams); consecutive
// threads take consecutive rows, eight at least in a workgroup, so that they read
// whole cache lines.
template <int P, bool COLS>
constexpr int DEC_MERGE_THREADS = COLS && P > 1 ? 1024 : 256;  // of a workgroup
template <int D, int P, bool EMPTY, bool COLS>
__global__ __launch_bounds__((DEC_MERGE_THREADS<P, COLS>)) void dec_combine_kernel(DecParams p) {
  constexpr int NT = DEC_MERGE_THREADS<P, COLS>;
  constexpr int TPR = D / 4, PST = D + 4, RPW = NT / (TPR * P);  // rows per workgroup
  static_assert(RPW >= 1, "a workgroup holds whole rows");
  __shared__ f32x4 so[P > 1 ? NT : 1];
  __shared__ float2 sml[P > 1 ? NT : 1];
  const int tid = threadIdx.x;
  constexpr int APART = COLS ? RPW * TPR : TPR;  // threads between the parts of a row's runs
  const int q4 = COLS ? tid / RPW % TPR : tid % TPR, part = COLS ? tid / APART : (tid / TPR) % P;
  const size_t qrow = (size_t)blockIdx.x * RPW + (COLS ? tid % RPW : tid / (TPR * P));  // row of Q: ((b * Hq + h) * S + s)
  const int GS = p.G * p.S;
  auto weight = [](float m, float mn) { return EMPTY && m == mn ? 1.f : fast_exp2(m - mn); };  // 2^(m - mn)
  DecRuns d = {0, -1};
  float M = -INFINITY, Lr = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (qrow < (size_t)p.B * p.Hkv * GS) {
    const int R = (int)(qrow % GS);
    const size_t bh = qrow / GS;  // b * Hkv + hkv
    const int g = R / p.grows, r = R - g * p.grows;
    d = p.desc[bh * p.ng + g];  // (last run -1: written by the decode kernel itself)
#pragma unroll 4
    for (int gw = d.first + part; gw <= d.last; gw += P) {
      float2 ml;
      f32x4 v;
      if constexpr (COLS) {
        const float* ps = p.part + (dec_slot_row(p, gw, bh, g) + (r & ~31)) * PST;
        ml = *reinterpret_cast<const float2*>(ps + 32 * D + 2 * (r & 31));
        v = *reinterpret_cast<const f32x4*>(ps + 4 * (32 * q4 + (r & 31)));
      } else {
        const float* ps = p.part + (dec_slot_row(p, gw, bh, g) + r) * PST;
        const f32x4 x = *reinterpret_cast<const f32x4*>(ps + D);
        ml = float2{x[0], x[1]};
        v = *reinterpret_cast<const f32x4*>(ps + 4 * q4);
      }
      const float Mn = fmaxf(M, ml.x);
      const float a = weight(M, Mn), c = weight(ml.x, Mn);  // a = 0 for the first run (M = -inf)
      Lr = Lr * a + ml.y * c;
      o = o * a + v * c;
      M = Mn;
    }
  }
  if constexpr (P > 1) {
    so[tid] = o;
    sml[tid] = float2{M, Lr};
    __syncthreads();
    if (part != 0 || d.last < 0) return;
    // (part 0 holds at least one run, so M is finite unless EMPTY)
#pragma unroll
    for (int u = 1; u < P; ++u) {
      const float2 ml = sml[tid + u * APART];
      const f32x4 v = so[tid + u * APART];
      const float Mn = fmaxf(M, ml.x);
      const float a = weight(M, Mn), c = weight(ml.x, Mn);  // c = 0 for a part without runs
      Lr = Lr * a + ml.y * c;
      o = o * a + v * c;
      M = Mn;
    }
  } else if (d.last < 0) {
    return;
  }
  const bool none = EMPTY && !(Lr > 0.f);
  const float inv = none ? 0.f : 1.f / Lr;
  st_bf16x4(p.O + qrow * D + 4 * q4, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (q4 == 0) p.LSE[qrow] = none ? -INFINITY : (M + __log2f(Lr)) * LN2;
}

// Enqueues the merge of the items held by several runs.
template <int D, bool EMPTY, bool COLS>
hipError_t launch_dec_combine(const DecodeShape& s, const DecodeGroups& g, const DecParams& p, hipStream_t st) {
  const size_t rows = (size_t)s.B * s.Hq * s.S, items = (size_t)s.B * s.Hkv * g.ng;
  const auto merge = [&](auto parts) {
    constexpr int P = decltype(parts)::value, NT = DEC_MERGE_THREADS<P, COLS>, RPW = NT / (D / 4 * P);
    hipLaunchKernelGGL((dec_combine_kernel<D, P, EMPTY, COLS>), dim3((unsigned)((rows + RPW - 1) / RPW)), dim3(NT), 0, st, p);
  };
  if (items * 8 <= (size_t)g.runs) merge(std::integral_constant<int, COLS ? 4 : 8>());
  else merge(std::integral_constant<int, 1>());
  return hipGetLastError();
}

}  // namespace
}  // namespace bd
