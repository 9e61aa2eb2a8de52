// Attention over chosen pages of a paged KV cache for gfx950: summaries of the
// pages, the choice, and the decoding over it.
//
// Summary of a page and KV head: for each feature the smallest and largest value
// lo_d, hi_d of its keys.  For a query row q, sum_d max(q_d lo_d, q_d hi_d) is an
// upper bound of q . k over the page's keys.  A page's score is the sum of these
// bounds over the G*S query rows of the KV head,
//   score = sum_d (Q+_d hi_d + Q-_d lo_d),  Q+ = sum_r max(q_r, 0), Q- = sum_r min(q_r, 0),
// so it costs 2 D multiply-adds a page however many rows there are, and reading
// the summaries, 4 D bytes a page and KV head, bounds the choice.  Scores are
// float64: which pages are chosen must not depend on the order of a sum.
#include "paged.hpp"

namespace bd {
namespace {

__device__ inline float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ inline float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// ---- summaries ----

// One wave a page and KV head: a load covers 512 / D rows, 16 bytes a lane.
template <int D>
__global__ __launch_bounds__(256) void summarize_kernel(SummaryArgs a) {
  constexpr int CPR = D / 8, RPI = 64 / CPR;  // 16-byte chunks of a row, rows of a load
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int z = blockIdx.x % a.split, bh = blockIdx.x / a.split, h = bh % a.Hkv, b = bh / a.Hkv;
  const int P = 1 << a.pages.log_size, room = a.width << a.pages.log_size;
  const int len = imin(imax(a.lens[b], 0), room), from = imin(imax(a.from[b], 0), len);
  const int j1 = (len + P - 1) >> a.pages.log_size;
  const int row = lane / CPR, chunk = lane % CPR;
  for (int j = (from >> a.pages.log_size) + 4 * z + w; j < j1; j += 4 * a.split) {
    const int id = a.table[(int64_t)b * a.table_stride + j];
    if ((unsigned)id >= (unsigned)a.pages.num) continue;
    const int rows = imin(P, len - (j << a.pages.log_size));
    const bf16* first = a.K + (int64_t)id * a.pages.sp + (int64_t)h * a.pages.sh + 8 * chunk;
    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = INFINITY;
      hi[e] = -INFINITY;
    }
    for (int r0 = 0; r0 < rows; r0 += 4 * RPI) {
      u32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)  // (a row past the last: the last again)
        x[u] = ld16(first + (int64_t)imin(r0 + u * RPI + row, rows - 1) * a.pages.sr);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = e & 1 ? bf16_hi(x[u][e / 2]) : bf16_lo(x[u][e / 2]);
          lo[e] = fminf(lo[e], v);
          hi[e] = fmaxf(hi[e], v);
        }
    }
#pragma unroll
    for (int o = CPR; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = fminf(lo[e], __shfl_xor(lo[e], o));
        hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o));
      }
    if (row < 2) {
      u32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t p = __float_as_uint(row ? hi[2 * e] : lo[2 * e]), q = __float_as_uint(row ? hi[2 * e + 1] : lo[2 * e + 1]);
        y[e] = p >> 16 | (q & 0xffff0000u);
      }
      st16(a.summaries + (((int64_t)id * a.Hkv + h) * 2 + row) * D + 8 * chunk, y);
    }
  }
}

// ---- scores ----

// Order of keys: that of the scores.  0: not to be chosen; ~0: chosen whatever the others are.
__device__ inline uint64_t score_key(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);  // (-0 is 0)
  return u >> 63 ? ~u : u | 1ull << 63;
}

constexpr int SCORE_PAGES = 256;  // of a workgroup

// Keys of SCORE_PAGES pages of one sequence and KV head.
template <int D>
__global__ __launch_bounds__(256) void score_kernel(SelectArgs a) {
  constexpr int CPP = D / 4, PPI = 64 / CPP, U = 8;  // 16-byte chunks of a summary, summaries a load, loads in flight
  __shared__ double sums[2][256];
  const int chunks = cdiv(a.width, SCORE_PAGES);
  const int c = blockIdx.x % chunks, bh = blockIdx.x / chunks, h = bh % a.Hkv, b = bh / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int P = 1 << a.log_size;
  const int len = imin(imax(a.lens[b], 0), a.width << a.log_size), used = (len + P - 1) >> a.log_size;
  if (c * SCORE_PAGES >= used) return;

  // Q+ and Q-
  {
    const int d = tid % D;
    double up = 0, down = 0;
    for (int r = tid / D; r < a.rows; r += 256 / D) {
      const double q = (double)(float)a.Q[((int64_t)bh * a.rows + r) * D + d];
      up += fmax(q, 0.0);
      down += fmin(q, 0.0);
    }
    sums[1][tid] = up;
    sums[0][tid] = down;
    __syncthreads();
    if (tid < D) {
#pragma unroll
      for (int u = 1; u < 256 / D; ++u) {
        up += sums[1][tid + u * D];
        down += sums[0][tid + u * D];
      }
      sums[1][tid] = up;
      sums[0][tid] = down;
    }
    __syncthreads();
  }
  const int part = lane % CPP, side = part / (CPP / 2), d0 = part % (CPP / 2) * 8;  // side: of the smallest, of the largest values
  double weight[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) weight[e] = sums[side][d0 + e];

  const int* row = a.table + (int64_t)b * a.table_stride;
  const int end = imin(used, (c + 1) * SCORE_PAGES);
  for (int j0 = c * SCORE_PAGES + w * U * PPI; j0 < end; j0 += 4 * U * PPI) {
    int id[U];
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = row[imin(j0 + u * PPI + lane / CPP, used - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int some = (unsigned)id[u] < (unsigned)a.num_pages ? id[u] : 0;
      x[u] = ld16(a.summaries + (((int64_t)some * a.Hkv + h) * 2 + side) * D + d0);
    }
    double s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = weight[e] * (double)(e & 1 ? bf16_hi(x[u][e / 2]) : bf16_lo(x[u][e / 2]));
      s[u] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
#pragma unroll
      for (int o = CPP / 2; o > 0; o >>= 1) s[u] += __shfl_xor(s[u], o);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * PPI + lane / CPP;
      if (part == u && j < end) {
        uint64_t key = score_key(s[u]);
        if (j < a.first || j >= used - a.last) key = ~0ull;
        if ((unsigned)id[u] >= (unsigned)a.num_pages) key = 0;
        a.keys[(int64_t)bh * a.width + j] = key;
      }
    }
  }
}

// ---- the choice ----

constexpr int SELECT_NT = 512;

// One workgroup a sequence and KV head: the highest `budget` keys, equal ones by
// position.  The lowest of them is found eight bits at a time, from counts of the
// keys that agree with it so far; then a pass in order of positions writes the list.
__global__ __launch_bounds__(SELECT_NT) void select_kernel(SelectArgs a) {
  constexpr int NW = SELECT_NT / 64;
  __shared__ int bins[256];
  __shared__ int found[3];  // digit, keys above it, keys in it
  __shared__ int wabove[NW], wequal[NW];
  const int bh = blockIdx.x, b = bh / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int P = 1 << a.log_size;
  const int len = imin(imax(a.lens[b], 0), a.width << a.log_size), used = (len + P - 1) >> a.log_size;
  const uint64_t* keys = a.keys + (int64_t)bh * a.width;

  // the threshold: keys above it are chosen, and the first `equal` of those that are it
  uint64_t low = 1;
  int equal = INT32_MAX;
  if (used > a.budget) {
    uint64_t prefix = 0;
    int need = a.budget;
    for (int shift = 56; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += SELECT_NT) bins[i] = 0;
      __syncthreads();
      for (int j0 = 0; j0 < used; j0 += SELECT_NT) {
        const int j = j0 + tid;
        const uint64_t key = j < used ? keys[j] : 0;
        const bool in = j < used && (shift == 56 || key >> (shift + 8) == prefix);
        const int digit = (int)(key >> shift) & 255;
        const uint64_t all = __ballot(in);
        if (all == 0) continue;
        // (one addition where a wave's keys agree, as in the first digits)
        const int one = __builtin_amdgcn_readlane(digit, __builtin_ctzll(all));
        if (__ballot(in && digit == one) == all) {
          if (lane == 0) atomicAdd(&bins[one], __builtin_popcountll(all));
        } else if (in) {
          atomicAdd(&bins[digit], 1);
        }
      }
      __syncthreads();
      if (w == 0) {
        // four bins a lane, the highest first
        int n[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += n[e] = bins[255 - 4 * lane - e];
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int u = __shfl_up(incl, o);
          if (lane >= o) incl += u;
        }
        int above = incl - sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (above < need && above + n[e] >= need) {
            found[0] = 255 - 4 * lane - e;
            found[1] = above;
            found[2] = n[e];
          }
          above += n[e];
        }
      }
      __syncthreads();
      prefix = prefix << 8 | (uint64_t)found[0];
      need -= found[1];
      const bool all = found[2] == need;  // all keys with these digits are chosen
      low = prefix << shift;
      equal = shift == 0 ? need : INT32_MAX;
      if (all) break;
      __syncthreads();
    }
    // (keys are counted from `low` on; without the last digits' count, all that begin with it are chosen)
    if (low == 0) low = 1, equal = INT32_MAX;  // fewer pages than the budget can be chosen
  }
  int* out = a.lists + (int64_t)bh * a.budget;
  const int* row = a.table + (int64_t)b * a.table_stride;
  int count = 0, met = 0;
  bool tail = false;
  const bool ties = equal != INT32_MAX;
  for (int j0 = 0; j0 < used; j0 += SELECT_NT) {
    const int j = j0 + tid;
    const uint64_t key = j < used ? keys[j] : 0;
    const bool same = ties && key == low;
    const uint64_t eq = __ballot(same);
    const uint64_t gt = __ballot(!same && key >= low);
    const uint64_t below = (1ull << lane) - 1;
    if (lane == 0) wequal[w] = __builtin_popcountll(eq);
    if (lane == 0) wabove[w] = __builtin_popcountll(gt);
    __syncthreads();
    int e0 = met, g0 = 0, all_e = 0, all_g = 0;  // equal keys and others chosen before this wave's
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      e0 += v < w ? wequal[v] : 0;
      g0 += v < w ? wabove[v] : 0;
      all_e += wequal[v];
      all_g += wabove[v];
    }
    const int er = e0 + __builtin_popcountll(eq & below);  // rank among equal keys
    const bool chosen = (gt >> lane & 1) || (same && er < equal);
    const int at = count + g0 + __builtin_popcountll(gt & below) + imin(er, equal) - imin(met, equal);
    if (chosen) {
      out[at] = row[j];
      if (j == used - 1) a.rows_out[bh] = ((at + 1) << a.log_size) - ((used << a.log_size) - len);
      tail |= j == used - 1;
    }
    count += all_g + imin(met + all_e, equal) - imin(met, equal);
    met += all_e;
    __syncthreads();
  }
  for (int i = count + tid; i < a.budget; i += SELECT_NT) out[i] = -1;
  if (!__syncthreads_or(tail) && tid == 0) a.rows_out[bh] = count << a.log_size;
}

}  // namespace

hipError_t launch_summarize(const SummaryArgs& in, int D, hipStream_t st) {
  SummaryArgs a = in;
  // about 2048 workgroups, as far as there are pages for four waves each
  a.split = imax(1, imin(2048 / imin(a.B * a.Hkv, 2048), cdiv(a.width, 4)));
  const dim3 grid((unsigned)a.B * a.Hkv * a.split);
  if (D == 128) hipLaunchKernelGGL(summarize_kernel<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(summarize_kernel<64>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_select(const SelectArgs& a, int D, hipStream_t st) {
  const dim3 grid((unsigned)a.B * a.Hkv * cdiv(a.width, SCORE_PAGES));
  if (D == 128) hipLaunchKernelGGL(score_kernel<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(score_kernel<64>, grid, dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)a.B * a.Hkv), dim3(SELECT_NT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_sparse_decode(const DecodeShape& s, const PagedArgs& a, int heads, void* ws, hipStream_t st) {
  return s.D == 128 ? launch_paged_decode_d<128, PagedMode::Lists>(s, a, heads, ws, st)
                    : launch_paged_decode_d<64, PagedMode::Lists>(s, a, heads, ws, st);
}

}  // namespace bd
