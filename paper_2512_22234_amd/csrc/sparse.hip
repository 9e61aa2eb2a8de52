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
// float64, summed in an order that is the same for every page and form of the choice,
// so that equal summaries score equally and results repeat.  In another order of the
// 2 D terms a score differs by up to about 2^-45 of their absolute sum: only pages nearer
// to each other than that could be chosen differently there.
#include "paged.hpp"

namespace bd {
namespace {

__device__ inline float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ inline float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// ---- summaries ----

// One wave a page and KV head: a load covers 512 / D rows, 16 bytes a lane.  Neighbouring waves take neighbouring
// heads of a page, whose rows lie side by side if the page is kept token by token; the next page's id comes meanwhile.
// HBM bounds it: 40 prompts of 100 to 4000 tokens (97 MB, pages of 16, D = 128, 8 heads) 24 us, 4.0 TB/s.
template <int D>
__global__ __launch_bounds__(256) void summarize_kernel(SummaryArgs a) {
  constexpr int CPR = D / 8, RPI = 64 / CPR;  // 16-byte chunks of a row, rows of a load
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = blockIdx.x / a.B, b = blockIdx.x % a.B;  // (few pages of each sequence: their workgroups on all dies)
  const int P = 1 << a.pages.log_size, room = a.width << a.pages.log_size;
  const int len = imin(imax(a.lens[b], 0), room), from = imin(imax(a.from[b], 0), len);
  // (no new position, no page: the last one of a sequence that waits or is done may have another owner)
  const int j1 = from < len ? (len + P - 1) >> a.pages.log_size : 0;
  const int row = lane / CPR, chunk = lane % CPR;
  const int* table = a.table + (int64_t)b * a.table_stride;
  const int i0 = 4 * z + w, dj = 4 * a.split / a.Hkv, dh = 4 * a.split % a.Hkv;
  int j = (from >> a.pages.log_size) + i0 / a.Hkv, h = i0 % a.Hkv;
  int next = j < j1 ? table[j] : -1;
  while (j < j1) {
    const int id = next, jp = j, hp = h;
    j += dj;
    h += dh;
    if (h >= a.Hkv) {
      h -= a.Hkv;
      ++j;
    }
    next = j < j1 ? table[j] : -1;
    if ((unsigned)id >= (unsigned)a.pages.num) continue;
    const int rows = imin(P, len - (jp << a.pages.log_size));
    const bf16* first = a.K + (int64_t)id * a.pages.sp + (int64_t)hp * a.pages.sh + 8 * chunk;
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
      st16(a.summaries + (((int64_t)id * a.Hkv + hp) * 2 + row) * D + 8 * chunk, y);
    }
  }
}

// ---- scores ----

// Order of keys: that of the scores.  0: not to be chosen; ~0: chosen whatever the others are.
__device__ inline uint64_t score_key(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);  // (-0 is 0)
  return u >> 63 ? ~u : u | 1ull << 63;
}

// Pages of a sequence that hold its tokens, and the tokens.
struct SelectSeq {
  int len, used;
};
__device__ inline SelectSeq select_seq(const SelectArgs& a, int b) {
  SelectSeq q;
  q.len = imin(imax(a.lens[b], 0), a.width << a.log_size);
  q.used = (q.len + (1 << a.log_size) - 1) >> a.log_size;
  return q;
}

// Keys of the pages j0 <= j < j1 of KV head h of sequence b, by NW waves, to put(j, key); ids: room
// for the j1 - j0 entries of the table, which are left there.
//   A load covers 1 KiB, PPI summaries of CPP lanes each: half of the lanes of a page hold
//   smallest values, half largest ones, eight features a lane.  U loads are in flight while
//   the U before them are summed, and the first while the query rows are.  A page's lanes are
//   summed U pages at a time: at each step a lane keeps half of its pages and sends the others,
//   so that 1 + 2 + 4 numbers go instead of 8 a step, in the same order for every page.
template <int D, int NW>
struct ScoreSmem {
  double part[NW][2 * D], sum[2 * D];  // at e * CPP + (lane of a page): feature e of eight (no two lanes in one bank)
};
template <int D, int NW, int U = 8, class Put>
__device__ inline void score_pages(const SelectArgs& a, ScoreSmem<D, NW>& sm, int* ids, int b, int h, int used, int j0, int j1,
                                   Put put) {
  constexpr int CPP = D / 4, PPI = 64 / CPP, UQ = 4;
  static_assert(2 * D <= 64 * NW, "a thread a sum");
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int in_page = lane % CPP, side = in_page / (CPP / 2), d0 = in_page % (CPP / 2) * 8;
  // query rows r0, r0 + NW * PPI, ...: UQ in flight
  const bf16* q = a.Q + ((int64_t)b * a.Hkv + h) * a.rows * D + d0;
  int r0 = w * PPI + lane / CPP;
  u32x4 v[UQ];
  auto load_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UQ; ++u) v[u] = ld16(q + (int64_t)imin(r0 + u * NW * PPI, a.rows - 1) * D);
  };
  load_rows();
  {
    const int* row = a.table + (int64_t)b * a.table_stride;
    for (int j = j0 + tid; j < j1; j += 64 * NW) ids[j - j0] = row[j];
  }
  __syncthreads();
  int id[U];
  u32x4 x[U];
  auto load = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = ids[imin(j + u * PPI + lane / CPP, j1 - 1) - j0];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int some = (unsigned)id[u] < (unsigned)a.num_pages ? id[u] : 0;
      x[u] = ld16(a.summaries + (((int64_t)some * a.Hkv + h) * 2 + side) * D + d0);
    }
  };
  int j = j0 + w * U * PPI;
  if (j < j1) load(j);

  // Q- and Q+: every lane the features and the side that it weighs, of its rows
  double weight[8];
  {
#pragma unroll
    for (int e = 0; e < 8; ++e) weight[e] = 0;
    while (r0 < a.rows) {
#pragma unroll
      for (int u = 0; u < UQ; ++u) {
        if (r0 + u * NW * PPI >= a.rows) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = e & 1 ? bf16_hi(v[u][e / 2]) : bf16_lo(v[u][e / 2]);
          weight[e] += (double)(side ? fmaxf(y, 0.f) : fminf(y, 0.f));
        }
      }
      r0 += UQ * NW * PPI;
      if (r0 < a.rows) load_rows();
    }
#pragma unroll
    for (int o = CPP; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) weight[e] += __shfl_xor(weight[e], o);
    if (lane < CPP) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sm.part[w][e * CPP + lane] = weight[e];
    }
    __syncthreads();
    if (tid < 2 * D) {
      double y = sm.part[0][tid];
#pragma unroll
      for (int p = 1; p < NW; ++p) y += sm.part[p][tid];
      sm.sum[tid] = y;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) weight[e] = sm.sum[e * CPP + in_page];
  }

  for (; j < j1; j += NW * U * PPI) {
    double s[U];
    unsigned bad = 0;  // pages that are none
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double t[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e & 1] = fma(weight[e], (double)(e & 1 ? bf16_hi(x[u][e / 2]) : bf16_lo(x[u][e / 2])), t[e & 1]);
      s[u] = t[0] + t[1];
      bad |= (unsigned)id[u] < (unsigned)a.num_pages ? 0u : 1u << u;
    }
    if (j + NW * U * PPI < j1) load(j + NW * U * PPI);
    int mine = 0;  // the load whose page this lane ends with
#pragma unroll
    for (int o = CPP / 2, n = U; o > 0; o >>= 1) {
      if (n > 1) {
        const bool high = lane & o;
        n /= 2;
#pragma unroll
        for (int u = 0; u < U / 2; ++u)
          if (u < n) {
            const double x0 = s[u], x1 = s[u + n];  // (a choice of the elements themselves would put s in memory)
            s[u] = (high ? x1 : x0) + __shfl_xor(high ? x0 : x1, o);
          }
        mine = 2 * mine + (high ? 1 : 0);
      } else {
        s[0] += __shfl_xor(s[0], o);
      }
    }
    const int at = j + mine * PPI + lane / CPP;
    uint64_t key = score_key(s[0]);
    if (at < a.first || at >= used - a.last) key = ~0ull;
    if (bad >> mine & 1) key = 0;
    if (in_page % (CPP / U) == 0 && at < j1) put(at, key);
  }
}

// ---- the choice ----

constexpr int CHOOSE_NT = 512, SCORE_NT = 512, SELECT_NT = 1024;  // threads of the kernels below
constexpr int SCORE_WORKGROUPS = 4096;  // at most
constexpr int SELECT_KEYS = 4096;   // of a sequence and KV head, in LDS
constexpr int SCORE_PAGES = 128;    // of a workgroup at a time, where several share a sequence and KV head

template <int NT>
struct SelectSmem {
  int bins[2][256];
  int found[3];  // digit, keys above it, keys in it
  int above[NT / 64], equal[NT / 64];
};

// The list of sequence and KV head bh, of the keys key_of(0 .. used - 1) of the pages id_of(...): the highest `budget`,
// equal ones by position.  The lowest of them is found eight bits at a time, from counts of the
// keys that agree with it so far; then a pass in order of positions writes the list.
template <int NT, class Key, class Id>
__device__ inline void select_pages(const SelectArgs& a, SelectSmem<NT>& sm, int bh, const SelectSeq& seq, Key key_of, Id id_of) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, used = seq.used;
  // the threshold: keys from `low` on are chosen, of those that are `low` the first `equal`
  uint64_t low = 1;
  int equal = INT32_MAX;
  if (used > a.budget) {
    uint64_t prefix = 0;
    int need = a.budget;
    if (tid < 256) sm.bins[0][tid] = 0;
    __syncthreads();
    for (int shift = 56; shift >= 0; shift -= 8) {
      int* const bins = sm.bins[shift >> 3 & 1 ? 0 : 1];
      for (int j0 = 0; j0 < used; j0 += NT) {
        const int j = j0 + tid;
        const uint64_t key = j < used ? key_of(j) : 0;
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
        int above = wave_scan(sum) - sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (above < need && above + n[e] >= need) {
            sm.found[0] = 255 - 4 * lane - e;
            sm.found[1] = above;
            sm.found[2] = n[e];
          }
          above += n[e];
        }
      } else if (tid >= NT - 256) {  // (the next digit's counts)
        sm.bins[shift >> 3 & 1][tid - (NT - 256)] = 0;
      }
      __syncthreads();
      prefix = prefix << 8 | (uint64_t)sm.found[0];
      need -= sm.found[1];
      low = prefix << shift;
      if (sm.found[2] == need) break;  // all keys that begin so are chosen
      if (shift == 0) equal = need;
    }
    if (low == 0) {  // fewer pages than the budget can be chosen
      low = 1;
      equal = INT32_MAX;
    }
  }
  int* out = a.lists + (int64_t)bh * a.budget;
  int count = 0, met = 0, tail = -1;  // tail: keys up to the sequence's last page, if that is chosen (its own thread)
  const bool ties = equal != INT32_MAX;
  for (int j0 = 0; j0 < used; j0 += NT) {
    const int j = j0 + tid;
    const uint64_t key = j < used ? key_of(j) : 0;
    const bool same = ties && key == low;
    const uint64_t eq = __ballot(same), gt = __ballot(!same && key >= low), below = (1ull << lane) - 1;
    if (lane == 0) {
      sm.equal[w] = __builtin_popcountll(eq);
      sm.above[w] = __builtin_popcountll(gt);
    }
    __syncthreads();
    int e0 = met, g0 = 0, all_e = 0, all_g = 0;  // equal keys and others chosen before this wave's
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) {
      e0 += v < w ? sm.equal[v] : 0;
      g0 += v < w ? sm.above[v] : 0;
      all_e += sm.equal[v];
      all_g += sm.above[v];
    }
    const int er = e0 + __builtin_popcountll(eq & below);  // rank among equal keys
    const bool chosen = (gt >> lane & 1) || (same && er < equal);
    const int at = count + g0 + __builtin_popcountll(gt & below) + imin(er, equal) - imin(met, equal);
    if (chosen) {
      out[at] = id_of(j);
      if (j == used - 1) tail = ((at + 1) << a.log_size) - ((used << a.log_size) - seq.len);
    }
    count += all_g + imin(met + all_e, equal) - imin(met, equal);
    met += all_e;
    __syncthreads();
  }
  for (int i = count + tid; i < a.budget; i += NT) out[i] = -1;
  if (tid == (used > 0 ? (used - 1) % NT : 0)) a.rows_out[bh] = tail >= 0 ? tail : count << a.log_size;
}

// One workgroup a sequence and KV head, its pages and keys in LDS (past KEYS pages, keys in the workspace).  64 sequences of
// 512 to 8192 tokens in pages of 16 (61 MB of summaries, D = 128, 8 KV heads, 16 query rows) 21 us: 12 for the reading, as
// fast as HBM gives it, and 7, all that one sequence of 94 pages takes, for the chain of query rows, first pages, and the
// digits of the choice.
// (four waves a SIMD: two workgroups a CU)
// LONG: tables of more than KEYS pages.  (Four loads in flight a wave: with eight, and the longer lists' loop, a wave's
// registers would not do.)
template <int D, int KEYS, bool LONG>
__global__ __launch_bounds__(CHOOSE_NT, 4) void choose_kernel(SelectArgs a) {
  __shared__ struct {
    uint64_t keys[KEYS];
    int ids[KEYS];
    ScoreSmem<D, CHOOSE_NT / 64> score;
    SelectSmem<CHOOSE_NT> select;
  } sm;
  const int bh = blockIdx.x, h = bh % a.Hkv, b = bh / a.Hkv;
  const SelectSeq seq = select_seq(a, b);
  const int* row = a.table + (int64_t)b * a.table_stride;
  if (seq.used > a.budget) {
    const bool held = !LONG || seq.used <= KEYS;
    uint64_t* keys = a.keys + (int64_t)bh * a.width;
    int j0 = 0;
    do {
      const int j1 = LONG ? imin(seq.used, j0 + KEYS) : seq.used;
      score_pages<D, CHOOSE_NT / 64, LONG ? 4 : 8>(a, sm.score, sm.ids, b, h, seq.used, j0, j1, [&](int j, uint64_t key) {
        if (held) sm.keys[j] = key;
        else keys[j] = key;
      });
      __syncthreads();
      j0 += KEYS;
    } while (LONG && j0 < seq.used);
    select_pages(a, sm.select, bh, seq, [&](int j) { return held ? sm.keys[j] : keys[j]; },
                 [&](int j) { return held ? sm.ids[j] : row[j]; });
  } else {  // every page that there is
    select_pages(a, sm.select, bh, seq, [&](int j) -> uint64_t { return (unsigned)row[j] < (unsigned)a.num_pages; },
                 [&](int j) { return row[j]; });
  }
}

// Several workgroups a sequence and KV head: keys of SCORE_PAGES pages each, in the workspace ...  Two sequences of 120,000
// tokens in pages of 64 with 128 query rows (16 MB): 9.9 us, then 8.7 for the choice, a chain of loads and barriers each.
template <int D>
__global__ __launch_bounds__(SCORE_NT) void score_kernel(SelectArgs a) {
  __shared__ struct {
    ScoreSmem<D, SCORE_NT / 64> score;
    int ids[SCORE_PAGES];
  } sm;
  // (the first pages of all lists, then the next ones, ...: sequences far shorter than the table leave the last ones empty)
  const int chunks = cdiv(a.width, SCORE_PAGES), items = a.B * a.Hkv;
  const int64_t total = (int64_t)items * chunks;  // checked on the host
  for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
    const int c = (int)(t / items), bh = (int)(t - (int64_t)c * items), h = bh % a.Hkv, b = bh / a.Hkv;
    const SelectSeq seq = select_seq(a, b);
    if (c * SCORE_PAGES >= seq.used) continue;
    uint64_t* keys = a.keys + (int64_t)bh * a.width;
    score_pages<D, SCORE_NT / 64>(a, sm.score, sm.ids, b, h, seq.used, c * SCORE_PAGES, imin(seq.used, (c + 1) * SCORE_PAGES),
                                  [&](int j, uint64_t key) { keys[j] = key; });
    __syncthreads();
  }
}
// ... and the choice among them.
__global__ __launch_bounds__(SELECT_NT) void select_kernel(SelectArgs a) {
  __shared__ struct {
    uint64_t keys[SELECT_KEYS];
    SelectSmem<SELECT_NT> select;
  } sm;
  const int bh = blockIdx.x;
  const SelectSeq seq = select_seq(a, bh / a.Hkv);
  const uint64_t* keys = a.keys + (int64_t)bh * a.width;
  const int* row = a.table + (int64_t)(bh / a.Hkv) * a.table_stride;
  auto id_of = [&](int j) { return row[j]; };
  if (seq.used <= SELECT_KEYS) {
    for (int j = threadIdx.x; j < seq.used; j += SELECT_NT) sm.keys[j] = keys[j];
    __syncthreads();
    select_pages(a, sm.select, bh, seq, [&](int j) { return sm.keys[j]; }, id_of);
  } else {
    select_pages(a, sm.select, bh, seq, [&](int j) { return keys[j]; }, id_of);
  }
}

// Whether one workgroup takes a sequence and KV head on its own.  Device us a call (8 KV heads, one query), one workgroup and
// several of SCORE_PAGES, by sequences and their pages:
//   D = 128   one      1 of 250 380 510 1000   9.2 10.8 12.8 20.2    4 of 250 380 510 2000   9.4 11.1 12.8 36.2
//             several                         10.4 10.0 10.6 10.8                           10.5 10.7 10.8 18.2
//             one      8 of 510 1000 2000     13.0 21.4 36.8        12 of 510 2000          13.1 37.3
//             several                         11.0 16.1 31.2                                14.6 41.0
//             one     16 of 140 510 1000 2000 4062  8.1 13.9 22.2 37.3 67.6   32 of 510 1000 2000 4062  17.3 28.2 49.9 114
//             several                              10.5 16.0 28.9 50.4 94.2                             28.9 48.2 89.5 184
//   D = 64    one      1 of 250 380 510 1000   7.8  8.2  9.3 13.9    4 of 510 2000  9.7 22.7    16 of 510 2000  10.1 24.9
//             several                         10.0  9.7  9.8 10.6                  10.1 15.6                    13.9 40.4
// In a table of 8193 pages, which is all that the host knows of them (D = 128): 16 of 125, 2000, 8192 pages 8.1 41.6 213 and
// 21.2 57.4 195; 32 of 125, 8192 8.6 277 and 28.8 355; 64 of 500 27.2 and 77.7.
// (The sides meet between 64 and 96 lists; at the rule's own borders the worse side is up to a fifth slower.)
bool select_fused(const SelectArgs& a) {
  const int items = a.B * a.Hkv;
  return a.width <= (items <= 32 ? 320 : 512) || items >= 128;
}

template <int D>
void launch_choose(const SelectArgs& a, unsigned items, hipStream_t st) {
  if (a.width <= 1024) hipLaunchKernelGGL((choose_kernel<D, 1024, false>), dim3(items), dim3(CHOOSE_NT), 0, st, a);
  else if (a.width <= SELECT_KEYS) hipLaunchKernelGGL((choose_kernel<D, SELECT_KEYS, false>), dim3(items), dim3(CHOOSE_NT), 0, st, a);
  else hipLaunchKernelGGL((choose_kernel<D, SELECT_KEYS, true>), dim3(items), dim3(CHOOSE_NT), 0, st, a);
}

}  // namespace

hipError_t launch_summarize(const SummaryArgs& in, int D, hipStream_t st) {
  SummaryArgs a = in;
  // About 4096 workgroups, as far as there are pages and heads for four waves each: sequences of unequal lengths spread
  // better over more of them, those without a page cost their launch.  us, 2048, 4096, 8192 (D = 128, 8 heads): 40
  // prompts of 100 to 4000 tokens, pages of 16 25.1 24.4 22.4; the last pages of 400 sequences 5.1 5.1 6.4, of 64 3.7 3.7 5.4.
  const int64_t items = (int64_t)a.width * a.Hkv;
  a.split = imax(1, imin(4096 / imin(a.B, 4096), (int)((items < 16384 ? items : 16384) + 3) / 4));
  const dim3 grid((unsigned)a.B * a.split);
  if (D == 128) hipLaunchKernelGGL(summarize_kernel<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(summarize_kernel<64>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_select(const SelectArgs& a, int D, hipStream_t st) {
  const unsigned items = (unsigned)a.B * a.Hkv;
  if (select_fused(a)) {
    if (D == 128) launch_choose<128>(a, items, st);
    else launch_choose<64>(a, items, st);
    return hipGetLastError();
  }
  // 128 pages a workgroup at a time; us a call (D = 128, 8 KV heads), 128 and 256: one sequence of 1000 pages 11.1 12.7, of
  // 2048 14.1 15.8, of 8192 with 128 query rows 38.3 39.8; two of 2000, 128 rows 18.0 18.6; four of 4096 32.2 32.6.
  const int64_t tasks = (int64_t)items * cdiv(a.width, SCORE_PAGES);
  const dim3 grid((unsigned)(tasks < SCORE_WORKGROUPS ? tasks : SCORE_WORKGROUPS));
  if (D == 128) hipLaunchKernelGGL(score_kernel<128>, grid, dim3(SCORE_NT), 0, st, a);
  else hipLaunchKernelGGL(score_kernel<64>, grid, dim3(SCORE_NT), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(select_kernel, dim3(items), dim3(SELECT_NT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_sparse_decode(const DecodeShape& s, const PagedArgs& a, int heads, void* ws, hipStream_t st) {
  return s.D == 128 ? launch_paged_decode_d<128, PagedMode::Lists>(s, a, heads, ws, st)
                    : launch_paged_decode_d<64, PagedMode::Lists>(s, a, heads, ws, st);
}

}  // namespace bd
