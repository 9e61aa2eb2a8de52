// The kernel that decodes over a paged KV cache (paged.hip), and its forms for
// sequences that share a prefix (shared.hip) and for a list of pages for each KV
// head (sparse.hip).
#pragma once

#include "decode.hpp"

namespace bd {
namespace {

// Where the merge finds the prefix's part of a sequence and KV head: its first query row
// is row row0 of item `item`, which the runs first to last hold; rows past an item's grows
// are in the items behind it.
struct alignas(16) SharedRef {
  int item, row0, first, last;
};
static_assert(sizeof(SharedRef) == 16 && sizeof(DecRuns) == 16, "the workspace's layout (kernels.hpp)");

// What the copies of a tile need, in bytes.
struct PagedTile {
  uint64_t kp, vp, kn, vn;  // addresses: pages, block
  uint64_t table;           // ... page table
  int64_t table_stride;
  int64_t sh;               // head stride of the pages
  uint32_t sp, sr;          // page and row stride of the pages
  int num, log_size;        // pages, log2 of their rows
  int last;                 // last entry of a table row
};
// What a call's "sequences", the rows of the page table, are:
//   Plain   a sequence's keys, for all KV heads;
//   Lists   the keys of one KV head of one sequence: B * Hkv rows, one KV head each
//           (DecodeShape with B * Hkv sequences, G query heads and one KV head);
//   Own     as Plain, of sequences that also have a prefix: every item leaves a
//           partial result, which a kernel of its own joins with the prefix's;
//   Joint   the sequences' own keys; then, behind the sequences, the keys that those of
//           each group share, the query rows of a KV head being those of all members,
//           G * S each, in row groups of grows.  Items leave partial results.
enum class PagedMode { Plain, Lists, Own, Joint };

struct PagedParams {
  DecParams d;  // C: the table's room in keys
  PagedTile t;
  int Sn;  // the block's own keys (0: none)
  // Lists: KV heads of the pages
  int heads;
  // Prefixes (d.B, d.C, d.cache_lens and t's table are theirs): members of each group, sequences in all
  const int* sizes;
  int seqs;
  SharedRef* refs;  // [seqs][Hkv], for the merge
  int* members;     // the sequences that are in a group
  // Joint: the sequences' own keys, in a table of own.width entries a row
  struct {
    uint64_t table;
    int64_t table_stride;
    int last, C;
    const int* lens;
  } own;
};

// Key tiles of an item of a sequence with cache length len.
template <int KT>
__device__ inline int tiles_of(int keys) {
  return (int)((unsigned)(keys + KT - 1) / KT);
}
template <int KT>
__device__ inline int paged_tiles(const PagedParams& p, int len) {
  return imax(tiles_of<KT>(len) + tiles_of<KT>(p.Sn), 1);
}

// Runs that the T tiles of all items are cut into.  Every run that holds part of an
// item leaves partial results, for one wave up to 32 rows of D floats (as many bytes
// as a tile of keys and values), which are written, read and merged, so a call is cut
// no finer than its reading needs.  One wave: single tiles for up to 256 runs (one a
// CU), then three tiles a run; where these come to two runs on most CUs, two on all.
// Items of at most eight tiles on average end a run's chain of copies so often that
// three runs a CU are needed to fill the gaps; so are they at D = 64, with half the
// bytes a tile.  Measured, us (32/8 heads; * no more than one tile a run):
//                                               256   cdiv(T, 3)  512   768   1024 runs
//   one sequence of 1500, S = 8 (384 tiles)     11.3     -        13.7* 13.6* 14.1*
//   ... of 3000 (760)                           13.6    13.6      16.0  20.1  20.7*
//   ... of 6000 (1512)                          16.5    17.9      16.8  18.4  20.0
//   8 sequences of 3000, S = 8 (6080)           34.5     -        27.3  29.9  31.0
//   D = 64: 2 of 3000, S = 4 (1520)               -     12.8       -    13.5    -
//   D = 64: 64 of 512 to 8192, S = 1 (50,072)     -      -        84.8  70.7  75.6
// and by the tiles of an item, S = 1, 512 / 768 runs:
//   tiles an item       2            4            8           16           32           64
//    4,000 tiles   26.1  22.7   22.9  20.3   21.9  20.7   22.0  21.5   21.1  21.9   22.6  21.9
//   15,000         72.0  64.8   61.3  59.5   56.8  56.8   55.1  56.1   55.2  55.5   58.0  57.7
//   30,000        132.6 109.2  107.3  96.7   91.7  91.1   84.8  87.9   83.2  86.9   84.8  86.7
//   60,000        254.3 211.0  204.3 184.9  175.8 174.5  162.3 166.2  159.2 164.2  157.7 162.3
// (64 sequences of 512 to 8192, 98 tiles an item: heads outermost 137.8 and 138.5, tokens 133.4 and 139.8).
// Teams take two tiles at least (dec_runs).
// Where every item leaves partial results, its run waits for its stores: three runs a CU (16 groups of
// 6 to 8 sequences, one token: 92.8 us a call, with the rule above 96.0).
template <int D, int TW, bool PARTS>
__device__ inline int paged_runs(int T, int items) {
  if (TW > 1) return dec_runs<TW>(DEC_WAVES / TW, T);
  const int three = imax(256, cdiv(T, 3));
  return imin(T, D == 64 || PARTS ? imin(three, 768) : T < 1152 ? three : T >> 3 <= items ? 768 : 512);
}
// First tile of run gw <= n (the runs cut T tiles into n near-equal pieces).
__device__ inline int paged_run_start(int gw, int n, int T) {
  if (T < 1 << 22) return (int)((unsigned)gw * (unsigned)T / (unsigned)n);
  return (int)((unsigned)(((unsigned long long)gw * T) >> 8) / ((unsigned)n >> 8));  // (n is a multiple of 256 here)
}

// Position of a tile: sequence b (cache length len, nt tiles per item), KV head
// h and row group g of the item, tile j of it.
struct PagedPos {
  int b, len, nt, h, g, j;
};
// Prefixes: also the group's row groups, first member and members, the members of all
// groups behind it, and the row groups before it; tiles of cached keys, the entry's row of its
// table and the last entry of that.
struct PrefixPos : PagedPos {
  int ng, first, n, left, row, ntc, last;
  uint64_t table;
};

// The tiles of all prefixes in order of (group, KV head, row group), JOINT: behind those of the
// sequences' own keys: how many there are, where a run starts, and what follows a tile.
// Entry b of the list is group b, JOINT: sequence b or, from seqs on, group b - seqs.  NW waves scan it.
template <int KT, int TW, int NW, int TEAMS, bool JOINT>
struct PrefixWork {
  struct Smem {
    int wmem[NW], wrow[NW], wsum[NW];  // per-wave sums: members, row groups, tiles of a KV head
    int b[TEAMS], off[TEAMS], first[TEAMS], n[TEAMS], left[TEAMS], row[TEAMS], len[TEAMS];  // where each team's run starts
  };
  const PagedParams& p;
  int c0, c1, before_members, before_rows, before_tiles, tiles;  // this thread's entries, what lies before them, their tiles
  int size0, keys0;                                              // of its first entry: members that it names, keys
  int all;                                                       // members of all groups

  typedef const __attribute__((address_space(4))) int* Uniform;  // (scalar loads: nothing writes these arrays meanwhile)
  __device__ int own() const { return JOINT ? p.seqs : 0; }      // entries ahead of the groups
  __device__ int entries() const { return own() + p.d.B; }
  __device__ int row_groups(int n) const { return tiles_of<32 * TW>(n * p.d.G * p.d.S); }
  // Members that entry b names (a sequence's own keys: none).
  template <class Ints>
  __device__ int size(int b) const {
    return JOINT && b < p.seqs ? 0 : imax(((Ints)(uintptr_t)p.sizes)[b - own()], 0);
  }
  // Members and first member of entry b, which names `size`, where the groups before it have `upto`, which it
  // adds to (sizes that pass the sequences end there); its keys; its tiles of a KV head and row group.
  __device__ void members(int b, int size, int& first, int& n, int& upto) const {
    if (JOINT && b < p.seqs) {
      first = b;
      n = 1;
    } else {
      first = upto;
      n = imin(size, p.seqs - upto);
      upto += n;
    }
  }
  template <class Ints>
  __device__ int keys(int b) const {
    if (JOINT && b < p.seqs) return imin(imax(((Ints)(uintptr_t)p.own.lens)[b], 0), p.own.C);
    return imin(imax(((Ints)(uintptr_t)p.d.cache_lens)[b - own()], 0), p.d.C);
  }
  __device__ int tiles_at(int b, int len) const {
    return imax(tiles_of<KT>(len) + (JOINT && b < p.seqs ? tiles_of<KT>(p.Sn) : 0), 1);
  }

  // Of an entry of this thread.
  __device__ int my_size(int b) const { return b == c0 ? size0 : size<const int*>(b); }
  __device__ int my_keys(int b) const { return b == c0 ? keys0 : keys<const int*>(b); }

  // Tiles of a KV head in all entries; the first workgroup notes what the merge needs.
  // (All that a thread with one entry reads, it reads at once, ahead of the sums.)
  __device__ int scan(Smem& sm, int tid) {
    const int lane = tid & 63, w = tid >> 6;
    const int cpt = cdiv(entries(), 64 * NW);
    c0 = imin(entries(), tid * cpt);
    c1 = imin(entries(), c0 + cpt);
    size0 = c0 < c1 ? size<const int*>(c0) : 0;
    keys0 = c0 < c1 ? keys<const int*>(c0) : 0;
    int mem = 0;
    for (int b = c0; b < c1; ++b) mem += imin(my_size(b), p.seqs - mem);
    const int imem = wave_scan(mem, p.seqs);
    if (lane == 63) sm.wmem[w] = imem;
    __syncthreads();
    const int last = __shfl_up(imem, 1, 64);
    before_members = lane == 0 ? 0 : last;
    all = 0;
    for (int v = 0; v < NW; ++v) {
      if (v < w) before_members = imin(before_members + sm.wmem[v], p.seqs);
      all = imin(all + sm.wmem[v], p.seqs);
    }
    if (blockIdx.x == 0 && tid == 0) *p.members = all;
    int rows = 0;
    tiles = 0;
    for (int b = c0, upto = before_members; b < c1; ++b) {
      int first, n;
      members(b, my_size(b), first, n, upto);
      const int r = row_groups(n);
      rows += r;
      tiles += tiles_at(b, my_keys(b)) * r;
    }
    const int irow = wave_scan(rows), itile = wave_scan(tiles);
    if (lane == 63) {
      sm.wrow[w] = irow;
      sm.wsum[w] = itile;
    }
    __syncthreads();
    before_rows = irow - rows;
    before_tiles = itile - tiles;
    int total = 0;
    for (int v = 0; v < NW; ++v) {
      before_rows += v < w ? sm.wrow[v] : 0;
      before_tiles += v < w ? sm.wsum[v] : 0;
      total += sm.wsum[v];
    }
    return __builtin_amdgcn_readfirstlane(total);
  }
  // Notes where team v's run starts, at tile x0 of all.  (A barrier before start().)
  __device__ void find(Smem& sm, int v, int x0) const {
    const int I = p.d.Hkv;
    if (tiles == 0 || x0 < before_tiles * I || x0 >= (before_tiles + tiles) * I) return;
    int pb = before_tiles, upto = before_members, row = before_rows;
    for (int b = c0; b < c1; ++b) {
      int first, n;
      members(b, my_size(b), first, n, upto);
      const int len = my_keys(b), r = row_groups(n), t = tiles_at(b, len) * r;
      if (x0 < (pb + t) * I) {
        sm.b[v] = b;
        sm.off[v] = x0 - pb * I;
        sm.first[v] = first;
        sm.n[v] = n;
        sm.left[v] = all - upto;
        sm.row[v] = row;
        sm.len[v] = len;
        return;
      }
      pb += t;
      row += r;
    }
  }
  // What q holds of its entry q.b, of q.n members and q.len keys.
  __device__ void enter(PrefixPos& q) const {
    const bool mine = JOINT && q.b < p.seqs;  // a sequence's own keys
    q.nt = tiles_at(q.b, q.len);
    q.ntc = mine ? tiles_of<KT>(q.len) : q.nt;
    q.ng = row_groups(q.n);
    q.last = mine ? p.own.last : p.t.last;
    q.table = mine ? p.own.table + (int64_t)q.b * p.own.table_stride : p.t.table + (int64_t)(q.b - own()) * p.t.table_stride;
  }
  __device__ PrefixPos start(const Smem& sm, int v) const {
    PrefixPos q;
    q.b = __builtin_amdgcn_readfirstlane(sm.b[v]);
    const int off = __builtin_amdgcn_readfirstlane(sm.off[v]);
    q.first = __builtin_amdgcn_readfirstlane(sm.first[v]);
    q.n = __builtin_amdgcn_readfirstlane(sm.n[v]);
    q.left = __builtin_amdgcn_readfirstlane(sm.left[v]);
    q.row = __builtin_amdgcn_readfirstlane(sm.row[v]);
    q.len = __builtin_amdgcn_readfirstlane(sm.len[v]);
    enter(q);
    const int item = off / q.nt;
    q.j = off - item * q.nt;
    q.h = item / q.ng;
    q.g = item - q.h * q.ng;
    return q;
  }
  // The first tile of the item behind that of q.
  __device__ __attribute__((always_inline)) void next_item(PrefixPos& q) const {
    q.j = 0;
    if (++q.g < q.ng) return;
    q.g = 0;
    if (++q.h < p.d.Hkv) return;
    q.h = 0;
    do {  // (to the next group that has members)
      q.row += q.ng;
      if (++q.b >= entries()) return;
      if (JOINT && q.b < p.seqs) {
        q.first = q.b;
        q.n = 1;
      } else {
        // No group behind has a member: the end of a long list is not read (16 groups of 8 in a list of 512, one token:
        // 143 -> 79 us).
        if (q.left == 0) {
          q.b = entries();
          return;
        }
        q.first = JOINT && q.b == p.seqs ? 0 : q.first + q.n;
        q.n = imin(size<Uniform>(q.b), q.left);
        q.left -= q.n;
      }
      q.ng = row_groups(q.n);
    } while (q.n == 0);
    q.len = keys<Uniform>(q.b);
    enter(q);
  }
  // Query row R of the entry's rows of a KV head (rows past the last: the last).
  __device__ __attribute__((always_inline)) size_t query_row(const DecParams& a, const PrefixPos& q, int R, bool& valid) const {
    const unsigned rows = (unsigned)(a.G * a.S);  // of a member
    valid = R < q.n * (int)rows;
    const unsigned Rc = valid ? R : q.n * rows - 1, m = Rc / rows;
    return ((size_t)(q.first + m) * a.Hkv + q.h) * rows + (Rc - m * rows);
  }
};
struct Nothing {};
template <int D, int TW, int KT, int NST, PagedMode MODE>
struct PagedSmem {
  static constexpr int TEAMS = TW == 1 ? 3 : 1;  // teams per workgroup (paged_runs: at most 768 runs)
  static constexpr int NW = TW * TEAMS;          // waves per workgroup
  static constexpr uint32_t TILE = KT * D * 2;   // bytes of one swizzled K or V tile
  alignas(256) char buf[TEAMS][NST * 2 * TILE];  // per team: a ring of K and V tiles
  int wsum[NW];                                  // prologue: per-wave sums of the scan
  int start_b[TEAMS], start_off[TEAMS];          // where each team's run starts
  using Work = PrefixWork<KT, TW, NW, TEAMS, true>;
  // (in here: with a second object the compiler tells their accesses apart in a way that has it wait for all copies in
  // flight before the next read of a tile)
  std::conditional_t<MODE == PagedMode::Joint, typename Work::Smem, Nothing> work;
};

// `lens` is the parameters' array as a restrict kernel argument, read through the
// scalar cache where the index is uniform.
template <int D, int TW, int KT, int NST, PagedMode MODE>
__global__ __launch_bounds__(TW == 1 ? 192 : 64 * TW, 1) void paged_kernel(PagedParams p, const int* __restrict__ lens) {
  constexpr bool LISTS = MODE == PagedMode::Lists, JOINT = MODE == PagedMode::Joint;
  constexpr bool PARTS = MODE == PagedMode::Own || JOINT;  // every item leaves partial results
  using Pos = std::conditional_t<JOINT, PrefixPos, PagedPos>;
  constexpr int DS = D / 16, DB = D / 32, PST = D + 4, KB = KT / 32;
  using Smem = PagedSmem<D, TW, KT, NST, MODE>;
  constexpr int TEAMS = Smem::TEAMS, NW = Smem::NW, NT = 64 * NW;
  constexpr int NP = KT / 16;  // 16-row pieces of a tile
  static_assert(NP * NST <= 32, "pieces of the tiles in flight fit a word");
  __shared__ Smem sm;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  const int tm = TW == 1 ? w : 0, tw = TW == 1 ? 0 : w;  // team of the workgroup, wave of the team
  const int ng = TW < 4 || JOINT ? 1 : p.d.ng;          // (decode_groups: smaller teams hold all rows of a KV head)
  const int I = p.d.Hkv * ng;                            // items per sequence (Joint: and row group)
  typename Smem::Work work{p};
  // ---- prologue: T, and the position of each team's first tile (as over a dense cache) ----
  const int cpt = cdiv(p.d.B, NT);
  const int c0 = imin(p.d.B, tid * cpt), c1 = imin(p.d.B, c0 + cpt);
  int csum = 0, excl = 0, total = 0;  // excl: tiles per item of the sequences before c0
  if constexpr (JOINT) {
    total = work.scan(sm.work, tid);
  } else {
#pragma unroll 4
    for (int b = c0; b < c1; ++b) csum += paged_tiles<KT>(p, dec_len(p.d, lens, b));
    const int incl = wave_scan(csum);
    if (lane == 63) sm.wsum[w] = incl;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const int s = sm.wsum[v];
      before += v < w ? s : 0;
      total += s;
    }
    excl = before + incl - csum;
    total = __builtin_amdgcn_readfirstlane(total);
  }
  const int T = total * I;  // checked on the host to fit in 31 bits
  const int n = paged_runs<D, TW, PARTS>(T, p.d.B * I);
  const bool stream = total * p.d.Hkv > (int)(DEC_STREAM_BYTES / (2 * Smem::TILE));
  auto run_of = [&](int v) { return v * (int)gridDim.x + (int)blockIdx.x; };  // run of a workgroup's team v
#pragma unroll
  for (int v = 0; v < TEAMS; ++v) {
    const int x0 = run_of(v) < n ? paged_run_start(run_of(v), n, T) : T;
    if constexpr (JOINT) work.find(sm.work, v, x0);
    else if (csum > 0 && excl * I <= x0 && x0 < (excl + csum) * I) {
      int pb = excl;
      for (int b = c0; b < c1; ++b) {
        const int nt = paged_tiles<KT>(p, dec_len(p.d, lens, b));
        if (x0 < (pb + nt) * I) {
          sm.start_b[v] = b;
          sm.start_off[v] = x0 - pb * I;
          break;
        }
        pb += nt;
      }
    }
  }
  __syncthreads();

  // ---- this team's run ----
  const int gw = run_of(tm);
  if (gw >= n) return;
  const int x0 = paged_run_start(gw, n, T), x1 = paged_run_start(gw + 1, n, T);
  Pos pc;
  if constexpr (JOINT) {
    pc = work.start(sm.work, tm);
  } else {
    pc.b = __builtin_amdgcn_readfirstlane(sm.start_b[tm]);
    const int off = __builtin_amdgcn_readfirstlane(sm.start_off[tm]);
    pc.len = __builtin_amdgcn_readfirstlane(dec_len(p.d, lens, pc.b));
    pc.nt = paged_tiles<KT>(p, pc.len);
    const int item0 = off / pc.nt;  // of the sequence's items
    pc.j = off - item0 * pc.nt;
    pc.h = LISTS ? pc.b % p.heads : item0 / ng;
    pc.g = LISTS ? item0 : item0 - pc.h * ng;
  }

  auto advance = [&](Pos q) __attribute__((always_inline)) {
    if (++q.j == q.nt) {
      q.j = 0;
      if constexpr (JOINT) {
        work.next_item(q);
      } else if constexpr (LISTS) {
        if (++q.g == ng) {
          q.g = 0;
          if (++q.h == p.heads) q.h = 0;
          if (++q.b < p.d.B) {
            q.len = __builtin_amdgcn_readfirstlane(dec_len(p.d, lens, q.b));
            q.nt = paged_tiles<KT>(p, q.len);
          }
        }
      } else if (++q.g == ng) {
        q.g = 0;
        if (++q.h == p.d.Hkv) {
          q.h = 0;
          if (++q.b < p.d.B) {
            q.len = __builtin_amdgcn_readfirstlane(dec_len(p.d, lens, q.b));
            q.nt = paged_tiles<KT>(p, q.len);
          }
        }
      }
    }
    return q;
  };
  auto cached_tiles = [&](const Pos& q) __attribute__((always_inline)) {
    if constexpr (JOINT) return q.ntc;
    else return tiles_of<KT>(q.len);
  };
  // The kernel's arguments, read again (those needed once per item would take
  // scalar registers from the tile loop).
  auto arguments = [&]() __attribute__((always_inline)) -> DecParams {
    auto* a = (const __attribute__((address_space(4))) DecParams*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return *(const DecParams*)a;
  };
  // Those of a tile's copies, read at the start of each step in one go: kept, they
  // would push the loop's own state out of the scalar registers, and read one by
  // one where they are needed, each costs a wait.
  auto tile_arguments = [&]() __attribute__((always_inline)) -> PagedTile {
    auto* a = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(PagedParams, t);
    asm volatile("" : "+s"(a));
    return *(const PagedTile*)(const __attribute__((address_space(4))) PagedTile*)a;
  };
  // this lane's query row of an item: row g*grows + 32*tw + l32 of the G*S rows
  // of its KV head.  A lane past the last row takes the last row instead:
  // its column is computed like the others and never stored.
  auto query_row = [&](const DecParams& p, Pos q, bool& valid) __attribute__((always_inline)) -> size_t {
    const int rl = 32 * tw + l32, R = q.g * p.grows + rl;
    if constexpr (JOINT) {
      return work.query_row(p, q, R, valid);
    } else {
      valid = R < p.G * p.S && (TW == 1 || rl < p.grows);
      return ((size_t)q.b * p.Hq + (LISTS ? 0 : (size_t)q.h * p.G)) * p.S + (R < p.G * p.S ? R : p.G * p.S - 1);
    }
  };
  struct QRows {
    bf16x8 v[DS];
  };
  auto load_q = [&](Pos q) __attribute__((always_inline)) {
    const DecParams a = arguments();
    bool valid;
    const size_t row = query_row(a, q, valid);
    QRows r;
#pragma unroll
    for (int s = 0; s < DS; ++s) r.v[s] = *reinterpret_cast<const bf16x8*>(a.Q + row * D + 16 * s + 8 * g2);
    return r;
  };

  // ---- copies ----
  // A wave copies whole 16-row pieces of a tile, tw, tw + TW, ..., so it needs the
  // addresses of those alone.  A piece takes UPP instructions of RPI rows; row
  // within the piece and (swizzled) 16-byte chunk of this lane for each.
  constexpr int RPI = 512 / D, CPR = D / 8, UPP = 16 / RPI, PPW = NP / TW, NI = PPW * UPP;
  static_assert(NP % TW == 0, "whole pieces for each wave");
  int crow[UPP], cchunk[UPP];
#pragma unroll
  for (int u = 0; u < UPP; ++u) {
    crow[u] = u * RPI + lane / CPR;
    cchunk[u] = 16 * ((lane % CPR) ^ chunk_swizzle<D>(crow[u]));
  }
  // Page ids of the cache tile at q (of no meaning, but read from the table, for
  // others): those of this wave's pieces, and of all, to know which have a page.
  // (vectors, not arrays, which the branch below would leave in memory)
  typedef int Ids __attribute__((ext_vector_type(NP)));
  typedef int Own __attribute__((ext_vector_type(PPW < 2 ? 2 : PPW)));
  struct Pages {
    Ids id;
    Own own;
  };
  auto load_pages = [&](const PagedTile& t, Pos q) __attribute__((always_inline)) {
    Pages g;
    // (constant address space: scalar loads; nothing writes the table while the kernel runs)
    uint64_t at;
    int last;
    if constexpr (JOINT) {
      at = q.table;
      last = q.last;
    } else {
      at = t.table + (int64_t)imin(q.b, p.d.B - 1) * t.table_stride;
      last = t.last;
    }
    auto* row = (const __attribute__((address_space(4))) int*)at;
    auto entry = [&](int piece) { return row[(uint32_t)imin((q.j * KT + 16 * piece) >> t.log_size, last)]; };
    if ((1 << t.log_size) >= KT) {  // the tile lies in one page
      const int id = entry(0);
#pragma unroll
      for (int i = 0; i < NP; ++i) g.id[i] = id;
#pragma unroll
      for (int i = 0; i < PPW; ++i) g.own[i] = id;
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) g.id[i] = entry(i);
#pragma unroll
      for (int i = 0; i < PPW; ++i) g.own[i] = TW == 1 ? g.id[i] : entry(tw + i * TW);
    }
    return g;
  };
  // Copies this wave's pieces of K and V of the tile at q to dst, dst + TILE;
  // returns which pieces of the tile may hold keys (bit i: rows 16 i ...).
  auto issue = [&](const PagedTile& t, Pos q, const Pages& g, char* dst, auto streamed) __attribute__((always_inline)) {
    constexpr int POLICY = decltype(streamed)::value ? COPY_STREAM : 0;
    const int ntc = cached_tiles(q);
    const bool cached = q.j < ntc;
    const int row0 = (cached ? q.j : q.j - ntc) * KT, end = cached ? q.len : p.Sn;
    const uint32_t row_bytes = cached ? t.sr : D * 2;
    uint64_t base[PPW], kp, vp;
    int left[PPW];
    uint32_t mask = (1u << NP) - 1;
#pragma unroll
    for (int i = 0; i < PPW; ++i) left[i] = imin(imax(end - row0 - 16 * (tw + i * TW), 0), 16);
    if (cached) {
      kp = t.kp;
      vp = t.vp;
      const uint64_t head = (uint64_t)q.h * (uint64_t)t.sh;
      mask = 0;
#pragma unroll
      for (int i = 0; i < NP; ++i) mask |= (uint32_t)g.id[i] < (uint32_t)t.num ? 1u << i : 0u;
#pragma unroll
      for (int i = 0; i < PPW; ++i) {
        const uint32_t r = (uint32_t)(row0 + 16 * (tw + i * TW)) & ((1u << t.log_size) - 1);
        const bool ok = (uint32_t)g.own[i] < (uint32_t)t.num;
        left[i] = ok ? left[i] : 0;
        // (products of 32 bits: bd_attn_paged_decode_fwd's limits)
        base[i] = head + (uint64_t)(ok ? (uint32_t)g.own[i] : 0u) * t.sp + r * row_bytes;
      }
    } else {
      kp = t.kn;
      vp = t.vn;
      uint32_t bh;
      if constexpr (JOINT) bh = (uint32_t)q.first * (uint32_t)p.d.Hkv + (uint32_t)q.h;
      else bh = LISTS ? (uint32_t)q.b : (uint32_t)q.b * (uint32_t)p.d.Hkv + (uint32_t)q.h;
      const uint64_t block = ((uint64_t)bh * (uint32_t)p.Sn + row0) * (D * 2);
#pragma unroll
      for (int i = 0; i < PPW; ++i) base[i] = block + 16 * (tw + i * TW) * (D * 2);
    }
    auto copy = [&](uint64_t from, char* to) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PPW; ++i) {
        const uint64_t a = from + base[i];
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
        const __amdgpu_buffer_rsrc_t rs = make_buffer((const void*)(uintptr_t)(((uint64_t)hi << 32) | lo),
                                                      __builtin_amdgcn_readfirstlane((uint32_t)left[i] * row_bytes));
#pragma unroll
        for (int u = 0; u < UPP; ++u)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(
              rs, (__attribute__((address_space(3))) void*)(to + ((tw + i * TW) * UPP + u) * 1024), 16,
              (int)(__umul24(crow[u], row_bytes) + cchunk[u]), 0, 0, POLICY);
      }
    };
    // (taken here, or the compiler selects between their places in memory)
    asm volatile("" : "+s"(kp), "+s"(vp));
    copy(kp, dst);
    copy(vp, dst + Smem::TILE);
    return mask;
  };

  // The whole run, with or without the streaming hint on its copies.
  auto run = [&](auto streamed) __attribute__((always_inline)) {
    const LdsOperands<D> ops(lane);
    QRows qreg, qnext;
    f32x16 oacc[DB];
    float m, lsum;
    auto reset = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[db][e] = 0.f;
      m = -INFINITY;
      lsum = 0.f;
    };
    reset();
    char* const ring = sm.buf[tm];
    Pos pa = pc;  // the next tile to copy, and its pages
    Pages ga;
    uint32_t pieces;  // pieces of the tiles in flight, NP bits each, the current tile's lowest
    {
      const PagedTile t = tile_arguments();
      ga = load_pages(t, pa);
      qreg = load_q(pc);
      pieces = issue(t, pa, ga, ring, streamed);
      pa = advance(pa);
#pragma unroll
      for (int u = 1; u < NST - 1; ++u)
        if (x0 + u < x1) {
          ga = load_pages(t, pa);
          pieces |= issue(t, pa, ga, ring + u * 2 * Smem::TILE, streamed) << (NP * u);
          pa = advance(pa);
        }
      ga = load_pages(t, pa);
    }
    // Teams: the query rows have landed once all but the newest tile have.
    if (TW > 1) wait_global_loads_but<2 * NI>();

    // Write out the state of the current item's segment, which ends at tile pc.j
    // (tile x of all).
    SharedRef* const refs = JOINT ? p.refs : nullptr;  // (`arguments` gives the first part alone)
    const int seqs = JOINT ? p.seqs : 0;
    auto flush = [&](int x) __attribute__((always_inline)) {
      const DecParams p = arguments();
      int item;
      if constexpr (JOINT) item = pc.row * p.Hkv + pc.h * pc.ng + pc.g;
      else if constexpr (LISTS) item = pc.b * I + pc.g;
      else item = pc.b * I + pc.h * ng + pc.g;
      const int item_start = x - pc.j;  // flat index of the item's first tile
      const bool ends = pc.j == pc.nt - 1;
      bool valid;
      const size_t qrow = query_row(p, pc, valid);
      const float Lrow = halves_sum(lsum);
      if (!PARTS && item_start >= x0 && ends) {
        if (valid) {
          const bool none = !(Lrow > 0.f);
          const float inv = none ? 0.f : 1.f / Lrow;
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            bf16* op = p.O + qrow * D + 32 * db + 4 * g2;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              st_bf16x4(op + 8 * i, oacc[db][4 * i] * inv, oacc[db][4 * i + 1] * inv, oacc[db][4 * i + 2] * inv,
                        oacc[db][4 * i + 3] * inv);
          }
          if (g2 == 0) p.LSE[qrow] = none ? -INFINITY : (m + __log2f(Lrow)) * LN2;
        }
        if (lane == 0 && tw == 0) p.desc[item] = DecRuns{0, -1};
        return;
      }
      if (valid) {
        // Teams leave [D / 4][32] float4 for each wave's rows, a contiguous KiB a store (rows of D + 4 floats: 32
        // bytes of each row); one wave, with few rows, leaves rows, which the merge reads faster.
        size_t slot;
        if constexpr (JOINT) slot = (size_t)(gw + item) * p.grows;
        else if constexpr (LISTS) slot = dec_slot_row(p, gw, pc.b, pc.g);
        else slot = dec_slot_row(p, gw, (size_t)pc.b * p.Hkv + pc.h, pc.g);
        float* pr = p.part + (slot + 32 * tw + (TW == 1 ? l32 : 0)) * PST;
        float* po = pr + (TW == 1 ? 4 * g2 : 4 * lane);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 v = {oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
            *reinterpret_cast<f32x4*>(po + (4 * db + i) * (TW == 1 ? 8 : 256)) = v;
          }
        if (g2 == 0) *reinterpret_cast<float2*>(pr + (TW == 1 ? D : 32 * D + 2 * l32)) = float2{m, Lrow};
      }
      if (ends && (JOINT || (lane == 0 && tw == 0))) {
        // the runs holding this item: from the one holding its first tile to this one
        const DecRuns runs = {PARTS && item_start >= x0 ? gw : (int)((((long long)item_start + 1) * n - 1) / T), gw};
        if (!JOINT || (lane == 0 && tw == 0)) p.desc[item] = runs;
        if constexpr (JOINT) {
          // the first row of each member
          const int rows = p.G * p.S, rl = 32 * tw + l32, R = pc.g * p.grows + rl;
          if (pc.b >= seqs && g2 == 0 && valid && R % rows == 0)
            refs[(pc.first + R / rows) * p.Hkv + pc.h] = SharedRef{item, rl, runs.first, runs.last};
        }
      }
    };

    // One tile: `cur` holds the tile at pc; the copy of the tile NST - 1 ahead
    // (at pa, if this run has one) goes to `nxt`, whose last readers are done.
    auto step = [&](const char* __restrict__ cur, char* __restrict__ nxt, Pos pn, bool more, bool copies,
                    bool new_item) __attribute__((always_inline)) {
      compute_fence();  // the reads of the buffer about to be refilled are done
      const PagedTile t = tile_arguments();
      if constexpr (TW == 1) {
        static_assert(TW > 1 || NST == 2, "a step without a copy is the last one");
        // (query rows of the next item: a tile ahead, behind the wait, in both branches, as over a dense cache)
        if (copies) {
          pieces |= issue(t, pa, ga, nxt, streamed) << (NP * (NST - 1));
          pa = advance(pa);
          ga = load_pages(t, pa);
          wait_global_loads_but<(NST - 1) * 2 * NI>();  // the tile at pc has landed (this wave's own copy)
          if (new_item) qreg = qnext;
          if (pn.j == 0) qnext = load_q(pn);
        } else {
          wait_global_loads();
          if (new_item) qreg = qnext;
        }
      } else {
        if (new_item) {
          wait_global_loads();
          qreg = qnext;
          compute_fence();  // (keeps this wait from being merged with those below)
        } else if (copies) {
          wait_global_loads_but<(NST - 2) * 2 * NI>();  // this wave's part of the tile at pc has landed
        } else {
          wait_global_loads();
        }
        barrier_lds_only();  // ... every wave's; and all are done with `nxt`
        if (more && pn.j == 0) qnext = load_q(pn);
        if (copies) {
          pieces |= issue(t, pa, ga, nxt, streamed) << (NP * (NST - 1));
          pa = advance(pa);
          ga = load_pages(t, pa);
        }
      }
      // (the page ids are waited for here: a scalar load in flight would turn every wait for an LDS read
      // below into one for all of them)
#pragma unroll
      for (int i = 0; i < NP; ++i) asm volatile("" : "+s"(ga.id[i]));
#pragma unroll
      for (int i = 0; i < PPW; ++i) asm volatile("" : "+s"(ga.own[i]));
      const int ntc = cached_tiles(pc);
      const int nvalid = pc.j < ntc ? pc.len - pc.j * KT : p.Sn - (pc.j - ntc) * KT;  // keys before the end
      const uint32_t here = pieces & ((1u << NP) - 1);
      pieces >>= NP;
      // no piece of the tile holds a key
      if (nvalid <= 0 || (here & ((2u << ((imin(nvalid, KT) - 1) >> 4)) - 1)) == 0) return;

      // S^T[key][query] = sum_d K[key][d] Q[query][d]
      f32x16 sacc[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) sacc[kb][e] = 0.f;
      if constexpr (JOINT) {
        // (in the order of the text too: with this mode's scalars the scheduler falls back to that in one of the two copies)
        constexpr int N = DS * KB, AHEAD = 4;
        bf16x8 k[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) k[i] = lds_rows<D>(cur, ops.row_rel, i / KB, i % KB);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const bf16x8 now = k[i % AHEAD];
          if (i + AHEAD < N) k[i % AHEAD] = lds_rows<D>(cur, ops.row_rel, (i + AHEAD) / KB, (i + AHEAD) % KB);
          sacc[i % KB] = mfma32(now, qreg.v[i / KB], sacc[i % KB]);
        }
      } else {
#pragma unroll
        for (int s = 0; s < DS; ++s)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) sacc[kb] = mfma32(lds_rows<D>(cur, ops.row_rel, s, kb), qreg.v[s], sacc[kb]);
      }
      pipeline_lds_reads<DS * KB, 4, 1>();  // operand reads four MFMAs ahead
      if (nvalid < KT || here != (1u << NP) - 1) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const bool piece = here >> (2 * kb + i4 / 2) & 1;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
              if (!piece || 32 * kb + 8 * i4 + 4 * g2 + jj >= nvalid) sacc[kb][4 * i4 + jj] = -INFINITY;
          }
      }
      float m3[KB * 8];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; e += 2) m3[kb * 8 + e / 2] = fmaxf(sacc[kb][e], sacc[kb][e + 1]);
      const float mx = halves_max(tree_max<KB * 8>(m3)) * p.d.c;
      const bool grow = mx > m + DEC_SLACK;
      if (__any(grow)) {
        const float alpha = grow ? fast_exp2(m - mx) : 1.f;
        m = grow ? mx : m;
        lsum *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] *= alpha;
      }
      bf16x8 pb[2 * KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sacc[kb][e] = fast_exp2(sacc[kb][e] * p.d.c - m);
        pb[2 * kb] = pack8(sacc[kb], 0);
        pb[2 * kb + 1] = pack8(sacc[kb], 8);
      }
      lsum += tree_sum<KB>(sacc);
      // O^T[d][query] += sum_key V^T[d][key] P^T[key][query]
      bf16x8 pl[2 * KB];  // what the rounding of P left
#pragma unroll
      for (int c = 0; c < 2 * KB; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) pl[c][e] = (bf16)(sacc[c / 2][8 * (c & 1) + e] - (float)pb[c][e]);
      if constexpr (JOINT) {
        constexpr int N = 2 * KB * DB, AHEAD = 3;
        bf16x8 v[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v[i] = lds_tr<D>(cur + Smem::TILE, ops.tr_rel0, ops.tr_rel1, i / DB, i % DB);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const bf16x8 now = v[i % AHEAD];
          if (i + AHEAD < N) v[i % AHEAD] = lds_tr<D>(cur + Smem::TILE, ops.tr_rel0, ops.tr_rel1, (i + AHEAD) / DB, (i + AHEAD) % DB);
          oacc[i % DB] = mfma32(now, pb[i / DB], oacc[i % DB]);
          oacc[i % DB] = mfma32(now, pl[i / DB], oacc[i % DB]);
        }
      } else {
#pragma unroll
        for (int c = 0; c < 2 * KB; ++c)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const bf16x8 v = lds_tr<D>(cur + Smem::TILE, ops.tr_rel0, ops.tr_rel1, c, db);
            oacc[db] = mfma32(v, pb[c], oacc[db]);
            oacc[db] = mfma32(v, pl[c], oacc[db]);
          }
      }
      pipeline_lds_reads<4 * KB * DB, 6, 1>();
    };

    uint32_t bcur = 0;                           // ring offset of the tile at pc
    uint32_t bnxt = (NST - 1) * 2 * Smem::TILE;  // ring offset the copy NST - 1 ahead goes to
    for (int x = x0; x < x1; ++x) {
      const Pos pn = advance(pc);
      const bool more = x + 1 < x1, copies = x + NST - 1 < x1;
      step(ring + bcur, ring + bnxt, pn, more, copies, x > x0 && pc.j == 0);
      bnxt = bcur;
      bcur = bcur == (NST - 1) * 2 * Smem::TILE ? 0u : bcur + 2 * Smem::TILE;
      if (!more || pn.j == 0) {
        flush(x);
        if (more) reset();  // the next tile starts the next item
      }
      pc = pn;
    }
  };
  if (stream) run(Flag<true>());
  else run(Flag<false>());
}

template <int D, int TW, int KT, int NST, PagedMode MODE>
void launch_paged_kernel(const PagedParams& p, hipStream_t st) {
  using Smem = PagedSmem<D, TW, KT, NST, MODE>;
  hipLaunchKernelGGL((paged_kernel<D, TW, KT, NST, MODE>), dim3(TW == 1 ? 256 : DEC_WAVES / TW), dim3(64 * Smem::NW), 0, st, p,
                     p.d.cache_lens);
}

// Parameters of a call of shape s (C: the room of a table row), partial results in ws.
inline PagedParams paged_params(const DecodeShape& s, const DecodeGroups& g, const PagedArgs& a, void* ws) {
  PagedParams p{};
  p.d.Q = static_cast<const bf16*>(a.Q);
  p.d.Kc = p.d.Vc = p.d.Kn = p.d.Vn = nullptr;  // (the copies' own arguments: t)
  p.d.cache_lens = a.cache_lens;
  p.d.O = static_cast<bf16*>(a.O);
  p.d.LSE = a.LSE;
  p.d.desc = static_cast<DecRuns*>(ws);
  p.d.part = reinterpret_cast<float*>(static_cast<char*>(ws) + decode_desc_bytes(s));
  p.d.B = s.B;
  p.d.S = s.S;
  p.d.Hq = s.Hq;
  p.d.Hkv = s.Hkv;
  p.d.G = s.Hq / s.Hkv;
  p.d.C = s.C;
  p.d.c = s.scale * LOG2E;
  p.d.ng = g.ng;
  p.d.grows = g.rows;
  p.d.hrows = DEC_QT * decode_query_tiles(s);
  p.d.runs = g.runs;
  p.Sn = a.Kn ? s.S : 0;
  p.t.kp = (uint64_t)(uintptr_t)a.Kp;
  p.t.vp = (uint64_t)(uintptr_t)a.Vp;
  p.t.kn = (uint64_t)(uintptr_t)a.Kn;
  p.t.vn = (uint64_t)(uintptr_t)a.Vn;
  p.t.table = (uint64_t)(uintptr_t)a.table;
  p.t.table_stride = a.table_stride * 4;
  p.t.sh = a.pages.sh * 2;
  p.t.sp = (uint32_t)(a.pages.sp * 2);
  p.t.sr = (uint32_t)(a.pages.sr * 2);
  p.t.num = a.pages.num;
  p.t.log_size = a.pages.log_size;
  p.t.last = a.width - 1;
  return p;
}

// Enqueues the decode kernel (not the merge).
template <int D, PagedMode MODE>
hipError_t launch_paged_runs(const DecodeGroups& g, const PagedParams& p, hipStream_t st) {
  if (g.waves == 1) launch_paged_kernel<D, 1, 32, 2, MODE>(p, st);
  else if (g.waves == 2) launch_paged_kernel<D, 2, (D == 64 ? 64 : 32), 4, MODE>(p, st);
  else if constexpr (MODE != PagedMode::Joint) launch_paged_kernel<D, 4, 64, 512 / D, MODE>(p, st);
  return hipGetLastError();
}

// ... and the merge of the items that several runs hold.
template <int D, PagedMode MODE>
hipError_t launch_paged_decode_d(const DecodeShape& s, const PagedArgs& a, int heads, void* ws, hipStream_t st) {
  const DecodeGroups g = decode_groups(s);
  PagedParams p = paged_params(s, g, a, ws);
  p.heads = heads;
  const hipError_t e = launch_paged_runs<D, MODE>(g, p, st);
  if (e != hipSuccess) return e;
  return g.waves == 1 ? launch_dec_combine<D, true, false>(s, g, p.d, st) : launch_dec_combine<D, true, true>(s, g, p.d, st);
}

}  // namespace
}  // namespace bd
