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

// ---- prefixes with many query rows ----
//
// With more than 64 rows a row group the matrix products bound a prefix (512 bytes of K
// and V a key for 4 D flops a row, at D = 128 256 rows for each byte per cycle and CU that HBM gives), so this kernel
// differs from the paged one in what its tile loop spends beside them: a wave copies
// one 16-row piece of K or of V a tile (TW = 8), page ids come one tile ahead of the
// copies with the wait of the copies over them, and tiles without absent or missing
// keys, nearly all, take no test a key.
//   TW = 8: 256 rows, one workgroup a CU, two waves a SIMD.  Waves 4 to 7 (LAG) take the product with V
//   of a tile after the scores of their partners' next one, so that the two waves of a SIMD are
//   not at the same products and exponentials at the same time.
//   TW = 4: 128 rows, two workgroups a CU.
template <int D, int TW>
struct PrefixShape {
  static constexpr int KT = 64, NP = KT / 16;
  static constexpr bool PAIRS = TW == 8;                     // a wave copies a piece of K or of V, else of both
  static constexpr int NST = PAIRS || D == 64 ? 4 : 2;       // tiles in the ring
  static constexpr int AHEAD = PAIRS ? NST - 2 : NST - 1;    // copies run this many tiles ahead
  static constexpr uint32_t TILE = KT * D * 2;
  static constexpr int WORKGROUPS = 8 / TW;                  // a CU
};
// Scalars that stay in registers (and are not read again where they are needed).
template <class A, class B>
__device__ inline void keep(A& a, B& b) { asm volatile("" : "+s"(a), "+s"(b)); }

// A value that is the same in all lanes, in scalar registers.
__device__ inline uint64_t uniform(uint64_t a) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return (uint64_t)hi << 32 | lo;
}

// A value that the compiler knows nothing of from here on (so that nothing is computed from it before).
__device__ inline void opaque(int& a) { asm volatile("" : "+v"(a)); }

// (One object: with two, the compiler tells their accesses apart in a way that has it
// wait for all copies in flight before the next read of a tile.)
template <int D, int TW>
struct PrefixSmem {
  using Shape = PrefixShape<D, TW>;
  alignas(256) char buf[Shape::NST * 2 * Shape::TILE];  // K and V tiles
  typename PrefixWork<Shape::KT, TW, TW, 1>::Smem work;
};

template <int D, int TW>
__global__ __launch_bounds__(64 * TW, 2) void prefix_kernel(PagedParams p, const int* __restrict__ lens) {
  using Shape = PrefixShape<D, TW>;
  constexpr int KT = Shape::KT, NP = Shape::NP, NST = Shape::NST, AHEAD = Shape::AHEAD, ROWS = 32 * TW;
  constexpr int DS = D / 16, DB = D / 32, PST = D + 4, KB = KT / 32;
  constexpr uint32_t TILE = Shape::TILE;
  constexpr int RPI = 512 / D, CPR = D / 8, UPP = 16 / RPI;  // rows of an instruction, 16-byte chunks of a row, instructions of a piece
  constexpr int COPIES = Shape::PAIRS ? UPP : 2 * UPP;       // instructions of a wave and tile
  using Work = PrefixWork<KT, TW, TW, 1>;
  __shared__ PrefixSmem<D, TW> sm;

  const int tid = threadIdx.x, lane = tid & 63;
  const int tw = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  // The kernel's arguments, read again: what is needed once an item, kept, would take the
  // scalar registers of the tile loop, which would then read its own arguments again and again.
  auto arguments = [&]() __attribute__((always_inline)) -> PagedParams {
    auto* a = (const __attribute__((address_space(4))) PagedParams*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return *(const PagedParams*)a;
  };
  Work work{p, lens};
  const int T = work.scan(sm.work, tid) * p.d.Hkv;  // checked on the host to fit in 31 bits
  const int n = imin(256 * Shape::WORKGROUPS, cdiv(T, 2));  // runs (two tiles at least, as dec_runs)
  const int gw = blockIdx.x;
  if (gw >= n) return;
  const int x0 = paged_run_start(gw, n, T), x1 = paged_run_start(gw + 1, n, T);
  work.find(sm.work, 0, x0);
  __syncthreads();
  PrefixPos pc = work.start(sm.work, 0), pa = pc;  // the tile to compute, the tile to copy
  const LdsOperands<D> ops(lane);

  // ---- copies ----
  const int piece = tw & (NP - 1);
  // What the tile loop needs of the arguments, in registers of its own.
  uint32_t sp = p.t.sp, sr = p.t.sr;
  int num = p.t.num, log_size = p.t.log_size, last_entry = p.t.last;
  float c = p.d.c;
  keep(sp, sr);
  keep(num, log_size);
  keep(last_entry, c);
  int coff[UPP];  // bytes from a piece to this lane's chunk of each instruction
#pragma unroll
  for (int u = 0; u < UPP; ++u) {
    const int row = u * RPI + lane / CPR;
    coff[u] = row * (int)sr + 16 * ((lane % CPR) ^ chunk_swizzle<D>(row));
  }
  // Of the item at pa: the arrays at its KV head (PAIRS: the one this wave copies from), its row of the table.
  uint64_t k_head, v_head, table_row;
  auto copy_item = [&]() __attribute__((always_inline)) {
    const PagedParams a = arguments();
    const uint64_t head = (uint64_t)pa.h * (uint64_t)a.t.sh;
    k_head = (Shape::PAIRS && tw >= NP ? a.t.vp : a.t.kp) + head;
    v_head = a.t.vp + head;
    table_row = a.t.table + (int64_t)imin(pa.b, a.d.B - 1) * a.t.table_stride;
  };
  // Ids of the pages that hold the pieces of the tile at pa, and of this wave's piece.
  struct Pages {
    int id[NP], own;
  };
  auto pages_of = [&]() __attribute__((always_inline)) {
    Pages g;
    auto* row = (const __attribute__((address_space(4))) int*)table_row;
    auto entry = [&](int i) { return row[(uint32_t)imin((pa.j * KT + 16 * i) >> log_size, last_entry)]; };
    if ((1 << log_size) >= KT) {  // the tile lies in one page
      g.own = entry(0);
#pragma unroll
      for (int i = 0; i < NP; ++i) g.id[i] = g.own;
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) g.id[i] = entry(i);
      g.own = entry(piece);
    }
    return g;
  };
  // (a scalar load in flight lengthens every wait for an LDS read)
  auto landed = [&](Pages& g) __attribute__((always_inline)) {
    keep(g.id[0], g.id[1]);
    keep(g.id[2], g.id[3]);
    keep(g.own, last_entry);
  };
  auto next_item = [&](PrefixPos& q) __attribute__((always_inline)) {
    const PagedParams a = arguments();
    Work{a, a.d.cache_lens}.next_item(q);
  };
  int next = 0;           // ring slot of the next copy
  uint32_t present = 0;  // pieces of the tiles in flight that have a page, NP bits each, the next tile's lowest
  Pages pages;            // of the tile at pa
  uint64_t k_rows = 0, v_rows = 0;  // where its rows start, and their bytes
  uint32_t row_bytes = 0;
  // Readies the copy of the tile at pa (not `some`: one that reads nothing), the `ahead`-th from the one computed, and moves on.
  auto prepare = [&](bool some, int ahead) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NP; ++i) present |= (uint32_t)pages.id[i] < (uint32_t)num ? 1u << (NP * ahead + i) : 0u;
    const int row0 = pa.j * KT + 16 * piece;
    const bool ok = some && (uint32_t)pages.own < (uint32_t)num;
    const int left = ok ? imin(imax(pa.len - row0, 0), 16) : 0;
    const uint32_t r = (uint32_t)row0 & ((1u << log_size) - 1);
    // (products of 32 bits: the limits of the paged calls)
    const uint64_t off = (uint64_t)(ok ? (uint32_t)pages.own : 0u) * sp + r * sr;
    k_rows = uniform(k_head + off);
    if constexpr (!Shape::PAIRS) v_rows = uniform(v_head + off);
    row_bytes = __builtin_amdgcn_readfirstlane((uint32_t)left * sr);
    next = next + 1 == NST ? 0 : next + 1;
    if (some && ++pa.j == pa.nt) {
      next_item(pa);
      copy_item();
    }
  };
  // Instruction u of it, into the slot at dst.
  auto copy = [&](char* dst, int u) __attribute__((always_inline)) {
    const bool value = Shape::PAIRS ? tw >= NP : u >= UPP;
    const int i = u % UPP;
    const __amdgpu_buffer_rsrc_t rs = make_buffer((const void*)(uintptr_t)(!Shape::PAIRS && u >= UPP ? v_rows : k_rows), row_bytes);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rs, (__attribute__((address_space(3))) void*)(dst + (value ? TILE : 0) + (piece * UPP + i) * 1024), 16, (int)(coff[i] + 0), 0, 0, 0);
  };

  // ---- one wave's rows ----
  bf16x8 qreg[DS];
  auto load_q = [&]() __attribute__((always_inline)) {
    const PagedParams a = arguments();
    bool valid;
    const size_t row = Work{a, nullptr}.query_row(a.d, pc, pc.g * ROWS + 32 * tw + l32, valid);
#pragma unroll
    for (int s = 0; s < DS; ++s) qreg[s] = *reinterpret_cast<const bf16x8*>(a.d.Q + row * D + 16 * s + 8 * g2);
  };
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
  uint32_t ph[KB * 8], pl[KB * 8];  // P in pairs of keys: rounded, and what the rounding left
  bool some = false;                // does the last tile of `scores` hold a key?
  // P of a tile of scores, of whose first `valid` rows those in the pieces `here` are keys.
  auto softmax = [&](f32x16* sacc, int valid, uint32_t here) __attribute__((always_inline)) {
    some = valid > 0 && (here & ((2u << ((imin(valid, KT) - 1) >> 4)) - 1)) != 0;
    if (!some) return;
    if (valid < KT || here != (1u << NP) - 1) {
      int above = 4 * g2;
      opaque(above);  // (a branch that nearly all tiles pass: nothing of it is computed before)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int end = here >> (2 * kb + i4 / 2) & 1 ? valid - 32 * kb - 8 * i4 : 0;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj)
            if (above + jj >= end) sacc[kb][4 * i4 + jj] = -INFINITY;
        }
    }
    float m3[KB * 8];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; e += 2) m3[kb * 8 + e / 2] = fmaxf(sacc[kb][e], sacc[kb][e + 1]);
    const float mx = halves_max(tree_max<KB * 8>(m3)) * c;
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
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sacc[kb][e] = fast_exp2(sacc[kb][e] * c - m);
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const uint32_t h = pack2(sacc[kb][e], sacc[kb][e + 1]);
        ph[kb * 8 + e / 2] = h;
        pl[kb * 8 + e / 2] = pack2(sacc[kb][e] - __uint_as_float(h << 16), sacc[kb][e + 1] - __uint_as_float(h & 0xffff0000u));
      }
    }
    lsum += tree_sum<KB>(sacc);
  };
  // Leaves the partial result of the item that ends at, or is cut behind, tile x (at q).
  auto flush = [&](const PrefixPos& q, int x) __attribute__((always_inline)) {
    const PagedParams p = arguments();
    const int item = q.row * p.d.Hkv + q.h * q.ng + q.g;
    const bool ends = q.j == q.nt - 1;
    const int R = q.g * ROWS + 32 * tw + l32, per = p.d.G * p.d.S;
    const bool valid = R < q.n * per;
    const float Lrow = halves_sum(lsum);
    if (valid) {
      float* pr = p.d.part + ((size_t)(gw + item) * ROWS + 32 * tw) * PST;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 v = {oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
          *reinterpret_cast<f32x4*>(pr + 4 * lane + (4 * db + i) * 256) = v;
        }
      if (g2 == 0) *reinterpret_cast<float2*>(pr + 32 * D + 2 * l32) = float2{m, Lrow};
      if (ends && q.h == 0 && g2 == 0 && R % per == 0) p.refs[q.first + R / per] = SharedRef{q.row * p.d.Hkv, q.ng, R};
    }
    if (ends && lane == 0 && tw == 0)
      p.d.desc[item] = DecRuns{x - q.j >= x0 ? gw : (int)((((long long)(x - q.j) + 1) * n - 1) / T), gw};
  };

  // ---- the run ----
  copy_item();
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) {
    pages = pages_of();
    char* const dst = sm.buf + next * (2 * TILE);
    prepare(x0 + a < x1, a);
#pragma unroll
    for (int u = 0; u < COPIES; ++u) copy(dst, u);
  }
  pages = pages_of();
  landed(pages);
  load_q();
  wait_global_loads();
  compute_fence();
  reset();

  // The tile at x has landed for all waves, and the slot of the copy AHEAD tiles on is read no more.
  auto arrive = [&]() __attribute__((always_inline)) {
    compute_fence();
    wait_global_loads_but<(AHEAD - 1) * COPIES>();
    barrier_lds_only();
    compute_fence();
  };
  auto begin = [&]() __attribute__((always_inline)) {  // the next item's rows
    load_q();
    wait_global_loads();
    compute_fence();
    reset();
  };
  PrefixPos last = pc;
  // (restrict: tiles are read from cur and old, and copied to nxt.  Otherwise the compiler waits for every copy before
  // it reads any.  It has to see these reads here, not in a lambda.)
  auto step = [&](const char* __restrict__ cur, const char* __restrict__ values, char* __restrict__ nxt, int x,
                  auto lag) __attribute__((always_inline)) {
    constexpr bool LAG = decltype(lag)::value;
    if (!LAG || x < x1) arrive();
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      if (part == (LAG ? 0 : 1)) {
        // O^T[d][query] += sum_key V^T[d][key] P^T[key][query]
        if (some) {
#pragma unroll
          for (int c = 0; c < 2 * KB; ++c) {
            const bf16x8 hi = __builtin_bit_cast(bf16x8, (u32x4{ph[4 * c], ph[4 * c + 1], ph[4 * c + 2], ph[4 * c + 3]}));
            const bf16x8 lo = __builtin_bit_cast(bf16x8, (u32x4{pl[4 * c], pl[4 * c + 1], pl[4 * c + 2], pl[4 * c + 3]}));
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              const bf16x8 v = lds_tr<D>(values + TILE, ops.tr_rel0, ops.tr_rel1, c, db);
              oacc[db] = mfma32(v, hi, oacc[db]);
              oacc[db] = mfma32(v, lo, oacc[db]);
            }
          }
          pipeline_lds_reads<4 * KB * DB, 6, 1>();
        }
        if (LAG && x > x0 && (pc.j == 0 || x == x1)) {
          flush(last, x - 1);
          if (x < x1) begin();
        }
      } else if (!LAG || x < x1) {
        if (!LAG && x > x0 && pc.j == 0) begin();
        prepare(x + AHEAD < x1, AHEAD);
        compute_fence();
        // S^T[key][query] = sum_d K[key][d] Q[query][d]
        f32x16 sacc[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) sacc[kb][e] = 0.f;
#pragma unroll
        for (int s = 0; s < DS; ++s)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) sacc[kb] = mfma32(lds_rows<D>(cur, ops.row_rel, s, kb), qreg[s], sacc[kb]);
#pragma unroll
        for (int u = 0; u < COPIES; ++u) copy(nxt, u);
        pipeline_reads_and_copies<DS * KB, 4, 1, COPIES>();
        compute_fence();
        pages = pages_of();
        softmax(sacc, pc.len - pc.j * KT, present & ((1u << NP) - 1));
        landed(pages);
        present >>= NP;
      }
    }
    if (!LAG && (pc.j == pc.nt - 1 || x + 1 == x1)) flush(pc, x);
  };
  auto tiles = [&](auto lag) __attribute__((always_inline)) {
    int slot = 0, before = 0;
    for (int x = x0; x < (decltype(lag)::value ? x1 + 1 : x1); ++x) {
      step(sm.buf + slot * (2 * TILE), sm.buf + (decltype(lag)::value ? before : slot) * (2 * TILE), sm.buf + next * (2 * TILE), x, lag);
      before = slot;
      slot = slot + 1 == NST ? 0 : slot + 1;
      last = pc;
      if (++pc.j == pc.nt) next_item(pc);
    }
  };
  if (Shape::PAIRS && tw >= NP) tiles(Flag<true>());
  else tiles(Flag<false>());
  wait_global_loads();
}

template <int D, int TW>
hipError_t launch_prefix(const PagedParams& p, hipStream_t st) {
  hipLaunchKernelGGL((prefix_kernel<D, TW>), dim3(256 * PrefixShape<D, TW>::WORKGROUPS), dim3(64 * TW), 0, st, p, p.d.cache_lens);
  return hipGetLastError();
}

// ---- the merge ----

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
__global__ __launch_bounds__((DEC_MERGE_THREADS<P, OWN_COLS || PRE_COLS>)) void shared_merge_kernel(MergeParams p) {
  constexpr bool COLS = OWN_COLS || PRE_COLS;  // consecutive threads take consecutive rows
  constexpr int NT = DEC_MERGE_THREADS<P, COLS>, TPR = D / 4, RPW = NT / (TPR * P);
  static_assert(RPW >= 1, "a workgroup holds whole rows");
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

template <int D, bool OWN_COLS, bool PRE_COLS>
void launch_merge_as(const MergeParams& p, bool many, hipStream_t st) {
  constexpr bool COLS = OWN_COLS || PRE_COLS;
  const size_t rows = (size_t)p.own.B * p.own.Hq * p.own.S;
  const auto merge = [&](auto parts) {
    constexpr int P = decltype(parts)::value, NT = DEC_MERGE_THREADS<P, COLS>, RPW = NT / (D / 4 * P);
    hipLaunchKernelGGL((shared_merge_kernel<D, P, OWN_COLS, PRE_COLS>), dim3((unsigned)((rows + RPW - 1) / RPW)), dim3(NT), 0,
                       st, p);
  };
  if (many) merge(std::integral_constant<int, COLS ? 4 : 8>());
  else merge(std::integral_constant<int, 1>());
}
template <int D>
void launch_merge(const MergeParams& p, bool own_cols, bool pre_cols, bool many, hipStream_t st) {
  if (own_cols) {
    if (pre_cols) launch_merge_as<D, true, true>(p, many, st);
    else launch_merge_as<D, true, false>(p, many, st);
  } else {
    if (pre_cols) launch_merge_as<D, false, true>(p, many, st);
    else launch_merge_as<D, false, false>(p, many, st);
  }
}

template <int D>
hipError_t launch_shared_d(const DecodeShape& s, const SharedArgs& a, void* ws, hipStream_t st) {
  char* const pre_ws = static_cast<char*>(ws) + shared_own_bytes(s);
  const DecodeGroups g = decode_groups(s);
  const PagedParams own = paged_params(s, g, a.own, ws);

  const int waves = shared_waves(s, a.groups);
  const DecodeGroups gp = {waves, 1, DEC_QT * waves, shared_runs(waves)};
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

  hipError_t e = waves == 8   ? launch_prefix<D, 8>(pre, st)
                 : waves == 4 ? launch_prefix<D, 4>(pre, st)
                              : launch_paged_runs<D, PagedMode::Prefix>(gp, pre, st);
  if (e != hipSuccess) return e;
  e = launch_paged_runs<D, PagedMode::Own>(g, own, st);
  if (e != hipSuccess) return e;
  const MergeParams m = {own.d, pre.d, pre.refs, pre.members};
  // (as launch_dec_combine: eight runs or more an item)
  const size_t prefixes = (size_t)s.Hkv * ((size_t)s.B * (s.Hq / s.Hkv) * s.S / gp.rows + 1);
  const bool many = decode_items(s) * 8 <= (size_t)g.runs || prefixes * 8 <= (size_t)gp.runs;
  launch_merge<D>(m, g.waves > 1, waves > 1, many, st);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_decode(const DecodeShape& s, const SharedArgs& a, void* ws, hipStream_t st) {
  return s.D == 128 ? launch_shared_d<128>(s, a, ws, st) : launch_shared_d<64>(s, a, ws, st);
}

}  // namespace bd
