// Decoding over a paged KV cache for gfx950 where groups of consecutive sequences
// share a prefix, as the samples of one prompt do: the S queries of each sequence
// attend to the prefix_lens[g] keys of their group's prefix, to the cache_lens[b]
// keys of their own, and, if given, to the block's own S keys.
//
// The softmax splits over any partition of the keys: with (m, l, o) the maximum,
// sum and unnormalised output over a part,
//   M = max_i m_i,  O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.
// So the prefix is taken once for the n G S query rows that all members have for
// a KV head, in groups of rows that run at about the same time and read its K and V
// from HBM once.  Few rows, or short prefixes (kernels.hpp): prefixes and own keys
// are items of one launch of the paged kernel (paged.hpp, Joint).  Else one launch
// does the prefixes, here, and one the own keys.  A last one joins the partial results.
#include "paged.hpp"

namespace bd {
namespace {

// ---- prefixes with many query rows ----
//
// The matrix products bound a prefix with many rows: a key's 512 bytes of K and V (D = 128) go
// with 6 D flops a row, P being two bfloat16 parts.  What the tile loop spends beside them is kept
// small: a workgroup takes 128 rows, and a wave copies one 16-row piece of K and of V a tile;
// page ids come a tile ahead of the copies, by scalar loads that are waited for under the softmax;
// tiles without absent or missing keys, nearly all, take no test a key.  Two workgroups share
// a CU, so that one is at its products while the other is at its exponentials.
//   One group of 24 sequences of 32 queries, 4 query heads a KV head, 8 KV heads, D = 128: on a prefix of 8000 keys 176 us
//   a call, 573 TFLOP/s of the two products as they are defined (860 executed); on one of 64,000 1167 us, 690 TFLOP/s.
// MFMA busy 0.41: a wave's products and its exponentials take about as long and overlap with the other workgroup's only.
// Measured against it: 256 rows a workgroup of eight waves, half of them a product behind the
// others, the same there and 5% to 2% either way elsewhere.
constexpr int PREFIX_WAVES = 4, PREFIX_WORKGROUPS = 2;  // of a workgroup; a CU
template <int D>
struct PrefixShape {
  static constexpr int KT = 64, NP = KT / 16;
  static constexpr int NST = D == 64 ? 4 : 2;  // tiles in the ring
  static constexpr int AHEAD = NST - 1;        // copies run this many tiles ahead
  static constexpr uint32_t TILE = KT * D * 2;
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
template <int D>
struct PrefixSmem {
  using Shape = PrefixShape<D>;
  alignas(256) char buf[Shape::NST * 2 * Shape::TILE];  // K and V tiles
  typename PrefixWork<Shape::KT, PREFIX_WAVES, PREFIX_WAVES, 1, false>::Smem work;
};

template <int D>
__global__ __launch_bounds__(64 * PREFIX_WAVES, PREFIX_WORKGROUPS) void prefix_kernel(PagedParams p) {
  using Shape = PrefixShape<D>;
  constexpr int TW = PREFIX_WAVES, KT = Shape::KT, NP = Shape::NP, NST = Shape::NST, AHEAD = Shape::AHEAD, ROWS = 32 * TW;
  constexpr int DS = D / 16, DB = D / 32, PST = D + 4, KB = KT / 32;
  constexpr uint32_t TILE = Shape::TILE;
  constexpr int RPI = 512 / D, CPR = D / 8, UPP = 16 / RPI;  // rows of an instruction, 16-byte chunks of a row, instructions of a piece
  constexpr int COPIES = 2 * UPP;                            // instructions of a wave and tile
  using Work = PrefixWork<KT, TW, TW, 1, false>;
  __shared__ PrefixSmem<D> sm;

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
  Work work{p};
  const int T = work.scan(sm.work, tid) * p.d.Hkv;  // checked on the host to fit in 31 bits
  const int n = imin(256 * PREFIX_WORKGROUPS, cdiv(T, 2));  // runs (two tiles at least, as dec_runs)
  // Consecutive runs on one die, whose L2 then holds more of the prefix for the row groups of a KV head: three groups
  // of 8, blocks of 32, prefixes of 4096 to 8192, 526 -> 304 MB fetched, 141.7 -> 139.1 us; the 8000 keys above 179 -> 175,
  // the 64,000 1152 -> 1168.
  const int per = cdiv(n, 8), gw = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || gw >= n) return;
  const int x0 = paged_run_start(gw, n, T), x1 = paged_run_start(gw + 1, n, T);
  work.find(sm.work, 0, x0);
  __syncthreads();
  PrefixPos pc = work.start(sm.work, 0), pa = pc;  // the tile to compute, the tile to copy
  const LdsOperands<D> ops(lane);

  // ---- copies ----
  static_assert(NP == TW, "a wave copies one 16-row piece of K and of V");
  const int piece = tw;
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
  // Of the item at pa: the arrays at its KV head, its row of the table.
  uint64_t k_head, v_head, table_row;
  auto copy_item = [&]() __attribute__((always_inline)) {
    const PagedParams a = arguments();
    const uint64_t head = (uint64_t)pa.h * (uint64_t)a.t.sh;
    k_head = a.t.kp + head;
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
    Work{a}.next_item(q);
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
    v_rows = uniform(v_head + off);
    row_bytes = __builtin_amdgcn_readfirstlane((uint32_t)left * sr);
    next = next + 1 == NST ? 0 : next + 1;
    if (some && ++pa.j == pa.nt) {
      next_item(pa);
      copy_item();
    }
  };
  // Instruction u of it, into the slot at dst.
  auto copy = [&](char* dst, int u) __attribute__((always_inline)) {
    const bool value = u >= UPP;
    const int i = u % UPP;
    const __amdgpu_buffer_rsrc_t rs = make_buffer((const void*)(uintptr_t)(value ? v_rows : k_rows), row_bytes);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rs, (__attribute__((address_space(3))) void*)(dst + (value ? TILE : 0) + (piece * UPP + i) * 1024), 16, (int)(coff[i] + 0), 0, 0, 0);
  };

  // ---- one wave's rows ----
  bf16x8 qreg[DS];
  auto load_q = [&]() __attribute__((always_inline)) {
    const PagedParams a = arguments();
    bool valid;
    const size_t row = Work{a}.query_row(a.d, pc, pc.g * ROWS + 32 * tw + l32, valid);
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
    }
    if (ends) {
      const DecRuns runs = {x - q.j >= x0 ? gw : (int)((((long long)(x - q.j) + 1) * n - 1) / T), gw};
      if (lane == 0 && tw == 0) p.d.desc[item] = runs;
      if (valid && g2 == 0 && R % per == 0)  // the first row of each member
        p.refs[(q.first + R / per) * p.d.Hkv + q.h] = SharedRef{item, 32 * tw + l32, runs.first, runs.last};
    }
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
  // (restrict: a tile is read from cur and one copied to nxt.  Otherwise the compiler waits for every copy before
  // it reads any.  It has to see these reads here, not in a lambda.)
  auto step = [&](const char* __restrict__ cur, char* __restrict__ nxt, int x) __attribute__((always_inline)) {
    arrive();
    if (x > x0 && pc.j == 0) begin();
    prepare(x + AHEAD < x1, AHEAD);
    compute_fence();
    // S^T[key][query] = sum_d K[key][d] Q[query][d]
    f32x16 sacc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) sacc[kb][e] = 0.f;
    constexpr int K_AHEAD = 4;
    bf16x8 k[K_AHEAD];
#pragma unroll
    for (int i = 0; i < K_AHEAD; ++i) k[i] = lds_rows<D>(cur, ops.row_rel, i / KB, i % KB);
#pragma unroll
    for (int i = 0; i < DS * KB; ++i) {
      const bf16x8 now = k[i % K_AHEAD];
      if (i + K_AHEAD < DS * KB) k[i % K_AHEAD] = lds_rows<D>(cur, ops.row_rel, (i + K_AHEAD) / KB, (i + K_AHEAD) % KB);
      sacc[i % KB] = mfma32(now, qreg[i / KB], sacc[i % KB]);
      if (i % (DS * KB / COPIES) == 0) copy(nxt, i / (DS * KB / COPIES));
    }
    pipeline_reads_and_copies<DS * KB, 4, 1, COPIES>();
    compute_fence();
    pages = pages_of();
    softmax(sacc, pc.len - pc.j * KT, present & ((1u << NP) - 1));
    landed(pages);
    present >>= NP;
    // O^T[d][query] += sum_key V^T[d][key] P^T[key][query]
    if (some) {
      // (the reads ahead are in the order of the text too: the scheduler, short of registers, may keep that)
      constexpr int N = 2 * KB * DB, V_AHEAD = 3;
      bf16x8 v[V_AHEAD];
#pragma unroll
      for (int i = 0; i < V_AHEAD; ++i) v[i] = lds_tr<D>(cur + TILE, ops.tr_rel0, ops.tr_rel1, i / DB, i % DB);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = i / DB, db = i % DB;
        const bf16x8 hi = __builtin_bit_cast(bf16x8, (u32x4{ph[4 * c], ph[4 * c + 1], ph[4 * c + 2], ph[4 * c + 3]}));
        const bf16x8 lo = __builtin_bit_cast(bf16x8, (u32x4{pl[4 * c], pl[4 * c + 1], pl[4 * c + 2], pl[4 * c + 3]}));
        const bf16x8 now = v[i % V_AHEAD];
        if (i + V_AHEAD < N)
          v[i % V_AHEAD] = lds_tr<D>(cur + TILE, ops.tr_rel0, ops.tr_rel1, (i + V_AHEAD) / DB, (i + V_AHEAD) % DB);
        oacc[db] = mfma32(now, hi, oacc[db]);
        oacc[db] = mfma32(now, lo, oacc[db]);
      }
      pipeline_lds_reads<4 * KB * DB, 6, 1>();
    }
    if (pc.j == pc.nt - 1 || x + 1 == x1) flush(pc, x);
  };
  int slot = 0;
  for (int x = x0; x < x1; ++x) {
    step(sm.buf + slot * (2 * TILE), sm.buf + next * (2 * TILE), x);
    slot = slot + 1 == NST ? 0 : slot + 1;
    if (++pc.j == pc.nt) next_item(pc);
  }
  wait_global_loads();
}

template <int D>
hipError_t launch_prefix(const PagedParams& p, hipStream_t st) {
  hipLaunchKernelGGL((prefix_kernel<D>), dim3(256 * PREFIX_WORKGROUPS), dim3(64 * PREFIX_WAVES), 0, st, p);
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
// JOINT: both in the prefixes' arrays, the sequences' own items first.
template <int D, int P, bool OWN_COLS, bool PRE_COLS, bool JOINT>
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
    const int g = R / p.own.grows, b = (int)(bh / p.own.Hkv);
    const int mine = (int)bh * p.own.ng + g;
    const DecRuns d = p.own.desc[mine];
    const SharedRef ref = p.refs[bh];  // (of no meaning without a prefix)
    DecRuns e = {0, -1};
    int r2 = 0, item = 0;
    if (b < *p.members) {
      const int G2 = (ref.row0 + R) / p.pre.grows;  // items behind that of the member's first row
      r2 = ref.row0 + R - G2 * p.pre.grows;
      item = ref.item + G2;
      e = G2 == 0 ? DecRuns{ref.first, ref.last} : p.pre.desc[item];
    }
#pragma unroll 4
    for (int gw = d.first + part; gw <= d.last; gw += P)
      merge_part<D, OWN_COLS>(s, p.own.part,
                              JOINT ? (size_t)(gw + mine) * p.own.grows : dec_slot_row(p.own, gw, bh, g), R - g * p.own.grows, q4);
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

// What bounds it: reading the partial results, 528 bytes a row and run (D = 128; 21,504 rows, 6.2 runs each, 71 MB: 14 us,
// 5.5 TB/s with what it writes), and below 20 MB the latency of two dependent loads.
// Several threads a row's runs where the rows alone do not fill the card, us (D = 128, one thread, several):
//   512 rows 25.5 21.9; 1024 rows 32.2 29.4 and 30.8 29.3; 2048 rows 34.2 32.6; 4096 rows 39.5 41.2 and 40.4 41.5.
template <int D, bool OWN_COLS, bool PRE_COLS, bool JOINT = false>
void launch_merge_as(const MergeParams& p, hipStream_t st) {
  constexpr bool COLS = OWN_COLS || PRE_COLS;
  const size_t rows = (size_t)p.own.B * p.own.Hq * p.own.S;
  const bool many = rows * (D / 4) <= 65536;
  const auto merge = [&](auto parts) {
    constexpr int P = decltype(parts)::value, NT = DEC_MERGE_THREADS<P, COLS>, RPW = NT / (D / 4 * P);
    hipLaunchKernelGGL((shared_merge_kernel<D, P, OWN_COLS, PRE_COLS, JOINT>), dim3((unsigned)((rows + RPW - 1) / RPW)), dim3(NT), 0,
                       st, p);
  };
  if (many) merge(std::integral_constant<int, COLS ? 4 : 8>());
  else merge(std::integral_constant<int, 1>());
}
template <int D>
hipError_t launch_shared_d(const SharedShape& sh, const SharedArgs& a, void* ws, hipStream_t st) {
  const DecodeShape& s = sh.s;
  const int waves = shared_waves(sh);
  const bool joint = shared_joint(sh);
  char* const pre_ws = static_cast<char*>(ws) + (joint ? 0 : shared_own_bytes(s));
  const size_t items = shared_items(sh);
  const DecodeGroups gp = {waves, 1, DEC_QT * waves, shared_runs(waves)};
  PagedArgs pa = a.own;
  pa.table = a.table;
  pa.width = a.width;
  pa.table_stride = a.table_stride;
  pa.cache_lens = a.lens;
  PagedParams pre = paged_params(s, gp, pa, ws);
  pre.d.B = sh.groups;
  pre.d.C = sh.C;
  pre.d.desc = reinterpret_cast<DecRuns*>(pre_ws);
  pre.d.part = reinterpret_cast<float*>(pre_ws + shared_desc_bytes(sh));
  pre.sizes = a.sizes;
  pre.seqs = s.B;
  pre.refs = reinterpret_cast<SharedRef*>(pre_ws) + items;
  pre.members = reinterpret_cast<int*>(pre.refs + (size_t)s.B * s.Hkv);
  MergeParams m = {pre.d, pre.d, pre.refs, pre.members};
  m.own.B = s.B;

  if (joint) {
    pre.own = {(uint64_t)(uintptr_t)a.own.table, a.own.table_stride * 4, a.own.width - 1, s.C, a.own.cache_lens};
    m.own.ng = (m.own.G * s.S + gp.rows - 1) / gp.rows;
    const hipError_t e = launch_paged_runs<D, PagedMode::Joint>(gp, pre, st);
    if (e != hipSuccess) return e;
    if (waves == 1) launch_merge_as<D, false, false, true>(m, st);
    else launch_merge_as<D, true, true, true>(m, st);
    return hipGetLastError();
  }

  const DecodeGroups g = decode_groups(s);
  const PagedParams own = paged_params(s, g, a.own, ws);
  pre.Sn = 0;
  hipError_t e = launch_prefix<D>(pre, st);
  if (e != hipSuccess) return e;
  e = launch_paged_runs<D, PagedMode::Own>(g, own, st);
  if (e != hipSuccess) return e;
  m.own = own.d;
  if (g.waves > 1) launch_merge_as<D, true, true>(m, st);
  else launch_merge_as<D, false, true>(m, st);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_decode(const SharedShape& s, const SharedArgs& a, void* ws, hipStream_t st) {
  return s.s.D == 128 ? launch_shared_d<128>(s, a, ws, st) : launch_shared_d<64>(s, a, ws, st);
}

}  // namespace bd
