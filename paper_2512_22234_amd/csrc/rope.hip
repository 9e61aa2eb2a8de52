// Norms of queries and keys for each head with the rotary embedding, in one
// pass from the projections' layout into the attention's, for gfx950.
//
// For a head row x of D values at position p, with the norm's weight w:
//   r = (mean(x^2) + eps)^(-1/2),   n = x r,   y = w n
//   out1 = y1 c - y2 s,   out2 = y2 c + y1 s        (halves 1, 2 of the head)
// where c, s are row p of the table (cos and sin of p f_j).  Values are only
// laid out.  The backward, for gradients d of the outputs, recomputes r from x:
//   g1 = d1 c + d2 s,   g2 = d2 c - d1 s            (the rotation's inverse)
//   dw = sum over rows of g n,   h = g w,   dx = r (h - n mean(h n)).
// Float32 throughout; each result is rounded once, when it is stored.
//
// Projections are token-major (any batch, token and head strides), outputs
// head-major [B][H][N][D]: the pass is the transposition that the attention
// needs anyway, and is bound by HBM.  A lane holds the same 8 values of both
// halves of a row (16-byte accesses, pairs of the rotation in one lane), D / 16
// lanes a row; a workgroup takes 256 / (D / 16) consecutive tokens, whose cos
// and sin stay in registers, and a run of heads of one kind (q, k or v).
// Measured: 16384 tokens of 32/8 heads of 128, forward: 76 us, 5.4 TB/s (a copy
// of 1 GiB: 5.1).
#include "device.hpp"
#include "kernels.hpp"

namespace bd {
namespace {

constexpr int ROPE_NT = 256;
// Lanes of a row, and rows (tokens) of a workgroup.
template <int D>
constexpr int ROPE_LPR = D / 16;
template <int D>
constexpr int ROPE_RPB = ROPE_NT / ROPE_LPR<D>;

// 16 bytes from or to memory; NT: nontemporal.
template <bool NT>
__device__ inline u32x4 ld16(const void* p) {
  return NT ? __builtin_nontemporal_load(static_cast<const u32x4*>(p)) : *static_cast<const u32x4*>(p);
}
template <bool NT>
__device__ inline void st16(void* p, const u32x4& v) {
  if constexpr (NT) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = v;
}
// 8 consecutive values as float32.
template <bool NT = false>
__device__ inline void ld8(const bf16* p, float* x) {
  const bf16x8 v = __builtin_bit_cast(bf16x8, ld16<NT>(p));
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
template <bool NT = false>
__device__ inline void ld8(const float* p, float* x) {
  const f32x4 a = __builtin_bit_cast(f32x4, ld16<NT>(p)), b = __builtin_bit_cast(f32x4, ld16<NT>(p + 4));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[e + 4] = b[e];
  }
}
template <bool NT = false>
__device__ inline void st8(bf16* p, const float* x) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16)x[e];
  st16<NT>(p, __builtin_bit_cast(u32x4, v));
}
template <bool NT = false>
__device__ inline void st8(float* p, const float* x) {
  st16<NT>(p, __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}));
  st16<NT>(p + 4, __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}));
}

// Copies a lane's values of a row, 8 in either half, bit for bit.
template <int D, bool NTL, bool NTS, typename T>
__device__ inline void copy_row(const T* from, T* to, bool store) {
  constexpr int PER = 16 / sizeof(T), N = 8 / PER;
  u32x4 v[2 * N];
#pragma unroll
  for (int e = 0; e < 2 * N; ++e) v[e] = ld16<NTL>(from + e / N * (D / 2) + e % N * PER);
  if (store) {
#pragma unroll
    for (int e = 0; e < 2 * N; ++e) st16<NTS>(to + e / N * (D / 2) + e % N * PER, v[e]);
  }
}

// Sum over the 4 or 8 consecutive lanes of a row.
template <int LPR>
__device__ inline float row_sum(float x) {
  x += __shfl_xor(x, 1);
  x += __shfl_xor(x, 2);
  if constexpr (LPR == 8) x += __shfl_xor(x, 4);
  return x;
}

// What a workgroup works on: heads [h0, h1) of a kind (0: q, 1: k, 2: v).  The
// grid's second index counts runs of hpb heads, those of q first, then k, then v.
struct HeadRun {
  int kind, h0, h1, part;  // part: the run among those of its kind
};
__device__ inline HeadRun head_run(const RopeShape& s, int y) {
  const int cq = cdiv(s.Hq, s.hpb), ck = cdiv(s.Hkv, s.hpb);
  HeadRun r;
  r.kind = y < cq ? 0 : y < cq + ck ? 1 : 2;
  r.part = y - (r.kind == 0 ? 0 : r.kind == 1 ? cq : cq + ck);
  r.h0 = r.part * s.hpb;
  r.h1 = imin(r.h0 + s.hpb, r.kind == 0 ? s.Hq : s.Hkv);
  return r;
}

// The block of tokens that a workgroup takes.  Workgroups go to the eight dies in
// turn; the blocks of a run of heads start at an offset with which all runs of one
// block (but for the last seven) are on one die and read its rows of the table into
// one L2.  32/8 heads of 128, one sequence, without / with, us: into pages, 1100
// tokens 7.5 / 7.1, 2052 11.5 / 10.6, 8194 40.6 / 41.2, 9001 45.0 / 43.9; forward and
// backward, 1500 23.4 / 22.9, 2200 32.5 / 31.5, 4356 56.9 / 55.3, 8200 96.3 / 96.5.
// (Rounding the grid up to whole rounds of the dies instead: 8200 98.2.  Where the
// number of blocks is a multiple of 8 nothing changes; runs put on different dies
// there cost 1 to 10%.)
__device__ inline int token_block() {
  const unsigned n = gridDim.x;
  if (n < 8) return (int)blockIdx.x;
  const unsigned x = blockIdx.x + blockIdx.y * n % 8;
  return (int)(x < n ? x : x - n);
}

// A lane's token: row t of the B*N (the last one again past the end, not stored).
struct Token {
  bool valid;
  int t, b, n;
};
template <int D>
__device__ inline Token lane_token(const RopeShape& s, int x) {
  const unsigned rows = (unsigned)s.B * (unsigned)s.N;
  const unsigned t = (unsigned)x * ROPE_RPB<D> + threadIdx.x / ROPE_LPR<D>;
  Token k;
  k.valid = t < rows;
  k.t = (int)(k.valid ? t : rows - 1);
  k.b = (int)((unsigned)k.t / (unsigned)s.N);
  k.n = k.t - k.b * s.N;
  return k;
}
// cos and sin of this lane's 8 pairs at its token's position (clamped to the table).
template <int D>
__device__ inline void lane_angles(const RopeShape& s, const Token& k, int i, float* c, float* sn) {
  const int p = imin(imax(s.pos[(size_t)k.b * s.pos_stride + k.n], 0), s.n_rope - 1);
  const float* row = s.rope + (size_t)p * D + 8 * i;
  ld8(row, c);
  ld8(row + D / 2, sn);
}

// NT: nontemporal loads (1), and stores (2).
template <typename T, typename W, int D, bool PAGED, int NT>
__global__ __launch_bounds__(ROPE_NT) void rope_fwd_kernel(RopeShape s, RopeFwdArgs a) {
  constexpr int LPR = ROPE_LPR<D>;
  const int i = threadIdx.x % LPR;
  const HeadRun run = head_run(s, blockIdx.y);
  const Token k = lane_token<D>(s, token_block());
  const int H = run.kind == 0 ? s.Hq : s.Hkv;
  const HeadRows in = run.kind == 0 ? a.sq : run.kind == 1 ? a.sk : a.sv;
  const T* src = static_cast<const T*>(run.kind == 0 ? a.q : run.kind == 1 ? a.k : a.v) + k.b * in.sb + k.n * in.sn + 8 * i;
  // where the rows go: [B][H][N][D], or the token's slot of the pages
  T* dst;
  int64_t dst_h;
  bool store = k.valid;
  if (PAGED && run.kind != 0) {
    const int slot = a.slots[k.t];
    const int page = slot >> s.pages.log_size;
    store = store && slot >= 0 && page < s.pages.num;
    dst = static_cast<T*>(run.kind == 1 ? a.ko : a.vo) +
          (store ? page * s.pages.sp + (slot & ((1 << s.pages.log_size) - 1)) * s.pages.sr : 0) + 8 * i;
    dst_h = s.pages.sh;
  } else {
    dst = static_cast<T*>(run.kind == 0 ? a.qo : run.kind == 1 ? a.ko : a.vo) + ((size_t)k.b * H * s.N + k.n) * D + 8 * i;
    dst_h = (int64_t)s.N * D;
  }
  if (run.kind == 2) {
    for (int h = run.h0; h < run.h1; ++h) copy_row<D, (NT > 0), (NT > 1)>(src + h * in.sh, dst + h * dst_h, store);
    return;
  }
  float c[8], sn[8], w1[8], w2[8];
  lane_angles<D>(s, k, i, c, sn);
  const W* w = static_cast<const W*>(run.kind == 0 ? a.wq : a.wk) + 8 * i;
  ld8(w, w1);
  ld8(w + D / 2, w2);
  for (int h = run.h0; h < run.h1; ++h) {
    float x1[8], x2[8];
    ld8<(NT > 0)>(src + h * in.sh, x1);
    ld8<(NT > 0)>(src + h * in.sh + D / 2, x2);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x1[e] * x1[e] + x2[e] * x2[e];
    const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + s.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y1 = x1[e] * r * w1[e], y2 = x2[e] * r * w2[e];
      x1[e] = y1 * c[e] - y2 * sn[e];
      x2[e] = y2 * c[e] + y1 * sn[e];
    }
    if (store) {
      st8<(NT > 1)>(dst + h * dst_h, x1);
      st8<(NT > 1)>(dst + h * dst_h + D / 2, x2);
    }
  }
}

// The gradients of the projections, and of each workgroup's rows the sums g n
// per weight (`part`: [workgroup of a kind][D], those of q first).
template <typename T, typename W, int D, bool NT>
__global__ __launch_bounds__(ROPE_NT) void rope_bwd_kernel(RopeShape s, RopeBwdArgs a) {
  constexpr int LPR = ROPE_LPR<D>;
  __shared__ float sums[ROPE_NT / 64][D];
  const int i = threadIdx.x % LPR;
  const HeadRun run = head_run(s, blockIdx.y);
  const int x = token_block();
  const Token k = lane_token<D>(s, x);
  const int H = run.kind == 0 ? s.Hq : s.Hkv;
  const HeadRows gs = run.kind == 0 ? a.gq : run.kind == 1 ? a.gk : a.gv;
  const T* dy = static_cast<const T*>(run.kind == 0 ? a.dqo : run.kind == 1 ? a.dko : a.dvo) +
                ((size_t)k.b * H * s.N + k.n) * D + 8 * i;
  const int64_t dy_h = (int64_t)s.N * D;
  T* dst = static_cast<T*>(run.kind == 0 ? a.dq : run.kind == 1 ? a.dk : a.dv) + k.b * gs.sb + k.n * gs.sn + 8 * i;
  if (run.kind == 2) {
    for (int h = run.h0; h < run.h1; ++h) copy_row<D, NT, false>(dy + h * dy_h, dst + h * gs.sh, k.valid);
    return;
  }
  const HeadRows in = run.kind == 0 ? a.sq : a.sk;
  const T* src = static_cast<const T*>(run.kind == 0 ? a.q : a.k) + k.b * in.sb + k.n * in.sn + 8 * i;
  float c[8], sn[8], w1[8], w2[8], a1[8], a2[8];
  lane_angles<D>(s, k, i, c, sn);
  const W* w = static_cast<const W*>(run.kind == 0 ? a.wq : a.wk) + 8 * i;
  ld8(w, w1);
  ld8(w + D / 2, w2);
#pragma unroll
  for (int e = 0; e < 8; ++e) a1[e] = a2[e] = 0.f;
  for (int h = run.h0; h < run.h1; ++h) {
    float x1[8], x2[8], d1[8], d2[8];
    ld8<NT>(src + h * in.sh, x1);
    ld8<NT>(src + h * in.sh + D / 2, x2);
    ld8<NT>(dy + h * dy_h, d1);
    ld8<NT>(dy + h * dy_h + D / 2, d2);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x1[e] * x1[e] + x2[e] * x2[e];
    const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + s.eps);
    float hn = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g1 = d1[e] * c[e] + d2[e] * sn[e], g2 = d2[e] * c[e] - d1[e] * sn[e];
      x1[e] *= r;
      x2[e] *= r;
      if (k.valid) {
        a1[e] += g1 * x1[e];
        a2[e] += g2 * x2[e];
      }
      d1[e] = g1 * w1[e];
      d2[e] = g2 * w2[e];
      hn += d1[e] * x1[e] + d2[e] * x2[e];
    }
    const float m = row_sum<LPR>(hn) * (1.f / D);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      d1[e] = r * (d1[e] - x1[e] * m);
      d2[e] = r * (d2[e] - x2[e] * m);
    }
    if (k.valid) {
      st8(dst + h * gs.sh, d1);
      st8(dst + h * gs.sh + D / 2, d2);
    }
  }
  // sums over the workgroup's rows, in a fixed order
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
      a1[e] += __shfl_xor(a1[e], o);
      a2[e] += __shfl_xor(a2[e], o);
    }
  if (lane < LPR) {
    st8(&sums[wave][8 * i], a1);
    st8(&sums[wave][8 * i + D / 2], a2);
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < ROPE_NT / 64; ++u) v += sums[u][threadIdx.x];
    const int cq = cdiv(s.Hq, s.hpb), ck = cdiv(s.Hkv, s.hpb);
    const size_t row = run.kind == 0 ? (size_t)x * cq + run.part
                                     : (size_t)gridDim.x * cq + (size_t)x * ck + run.part;
    a.part[row * D + threadIdx.x] = v;
  }
}

// dw: column sums of the rows of `part` of each kind (blockIdx.y: 0 q, 1 k), 32
// columns a workgroup, in a fixed order.
template <typename W>
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* part, int nq, int nk, int D, W* dwq, W* dwk) {
  __shared__ float sums[32][33];
  const int col = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int n = blockIdx.y == 0 ? nq : nk;
  const float* p = part + (size_t)(blockIdx.y == 0 ? 0 : nq) * D + blockIdx.x * 32 + col;
  float v = 0.f;
#pragma unroll 8
  for (int u = r; u < n; u += 32) v += p[(size_t)u * D];
  sums[r][col] = v;
  __syncthreads();
  if (r == 0) {
    v = 0.f;
#pragma unroll
    for (int u = 0; u < 32; ++u) v += sums[u][col];
    (blockIdx.y == 0 ? dwq : dwk)[blockIdx.x * 32 + col] = (W)v;
  }
}

// Row p of the table: cos(p f_j), then sin(p f_j), from angles in float64 (a
// float32 angle is off by up to p 2^-24 rad).
__global__ __launch_bounds__(256) void rope_table_kernel(const double* inv_freq, int n, int half, float* table) {
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (size_t)n * half) return;
  const size_t p = at / half;
  const int j = (int)(at - p * half);
  double sn, c;
  sincos((double)p * inv_freq[j], &sn, &c);
  table[p * 2 * half + j] = (float)c;
  table[p * 2 * half + half + j] = (float)sn;
}

// Heads a workgroup takes: 1, 2, 4 or 8, as many as leave 768 workgroups (three
// a CU), so that its tokens' cos and sin are read once for all of them.  Forward of
// 16384 tokens, 32/8 heads of 128, one head each 95 us, two 87, eight 82 (before the
// nontemporal accesses below); forward and backward of 2048 tokens, one 30.0, four
// 26.5; 12/4 heads, 4096 tokens, one 25.9, two 22.3.  Powers of two divide most head
// counts: 4096 tokens of 32/8 heads, runs of six 52.5 us, of eight 48.2.
RopeShape with_runs(const RopeShape& shape) {
  RopeShape s = shape;
  const long long work = (long long)rope_token_blocks(s) * (s.Hq + 2 * s.Hkv);
  s.hpb = 1;
  while (s.hpb < 8 && work >= 768 * 2 * s.hpb) s.hpb *= 2;
  return s;
}
dim3 rope_grid(const RopeShape& s) {
  return dim3((unsigned)rope_token_blocks(s), (unsigned)(cdiv(s.Hq, s.hpb) + 2 * cdiv(s.Hkv, s.hpb)));
}

// Bytes of a call's rows, `heads` of D values read or written per token: beyond
// 64 MiB their loads are nontemporal, and in the forward beyond 128 MiB (half the
// last-level cache) the stores too.  Measured between a kernel that writes the
// call's inputs and one that reads its results, on a GiB of arrays in turn, as the
// layers of a model have them (32/8 heads of 128; us for the three kernels with
// neither, the loads, both):
//   tokens     forward                backward
//     1024      15.1  15.4  15.2      21.9  21.9  22.9
//     2048      24.1  24.1  25.4      33.0  32.7  35.2    (48 and 68 MiB)
//     4096      48.0  43.6  45.8      61.2  54.9  59.3
//     8192     107.7 102.8  89.6     124.9 115.3 117.7
//    16384     207.6 209.8 200.4     251.5 238.2 236.9
// and the forward alone, us: 2048 tokens 10.1, 12.5, 11.6; 4096 20.7, 20.0, 20.2;
// 8192 43.2, 38.3, 38.9; 16384 83.3, 82.2, 77.0.
constexpr size_t ROPE_NT_LOADS = (size_t)64 << 20, ROPE_NT_STORES = (size_t)128 << 20;
size_t rope_bytes(const RopeShape& s, int heads) { return (size_t)s.B * s.N * heads * s.D * (s.f32 ? 4 : 2); }

template <typename T, typename W, int D>
hipError_t launch_rope_fwd_t(const RopeShape& s, const RopeFwdArgs& a, bool paged, hipStream_t st) {
  const auto kernel = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (paged) {
      if constexpr (std::is_same_v<T, bf16>)
        hipLaunchKernelGGL((rope_fwd_kernel<T, W, D, true, NT>), rope_grid(s), dim3(ROPE_NT), 0, st, s, a);
    } else {
      hipLaunchKernelGGL((rope_fwd_kernel<T, W, D, false, NT>), rope_grid(s), dim3(ROPE_NT), 0, st, s, a);
    }
  };
  const size_t bytes = rope_bytes(s, 2 * (s.Hq + 2 * s.Hkv));
  if (bytes > ROPE_NT_STORES) kernel(std::integral_constant<int, 2>());
  else if (bytes > ROPE_NT_LOADS) kernel(std::integral_constant<int, 1>());
  else kernel(std::integral_constant<int, 0>());
  return hipGetLastError();
}
template <typename T, typename W, int D>
hipError_t launch_rope_bwd_t(const RopeShape& s, const RopeBwdArgs& a, hipStream_t st) {
  int nq = 0, nk = 0;
  if (s.B > 0 && s.N > 0) {
    if (rope_bytes(s, 3 * s.Hq + 5 * s.Hkv) > ROPE_NT_LOADS)
      hipLaunchKernelGGL((rope_bwd_kernel<T, W, D, true>), rope_grid(s), dim3(ROPE_NT), 0, st, s, a);
    else
      hipLaunchKernelGGL((rope_bwd_kernel<T, W, D, false>), rope_grid(s), dim3(ROPE_NT), 0, st, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    nq = rope_token_blocks(s) * cdiv(s.Hq, s.hpb);
    nk = rope_token_blocks(s) * cdiv(s.Hkv, s.hpb);
  }
  hipLaunchKernelGGL((rope_dw_kernel<W>), dim3(D / 32, 2), dim3(1024), 0, st, a.part, nq, nk, D,
                     static_cast<W*>(a.dwq), static_cast<W*>(a.dwk));
  return hipGetLastError();
}

// f(T, W, D) for the element type, the weights' type and the head size of s.
template <typename F>
hipError_t rope_dispatch(const RopeShape& s, F f) {
  auto with_d = [&](auto t, auto w) {
    return s.D == 128 ? f(t, w, std::integral_constant<int, 128>()) : f(t, w, std::integral_constant<int, 64>());
  };
  if (s.f32) return with_d(float(), float());
  if (s.w32) return with_d(bf16(), float());
  return with_d(bf16(), bf16());
}

}  // namespace

size_t rope_bwd_workspace_bytes(const RopeShape& shape) {
  const RopeShape s = with_runs(shape);
  return (size_t)rope_token_blocks(s) * (cdiv(s.Hq, s.hpb) + cdiv(s.Hkv, s.hpb)) * s.D * 4;
}

hipError_t launch_rope_fwd(const RopeShape& shape, const RopeFwdArgs& a, bool paged, hipStream_t st) {
  const RopeShape s = with_runs(shape);
  return rope_dispatch(s, [&](auto t, auto w, auto d) {
    return launch_rope_fwd_t<decltype(t), decltype(w), decltype(d)::value>(s, a, paged, st);
  });
}

hipError_t launch_rope_bwd(const RopeShape& shape, const RopeBwdArgs& a, hipStream_t st) {
  const RopeShape s = with_runs(shape);
  return rope_dispatch(s, [&](auto t, auto w, auto d) {
    return launch_rope_bwd_t<decltype(t), decltype(w), decltype(d)::value>(s, a, st);
  });
}

hipError_t launch_rope_table(const double* inv_freq, int n, int D, float* table, hipStream_t st) {
  const size_t work = (size_t)n * (D / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((work + 255) / 256)), dim3(256), 0, st, inv_freq, n, D / 2, table);
  return hipGetLastError();
}

}  // namespace bd
