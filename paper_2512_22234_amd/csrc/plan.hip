// Page tables and slot maps for the next tokens of a batch of sequences, from
// their lengths on the device, for gfx950: the host neither knows the lengths
// nor waits for them.
//
// Sequence b holds len_b tokens in the pages of row b of the table (2^log_size
// tokens each) and gets new_b more; with cap the row's room,
//   end_b  = min(len_b + new_b, cap)
//   need_b = ceil(end_b / P) - ceil(len_b / P)    pages, taken from the free list
//            in sequence order from its head on: page j of the row, j from
//            ceil(len_b / P), is free[head + sum_{b' < b} need_b' + j - ceil(len_b / P)]
//   slot   = page * P + position mod P            of each new token.
//
// The work is a prefix sum over the sequences and a few integer operations a
// token: bound by launch and load latency.  One launch: every workgroup scans
// all lengths (8 bytes a sequence, from L2) and then takes a contiguous run of
// tokens, the first one the state; a token finds its sequence by a search of the scan.
// The token that starts a page writes the page's table entry, the others read the
// same entry of the free list, so no workgroup waits for another.  The kernel takes 3.7 us for
// 64 sequences of 4 tokens and 6.1 for 82,000 tokens of 700 sequences; a call 30 to
// 33 us for 8192 sequences and 300 to 390 for 65,536, whose lengths a thread walks
// 256 at a time.
#include "device.hpp"
#include "kernels.hpp"

namespace bd {
namespace {

constexpr int PLAN_NT = 256;

// Lengths of a sequence within the table's room and the pages it needs.
struct PlanSeq {
  int len, fresh, end, p0, need;
};
__device__ inline PlanSeq plan_seq(const PlanArgs& a, int b) {
  const int cap = a.width << a.log_size, up = (1 << a.log_size) - 1;
  PlanSeq q;
  q.len = imin(imax(a.lens[b], 0), cap);
  q.fresh = imax(a.fresh[b], 0);
  if (a.S > 0) q.fresh = imin(q.fresh, a.S);
  q.end = q.len + imin(q.fresh, cap - q.len);
  q.p0 = (q.len + up) >> a.log_size;
  q.need = ((q.end + up) >> a.log_size) - q.p0;
  return q;
}
// Id of entry `at` of the free list, or -1 if there is none.
__device__ inline int plan_free(const PlanArgs& a, long long at) {
  if (at >= a.n_free) return -1;
  const int id = a.free_pages[at];
  return id >= 0 && id < a.num_pages ? id : -1;
}
// New tokens of a sequence that have a row in the results; t: tokens before it.
__device__ inline int plan_seen(const PlanArgs& a, const PlanSeq& q, long long t) {
  if (a.S > 0 || t + q.fresh <= a.T) return q.fresh;
  return t < a.T ? (int)(a.T - t) : 0;
}
// The last thread whose sequences start at or before token (or page) x, by the sums before each thread.
__device__ inline int plan_find(const long long* before, long long x) {
  int c = 0;
#pragma unroll
  for (int step = PLAN_NT / 2; step > 0; step >>= 1)
    if (before[c + step] <= x) c += step;
  return c;
}

__global__ __launch_bounds__(PLAN_NT) void plan_kernel(PlanArgs a) {
  // tokens and pages of the sequences before those of thread t
  __shared__ long long tok0[PLAN_NT + 1];
  __shared__ long long need0[PLAN_NT + 1];
  __shared__ long long wtok[PLAN_NT / 64];
  __shared__ long long wneed[PLAN_NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cpt = cdiv(a.B, PLAN_NT);  // consecutive sequences of a thread
  const int c0 = imin(a.B, tid * cpt), c1 = imin(a.B, c0 + cpt);
  long long tok = 0, need = 0;
  for (int b = c0; b < c1; ++b) {
    const PlanSeq q = plan_seq(a, b);
    tok += q.fresh;
    need += q.need;
  }
  long long itok = tok, ineed = need;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long u = __shfl_up(itok, o, 64), v = __shfl_up(ineed, o, 64);
    if (lane >= o) {
      itok += u;
      ineed += v;
    }
  }
  if (lane == 63) {
    wtok[wave] = itok;
    wneed[wave] = ineed;
  }
  __syncthreads();
  for (int v = 0; v < wave; ++v) {
    itok += wtok[v];
    ineed += wneed[v];
  }
  tok0[tid + 1] = itok;
  need0[tid + 1] = ineed;
  if (tid == 0) {
    tok0[0] = 0;
    need0[0] = 0;
  }
  __syncthreads();
  const long long total = tok0[PLAN_NT];
  const long long head = imin(imax(a.free_head[0], 0), a.n_free);
  const int P = 1 << a.log_size, cap = a.width << a.log_size;

  // The first workgroup: the new head of the free list, and the tokens that have no page.
  const int workers = (int)gridDim.x - 1, worker = (int)blockIdx.x - 1;
  if (worker < 0) {
    // (packed tokens past T are lost once, wherever else they would be)
    long long lost = 0;
    long long first = need0[tid], t = tok0[tid];
    for (int b = c0; b < c1; ++b) {
      const PlanSeq q = plan_seq(a, b);
      const int seen = plan_seen(a, q, t);
      const int end = q.len + imin(seen, cap - q.len);  // of the tokens below T
      lost += q.fresh - (end - q.len);
      const long long left = a.n_free - head - first;  // entries of the free list for this sequence
      const int given = left <= 0 ? 0 : (int)(left < q.need ? left : q.need);
      if (given < q.need) lost += imax(end - imax(q.len, (q.p0 + given) << a.log_size), 0);
      // tokens behind the cached ones in a page that is none
      const int tail = imin(end, q.p0 << a.log_size) - q.len;
      if (tail > 0) {
        const int id = a.table[b * a.table_stride + (q.len >> a.log_size)];
        if (id < 0 || id >= a.num_pages) lost += tail;
      }
      t += q.fresh;
      first += q.need;
    }
    // tokens in pages whose entry of the list is no page: every entry taken is looked at, 32 loads at a time (four prompts
    // of 62,500 tokens in pages of 16: 5.9 us a call, eight at a time 8.2); a sequence is sought for the bad ones alone
    const long long pages = need0[PLAN_NT];
    const long long given = pages < a.n_free - head ? pages : a.n_free - head;
    for (long long u0 = tid; u0 < given; u0 += 32 * PLAN_NT) {
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const long long u = u0 + e * PLAN_NT;
        bad |= (unsigned)a.free_pages[head + (u < given ? u : given - 1)] >= (unsigned)a.num_pages;
      }
      if (!bad) continue;
      const long long end_u = given < u0 + 32 * PLAN_NT ? given : u0 + 32 * PLAN_NT;
      for (long long u = u0; u < end_u; u += PLAN_NT) {
        if (plan_free(a, head + u) >= 0) continue;
        const int c = plan_find(need0, u);
        int b = c * cpt;
        long long at = u - need0[c], t = tok0[c];  // page, and token, among those of the sequences of thread c
        PlanSeq q = plan_seq(a, b);
        while (at >= q.need) {  // (ends: thread c's sequences need need0[c + 1] - need0[c] > u - need0[c] pages)
          at -= q.need;
          t += q.fresh;
          q = plan_seq(a, ++b);
        }
        const int begin = (q.p0 + (int)at) << a.log_size, end = q.len + imin(plan_seen(a, q, t), cap - q.len);
        lost += imax(imin(end - begin, P), 0);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) lost += __shfl_xor(lost, o);
    if (lane == 0) wtok[wave] = lost;
    __syncthreads();
    if (tid == 0) {
      long long sum = 0;
      for (int v = 0; v < PLAN_NT / 64; ++v) sum += wtok[v];
      const long long used = head + pages;
      a.state[0] = (int)(used < a.n_free ? used : a.n_free);
      a.state[1] = (int)(sum < INT32_MAX ? sum : INT32_MAX);
    }
    return;
  }

  // the sequences' own outputs: thread t's are written by worker t mod workers
  if (tid % workers == worker) {
    long long t = tok0[tid];
    for (int b = c0; b < c1; ++b) {
      const PlanSeq q = plan_seq(a, b);
      a.lens_out[b] = q.end;
      a.cu[b] = (int)(t < INT32_MAX ? t : INT32_MAX);
      t += q.fresh;
    }
    if (c0 < c1 && c1 == a.B) a.cu[a.B] = (int)(t < INT32_MAX ? t : INT32_MAX);
  }

  // tokens: a contiguous run for each workgroup
  const int t0 = (int)((long long)a.T * worker / workers), t1 = (int)((long long)a.T * (worker + 1) / workers);
  for (int t = t0 + tid; t < t1; t += PLAN_NT) {
    int b, c, i;  // token i of sequence b
    PlanSeq q;
    long long first;  // pages of the sequences before b
    bool real = true;
    if (a.S > 0) {
      b = t / a.S;
      i = t - b * a.S;
      c = b / cpt;
      first = need0[c];
      for (int u = c * cpt; u < b; ++u) first += plan_seq(a, u).need;
      q = plan_seq(a, b);
      real = i < q.fresh;
    } else if (t < total) {
      c = plan_find(tok0, t);
      i = t - (int)tok0[c];
      first = need0[c];
      b = c * cpt;
      q = plan_seq(a, b);
      while (i >= q.fresh) {  // (ends: the sequences of thread c hold tok0[c + 1] - tok0[c] > i tokens)
        i -= q.fresh;
        first += q.need;
        q = plan_seq(a, ++b);
      }
    } else {
      real = false;
    }
    int slot = -1, position = 0;
    if (real) {
      position = q.len + i;
      if (position < cap) {
        const int j = position >> a.log_size;
        int id;
        if (j >= q.p0) {
          id = plan_free(a, head + first + (j - q.p0));
          if ((position & (P - 1)) == 0) a.table[b * a.table_stride + j] = id;
        } else {
          id = a.table[b * a.table_stride + j];
          if (id >= a.num_pages) id = -1;
        }
        if (id >= 0) slot = (id << a.log_size) + (position & (P - 1));
      }
    }
    a.slots[t] = slot;
    a.positions[t] = position;
  }

  // Packed tokens past T: the pages that they begin are taken from the list like the others, and are entered too (a row
  // may hold ids of an earlier sequence there).  A sequence at a time for each workgroup.
  if (a.S == 0 && total > a.T) {
    for (int b = worker; b < a.B; b += workers) {
      const int c = b / cpt;
      long long t = tok0[c], first = need0[c];
      for (int u = c * cpt; u < b; ++u) {
        const PlanSeq q = plan_seq(a, u);
        t += q.fresh;
        first += q.need;
      }
      const PlanSeq q = plan_seq(a, b);
      // entered above: pages that begin with one of the tokens below T
      const int seen = plan_seen(a, q, t), begun = (q.len + imin(seen, cap - q.len) + P - 1) >> a.log_size;
      for (int j = imax(begun, q.p0) + tid; j < q.p0 + q.need; j += PLAN_NT)
        a.table[b * a.table_stride + j] = plan_free(a, head + first + (j - q.p0));
    }
  }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t st) {
  // a workgroup for each 256 tokens (one a thread) and 256 sequences, and one for the state: 82,000 tokens of 700
  // sequences 5.9 us a call, with 1024 tokens a workgroup 8.5
  const int work = imax(a.T / PLAN_NT, a.B / PLAN_NT);
  hipLaunchKernelGGL(plan_kernel, dim3(imin(imax(work, 1), 2048) + 1), dim3(PLAN_NT), 0, st, a);
  return hipGetLastError();
}

}  // namespace bd
