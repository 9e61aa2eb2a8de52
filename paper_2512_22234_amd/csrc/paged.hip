// Decoding over a paged KV cache for gfx950: the S queries of each sequence
// attend to the first cache_lens[b] keys of its pages (row b of the page table)
// and, if given, to the block's own S keys.  A page outside the pool holds no
// keys; a row that sees no key at all gets O = 0 and LSE = -inf.
//
// For each query row, over the keys j that it sees:
//   s_j = scale q . k_j,   M = max_j s_j,   l = sum_j exp(s_j - M),
//   O = sum_j exp(s_j - M) v_j / l,   LSE = M + log l.
// Every cached K and V row is read once and serves all G*S query rows of its KV
// head: 4 D bytes of HBM a key for 4 D G S flops, so the work is bound by HBM.
//
// The work is shared out as over a dense cache (decode.hip): the KT-key tiles of
// all (sequence, KV head, row group) items end to end, in equal contiguous runs
// over teams of TW waves, one per 32 query rows; a run that holds part of an
// item leaves unnormalised sums, which a second kernel joins.  What differs:
//   - A tile's rows lie in pages: each piece of 16 rows (a page holds a multiple
//     of 16) is copied by one wave through a buffer descriptor of its own, which
//     ends with the last valid row.  So pages cost scalar work only, whatever
//     their size and strides.  The page ids of the next tile are read (scalar
//     loads) while the current one is waited for.
//   - Items have at least one tile, empty where there is no key, so that their
//     rows are written.  Tiles without a key are not computed; 16-row pieces
//     without one are masked.
//
// Roundings: O to bfloat16, relative error against float64 1.7e-3.  P enters the
// product with V as two bfloat16 parts, the second being what the rounding of the
// first left: 16 bits of P in all, so that O is off by its own rounding alone.  In one
// part (2.3e-3, values that cancel by several of their steps) a call takes 1% less for
// 64 sequences of 512 to 8192 tokens, 3% for one of 1500, 5 to 7% for 64 rows per KV head
// (32 sequences of 128 to 2048, D = 128: 31.0 us, two parts 32.4; D = 64: 22.2, 23.7) and
// 10% for 128 rows (24 sequences: 62.9, 69.5).  Scores, maxima, sums and O's sums are
// float32.
//
// Measured (32/8 heads of 128): 64 sequences of 512 to 8192 tokens (816 MB), one
// token each, 133 to 143 us whatever the pages (16 to 128 rows; heads or tokens
// outermost), 5.7 to 6.1 TB/s; blocks of 4, 139 to 141 us (over a dense cache 143);
// 24 sequences of 200 to 4096 (184 MB), blocks of 32, 66 to 71 us (dense, with P in one
// part, 63 to 66): 7 are the merge of 27 MB of partial results, and without any product the
// call takes 56, one team of four waves a CU waiting for each tile in turn.
#include "paged.hpp"

namespace bd {

hipError_t launch_paged_decode(const DecodeShape& s, const PagedArgs& a, void* ws, hipStream_t st) {
  return s.D == 128 ? launch_paged_decode_d<128, PagedMode::Plain>(s, a, 0, ws, st)
                    : launch_paged_decode_d<64, PagedMode::Plain>(s, a, 0, ws, st);
}

}  // namespace bd
