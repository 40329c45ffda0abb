// How a gradient call is cut up (host code): the key ranges of the dQ pass, the
// query ranges of the dK/dV pass, and the workspace that follows from them.  The
// kernels (attn_bwd.hip) take the cut through BwdArgs.
#pragma once

#include <math.h>

#include <algorithm>

#include "launch.h"

namespace sparstar {

struct BwdPlan {
  int dq_ranges, dkv_ranges;
  int slots;    // partial results of pieces of key blocks (0: blocks are not cut)
  int extra;    // pieces that there may be beyond one per block
  bool rounds;  // the dK/dV pass has more work-groups than the chip holds
  // byte offsets of the workspace's regions, and its size
  size_t stats, bits, count, pieces, listed, part, part_kv, part_piece, total;
};

constexpr int kBwdMaxRanges = 16;

// Ranges of one pass: `groups` work-groups of `waves` waves that each walk `tiles` tiles at
// most.  A SIMD works off its waves at the rate of its matrix core whether it holds one or
// two, so the pass takes as long as the SIMDs with the most of them: ceil(x) / x of the even
// share, x waves per SIMD.  More ranges even that out (24 dense heads of 2,880 rows: 2.2
// work-groups of 4 waves per CU; dQ takes 3.4 ms in 2 ranges and 3.0 in 4) and cost their
// partial results, `bytes` written and read again each, and a launch; both against a time of
// the pass estimated from its operations.  A gain below 3 % is not worth the memory.  The
// estimate's rates (1.1 PFLOP/s, 4.5 TB/s, 4 us) are round figures of large calls, not fitted to a
// sweep.  Lists are taken to hold a quarter of the keys: 6 heads of 691 x 40,407, of another
// density, take 181 us where another cut takes 138; but cuts by kv_stride's density, tried on 125
// drawn gradients, made 10 of them 5 to 24% faster, as many 3 to 40% slower, and all 0.3% faster.
inline int bwd_ranges(int64_t groups, int waves, int64_t tiles, double flops, double bytes) {
  const double pass_us = flops / 1.1e9;
  int best = 1;
  double least = 0.0;
  for (int r = 1; r <= kBwdMaxRanges && (r == 1 || tiles >= 16 * r); r *= 2) {
    const double x = double(groups) * r * waves / 1024.0;
    const double t = pass_us * ceil(x) / x + (r > 1 ? 4.0 + 2.0 * r * bytes / 4.5e6 : 0.0);
    if (r == 1 || t < 0.97 * least) {
      least = t;
      best = r;
    }
  }
  return best;
}

// The sparse dK/dV pass is not cut into ranges: some key blocks are on far more lists than
// others (forced ones on all), and the pass would wait for those.  Instead a block is cut
// that would take more than 1 / kPieceShare of what each of the work-groups that the chip
// holds at a time has to do, into pieces of no more than that, and of kPieceRows query rows
// or more: pieces cost partial results.  As entries / piece_max <= kPieceShare held, whatever
// the lists, pieces take kPieceShare held work-groups beyond one per block at most, and cut
// blocks have at most twice as many pieces.  5 heads of 70,409 x 2,634, D = 64, block 128,
// budget 0.1: 231 us, whole blocks 683; 3 heads of 9,013 x 30,247, budget 0.05: 195 and 270;
// 24 heads of 11,520 x 84,032, budget 0.25, where nothing is cut: 10.5 ms.  Pieces hold even
// shares of a block's lists: where neighbouring query blocks list the same keys, 5 heads of
// 70,409 x 2,634 take 221 us (cut at even shares of all query blocks, 304), 3 heads of
// 72,000 x 9,000 at D = 128 422 (495).
constexpr int kPieceShare = 2;
constexpr int kPieceRows = 1024;

// Work-groups of the pass that the chip runs at full rate (four waves per CU).
inline int bwd_held(int block) { return 1024 / (block / 32); }

// The most lists per piece, for bh heads of n_q lists of `entries` at most.
inline int attn_bwd_piece_max(int64_t bh, int64_t nq, int64_t entries, int block) {
  const double share = double(bh) * double(nq) * double(entries) / (double(kPieceShare) * bwd_held(block));
  return (int)std::min(std::max(ceil(share), double(kPieceRows / block)), 1e9);
}

// What the sparse dK/dV pass does with its key blocks (see BwdArgs), for lists of `entries` at most.
struct BwdPieces {
  int list_min, piece_max, most_pieces;
};

inline BwdPieces attn_bwd_pieces(const BwdPlan& p, int64_t bh, int64_t nq, int64_t nk, int64_t entries, int block) {
  BwdPieces c{};
  c.piece_max = p.slots > 0 ? attn_bwd_piece_max(bh, nq, entries, block) : int(nq);
  // (in order of rounds: also those on twice as many lists as the average, if rows fill their stride)
  if (p.rounds) c.list_min = int(std::max<int64_t>(1, std::min<int64_t>(c.piece_max, 2 * nq * entries / nk)));
  else if (c.piece_max < nq) c.list_min = c.piece_max;
  // blocks on more than twice the average are fewer than half, cut ones have 2 * extra pieces at most
  c.most_pieces = (p.rounds ? int(bh * nk / 2) : 0) + (c.piece_max < nq ? 2 * p.extra : 0);
  return c;
}

inline BwdPlan attn_bwd_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, bool dense) {
  const int rows = dense ? 128 : block;
  const int64_t nq = (lq + block - 1) / block, nk = (lk + block - 1) / block;
  const int64_t q_groups = bh * ((lq + rows - 1) / rows), k_groups = bh * ((lk + rows - 1) / rows);
  // (the cut does not depend on the lists: a quarter of the keys is taken for them)
  const double products = 2.0 * d * double(bh) * double(lq) * double(lk) * (dense ? 1.0 : 0.25);
  BwdPlan p{};
  p.dq_ranges = bwd_ranges(std::max<int64_t>(1, q_groups), rows / 32, (lk + 31) / 32, 3.0 * products,
                           4.0 * bh * lq * d);
  p.dkv_ranges = dense ? bwd_ranges(k_groups, rows / 32, (lq + 31) / 32, 4.0 * products, 8.0 * bh * lk * d) : 1;
  p.rounds = lq > 0 && k_groups * (rows / 32) > (d == 128 ? 1024 : 2048);
  if (!dense && lq >= 2 * kPieceRows) {
    p.extra = kPieceShare * bwd_held(block);
    const double most = double(bh * nk) * double((nq + kPieceRows / block - 1) / (kPieceRows / block));
    p.slots = (int)std::min(2.0 * p.extra, most);
  }
  auto align = [](size_t x) { return (x + 255) & ~size_t(255); };
  p.stats = 0;
  p.bits = align(size_t(bh * nq * block) * 2 * sizeof(float));
  p.count = p.bits + (dense ? 0 : align(size_t(bh * nk * ((nq + 31) / 32)) * sizeof(uint32_t)));
  const bool list = !dense && (p.rounds || p.slots > 0);
  p.pieces = p.count + (list ? 256 : 0);
  p.listed = p.pieces + (list ? align(size_t(bh * nk + p.extra) * sizeof(BwdPiece)) : 0);
  p.part = p.listed + (list ? align(size_t(bh * nk)) : 0);
  const size_t dq = p.dq_ranges > 1 ? size_t(bh * lq * d) * p.dq_ranges * sizeof(float) : 0;
  const size_t dkv = p.dkv_ranges > 1 ? 2 * size_t(bh * lk * d) * p.dkv_ranges * sizeof(float) : 0;
  p.part_kv = p.part + align(dq);
  p.part_piece = p.part_kv + align(dkv);
  p.total = p.part_piece + 2 * size_t(p.slots) * block * d * sizeof(float);
  return p;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32 (launch_bwd).
inline int64_t attn_bwd_threads(const BwdPlan& p, int64_t bh, int64_t lq, int64_t lk, int d, int block, bool dense,
                                int64_t most_pieces) {
  const int64_t rows = dense ? 128 : block, nq = (lq + block - 1) / block, nk = (lk + block - 1) / block;
  const int64_t prepare = bh * nq * block * (d / 8) + (dense ? 0 : 256 * bh * ((nq + 31) / 32) * (nk / kBitsChunk + 1)) + 256;
  const int64_t dq = bh * p.dq_ranges * ((lq + rows - 1) / rows) * 2 * rows;
  const int64_t dkv = (bh * p.dkv_ranges * ((lk + rows - 1) / rows) + most_pieces) * 2 * rows;
  const int64_t sum = bh * std::max(p.dq_ranges > 1 ? lq : 0, p.dkv_ranges > 1 ? lk : 0) * (d / 8) + 256;
  return std::max({prepare, dq, dkv, sum, 8 * bh * nk + 256});
}

}  // namespace sparstar
