// How a projection with adapters splits a call: no GPU headers, so that a host
// compiler alone can check it.
#pragma once

#include "sizes.h"

namespace nsc {

// How a product is split: tiles of tn outputs x tm rows and parts of the
// reduction, chosen by the sizes alone.
struct GemmPlan {
  int32_t tn, tm, parts;
};

inline GemmPlan plan_gemm(int64_t max_rows, int64_t outs, int64_t len, int64_t es, bool tr) {
  GemmPlan p{};
  // Large tiles read each operand least often; they need enough of them to
  // fill the chip
  auto tiles = [&](int64_t tn, int64_t tm) {
    return (outs + tn - 1) / tn * ((max_rows + tm - 1) / tm);
  };
  const int64_t blocks = (len * es + 127) / 128;
  const bool few = !tr && outs <= 64 && max_rows > 16;
  const bool big = !few && tiles(256, 128) >= kNumCU && blocks >= 16;
  p.tn = big ? 256 : 128;
  p.tm = big ? 128 : max_rows <= 16 ? 16 : 64;
  // Up to 64 outputs would leave half of a tile of 128 to multiply zeros, which
  // counts where the matrix instructions are slow: 3,038 rows of 4,608 values
  // onto 32 outputs in fp32 took 91 us with 128 and take 61 with 64.  Backward
  // the tiles run over the inputs, which are many.
  if (few) p.tn = 64;
  const int64_t t = tiles(p.tn, p.tm);
  // parts for about a workgroup per CU, each of at least four blocks
  int64_t parts = t > 0 ? kNumCU / t : 1;
  if (parts > blocks / 4) parts = blocks / 4;
  if (parts > 64) parts = 64;
  p.parts = parts < 1 ? 1 : (int32_t)parts;
  return p;
}

inline size_t gemm_part_bytes(const GemmPlan& p, int64_t max_rows, int64_t outs) {
  if (p.parts == 1) return 0;
  return (size_t)((outs + p.tn - 1) / p.tn * p.tn) * ((max_rows + p.tm - 1) / p.tm * p.tm) *
         p.parts * 4;
}

// Waves of a workgroup for the rank-wide rows, alone in a launch and beside a
// split product, and most parts of their reduction.
constexpr int kDownWaves = 8, kGemmDownWaves = 4;
constexpr int kMaxDownParts = 4, kMaxJoinParts = 8;

// Parts of the rank-wide rows' reduction: about two workgroups per CU, four of
// the smaller ones beside a split product, each wave of at least two chunks of
// 128 bytes.
inline int32_t down_parts(int64_t max_rows, int64_t len, int64_t es, bool split) {
  const int64_t tiles = (max_rows + 15) / 16, per = split ? 4 : 2;
  int64_t parts = tiles > 0 ? per * kNumCU / tiles : 1;
  const int64_t most = len * es / (128 * 2 * (split ? kGemmDownWaves : kDownWaves));
  if (parts > most) parts = most;
  const int64_t room = split ? kMaxJoinParts : kMaxDownParts;
  if (parts > room) parts = room;
  return parts < 1 ? 1 : (int32_t)parts;
}

// From this many rows on they are taken in the order of their adapters, so that
// 16 neighbours mostly share one.
constexpr int64_t kListRows = 256;

// Workspace: the rank-wide rows t (backward: and u) by part, the product's
// partial sums, the rows by adapter, and backward b transposed.
struct AdapterLayout {
  size_t t, u, part, off, rows, bt, total;
  int32_t t_parts, u_parts;
  GemmPlan g;
  bool list;
};

inline AdapterLayout adapter_layout(const nsc_adapter_desc& d, int64_t max_rows, bool backward) {
  AdapterLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = align_up(o + bytes, 256);
    return at;
  };
  const int64_t es = type_bytes(d.dtype);
  const size_t rp = align_up(d.rank, 16);
  L.g = backward ? plan_gemm(max_rows, d.k, d.d, es, true)
                 : plan_gemm(max_rows, d.d, d.k, es, false);
  L.t_parts = down_parts(max_rows, d.k, es, !backward && L.g.parts > 1);
  L.u_parts = down_parts(max_rows, d.d, es, false);
  L.list = backward || max_rows >= kListRows;
  L.t = take((size_t)max_rows * rp * 4 * L.t_parts);
  if (backward) {
    L.u = take((size_t)max_rows * rp * 4 * L.u_parts);
    if (max_rows > 0) L.bt = take((size_t)d.n_adapters * d.rank * d.d * es);
  }
  L.part = take(gemm_part_bytes(L.g, max_rows, backward ? d.k : d.d));
  if (L.list) {
    L.off = take(((size_t)d.n_adapters + 1) * 4);
    L.rows = take((size_t)max_rows * 4);
  }
  L.total = o;
  return L;
}

// Of every call of up to max_rows rows.  Fewer rows are split into more parts,
// so that a smaller call can need more.  Between multiples of 16 rows a call
// only grows, and from 8,192 rows on neither reduction is split: 128 tiles of 64
// rows leave a tile fewer than two parts, 512 tiles of 16 its rank-wide rows.
inline size_t adapter_ws_bytes(const nsc_adapter_desc& d, int64_t max_rows, bool backward) {
  size_t most = adapter_layout(d, max_rows, backward).total;
  for (int64_t n = 16; n < max_rows && n <= 8192; n += 16) {
    const size_t b = adapter_layout(d, n, backward).total;
    if (b > most) most = b;
  }
  return most;
}

// Waves share an adapter's rows where its columns alone make too few of them
// (about two per SIMD) and it has two steps of 16 rows for each on average.
inline int grad_row_waves(int64_t cols, int32_t n_adapters, int64_t max_rows, int64_t es) {
  const int64_t waves = cols / (16 * (16 / es)) * n_adapters;
  int rw = 1;
  while (rw < 8 && waves * rw < 8 * kNumCU && max_rows / n_adapters >= 2 * 16 * 2 * rw) rw *= 2;
  return rw;
}

}  // namespace nsc
