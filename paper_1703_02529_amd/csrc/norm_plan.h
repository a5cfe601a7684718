// How group normalisation splits a call, and what of that arithmetic its kernels
// share: no GPU headers, so that a host compiler alone can check it.
#pragma once

#include "sizes.h"

#ifdef __HIPCC__
#define NSC_HD __host__ __device__ __forceinline__
#else
#define NSC_HD inline
#endif

namespace nsc {

// Of the ve values at position pos of step p, those that lie inside an image of
// hw pixels of c channels (none or less: the vector lies behind it).  A step is
// s pixels, and only the last of an image's steps can be ragged; an image may
// hold more than 2^31 values.
NSC_HD int values_inside(int32_t hw, int32_t c, int32_t s, int32_t steps, int32_t p, int32_t pos,
                         int32_t ve) {
  if (p + 1 < steps) return ve;
  const int64_t left = (int64_t)hw * c - ((int64_t)p * s * c + pos);
  return left < ve ? (int)left : ve;
}

constexpr int kMaxParts = 64;  // of an image

struct NormPlan {
  int32_t ve, s, cb, gpb, blocks, cv, pl, threads;
  int32_t v;                // vectors a thread keeps in registers; 0: read twice
  int32_t parts;            // 1: one launch
};

constexpr int64_t kPartBytes = 16384;  // a part is at least that much

// Vectors a thread that kernels are built for; the next larger one takes what
// lies between and leaves the rest of its vectors out.  Each step's size in the
// next step's kernel (bf16, 64 channels, forward): 16,384 maps of 60 pixels 78 us
// with 2 vectors, 83 with 4, 190 with 20; 2,048 maps of 1,270, 1,530 and 2,040
// pixels 140, 164 and 217 us with 10, 12 and 16, and 185, 203 and 252 with 20 (fp32
// without spills: alike).  6 and 8 are alike forward.  Read twice instead of 20:
// 1,031 maps of 50x50x64 201 against 166 us.
constexpr int32_t kResident[] = {2, 4, 6, 8, 10, 12, 16, 20};

// How a call is split, by its sizes and alignment alone.  max_count images.
inline NormPlan plan_norm(const nsc_norm_desc& d, uintptr_t ptrs, int64_t max_count,
                          bool backward) {
  NormPlan p{};
  const int32_t es = (int32_t)type_bytes(d.dtype), cpg = d.c / d.groups;
  const int64_t hw = (int64_t)d.h * d.w;
  // The widest vectors at which every image starts
  p.ve = 16 / es;
  while (p.ve > 1 && (ptrs % (uintptr_t)(p.ve * es) || d.x_stride % p.ve || d.y_stride % p.ve))
    p.ve /= 2;
  p.s = p.ve / (int32_t)gcd64(p.ve, d.c);
  const int32_t most_v = backward ? 10 : 20, most_t = backward ? 512 : 1024;
  if (p.s > 1) {
    // several pixels make whole vectors: a block is all channels
    if ((int64_t)p.s * d.c / p.ve > most_t) {
      p.ve = 1;
      p.s = 1;
    } else {
      p.gpb = d.groups;
    }
  }
  if (p.s == 1) {
    // A block is the fewest whole groups that make 128 bytes of a pixel, a cache
    // line (1,031 maps of 50x50x64 bf16 in registers: 172 us; as blocks of half
    // a line 199 us, of a quarter 328 us), fewer where the call has too few
    // blocks to fill the chip.
    auto groups_for = [&](int64_t bytes) {  // at most 256 vectors wide, if it can be
      int32_t best = 0;
      for (int32_t g = 1; g <= d.groups; ++g) {
        if (g * cpg / p.ve > (best ? 256 : most_t)) break;
        if (d.groups % g || (g * cpg) % p.ve) continue;
        best = g;
        if ((int64_t)g * cpg * es >= bytes) break;
      }
      return best;
    };
    p.gpb = groups_for(128);
    if (p.gpb == 0) {  // no such block: single elements, a group at a time
      p.ve = 1;
      p.gpb = groups_for(128);
      if (p.gpb == 0) p.gpb = 1;
    }
    if (hw * p.gpb * cpg * es > (int64_t)most_t * most_v * 16) {
      // too large for registers: with few images as contiguous as can be (they
      // are split by pixels), else as above
      const int32_t g = groups_for(4096);
      if (g > 0 && max_count * (d.groups / p.gpb) < 2 * kNumCU) p.gpb = g;
    } else {
      for (int64_t bytes = 64; bytes >= 16; bytes /= 2) {
        if (max_count * (d.groups / p.gpb) >= kNumCU || hw * p.gpb * cpg * es <= 8192) break;
        const int32_t g = groups_for(bytes);
        if (g == 0) break;
        p.gpb = g;
      }
    }
  }
  p.cb = p.gpb * cpg;
  p.blocks = d.groups / p.gpb;
  p.cv = p.s * p.cb / p.ve;
  const int64_t steps = (hw + p.s - 1) / p.s;
  // The smallest workgroup that holds the block, eight vectors a thread if it can
  p.threads = most_t;
  p.v = 0;
  for (int32_t t = 256; t <= most_t; t *= 2) {
    if (p.cv > t) continue;
    const int64_t v = (steps + t / p.cv - 1) / (t / p.cv);
    if (v > most_v || (v > 8 && t < most_t)) continue;
    p.threads = t;
    for (int32_t r : kResident)
      if (r >= v) {
        p.v = r;
        break;
      }
    break;
  }
  // Parts where the images do not fill the chip: about 1,024 workgroups of 256,
  // or what kMaxParts allows of larger ones, each part of at least 16 KB.  (A
  // workgroup of 1,024 has its CU alone: up to two rounds of them are split as
  // well; 300 maps of 37x41x45: 58 against 44 us.)
  p.parts = 1;
  const int64_t items = max_count * p.blocks, bytes = hw * p.cb * es;
  if (p.threads == 1024 && items < 2 * kNumCU && bytes > 32768) p.v = 0;
  if (p.v == 0) p.threads = p.cv > 512 ? 1024 : 512;  // (backward, 1,024: single elements)
  if (items > 0 && p.v == 0 && items < 2 * kNumCU) {
    int64_t parts = (4 * kNumCU + items - 1) / items;
    if (parts > bytes / kPartBytes) parts = bytes / kPartBytes;
    if (parts > steps) parts = steps;
    if (parts > kMaxParts) parts = kMaxParts;
    if (parts > 1) {
      p.parts = (int32_t)parts;
      const int32_t t = items * parts >= 3 * kNumCU ? 256 : items * parts > kNumCU ? 512 : most_t;
      if (p.cv <= t && p.threads < 1024) p.threads = t;
    }
  }
  p.pl = p.threads / p.cv;
  return p;
}

// The parts' statistics of a call of count images: for any alignment of its
// tensors (gradients: and for the sums over images).
inline size_t norm_call_bytes(const nsc_norm_desc& d, int64_t count, bool backward) {
  int64_t parts = 1;
  for (uintptr_t align = 16; align >= (uintptr_t)type_bytes(d.dtype); align /= 2) {
    const NormPlan p = plan_norm(d, align, count, backward);
    if (p.parts > parts) parts = p.parts;
  }
  if (backward) return (size_t)count * parts * d.c * 8;
  return parts > 1 ? (size_t)count * parts * d.groups * 8 : 0;
}

// Of every call of up to max_count images.  Fewer images are split into more
// parts, so that a smaller call can need more; from 2 kNumCU on, and where an
// image does not make two parts, none is split.
inline size_t norm_ws_bytes(const nsc_norm_desc& d, int64_t max_count, bool backward) {
  size_t most = norm_call_bytes(d, max_count, backward);
  if ((int64_t)d.h * d.w * d.c * type_bytes(d.dtype) < 2 * kPartBytes) return most;
  for (int64_t n = 1; n < max_count && n < 2 * kNumCU; ++n) {
    const size_t b = norm_call_bytes(d, n, backward);
    if (b > most) most = b;
  }
  return most;
}

}  // namespace nsc
