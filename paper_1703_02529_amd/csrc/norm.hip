// Group normalisation of channels-last maps with an activation, and its
// gradients (nsc_group_norm, nsc_group_norm_backward).
//
// A work item is one image's block of whole groups: a run of channels of every
// pixel.  Its threads are dealt over the block's vectors of VE channels first
// and over pixels second, so that every thread keeps the same channels for all
// its pixels: their parameters and sums stay in registers, and consecutive
// lanes read consecutive memory.  Where VE does not divide the channels, S
// pixels together are whole vectors and take a pixel's place ("step" below);
// the last step may then be ragged.
//
// Statistics: each thread takes the mean and the sum of squared deviations
// from it (M2) of a chunk of pixels it holds in registers, and chunks, threads
// and parts are joined by
//   mean = (na ma + nb mb) / n,  M2 = M2a + M2b + (mb - ma)^2 na nb / n,
// so that no sum of squares ever cancels against the square of a mean; all of
// it in fp32.
//
// Both directions move each byte once where a block fits a workgroup's
// registers (V vectors a thread): it is loaded, reduced and written back from
// there.  Larger blocks are read a second time, from the caches while they
// hold them.  A few large images are split over workgroups that leave their
// parts' statistics in the workspace for a second launch to join.
#include "layer_types.h"
#include "norm_plan.h"

#include <math.h>


namespace nsc {
namespace {

struct NormArgs {
  const void* x;
  const void* dy;
  void* out;                // y or dx
  const float* gamma;
  const float* beta;
  float* stats;             // forward: nullable output; backward: input
  float* part;              // workspace: [image][part][group] (mean, M2), or
                            // [image][part][channel] (sum dz, sum dz xh)
  const int32_t* count;     // nullable
  int64_t max_count;
  int64_t x_stride, y_stride;
  int32_t hw, c, cpg, groups;
  int32_t cb;               // channels of a block
  int32_t gpb;              // groups of a block
  int32_t blocks;           // blocks of an image
  int32_t cv;               // vectors of a block's step
  int32_t pl;               // steps the threads cover at once
  int32_t s;                // pixels of a step
  int32_t steps;            // of an image, the last one ragged unless s divides hw
  int32_t parts;            // parts of an image
  float eps;
  int32_t act;
};

__device__ __forceinline__ int64_t live_count(const NormArgs& a) {
  int64_t n = a.count ? *a.count : a.max_count;
  return n < a.max_count ? n : a.max_count;
}

// The activation of VE values; `floor` is what the values are cut at below (0
// for ReLU, minus infinity without an activation).  NaN stays.  SiLU's
// exponential and reciprocal are the instructions of the machine, for fp32 too:
// their error, |z| and a few roundings of 2^-24, is that of z itself (128 maps of
// 50x50x64 fp32: mean error 0.89 (gradient) and 1.01 of that of the elementary
// operations in fp32).
template <int VE>
__device__ __forceinline__ void activate(float (&z)[VE], int act, float floor) {
  if (act == NSC_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < VE; ++e) z[e] *= __builtin_amdgcn_rcpf(1.0f + __expf(-z[e]));
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) z[e] = __builtin_elementwise_maximum(z[e], floor);
  }
}
__device__ __forceinline__ float act_floor(int act) {
  return act == NSC_ACT_RELU ? 0.0f : -__builtin_inff();
}

// (na, ma, qa) joined with (nb, mb, qb), nb > 0.  (Joined with nothing, the
// means' distance is not squared: it is the mean itself.)
__device__ __forceinline__ void join(float& na, float& ma, float& qa, float nb, float mb,
                                     float qb) {
  const float n = na + nb, f = nb / n, d = mb - ma, dq = na > 0.0f ? d : 0.0f;
  ma += d * f;
  qa += qb + dq * dq * na * f;
  na = n;
}

// One work item's place: image, block, part, and this thread's vector in it.
template <typename T, int VE, bool RAG>
struct Place {
  int64_t img;
  int blk, part, v, p0;
  int first, last;          // the part's steps
  bool on;                  // the thread has vectors at all
  int ch0;                  // channel of the block's first
  __device__ __forceinline__ Place(const NormArgs& a, int64_t item) {
    const int64_t ib = item / a.parts;
    part = (int)(item - ib * a.parts);
    img = ib / a.blocks;
    blk = (int)(ib - img * a.blocks);
    p0 = threadIdx.x / a.cv;
    v = threadIdx.x - p0 * a.cv;
    on = p0 < a.pl;
    first = (int)((int64_t)part * a.steps / a.parts);
    last = (int)((int64_t)(part + 1) * a.steps / a.parts);
    ch0 = blk * a.cb;
  }
  // Channel of the block of the thread's value e.
  __device__ __forceinline__ int channel(const NormArgs& a, int e) const {
    return RAG ? (v * VE + e) % a.c : v * VE + e;
  }
  // Values of the thread's vector that lie inside the image at step p.
  __device__ __forceinline__ int inside(const NormArgs& a, int p) const {
    return RAG ? values_inside(a.hw, a.c, a.s, a.steps, p, v * VE, VE) : VE;
  }
  __device__ __forceinline__ int64_t offset(const NormArgs& a, int p) const {
    return (int64_t)p * a.s * a.c + ch0 + v * VE;
  }
  __device__ __forceinline__ Pack<T, VE> load(const NormArgs& a, const T* x, int p) const {
    const T* at = x + offset(a, p);
    if (!RAG || p + 1 < a.steps) return Pack<T, VE>::load(at);
    Pack<T, VE> r{};
    const int n = inside(a, p);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < n) r.set(e, at[e]);
    return r;
  }
  __device__ __forceinline__ void store(const NormArgs& a, T* y, int p, const float (&f)[VE]) const {
    T* at = y + offset(a, p);
    if (!RAG || p + 1 < a.steps) return Pack<T, VE>::from_f32(f).store(at);
    const int n = inside(a, p);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < n) at[e] = (T)f[e];
  }
  // Steps of pixel lane p in the part that hold position pos of a step.
  __device__ __forceinline__ int held(const NormArgs& a, int p, int pos) const {
    int n = last - first - p;
    n = n > 0 ? (n + a.pl - 1) / a.pl : 0;
    if (RAG && n > 0 && last == a.steps && (a.steps - 1 - first - p) % a.pl == 0 &&
        (int64_t)(a.steps - 1) * a.s * a.c + pos >= (int64_t)a.hw * a.c)
      --n;
    return n;
  }
};

constexpr int kNormChunk = 8;  // vectors of a thread in flight together

// Adds a chunk of C vectors, whose first cnt are inside, to the thread's
// statistics: K = 1, of all its channels (they lie in one group); K = VE, of
// each.  Ragged vectors leave out their values from `rag` on.  FULL: all of C
// are whole.
template <typename T, int VE, int K, bool RAG, bool FULL, int C>
__device__ __forceinline__ void add_chunk(Pack<T, VE> (&x)[C], int cnt, int rag,
                                          float (&n)[RAG ? K : 1], float (&m)[K], float (&q)[K]) {
  if (FULL) {
    cnt = C;
    rag = VE;
  }
  float s[K], mb[K], d2[K];
#pragma unroll
  for (int k = 0; k < K; ++k) s[k] = d2[k] = 0.0f;
#pragma unroll
  for (int u = 0; u < C; ++u) {
    x[u].renew();
    float f[VE];
    x[u].to_f32(f);
    if constexpr (K == 1) {
      float t = 0.0f;
#pragma unroll
      for (int e = 0; e < VE; ++e) t += f[e];
      if (FULL || u < cnt) s[0] += t;
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (FULL || (u < cnt && !(RAG && u + 1 == cnt && e >= rag))) s[e] += f[e];
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k)
    mb[k] = s[k] / (float)(K == 1 ? cnt * VE : RAG && k >= rag ? (cnt > 1 ? cnt - 1 : 1) : cnt);
#pragma unroll
  for (int u = 0; u < C; ++u) {
    x[u].renew();
    float f[VE];
    x[u].to_f32(f);
    if constexpr (K == 1) {
      float t = 0.0f;
#pragma unroll
      for (int e = 0; e < VE; ++e) t = fmaf(f[e] - mb[0], f[e] - mb[0], t);
      if (FULL || u < cnt) d2[0] += t;
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (FULL || (u < cnt && !(RAG && u + 1 == cnt && e >= rag)))
          d2[e] = fmaf(f[e] - mb[e], f[e] - mb[e], d2[e]);
    }
  }
  if constexpr (K == 1) {
    join(n[0], m[0], q[0], (float)(cnt * VE), mb[0], d2[0]);
  } else {
    const float na = n[0];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      if constexpr (RAG) {
        const int c = e >= rag ? cnt - 1 : cnt;
        if (c > 0) join(n[e], m[e], q[e], (float)c, mb[e], d2[e]);
      } else {
        n[0] = na;
        join(n[0], m[e], q[e], (float)cnt, mb[e], d2[e]);
      }
    }
  }
}

// Each group's statistics of an item's part from its threads' (mean, M2).  A
// wave takes a group at a time.  sm: 2 K blockDim floats; the results (mean,
// M2) in gs[group of the block].
template <typename T, int VE, int K, bool RAG>
__device__ __forceinline__ void reduce_groups(const NormArgs& a, const Place<T, VE, RAG>& at,
                                              const float (&m)[K], const float (&q)[K], float* sm,
                                              float2* gs, float total) {
  const int T_ = blockDim.x, lane = threadIdx.x & 63, waves = T_ >> 6;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    sm[(2 * k) * T_ + threadIdx.x] = m[k];
    sm[(2 * k + 1) * T_ + threadIdx.x] = q[k];
  }
  __syncthreads();
  // a group's entries per pixel lane: vectors (K = 1) or values
  const int one = K == 1 ? a.cpg / VE : a.cpg, per = RAG ? a.s * one : one;
  const int entries = a.pl * per;
  for (int g = threadIdx.x >> 6; g < a.gpb; g += waves) {
    auto entry = [&](int i, int& slot, float& n) {
      const int p = i / per, r = i - p * per;
      int pos = g * one + r;
      if (RAG) pos = r / one * a.c + g * one + r % one;
      slot = K == 1 ? p * a.cv + pos : (2 * (pos % VE)) * T_ + p * a.cv + pos / VE;
      n = (float)(at.held(a, p, pos) * (K == 1 ? VE : 1));
    };
    float sum = 0.0f;
    for (int i = lane; i < entries; i += 64) {
      int slot;
      float n;
      entry(i, slot, n);
      if (n > 0.0f) sum += sm[slot] * n;
    }
    const float mean = wave_sum(sum) / total;
    float dev = 0.0f;
    for (int i = lane; i < entries; i += 64) {
      int slot;
      float n;
      entry(i, slot, n);
      const float d = sm[slot] - mean;
      if (n > 0.0f) dev += sm[slot + T_] + d * d * n;
    }
    dev = wave_sum(dev);
    if (lane == 0) gs[g] = make_float2(mean, dev);
  }
  __syncthreads();
}

// Whole: statistics and output of whole images; Stats and Apply: the two
// launches of split ones.
enum class NormPass { Whole, Stats, Apply };

template <typename T, int VE, int K, bool RAG, int V, NormPass P>
__global__ void __launch_bounds__(1024) k_norm(NormArgs a) {
  extern __shared__ __align__(16) float sm[];
  float2* gs = reinterpret_cast<float2*>(sm + (P == NormPass::Apply ? 0 : 2 * K * blockDim.x));
  const int64_t items = live_count(a) * a.blocks * a.parts;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const Place<T, VE, RAG> at(a, P == NormPass::Whole && gridDim.x == items ? xcd_block(i, items) : i);
    const T* x = static_cast<const T*>(a.x) + at.img * a.x_stride;
    const int begin = at.on ? at.first + at.p0 : at.last;
    constexpr int C = V > 0 ? V : kNormChunk;
    Pack<T, VE> xv[C];
    if constexpr (P != NormPass::Apply) {
      float n[RAG ? K : 1], m[K], q[K];
#pragma unroll
      for (int k = 0; k < K; ++k) m[k] = q[k] = 0.0f;
#pragma unroll
      for (int k = 0; k < (RAG ? K : 1); ++k) n[k] = 0.0f;
      for (int p = begin; p < at.last; p += a.pl * C) {
        int cnt = 0, rag = VE;
#pragma unroll
        for (int u = 0; u < C; ++u) {
          const int pu = p + u * a.pl;
          if (pu < at.last) {
            xv[u] = at.load(a, x, pu);
            ++cnt;
            if (RAG && pu + 1 == a.steps) rag = at.inside(a, pu);
          }
        }
        if (cnt == C && rag == VE)
          add_chunk<T, VE, K, RAG, true>(xv, cnt, rag, n, m, q);
        else
          add_chunk<T, VE, K, RAG, false>(xv, cnt, rag, n, m, q);
        if constexpr (V > 0) break;
      }
      const float total = (float)(min((int64_t)at.last * a.s, (int64_t)a.hw) -
                                  (int64_t)at.first * a.s) * (float)a.cpg;
      reduce_groups<T, VE, K, RAG>(a, at, m, q, sm, gs, total);
    }
    const int64_t g0 = at.img * a.groups + at.blk * a.gpb;
    if constexpr (P == NormPass::Stats) {
      for (int g = threadIdx.x; g < a.gpb; g += blockDim.x)
        reinterpret_cast<float2*>(a.part)[(at.img * a.parts + at.part) * a.groups +
                                          at.blk * a.gpb + g] = gs[g];
    } else {
      // (mean, M2) of the image's groups as (mean, rstd)
      const float total = (float)a.hw * (float)a.cpg;
      auto put = [&](int g, float mean, float m2) {
        const float2 st = make_float2(mean, 1.0f / sqrtf(m2 / total + a.eps));
        gs[g] = st;
        if (a.stats && at.part == 0) reinterpret_cast<float2*>(a.stats)[g0 + g] = st;
      };
      if constexpr (P == NormPass::Apply) {
        // a wave per group and a lane per part: there are at most kMaxParts
        const int h = threadIdx.x & 63;
        const int64_t b = (int64_t)h * a.steps / a.parts * a.s;
        const int64_t e = (int64_t)(h + 1) * a.steps / a.parts * a.s;
        const float n = h < a.parts ? (float)((e < a.hw ? e : a.hw) - b) * (float)a.cpg : 0.0f;
        for (int g = threadIdx.x >> 6; g < a.gpb; g += blockDim.x >> 6) {
          const float2 t = h < a.parts
                               ? reinterpret_cast<const float2*>(
                                     a.part)[(at.img * a.parts + h) * a.groups + at.blk * a.gpb + g]
                               : make_float2(0.0f, 0.0f);
          const float mean = wave_sum(h < a.parts ? n * t.x : 0.0f) / total;
          const float m2 = wave_sum(h < a.parts ? t.y + n * (t.x - mean) * (t.x - mean) : 0.0f);
          if (h == 0) put(g, mean, m2);
        }
      } else {
        for (int g = threadIdx.x; g < a.gpb; g += blockDim.x) put(g, gs[g].x, gs[g].y);
      }
      __syncthreads();
      if (at.on) {
        T* y = static_cast<T*>(a.out) + at.img * a.y_stride;
        float mu[K], s[VE], b[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int ch = at.channel(a, e);
          const float2 st = gs[ch / a.cpg];
          if (K > 1 || e == 0) mu[K > 1 ? e : 0] = st.x;
          s[e] = a.gamma[at.ch0 + ch] * st.y;
          b[e] = a.beta[at.ch0 + ch];
        }
        arrive(s);
        arrive(b);
        const float floor = act_floor(a.act);
        auto apply = [&](Pack<T, VE>& xu, int p) __attribute__((always_inline)) {
          xu.renew();
          float f[VE];
          xu.to_f32(f);
#pragma unroll
          for (int e = 0; e < VE; ++e) f[e] = fmaf(f[e] - mu[K > 1 ? e : 0], s[e], b[e]);
          activate<VE>(f, a.act, floor);
          at.store(a, y, p, f);
        };
        if constexpr (V > 0) {
#pragma unroll
          for (int u = 0; u < C; ++u)
            if (begin + u * a.pl < at.last) apply(xv[u], begin + u * a.pl);
        } else {
          // backwards: what was read last is nearest
          int p = begin;
          while (p + a.pl * C < at.last) p += a.pl * C;
          for (; p >= begin; p -= a.pl * C) {
#pragma unroll
            for (int u = 0; u < C; ++u)
              if (p + u * a.pl < at.last) xv[u] = at.load(a, x, p + u * a.pl);
#pragma unroll
            for (int u = 0; u < C; ++u)
              if (p + u * a.pl < at.last) apply(xv[u], p + u * a.pl);
          }
        }
      }
      __syncthreads();  // gs and sm are read before the next item writes them
    }
  }
}

// ---------------------------------------------------------------- backward

template <typename T, int VE, int K, bool RAG, int V, NormPass P>
__global__ void __launch_bounds__(VE == 1 ? 1024 : 512) k_norm_grad(NormArgs a) {
  extern __shared__ __align__(16) float sm[];  // [2 VE][blockDim], then [cb][2], then [gpb][2]
  const int T_ = blockDim.x;
  float* chs = sm + (P == NormPass::Apply ? 0 : 2 * VE * T_);
  float2* grs = reinterpret_cast<float2*>(chs + 2 * a.cb);
  const int64_t items = live_count(a) * a.blocks * a.parts;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const Place<T, VE, RAG> at(a, P == NormPass::Whole && gridDim.x == items ? xcd_block(i, items) : i);
    const T* x = static_cast<const T*>(a.x) + at.img * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + at.img * a.y_stride;
    const float2* stats =
        reinterpret_cast<const float2*>(a.stats) + at.img * a.groups + at.blk * a.gpb;
    float mu[K], rs[K], s[VE], b[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int ch = at.channel(a, e);
      const float2 st = at.on ? stats[ch / a.cpg] : make_float2(0.f, 0.f);
      if (K > 1 || e == 0) {
        mu[K > 1 ? e : 0] = st.x;
        rs[K > 1 ? e : 0] = st.y;
      }
      s[e] = at.on ? a.gamma[at.ch0 + ch] * st.y : 0.0f;
      b[e] = at.on ? a.beta[at.ch0 + ch] : 0.0f;
    }
    arrive(mu);
    arrive(rs);
    arrive(s);
    arrive(b);
    const int begin = at.on ? at.first + at.p0 : at.last;
    constexpr int C = V > 0 ? V : 4;
    Pack<T, VE> xv[C], gv[C];
    auto load = [&](int p) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < C; ++u)
        if (p + u * a.pl < at.last) {
          xv[u] = at.load(a, x, p + u * a.pl);
          gv[u] = at.load(a, dy, p + u * a.pl);
        }
    };
    // xh and dz = dy act'(z) of vector u, z = (x - mean) gamma rstd + beta.  The
    // ReLU's sign is fp64's: fp32's z is within 2^-22 of its product of the exact
    // one, and values closer to zero are taken again in fp64.
    auto grads = [&](int u, float (&dz)[VE], float (&xh)[VE]) __attribute__((always_inline)) {
      xv[u].renew();
      gv[u].renew();
      float f[VE];
      xv[u].to_f32(f);
      gv[u].to_f32(dz);
      if (a.act == NSC_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float p = (f[e] - mu[K > 1 ? e : 0]) * s[e];
          float z = p + b[e];
          if (fabsf(z) <= 5e-7f * fabsf(p) + 1e-37f)
            z = ((double)f[e] - (double)mu[K > 1 ? e : 0]) * (double)rs[K > 1 ? e : 0] *
                            (double)a.gamma[at.ch0 + at.channel(a, e)] + (double)b[e] > 0.0
                    ? 1.0f : 0.0f;
          dz[e] = z > 0.0f ? dz[e] : 0.0f;
        }
      } else if (a.act == NSC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float z = fmaf(f[e] - mu[K > 1 ? e : 0], s[e], b[e]);
          const float t = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
          dz[e] *= t * (1.0f + z * (1.0f - t));
        }
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) xh[e] = (f[e] - mu[K > 1 ? e : 0]) * rs[K > 1 ? e : 0];
    };
    if constexpr (P != NormPass::Apply) {
      // (fp32 over an image's pixels, fp64 over images: of the sums of 128 maps of
      // 50x50x64 fp32 the mean error is 1.2 to 2.3 x 2^-24 of their mean size, that
      // of sums all in fp64 0.4 to 1.3)
      float s1[VE], s2[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) s1[e] = s2[e] = 0.0f;
      for (int p = begin; p < at.last; p += a.pl * C) {
        load(p);
#pragma unroll
        for (int u = 0; u < C; ++u)
          if (p + u * a.pl < at.last) {
            float dz[VE], xh[VE];
            grads(u, dz, xh);
            const int n = at.inside(a, p + u * a.pl);
#pragma unroll
            for (int e = 0; e < VE; ++e)
              if (!RAG || e < n) {
                s1[e] += dz[e];
                s2[e] = fmaf(dz[e], xh[e], s2[e]);
              }
          }
        if constexpr (V > 0) break;
      }
      // the channels' sums: a channel's pixel lanes in a fixed order, by as many
      // threads as there are for each channel's two sums
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        sm[(2 * e) * T_ + threadIdx.x] = s1[e];
        sm[(2 * e + 1) * T_ + threadIdx.x] = s2[e];
      }
      __syncthreads();
      const int per = RAG ? a.s : 1;  // positions of a channel in a step
      int width = 1;                  // lanes that share a sum
      while (width < 64 && width * 2 * (2 * a.cb) <= T_ && width * 2 <= a.pl * per) width *= 2;
      for (int j0 = 0; j0 < 2 * a.cb; j0 += T_ / width) {
        const int j = j0 + threadIdx.x / width;
        float t = 0.0f;
        if (j < 2 * a.cb)
          for (int k = threadIdx.x % width; k < a.pl * per; k += width) {
            const int pos = (j >> 1) + (RAG ? k % per * a.c : 0);
            t += sm[(2 * (pos % VE) + (j & 1)) * T_ + k / per * a.cv + pos / VE];
          }
        for (int o = width / 2; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
        if (j < 2 * a.cb && threadIdx.x % width == 0) {
          chs[j] = t;
          a.part[((at.img * a.parts + at.part) * a.c + at.ch0) * 2 + j] = t;
        }
      }
    } else {
      for (int j = threadIdx.x; j < 2 * a.cb; j += T_) {
        float t = 0.0f;
        for (int h = 0; h < a.parts; ++h)
          t += a.part[((at.img * a.parts + h) * a.c + at.ch0) * 2 + j];
        chs[j] = t;
      }
    }
    if constexpr (P != NormPass::Stats) {
      __syncthreads();
      // the groups' means of gamma dz and gamma dz xh
      const float inv = 1.0f / ((float)a.hw * (float)a.cpg);
      for (int g = threadIdx.x; g < a.gpb; g += T_) {
        float t1 = 0.0f, t2 = 0.0f;
        for (int k = g * a.cpg; k < (g + 1) * a.cpg; ++k) {
          const float ga = a.gamma[at.ch0 + k];
          t1 += ga * chs[2 * k];
          t2 += ga * chs[2 * k + 1];
        }
        grs[g] = make_float2(t1 * inv, t2 * inv);
      }
      __syncthreads();
      if (at.on) {
        T* dx = static_cast<T*>(a.out) + at.img * a.x_stride;
        float m1[K], m2[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const float2 t = grs[at.channel(a, k) / a.cpg];
          m1[k] = t.x;
          m2[k] = t.y;
        }
        auto apply = [&](int u, int p) __attribute__((always_inline)) {
          float dz[VE], xh[VE];
          grads(u, dz, xh);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const int k = K > 1 ? e : 0;
            dz[e] = fmaf(s[e], dz[e], -rs[k] * fmaf(xh[e], m2[k], m1[k]));
          }
          at.store(a, dx, p, dz);
        };
        int p = begin;
        if constexpr (V == 0)  // backwards: what was read last is nearest
          while (p + a.pl * C < at.last) p += a.pl * C;
        for (; p >= begin; p -= a.pl * C) {
          if constexpr (V == 0) load(p);
#pragma unroll
          for (int u = 0; u < C; ++u)
            if (p + u * a.pl < at.last) apply(u, p + u * a.pl);
          if constexpr (V > 0) break;
        }
      }
    }
    __syncthreads();  // chs and sm are read before the next item writes them
  }
}

// dgamma and dbeta: a workgroup per channel adds the images' (and their
// parts') sums, each thread its own in order, then the threads' in a tree, in fp64.
__global__ void __launch_bounds__(256) k_norm_grad_params(const float* part, const int32_t* count,
                                                          int64_t max_count, int32_t parts,
                                                          int32_t c, float* dgamma, float* dbeta) {
  __shared__ double red[2][256];
  int64_t n = count ? *count : max_count;
  if (n > max_count) n = max_count;
  n *= parts;
  const int ch = blockIdx.x, t = threadIdx.x;
  double s1 = 0.0, s2 = 0.0;
  for (int64_t i = t; i < n; i += 256) {
    const float2 v = reinterpret_cast<const float2*>(part)[i * c + ch];
    s1 += v.x;
    s2 += v.y;
  }
  red[0][t] = s1;
  red[1][t] = s2;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (t < o) {
      red[0][t] += red[0][t + o];
      red[1][t] += red[1][t + o];
    }
    __syncthreads();
  }
  if (t == 0) {
    dbeta[ch] = (float)red[0][0];
    dgamma[ch] = (float)red[1][0];
  }
}

// -------------------------------------------------------------------- host

int check_norm(const nsc_norm_desc* d) {
  NSC_REQUIRE_L(d != nullptr, NSC_E_INVAL, "norm description is NULL");
  NSC_REQUIRE_L(d->h >= 1 && d->w >= 1 && (int64_t)d->h * d->w <= (1 << 24), NSC_E_SHAPE,
                "map %dx%d outside 1x1 .. 2^24 pixels", d->h, d->w);
  NSC_REQUIRE_L(d->c >= 1 && d->c <= NSC_MAX_NORM_CHANNELS, NSC_E_SHAPE,
                "%d channels outside 1..%d", d->c, NSC_MAX_NORM_CHANNELS);
  NSC_REQUIRE_L(d->groups >= 1 && d->groups <= d->c && d->c % d->groups == 0, NSC_E_SHAPE,
                "%d groups do not divide %d channels", d->groups, d->c);
  NSC_REQUIRE_L(d->c / d->groups <= NSC_MAX_NORM_GROUP, NSC_E_SHAPE,
                "groups of %d channels exceed %d", d->c / d->groups, NSC_MAX_NORM_GROUP);
  NSC_REQUIRE_L(d->act >= NSC_ACT_NONE && d->act <= NSC_ACT_SILU, NSC_E_INVAL,
                "act %d is not one of NSC_ACT_NONE / RELU / SILU", d->act);
  NSC_REQUIRE_L(d->dtype >= NSC_T_F32 && d->dtype <= NSC_T_F16, NSC_E_DTYPE, "dtype %d is unknown",
                d->dtype);
  NSC_REQUIRE_L(isfinite(d->eps) && d->eps > 0.0f, NSC_E_INVAL, "eps must be finite and above 0");
  const int64_t e = (int64_t)d->h * d->w * d->c;
  NSC_REQUIRE_L(d->x_stride >= e && d->y_stride >= e, NSC_E_INVAL,
                "image strides %lld, %lld are below one map (%lld elements)",
                (long long)d->x_stride, (long long)d->y_stride, (long long)e);
  NSC_REQUIRE_L(d->x_stride <= ((int64_t)1 << 40) && d->y_stride <= ((int64_t)1 << 40),
                NSC_E_INVAL, "image strides beyond 2^40 elements");
  return NSC_OK;
}

constexpr int64_t kMaxImages = 0x7FFFFFFF;

NormArgs norm_args(const nsc_norm_desc& d, const NormPlan& p, const int32_t* count,
                   int64_t max_count) {
  NormArgs a{};
  a.count = count;
  a.max_count = max_count;
  a.x_stride = d.x_stride;
  a.y_stride = d.y_stride;
  a.hw = d.h * d.w;
  a.c = d.c;
  a.cpg = d.c / d.groups;
  a.groups = d.groups;
  a.cb = p.cb;
  a.gpb = p.gpb;
  a.blocks = p.blocks;
  a.cv = p.cv;
  a.pl = p.pl;
  a.s = p.s;
  a.steps = (a.hw + p.s - 1) / p.s;
  a.parts = p.parts;
  a.eps = d.eps;
  a.act = d.act;
  return a;
}

template <typename T, int VE, int K, bool RAG, int V, NormPass P>
int launch_norm(const NormArgs& a, const NormPlan& p, bool backward, hipStream_t st) {
  // (a launch has fewer than 2^32 threads; its workgroups take the items behind)
  int64_t grid = a.max_count * p.blocks * p.parts;
  const int64_t most = 0xFFFFFFFFll / p.threads;
  if (grid > most) grid = most;
  const dim3 g((unsigned)grid), b((unsigned)p.threads);
  if (backward) {
    if constexpr (V <= 10) {
      const size_t lds =
          (size_t)((P == NormPass::Apply ? 0 : 2 * VE * p.threads) + 2 * p.cb + 2 * p.gpb) * 4;
      hipLaunchKernelGGL((k_norm_grad<T, VE, K, RAG, V, P>), g, b, lds, st, a);
      NSC_CHECK_LAUNCH("k_norm_grad");
    }
    return NSC_OK;
  }
  const size_t lds = (size_t)((P == NormPass::Apply ? 0 : 2 * K * p.threads) + 2 * p.gpb) * 4;
  hipLaunchKernelGGL((k_norm<T, VE, K, RAG, V, P>), g, b, lds, st, a);
  NSC_CHECK_LAUNCH("k_norm");
  return NSC_OK;
}

template <typename T, int VE, int K, bool RAG>
int launch_form(const NormArgs& a, const NormPlan& p, bool backward, hipStream_t st) {
  if (p.parts > 1) {
    if (int rc = launch_norm<T, VE, K, RAG, 0, NormPass::Stats>(a, p, backward, st)) return rc;
    return launch_norm<T, VE, K, RAG, 0, NormPass::Apply>(a, p, backward, st);
  }
#define NSC_NORM_CASE(N) \
  case N:                \
    return launch_norm<T, VE, K, RAG, N, NormPass::Whole>(a, p, backward, st);
  switch (p.v) {
    NSC_NORM_CASE(2)
    NSC_NORM_CASE(4)
    NSC_NORM_CASE(6)
    NSC_NORM_CASE(8)
    NSC_NORM_CASE(10)
    NSC_NORM_CASE(12)
    NSC_NORM_CASE(16)
    NSC_NORM_CASE(20)
    default:
      return launch_norm<T, VE, K, RAG, 0, NormPass::Whole>(a, p, backward, st);
  }
#undef NSC_NORM_CASE
}

template <typename T>
int launch_type(const NormArgs& a, const NormPlan& p, bool backward, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  if (p.ve == 1) return launch_form<T, 1, 1, false>(a, p, backward, st);
  if (p.s == 1) {
    // a vector's channels lie in one group, or not
    if (p.ve == V)
      return a.cpg % V == 0 ? launch_form<T, V, 1, false>(a, p, backward, st)
                            : launch_form<T, V, V, false>(a, p, backward, st);
    if (p.ve == 2) return launch_form<T, 2, 2, false>(a, p, backward, st);
    if constexpr (V == 8) return launch_form<T, 4, 4, false>(a, p, backward, st);
  }
  if (p.ve == V) return launch_form<T, V, V, true>(a, p, backward, st);
  if constexpr (V == 8)
    if (p.ve == 4) return launch_form<T, 4, 4, true>(a, p, backward, st);
  return launch_form<T, 2, 2, true>(a, p, backward, st);
}

int launch_norm_typed(int32_t dtype, const NormArgs& a, const NormPlan& p, bool backward,
                      hipStream_t st) {
  if (dtype == NSC_T_BF16) return launch_type<__bf16>(a, p, backward, st);
  if (dtype == NSC_T_F16) return launch_type<_Float16>(a, p, backward, st);
  return launch_type<float>(a, p, backward, st);
}

int check_call(const nsc_norm_desc* d, int64_t max_count, const void* ws, size_t ws_bytes,
               bool backward) {
  if (int rc = check_norm(d)) return rc;
  NSC_REQUIRE_L(max_count >= 0 && max_count <= kMaxImages, NSC_E_INVAL,
                "max_count %lld out of range", (long long)max_count);
  const size_t need = norm_call_bytes(*d, max_count, backward);
  NSC_REQUIRE_L(need == 0 || (ws != nullptr && (uintptr_t)ws % 256 == 0 && ws_bytes >= need),
                NSC_E_WORKSPACE, "workspace needs %zu bytes (256-byte aligned), got %zu", need,
                ws_bytes);
  return NSC_OK;
}

bool misaligned(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }

}  // namespace
}  // namespace nsc

using namespace nsc;

extern "C" {

int nsc_norm_check(const nsc_norm_desc* desc) {
  fail(NSC_OK, "%s", "");
  return check_norm(desc);
}

int nsc_group_norm_workspace_bytes(const nsc_norm_desc* desc, int64_t max_count, int32_t backward,
                                   size_t* bytes) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_norm(desc)) return rc;
  NSC_REQUIRE_L(bytes != nullptr && max_count >= 0 && max_count <= kMaxImages &&
                    (backward == 0 || backward == 1),
                NSC_E_INVAL, "bad arguments");
  *bytes = norm_ws_bytes(*desc, max_count, backward != 0);
  return NSC_OK;
}

int nsc_group_norm(const nsc_norm_desc* desc, const void* x, const float* gamma, const float* beta,
                   const int32_t* count, int64_t max_count, void* y, float* stats, void* ws,
                   size_t ws_bytes, void* stream) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_call(desc, max_count, ws, ws_bytes, false)) return rc;
  if (max_count == 0) return NSC_OK;
  NSC_REQUIRE_L(x && gamma && beta && y, NSC_E_INVAL, "x, gamma, beta or y is NULL");
  const int64_t es = type_bytes(desc->dtype);
  NSC_REQUIRE_L(!misaligned(x, es) && !misaligned(y, es) && !misaligned(gamma, 4) &&
                    !misaligned(beta, 4) && !misaligned(stats, 8) && !misaligned(count, 4),
                NSC_E_INVAL, "a pointer is not aligned to its elements (stats to pairs)");
  NSC_REQUIRE_L(x != y || desc->x_stride == desc->y_stride, NSC_E_INVAL,
                "y may be x only with equal strides");
  const NormPlan p = plan_norm(*desc, (uintptr_t)x | (uintptr_t)y, max_count, false);
  NormArgs a = norm_args(*desc, p, count, max_count);
  a.x = x;
  a.out = y;
  a.gamma = gamma;
  a.beta = beta;
  a.stats = stats;
  a.part = static_cast<float*>(ws);
  return launch_norm_typed(desc->dtype, a, p, false, (hipStream_t)stream);
}

int nsc_group_norm_backward(const nsc_norm_desc* desc, const void* x, const void* dy,
                            const float* gamma, const float* beta, const float* stats,
                            const int32_t* count, int64_t max_count, void* dx, float* dgamma,
                            float* dbeta, void* ws, size_t ws_bytes, void* stream) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_call(desc, max_count, ws, ws_bytes, true)) return rc;
  NSC_REQUIRE_L(dgamma && dbeta, NSC_E_INVAL, "dgamma or dbeta is NULL");
  NSC_REQUIRE_L(max_count == 0 || (x && dy && gamma && beta && stats && dx), NSC_E_INVAL,
                "x, dy, gamma, beta, stats or dx is NULL");
  const int64_t es = type_bytes(desc->dtype);
  NSC_REQUIRE_L(!misaligned(x, es) && !misaligned(dy, es) && !misaligned(dx, es) &&
                    !misaligned(gamma, 4) && !misaligned(beta, 4) && !misaligned(stats, 8) &&
                    !misaligned(dgamma, 4) && !misaligned(dbeta, 4) && !misaligned(count, 4),
                NSC_E_INVAL, "a pointer is not aligned to its elements (stats to pairs)");
  const hipStream_t st = (hipStream_t)stream;
  int32_t parts = 1;
  if (max_count > 0) {
    const NormPlan p =
        plan_norm(*desc, (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx, max_count, true);
    parts = p.parts;
    NormArgs a = norm_args(*desc, p, count, max_count);
    a.x = x;
    a.dy = dy;
    a.out = dx;
    a.gamma = gamma;
    a.beta = beta;
    a.stats = const_cast<float*>(stats);
    a.part = static_cast<float*>(ws);
    if (int rc = launch_norm_typed(desc->dtype, a, p, true, st)) return rc;
  }
  hipLaunchKernelGGL(k_norm_grad_params, dim3((unsigned)desc->c), dim3(256), 0, st,
                     static_cast<const float*>(ws), max_count ? count : nullptr, max_count, parts,
                     desc->c, dgamma, dbeta);
  NSC_CHECK_LAUNCH("k_norm_grad_params");
  return NSC_OK;
}

}  // extern "C"
