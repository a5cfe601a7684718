// Group normalisation of channels-last maps with an activation, and its
// gradients (nsc_group_norm, nsc_group_norm_backward).
//
// A work item is one image's block of whole groups (a run of channels of every
// pixel).  Its threads are dealt over the block's vectors of VE channels first
// and over pixels second, so that every thread keeps the same channels for all
// its pixels: their parameters and sums stay in registers, and consecutive
// lanes read consecutive memory.
//
// Statistics: each thread takes the mean and the sum of squared deviations
// from it (M2) of a chunk of pixels it holds in registers, and chunks, threads
// and parts are joined by
//   mean = (na ma + nb mb) / n,  M2 = M2a + M2b + (mb - ma)^2 na nb / n,
// so that no sum of squares ever cancels against the square of a mean; all of
// it in fp32.
#include "layer_types.h"

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
  float* part;              // workspace (see the kernels)
  const int32_t* count;     // nullable
  int64_t max_count;
  int64_t x_stride, y_stride;
  int32_t hw, c, cpg, groups;
  int32_t cb;               // channels of a block
  int32_t gpb;              // groups of a block
  int32_t blocks;           // blocks of an image
  int32_t cv;               // vectors of a block's pixel
  int32_t pl;               // pixels the threads cover at once
  float eps;
  int32_t act;
};

__device__ __forceinline__ int64_t live_count(const NormArgs& a) {
  int64_t n = a.count ? *a.count : a.max_count;
  return n < a.max_count ? n : a.max_count;
}

__device__ __forceinline__ float activate(float z, int act) {
  if (act == NSC_ACT_RELU) return z < 0.0f ? 0.0f : z;
  if (act == NSC_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  return z;
}

// (na, ma, qa) joined with (nb, mb, qb), nb > 0.
__device__ __forceinline__ void join(float& na, float& ma, float& qa, float nb, float mb,
                                     float qb) {
  const float n = na + nb, f = nb / n, d = mb - ma;
  ma += d * f;
  qa += qb + d * d * na * f;
  na = n;
}

constexpr int kNormChunk = 8;  // pixels of a thread in flight together

// Each group's statistics of an item from its threads' (mean, M2): K = 1, of
// all the channels a thread holds (they lie in one group); K = VE, of each of
// them.  A wave takes a group at a time.  sm: 2 * K * blockDim floats, the
// results (mean, rstd) in gs[group of the block].
template <int VE, int K>
__device__ __forceinline__ void reduce_groups(const NormArgs& a, const float (&m)[K],
                                              const float (&q)[K], float* sm, float2* gs) {
  const int T = blockDim.x, lane = threadIdx.x & 63, waves = T >> 6;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    sm[(2 * k) * T + threadIdx.x] = m[k];
    sm[(2 * k + 1) * T + threadIdx.x] = q[k];
  }
  __syncthreads();
  const int per = K == 1 ? a.cpg / VE : a.cpg;  // a group's entries per pixel lane
  const int entries = a.pl * per;
  const float total = (float)a.hw * (float)a.cpg;
  for (int g = threadIdx.x >> 6; g < a.gpb; g += waves) {
    float sum = 0.0f;
    for (int i = lane; i < entries; i += 64) {
      const int p = i / per, j = g * per + (i - p * per);
      const int t = K == 1 ? p * a.cv + j : p * a.cv + j / VE;
      const int k = K == 1 ? 0 : j % VE;
      const int px = p < a.hw ? (a.hw - p + a.pl - 1) / a.pl : 0;  // pixels of the thread
      sum += sm[(2 * k) * T + t] * (float)(px * (K == 1 ? VE : 1));
    }
    const float mean = wave_sum(sum) / total;
    float dev = 0.0f;
    for (int i = lane; i < entries; i += 64) {
      const int p = i / per, j = g * per + (i - p * per);
      const int t = K == 1 ? p * a.cv + j : p * a.cv + j / VE;
      const int k = K == 1 ? 0 : j % VE;
      const int px = p < a.hw ? (a.hw - p + a.pl - 1) / a.pl : 0;
      const float d = sm[(2 * k) * T + t] - mean;
      if (px) dev += sm[(2 * k + 1) * T + t] + d * d * (float)(px * (K == 1 ? VE : 1));
    }
    const float var = wave_sum(dev) / total;
    if (lane == 0) gs[g] = make_float2(mean, 1.0f / sqrtf(var + a.eps));
  }
  __syncthreads();
}

template <typename T, int VE, int K>
__global__ void __launch_bounds__(1024) k_norm(NormArgs a) {
  extern __shared__ __align__(16) float sm[];
  float2* gs = reinterpret_cast<float2*>(sm + 2 * K * blockDim.x);
  const int64_t items = live_count(a) * a.blocks;
  const int p0 = threadIdx.x / a.cv, v = threadIdx.x - p0 * a.cv;
  const bool on = p0 < a.pl;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t img = item / a.blocks;
    const int blk = (int)(item - img * a.blocks);
    const int ch = blk * a.cb + v * VE;
    const T* x = static_cast<const T*>(a.x) + img * a.x_stride + ch;
    T* y = static_cast<T*>(a.out) + img * a.y_stride + ch;
    float m[K], q[K];
#pragma unroll
    for (int k = 0; k < K; ++k) m[k] = q[k] = 0.0f;
    float n = 0.0f;
    for (int p = on ? p0 : a.hw; p < a.hw; p += a.pl * kNormChunk) {
      float f[kNormChunk][VE];
      int cnt = 0;
#pragma unroll
      for (int u = 0; u < kNormChunk; ++u) {
        const int pu = p + u * a.pl;
        if (pu < a.hw) {
          to_f32(*reinterpret_cast<const Vec<T, VE>*>(x + (int64_t)pu * a.c), f[u]);
          ++cnt;
        }
      }
      const float nb = (float)(cnt * (K == 1 ? VE : 1)), na = n;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float s = 0.0f, d2 = 0.0f;
#pragma unroll
        for (int u = 0; u < kNormChunk; ++u)
          if (u < cnt) {
            if constexpr (K == 1) {
#pragma unroll
              for (int e = 0; e < VE; ++e) s += f[u][e];
            } else {
              s += f[u][k];
            }
          }
        const float mb = s / nb;
#pragma unroll
        for (int u = 0; u < kNormChunk; ++u)
          if (u < cnt) {
            if constexpr (K == 1) {
#pragma unroll
              for (int e = 0; e < VE; ++e) d2 += (f[u][e] - mb) * (f[u][e] - mb);
            } else {
              d2 += (f[u][k] - mb) * (f[u][k] - mb);
            }
          }
        n = na;
        join(n, m[k], q[k], nb, mb, d2);
      }
    }
    reduce_groups<VE, K>(a, m, q, sm, gs);
    if (a.stats)
      for (int g = threadIdx.x; g < a.gpb; g += blockDim.x)
        reinterpret_cast<float2*>(a.stats)[img * a.groups + blk * a.gpb + g] = gs[g];
    if (on) {
      float mu[VE], s[VE], b[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float2 st = gs[(v * VE + e) / a.cpg];
        mu[e] = st.x;
        s[e] = a.gamma[ch + e] * st.y;
        b[e] = a.beta[ch + e];
      }
      for (int p = p0; p < a.hw; p += a.pl) {
        float f[VE];
        to_f32(*reinterpret_cast<const Vec<T, VE>*>(x + (int64_t)p * a.c), f);
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = activate(fmaf(f[e] - mu[e], s[e], b[e]), a.act);
        *reinterpret_cast<Vec<T, VE>*>(y + (int64_t)p * a.c) = from_f32<T, VE>(f);
      }
    }
    __syncthreads();  // gs and sm are read before the next item writes them
  }
}

// ---------------------------------------------------------------- backward

// act'(z) of z = (x - mean) rstd gamma + beta for xm = x - mean and
// s = gamma rstd.  The ReLU's sign is that of the exact value: fp32's z is
// within 2^-22 |xm s| of it, and values closer to zero are taken again in
// fp64.
__device__ __forceinline__ float slope(float xm, float s, float beta, int act, float x, float mean,
                                       float rstd, const float* gamma) {
  if (act == NSC_ACT_NONE) return 1.0f;
  const float p = xm * s, z = p + beta;
  if (act == NSC_ACT_RELU) {
    if (fabsf(z) <= 5e-7f * fabsf(p) + 1e-37f)
      return ((double)x - (double)mean) * (double)rstd * (double)*gamma + (double)beta > 0.0 ? 1.0f
                                                                                           : 0.0f;
    return z > 0.0f ? 1.0f : 0.0f;
  }
  const float t = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  return t * (1.0f + z * (1.0f - t));
}

template <typename T, int VE>
__global__ void __launch_bounds__(1024) k_norm_grad(NormArgs a) {
  extern __shared__ __align__(16) float sm[];  // [2 VE][blockDim], then [cb][2]
  const int Tn = blockDim.x;
  float* chs = sm + 2 * VE * Tn;
  const int64_t items = live_count(a) * a.blocks;
  const int p0 = threadIdx.x / a.cv, v = threadIdx.x - p0 * a.cv;
  const bool on = p0 < a.pl;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t img = item / a.blocks;
    const int blk = (int)(item - img * a.blocks);
    const int ch = blk * a.cb + v * VE;
    const T* x = static_cast<const T*>(a.x) + img * a.x_stride + ch;
    const T* dy = static_cast<const T*>(a.dy) + img * a.y_stride + ch;
    T* dx = static_cast<T*>(a.out) + img * a.x_stride + ch;
    const float2* stats = reinterpret_cast<const float2*>(a.stats) + img * a.groups + blk * a.gpb;
    float mu[VE], rs[VE], s[VE], b[VE], s1[VE], s2[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float2 st = on ? stats[(v * VE + e) / a.cpg] : make_float2(0.f, 0.f);
      mu[e] = st.x;
      rs[e] = st.y;
      s[e] = on ? a.gamma[ch + e] * st.y : 0.0f;
      b[e] = on ? a.beta[ch + e] : 0.0f;
      s1[e] = s2[e] = 0.0f;
    }
    for (int p = on ? p0 : a.hw; p < a.hw; p += a.pl) {
      float f[VE], g[VE];
      to_f32(*reinterpret_cast<const Vec<T, VE>*>(x + (int64_t)p * a.c), f);
      to_f32(*reinterpret_cast<const Vec<T, VE>*>(dy + (int64_t)p * a.c), g);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float xm = f[e] - mu[e];
        const float dz = g[e] * slope(xm, s[e], b[e], a.act, f[e], mu[e], rs[e], a.gamma + ch + e);
        s1[e] += dz;
        s2[e] += dz * (xm * rs[e]);
      }
    }
    // the channels' sums: a channel's pixel lanes in a fixed order
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      sm[(2 * e) * Tn + threadIdx.x] = s1[e];
      sm[(2 * e + 1) * Tn + threadIdx.x] = s2[e];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * a.cb; j += Tn) {
      const int c = j >> 1, e = c % VE, w = c / VE;
      float t = 0.0f;
      for (int p = 0; p < a.pl; ++p) t += sm[(2 * e + (j & 1)) * Tn + p * a.cv + w];
      chs[j] = t;
      a.part[((img * a.c) + blk * a.cb) * 2 + j] = t;
    }
    __syncthreads();
    // the groups' means of gamma dz and gamma dz xh, where a thread needs them
    if (on) {
      const float inv = 1.0f / ((float)a.hw * (float)a.cpg);
      float m1[VE], m2[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int g = (v * VE + e) / a.cpg;
        float t1 = 0.0f, t2 = 0.0f;
        for (int k = 0; k < a.cpg; ++k) {
          const float ga = a.gamma[blk * a.cb + g * a.cpg + k];
          t1 += ga * chs[2 * (g * a.cpg + k)];
          t2 += ga * chs[2 * (g * a.cpg + k) + 1];
        }
        m1[e] = t1 * inv;
        m2[e] = t2 * inv;
      }
      for (int p = p0; p < a.hw; p += a.pl) {
        float f[VE], g[VE];
        to_f32(*reinterpret_cast<const Vec<T, VE>*>(x + (int64_t)p * a.c), f);
        to_f32(*reinterpret_cast<const Vec<T, VE>*>(dy + (int64_t)p * a.c), g);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float xm = f[e] - mu[e];
          const float dz =
              g[e] * slope(xm, s[e], b[e], a.act, f[e], mu[e], rs[e], a.gamma + ch + e);
          f[e] = s[e] * dz - rs[e] * (m1[e] + xm * rs[e] * m2[e]);
        }
        *reinterpret_cast<Vec<T, VE>*>(dx + (int64_t)p * a.c) = from_f32<T, VE>(f);
      }
    }
    __syncthreads();  // chs and sm are read before the next item writes them
  }
}

// dgamma and dbeta: a workgroup per channel adds the images' sums, each thread
// its images in order, then the threads' in a tree, in fp64.
__global__ void __launch_bounds__(256) k_norm_grad_params(const float* part, const int32_t* count,
                                                          int64_t max_count, int32_t c,
                                                          float* dgamma, float* dbeta) {
  __shared__ double red[2][256];
  int64_t n = count ? *count : max_count;
  if (n > max_count) n = max_count;
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

struct NormPlan {
  int32_t ve, cb, gpb, blocks, cv, pl, threads;
};

// Vectors of 16 bytes where every image, pixel and block starts at one, else
// single elements.  A block is the fewest whole groups that make 128 bytes of
// a pixel (a cache line per read).
NormPlan plan_norm(const nsc_norm_desc& d, uintptr_t ptrs) {
  NormPlan p{};
  const int32_t es = (int32_t)type_bytes(d.dtype), cpg = d.c / d.groups;
  p.ve = 16 / es;
  const bool aligned = ptrs % 16 == 0 && d.c % p.ve == 0 && d.x_stride % p.ve == 0 &&
                       d.y_stride % p.ve == 0;
  if (!aligned) p.ve = 1;
  p.gpb = 0;
  for (int32_t g = 1; g <= d.groups; ++g) {
    if (d.groups % g || (g * cpg) % p.ve) continue;
    p.gpb = g;
    if (g * cpg * es >= 128) break;
  }
  if (p.gpb * cpg / p.ve > 1024) {  // no such block of at most 1024 vectors: elements
    p.ve = 1;
    p.gpb = 1;
  }
  p.cb = p.gpb * cpg;
  p.blocks = d.groups / p.gpb;
  p.cv = p.cb / p.ve;
  const int64_t vecs = (int64_t)d.h * d.w * p.cv;
  p.threads = vecs <= 1024 && p.cv <= 256 ? 256 : 1024;
  p.pl = p.threads / p.cv;
  return p;
}

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
  a.eps = d.eps;
  a.act = d.act;
  return a;
}

template <typename T>
int launch_norm(const NormArgs& a, const NormPlan& p, bool backward, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  int64_t grid = a.max_count * p.blocks;
  if (grid > 64 * kNumCU) grid = 64 * kNumCU;
  const dim3 g((unsigned)grid), b((unsigned)p.threads);
  if (backward) {
    const size_t lds = (size_t)(2 * p.ve * p.threads + 2 * p.cb) * 4;
    if (p.ve == V)
      hipLaunchKernelGGL((k_norm_grad<T, V>), g, b, lds, st, a);
    else
      hipLaunchKernelGGL((k_norm_grad<T, 1>), g, b, lds, st, a);
    NSC_CHECK_LAUNCH("k_norm_grad");
    return NSC_OK;
  }
  const bool whole = a.cpg % p.ve == 0;  // a vector's channels lie in one group
  const size_t lds = (size_t)(2 * (whole ? 1 : p.ve) * p.threads + 2 * p.gpb) * 4;
  if (p.ve != V)
    hipLaunchKernelGGL((k_norm<T, 1, 1>), g, b, lds, st, a);
  else if (whole)
    hipLaunchKernelGGL((k_norm<T, V, 1>), g, b, lds, st, a);
  else
    hipLaunchKernelGGL((k_norm<T, V, V>), g, b, lds, st, a);
  NSC_CHECK_LAUNCH("k_norm");
  return NSC_OK;
}

int launch_norm_typed(int32_t dtype, const NormArgs& a, const NormPlan& p, bool backward,
                      hipStream_t st) {
  if (dtype == NSC_T_BF16) return launch_norm<__bf16>(a, p, backward, st);
  if (dtype == NSC_T_F16) return launch_norm<_Float16>(a, p, backward, st);
  return launch_norm<float>(a, p, backward, st);
}

size_t norm_ws_bytes(const nsc_norm_desc& d, int64_t max_count, bool backward) {
  return backward ? (size_t)max_count * d.c * 8 : 0;
}

int check_call(const nsc_norm_desc* d, int64_t max_count, const void* ws, size_t ws_bytes,
               bool backward) {
  if (int rc = check_norm(d)) return rc;
  NSC_REQUIRE_L(max_count >= 0 && max_count <= kMaxImages, NSC_E_INVAL, "max_count %lld out of range",
                (long long)max_count);
  const size_t need = norm_ws_bytes(*d, max_count, backward);
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
  const NormPlan p = plan_norm(*desc, (uintptr_t)x | (uintptr_t)y);
  NormArgs a = norm_args(*desc, p, count, max_count);
  a.x = x;
  a.out = y;
  a.gamma = gamma;
  a.beta = beta;
  a.stats = stats;
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
  if (max_count > 0) {
    const NormPlan p = plan_norm(*desc, (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx);
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
                     static_cast<const float*>(ws), max_count ? count : nullptr, max_count, desc->c,
                     dgamma, dbeta);
  NSC_CHECK_LAUNCH("k_norm_grad_params");
  return NSC_OK;
}

}  // extern "C"
