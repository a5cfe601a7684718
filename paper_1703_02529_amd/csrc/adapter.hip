// A projection that all rows share, each row with the low-rank adapter of its
// camera or request beside it, and its gradients (nsc_adapter_project,
// nsc_adapter_backward).
//
// The rank-wide rows t = scale x a^T (and u = scale dy b) are taken first, in
// fp32.  The shared product runs on 16x16 MFMA tiles with the weights as the
// first operand, so that a lane holds four neighbouring outputs of one row;
// its epilogue adds t b^T with the fp32 MFMA, adapter by adapter among the
// tile's rows: an adapter's products are taken for all 16 rows and kept for
// its own, so that no row's result depends on its neighbours.
//
// The gradients of the adapters are sums over an adapter's rows, which a list
// of the rows by adapter gives in ascending order.
#include "layer_types.h"

#include <limits.h>

namespace nsc {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A fragment is 16 bytes of a row's consecutive values per lane: lane (m, g)
// holds row m's values E g .. E g + E - 1 of a step of KS.  (The fp32 step is
// four MFMAs; which of a step's values meet in which is the same on both
// sides.)
template <typename T> struct Mma;
template <> struct Mma<__bf16> {
  static constexpr int E = 8, KS = 32;
  static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<_Float16> {
  static constexpr int E = 8, KS = 32;
  static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
__device__ __forceinline__ f32x4 mma_f32(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
template <> struct Mma<float> {
  static constexpr int E = 4, KS = 16;
  static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
    return mma_f32(__builtin_bit_cast(f32x4, a), __builtin_bit_cast(f32x4, b), c);
  }
};

// 16 bytes of values from p, of which `left` (any sign) are inside the row;
// zeros behind them.  VEC: p is 16-byte aligned and left a multiple of E.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load_frag(const T* p, int left) {
  constexpr int E = 16 / sizeof(T);
  if constexpr (VEC) {
    return left > 0 ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
  } else {
    Vec<T, E> v;
#pragma unroll
    for (int e = 0; e < E; ++e) v.e[e] = e < left ? p[e] : (T)0.0f;
    return __builtin_bit_cast(uint4, v);
  }
}
// Four values as fp32, of which `left` are inside.
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, int left) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < left ? (float)p[e] : 0.0f;
  return v;
}

struct AdapterArgs {
  const void* x;            // rows of the reduction's input (x, or dy)
  const void* w;            // [d][k]
  const float* bias;
  const void* a;            // [n_adapters][rank][k]
  const void* b;            // [n_adapters][d][rank]
  const float* scale;
  const int32_t* ids;
  const int32_t* count;     // nullable
  int64_t max_rows;
  int64_t in_stride, out_stride;
  void* out;
  float* t;                 // [rows][rp] rank-wide rows
  int32_t k, d, rank, rp, n_adapters;
};

__device__ __forceinline__ int64_t live_rows(const AdapterArgs& a) {
  int64_t n = a.count ? *a.count : a.max_rows;
  return n < a.max_rows ? n : a.max_rows;
}
// The adapter of row r, INT_MAX without one.
__device__ __forceinline__ int row_adapter(const AdapterArgs& a, int64_t r, int64_t n) {
  if (r >= n) return INT_MAX;
  const int p = a.ids[r];
  return p >= 0 && p < a.n_adapters ? p : INT_MAX;
}
// The smallest adapter above p among a wave's lanes (INT_MAX: none).
__device__ __forceinline__ int next_adapter(int mine, int p) {
  int v = mine > p ? mine : INT_MAX;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = min(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// Rank-wide rows: a workgroup per 16 rows, whose waves split the reduction and
// add their sums through LDS.  B = false: t = scale x a^T over k; B = true:
// u = scale dy b over d, whose values lie rank apart.
constexpr int kDownWaves = 8;

template <typename T, bool VEC, bool B>
__global__ void __launch_bounds__(64 * kDownWaves) k_adapter_down(AdapterArgs a) {
  using M = Mma<T>;
  __shared__ f32x4 red[kDownWaves][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int64_t n = live_rows(a);
  const int len = B ? a.d : a.k;
  for (int64_t row0 = blockIdx.x * 16ll; row0 < n; row0 += gridDim.x * 16ll) {
    const int64_t row = row0 + m < n ? row0 + m : n - 1;
    const int mine = row_adapter(a, row0 + m, n);
    const T* x = static_cast<const T*>(a.x) + row * a.in_stride;
    for (int j0 = 0; j0 < a.rp; j0 += 16) {
      f32x4 out = {0.f, 0.f, 0.f, 0.f};
      const int j = j0 + m;
      for (int p = next_adapter(mine, -1); p != INT_MAX; p = next_adapter(mine, p)) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        if constexpr (B) {
          const T* b = static_cast<const T*>(a.b) + (int64_t)p * a.d * a.rank + j;
          for (int k0 = wave * 16; k0 < len; k0 += 16 * kDownWaves) {
            const int k = k0 + 4 * g;
            f32x4 bv;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              bv[e] = j < a.rank && k + e < len ? (float)b[(int64_t)(k + e) * a.rank] : 0.0f;
            acc = mma_f32(bv, load4(x + k, len - k), acc);
          }
        } else {
          const T* ar = static_cast<const T*>(a.a) + ((int64_t)p * a.rank + j) * a.k;
          for (int k0 = wave * M::KS; k0 < len; k0 += M::KS * kDownWaves) {
            const int k = k0 + M::E * g;
            const uint4 av = load_frag<T, VEC>(ar + k, j < a.rank ? len - k : 0);
            acc = M::mma(av, load_frag<T, VEC>(x + k, len - k), acc);
          }
        }
        __syncthreads();  // red is read before it is written again
        red[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int w = 1; w < kDownWaves; ++w) acc += red[w][lane];
          if (mine == p) out = acc * a.scale[p];
        }
      }
      if (wave == 0 && row0 + m < n)
        *reinterpret_cast<f32x4*>(a.t + row * a.rp + j0 + 4 * g) = out;
    }
  }
}

// The shared product with the rank-wide rows' in its epilogue: 64 x 64 tiles
// of (outputs, rows), 128 bytes of the reduction at a time through LDS, whose
// 16-byte chunks c of row r lie at chunk c ^ (r & 7).  TR = false: outputs d
// from x w^T + t b^T; TR = true: outputs k from dy w + u a, the weights
// transposed on their way into LDS.
constexpr int kTile = 64;

template <typename T, bool VEC, bool TR>
__global__ void __launch_bounds__(256) k_adapter_gemm(AdapterArgs a) {
  using M = Mma<T>;
  constexpr int E = M::E, BK = 2 * M::KS;  // values per 128 bytes
  __shared__ uint4 wl[kTile][8], xl[kTile][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  const int64_t n = live_rows(a);
  const int outs = TR ? a.k : a.d, len = TR ? a.d : a.k;
  const int o0 = blockIdx.x * kTile, wo = (wave & 1) * 32, wr = (wave >> 1) * 32;
  const T* w = static_cast<const T*>(a.w);
  const T* xs = static_cast<const T*>(a.x);
  for (int64_t r0 = blockIdx.y * (int64_t)kTile; r0 < n; r0 += gridDim.y * (int64_t)kTile) {
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < len; k0 += BK) {
      __syncthreads();
      for (int c = threadIdx.x; c < kTile * 8; c += 256) {
        const int r = c >> 3, ch = c & 7, k = k0 + ch * E;
        const int64_t row = r0 + r < n ? r0 + r : n - 1;
        xl[r][ch ^ (r & 7)] = load_frag<T, VEC>(xs + row * a.in_stride + k, len - k);
        if constexpr (!TR) {
          const int o = o0 + r < outs ? o0 + r : outs - 1;
          wl[r][ch ^ (r & 7)] = load_frag<T, VEC>(w + (int64_t)o * a.k + k, len - k);
        }
      }
      if constexpr (TR) {
        for (int c = threadIdx.x; c < kTile * BK; c += 256) {
          const int o = c % kTile, k = c / kTile;  // lanes along the outputs
          const bool in = o0 + o < outs && k0 + k < len;
          reinterpret_cast<T*>(&wl[o][(k / E) ^ (o & 7)])[k % E] =
              in ? w[(int64_t)(k0 + k) * a.k + o0 + o] : (T)0.0f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint4 av[2], bv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int ro = wo + i * 16 + m, rr = wr + i * 16 + m;
          av[i] = wl[ro][(4 * s + g) ^ (ro & 7)];
          bv[i] = xl[rr][(4 * s + g) ^ (rr & 7)];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = M::mma(av[i], bv[j], acc[i][j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {  // 16 rows
      const int64_t row = r0 + wr + j * 16 + m;
      const int mine = row_adapter(a, row, n);
      for (int p = next_adapter(mine, -1); p != INT_MAX; p = next_adapter(mine, p)) {
        f32x4 add[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) add[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q0 = 0; q0 < a.rp; q0 += 16) {
          const int q = q0 + 4 * g;
          f32x4 tv = {0.f, 0.f, 0.f, 0.f};
          if (mine == p) tv = *reinterpret_cast<const f32x4*>(a.t + row * a.rp + q);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int o = o0 + wo + i * 16 + m;
            f32x4 bv = {0.f, 0.f, 0.f, 0.f};
            if (o < outs) {
              if constexpr (TR) {
                const T* ap = static_cast<const T*>(a.a) + (int64_t)p * a.rank * a.k + o;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (q + e < a.rank) bv[e] = (float)ap[(int64_t)(q + e) * a.k];
              } else {
                bv = load4(static_cast<const T*>(a.b) + ((int64_t)p * a.d + o) * a.rank + q,
                           a.rank - q);
              }
            }
            add[i] = mma_f32(bv, tv, add[i]);
          }
        }
        if (mine == p) {
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[i][j] += add[i];
        }
      }
      if (row < n) {
        T* y = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int o = o0 + wo + i * 16 + 4 * g;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (o + e < outs)
              y[o + e] = (T)(acc[i][j][e] + (a.bias ? a.bias[o + e] : 0.0f));
        }
      }
    }
  }
}

// The rows of each adapter in ascending order: rows[off[p] .. off[p + 1]).  A
// workgroup per adapter counts the rows of smaller adapters and its own, then
// writes its own.  Waves take consecutive ranges of the rows.
constexpr int kListWaves = 16;

__global__ void __launch_bounds__(64 * kListWaves) k_adapter_list(AdapterArgs a, int32_t* off,
                                                                  int32_t* rows) {
  __shared__ int32_t less[kListWaves], same[kListWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = live_rows(a);
  const int64_t per = (n + kListWaves * 64 - 1) / (kListWaves * 64) * 64;
  const int64_t b = wave * per < n ? wave * per : n, e = b + per < n ? b + per : n;
  for (int p = blockIdx.x; p < a.n_adapters; p += gridDim.x) {
    int32_t lo = 0, eq = 0;
    for (int64_t r = b; r < e; r += 64) {
      const int mine = r + lane < e ? a.ids[r + lane] : -1;
      lo += __popcll(__ballot(mine >= 0 && mine < p));
      eq += __popcll(__ballot(mine == p));
    }
    __syncthreads();
    if (lane == 0) {
      less[wave] = lo;
      same[wave] = eq;
    }
    __syncthreads();
    int32_t first = 0, at = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kListWaves; ++w) {
      first += less[w];
      at += w < wave ? same[w] : 0;
      all += same[w];
    }
    if (threadIdx.x == 0) {
      off[p] = first;
      if (p == a.n_adapters - 1) off[a.n_adapters] = first + all;
    }
    at += first;
    for (int64_t r = b; r < e; r += 64) {
      const bool mine = r + lane < e && a.ids[r + lane] == p;
      const uint64_t mask = __ballot(mine);
      if (mine) rows[at + __popcll(mask & ((1ull << lane) - 1))] = (int32_t)(r + lane);
      at += __popcll(mask);
    }
  }
}

// A gradient of the adapters: a workgroup takes 64 columns of the rows of one
// adapter, its waves every eighth step of 16 rows, 16 of the rank at a time.
// B = false: da[p][j][c] = sum u[r][j] x[r][c]; B = true: db[p][c][j] = sum
// t[r][j] dy[r][c].
constexpr int kGradWaves = 8;

struct GradArgs {
  const float* t;           // u, or t
  const void* v;            // x, or dy
  int64_t v_stride;
  const int32_t* off;
  const int32_t* rows;
  float* out;
  int32_t cols, rank, rp, n_adapters;
};

template <typename T, bool B>
__global__ void __launch_bounds__(64 * kGradWaves) k_adapter_grad(GradArgs a) {
  __shared__ f32x4 red[kGradWaves][4][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int c0 = blockIdx.x * 64, c = c0 + 4 * m;  // a lane's four columns
  for (int p = blockIdx.y; p < a.n_adapters; p += gridDim.y) {
    const int32_t b = a.off[p], e = a.off[p + 1];
    for (int j0 = 0; j0 < a.rp; j0 += 16) {
      f32x4 acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int32_t r = b + wave * 16; r < e; r += 16 * kGradWaves) {
        f32x4 uv, xv[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int32_t at = r + 4 * g + s;
          const bool in = at < e;
          const int64_t row = in ? a.rows[at] : 0;
          uv[s] = in ? a.t[row * a.rp + j0 + m] : 0.0f;
          const f32x4 v = load4(static_cast<const T*>(a.v) + row * a.v_stride + c,
                                in ? a.cols - c : 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) xv[i][s] = v[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma_f32(uv, xv[i], acc[i]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][i][lane] = acc[i];
      __syncthreads();
      // wave i adds column i of the lanes' four: rank values j0 + 4 g .. + 3
      if (wave < 4 && c + wave < a.cols) {
        f32x4 s = red[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kGradWaves; ++w) s += red[w][wave][lane];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int j = j0 + 4 * g + q;
          if (j < a.rank)
            a.out[B ? ((int64_t)p * a.cols + c + wave) * a.rank + j
                    : ((int64_t)p * a.rank + j) * a.cols + c + wave] = s[q];
        }
      }
      __syncthreads();
    }
  }
}

// -------------------------------------------------------------------- host

constexpr int64_t kMaxRows = 0x7FFFFFFF;

int check_adapter(const nsc_adapter_desc* d) {
  NSC_REQUIRE_L(d != nullptr, NSC_E_INVAL, "adapter description is NULL");
  NSC_REQUIRE_L(d->k >= 1 && d->k <= (1 << 24) && d->d >= 1 && d->d <= (1 << 24), NSC_E_SHAPE,
                "projection of %d inputs onto %d outputs outside 1 .. 2^24", d->k, d->d);
  NSC_REQUIRE_L(d->rank >= 1 && d->rank <= NSC_MAX_RANK, NSC_E_SHAPE, "rank %d outside 1..%d",
                d->rank, NSC_MAX_RANK);
  NSC_REQUIRE_L(d->n_adapters >= 1 && d->n_adapters <= NSC_MAX_ADAPTERS, NSC_E_INVAL,
                "n_adapters %d outside 1..%d", d->n_adapters, NSC_MAX_ADAPTERS);
  NSC_REQUIRE_L(d->dtype >= NSC_T_F32 && d->dtype <= NSC_T_F16, NSC_E_DTYPE, "dtype %d is unknown",
                d->dtype);
  NSC_REQUIRE_L(d->x_stride >= d->k && d->y_stride >= d->d, NSC_E_INVAL,
                "row strides %lld, %lld are below one row (%d, %d elements)",
                (long long)d->x_stride, (long long)d->y_stride, d->k, d->d);
  NSC_REQUIRE_L(d->x_stride <= ((int64_t)1 << 31) && d->y_stride <= ((int64_t)1 << 31),
                NSC_E_INVAL, "row strides beyond 2^31 elements");
  return NSC_OK;
}

// Workspace: the rank-wide rows t (backward: and u), and backward the rows by
// adapter.
struct AdapterLayout {
  size_t t, u, off, rows, total;
};

AdapterLayout adapter_layout(const nsc_adapter_desc& d, int64_t max_rows, bool backward) {
  AdapterLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = align_up(o + bytes, 256);
    return at;
  };
  const size_t rp = align_up(d.rank, 16);
  L.t = take((size_t)max_rows * rp * 4);
  if (backward) {
    L.u = take((size_t)max_rows * rp * 4);
    L.off = take(((size_t)d.n_adapters + 1) * 4);
    L.rows = take((size_t)max_rows * 4);
  }
  L.total = o;
  return L;
}

int check_adapter_call(const nsc_adapter_desc* d, int64_t max_rows, const void* ws,
                       size_t ws_bytes, bool backward) {
  if (int rc = check_adapter(d)) return rc;
  NSC_REQUIRE_L(max_rows >= 0 && max_rows <= kMaxRows, NSC_E_INVAL, "max_rows %lld out of range",
                (long long)max_rows);
  const size_t need = adapter_layout(*d, max_rows, backward).total;
  NSC_REQUIRE_L(need == 0 || (ws != nullptr && (uintptr_t)ws % 256 == 0 && ws_bytes >= need),
                NSC_E_WORKSPACE, "workspace needs %zu bytes (256-byte aligned), got %zu", need,
                ws_bytes);
  return NSC_OK;
}

bool misaligned(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }

template <typename T>
int launch_down(const AdapterArgs& a, bool vec, bool b, hipStream_t st) {
  int64_t grid = (a.max_rows + 15) / 16;
  if (grid > 16 * kNumCU) grid = 16 * kNumCU;
  const dim3 g((unsigned)grid), t(64 * kDownWaves);
  if (b)
    hipLaunchKernelGGL((k_adapter_down<T, false, true>), g, t, 0, st, a);
  else if (vec)
    hipLaunchKernelGGL((k_adapter_down<T, true, false>), g, t, 0, st, a);
  else
    hipLaunchKernelGGL((k_adapter_down<T, false, false>), g, t, 0, st, a);
  NSC_CHECK_LAUNCH("k_adapter_down");
  return NSC_OK;
}

template <typename T>
int launch_gemm(const AdapterArgs& a, bool vec, bool tr, hipStream_t st) {
  const int outs = tr ? a.k : a.d;
  int64_t gy = (a.max_rows + kTile - 1) / kTile;
  if (gy > 65535) gy = 65535;
  const dim3 g((unsigned)((outs + kTile - 1) / kTile), (unsigned)gy), t(256);
#define NSC_GEMM(V, TR) hipLaunchKernelGGL((k_adapter_gemm<T, V, TR>), g, t, 0, st, a)
  if (tr) {
    if (vec) NSC_GEMM(true, true);
    else NSC_GEMM(false, true);
  } else {
    if (vec) NSC_GEMM(true, false);
    else NSC_GEMM(false, false);
  }
#undef NSC_GEMM
  NSC_CHECK_LAUNCH("k_adapter_gemm");
  return NSC_OK;
}

template <typename T>
int launch_grad(const GradArgs& a, bool b, hipStream_t st) {
  const dim3 g((unsigned)((a.cols + 63) / 64), (unsigned)a.n_adapters), t(64 * kGradWaves);
  if (b)
    hipLaunchKernelGGL((k_adapter_grad<T, true>), g, t, 0, st, a);
  else
    hipLaunchKernelGGL((k_adapter_grad<T, false>), g, t, 0, st, a);
  NSC_CHECK_LAUNCH("k_adapter_grad");
  return NSC_OK;
}

AdapterArgs adapter_args(const nsc_adapter_desc& d, const void* w, const void* a, const void* b,
                         const float* scale, const int32_t* ids, const int32_t* count,
                         int64_t max_rows) {
  AdapterArgs g{};
  g.w = w;
  g.a = a;
  g.b = b;
  g.scale = scale;
  g.ids = ids;
  g.count = count;
  g.max_rows = max_rows;
  g.k = d.k;
  g.d = d.d;
  g.rank = d.rank;
  g.rp = (int32_t)align_up(d.rank, 16);
  g.n_adapters = d.n_adapters;
  return g;
}

template <typename T>
int project(AdapterArgs a, bool vec, hipStream_t st) {
  if (int rc = launch_down<T>(a, vec, false, st)) return rc;
  return launch_gemm<T>(a, vec, false, st);
}

template <typename T>
int backward(const nsc_adapter_desc& d, AdapterArgs a, const void* x, const void* dy, void* dx,
             float* da, float* db, float* t, float* u, int32_t* off, int32_t* rows, bool vec_x,
             bool vec_dy, hipStream_t st) {
  hipLaunchKernelGGL(k_adapter_list,
                     dim3((unsigned)(d.n_adapters < 8 * kNumCU ? d.n_adapters : 8 * kNumCU)),
                     dim3(64 * kListWaves), 0, st, a, off, rows);
  NSC_CHECK_LAUNCH("k_adapter_list");
  if (a.max_rows > 0) {
    a.x = x;
    a.in_stride = d.x_stride;
    a.t = t;
    if (int rc = launch_down<T>(a, vec_x, false, st)) return rc;
    a.x = dy;
    a.in_stride = d.y_stride;
    a.t = u;
    if (int rc = launch_down<T>(a, false, true, st)) return rc;
    if (dx) {
      a.out = dx;
      a.out_stride = d.x_stride;
      if (int rc = launch_gemm<T>(a, vec_dy, true, st)) return rc;
    }
  }
  GradArgs g{};
  g.off = off;
  g.rows = rows;
  g.rank = a.rank;
  g.rp = a.rp;
  g.n_adapters = d.n_adapters;
  g.t = u;
  g.v = x;
  g.v_stride = d.x_stride;
  g.cols = d.k;
  g.out = da;
  if (int rc = launch_grad<T>(g, false, st)) return rc;
  g.t = t;
  g.v = dy;
  g.v_stride = d.y_stride;
  g.cols = d.d;
  g.out = db;
  return launch_grad<T>(g, true, st);
}

}  // namespace
}  // namespace nsc

using namespace nsc;

extern "C" {

int nsc_adapter_check(const nsc_adapter_desc* desc) {
  fail(NSC_OK, "%s", "");
  return check_adapter(desc);
}

int nsc_adapter_workspace_bytes(const nsc_adapter_desc* desc, int64_t max_rows, int32_t backward,
                                size_t* bytes) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_adapter(desc)) return rc;
  NSC_REQUIRE_L(bytes != nullptr && max_rows >= 0 && max_rows <= kMaxRows &&
                    (backward == 0 || backward == 1),
                NSC_E_INVAL, "bad arguments");
  *bytes = adapter_layout(*desc, max_rows, backward != 0).total;
  return NSC_OK;
}

int nsc_adapter_project(const nsc_adapter_desc* desc, const void* x, const void* w,
                        const float* bias, const void* a, const void* b, const float* scale,
                        const int32_t* ids, const int32_t* count, int64_t max_rows, void* y,
                        void* ws, size_t ws_bytes, void* stream) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_adapter_call(desc, max_rows, ws, ws_bytes, false)) return rc;
  if (max_rows == 0) return NSC_OK;
  NSC_REQUIRE_L(x && w && a && b && scale && ids && y, NSC_E_INVAL,
                "x, w, a, b, scale, ids or y is NULL");
  const int64_t es = type_bytes(desc->dtype);
  NSC_REQUIRE_L(!misaligned(x, es) && !misaligned(w, es) && !misaligned(a, es) &&
                    !misaligned(b, es) && !misaligned(y, es) && !misaligned(bias, 4) &&
                    !misaligned(scale, 4) && !misaligned(ids, 4) && !misaligned(count, 4),
                NSC_E_INVAL, "a pointer is not aligned to its elements");
  AdapterArgs g = adapter_args(*desc, w, a, b, scale, ids, count, max_rows);
  g.x = x;
  g.bias = bias;
  g.in_stride = desc->x_stride;
  g.out = y;
  g.out_stride = desc->y_stride;
  g.t = static_cast<float*>(ws);
  const int64_t e = 16 / es;
  const bool vec = !misaligned(x, 16) && !misaligned(w, 16) && !misaligned(a, 16) &&
                   desc->k % e == 0 && desc->x_stride % e == 0;
  const hipStream_t st = (hipStream_t)stream;
  if (desc->dtype == NSC_T_BF16) return project<__bf16>(g, vec, st);
  if (desc->dtype == NSC_T_F16) return project<_Float16>(g, vec, st);
  return project<float>(g, vec, st);
}

int nsc_adapter_backward(const nsc_adapter_desc* desc, const void* x, const void* dy,
                         const void* w, const void* a, const void* b, const float* scale,
                         const int32_t* ids, const int32_t* count, int64_t max_rows, void* dx,
                         float* da, float* db, void* ws, size_t ws_bytes, void* stream) {
  fail(NSC_OK, "%s", "");
  if (int rc = check_adapter_call(desc, max_rows, ws, ws_bytes, true)) return rc;
  NSC_REQUIRE_L(da && db, NSC_E_INVAL, "da or db is NULL");
  NSC_REQUIRE_L(max_rows == 0 || (x && dy && w && a && b && scale && ids), NSC_E_INVAL,
                "x, dy, w, a, b, scale or ids is NULL");
  const int64_t es = type_bytes(desc->dtype);
  NSC_REQUIRE_L(!misaligned(x, es) && !misaligned(dy, es) && !misaligned(w, es) &&
                    !misaligned(a, es) && !misaligned(b, es) && !misaligned(dx, es) &&
                    !misaligned(scale, 4) && !misaligned(ids, 4) && !misaligned(count, 4) &&
                    !misaligned(da, 4) && !misaligned(db, 4),
                NSC_E_INVAL, "a pointer is not aligned to its elements");
  const AdapterArgs g =
      adapter_args(*desc, w, a, b, scale, ids, max_rows ? count : nullptr, max_rows);
  const AdapterLayout L = adapter_layout(*desc, max_rows, true);
  unsigned char* at = static_cast<unsigned char*>(ws);
  float* t = reinterpret_cast<float*>(at + L.t);
  float* u = reinterpret_cast<float*>(at + L.u);
  int32_t* off = reinterpret_cast<int32_t*>(at + L.off);
  int32_t* rows = reinterpret_cast<int32_t*>(at + L.rows);
  const int64_t e = 16 / es;
  const bool vec_x = !misaligned(x, 16) && !misaligned(a, 16) && desc->k % e == 0 &&
                     desc->x_stride % e == 0;
  const bool vec_dy = !misaligned(dy, 16) && desc->d % e == 0 && desc->y_stride % e == 0;
  const hipStream_t st = (hipStream_t)stream;
  if (desc->dtype == NSC_T_BF16)
    return backward<__bf16>(*desc, g, x, dy, dx, da, db, t, u, off, rows, vec_x, vec_dy, st);
  if (desc->dtype == NSC_T_F16)
    return backward<_Float16>(*desc, g, x, dy, dx, da, db, t, u, off, rows, vec_x, vec_dy, st);
  return backward<float>(*desc, g, x, dy, dx, da, db, t, u, off, rows, vec_x, vec_dy, st);
}

}  // extern "C"
