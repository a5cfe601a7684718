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
#include "adapter_plan.h"
#include "layer_types.h"

#include <limits.h>

#include <type_traits>

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
  static constexpr int E = 8, KS = 32, kParts = 1;
  static __device__ __forceinline__ f32x4 part(uint4 a, uint4 b, f32x4 c, int) {
    return mma(a, b, c);
  }
  static __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<_Float16> {
  static constexpr int E = 8, KS = 32, kParts = 1;
  static __device__ __forceinline__ f32x4 part(uint4 a, uint4 b, f32x4 c, int) {
    return mma(a, b, c);
  }
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
  static constexpr int E = 4, KS = 16, kParts = 4;
  static __device__ __forceinline__ f32x4 part(uint4 a, uint4 b, f32x4 c, int e) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, a)[e],
                                                __builtin_bit_cast(f32x4, b)[e], c, 0, 0, 0);
  }
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
  const int32_t* rows;      // the row at each position (k_adapter_list); null: itself
  const int32_t* count;     // nullable
  int64_t max_rows;
  int64_t in_stride, out_stride;
  void* out;
  float* t;                 // [t_parts][max_rows][rp] rank-wide rows, by position
  float* part;              // the product's partial sums (parts > 1)
  int32_t k, d, rank, rp, n_adapters;
  int32_t t_parts;          // parts of the rank-wide rows' reduction
  int32_t parts;            // parts of the product's reduction
  int32_t b4;               // four values of a row of b are one aligned load
  int32_t out4;             // four neighbouring outputs are one aligned store
  int64_t row_tiles;        // the product's grid: out_tiles x row_tiles x parts, after
  int32_t out_tiles;        // down_blocks workgroups of rank-wide rows
  int32_t down_blocks, down_sets;
  int64_t first;            // the launch's first workgroup of them
};

__device__ __forceinline__ int64_t live_rows(const AdapterArgs& a) {
  int64_t n = a.count ? *a.count : a.max_rows;
  return n < a.max_rows ? n : a.max_rows;
}
// The row at a position below n, and its adapter (INT_MAX without one).
__device__ __forceinline__ int64_t row_at(const AdapterArgs& a, int64_t pos) {
  return a.rows ? a.rows[pos] : pos;
}
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int64_t row) {
  const int p = a.ids[row];
  return p >= 0 && p < a.n_adapters ? p : INT_MAX;
}
// The lanes 0 .. 15 whose row has an adapter, and one of those rows' adapters.
__device__ __forceinline__ uint32_t with_adapter(int mine) {
  return (uint32_t)__ballot(mine != INT_MAX) & 0xFFFFu;
}
__device__ __forceinline__ int pick_adapter(int mine, uint32_t todo) {
  return __builtin_amdgcn_readlane(mine, __builtin_ctz(todo));
}
__device__ __forceinline__ uint32_t rows_of(int mine, int p) {
  return (uint32_t)__ballot(mine == p) & 0xFFFFu;
}

// 16 bytes per lane from memory straight to LDS, at the wave's lds + 16 * lane.
__device__ __forceinline__ void copy_to_lds(const void* from, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// Waits until at most N of the wave's copies are under way and its LDS
// accesses are done.  (The builtin's wait is one that the compiler counts with.)
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x70);  // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// Chunk c of 128-byte row r lies at chunk slot(r, c) of its row in LDS, so that
// 16 lanes that read one chunk of 16 rows fall on different banks.
__device__ __forceinline__ int row_slot(int r, int c) { return c ^ (r & 7); }

// Rank-wide rows of 16 positions: a workgroup per (tile, part of the
// reduction), whose W waves split the part and add their sums through LDS.
// Each wave copies 128 bytes of its 16 rows and of an adapter's 16 rank rows
// at a time to LDS of its own, two such chunks ahead (loaded as fragments, 16
// lanes read 16 rows and a CU takes 7 bytes a cycle: 1,501 rows of 9,216 fp32
// 85 us), adapter by adapter among the rows; a lane keeps the products of its
// own row's adapter.  What is not whole aligned chunks is loaded as fragments.
// Where rows of many adapters mix, `sets` workgroups share a tile's adapters.
template <typename T, bool VEC, int W>
__device__ __forceinline__ void adapter_down(const AdapterArgs& a, int64_t block, int64_t blocks,
                                             int part, int set, int sets, uint4* stage0,
                                             uint4* stage1, uint4* stage2, f32x4 (*red)[64]) {
  using M = Mma<T>;
  constexpr int E = M::E, BK = 2 * M::KS;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int64_t n = live_rows(a);
  const int whole = VEC ? a.k / BK : 0;  // chunks that are copied
  const int parts = a.t_parts * W, me = part * W + wave;
  const int c0 = (int)((int64_t)me * whole / parts), c1 = (int)((int64_t)(me + 1) * whole / parts);
  // the values behind them, by steps
  const int steps = (a.k - whole * BK + M::KS - 1) / M::KS;
  const int s0 = (int)((int64_t)me * steps / parts), s1 = (int)((int64_t)(me + 1) * steps / parts);
  const int cr = lane >> 3, cs = row_slot(cr, lane & 7) * E;  // a copy's row (and + 8), values
  for (int64_t pos0 = block * 16; pos0 < n; pos0 += blocks * 16) {
    bool in = pos0 + m < n;
    const int64_t row = row_at(a, in ? pos0 + m : n - 1);
    int mine = in ? adapter_of(a, row) : INT_MAX;
    if (sets > 1) {  // every sets-th of the rows' adapters; without one: set 0
      int at = 0, of = 0;
      for (uint32_t t = with_adapter(mine); t; at = at + 1 == sets ? 0 : at + 1) {
        const int p = pick_adapter(mine, t);
        t &= ~rows_of(mine, p);
        if (mine == p) of = at;
      }
      if (__ballot(in && of == set) == 0) continue;
      if (of != set) {
        in = false;
        mine = INT_MAX;
      }
    }
    const float scale = mine != INT_MAX ? a.scale[mine] : 0.0f;
    const uint32_t some = with_adapter(mine);
    const T* x = static_cast<const T*>(a.x) + row * a.in_stride;
    const T* xc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t pos = pos0 + cr + 8 * h;
      xc[h] = static_cast<const T*>(a.x) + row_at(a, pos < n ? pos : n - 1) * a.in_stride + cs;
    }
    for (int j0 = 0; j0 < a.rp; j0 += 16) {
      f32x4 out = {0.f, 0.f, 0.f, 0.f};
      int items = 0;  // (adapter, chunk) pairs
      for (uint32_t t = some; t; items += c1 - c0) t &= ~rows_of(mine, pick_adapter(mine, t));
      if (c1 == c0) items = 0;
      if (items) {
        uint32_t ftodo = some, todo = some;
        int fp = pick_adapter(mine, some), fc = c0, p = fp, c = c0;
        int64_t ac[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) ac[h] = (int64_t)min(j0 + cr + 8 * h, a.rank - 1) * a.k + cs;
        auto issue = [&](uint4* st) __attribute__((always_inline)) {
          const T* ap = static_cast<const T*>(a.a) + (int64_t)fp * a.rank * a.k + fc * BK;
#pragma unroll
          for (int h = 0; h < 2; ++h) copy_to_lds(xc[h] + fc * BK, st + wave * 256 + h * 64);
#pragma unroll
          for (int h = 0; h < 2; ++h) copy_to_lds(ap + ac[h], st + wave * 256 + 128 + h * 64);
          if (++fc == c1) {
            fc = c0;
            ftodo &= ~rows_of(mine, fp);
            if (ftodo) fp = pick_adapter(mine, ftodo);
          }
        };
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        auto step = [&](int i, const uint4* now, uint4* next) __attribute__((always_inline)) {
          if (i + 1 < items)
            wait_copies<4>();
          else
            wait_copies<0>();
          if (i + 2 < items) issue(next);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint4* at = now + wave * 256 + m * 8 + row_slot(m, 4 * s + g);
            acc = M::mma(at[128], at[0], acc);
          }
          if (++c == c1) {
            c = c0;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] += mine == p ? acc[e] : 0.0f;
            acc = f32x4{0.f, 0.f, 0.f, 0.f};
            todo &= ~rows_of(mine, p);
            if (todo) p = pick_adapter(mine, todo);
          }
        };
        wait_copies<0>();  // of the loads above, not of the copies in the loop
        issue(stage0);
        issue(stage1);  // behind a single item: that item's again
        for (int i = 0; i < items; i += 3) {
          step(i, stage0, stage2);
          if (i + 1 < items) step(i + 1, stage1, stage0);
          if (i + 2 < items) step(i + 2, stage2, stage1);
        }
      }
      if (s0 < s1)
        for (uint32_t todo = some; todo;) {
          const int p = pick_adapter(mine, todo), j = j0 + m;
          todo &= ~rows_of(mine, p);
          const T* ap = static_cast<const T*>(a.a) + ((int64_t)p * a.rank + j) * a.k;
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
          for (int s = s0; s < s1; ++s) {
            const int k = whole * BK + s * M::KS + E * g;
            const uint4 av = load_frag<T, VEC>(ap + k, j < a.rank ? a.k - k : 0);
            acc = M::mma(av, load_frag<T, VEC>(x + k, a.k - k), acc);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) out[e] += mine == p ? acc[e] : 0.0f;
        }
      __syncthreads();  // red is read before it is written again
      red[wave][lane] = out;
      __syncthreads();
      if (wave == 0 && in) {
#pragma unroll
        for (int w = 1; w < W; ++w) out += red[w][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = j0 + 4 * g + e < a.rank ? out[e] * scale : 0.0f;
        *reinterpret_cast<f32x4*>(a.t + (part * a.max_rows + pos0 + m) * a.rp + j0 + 4 * g) = out;
      }
    }
  }
}

// The rank-wide rows alone in a launch: of one reduction (t of x and a), or of
// two (and u of dy and the transposed b).

struct DownArgs {
  AdapterArgs of[2];
  int32_t vec[2];
};

template <typename T>
__global__ void __launch_bounds__(64 * kDownWaves) k_adapter_down(DownArgs d) {
  __shared__ uint4 stage0[kDownWaves * 256], stage1[kDownWaves * 256], stage2[kDownWaves * 256];
  __shared__ f32x4 red[kDownWaves][64];
  const AdapterArgs& a = blockIdx.z ? d.of[1] : d.of[0];
  if ((int)blockIdx.y >= a.t_parts) return;
  if (blockIdx.z ? d.vec[1] : d.vec[0])
    adapter_down<T, true, kDownWaves>(a, blockIdx.x, gridDim.x, blockIdx.y, 0, 1, stage0, stage1,
                                      stage2, red);
  else
    adapter_down<T, false, kDownWaves>(a, blockIdx.x, gridDim.x, blockIdx.y, 0, 1, stage0, stage1,
                                       stage2, red);
}

// The shared product with the rank-wide rows' in its epilogue, in tiles of TN
// outputs x TM rows.  The reduction goes through LDS 128 bytes of a row at a
// time, copied there directly from memory: STAGES blocks lie in LDS, one being
// multiplied while the copies of the others are under way (with one block
// ahead, its copies' latency of about 2 us was longer than the products of a
// block).  What lies behind the reduction's end, or is not aligned to 16 bytes,
// is loaded through registers and filled with zeros.
// TR = false: outputs d from x w^T + t b^T.  TR = true: outputs k from
// dy w + u a; the weights' reduction then runs down the columns of w, whose
// tile keeps its rows in LDS and is transposed as it is read.
// With parts > 1 the workgroups of a tile share its reduction and write their
// sums, which k_adapter_join adds in order before the same epilogue.
template <typename T, bool TR, int TN, int TM>
struct Gemm {
  using M = Mma<T>;
  static constexpr int E = M::E, BK = 2 * M::KS;      // values per 16 and per 128 bytes
  static constexpr int kWaves = TN >= 256 ? 8 : 4, kThreads = 64 * kWaves;
  static constexpr int WM = TM >= 64 ? 2 : 1;         // waves along the rows
  static constexpr int WN = kWaves / WM;              // and along the outputs
  static constexpr int NI = TN / WN / 16, NJ = TM / WM / 16;
  static constexpr int WCH = TN * BK * sizeof(T) / 16, XCH = TM * 8;  // 16-byte chunks of a tile
  static constexpr int RCH = TR ? TN / E : 8;         // chunks of a row of the weights' tile
  static constexpr int kStages = TM >= 64 ? (TR && TN < 256 ? 2 : 3) : 4;
  // copies per thread and block, at least (a wave's outstanding ones of a whole block)
  static constexpr int kCopies = WCH / kThreads + XCH / kThreads;

  // Chunk c of row r lies at chunk slot(r, c) of its row, so that the lanes of
  // a read fall on different banks: x and w by rows (16 lanes read one chunk
  // of 16 rows), and w transposed (16-bit: 32-byte blocks of rows 8 g + 0..3
  // of 2 lane groups at once; 32-bit: 64-byte blocks of rows 4 g of 4).
  static __device__ __forceinline__ int xslot(int r, int c) { return row_slot(r, c); }
  static __device__ __forceinline__ int wslot(int r, int c) {
    if constexpr (!TR) return c ^ (r & 7);
    if constexpr (sizeof(T) == 2) return c ^ ((((r & 3) | ((r >> 1) & 4)) << 1) & (RCH - 1));
    return c ^ ((((r >> 2) & 3) << 2) & (RCH - 1));
  }
  // The weights' fragment of outputs o .. o + 15 at step s.
  static __device__ __forceinline__ uint4 wfrag(const uint4* wl, int o, int s, int m, int g) {
    if constexpr (!TR) {
      return wl[(o + m) * 8 + xslot(o + m, 4 * s + g)];
    } else if constexpr (sizeof(T) == 2) {
      uint2 h[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = s * 32 + 8 * g + 4 * i + (m >> 2), c = (o >> 3) + ((m >> 1) & 1);
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        const char* at = reinterpret_cast<const char*>(wl + r * RCH + wslot(r, c)) + (m & 1) * 8;
        h[i] = __builtin_bit_cast(
            uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4*)(at)));
      }
      return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
    } else {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = s * 16 + 4 * g + e;
        v[e] = reinterpret_cast<const float*>(wl + r * RCH + wslot(r, (o + m) >> 2))[m & 3];
      }
      return __builtin_bit_cast(uint4, v);
    }
  }
};

// The rows at 16 NJ positions and their adapters.
template <int NJ>
struct TileRows {
  int64_t row[NJ];
  int mine[NJ];
  __device__ __forceinline__ TileRows(const AdapterArgs& a, int64_t pos0, int64_t n, int m) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t pos = pos0 + j * 16 + m;
      row[j] = pos < n ? row_at(a, pos) : 0;
      mine[j] = pos < n ? adapter_of(a, row[j]) : INT_MAX;
    }
  }
};

// Adds the rank-wide rows' products to outputs o0 .. of positions pos0 .. .
template <typename T, bool TR, int NI, int NJ>
__device__ __forceinline__ void add_ranks(const AdapterArgs& a, f32x4 (&acc)[NI][NJ],
                                          const int (&mine)[NJ], int o0, int64_t pos0, int m,
                                          int g) {
  const int outs = TR ? a.k : a.d;
  for (int q0 = 0; q0 < a.rp; q0 += 16) {
    const int q = q0 + 4 * g;
    f32x4 tv[NJ];
    uint32_t todo[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      tv[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      todo[j] = with_adapter(mine[j]);
      if (mine[j] != INT_MAX) {
        f32x4 v[kMaxDownParts];
#pragma unroll
        for (int h = 0; h < kMaxDownParts; ++h) {
          v[h] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (h == 0 || h < a.t_parts)
            v[h] = *reinterpret_cast<const f32x4*>(
                a.t + (h * a.max_rows + pos0 + j * 16 + m) * a.rp + q);
        }
#pragma unroll
        for (int h = 0; h < kMaxDownParts; ++h) tv[j] += v[h];
      }
    }
    auto load_b = [&](int p, f32x4 (&bv)[NI]) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int o = o0 + i * 16 + m;
        bv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (o < outs) {
          if constexpr (TR) {
            const T* ap = static_cast<const T*>(a.a) + (int64_t)p * a.rank * a.k + o;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (q + e < a.rank) bv[i][e] = (float)ap[(int64_t)(q + e) * a.k];
          } else {
            const T* bp = static_cast<const T*>(a.b) + ((int64_t)p * a.d + o) * a.rank + q;
            if (a.b4) {
              if (q < a.rank) {
                const Vec<T, 4> v = *reinterpret_cast<const Vec<T, 4>*>(bp);
#pragma unroll
                for (int e = 0; e < 4; ++e) bv[i][e] = (float)v.e[e];
              }
            } else {
              bv[i] = load4(bp, a.rank - q);
            }
          }
        }
      }
    };
    auto add_b = [&](int p, const f32x4 (&bv)[NI]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        if (rows_of(mine[j], p)) {
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const f32x4 add = mma_f32(bv[i], tv[j], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] += mine[j] == p ? add[e] : 0.0f;
          }
        }
      }
    };
    auto next = [&]() __attribute__((always_inline)) {
      int p = INT_MAX;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (p == INT_MAX && todo[j]) p = pick_adapter(mine[j], todo[j]);
#pragma unroll
      for (int j = 0; j < NJ; ++j) todo[j] &= ~rows_of(mine[j], p);
      return p;
    };
    for (int p = next(); p != INT_MAX; p = next()) {
      f32x4 bv[NI];
      load_b(p, bv);
      add_b(p, bv);
    }
  }
}

// The rank-wide row's products of four neighbouring outputs of one position by
// a lane alone, with its adapter's own values: no adapter waits for another
// one's loads.
template <typename T, bool TR>
__device__ __forceinline__ void row_ranks(const AdapterArgs& a, f32x4& acc, int p, int o,
                                          int64_t pos) {
  const int outs = TR ? a.k : a.d;
  for (int q0 = 0; q0 < a.rank; q0 += 8) {
    f32x4 t[2] = {}, tp[kMaxJoinParts][2];
#pragma unroll
    for (int h = 0; h < kMaxJoinParts; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        tp[h][i] = h < a.t_parts ? *reinterpret_cast<const f32x4*>(
                                       a.t + (h * a.max_rows + pos) * a.rp + q0 + 4 * i)
                                 : f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 b[4][2];  // TR: of rank values q0 + 2 e + i (outputs o ..); else of output o + e
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (TR) {
          const int q = q0 + 2 * e + i;
          const T* at = static_cast<const T*>(a.a) + ((int64_t)p * a.rank + q) * a.k + o;
          b[e][i] = load4(at, q < a.rank ? outs - o : 0);
        } else {
          const int q = q0 + 4 * i, oe = o + e < outs ? o + e : outs - 1;
          const T* at = static_cast<const T*>(a.b) + ((int64_t)p * a.d + oe) * a.rank + q;
          if (a.b4) {
            b[e][i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (q < a.rank) {
              const Vec<T, 4> v = *reinterpret_cast<const Vec<T, 4>*>(at);
              b[e][i] = f32x4{(float)v.e[0], (float)v.e[1], (float)v.e[2], (float)v.e[3]};
            }
          } else {
            b[e][i] = load4(at, a.rank - q);
          }
        }
      }
#pragma unroll
    for (int h = 0; h < kMaxJoinParts; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) t[i] += tp[h][i];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (TR) {
          acc += t[(2 * e + i) / 4][(2 * e + i) % 4] * b[e][i];
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[e] = fmaf(t[i][k], b[e][i][k], acc[e]);
        }
      }
  }
}

// Adds the bias to outputs o0 .. of positions pos0 .. and stores them.
template <typename T, bool TR, int NI, int NJ>
__device__ __forceinline__ void store_outputs(const AdapterArgs& a, const f32x4 (&acc)[NI][NJ],
                                              const int64_t (&row)[NJ], int o0, int64_t pos0,
                                              int64_t n, int m, int g) {
  const int outs = TR ? a.k : a.d;
  f32x4 bias[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i)
    bias[i] = a.bias ? load4(a.bias + o0 + i * 16 + 4 * g, outs - o0 - i * 16 - 4 * g)
                     : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    __builtin_amdgcn_sched_barrier(0);  // one row at a time: registers
    if (pos0 + j * 16 + m < n) {
      T* y = static_cast<T*>(a.out) + row[j] * a.out_stride;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int o = o0 + i * 16 + 4 * g;
        Vec<T, 4> v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v.e[e] = (T)(acc[i][j][e] + bias[i][e]);
        if (a.out4) {
          if (o < outs) *reinterpret_cast<Vec<T, 4>*>(y + o) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (o + e < outs) y[o + e] = v.e[e];
        }
      }
    }
  }
}

// A block's products from its tiles.
template <typename G, typename M, int NI, int NJ>
__device__ __forceinline__ void multiply(const uint4* wl, const uint4* xl, f32x4 (&acc)[NI][NJ],
                                         int wo, int wr, int m, int g) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    uint4 av[NI], bv[NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i) av[i] = G::wfrag(wl, wo + i * 16, s, m, g);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int r = wr + j * 16 + m;
      bv[j] = xl[r * 8 + G::xslot(r, 4 * s + g)];
    }
    // (of the four fp32 products of a step, one of every block before the next:
    // none waits for the one before it)
#pragma unroll
    for (int e = 0; e < M::kParts; ++e)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = M::part(av[i], bv[j], acc[i][j], e);
  }
}

// Tile of a logical index: panels of four tiles of outputs, row tile by row
// tile, so that neighbours share both operands in a cache.
__device__ __forceinline__ void tile_at(const AdapterArgs& a, int64_t i, int& tx, int64_t& ty) {
  const int64_t panel = i / (4 * a.row_tiles);
  const int width = min(4, a.out_tiles - (int)panel * 4);
  i -= panel * 4 * a.row_tiles;
  ty = i / width;
  tx = (int)(panel * 4 + i % width);
}

template <typename T, bool VEC, bool TR, int TN, int TM>
__global__ void __launch_bounds__(TN >= 256 ? 512 : 256) k_adapter_gemm(AdapterArgs a) {
  using G = Gemm<T, TR, TN, TM>;
  using M = Mma<T>;
  constexpr int E = G::E, BK = G::BK, NI = G::NI, NJ = G::NJ, TH = G::kThreads, ST = G::kStages;
  // A variable per stage, each named where it is used: of one array, the
  // compiler takes every read to need all the copies under way and waits for
  // them before it.
  constexpr int kStage = G::WCH + G::XCH;
  __shared__ uint4 stage0[kStage], stage1[kStage], stage2[ST > 2 ? kStage : 1];
  __shared__ uint4 stage3[ST > 3 ? kStage : 1];
  uint4* const last = ST > 3 ? stage3 : ST > 2 ? stage2 : stage1;
  int64_t block = a.first + blockIdx.x;
  if constexpr (!TR && TN < 256) {  // a call whose product is split takes its rank-wide rows here
    if (block < a.down_blocks) {
      static_assert(kStage >= kGemmDownWaves * 256 && kGemmDownWaves * 64 == TH, "in the stages");
      const int per = a.t_parts * a.down_sets;
      adapter_down<T, VEC, kGemmDownWaves>(
          a, block / per, a.down_blocks / per, (int)(block % a.t_parts),
          (int)(block % per / a.t_parts), a.down_sets, stage0, stage1, stage2,
          reinterpret_cast<f32x4(*)[64]>(stage0));
      return;
    }
    block -= a.down_blocks;
  }
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int64_t n = live_rows(a);
  const int outs = TR ? a.k : a.d, len = TR ? a.d : a.k;
  const int64_t tiles = a.out_tiles * a.row_tiles;
  const int z = (int)(block / tiles);
  int tx;
  int64_t ty;
  tile_at(a, a.parts > 1 ? block - z * tiles : xcd_block(block, tiles), tx, ty);
  const int o0 = tx * TN;
  const int wo = (wave % G::WN) * NI * 16, wr = (wave / G::WN) * NJ * 16;
  const T* w = static_cast<const T*>(a.w);
  const T* xs = static_cast<const T*>(a.x);
  const int blocks = (len + BK - 1) / BK;
  const int b0 = (int)((int64_t)z * blocks / a.parts);
  const int b1 = (int)((int64_t)(z + 1) * blocks / a.parts);
  constexpr int XC = (G::XCH + TH - 1) / TH, WC = G::WCH / TH;  // chunks per thread
  static_assert(G::WCH % TH == 0, "whole chunks per thread");
  const int64_t pos0 = ty * TM;
  if (pos0 >= n) return;
  f32x4 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // this thread's chunks: LDS slot c = TH i + thread holds its row's chunk
  // slot(row, c), as the slots are their own inverses
  const T* xp[XC];
  const T* wp[WC];
#pragma unroll
  for (int i = 0; i < XC; ++i) {
    const int c = i * TH + threadIdx.x, r = c >> 3;
    const int64_t pos = pos0 + r < n ? pos0 + r : n - 1;
    xp[i] = xs + row_at(a, pos) * a.in_stride + G::xslot(r, c & 7) * E;
  }
#pragma unroll
  for (int i = 0; i < WC; ++i) {
    const int c = i * TH + threadIdx.x, r = c / G::RCH;
    const int ch = G::wslot(r, c % G::RCH);
    if constexpr (TR) {
      const int o = o0 + ch * E < outs ? o0 + ch * E : 0;
      wp[i] = w + (int64_t)r * a.k + o;
    } else {
      const int o = o0 + r < outs ? o0 + r : outs - 1;
      wp[i] = w + (int64_t)o * a.k + ch * E;
    }
  }
  auto whole = [&](int b) { return VEC && (b + 1) * BK <= len; };  // copied directly
  auto copy = [&](int b, uint4* wl) __attribute__((always_inline)) {
    uint4* xl = wl + G::WCH;
    const int k0 = b * BK;
#pragma unroll
    for (int i = 0; i < WC; ++i)
      copy_to_lds(wp[i] + (TR ? (int64_t)k0 * a.k : k0), wl + i * TH + wave * 64);
#pragma unroll
    for (int i = 0; i < XC; ++i)
      if (G::XCH % TH == 0 || i * TH + wave * 64 < G::XCH)
        copy_to_lds(xp[i] + k0, xl + i * TH + wave * 64);
  };
  auto stage = [&](int b, uint4* wl) __attribute__((always_inline)) {
    if (whole(b)) return copy(b, wl);
    uint4* xl = wl + G::WCH;
    const int k0 = b * BK;
#pragma unroll
    for (int i = 0; i < WC; ++i) {
      const int c = i * TH + threadIdx.x, r = c / G::RCH;
      const int ch = G::wslot(r, c % G::RCH);
      if constexpr (TR)
        wl[c] = load_frag<T, VEC>(w + (int64_t)(k0 + r) * a.k + o0 + ch * E,
                                  k0 + r < len ? outs - o0 - ch * E : 0);
      else
        wl[c] = load_frag<T, VEC>(wp[i] + k0, len - k0 - ch * E);
    }
#pragma unroll
    for (int i = 0; i < XC; ++i) {
      const int c = i * TH + threadIdx.x;
      if (c < G::XCH) xl[c] = load_frag<T, VEC>(xp[i] + k0, len - k0 - G::xslot(c >> 3, c & 7) * E);
    }
  };
  // Long reductions run in rounds of ST blocks that are all copied directly: a
  // block is multiplied once it has landed (of the ST - 2 behind it each has at
  // least kCopies copies under way) and the block before it is done with in
  // every wave, while the block ST - 1 behind it is copied to that one's stage.
  int b = b0;
  const int bw = VEC ? min(b1, len / BK) : 0;  // blocks that are copied directly
  if (bw - b0 >= 2 * ST - 1) {
    auto step = [&](int c, const uint4* now, uint4* next) __attribute__((always_inline)) {
      wait_copies<(ST - 2) * G::kCopies>();
      __builtin_amdgcn_s_barrier();
      copy(c + ST - 1, next);
      __builtin_amdgcn_sched_barrier(0);  // the copies first
      multiply<G, M, NI, NJ>(now, now + G::WCH, acc, wo, wr, m, g);
    };
    copy(b0, stage0);
    if constexpr (ST > 2) copy(b0 + 1, stage1);
    if constexpr (ST > 3) copy(b0 + 2, stage2);
    for (; b + 2 * ST - 1 <= bw; b += ST) {
      step(b, stage0, last);
      step(b + 1, stage1, stage0);
      if constexpr (ST > 2) step(b + 2, stage2, stage1);
      if constexpr (ST > 3) step(b + 3, stage3, stage2);
    }
  } else {
    if (b0 < b1) stage(b0, stage0);
    if (ST > 2 && b0 + 1 < b1) stage(b0 + 1, stage1);
    if (ST > 3 && b0 + 2 < b1) stage(b0 + 2, stage2);
  }
  // The last blocks, and short reductions: as above, each block as it may be
  // loaded.
  auto step = [&](int c, const uint4* now, uint4* next) __attribute__((always_inline)) {
    if (c + ST - 2 < b1 && whole(c + ST - 2))
      wait_copies<(ST - 2) * G::kCopies>();
    else
      wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    if (c + ST - 1 < b1) stage(c + ST - 1, next);
    multiply<G, M, NI, NJ>(now, now + G::WCH, acc, wo, wr, m, g);
  };
  for (; b < b1; b += ST) {
    step(b, stage0, last);
    if (b + 1 < b1) step(b + 1, stage1, stage0);
    if (ST > 2 && b + 2 < b1) step(b + 2, stage2, stage1);
    if (ST > 3 && b + 3 < b1) step(b + 3, stage3, stage2);
  }
  if (a.parts > 1) {
    f32x4* out = reinterpret_cast<f32x4*>(a.part) +
                 ((ty * a.out_tiles + tx) * a.parts + z) * (TN * TM / 4) + wave * NI * NJ * 64 +
                 lane;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) out[(i * NJ + j) * 64] = acc[i][j];
  } else {
    const TileRows<NJ> rows(a, pos0 + wr, n, m);
    add_ranks<T, TR, NI, NJ>(a, acc, rows.mine, o0 + wo, pos0 + wr, m, g);
    store_outputs<T, TR>(a, acc, rows.row, o0 + wo, pos0 + wr, n, m, g);
  }
}

// Adds a tile's parts in order, then its epilogue: a wave per 16 outputs of 16
// rows.  The rows' adapters are loaded first and everything else at once after
// them: the kernel's time is its chain of loads.
template <typename T, bool TR, int TN, int TM>
__global__ void __launch_bounds__(256) k_adapter_join(AdapterArgs a) {
  using G = Gemm<T, TR, TN, TM>;
  constexpr int NI = G::NI, NJ = G::NJ, F = TN * TM / 256;  // 16 x 16 blocks of a tile
  const int lane = threadIdx.x & 63;
  const int64_t item = blockIdx.x * 4ll + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tile = item / F;
  const int f = (int)(item % F), wave = f / (NI * NJ), i = f % (NI * NJ) / NJ, j = f % NJ;
  const int64_t n = live_rows(a);
  const int64_t pos0 = tile / a.out_tiles * TM + (wave / G::WN) * NJ * 16 + j * 16;
  const int o0 = (int)(tile % a.out_tiles) * TN + (wave % G::WN) * NI * 16 + i * 16;
  if (pos0 >= n || o0 >= (TR ? a.k : a.d)) return;
  const f32x4* in =
      reinterpret_cast<const f32x4*>(a.part) + tile * a.parts * (TN * TM / 4) + f * 64 + lane;
  const int m = lane & 15, g = lane >> 4;
  const TileRows<1> rows(a, pos0, n, m);
  constexpr int P = 8;  // parts whose loads are under way while the adapters' are
  f32x4 part[P];
#pragma unroll
  for (int h = 0; h < P; ++h)
    part[h] = h < a.parts ? in[(int64_t)h * (TN * TM / 4)] : f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 acc[1][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}};
  if (rows.mine[0] != INT_MAX)
    row_ranks<T, TR>(a, acc[0][0], rows.mine[0], o0 + 4 * g, pos0 + m);
  f32x4 sum = part[0];
#pragma unroll
  for (int h = 1; h < P; ++h) sum += part[h];
  for (int h0 = P; h0 < a.parts; h0 += P) {
#pragma unroll
    for (int h = 0; h < P; ++h)
      part[h] = h0 + h < a.parts ? in[(int64_t)(h0 + h) * (TN * TM / 4)]
                                 : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < P; ++h) sum += part[h];
  }
  acc[0][0] += sum;
  store_outputs<T, TR>(a, acc, rows.row, o0, pos0, n, m, g);
}

// The rows of each adapter in ascending order: rows[off[p] .. off[p + 1]), and
// those without one last.  A workgroup per adapter (and one for the rest)
// counts the rows of smaller adapters and its own, then writes its own.  Waves
// take consecutive ranges of the rows.
constexpr int kListWaves = 16;

// b[p] [d][rank] as [rank][d], 64 rows at a time through LDS: the rank-wide
// rows u then read b as t read a.  Of all such items, every `of`-th from `item`.
template <typename T>
__device__ __forceinline__ void adapter_flip(const AdapterArgs& a, int64_t item, int64_t of,
                                             T* bt) {
  __shared__ T tile[64 * (NSC_MAX_RANK + 1)];
  const int blocks = (a.d + 63) / 64;
  for (; item < (int64_t)a.n_adapters * blocks; item += of) {
    const int64_t p = item / blocks;
    const int d0 = (int)(item % blocks) * 64, nd = min(64, a.d - d0);
    const T* from = static_cast<const T*>(a.b) + (p * a.d + d0) * a.rank;
    for (int i = threadIdx.x; i < nd * a.rank; i += 64 * kListWaves)
      tile[i / a.rank * (a.rank + 1) + i % a.rank] = from[i];
    __syncthreads();
    T* to = bt + p * a.rank * a.d + d0;
    for (int i = threadIdx.x; i < 64 * a.rank; i += 64 * kListWaves) {
      const int j = i / 64, r = i % 64;
      if (r < nd) to[(int64_t)j * a.d + r] = tile[r * (a.rank + 1) + j];
    }
    __syncthreads();  // the tile is read before the next item writes it
  }
}

template <typename T>
__global__ void __launch_bounds__(64 * kListWaves) k_adapter_list(AdapterArgs a, int32_t* off,
                                                                  int32_t* rows, int32_t listers,
                                                                  T* bt) {
  if ((int)blockIdx.x >= listers)
    return adapter_flip<T>(a, blockIdx.x - listers, gridDim.x - listers, bt);
  __shared__ int32_t less[kListWaves], same[kListWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = live_rows(a);
  const int64_t per = (n + kListWaves * 64 - 1) / (kListWaves * 64) * 64;
  const int64_t b = wave * per < n ? wave * per : n, e = b + per < n ? b + per : n;
  for (int p = blockIdx.x; p <= a.n_adapters; p += listers) {
    auto of = [&](int64_t r) {
      const int q = r < e ? a.ids[r] : -1;
      return q >= 0 && q < a.n_adapters ? q : (r < e ? a.n_adapters : INT_MAX);
    };
    int32_t lo = 0, eq = 0;
    for (int64_t r = b; r < e; r += 64) {
      const int mine = of(r + lane);
      lo += __popcll(__ballot(mine < p));
      eq += __popcll(__ballot(mine == p));
    }
    __syncthreads();
    if (lane == 0) {
      less[wave] = lo;
      same[wave] = eq;
    }
    __syncthreads();
    int32_t at = 0;
#pragma unroll
    for (int w = 0; w < kListWaves; ++w) at += less[w] + (w < wave ? same[w] : 0);
    if (threadIdx.x == 0) off[p] = at;
    for (int64_t r = b; r < e; r += 64) {
      const bool mine = of(r + lane) == p;
      const uint64_t mask = __ballot(mine);
      if (mine) rows[at + __popcll(mask & ((1ull << lane) - 1))] = (int32_t)(r + lane);
      at += __popcll(mask);
    }
  }
}

// The gradients of the adapters: a wave takes the 16 rank values j0 .. of one
// adapter and 16 x CPL columns, a lane CPL neighbouring ones (16 bytes of a
// row), and adds u^T x (or t^T dy) over the adapter's rows, 16 at a time.  RW
// waves share them and add their sums through LDS; the other waves of a
// workgroup take other columns.
struct GradArgs {
  const float* t[2];        // u, t: [parts][max_rows][rp]
  int32_t parts[2];
  int64_t max_rows;
  const void* v[2];         // x, dy
  float* out[2];            // da, db
  int64_t v_stride[2];
  int32_t cols[2];
  int32_t vec[2];           // a lane's columns are one aligned load
  int32_t blocks0;          // workgroups per adapter that take da's columns
  const int32_t* off;
  const int32_t* rows;
  int32_t rank, rp;
};

template <typename T, int RW>
__global__ void __launch_bounds__(512) k_adapter_grad(GradArgs a) {
  constexpr int CPL = 16 / sizeof(T), CW = 8 / RW;  // waves along the columns
  __shared__ f32x4 red[RW > 1 ? 8 : 1][CPL][RW > 1 ? 64 : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4, rw = wave % RW;
  const int which = (int)blockIdx.x >= a.blocks0, p = blockIdx.y;
  const int blk = (int)blockIdx.x - (which ? a.blocks0 : 0);
  const int cols = which ? a.cols[1] : a.cols[0], parts = which ? a.parts[1] : a.parts[0];
  const bool vec = (which ? a.vec[1] : a.vec[0]) != 0;
  const int64_t stride = which ? a.v_stride[1] : a.v_stride[0];
  const float* t = which ? a.t[1] : a.t[0];
  const T* v = static_cast<const T*>(which ? a.v[1] : a.v[0]);
  float* out = which ? a.out[1] : a.out[0];
  const int c = (blk * CW + wave / RW) * 16 * CPL + m * CPL;
  const int32_t b = a.off[p], e = a.off[p + 1];
  for (int j0 = 0; j0 < a.rp; j0 += 16) {
    f32x4 acc[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    int32_t row[4];  // of the next 16 rows, -1 behind the last
    auto next_rows = [&](int32_t r) {
#pragma unroll
      for (int s = 0; s < 4; ++s) row[s] = r + 4 * g + s < e ? a.rows[r + 4 * g + s] : -1;
    };
    auto all_rows = [&](auto one) __attribute__((always_inline)) {  // one part of t, or more
      next_rows(b + rw * 16);
      for (int32_t r = b + rw * 16; r < e; r += 16 * RW) {
        f32x4 uv;
        uint4 xv[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const bool in = row[s] >= 0;
          const T* x = v + (in ? row[s] : 0) * stride + c;
          xv[s] = vec ? load_frag<T, true>(x, in ? cols - c : 0)
                      : load_frag<T, false>(x, in ? cols - c : 0);
          const float* ts = t + (int64_t)(r + 4 * g + s) * a.rp + j0 + m;
          uv[s] = in ? *ts : 0.0f;
          if constexpr (!decltype(one)::value) {
            float part[kMaxDownParts - 1];
#pragma unroll
            for (int h = 1; h < kMaxDownParts; ++h)
              part[h - 1] = in && h < parts ? ts[h * a.max_rows * a.rp] : 0.0f;
#pragma unroll
            for (int h = 1; h < kMaxDownParts; ++h) uv[s] += part[h - 1];
          }
        }
        next_rows(r + 16 * RW);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          f32x4 xi;
#pragma unroll
          for (int s = 0; s < 4; ++s) xi[s] = (float)__builtin_bit_cast(Vec<T, CPL>, xv[s]).e[i];
          acc[i] = mma_f32(uv, xi, acc[i]);
        }
      }
    };
    if (parts == 1)
      all_rows(std::true_type{});
    else
      all_rows(std::false_type{});
    if constexpr (RW > 1) {
      __syncthreads();  // red is read before it is written again
#pragma unroll
      for (int i = 0; i < CPL; ++i) red[wave][i][lane] = acc[i];
      __syncthreads();
      if (rw == 0) {
#pragma unroll 1
        for (int w = 1; w < RW; ++w)
#pragma unroll
          for (int i = 0; i < CPL; ++i) acc[i] += red[wave + w][i][lane];
      }
    }
    if (rw == 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + 4 * g + q;
#pragma unroll
        for (int i = 0; i < CPL; ++i)
          if (j < a.rank && c + i < cols)
            out[which ? ((int64_t)p * cols + c + i) * a.rank + j
                      : ((int64_t)p * a.rank + j) * cols + c + i] = acc[i][q];
      }
    }
  }
}

// -------------------------------------------------------------------- host

constexpr int64_t kMaxRows = 0x7FFFFFFF;
// Backward: k_adapter_grad looks up to 16 x 8 + 15 positions past the last row,
// in 32 bits.
constexpr int64_t kMaxGradRows = kMaxRows - 255;
constexpr int64_t kLaunchThreads = 0xFFFFFFFFll;  // of one launch

bool misaligned(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }

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

int check_adapter_call(const nsc_adapter_desc* d, int64_t max_rows, const void* ws,
                       size_t ws_bytes, bool backward) {
  if (int rc = check_adapter(d)) return rc;
  NSC_REQUIRE_L(max_rows >= 0 && max_rows <= (backward ? kMaxGradRows : kMaxRows), NSC_E_INVAL,
                "max_rows %lld out of range", (long long)max_rows);
  const size_t need = adapter_layout(*d, max_rows, backward).total;
  NSC_REQUIRE_L(need == 0 || (ws != nullptr && (uintptr_t)ws % 256 == 0 && ws_bytes >= need),
                NSC_E_WORKSPACE, "workspace needs %zu bytes (256-byte aligned), got %zu", need,
                ws_bytes);
  return NSC_OK;
}

template <typename T>
int launch_down(const DownArgs& d, int n, hipStream_t st) {
  int64_t grid = (d.of[0].max_rows + 15) / 16;
  if (grid > 16 * kNumCU) grid = 16 * kNumCU;
  int32_t parts = d.of[0].t_parts;
  if (n > 1 && d.of[1].t_parts > parts) parts = d.of[1].t_parts;
  hipLaunchKernelGGL(k_adapter_down<T>, dim3((unsigned)grid, (unsigned)parts, (unsigned)n),
                     dim3(64 * kDownWaves), 0, st, d);
  NSC_CHECK_LAUNCH("k_adapter_down");
  return NSC_OK;
}

template <typename T, bool VEC, bool TR, int TN, int TM>
int launch_tiles(AdapterArgs a, hipStream_t st) {
  using G = Gemm<T, TR, TN, TM>;
  a.out_tiles = ((TR ? a.k : a.d) + TN - 1) / TN;
  a.row_tiles = (a.max_rows + TM - 1) / TM;
  const int64_t tiles = a.out_tiles * a.row_tiles, grid = tiles * a.parts + a.down_blocks;
  const int64_t most = kLaunchThreads / G::kThreads;  // in launches of that many
  for (a.first = 0; a.first < grid; a.first += most) {
    hipLaunchKernelGGL((k_adapter_gemm<T, VEC, TR, TN, TM>),
                       dim3((unsigned)(grid - a.first < most ? grid - a.first : most)),
                       dim3(G::kThreads), 0, st, a);
    NSC_CHECK_LAUNCH("k_adapter_gemm");
  }
  if constexpr (TN < 256) {
    if (a.parts > 1) {
      hipLaunchKernelGGL((k_adapter_join<T, TR, TN, TM>),
                         dim3((unsigned)(tiles * (TN * TM / 1024))), dim3(256), 0, st, a);
      NSC_CHECK_LAUNCH("k_adapter_join");
    }
  }
  return NSC_OK;
}

template <typename T, bool VEC, bool TR>
int launch_plan(const AdapterArgs& a, const GemmPlan& p, hipStream_t st) {
  if (p.tn == 256) return launch_tiles<T, VEC, TR, 256, 128>(a, st);
  if constexpr (!TR)
    if (p.tn == 64) return launch_tiles<T, VEC, TR, 64, 64>(a, st);
  if (p.tm == 64) return launch_tiles<T, VEC, TR, 128, 64>(a, st);
  return launch_tiles<T, VEC, TR, 128, 16>(a, st);
}

template <typename T, bool TR>
int launch_gemm(const AdapterArgs& a, const GemmPlan& p, bool vec, hipStream_t st) {
  return vec ? launch_plan<T, true, TR>(a, p, st) : launch_plan<T, false, TR>(a, p, st);
}

template <typename T>
int launch_grad(GradArgs a, int32_t n_adapters, int64_t max_rows, hipStream_t st) {
  constexpr int CPL = 16 / sizeof(T);
  const int rw = grad_row_waves((int64_t)a.cols[0] + a.cols[1], n_adapters, max_rows, sizeof(T));
  const int32_t width = 16 * CPL * (8 / rw);
  a.blocks0 = (a.cols[0] + width - 1) / width;
  const dim3 g((unsigned)(a.blocks0 + (a.cols[1] + width - 1) / width), (unsigned)n_adapters),
      t(512);
  switch (rw) {
    case 1: hipLaunchKernelGGL((k_adapter_grad<T, 1>), g, t, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_adapter_grad<T, 2>), g, t, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_adapter_grad<T, 4>), g, t, 0, st, a); break;
    default: hipLaunchKernelGGL((k_adapter_grad<T, 8>), g, t, 0, st, a); break;
  }
  NSC_CHECK_LAUNCH("k_adapter_grad");
  return NSC_OK;
}

// The rows by adapter, and (bt) b transposed.
template <typename T>
int launch_list(AdapterArgs* a, int32_t* off, int32_t* rows, T* bt, hipStream_t st) {
  const int32_t most = 8 * kNumCU, listers = a->n_adapters < most ? a->n_adapters + 1 : most;
  int64_t flips = bt ? (int64_t)a->n_adapters * ((a->d + 63) / 64) : 0;
  const int64_t room = kLaunchThreads / (64 * kListWaves) - listers;
  if (flips > room) flips = room;  // its workgroups take the ones behind
  hipLaunchKernelGGL(k_adapter_list<T>, dim3((unsigned)(listers + flips)), dim3(64 * kListWaves), 0,
                     st, *a, off, rows, listers, bt);
  NSC_CHECK_LAUNCH("k_adapter_list");
  a->rows = rows;
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
  g.b4 = d.rank % 4 == 0 && !misaligned(b, 4 * type_bytes(d.dtype));
  return g;
}

template <typename T>
int project(const nsc_adapter_desc& d, AdapterArgs a, unsigned char* ws, hipStream_t st) {
  constexpr int E = 16 / sizeof(T);
  const AdapterLayout L = adapter_layout(d, a.max_rows, false);
  if (L.list)
    if (int rc = launch_list<T>(&a, reinterpret_cast<int32_t*>(ws + L.off),
                                reinterpret_cast<int32_t*>(ws + L.rows), nullptr, st))
      return rc;
  a.in_stride = d.x_stride;
  a.out_stride = d.y_stride;
  a.out4 = d.d % 4 == 0 && d.y_stride % 4 == 0 && !misaligned(a.out, 4 * sizeof(T));
  a.t = reinterpret_cast<float*>(ws + L.t);
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.t_parts = L.t_parts;
  a.parts = L.g.parts;
  const bool vec = !misaligned(a.x, 16) && !misaligned(a.a, 16) && !misaligned(a.w, 16) &&
                   d.k % E == 0 && d.x_stride % E == 0;
  if (a.parts > 1) {
    // few tiles: several workgroups share the adapters of each
    const int32_t tiles = (int32_t)((a.max_rows + 15) / 16) * a.t_parts;
    a.down_sets = tiles * 8 <= kNumCU ? 8 : tiles * 2 <= kNumCU ? kNumCU / tiles : 1;
    a.down_blocks = tiles * a.down_sets;
  } else {
    DownArgs t{};
    t.of[0] = a;
    t.vec[0] = vec;
    if (int rc = launch_down<T>(t, 1, st)) return rc;
  }
  return launch_gemm<T, false>(a, L.g, vec, st);
}

template <typename T>
int backward(const nsc_adapter_desc& d, AdapterArgs a, const void* x, const void* dy, void* dx,
             float* da, float* db, unsigned char* ws, hipStream_t st) {
  constexpr int E = 16 / sizeof(T);
  const AdapterLayout L = adapter_layout(d, a.max_rows, true);
  float* t = reinterpret_cast<float*>(ws + L.t);
  float* u = reinterpret_cast<float*>(ws + L.u);
  int32_t* off = reinterpret_cast<int32_t*>(ws + L.off);
  int32_t* rows = reinterpret_cast<int32_t*>(ws + L.rows);
  T* bt = a.max_rows > 0 ? reinterpret_cast<T*>(ws + L.bt) : nullptr;
  if (int rc = launch_list<T>(&a, off, rows, bt, st)) return rc;
  if (a.max_rows > 0) {
    DownArgs r{};
    r.of[0] = a;  // t = scale x a^T
    r.of[0].x = x;
    r.of[0].in_stride = d.x_stride;
    r.of[0].t = t;
    r.of[0].t_parts = L.t_parts;
    r.vec[0] = !misaligned(x, 16) && !misaligned(a.a, 16) && d.k % E == 0 && d.x_stride % E == 0;
    a.x = dy;
    a.in_stride = d.y_stride;
    a.t = u;
    a.t_parts = L.u_parts;
    r.of[1] = a;  // u = scale dy b
    r.of[1].a = bt;
    r.of[1].k = d.d;
    r.vec[1] = !misaligned(dy, 16) && d.d % E == 0 && d.y_stride % E == 0;
    if (int rc = launch_down<T>(r, 2, st)) return rc;
    if (dx) {
      a.out = dx;
      a.out_stride = d.x_stride;
      a.out4 = d.k % 4 == 0 && d.x_stride % 4 == 0 && !misaligned(dx, 4 * sizeof(T));
      a.part = reinterpret_cast<float*>(ws + L.part);
      a.parts = L.g.parts;
      const bool vec = !misaligned(dy, 16) && !misaligned(a.w, 16) && d.d % E == 0 &&
                       d.y_stride % E == 0 && d.k % E == 0;
      if (int rc = launch_gemm<T, true>(a, L.g, vec, st)) return rc;
    }
  }
  GradArgs g{};
  g.off = off;
  g.rows = rows;
  g.max_rows = a.max_rows;
  g.rank = a.rank;
  g.rp = a.rp;
  const void* v[2] = {x, dy};
  const int64_t strides[2] = {d.x_stride, d.y_stride};
  const int32_t cols[2] = {d.k, d.d};
  for (int i = 0; i < 2; ++i) {
    g.t[i] = i ? t : u;
    g.parts[i] = i ? L.t_parts : L.u_parts;
    g.v[i] = v[i];
    g.v_stride[i] = strides[i];
    g.cols[i] = cols[i];
    g.vec[i] = !misaligned(v[i], 16) && strides[i] % E == 0 && cols[i] % E == 0;
    g.out[i] = i ? db : da;
  }
  return launch_grad<T>(g, d.n_adapters, a.max_rows, st);
}

}  // namespace

size_t adapter_call_bytes(const nsc_adapter_desc& d, int64_t rows) {
  return adapter_layout(d, rows, false).total;
}

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
  NSC_REQUIRE_L(bytes != nullptr && max_rows >= 0 && (backward == 0 || backward == 1) &&
                    max_rows <= (backward ? kMaxGradRows : kMaxRows),
                NSC_E_INVAL, "bad arguments");
  *bytes = adapter_ws_bytes(*desc, max_rows, backward != 0);
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
  NSC_REQUIRE_L(y != x, NSC_E_INVAL, "y overlaps x");
  AdapterArgs g = adapter_args(*desc, w, a, b, scale, ids, count, max_rows);
  g.x = x;
  g.bias = bias;
  g.out = y;
  unsigned char* at = static_cast<unsigned char*>(ws);
  const hipStream_t st = (hipStream_t)stream;
  if (desc->dtype == NSC_T_BF16) return project<__bf16>(*desc, g, at, st);
  if (desc->dtype == NSC_T_F16) return project<_Float16>(*desc, g, at, st);
  return project<float>(*desc, g, at, st);
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
  NSC_REQUIRE_L(!dx || max_rows == 0 || (dx != x && dx != dy), NSC_E_INVAL,
                "dx overlaps x or dy, which are read after it is written");
  const AdapterArgs g =
      adapter_args(*desc, w, a, b, scale, ids, max_rows ? count : nullptr, max_rows);
  unsigned char* at = static_cast<unsigned char*>(ws);
  const hipStream_t st = (hipStream_t)stream;
  if (desc->dtype == NSC_T_BF16) return backward<__bf16>(*desc, g, x, dy, dx, da, db, at, st);
  if (desc->dtype == NSC_T_F16) return backward<_Float16>(*desc, g, x, dy, dx, da, db, at, st);
  return backward<float>(*desc, g, x, dy, dx, da, db, at, st);
}

}  // extern "C"
