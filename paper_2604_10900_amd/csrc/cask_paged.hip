// Rows into the pages of a cache, quantised as they are written, and back out of them.
#include <hip/hip_runtime.h>

#include "cask.h"
#include "cask_common.h"

namespace cask {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kE4m3Max = 448.f;
// Lanes that share a row.  Both directions only move rows and run at the rate of a copy once a lane moves enough of one:
// sixteen / eight lanes, inputs not in the last-level cache: 229 376 rows of 128 bf16 values and as many of V into e4m3
// pages 48.5 / 40.7 us (4.4 TB/s), 946 176 back 191 / 160.5 (4.6), ragged fp32 rows of 64 channels 67 / 52 (4.65).
constexpr int kRowLanes = 8;
constexpr int kBlockRows = 256 / kRowLanes;      // rows of K and of V a workgroup takes

// Largest over the eight lanes of a row.
__device__ inline float max8(float v) {
#define CASK_STEP(how) \
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), how, 0xf, 0xf, true)))
  CASK_STEP(0xb1);   // neighbours
  CASK_STEP(0x4e);   // pairs of a quad
  CASK_STEP(0x141);  // the half row turned round
#undef CASK_STEP
  return v;
}

// A lane's share of a row: N consecutive elements as raw words.
template <typename T, int N>
struct Share {
  static constexpr int kWords = N * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ void load(const T* p) {
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
      }
    } else {
      const u32x2 v = *reinterpret_cast<const u32x2*>(p);
      w[0] = v[0];
      w[1] = v[1];
    }
  }
  __device__ void store(void* p) const {
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[4 * i + e];
        reinterpret_cast<u32x4*>(p)[i] = v;
      }
    } else if constexpr (kWords == 2) {
      *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
    } else {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    }
  }
  __device__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
};

// A row's scale and the lane's N values of it as e4m3.  448 x / a: for bf16 rows one quotient in 500 lies exactly
// between two e4m3 values, so it is the quotient that is rounded and not a product with a rounded 448 / a.  One
// Newton step on the product's remainder gives such quotients exactly, and any other to 2^-23 of itself, with three
// instructions; row and a are brought to a's binade first, where neither 448 x nor the remainder can overflow or
// lose its low bits.
template <typename T, int N>
__device__ inline float quantise(const Share<T, N>& x, uint32_t (&q)[N / 4]) {
  float a = 0.f;
  bool odd = false;  // an infinity or NaN among the lane's values
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float m = fabsf(x.get(i));
    const bool fin = m < __builtin_inff();
    odd |= !fin;
    a = fmaxf(a, fin ? m : 0.f);
  }
  a = fmaxf(max8(a), kE4m3Max * 0x1p-126f);
  const int e = (int)(__float_as_uint(a) >> 23) - 127;              // a is a normal number
  const float f = __builtin_ldexpf(1.f, -e);                        // (2^-127 at the least: a denormal, exact)
  const float as = a * f, inv = 1.f / as, up = kE4m3Max * f;
  float y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float n = x.get(i) * up, y0 = n * inv;
    y[i] = __builtin_fmaf(__builtin_fmaf(-y0, as, n), inv, y0);
  }
  if (odd) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float v = x.get(i);
      if (fabsf(v) == __builtin_inff()) y[i] = v > 0.f ? kE4m3Max : -kE4m3Max;
      if (v != v) y[i] = v;
    }
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
  }
  return a / kE4m3Max;
}

// The row that a group of lanes takes: unit, place in the unit's rows, in the arrays and in the pools.
struct RowPlace {
  int64_t array, pool;  // -1: none
};
__device__ inline RowPlace place_of(const PagesView& pg, const RowsView& rw, int64_t item) {  // item < 2^31, see resolve_rows
  RowPlace at{-1, -1};
  if (item >= (int64_t)pg.n_units * rw.max_n) return at;
  const int u = (int)((uint32_t)item / (uint32_t)rw.max_n), t = (int)((uint32_t)item % (uint32_t)rw.max_n);
  if (t >= rows_of_unit(rw, u)) return at;
  at.array = array_row(rw, first_of_unit(rw, u), t);
  const int64_t r = (rw.start ? rw.start[u] : 0) + (int64_t)t;
  if (r >= 0 && r < pg.cap) at.pool = pool_row(pg, u, (int)r);
  return at;
}

// Eight lanes take a row of K and the same row of V: both on their way before the first is looked at.
template <typename T, bool E4M3, int D>
__global__ __launch_bounds__(256) void cache_write_kernel(PagesView pg, RowsView rw, const T* __restrict__ K,
                                                          const T* __restrict__ V) {
  constexpr int N = D / kRowLanes;
  const int lane = threadIdx.x % kRowLanes;
  const int64_t items = (int64_t)pg.n_units * rw.max_n;
  for (int64_t item = (int64_t)blockIdx.x * kBlockRows + threadIdx.x / kRowLanes; item < items; item += (int64_t)gridDim.x * kBlockRows) {
    const RowPlace at = place_of(pg, rw, item);
    if (at.array < 0 || at.pool < 0) continue;  // (the lanes of a row go on together)
    Share<T, N> k, v;
    k.load(K + at.array * D + lane * N);
    v.load(V + at.array * D + lane * N);
    if constexpr (E4M3) {
      uint32_t qk[N / 4], qv[N / 4];
      const float sk = quantise(k, qk), sv = quantise(v, qv);
      Share<uint8_t, N> out;
#pragma unroll
      for (int i = 0; i < N / 4; ++i) out.w[i] = qk[i];
      out.store(pg.K + at.pool * D + lane * N);
#pragma unroll
      for (int i = 0; i < N / 4; ++i) out.w[i] = qv[i];
      out.store(pg.V + at.pool * D + lane * N);
      if (lane == 0) {
        pg.K_scale[at.pool] = sk;
        pg.V_scale[at.pool] = sv;
      }
    } else {
      k.store(reinterpret_cast<T*>(pg.K) + at.pool * D + lane * N);
      v.store(reinterpret_cast<T*>(pg.V) + at.pool * D + lane * N);
    }
  }
}

// value * scale, rounded once to the array's type
template <typename T, int N>
__device__ inline void widen(const uint32_t (&q)[N / 4], float scale, Share<T, N>& out) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
    const float y[4] = {lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) out.w[4 * i + e] = __float_as_uint(y[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        out.w[2 * i + e] = (uint32_t)float_to_bf16_bits(y[2 * e]) | ((uint32_t)float_to_bf16_bits(y[2 * e + 1]) << 16);
    }
  }
}

template <typename T, bool E4M3, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(PagesView pg, RowsView rw, T* __restrict__ K, T* __restrict__ V) {
  constexpr int N = D / kRowLanes;
  const int lane = threadIdx.x % kRowLanes;
  const int64_t items = (int64_t)pg.n_units * rw.max_n;
  for (int64_t item = (int64_t)blockIdx.x * kBlockRows + threadIdx.x / kRowLanes; item < items; item += (int64_t)gridDim.x * kBlockRows) {
    const RowPlace at = place_of(pg, rw, item);
    if (at.array < 0) continue;
    Share<T, N> k, v;
#pragma unroll
    for (int i = 0; i < k.kWords; ++i) k.w[i] = v.w[i] = 0u;
    if (at.pool >= 0) {
      if constexpr (E4M3) {
        uint32_t qk[N / 4], qv[N / 4];
        const uint32_t* pk = reinterpret_cast<const uint32_t*>(pg.K + at.pool * D + lane * N);
        const uint32_t* pv = reinterpret_cast<const uint32_t*>(pg.V + at.pool * D + lane * N);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          qk[i] = pk[i];
          qv[i] = pv[i];
        }
        const float sk = pg.K_scale[at.pool], sv = pg.V_scale[at.pool];
        widen<T, N>(qk, sk, k);
        widen<T, N>(qv, sv, v);
      } else {
        k.load(reinterpret_cast<const T*>(pg.K) + at.pool * D + lane * N);
        v.load(reinterpret_cast<const T*>(pg.V) + at.pool * D + lane * N);
      }
    }
    k.store(K + at.array * D + lane * N);
    v.store(V + at.array * D + lane * N);
  }
}

// Workgroups of a call; they go round again where there would be 2^32 threads.
int row_blocks(const PagesView& pg, const RowsView& rw) {
  const int64_t blocks = ((int64_t)pg.n_units * rw.max_n + kBlockRows - 1) / kBlockRows;
  return (int)(blocks < (1 << 23) ? blocks : (1 << 23));
}

}  // namespace

hipError_t launch_cache_write(const KParams& kp, const PagesView& pg, const RowsView& rw, bool e4m3, const void* K,
                              const void* V, hipStream_t st) {
  auto go = [&](auto* k, auto fn) { fn<<<dim3(row_blocks(pg, rw)), dim3(256), 0, st>>>(pg, rw, k, static_cast<decltype(k)>(V)); };
  const float* kf = static_cast<const float*>(K);
  const uint16_t* kb = static_cast<const uint16_t*>(K);
#define CASK_PW(T, k) \
  if (e4m3) kp.d == 64 ? go(k, &cache_write_kernel<T, true, 64>) : go(k, &cache_write_kernel<T, true, 128>); \
  else kp.d == 64 ? go(k, &cache_write_kernel<T, false, 64>) : go(k, &cache_write_kernel<T, false, 128>)
  if (kp.dtype == CASK_F32) { CASK_PW(float, kf); } else { CASK_PW(uint16_t, kb); }
#undef CASK_PW
  return hipGetLastError();
}

hipError_t launch_cache_read(const KParams& kp, const PagesView& pg, const RowsView& rw, bool e4m3, void* K, void* V,
                             hipStream_t st) {
  auto go = [&](auto* k, auto fn) { fn<<<dim3(row_blocks(pg, rw)), dim3(256), 0, st>>>(pg, rw, k, static_cast<decltype(k)>(V)); };
  float* kf = static_cast<float*>(K);
  uint16_t* kb = static_cast<uint16_t*>(K);
#define CASK_PR(T, k) \
  if (e4m3) kp.d == 64 ? go(k, &cache_read_kernel<T, true, 64>) : go(k, &cache_read_kernel<T, true, 128>); \
  else kp.d == 64 ? go(k, &cache_read_kernel<T, false, 64>) : go(k, &cache_read_kernel<T, false, 128>)
  if (kp.dtype == CASK_F32) { CASK_PR(float, kf); } else { CASK_PR(uint16_t, kb); }
#undef CASK_PR
  return hipGetLastError();
}

}  // namespace cask
