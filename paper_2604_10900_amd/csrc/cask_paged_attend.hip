// Attention of the newest tokens of every unit, one or a chunk of them, over the pages of its cache: causal,
// proportional to the rows' token counts, with a sliding window and first rows that stay visible.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cask.h"
#include "cask_common.h"

namespace cask {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_inff();
constexpr int kCols = 16;  // query rows (token, head) of a 16x16 product: its columns

// The rows of a unit that a block of queries sees, in tiles of TR rows: tiles [0, n_sink) of the cache, then the
// tiles from `first` on; n_tiles of both.
struct TileRange {
  int n_sink, first, n_tiles;
  __device__ int tile(int t) const { return t < n_sink ? t : t - n_sink + first; }
};
template <int TR>
__device__ inline TileRange tiles_of(int i_lo, int i_hi, int end, int causal, int window, int sinks) {
  const int hi = causal ? min(end, i_hi + 1) : end;  // rows [lo, hi) and the first `sinks`
  const int lo = window > 0 ? max(0, i_lo - window + 1) : 0;
  TileRange r{0, lo / TR, 0};
  if (hi <= 0) return r;
  if (window > 0) r.n_sink = min((min(sinks, hi) + TR - 1) / TR, r.first);
  r.n_tiles = r.n_sink + max(0, (hi + TR - 1) / TR - r.first);
  return r;
}

// What a unit brings to a call.
struct UnitRows {
  int n, start, end;  // tokens, row of the first of them, rows of the unit (start + n, inside the capacity)
  int64_t first;
  __device__ UnitRows(const PagesView& pg, const RowsView& rw, int u) {
    n = rows_of_unit(rw, u);
    const int s = rw.start ? rw.start[u] : 0;
    start = max(-(1 << 30), min(s, 1 << 30));  // (no capacity is larger, and sums with n stay inside 32 bits)
    end = min(start + n, pg.cap);
    first = first_of_unit(rw, u);
  }
};

// Sizes that follow from the types and the head dimension.  T: queries and results, E4M3: of the cache's rows.
template <typename T, bool E4M3, int D>
struct RowsGeom {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kEl = E4M3 ? 1 : (int)sizeof(T);      // bytes of a cached element
  static constexpr int kTileRows = kBf16 ? 32 : 16;          // cache rows a wave takes at a time
  static constexpr int kKeys = kTileRows / 4;                // of them per lane group (16 lanes)
  static constexpr int kSub = kTileRows / 16;                // 16-row subtiles of the logit product
  // key row: pieces of a lane.  A piece holds what the query operand's kPieceQ 16-byte pieces are multiplied with.
  static constexpr int kPieceEl = kBf16 ? (E4M3 ? 16 : 8) : 4;  // elements
  static constexpr int kPieces = D / (4 * kPieceEl);
  static constexpr int kPieceQ = kPieceEl * (int)sizeof(T) / 16;
  static constexpr int kQ = kPieces * kPieceQ;
  static constexpr int kPieceWords = kPieceEl * kEl / 4;
  static constexpr int EPV = (kBf16 && D == 128) ? 8 : 4;    // elements of a value row per lane and load
  static constexpr int kValLoads = D / (16 * EPV);           // loads per value row
  static constexpr int kValWords = EPV * kEl / 4;
  static constexpr int kBlocks = D / 16;                     // 16-channel blocks of the value product
  // channel of row m of block b of the value product
  __device__ static int channel(int b, int m) { return (b / EPV) * (16 * EPV) + m * EPV + b % EPV; }
};

template <int WORDS>
struct Words {
  uint32_t w[WORDS];
};
template <int WORDS, int AUX>
__device__ inline Words<WORDS> load_words(__amdgpu_buffer_rsrc_t rs, int off, int soff) {
  Words<WORDS> r;
  if constexpr (WORDS == 4) {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rs, off, soff, AUX);
#pragma unroll
    for (int e = 0; e < 4; ++e) r.w[e] = v[e];
  } else if constexpr (WORDS == 2) {
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rs, off, soff, AUX);
    r.w[0] = v[0];
    r.w[1] = v[1];
  } else {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, soff, AUX);
  }
  return r;
}

// Masks as bits and words: a predicate for every element would not fit the scalar registers.
__device__ inline uint32_t rows_below(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
// Bit o: the query at row i sees row r + o, as far as places go.
__device__ inline uint32_t seen_rows(int r, int i, int causal, int window, int sinks) {
  uint32_t bits = causal ? rows_below(i + 1 - r) : ~0u;
  if (window > 0) bits &= ~rows_below(i + 1 - window - r) | rows_below(sinks - r);
  return bits;
}
__device__ inline uint32_t bit_mask(uint32_t bits, int b) { return (uint32_t)((int32_t)(bits << (31 - b)) >> 31); }
__device__ inline float masked(float x, uint32_t m) { return __uint_as_float((__float_as_uint(x) & m) | (__float_as_uint(kNegInf) & ~m)); }
// 1 where a value is no finite number; of the two bf16 of a word in bits 0 and 16.
__device__ inline uint32_t not_finite(float x) { return ((__float_as_uint(x) & 0x7fffffffu) + 0x00800000u) >> 31; }
__device__ inline uint32_t not_finite2(uint32_t w) { return (((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15; }

// two e4m3 values of a word as two bf16 in a word (exact)
__device__ inline uint32_t e4m3_to_bf16(uint32_t w, bool upper) {
  const bf16x2 v = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
  return __builtin_bit_cast(uint32_t, v);
}

__device__ inline float exp2_from(float x, float reference) { return __builtin_amdgcn_exp2f(x - reference); }

// Factor of a state with reference m that is joined under the reference `top` >= m.  A state that has seen no finite
// logit holds zeros, or the NaN of a logit, which has to come through.
__device__ inline float share(float m, float top) { return m == kNegInf ? 1.f : exp2_from(m, top); }
// The result of joined sums: zero where no row was seen.
__device__ inline float joined(float num, float den) { return den == 0.f ? num : num / den; }

// Partial results of the splits: [unit][query row][split] of D sums, behind all of them one reference and one
// denominator each.
__device__ inline f32x2* part_state(const PagedAttend& pa, int G, int D) {
  return reinterpret_cast<f32x2*>(pa.part + (int64_t)pa.pg.n_units * pa.rw.max_n * G * pa.splits * D);
}

// A wave takes tiles of kTileRows rows of one unit for NQ groups of 16 query rows (token, head): the waves of a
// workgroup, and the `splits` workgroups that share a block of queries, take them in turn.  Per tile two products
// on 16x16 matrix tiles, as in the one-token attention over dense caches:
//   logits   S[key][query]     = K_tile . Q^T       (lane: key or query = lane % 16, 16 bytes of channels)
//   values   O[channel][query] += V_tile^T . P      (lane: channel or query = lane % 16, keys of group lane / 16)
// A lane ends the first product with one query's logits of the kKeys keys 16 y + 4 (lane / 16) + r and holds its
// weights as the second product's operand as they stand; the channel rows of that product are numbered so that a
// lane already holds its share of them (RowsGeom::channel).
// e4m3 rows become bf16 (exact) in registers; a key's scale multiplies its logits, a value row's scale the weights.
// bf16 weights enter as two terms, p = hi + lo (2^-17 in all); fp32 products are summed in short chains.
// Every 16 rows of a tile lie in one page: a descriptor each, that ends behind the unit's last row and is empty where
// no page is.
// A row that some query of the block does not see must not reach it, whatever it holds: a NaN key gives a NaN logit,
// which the mask replaces; a value that is not finite would give 0 * inf.  Tiles where the mask hides rows from some
// queries are looked through for such values; if there are any, they are taken out of the product, and one more
// product, of zeros and ones, says which results are NaN because a query sees one.
template <typename T, bool E4M3, int D, int NQ, int WAVES, bool NT>
__global__ __launch_bounds__(WAVES * 64, 8 / WAVES) void paged_rows_kernel(KParams kp, PagedAttend pa, int q_blocks) {
  using A = RowsGeom<T, E4M3, D>;
  constexpr int TR = A::kTileRows, KEYS = A::kKeys, SUB = A::kSub, NB = A::kBlocks, EPV = A::EPV, NV = A::kValLoads;
  constexpr int kAccPitch = D + 4;
  constexpr int ROWB = D * A::kEl;
  constexpr int kAux = NT ? 2 : 0;  // cache policy of the row loads: non-temporal or default
  extern __shared__ __align__(16) unsigned char rows_lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  int u, part_of;
  if (!map_block(pa.pg.n_units, q_blocks * pa.splits, u, part_of)) return;
  const int qb = part_of / pa.splits, sp = part_of % pa.splits;
  const int G = kp.G;
  const UnitRows ur(pa.pg, pa.rw, u);
  const int m0 = qb * (NQ * kCols), m_all = ur.n * G;
  if (m0 >= m_all) return;
  float* bias_s = reinterpret_cast<float*>(rows_lds) + wv * 32;
  float* st_m = reinterpret_cast<float*>(rows_lds) + WAVES * 32;  // [WAVES][16]
  float* st_l = st_m + WAVES * kCols;
  float* st_acc = st_l + WAVES * kCols;                           // [WAVES][16][kAccPitch]
  const int32_t* cu = pa.count ? pa.count + (size_t)u * pa.count_pitch : nullptr;
  const float c = kp.scale_log2;
  const int step = pa.splits * WAVES;

  const int m1 = min(m_all, m0 + NQ * kCols);
  const int i_lo = ur.start + m0 / G, i_hi = ur.start + (m1 - 1) / G;
  const TileRange range = tiles_of<TR>(i_lo, i_hi, ur.end, kp.causal, pa.window, pa.sinks);

  // the queries of this lane: column l16 of every group
  u32x4 q[NQ][A::kQ];
  int qi[NQ];  // row of the query's token
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int m = m0 + n * kCols + l16;
    const int t = m / G;
    const int64_t at = m < m1 ? array_row(pa.rw, ur.first, t) : -1;
    qi[n] = ur.start + t;
    const T* qp = static_cast<const T*>(pa.Q) + ((at < 0 ? 0 : at) * G + (at < 0 ? 0 : m % G)) * D;
#pragma unroll
    for (int i = 0; i < A::kQ; ++i) {
      const int ch = (i / A::kPieceQ * 4 + g) * A::kPieceEl + (i % A::kPieceQ) * (16 / (int)sizeof(T));
      q[n][i] = at < 0 ? u32x4{0u, 0u, 0u, 0u} : *reinterpret_cast<const u32x4*>(qp + ch);
    }
  }

  Words<A::kPieceWords> ka[SUB][A::kPieces];
  Words<A::kValWords> va[KEYS][NV];
  f32x4 ks4[SUB], vs4[SUB];  // scales of the lane's keys
  int cn = 1;
  // Subtile y of tile t: its first pool row, -1 where no page is or no row of the unit
  auto sub_row = [&](int t, int y) -> int64_t {
    const int r = t * TR + y * 16;
    return r < ur.end ? pool_row(pa.pg, u, r) : -1;
  };
  auto sub_rsrc = [&](const unsigned char* pool, int64_t row, int t, int y) {
    const int left = row >= 0 ? min(16, ur.end - (t * TR + y * 16)) : 0;
    const int bytes = __builtin_amdgcn_readfirstlane(left * ROWB);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(pool) + (row >= 0 ? row : 0) * ROWB, 0, bytes, 0x00020000);
  };
  auto sub_scales = [&](const float* s, int64_t row) {
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(s) + (row >= 0 ? row : 0), 0, row >= 0 ? 64 : 0, 0x00020000);
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, g * 16, 0, 0));
  };
  const int k_off = l16 * ROWB + g * (A::kPieceEl * A::kEl), v_off = g * 4 * ROWB + l16 * (EPV * A::kEl);
  auto load_keys = [&](int t, const int64_t (&row)[SUB]) {
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      const __amdgpu_buffer_rsrc_t rs = sub_rsrc(pa.pg.K, row[y], t, y);
#pragma unroll
      for (int i = 0; i < A::kPieces; ++i) ka[y][i] = load_words<A::kPieceWords, kAux>(rs, k_off, i * (4 * A::kPieceEl * A::kEl));
      if constexpr (E4M3) ks4[y] = sub_scales(pa.pg.K_scale, row[y]);
    }
    if (cu) {
      const int r = t * TR + (lane & (TR - 1));
      cn = cu[min(r, pa.count_pitch - 1)];
      if (r >= pa.count_pitch) cn = 1;  // rows behind the counted ones stand for themselves
    }
  };
  auto load_values = [&](int t, const int64_t (&row)[SUB]) {
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      const __amdgpu_buffer_rsrc_t rs = sub_rsrc(pa.pg.V, row[y], t, y);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          va[y * 4 + j][i] = load_words<A::kValWords, kAux>(rs, v_off + j * ROWB, i * (16 * EPV * A::kEl));
      if constexpr (E4M3) vs4[y] = sub_scales(pa.pg.V_scale, row[y]);
    }
  };

  float m_run[NQ], l_run[NQ];
  uint32_t marks[NQ];  // bit 4 b + r: the result of acc[n][b][r] is NaN
  f32x4 acc[NQ][NB];  // acc[n][b][r] = O[channel(b, 4 g + r)][query n, l16]
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = kNegInf;
    l_run[n] = 0.f;
    marks[n] = 0u;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // The next tile's keys are requested behind the logits, its values behind the product with the weights, the pages of
  // the tile after that before both.
  auto key_mask = [](uint32_t bits, int j) { return bit_mask(bits, (j >> 2) * 16 + (j & 3)); };
  auto rows_at = [&](int t0, int64_t (&row)[SUB]) {
#pragma unroll
    for (int y = 0; y < SUB; ++y) row[y] = t0 < range.n_tiles ? sub_row(range.tile(t0), y) : -1;
  };
  const int t_first = sp * WAVES + wv;
  int64_t row[SUB], row_next[SUB];
  rows_at(t_first, row);
  load_keys(range.tile(t_first), row);
  load_values(range.tile(t_first), row);
  rows_at(t_first + step, row_next);
  for (int t0 = t_first; t0 < range.n_tiles; t0 += step) {
    const int t = range.tile(t0), t_next = range.tile(t0 + step);
    bool there[SUB];  // the subtile has a page
#pragma unroll
    for (int y = 0; y < SUB; ++y) {
      there[y] = row[y] >= 0;
      row[y] = row_next[y];
    }
    rows_at(t0 + 2 * step, row_next);
    // Does every query of the block see every row of the tile?
    bool all = t * TR + TR <= ur.end && (!kp.causal || t * TR + TR - 1 <= i_lo);
#pragma unroll
    for (int y = 0; y < SUB; ++y) all = all && there[y];
    if (pa.window > 0) all = all && (t * TR > i_hi - pa.window || t * TR + TR <= pa.sinks);
    f32x4 bias4[SUB];
#pragma unroll
    for (int y = 0; y < SUB; ++y) bias4[y] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (cu) {
      if (lane < TR) bias_s[lane & (TR - 1)] = cn > 1 ? __log2f((float)cn) : 0.f;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int y = 0; y < SUB; ++y) bias4[y] = *reinterpret_cast<const f32x4*>(&bias_s[y * 16 + g * 4]);
      __builtin_amdgcn_wave_barrier();
    }
    // the lane's values as the product takes them: bf16 words of (key pair, channel), or floats
    u32x4 vb[A::kBf16 ? NB : 1];
    auto value_words = [&](int j, int i, int w) -> uint32_t {  // bf16: channels 2 w, 2 w + 1 of load i of key j
      if constexpr (E4M3) return e4m3_to_bf16(va[j][i].w[w / 2], w & 1);
      else return va[j][i].w[w];
    };
    if constexpr (A::kBf16) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int w = 0; w < EPV / 2; ++w)
#pragma unroll
          for (int k2 = 0; k2 < 4; ++k2) {  // the halves of two keys' words that hold a block's channel
            const uint32_t a = value_words(2 * k2, i, w), b = value_words(2 * k2 + 1, i, w);
            vb[i * EPV + 2 * w][k2] = __builtin_amdgcn_perm(b, a, 0x05040100u);
            vb[i * EPV + 2 * w + 1][k2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
          }
    }
    float vf[A::kBf16 ? 1 : KEYS][A::kBf16 ? 1 : NB];
    if constexpr (!A::kBf16) {
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if constexpr (E4M3) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)va[j][i].w[0], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)va[j][i].w[0], true);
            vf[j][i * 4] = lo[0], vf[j][i * 4 + 1] = lo[1], vf[j][i * 4 + 2] = hi[0], vf[j][i * 4 + 3] = hi[1];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[j][i * 4 + e] = __uint_as_float(va[j][i].w[e]);
          }
        }
    }
    f32x4 s[NQ][SUB];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int y = 0; y < SUB; ++y) {
        s[n][y] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (A::kBf16) {
#pragma unroll
          for (int i = 0; i < A::kPieces; ++i)
#pragma unroll
            for (int e = 0; e < A::kPieceQ; ++e) {
              u32x4 kw;
              if constexpr (E4M3) {
#pragma unroll
                for (int w = 0; w < 4; ++w) kw[w] = e4m3_to_bf16(ka[y][i].w[2 * e + w / 2], w & 1);
              } else {
#pragma unroll
                for (int w = 0; w < 4; ++w) kw[w] = ka[y][i].w[w];
              }
              s[n][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw),
                                                             __builtin_bit_cast(bf16x8, q[n][i * A::kPieceQ + e]), s[n][y], 0, 0, 0);
            }
        } else {
          // chains of eight products, the chains in pairs
          f32x4 chain[A::kPieces / 2];
#pragma unroll
          for (int pair = 0; pair < A::kPieces / 2; ++pair) {
            f32x4 a[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f32x4 kf;
              const int i = 2 * pair + (e >> 1);
              if constexpr (E4M3) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)ka[y][i].w[0], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)ka[y][i].w[0], true);
                kf = f32x4{lo[0], lo[1], hi[0], hi[1]};
              } else {
#pragma unroll
                for (int w = 0; w < 4; ++w) kf[w] = __uint_as_float(ka[y][i].w[w]);
              }
              const f32x4 qf = __builtin_bit_cast(f32x4, q[n][i]);
              a[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[2 * (e & 1)], qf[2 * (e & 1)], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
              a[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[2 * (e & 1) + 1], qf[2 * (e & 1) + 1], a[e], 0, 0, 0);
            }
            chain[pair] = (a[0] + a[1]) + (a[2] + a[3]);
          }
#pragma unroll
          for (int o = A::kPieces / 4; o > 0; o >>= 1)
#pragma unroll
            for (int h = 0; h < o; ++h) chain[h] += chain[h + o];
          s[n][y] = chain[0];
        }
        if constexpr (E4M3) s[n][y] *= ks4[y];
      }
    }
    load_keys(t_next, row);
    // s[n][y][r] = <key 16 y + 4 g + r, query n, l16>
    uint32_t bits[NQ];  // bit 16 y + r: the lane's query sees its key of (y, r)
    if (!all) {
      uint32_t here = rows_below(ur.end - t * TR);
#pragma unroll
      for (int y = 0; y < SUB; ++y)
        if (!there[y]) here &= ~(0xffffu << (16 * y));
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        bits[n] = (seen_rows(t * TR, qi[n], kp.causal, pa.window, pa.sinks) & here) >> (4 * g);
        // values that are not finite leave the product; marks stay for those that see one
      }
      uint32_t odd = 0u;
      if constexpr (A::kBf16) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= not_finite2(vb[b][e]);
      } else {
#pragma unroll
        for (int j = 0; j < KEYS; ++j)
#pragma unroll
          for (int b = 0; b < NB; ++b) odd |= not_finite(vf[j][b]);
      }
      if (__any(odd != 0u)) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          f32x4 seen[NQ];
#pragma unroll
          for (int n = 0; n < NQ; ++n) seen[n] = f32x4{0.f, 0.f, 0.f, 0.f};
          if constexpr (A::kBf16) {
            u32x4 bad;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t k = not_finite2(vb[b][e]);
              bad[e] = k * 0x3f80u;  // one or zero
              vb[b][e] &= ~(k * 0xffffu);
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
              u32x4 see;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                see[e] = (key_mask(bits[n], 2 * e) & 0x3f80u) | (key_mask(bits[n], 2 * e + 1) & 0x3f800000u);
              seen[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, see), seen[n], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int j = 0; j < KEYS; ++j) {
              const uint32_t k = not_finite(vf[j][b]);
              vf[j][b] = __uint_as_float(__float_as_uint(vf[j][b]) & (k - 1u));
#pragma unroll
              for (int n = 0; n < NQ; ++n)
                seen[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k * 0x3f800000u), __uint_as_float(key_mask(bits[n], j) & 0x3f800000u), seen[n], 0, 0, 0);
            }
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) marks[n] |= min(__float_as_uint(seen[n][r]), 1u) << (4 * b + r);
          __builtin_amdgcn_sched_barrier(0);  // (or all blocks' temporaries live at once)
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float p[KEYS], mx = kNegInf;
#pragma unroll
      for (int j = 0; j < KEYS; ++j) p[j] = __builtin_fmaf(s[n][j >> 2][j & 3], c, bias4[j >> 2][j & 3]);
      if (!all) {
#pragma unroll
        for (int j = 0; j < KEYS; ++j) p[j] = masked(p[j], key_mask(bits[n], j));
      }
#pragma unroll
      for (int j = 0; j < KEYS; ++j) mx = fmaxf(mx, p[j]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m_run[n], mx);
      const float ref = mn == kNegInf ? 0.f : mn;  // (a query that has seen no row yet)
      const float corr = exp2_from(m_run[n], ref);
      if constexpr (!A::kBf16) {  // (fp32: the logit meets its reference inside one rounding)
#pragma unroll
        for (int j = 0; j < KEYS; ++j) p[j] = __builtin_fmaf(s[n][j >> 2][j & 3], c, bias4[j >> 2][j & 3] - ref);
        if (!all) {
#pragma unroll
          for (int j = 0; j < KEYS; ++j) p[j] = masked(p[j], key_mask(bits[n], j));
        }
      }
      float ps = 0.f;
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        p[j] = __builtin_amdgcn_exp2f(A::kBf16 ? p[j] - ref : p[j]);
        ps += p[j];
        if constexpr (E4M3) p[j] *= vs4[j >> 2][j & 3];
      }
      if constexpr (E4M3) {
        if (!all) {  // (the scale of a row that is not seen may be anything)
#pragma unroll
          for (int j = 0; j < KEYS; ++j) p[j] = __uint_as_float(__float_as_uint(p[j]) & key_mask(bits[n], j));
        }
      }
      l_run[n] = __builtin_fmaf(l_run[n], corr, ps);
      m_run[n] = mn;
      if (__any(corr != 1.f)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[n][b][r] *= corr;
      }
      if constexpr (A::kBf16) {
        bf16x8 ph, pl;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const __bf16 hi = (__bf16)p[j];
          ph[j] = hi;
          pl[j] = (__bf16)(p[j] - (float)hi);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vb[b]), ph, acc[n][b], 0, 0, 0);
          acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vb[b]), pl, acc[n][b], 0, 0, 0);
        }
      } else {
        // (a tile's products are summed on their own: the long sum has as many addends as there are tiles)
#pragma unroll
        for (int b0 = 0; b0 < NB; b0 += 4) {
          f32x4 a[4];
#pragma unroll
          for (int j = 0; j < KEYS; ++j)
#pragma unroll
            for (int b = 0; b < 4; ++b)
              a[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][b0 + b], p[j], j ? a[b] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int b = 0; b < 4; ++b) acc[n][b0 + b] += a[b];
        }
      }
    }
    load_values(t_next, row);
  }

  // The waves' states are merged in wave order: the same bits every run.
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (m0 + n * kCols >= m1) break;
    float l = l_run[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
      st_m[wv * kCols + l16] = m_run[n];
      st_l[wv * kCols + l16] = l;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x4 o = acc[n][b];
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = __uint_as_float(__float_as_uint(o[r]) | bit_mask(marks[n], 4 * b + r));  // (all ones: a NaN)
      *reinterpret_cast<f32x4*>(&st_acc[(wv * kCols + l16) * kAccPitch + b * 16 + g * 4]) = o;
    }
    __syncthreads();
    const int rows_here = min(kCols, m1 - (m0 + n * kCols));
    for (int o = tid; o < rows_here * D; o += WAVES * 64) {
      const int h = o / D, ch = o % D, m = m0 + n * kCols + h;
      // where channel `ch` waits: block b, row r with RowsGeom::channel(b, r) == ch
      const int at = ((ch / (16 * EPV)) * EPV + ch % EPV) * 16 + (ch % (16 * EPV)) / EPV;
      float top = kNegInf;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, st_m[w * kCols + h]);
      float num = 0.f, den = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = share(st_m[w * kCols + h], top);
        den = __builtin_fmaf(st_l[w * kCols + h], f, den);
        num = __builtin_fmaf(st_acc[(w * kCols + h) * kAccPitch + at], f, num);
      }
      if (pa.splits == 1) {
        const int64_t row = array_row(pa.rw, ur.first, m / G);
        if (row >= 0) Elem<T>::store(static_cast<T*>(pa.out) + (row * G + m % G) * D + ch, joined(num, den));
      } else {
        const int64_t at = ((int64_t)u * pa.rw.max_n * G + m) * pa.splits + sp;
        pa.part[at * D + ch] = num;
        if (ch == 0) part_state(pa, G, D)[at] = f32x2{top, den};
      }
    }
    __syncthreads();
  }
}

constexpr int kMostSplits = 64, kFewSplits = 8;

// Adds the splits of a query row under their common reference, in their order.
// FEW: D / 4 threads a row, which hold all of its splits at once (28 672 rows of 2 splits: a workgroup each 40 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_combine_few_kernel(int G, PagedAttend pa, int64_t rows) {
  constexpr int kLanes = D / 4;
  const int64_t o = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (o >= rows) return;
  const int ch = (threadIdx.x % kLanes) * 4, S = pa.splits;
  const uint32_t per_unit = (uint32_t)(pa.rw.max_n * G);  // (no more rows than kMostBlocks in all where there are splits)
  const int u = (int)((uint32_t)o / per_unit), m = (int)((uint32_t)o % per_unit);
  // (asked for at once with the partial results, which lie there whether the row exists or not)
  const bool there = m < rows_of_unit(pa.rw, u) * G;
  const int64_t row = array_row(pa.rw, first_of_unit(pa.rw, u), m / G);
  f32x2 st[kFewSplits];
  f32x4 v[kFewSplits];
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < kFewSplits; ++i) {
    st[i] = i < S ? part_state(pa, G, D)[o * S + i] : f32x2{kNegInf, 0.f};
    v[i] = i < S ? *reinterpret_cast<const f32x4*>(pa.part + (o * S + i) * D + ch) : f32x4{0.f, 0.f, 0.f, 0.f};
    top = fmaxf(top, st[i][0]);
  }
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
#pragma unroll
  for (int i = 0; i < kFewSplits; ++i)
    if (i < S) {
      const float f = share(st[i][0], top);
      num += v[i] * f;
      den = __builtin_fmaf(st[i][1], f, den);
    }
  if (!there || row < 0) return;
  T* out = static_cast<T*>(pa.out) + (row * G + m % G) * D + ch;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(out) = f32x4{joined(num[0], den), joined(num[1], den), joined(num[2], den), joined(num[3], den)};
  } else {
    u32x2 w;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      w[e] = (uint32_t)float_to_bf16_bits(joined(num[2 * e], den)) | (uint32_t)float_to_bf16_bits(joined(num[2 * e + 1], den)) << 16;
    *reinterpret_cast<u32x2*>(out) = w;
  }
}

// Many splits: a wave finds the reference, a workgroup's 256 / (D / 4) groups of threads take every so many-th split,
// the groups' sums are added in order.  (A thread per channel that goes through the splits one by one: 28 rows of 64
// splits 20 us, this 4.)
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_combine_kernel(int G, PagedAttend pa) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kMost = kMostSplits;
  __shared__ float factor[kMost];
  __shared__ float total;
  __shared__ __align__(16) float sums[kGroups][D];
  const int64_t o = blockIdx.x;
  const uint32_t per_unit = (uint32_t)(pa.rw.max_n * G);
  const int u = (int)(blockIdx.x / per_unit), m = (int)(blockIdx.x % per_unit);
  const bool there = m < rows_of_unit(pa.rw, u) * G;  // (see above)
  const int64_t row = array_row(pa.rw, first_of_unit(pa.rw, u), m / G);
  const int S = pa.splits, tid = threadIdx.x, grp = tid / kLanes, ch = (tid % kLanes) * 4;
  if (tid < 64) {
    const f32x2 st = tid < S ? part_state(pa, G, D)[o * S + tid] : f32x2{kNegInf, 0.f};
    float top = st[0];
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float f = share(st[0], top);
    if (tid < S) factor[tid] = f;
    const float den = wave_sum(tid < S ? st[1] * f : 0.f);
    if (tid == 0) total = den;
  }
  const float* pp = pa.part + o * S * D + ch;
  f32x4 v[kMost / kGroups];
#pragma unroll
  for (int i = 0; i < kMost / kGroups; ++i)
    v[i] = grp + i * kGroups < S ? *reinterpret_cast<const f32x4*>(pp + (int64_t)(grp + i * kGroups) * D) : f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kMost / kGroups; ++i)
    if (grp + i * kGroups < S) sum += v[i] * factor[grp + i * kGroups];
  *reinterpret_cast<f32x4*>(&sums[grp][ch]) = sum;
  __syncthreads();
  if (there && row >= 0 && tid < D) {
    float num = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) num += sums[g][tid];
    Elem<T>::store(static_cast<T*>(pa.out) + (row * G + m % G) * D + tid, joined(num, total));
  }
}

// ---------------------------------------------------------------- chunks of many query rows

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct ChunkParams {
  int G, causal;
  float scale_log2;
};

template <bool E4M3, int D>
struct ChunkGeom {
  // 64 channels: four waves, so that two workgroups share a compute unit and one's start and end overlap the other's work
  // (102 -> 96 us with a window of 512 rows over 4096 tokens, e4m3 turns of conversations 161 -> 147; 128 channels would
  // need 2 x 137 KB of LDS)
  static constexpr int kWaveQ = 32, kWaves = D / 16, kBlockQ = kWaveQ * kWaves;  // query rows of a wave, of a workgroup
  static constexpr int kStage = 64;                     // cache rows of a ring slot
  static constexpr int kBring = kStage / kWaves;        // of them from each wave: 8 or 16
  static constexpr int kRowB = D * 2;                   // bytes of a row in LDS: bf16
  static constexpr int kEight = 8 * kRowB + (E4M3 && D == 64 ? 0 : 128);  // bytes of eight rows
  static constexpr int kSlotK = kStage / 8 * kEight;        // keys of a slot; its values lie behind them
  static constexpr int kSlot = 2 * kSlotK;
  static constexpr int kDepth = 4;
  static constexpr int kAux = kStage * 3;               // words of a slot: count, later its logarithm, key scale, value scale of a row
  static constexpr int kRaw = kStage * D;               // e4m3: bytes of a stage's keys as they come, values behind them
  static constexpr int kMarks = (D + 63) / 64;          // words of a lane
  static constexpr int kLds = kDepth * (kSlot + kAux * 4 + 8) + kWaves * 64 * kMarks * 4, kLdsE4m3 = kLds + 2 * kRaw;
  // Rows lie in LDS in groups of four, the group's 16-byte pieces one behind the other, each of them for its four
  // rows; every other group has its neighbouring pieces swapped, and 128 bytes stay free behind every other one.
  // Sixteen rows' reads of one piece (keys), and four rows' reads of four neighbouring pieces (values), then meet all
  // 256 bytes that the banks give in a cycle.  (Keys without the free bytes: 8 cycles a read for 4, and 533 us for 528
  // of 2048 x 7 query rows behind 16 384 rows; an e4m3 cache waits for its conversions and has no gain from them.)
  __device__ static int place(int row, int piece) {
    const int odd = (row >> 2) & 1;
    return (row >> 3) * kEight + odd * (4 * kRowB) + ((piece ^ odd) * 4 + (row & 3)) * 16;
  }
};

// A wave holds 32 query rows in registers, a workgroup of eight waves 256 (64 channels: of four, 128); the cache's rows come through a ring of
// 64-row slots in LDS.  Per 32 rows of the cache, on 32x32 matrix tiles:
//   logits   S[key][query]     = K . Q^T      (lane: query = lane % 32; keys (i & 3) + 8 (i >> 2) + 4 (lane / 32))
//   values   O[channel][query] += V^T . P     (P as the lane has it: the product's key order is that of S; V^T by
//                                              transposing reads of four keys)
// Softmax: weights relative to a reference 2^8 above the largest weight at the time that it was set, which follows only
// when a logit passes it (results are quotients of two sums with the same reference): then, and only then, the sums are
// rescaled.  So no weight is larger than one, as in paged_rows_kernel, and a sum overflows where that of the values'
// magnitudes does.  (With the largest weight itself as the reference, followed 2^8 later, 300 rows of 2^118 gave
// infinities; the time is the same.  The other end: the weights of e4m3 rows whose scale is below 2^-118 are denormal.)
// The three parts work on different rows in one turn of the loop -- the logits of the next 32, the weights of these, the
// values of those before -- so that matrix and vector pipes are both busy.
// bf16 weights are rounded once (2^-8 of a weight at the most): two terms as for single tokens would cost as many
// matrix instructions again where these are the bound.
// Bound: matrix and vector pipes, which a SIMD's two waves keep busy in turn.  2048 x 7 query rows of 4 units behind 16 384 rows:
// 523 to 542 us, 978 to 944 TFLOP/s (a library product of 8192^3: 1253); without the exponentials 3 % less, without either product
// 5 to 13 %: no single part holds it up.
template <bool E4M3, int D>
__global__ __launch_bounds__(D * 4, 2) void paged_chunk_kernel(ChunkParams kp, PagedAttend pa, int q_blocks) {
  using A = ChunkGeom<E4M3, D>;
  constexpr int NK = D / 16, CB = D / 32;
  extern __shared__ __align__(16) unsigned char ring[];
  float* aux_all = reinterpret_cast<float*>(ring + A::kDepth * A::kSlot);
  unsigned char* flag_all = reinterpret_cast<unsigned char*>(aux_all + A::kDepth * A::kAux);
  // results that are NaN because their query sees a value that is not finite, a bit each (rarely any: not in registers)
  uint32_t* marks = reinterpret_cast<uint32_t*>(flag_all + A::kDepth * 8) + threadIdx.x * A::kMarks;
  unsigned char* raw_all = flag_all + A::kDepth * 8 + A::kWaves * 64 * A::kMarks * 4;  // (16-byte aligned)
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, h = lane >> 5;
  int u, part_of;
  if (!map_block(pa.pg.n_units, q_blocks * pa.splits, u, part_of)) return;
  const int qb = q_blocks - 1 - part_of / pa.splits, sp = part_of % pa.splits;  // (blocks that see most rows first)
  const int G = kp.G;
  const UnitRows ur(pa.pg, pa.rw, u);
  const int m0 = qb * A::kBlockQ, m_all = ur.n * G;
  if (m0 >= m_all) return;
  const int m1 = min(m_all, m0 + A::kBlockQ);
  const TileRange range = tiles_of<A::kStage>(ur.start + m0 / G, ur.start + (m1 - 1) / G, ur.end, kp.causal, pa.window, pa.sinks);
  // this workgroup's share of the stages
  const int per = (range.n_tiles + pa.splits - 1) / pa.splits;
  const int s_begin = min(range.n_tiles, sp * per), n_stages = min(range.n_tiles, s_begin + per) - s_begin;

  const float c = kp.scale_log2;
  const int32_t* cu = pa.count ? pa.count + (size_t)u * pa.count_pitch : nullptr;
  // the wave's queries
  const int w0 = m0 + wv * A::kWaveQ;
  const int w_lo = ur.start + min(w0, m_all - 1) / G, w_hi = ur.start + min(w0 + A::kWaveQ - 1, m_all - 1) / G;
  bf16x8 q[NK];
  int qi;
  {
    const int m = w0 + c32, t = m / G;
    const int64_t at = m < m1 ? array_row(pa.rw, ur.first, t) : -1;
    qi = ur.start + t;
    const uint16_t* qp = static_cast<const uint16_t*>(pa.Q) + ((at < 0 ? 0 : at) * G + (at < 0 ? 0 : m % G)) * D + h * 8;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(qp + k * 16);
      q[k] = __builtin_bit_cast(bf16x8, at < 0 ? u32x4{0u, 0u, 0u, 0u} : v);
    }
  }

  // ---- the ring: wave wv brings rows [kBring wv, kBring wv + kBring) of a stage, all of one page
  constexpr int kBring = A::kBring;
  auto stage_row = [&](int s) { return range.tile(s_begin + s) * A::kStage; };
  constexpr int EL = E4M3 ? 1 : 2, ROWB = D * EL;
  // Page of the wave's rows of stage 64 k + lane: one load for 64 stages.  (Looked up at its stage, each entry made
  // the whole wave wait for it.)
  int entries = -1;
  auto load_entries = [&](int s0) {
    const int s = s0 + lane, r = stage_row(s) + wv * kBring;
    entries = -1;
    if (s < n_stages && r < ur.end) entries = pa.pg.table ? pa.pg.table[(int64_t)u * pa.pg.table_pitch + (r >> pa.pg.shift)] : u;
    asm volatile("" : "+v"(entries));  // (the wait for them here, or every stage waits for all loads under way before it reads one)
  };
  struct Place {
    int64_t at;  // pool row of the first of the wave's rows of a stage
    int rows;    // how many are there
  };
  auto find = [&](int s, int r_stage) {
    const int e = __builtin_amdgcn_readlane(entries, s & 63), r = r_stage + wv * kBring;
    Place p{0, 0};
    if ((unsigned)e < (unsigned)pa.pg.n_pages) p = Place{e * pa.pg.pitch + (r & pa.pg.mask), min(kBring, ur.end - r)};
    // (bit o of a stage's eight bytes: row o of it is there; read by all waves a stage before its own)
    typedef typename std::conditional<kBring == 8, uint8_t, uint16_t>::type Flags;
    if (lane == 0) reinterpret_cast<Flags*>(flag_all + (s & (A::kDepth - 1)) * 8)[wv] = (Flags)((1 << p.rows) - 1);
    return p;
  };
  auto rsrc_of = [&](const void* base, int64_t at, int bytes) {  // words of a buffer descriptor
    const uint64_t p = reinterpret_cast<uint64_t>(base) + at;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)p), (uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32) & 0xffff),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
  };
  auto buffer = [&](const void* base, int64_t at, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<unsigned char*>(const_cast<void*>(base)) + at, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000u);
  };
  // (places in LDS as numbers: a generic pointer is tested for null at every use)
  const int ring_lds = __builtin_amdgcn_readfirstlane((int)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring);
  // Waits and barriers for the written-out loads: to the compiler they touch no memory, and it may move reads and writes of
  // LDS over them unless it is told.
  auto wait_for = [](auto what) {
    asm volatile("" ::: "memory");
    what();
    asm volatile("" ::: "memory");
  };
  // Loads to LDS, written out: m0 holds the place (reserved: the compiler keeps nothing there, and nothing else here uses it);
  // between a vector instruction that writes a word of the descriptor and the load that reads it there have to be five wait
  // states, which the compiler does not see to here: the move's and s_nop's four.
  // A kilobyte to LDS, sixteen bytes a lane.  (Written out because the compiler lets every transposing read wait for
  // all such loads that it knows of: as measured when this was written, a chunk of 2048 x 7 query rows behind 16 384 rows took
  // 695 us so and 559 without that wait.  The waits are in `meet`; the loads return no register.)
  auto load_lds = [&](int dst, u32x4 rs, int off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "v"(off), "s"(rs) : "memory");
  };
  // bf16: straight to LDS, a KB an instruction.  Lane -> group of four rows, piece, row of the group as they lie there.
  constexpr int kLoads = kBring * A::kRowB / 1024, kGroupLanes = D / 2;   // instructions of a wave's rows; lanes of a group
  auto load_rows = [&](int dst, const unsigned char* pool, const Place& p) {
    static_assert(kLoads == 2, "");
    int to[2], off[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int grp = j * (64 / kGroupLanes) + lane / kGroupLanes;
      const int piece = (lane % kGroupLanes) / 4 ^ (grp & 1);
      to[j] = __builtin_amdgcn_readfirstlane(dst + j * 1024 / (8 * A::kRowB) * A::kEight + j * 1024 % (8 * A::kRowB));
      off[j] = (grp * 4 + lane % 4) * ROWB + piece * 16;
    }
    // (both in one, so that the wait states are taken once)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds"
                 ::"s"(to[0]), "s"(to[1]), "v"(off[0]), "v"(off[1]), "s"(rsrc_of(pool, p.at * ROWB, p.rows * ROWB)) : "memory");
  };
  auto slot_at = [&](int s) { return ring + (s & (A::kDepth - 1)) * A::kSlot; };
  auto slot_lds = [&](int s) { return ring_lds + (s & (A::kDepth - 1)) * A::kSlot; };
  constexpr int kAuxAt = A::kDepth * A::kSlot, kRawAt = kAuxAt + A::kDepth * (A::kAux * 4 + 8) + A::kWaves * 64 * A::kMarks * 4;
  auto load_counts = [&](int s, int r_stage) {  // of a stage's rows, by one of the waves
    if (s >= n_stages || r_stage >= pa.count_pitch || wv != (s & (A::kWaves - 1))) return;
    const u32x4 rs = rsrc_of(cu, (int64_t)r_stage * 4, min(pa.count_pitch - r_stage, A::kStage) * 4);  // (behind them: 0, which counts as one)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(ring_lds + kAuxAt + (s & (A::kDepth - 1)) * A::kAux * 4)),
                 "v"(lane * 4), "s"(rs) : "memory");
  };
  // Counts of stage s into their logarithms, a stage before it: by the wave that asked for them, once they are there (bf16:
  // `meet` has waited, e4m3: commit).
  auto convert_counts = [&](int s) {
    if (s >= n_stages || stage_row(s) >= pa.count_pitch || wv != (s & (A::kWaves - 1))) return;
    float* at = aux_all + (s & (A::kDepth - 1)) * A::kAux + lane;
    asm volatile("" ::: "memory");
    *at = __builtin_amdgcn_logf((float)max((int)__float_as_uint(*at), 1));
  };
  auto load_keys = [&](int s, int r_stage, const Place& p) {
    if (cu) load_counts(s, r_stage);
    load_rows(slot_lds(s) + wv * (kBring / 8 * A::kEight), pa.pg.K, p);
  };
  auto load_values = [&](int s, const Place& p) { load_rows(slot_lds(s) + A::kSlotK + wv * (kBring / 8 * A::kEight), pa.pg.V, p); };
  // e4m3: sixteen bytes a lane to a place of the wave's own in LDS, a stage later from there into the ring as bf16
  // (held in registers until then they made the wave spill others).  Lane l brings piece l / kBring of row l % kBring: eight lanes
  // then write 128 bytes of the ring that lie together (a row's lanes next to each other: an eight-way bank conflict).
  static_assert(kBring * D == 64 * 16, "");
  uint32_t a_ks = 0u, a_vs = 0u;                    // scales of the wave's row lane % kBring
  auto issue = [&](int s) {
    const int r_stage = stage_row(s);
    const Place p = find(s, r_stage);
    if (cu) load_counts(s, r_stage);
    wait_for([] { __builtin_amdgcn_s_waitcnt(0xc07f); });  // lgkmcnt(0): what commit read from there has been read
    const int off = lane % kBring * ROWB + lane / kBring * 16;
    load_lds(ring_lds + kRawAt + wv * 1024, rsrc_of(pa.pg.K, p.at * ROWB, p.rows * ROWB), off);
    load_lds(ring_lds + kRawAt + A::kRaw + wv * 1024, rsrc_of(pa.pg.V, p.at * ROWB, p.rows * ROWB), off);
    a_ks = __builtin_amdgcn_raw_buffer_load_b32(buffer(pa.pg.K_scale, p.at * 4, p.rows * 4), lane % kBring * 4, 0, 0);   // (behind the rows: 0)
    a_vs = __builtin_amdgcn_raw_buffer_load_b32(buffer(pa.pg.V_scale, p.at * 4, p.rows * 4), lane % kBring * 4, 0, 0);
  };
  auto commit = [&](int s) {
    wait_for([] { __builtin_amdgcn_s_waitcnt(0x0f70); });  // vmcnt(0)
    const u32x4 ek = *reinterpret_cast<const u32x4*>(raw_all + wv * 1024 + lane * 16);
    const u32x4 ev = *reinterpret_cast<const u32x4*>(raw_all + A::kRaw + wv * 1024 + lane * 16);
    float* aux = aux_all + (s & (A::kDepth - 1)) * A::kAux + wv * kBring;
    const float ks = __uint_as_float(a_ks) * c, vs = __uint_as_float(a_vs);
    if (lane < kBring) {
      aux[A::kStage + lane] = ks;
      aux[2 * A::kStage + lane] = fabsf(vs) < __builtin_inff() ? vs : 0.f;
    }
    if (cu) convert_counts(s);
    unsigned char* slot = slot_at(s);
    const int r = wv * kBring + lane % kBring, piece = lane / kBring * 2;
    // a row of values whose scale is not finite lies there as a row of NaN with a scale of zero
    const bool lost = !(fabsf(vs) < __builtin_inff());
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      u32x4 k, v;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        k[w] = e4m3_to_bf16(ek[2 * e + w / 2], w & 1);
        v[w] = lost ? 0x7fc07fc0u : e4m3_to_bf16(ev[2 * e + w / 2], w & 1);
      }
      *reinterpret_cast<u32x4*>(slot + A::place(r, piece + e)) = k;
      *reinterpret_cast<u32x4*>(slot + A::kSlotK + A::place(r, piece + e)) = v;
    }
  };
  // Between stages: every wave's rows that the next one reads have landed, and it reads none of those that will be
  // written over.  bf16: the loads of the stage that ends here may still be under way.
  auto meet = [&]() {
    wait_for([] {
      __builtin_amdgcn_s_waitcnt(E4M3 ? 0xc07f : 0x0070 | 2 * kLoads);  // lgkmcnt(0), and vmcnt(2 kLoads)
      __builtin_amdgcn_s_barrier();
    });
  };

  // ---- operands of 32 rows: tile t, half t & 1 of stage t / 2
  const int k_at = A::place(c32, h);  // (piece 2 ks + h: the swap moves bit 0 alone)
  const int i16 = lane & 15, half16 = (lane >> 4) & 1;
  const int v_at = A::place(4 * h + (i16 >> 2), 2 * half16 + ((i16 & 3) >> 1)) + 8 * (i16 & 1);
  // (a tile is named by its stage's place in the ring, in slots, and its half)
  auto load_k = [&](bf16x8 (&a)[NK], int place, int half) {
    const unsigned char* p = ring + place * A::kSlot + half * 4 * A::kEight + k_at;
#pragma unroll
    for (int k = 0; k < NK; ++k) a[k] = *reinterpret_cast<const bf16x8*>(p + k * 128);
  };
  auto load_v = [&](bf16x8 (&a)[2], int place, int half, int cb) {
    const unsigned char* p = ring + place * A::kSlot + A::kSlotK + half * 4 * A::kEight + v_at;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      union { s16x4 s[2]; bf16x8 b; } x;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        x.s[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)(p + (2 * m + e) * A::kEight + cb * 256));
      a[m] = x.b;
    }
  };
  constexpr float kHeadroom = 8.f;
  f32x16 acc[CB], s[2];  // s[t & 1]: logits of tile t
  bf16x8 p[2][2];        // p[t & 1]: weights of tile t
  float ref = 0.f, l = 0.f;
  float limit = kNegInf;            // exponents above it make the reference follow: zero, -inf before the first that is seen
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    marks[cb / 2] = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[cb][i] = 0.f;
  }
  // words of a tile's rows: what 0 logarithms of counts, 1 key scales, 2 value scales
  auto aux_of = [&](int place, int half, int what) { return aux_all + place * A::kAux + what * A::kStage + half * 32 + 4 * h; };
  // some query of the wave does not see some row of the 32 from r on, though the row is there
  auto edge = [&](int r) {
    return (kp.causal && r + 31 > w_lo) || (pa.window > 0 && r <= w_hi - pa.window && r + 32 > pa.sinks);
  };
  // Bit (i & 3) + 8 (i >> 2): the lane's query sees the row of its element i, of the 32 from r on.
  auto seen_bits = [&](int r) { return seen_rows(r, qi, kp.causal, pa.window, pa.sinks) >> (4 * h); };
  auto elem_mask = [](uint32_t bits, int i) { return bit_mask(bits, (i & 3) + 8 * (i >> 2)); };
  auto logits = [&](f32x16& o, const bf16x8 (&a)[NK]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[k], q[k], o, 0, 0, 0);
  };
  auto values = [&](const bf16x8 (&a)[2], const bf16x8 (&w)[2], int cb) {
#pragma unroll
    for (int m = 0; m < 2; ++m) acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[m], w[m], acc[cb], 0, 0, 0);
  };
  // Are a tile's values all finite? (The largest of their bits says so. One answer for all column blocks of a stage's half,
  // not one each in clean: 103 us for 108 with a window of 512 rows over 4096 tokens. An e4m3 cache pays for the registers
  // with spills, 218 to 230 us for 212 over sixteen turns of conversations, and keeps clean's own.)
  auto all_finite = [&](const bf16x8 (&v)[CB][2]) {
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < CB * 8; ++i)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, __builtin_bit_cast(u32x4, v[i / 8][i / 4 % 2])[i % 4] & 0x7fff7fffu));
    return __any(most[0] >= 0x7f80 || most[1] >= 0x7f80) == 0;
  };
  // A tile that some query does not see whole: values that are not finite out of the product, and marks for those
  // that see one.
  auto clean = [&](bf16x8 (&a)[2], uint32_t bits, int cb) {  // (bits: seen_bits of the tile; rows that are not there hold zeros)
    uint32_t odd = 0u;  // (bits 15 and 31 alone: see not_finite2)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= (__builtin_bit_cast(u32x4, a[m])[e] & 0x7f807f80u) + 0x00800080u;
    if (!__any((odd & 0x80008000u) != 0u)) return;
    f32x16 seen;
#pragma unroll
    for (int i = 0; i < 16; ++i) seen[i] = 0.f;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      u32x4 see;
#pragma unroll
      for (int e = 0; e < 4; ++e) see[e] = (elem_mask(bits, 8 * m + 2 * e) & 0x3f80u) | (elem_mask(bits, 8 * m + 2 * e + 1) & 0x3f800000u);
      u32x4 w = __builtin_bit_cast(u32x4, a[m]), bad;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t n = not_finite2(w[e]);
        bad[e] = n * 0x3f80u;  // one or zero
        w[e] &= ~(n * 0xffffu);
      }
      a[m] = __builtin_bit_cast(bf16x8, w);
      seen = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, see), seen, 0, 0, 0);
    }
    uint32_t mark = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) mark |= min(__float_as_uint(seen[i]), 1u) << (16 * (cb & 1) + i);
    marks[cb / 2] |= mark;
    __builtin_amdgcn_sched_barrier(0);  // (or all blocks' temporaries live at once)
  };
  // Exponents of tile t, in place of its logits ...
  auto exponents = [&](int place, int half, f32x16& x) {
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      f32x4 ck = {c, c, c, c};
      if constexpr (E4M3) ck = *reinterpret_cast<const f32x4*>(aux_of(place, half, 1) + 8 * i4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i4 + e] = __builtin_fmaf(x[4 * i4 + e], ck[e], -ref);
    }
  };
  // ... and where a query does not see every row or a row has a count.
  auto mask = [&](int place, int half, int r, f32x16& x, uint32_t here, bool counted) {
    if (counted) {
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 bias = *reinterpret_cast<const f32x4*>(aux_of(place, half, 0) + 8 * i4);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i4 + e] += bias[e];
      }
    }
    const uint32_t bits = seen_bits(r) & (here >> (4 * h));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = masked(x[i], elem_mask(bits, i));
  };
  // The reference follows; the result is what the sums so far are to be multiplied with.
  auto follow = [&](f32x16& x, float mx) {
    const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false));
    const float top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    const float d = top > limit ? top + kHeadroom : 0.f;
    const float corr = limit == kNegInf ? 1.f : __builtin_amdgcn_exp2f(-d);
    if (top > limit) limit = 0.f;
    ref += d;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] -= d;
    return corr;
  };
  auto rescale = [&](float corr) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[cb][i] *= corr;
  };
  // Weights from exponents, and their sum.
  auto weights = [&](int place, int half, const f32x16& x, bf16x8 (&w)[2]) {
    float sum = 0.f;
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      f32x4 vs;
      if constexpr (E4M3) vs = *reinterpret_cast<const f32x4*>(aux_of(place, half, 2) + 8 * i4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y = __builtin_amdgcn_exp2f(x[4 * i4 + e]);
        sum += y;
        if constexpr (E4M3) y *= vs[e];  // (finite, see commit: the weight of a row that is not seen stays zero)
        w[i4 / 2][4 * (i4 % 2) + e] = (__bf16)y;
      }
    }
    return sum;
  };

  if (n_stages > 0) {
    // Keys are requested three stages ahead and values two: turn t reads keys of tile t + 2 and values of tile t - 1.
    load_entries(0);
    Place next_v;
    if constexpr (E4M3) {
      issue(0);
      commit(0);
      issue(1);
      commit(1);
      issue(2);
    } else {
      const Place p0 = find(0, stage_row(0)), p1 = find(1, stage_row(1));
      load_keys(0, stage_row(0), p0);
      load_values(0, p0);
      load_keys(1, stage_row(1), p1);
      next_v = find(2, stage_row(2));
      load_keys(2, stage_row(2), next_v);
      load_values(1, p1);
    }
    meet();
    if constexpr (!E4M3)
      if (cu) {
        convert_counts(0);
        meet();
      }
    bf16x8 a[NK];
    load_k(a, 0, 0);
    logits(s[0], a);
    load_k(a, 0, 1);
    auto flags_of = [&](int place) { return *reinterpret_cast<const u32x2*>(flag_all + place * 8); };
    u32x2 flag_next = flags_of(0);
    // (Behind the last tile lie zeros; in front of the first, weights of zero meet the first tile's own values.)
    int r_prev = -1;             // first row of the tile before
    bool edge_prev = true, grown_prev = false;
    float corr = 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[1][0][e] = p[1][1][e] = (__bf16)0.f;
    for (int st = 0; st < n_stages; ++st) {
      if (st > 0) meet();
      const int place = st & (A::kDepth - 1), after = (st + 1) & (A::kDepth - 1), before = st > 0 ? (st - 1) & (A::kDepth - 1) : 0;
      const int r_stage = stage_row(st);
      const uint32_t here[2] = {(uint32_t)__builtin_amdgcn_readfirstlane((int)flag_next[0]), (uint32_t)__builtin_amdgcn_readfirstlane((int)flag_next[1])};
      flag_next = flags_of(after);
      const bool counted = cu && r_stage < pa.count_pitch;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = r_stage + 32 * half;
        const bool at_edge = edge(r);
        bf16x8 v[CB][2];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) load_v(v[cb], half ? place : before, half ^ (st > 0 || half), cb);
        logits(s[half ^ 1], a);
        // what brings rows, while the matrix cores work on the logits
        if (half == (E4M3 ? 1 : 0)) {
          if (((st + 3) & 63) == 0) load_entries(st + 3);
          if constexpr (E4M3) {
            commit(st + 2);
            issue(st + 3);
          } else {
            const int r_next = stage_row(st + 3);
            const Place next_k = find(st + 3, r_next);
            load_keys(st + 3, r_next, next_k);
            load_values(st + 2, next_v);
            next_v = next_k;
            if (cu) convert_counts(st + 1);
          }
        }
        exponents(place, half, s[half]);
        if (at_edge || counted || here[half] != ~0u) mask(place, half, r, s[half], here[half], counted);
        float mx = s[half][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[half][i]);
        if (edge_prev || grown_prev) {
          if (grown_prev) rescale(corr);
          if (edge_prev && (E4M3 || !all_finite(v))) {
            const uint32_t bits = r_prev < 0 ? 0u : seen_bits(r_prev);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) clean(v[cb], bits, cb);
          }
        }
        grown_prev = __any(mx > limit) != 0;  // some query's exponents have passed its reference, or are its first:
        if (grown_prev) corr = follow(s[half], mx);  // its sums follow when this tile's values join them
        load_k(a, after, half);
        // (bf16: 552 -> 543 us for 2048 x 7 query rows behind 16 384 rows; e4m3, whose waves convert rows meanwhile, lost)
        if constexpr (!E4M3) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) values(v[cb], p[half ^ 1], cb);
        float ps = weights(place, half, s[half], p[half]);
        asm volatile("" : "+v"(ps));  // (or the weights move behind the branch below, away from the products they run beside)
#pragma unroll
        for (int k = 0; k < 2 * CB; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);            // a matrix instruction,
          __builtin_amdgcn_sched_group_barrier(0x100, NK / (2 * CB), 0);  // key reads,
          __builtin_amdgcn_sched_group_barrier(0x400, 16 / (2 * CB), 0);  // exponentials
          __builtin_amdgcn_sched_group_barrier(0x002, 24 / (2 * CB) + 1, 0);
        }
        if constexpr (!E4M3) __builtin_amdgcn_s_setprio(0);
        l = __builtin_fmaf(l, grown_prev ? corr : 1.f, ps);
        edge_prev = at_edge;
        r_prev = r;
      }
    }
    wait_for([] { __builtin_amdgcn_s_waitcnt(0x0f70); });  // vmcnt(0): the requests of stages behind the last
    if (grown_prev) rescale(corr);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      bf16x8 v[2];
      load_v(v, (n_stages - 1) & (A::kDepth - 1), 1, cb);
      if (edge_prev) clean(v, seen_bits(r_prev), cb);
      values(v, p[1], cb);
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const uint32_t mark = marks[cb / 2];
#pragma unroll
      for (int i = 0; i < 16; ++i)  // (all ones: a NaN)
        acc[cb][i] = __uint_as_float(__float_as_uint(acc[cb][i]) | bit_mask(mark, 16 * (cb & 1) + i));
    }
  }

  const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false));
  const float den = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  const int m = w0 + c32;
  if (m >= m1) return;
  if (pa.splits == 1) {
    const int64_t at = array_row(pa.rw, ur.first, m / G);
    if (at < 0) return;
    const float inv = den == 0.f ? 1.f : 1.f / den;   // (nothing seen: the sums are zero)
    uint16_t* o = static_cast<uint16_t*>(pa.out) + (at * G + m % G) * D + 4 * h;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        u32x2 w;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          w[e] = (uint32_t)float_to_bf16_bits(acc[cb][4 * i4 + 2 * e] * inv) | (uint32_t)float_to_bf16_bits(acc[cb][4 * i4 + 2 * e + 1] * inv) << 16;
        *reinterpret_cast<u32x2*>(o + cb * 32 + 8 * i4) = w;
      }
  } else {
    const int64_t at = ((int64_t)u * pa.rw.max_n * G + m) * pa.splits + sp;
    float* pp = pa.part + at * D + 4 * h;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        *reinterpret_cast<f32x4*>(pp + cb * 32 + 8 * i4) = f32x4{acc[cb][4 * i4], acc[cb][4 * i4 + 1], acc[cb][4 * i4 + 2], acc[cb][4 * i4 + 3]};
    if (h == 0) part_state(pa, G, D)[at] = f32x2{limit == kNegInf ? kNegInf : ref, den};
  }
}

template <bool E4M3, int D>
hipError_t launch_chunk(const KParams& kp, const PagedAttend& pa, hipStream_t st) {
  using A = ChunkGeom<E4M3, D>;
  const int q_blocks = (int)(((int64_t)pa.rw.max_n * kp.G + A::kBlockQ - 1) / A::kBlockQ);
  static LdsLimitOnce lim;
  const hipError_t e = lim.ensure(reinterpret_cast<const void*>(&paged_chunk_kernel<E4M3, D>), 160 * 1024);
  if (e != hipSuccess) return e;
  paged_chunk_kernel<E4M3, D><<<dim3(mapped_blocks(pa.pg.n_units, q_blocks * pa.splits)), dim3(A::kWaves * 64), E4M3 ? A::kLdsE4m3 : A::kLds, st>>>(ChunkParams{kp.G, kp.causal, kp.scale_log2}, pa, q_blocks);
  return hipSuccess;
}

template <typename T, bool E4M3, int D, int NQ, int WAVES, bool NT>
hipError_t launch_rows_as(const KParams& kp, const PagedAttend& pa, hipStream_t st) {
  const int q_blocks = (int)(((int64_t)pa.rw.max_n * kp.G + NQ * kCols - 1) / (NQ * kCols));
  const int lds = WAVES * (32 + 2 * kCols + kCols * (D + 4)) * (int)sizeof(float);
  static LdsLimitOnce lim;  // one per instantiation
  const hipError_t e = lim.ensure(reinterpret_cast<const void*>(&paged_rows_kernel<T, E4M3, D, NQ, WAVES, NT>), 160 * 1024);
  if (e != hipSuccess) return e;
  paged_rows_kernel<T, E4M3, D, NQ, WAVES, NT><<<dim3(mapped_blocks(pa.pg.n_units, q_blocks * pa.splits)), dim3(WAVES * 64), lds, st>>>(kp, pa, q_blocks);
  return hipSuccess;
}

// Which form of the rows kernel (us, 128 channels, 4 heads a unit, e4m3 unless noted):
//   two groups of 16 query rows instead of one from 17 query rows on: 5 tokens of 256 bf16 units of 1500 rows 43.9 for 47.0 (64 units,
//     whose rows the caches hold for the second group: 20.5 for 19.0)
//   four waves where there are more workgroups than compute units, else eight: 1024 units of 600 rows 38.4 / 49.2, 300 of
//     2100 46.1 / 51.3, 512 52.8 / 55.8; 256 31.5 / 30.6
//   non-temporal loads from 64 MB of rows on, which a program's other layers push out of the caches before the next step: 256
//     units of 2100 rows, six caches in turn, 29.1 for 30.8, 128 bf16 units of 1500 22.9 for 24.8, 512 bf16 units of 2100 86.2
//     for 96.8 (one cache alone, which stays there: 27.9 for 27.0, 23.0 for 23.2)
template <typename T, bool E4M3, int D>
hipError_t launch_rows(const KParams& kp, const PagedAttend& pa, int64_t bytes, hipStream_t st) {
  const int64_t m = (int64_t)pa.rw.max_n * kp.G;
  constexpr bool kTwo = sizeof(T) == 2 || D == 64;  // (fp32, 128 channels: two groups do not fit the registers)
  const bool two = kTwo && m > kCols, nt = bytes > (64ll << 20);
  const int64_t groups = (int64_t)pa.pg.n_units * ((m + (two ? 2 : 1) * kCols - 1) / ((two ? 2 : 1) * kCols)) * pa.splits;
  auto go = [&](auto f) { return f(kp, pa, st); };
  if constexpr (kTwo)
    if (two) return go(&launch_rows_as<T, E4M3, D, 2, 8, false>);
  if (groups > 256) return nt ? go(&launch_rows_as<T, E4M3, D, 1, 4, true>) : go(&launch_rows_as<T, E4M3, D, 1, 4, false>);
  return nt ? go(&launch_rows_as<T, E4M3, D, 1, 8, true>) : go(&launch_rows_as<T, E4M3, D, 1, 8, false>);
}

template <typename T, int D>
hipError_t launch_combine(const KParams& kp, const PagedAttend& pa, hipStream_t st) {
  const int64_t rows = (int64_t)pa.pg.n_units * pa.rw.max_n * kp.G;
  constexpr int kRows = 256 / (D / 4);
  if (pa.splits > kFewSplits) paged_combine_kernel<T, D><<<dim3((unsigned)rows), dim3(256), 0, st>>>(kp.G, pa);
  else if (pa.splits > 1)
    paged_combine_few_kernel<T, D><<<dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(256), 0, st>>>(kp.G, pa, rows);
  return hipGetLastError();
}

}  // namespace

// Blocks of queries that a launch may have: below 2^32 threads.
constexpr int64_t kMostBlocks = 1 << 22;
static int64_t query_blocks(const KParams& kp, int n_units, int max_n, int64_t block) {
  return (int64_t)n_units * (((int64_t)max_n * kp.G + block - 1) / block);
}
bool paged_fits(const KParams& kp, int n_units, int max_n) {
  return query_blocks(kp, n_units, max_n, kp.dtype == CASK_F32 ? kCols : 256) <= kMostBlocks;
}

// Which kernel, and how many workgroups share the rows of a block of queries.  By what a call takes, as measured (us):
// rounds of the 256 compute units, each `start` + `row` for every row that a workgroup goes through; with splits 4 for
// the launch that adds them and their results' way to memory and back at 4 TB/s.
//   query rows                 start   us per 1000 rows, 128 / 64 channels
//   up to 16 query rows          4       9 / 5      (4 units of 32 768 rows 15 in all; 512 of 2100 52)
//   up to 32                     4      15.5 / 9    (64 units of 4000 rows, 64 query rows 41; 256 of 1500 55)
//   the same, fp32               4      32 / 32
//   256, bf16 / e4m3             6      36 / 45 (both 128 channels)
//   128, bf16 / e4m3             6      23 / 27 (both 64 channels, two workgroups a compute unit)
// The form of 256 query rows is slower per row of the cache and takes eight times as many queries along: 4 units of
// 30 000 rows with 128 / 192 / 256 query rows each 38 / 47 / 53 by 32, 35 / 37 / 40 by 256; 64 of 500 19 / 34 / 36 and
// 33 / 38 / 44; 256 of 1500 with 64 / 96 / 128 55 / 78 / 101 and 55 / 56 / 57.
PagedPlan paged_plan(const KParams& kp, int n_units, int max_n, bool e4m3, int window, int sinks, int max_rows) {
  const int64_t m = (int64_t)max_n * kp.G;
  const bool f32 = kp.dtype == CASK_F32, wide = kp.d == 128;
  auto cost = [&](int64_t block, int slots, int least, double start, double per_row, int* splits) {
    const int64_t blocks = query_blocks(kp, n_units, max_n, block);
    int64_t rows = max_rows;
    const int64_t tokens = (block < m ? block : m) / kp.G + 1;
    if (window > 0 && window + tokens + sinks < rows) rows = window + tokens + sinks;
    double best = 0.0;
    for (int s = 1; s <= kMostSplits && (s == 1 || rows >= (int64_t)s * least); ++s) {
      if (s > 1 && (blocks * s > kMostBlocks || n_units * m > kMostBlocks)) break;
      double c = (double)((blocks * s + slots - 1) / slots) * (start + per_row * 1e-3 * (double)((rows + s - 1) / s));
      if (s > 1) c += 4.0 + (double)n_units * m * s * kp.d * 8.0 / 4.0e6;
      if (s == 1 || c < best) best = c, *splits = s;
    }
    return best;
  };
  PagedPlan few{false, 1}, many{true, 1};
  const bool two = m > kCols && (!f32 || !wide);
  const double c_few = cost(two ? 2 * kCols : kCols, 256, 256, 4.0, f32 ? 32.0 : two ? (wide ? 15.5 : 9.0) : (wide ? 9.0 : 5.0), &few.splits);
  const bool ask_many = (kp.path_flags & CASK_PATH_PAGED_MANY) != 0, ask_few = (kp.path_flags & CASK_PATH_PAGED_FEW) != 0;
  const bool few_fit = query_blocks(kp, n_units, max_n, kCols) <= kMostBlocks;
  if (f32 || (few_fit && (ask_few || (m <= 2 * kCols && !ask_many)))) return few;
  const double c_many = cost(wide ? 256 : 128, wide ? 256 : 512, 128, 6.0, wide ? (e4m3 ? 45.0 : 36.0) : (e4m3 ? 27.0 : 23.0), &many.splits);
  return c_many < c_few || ask_many || !few_fit ? many : few;
}

size_t paged_part_bytes(const KParams& kp, int n_units, int max_n, int splits) {
  return splits <= 1 ? 0 : (size_t)n_units * max_n * kp.G * splits * (kp.d + 2) * sizeof(float);
}

hipError_t launch_attend_paged(const KParams& kp, const PagedAttend& pa, bool chunk, bool e4m3, int max_rows, hipStream_t st) {
  int64_t rows = max_rows;  // what a unit's queries see, at the most
  if (pa.window > 0 && (int64_t)pa.window + pa.rw.max_n + pa.sinks < rows) rows = (int64_t)pa.window + pa.rw.max_n + pa.sinks;
  const int64_t bytes = pa.pg.n_units * rows * 2 * kp.d * (e4m3 ? 1 : kp.dtype == CASK_F32 ? 4 : 2);
  hipError_t e;
  if (chunk) {
    if (kp.d == 64) e = e4m3 ? launch_chunk<true, 64>(kp, pa, st) : launch_chunk<false, 64>(kp, pa, st);
    else e = e4m3 ? launch_chunk<true, 128>(kp, pa, st) : launch_chunk<false, 128>(kp, pa, st);
  } else {
#define CASK_PA(T, D) e = e4m3 ? launch_rows<T, true, D>(kp, pa, bytes, st) : launch_rows<T, false, D>(kp, pa, bytes, st)
    if (kp.dtype == CASK_F32) {
      if (kp.d == 64) CASK_PA(float, 64); else CASK_PA(float, 128);
    } else {
      if (kp.d == 64) CASK_PA(uint16_t, 64); else CASK_PA(uint16_t, 128);
    }
#undef CASK_PA
  }
  if (e != hipSuccess) return e;
  if (kp.dtype == CASK_F32) return kp.d == 64 ? launch_combine<float, 64>(kp, pa, st) : launch_combine<float, 128>(kp, pa, st);
  return kp.d == 64 ? launch_combine<uint16_t, 64>(kp, pa, st) : launch_combine<uint16_t, 128>(kp, pa, st);
}

}  // namespace cask
