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
template <int WORDS>
__device__ inline Words<WORDS> load_words(__amdgpu_buffer_rsrc_t rs, int off, int soff) {
  Words<WORDS> r;
  if constexpr (WORDS == 4) {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rs, off, soff, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) r.w[e] = v[e];
  } else if constexpr (WORDS == 2) {
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rs, off, soff, 0);
    r.w[0] = v[0];
    r.w[1] = v[1];
  } else {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, soff, 0);
  }
  return r;
}

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
template <typename T, bool E4M3, int D, int NQ, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void paged_rows_kernel(KParams kp, PagedAttend pa, int q_blocks) {
  using A = RowsGeom<T, E4M3, D>;
  constexpr int TR = A::kTileRows, KEYS = A::kKeys, SUB = A::kSub, NB = A::kBlocks, EPV = A::EPV, NV = A::kValLoads;
  constexpr int kAccPitch = D + 4;
  constexpr int ROWB = D * A::kEl;
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
  bool there[SUB];  // the subtile has a page
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
      for (int i = 0; i < A::kPieces; ++i) ka[y][i] = load_words<A::kPieceWords>(rs, k_off, i * (4 * A::kPieceEl * A::kEl));
      if constexpr (E4M3) ks4[y] = sub_scales(pa.pg.K_scale, row[y]);
      there[y] = row[y] >= 0;
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
          va[y * 4 + j][i] = load_words<A::kValWords>(rs, v_off + j * ROWB, i * (16 * EPV * A::kEl));
      if constexpr (E4M3) vs4[y] = sub_scales(pa.pg.V_scale, row[y]);
    }
  };

  float m_run[NQ], l_run[NQ];
  f32x4 acc[NQ][NB];  // acc[n][b][r] = O[channel(b, 4 g + r)][query n, l16]
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = kNegInf;
    l_run[n] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int t0 = sp * WAVES + wv; t0 < range.n_tiles; t0 += step) {
    const int t = range.tile(t0);
    int64_t row[SUB];
#pragma unroll
    for (int y = 0; y < SUB; ++y) row[y] = sub_row(t, y);
    load_keys(t, row);
    load_values(t, row);
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
    // values that are not finite, in a tile that some query does not see whole
    bool odd = false;
    if (!all) {
      if constexpr (A::kBf16) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int k2 = 0; k2 < 4; ++k2)
            odd |= (vb[b][k2] & 0x7f80u) == 0x7f80u || (vb[b][k2] & 0x7f800000u) == 0x7f800000u;
      } else {
#pragma unroll
        for (int j = 0; j < KEYS; ++j)
#pragma unroll
          for (int b = 0; b < NB; ++b) odd |= !(fabsf(vf[j][b]) < __builtin_inff());
      }
      odd = __any(odd);
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      f32x4 s[SUB];
#pragma unroll
      for (int y = 0; y < SUB; ++y) {
        s[y] = f32x4{0.f, 0.f, 0.f, 0.f};
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
              s[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw),
                                                             __builtin_bit_cast(bf16x8, q[n][i * A::kPieceQ + e]), s[y], 0, 0, 0);
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
          s[y] = chain[0];
        }
        if constexpr (E4M3) s[y] *= ks4[y];
      }
      // s[y][r] = <key 16 y + 4 g + r, query l16>
      float p[KEYS], mx = kNegInf;
      bool sees[KEYS];
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        sees[j] = true;
        if (!all) {
          const int r = t * TR + (j >> 2) * 16 + g * 4 + (j & 3);
          sees[j] = there[j >> 2] && r < ur.end && (!kp.causal || r <= qi[n]) && (pa.window <= 0 || r > qi[n] - pa.window || r < pa.sinks);
        }
        p[j] = sees[j] ? __builtin_fmaf(s[j >> 2][j & 3], c, bias4[j >> 2][j & 3]) : kNegInf;
        mx = fmaxf(mx, p[j]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m_run[n], mx);
      const float ref = mn == kNegInf ? 0.f : mn;  // (a query that has seen no row yet)
      const float corr = exp2_from(m_run[n], ref);
      float ps = 0.f;
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        if constexpr (A::kBf16) p[j] = exp2_from(p[j], ref);
        else p[j] = sees[j] ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 2][j & 3], c, bias4[j >> 2][j & 3] - ref)) : 0.f;  // (the logit meets its reference inside one rounding)
        ps += p[j];
        if constexpr (E4M3) p[j] = sees[j] ? p[j] * vs4[j >> 2][j & 3] : 0.f;
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
        if (!odd) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vb[b]), ph, acc[n][b], 0, 0, 0);
            acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vb[b]), pl, acc[n][b], 0, 0, 0);
          }
        } else {
          bf16x8 see8;
#pragma unroll
          for (int j = 0; j < 8; ++j) see8[j] = (__bf16)(sees[j] ? 1.f : 0.f);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            bf16x8 fin, bad;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float x = __uint_as_float(j & 1 ? vb[b][j >> 1] & 0xffff0000u : vb[b][j >> 1] << 16);
              const bool ok = fabsf(x) < __builtin_inff();
              fin[j] = (__bf16)(ok ? x : 0.f);
              bad[j] = (__bf16)(ok ? 0.f : 1.f);
            }
            acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fin, ph, acc[n][b], 0, 0, 0);
            acc[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fin, pl, acc[n][b], 0, 0, 0);
            const f32x4 seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, see8, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (seen[r] > 0.f) acc[n][b][r] = __builtin_nanf("");
          }
        }
      } else {
        // (a tile's products are summed on their own: the long sum has as many addends as there are tiles)
#pragma unroll
        for (int b0 = 0; b0 < NB; b0 += 4) {
          f32x4 a[4];
#pragma unroll
          for (int j = 0; j < KEYS; ++j)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              float x = vf[j][b0 + b];
              if (odd) x = fabsf(x) < __builtin_inff() ? x : 0.f;
              a[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p[j], j ? a[b] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
#pragma unroll
          for (int b = 0; b < 4; ++b) acc[n][b0 + b] += a[b];
        }
        if (odd) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            f32x4 seen = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
              seen = __builtin_amdgcn_mfma_f32_16x16x4f32(fabsf(vf[j][b]) < __builtin_inff() ? 0.f : 1.f, sees[j] ? 1.f : 0.f, seen, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (seen[r] > 0.f) acc[n][b][r] = __builtin_nanf("");
          }
        }
      }
    }
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
    for (int b = 0; b < NB; ++b)
      *reinterpret_cast<f32x4*>(&st_acc[(wv * kCols + l16) * kAccPitch + b * 16 + g * 4]) = acc[n][b];
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
      } else {  // [unit][query row][split]: D sums, then the reference and the denominator
        float* pp = pa.part + (((int64_t)u * pa.rw.max_n * G + m) * pa.splits + sp) * (D + 2);
        pp[ch] = num;
        if (ch == 0) {
          pp[D] = top;
          pp[D + 1] = den;
        }
      }
    }
    __syncthreads();
  }
}

// Adds the splits of a query row in their order.  D threads per row.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_combine_kernel(int G, PagedAttend pa) {
  const int64_t o = (int64_t)blockIdx.x * (256 / D) + threadIdx.x / D;
  const int ch = threadIdx.x % D;
  const int64_t per_unit = (int64_t)pa.rw.max_n * G;
  if (o >= per_unit * pa.pg.n_units) return;
  const int u = (int)(o / per_unit), m = (int)(o % per_unit);
  if (m >= rows_of_unit(pa.rw, u) * G) return;
  const int64_t row = array_row(pa.rw, first_of_unit(pa.rw, u), m / G);
  if (row < 0) return;
  const float* pp = pa.part + o * pa.splits * (D + 2);
  float mx = kNegInf, num = 0.f, den = 0.f;
  for (int s = 0; s < pa.splits; ++s) {
    const float* ps = pp + (int64_t)s * (D + 2);
    const float pm = ps[D], mn = fmaxf(mx, pm);
    const float fa = share(mx, mn), fb = share(pm, mn);
    den = __builtin_fmaf(den, fa, ps[D + 1] * fb);
    num = __builtin_fmaf(num, fa, ps[ch] * fb);
    mx = mn;
  }
  Elem<T>::store(static_cast<T*>(pa.out) + (row * G + m % G) * D + ch, joined(num, den));
}

template <typename T, bool E4M3, int D, int NQ, int WAVES>
hipError_t launch_rows(const KParams& kp, const PagedAttend& pa, hipStream_t st) {
  const int q_blocks = (int)(((int64_t)pa.rw.max_n * kp.G + NQ * kCols - 1) / (NQ * kCols));
  const int lds = WAVES * (32 + 2 * kCols + kCols * (D + 4)) * (int)sizeof(float);
  static LdsLimitOnce lim;  // one per instantiation
  const hipError_t e = lim.ensure(reinterpret_cast<const void*>(&paged_rows_kernel<T, E4M3, D, NQ, WAVES>), 160 * 1024);
  if (e != hipSuccess) return e;
  paged_rows_kernel<T, E4M3, D, NQ, WAVES><<<dim3(mapped_blocks(pa.pg.n_units, q_blocks * pa.splits)), dim3(WAVES * 64), lds, st>>>(kp, pa, q_blocks);
  if (pa.splits > 1) {
    const int64_t rows = (int64_t)pa.pg.n_units * pa.rw.max_n * kp.G;
    paged_combine_kernel<T, D><<<dim3((unsigned)((rows + 256 / D - 1) / (256 / D))), dim3(256), 0, st>>>(kp.G, pa);
  }
  return hipGetLastError();
}

}  // namespace

int paged_splits(const KParams& kp, int n_units, int max_n, bool e4m3, int window, int sinks, int max_rows) {
  (void)e4m3;
  const int64_t blocks = (int64_t)n_units * (((int64_t)max_n * kp.G + kCols - 1) / kCols);
  int64_t rows = max_rows;
  if (window > 0) rows = rows < (int64_t)window + max_n + sinks ? rows : (int64_t)window + max_n + sinks;
  const int tile = kp.dtype == CASK_BF16 ? 32 : 16;
  const int rounds = (int)((rows + tile * 8 - 1) / (tile * 8));
  if (blocks > 128 || rounds < 4) return 1;
  int s = (int)(256 / blocks);
  if (s > rounds / 2) s = rounds / 2;
  return s > 64 ? 64 : (s < 1 ? 1 : s);
}

size_t paged_part_bytes(const KParams& kp, int n_units, int max_n, int splits) {
  return splits <= 1 ? 0 : (size_t)n_units * max_n * kp.G * splits * (kp.d + 2) * sizeof(float);
}

hipError_t launch_attend_paged(const KParams& kp, const PagedAttend& pa, bool e4m3, hipStream_t st) {
#define CASK_PA(T, D) return e4m3 ? launch_rows<T, true, D, 1, 8>(kp, pa, st) : launch_rows<T, false, D, 1, 8>(kp, pa, st)
  if (kp.dtype == CASK_F32) {
    if (kp.d == 64) CASK_PA(float, 64); else CASK_PA(float, 128);
  } else {
    if (kp.d == 64) CASK_PA(uint16_t, 64); else CASK_PA(uint16_t, 128);
  }
#undef CASK_PA
}

}  // namespace cask
