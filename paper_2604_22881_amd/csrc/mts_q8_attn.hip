// Incremental attention over the 8-bit pool (mts_q8.hpp), query heads sharing key heads:
//   out[i, h] = sum_j softmax_j(sm_scale * q[i, h] . K[j, h / G]) V[j, h / G],  j in [0, prefix + i].
//
// The query rows of a (user, key head) are its new tokens times the G query heads of the key head.  Of few rows a workgroup takes a
// tile of 16 or 32 and a stretch of the user's keys, its four wavefronts every fourth tile of 32 keys, each with all the rows;
// their sums are joined through LDS.  Of many (128 and more) it takes 128, 32 a wavefront, and all go through the same keys.
// Where the keys are cut into several stretches (a few rows behind a long history would leave most of the chip idle) a second
// kernel joins them.
//
// Operand flow: S^T = K Q^T in bf16 and O^T = V^T P^T in fp16.  A code times its row's power of two is a bf16 value, so the
// logits are those of the stored values with fp32 sums; rows of K meet that power in the conversion.  S^T leaves a lane with
// tokens of one query, the ones whose codes of V it holds (16x16x32 instructions, few rows) or reads (32x32x16, many).
//
// V's power of two e varies along the index that P V sums over, so it goes to the weight: with references Y of the logits
// (base 2) and E, both of them per query and wavefront,
//   w_j = 2^(y_j - Y + e_j - E),  O = sum w_j code_j,  l = sum w_j 2^(E - e_j),  out = 2^E O / l.
// Y is some largest y_j and E some largest y_j - Y + e_j, so that a large row of V which nothing weighs takes no bits from the others.
// w is rounded to fp16 for the product (11 bits, half a step 2^-12: next to it the output's own rounding to bf16, 2^-9, is
// what counts) and taken into l unrounded; weights are scaled so that the references' own is 2^8 and nothing above 2^-22 of it
// is below fp16's normal numbers.  Y and E move only when some w would leave fp16, and all sums are then scaled.  y_j - Y is one fma; where logits are so large that their rounding is a matter of whole powers of two, the
// product is rounded first, as the reference was, so that the largest logit's weight is the reference's.  fp32 rows: queries as three bf16 parts, weights as two
// fp16 ones, which keep 24 and 22 bits.
//
// Bound: few rows, reading K and V once (2 (D + 1) bytes a token); many, the vector instructions beside the products (per weight
// an fma, an addition, a maximum, an exponential, an fma and half a conversion, and per code of the tile half a conversion
// that the tile's rows share).  Measured: 32 users' single tokens behind 6-16 K keys x 8 heads of 128, 722 MB, 130 us with its
// join (5.6 TB/s); first visits of 4096 tokens x 8 users x 8 (2 query heads each) of 128, 550 GFLOP, 665 us (827 TFLOP/s).
#include <type_traits>

#include "mts_internal.hpp"
#include "mts_q8.hpp"

namespace mts {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// log2 of the weight of the references, and of the largest, which fp16's 65504 bounds.  The room between them is for later keys
// that weigh more, for which all sums would be scaled; below the references, fp16's half step of 2^-25 is 2^-33 of theirs.
// us a call with 5, 7, 9 bits of room: 8 first visits of 4096 x 8 (2 query heads each) of 128 706, 682, 666; 120 users' 48 rows x 5
// (8) of 64 in fp32 45.6, 44.9, 44.4.
constexpr float kRef = 8.f;
constexpr float kMost = 15.99f;
// A reference is a rounded logit, an fma's product is not: up to this size the two differ by 1/4 at most.
constexpr float kFused = 4194304.f;
constexpr float kNoExp = (float)(kQ8ExpMin + 127);   // what keys without a row count as
constexpr float kLog2e = 1.44269504088896340736f;

struct Q8AttnArgs {
  Q8Geom      g;
  const char* q;
  char*       out;
  BatchDev    b;
  float       scale;               // sm_scale * log2(e)
  int32_t     G;                   // query heads of a key head
  // of the launch, as in Q8AttnLaunch
  int32_t     above, upto;
  int32_t     q_tiles;
  bool        by_rank;
  int32_t     chunk_shift;
  int32_t     part_rows;
  int32_t     user_rows;
  int64_t     slots;
  float*      part_o;              // [item][part_rows][D]
  float*      part_ml;             // [item][part_rows][2]
};

// a product that no later addition is fused with
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename F>
__device__ __forceinline__ float over_groups(float v, F f) {       // the four lanes of a query
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Where a user's rows and keys lie, from the tables; what does not fit the host's bounds is cut to them.
constexpr int kMostKeys = 1 << 30;  // of a user
struct UserSpan {
  int row0, n;                     // first row and rows of the step's tokens
  int prefix;
  int page0;                       // its page list
  int held;                        // tokens its pages hold
};
__device__ __forceinline__ UserSpan user_span(const BatchDev& b, int S, int u) {
  UserSpan s;
  s.row0 = min(max(b.new_indptr[u], 0), b.total_new);
  s.n = min(max(min(b.new_indptr[u + 1], b.total_new) - s.row0, 0), b.max_new);
  s.prefix = min(max(b.prefix_lens[u], 0), kMostKeys);
  s.page0 = min(max(b.page_indptr[u], 0), b.total_pages);
  s.held = min(max(min(b.page_indptr[u + 1], b.total_pages) - s.page0, 0), kMostKeys / S) * S;
  return s;
}
// keys that a tile's last row sees
__device__ __forceinline__ int keys_of(const UserSpan& s, int last_row, int G) {
  return min(s.prefix + min(last_row / G, kMostKeys - 1) + 1, s.held);
}

// The codes of one granule as a matrix operand: 8 dims of K times the row's power of two; 4 + 4 keys of V of one dim.
__device__ __forceinline__ bf16x8 k_operand(uint32_t a, uint32_t b, float scale) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true));
  return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ u32x2 v_values(uint32_t a) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true))};
}
// byte r of a word of exponent bytes as e + 127 and as 2^-e
__device__ __forceinline__ float exp_of(uint32_t w, int r) { return (float)((w >> (8 * r)) & 255u); }
__device__ __forceinline__ float inverse_of(uint32_t w, int r) { return __uint_as_float((254u - ((w >> (8 * r)) & 255u)) << 23); }
// 0xff where a byte is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return top | (top - (top >> 7));
}

// A wavefront's query rows and sums.
template <int D, int MT, typename T>
struct Attn {
  static constexpr int GB = D >= 64 ? 16 : 8;          // bytes of a lane's granule
  static constexpr int NJ = D >= 64 ? D / 64 : 1;      // granules of a row / 4
  static constexpr int NE = GB / 8;                    // matrix steps of a granule
  static constexpr int KS = NJ * NE;
  static constexpr int W = GB / 4;                     // 16-dim tiles of a granule of V
  static constexpr int DT = D / 16;
  static constexpr bool kF32 = std::is_same<T, float>::value;
  static constexpr int QP = kF32 ? 3 : 1, PP = kF32 ? 2 : 1;
  using Granule = typename std::conditional<GB == 16, u32x4, u32x2>::type;

  bf16x8 q[MT][KS][QP];
  f32x4  o[MT][DT];
  float  neg_y[MT];                // -(Y - kRef)
  float  neg_r[MT];                // the same less E, for a fused subtraction
  float  E[MT];                    // + 127
  float  l[MT];                    // sums of this lane's keys, times 2^(127 - E)
  bool   first;                    // no keys yet
  bool   huge;                     // some reference is beyond what an fma may be exact to

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      neg_y[m] = neg_r[m] = l[m] = 0.f;
      E[m] = kNoExp;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    first = true;
    huge = false;
  }

  __device__ __forceinline__ void load_queries(int mt, const char* row, int grp) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = (s / NE) * 4 * GB + grp * GB + (s % NE) * 8;
      if constexpr (kF32) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + d * 4), b = *reinterpret_cast<const f32x4*>(row + d * 4 + 16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = j < 4 ? a[j & 3] : b[j & 3];
          const __bf16 h = (__bf16)x;
          const float r = x - (float)h;
          const __bf16 m = (__bf16)r;
          q[mt][s][0][j] = h;
          q[mt][s][1 % QP][j] = m;
          q[mt][s][2 % QP][j] = (__bf16)(r - (float)m);
        }
      } else {
        q[mt][s][0] = *reinterpret_cast<const bf16x8*>(row + d * 2);
      }
    }
  }

  // One tile of 32 keys, the first of them key0, in the parts that a wavefront goes through.  A lane's accumulators hold keys key0
  // + 16 h + 4 grp + r of query lane & 15; ef, iv: e + 127 and 2^-e of these keys of V; `edge`: some row does not see all keys of the
  // tile; lim: the last key that this lane's query sees.
  using Scores = f32x4[2][MT];
  using Weights = f16x8[MT][PP];

  template <typename K>
  __device__ __forceinline__ void scores(K&& k_op, Scores& s) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int m = 0; m < MT; ++m) s[h][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const bf16x8 k = k_op(h, i);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int p = QP - 1; p >= 0; --p) s[h][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[m][i][p], s[h][m], 0, 0, 0);
      }
    }
  }

  // x: log2 of the weights, if no reference moves
  __device__ __forceinline__ void weigh(const Scores& s, const float (&ef)[2][4], float scale, Scores& x) const {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[h][m][r] = __builtin_fmaf(s[h][m][r], scale, neg_r[m]) + ef[h][r];
  }
  __device__ __forceinline__ void hide(int key0, const int (&lim)[MT], int grp, Scores& x) const {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[h][m][r] = key0 + 16 * h + 4 * grp + r > lim[m] ? -__builtin_inff() : x[h][m][r];
  }
  __device__ __forceinline__ bool over(const Scores& x) const {
    float most = -__builtin_inff();
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) most = fmaxf(most, x[h][m][r]);
    return first || huge || __any(most > kMost);
  }
  // References that hold for this tile too, and the sums scaled to them.
  __device__ __forceinline__ void move_references(const Scores& s, const float (&ef)[2][4], int key0, bool edge, const int (&lim)[MT],
                                                  float scale, int grp, Scores& x) {
    float largest = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float y = -__builtin_inff(), py[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          py[h][r] = edge && key0 + 16 * h + 4 * grp + r > lim[m] ? -__builtin_inff() : rounded_product(s[h][m][r], scale);
          y = fmaxf(y, py[h][r]);
        }
      y = over_groups(y, [](float a, float b) { return fmaxf(a, b); });
      // a query that sees none of the tile keeps its references (0 and the least at first: its sums are 0)
      const float was = neg_y[m], e_was = E[m];
      const bool seen = y > -__builtin_inff();
      const float now = seen ? (first ? kRef - y : fminf(was, kRef - y)) : was;
      float e = kNoExp;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) e = fmaxf(e, (py[h][r] + now) + (ef[h][r] - kRef));
      e = over_groups(e, [](float a, float b) { return fmaxf(a, b); });
      E[m] = first ? e : fmaxf(e, e_was + (now - was));
      const float f = first ? 0.f : exp2_of((now - was) + (e_was - E[m]));
      neg_y[m] = now;
      neg_r[m] = now - E[m];
      l[m] *= f;
#pragma unroll
      for (int c = 0; c < DT; ++c) o[m][c] *= f;
      largest = fmaxf(largest, __builtin_fabsf(now));
    }
    huge = __any(largest > kFused);
    first = false;
    if (huge) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[h][m][r] = (rounded_product(s[h][m][r], scale) + neg_y[m]) + (ef[h][r] - E[m]);
    } else {
      weigh(s, ef, scale, x);
    }
    if (edge) hide(key0, lim, grp, x);
  }
  __device__ __forceinline__ void weights(const Scores& x, const float (&iv)[2][4], Weights& p) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = exp2_of(x[h][m][r]);
          l[m] = __builtin_fmaf(w[r], iv[h][r], l[m]);
        }
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const f16x2 a = __builtin_convertvector((f32x2{w[r], w[r + 1]}), f16x2);
          p[m][0][4 * h + r] = a[0];
          p[m][0][4 * h + r + 1] = a[1];
          if constexpr (PP == 2) {
            const f16x2 b = __builtin_convertvector((f32x2{w[r] - (float)a[0], w[r + 1] - (float)a[1]}), f16x2);
            p[m][PP - 1][4 * h + r] = b[0];
            p[m][PP - 1][4 * h + r + 1] = b[1];
          }
        }
      }
  }
  template <typename V>
  __device__ __forceinline__ void add_products(V&& v_op, const Weights& p) {
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      const f16x8 v = v_op(c);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = PP - 1; i >= 0; --i) o[m][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[m][i], o[m][c], 0, 0, 0);
    }
  }

  // NaN in V among keys that not all rows see: their codes were left out of the products (0 * NaN would reach every row), and are
  // brought in here, key by key for the queries that see it.  v: the codes of the lane's granules, of both sub-blocks.
  __device__ __forceinline__ void add_nan(const Granule (&v)[2][NJ], int key0, const int (&lim)[MT], int grp) {
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
      const bool mine = grp == ((key >> 2) & 3);
      uint32_t byte[DT], any = 0;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        byte[c] = ((key < 16 ? v[0][c / W][c % W] : v[1][c / W][c % W]) >> (8 * (key & 3))) & 0x7fu;
        any |= mine && byte[c] == 0x7fu;
      }
      if (!__any(any)) continue;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        const u32x4 a{mine && byte[c] == 0x7fu ? 0x7e00u : 0u, 0u, 0u, 0u}, one{0x3c00u, 0u, 0u, 0u};
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, one), o[m][c], 0, 0, 0);
          o[m][c] = key0 + key <= lim[m] ? n : o[m][c];
        }
      }
    }
  }

  // sum of the weights over all keys, in units of the output's
  __device__ __forceinline__ float total(int m) const {
    return over_groups(l[m], [](float a, float b) { return a + b; }) * exp2_of(E[m] - 127.f);
  }
};

// bytes of the first n of four keys
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// What a workgroup is to do: a tile of M rows of user u's head h from row_first on, keys [key_first, key_last).  Workgroups are
// numbered head after head inside
//   kUsers:  user, tile of rows                             few rows, keys not cut
//   kKeys:   stretch of keys of all users, tile of rows     few rows: stretches of user u start at its first page's tokens / 2^shift + u
//   kRows:   tile of rows of all users                      many rows: tiles of user u start at its first row / M + u, the last first
//                                                           (by_rank: the last tiles of all users, then those before them, ..)
//   kBoth:   stretch of a user's keys, tile of all users    many rows of few users, keys cut
// so that both the stretches and the tiles of users of unlike size follow one another with one place per user left over at most,
// and a place's user is found from a table that never falls.
enum class Numbered { kUsers, kKeys, kRows, kBoth };
struct Work {
  UserSpan us;
  int64_t  item;
  int      h, row_first, row_last;
  int      key_first, key_last;
  int      keys;                   // of the whole tile of rows
  bool     partial;                // one of several stretches
};
template <int M>
__device__ __forceinline__ int64_t first_tile(const Q8AttnArgs& a, int u) { return (int64_t)a.b.new_indptr[u] * a.G / M + u; }
// the place of the tile that `back` others of the user come behind, and the other way round
template <int M>
__device__ __forceinline__ int64_t tile_place(const Q8AttnArgs& a, int u, int64_t back) {
  return a.by_rank ? back * a.b.batch + u : first_tile<M>(a, u) + back;
}
template <int M>
__device__ __forceinline__ int64_t tile_at(const Q8AttnArgs& a, int64_t place, int& u) {
  if (a.by_rank) {
    u = (int)(place % a.b.batch);
    return place / a.b.batch;
  }
  u = find_user(a.b.batch, place, [&](int s) -> int64_t { return first_tile<M>(a, s); });
  return place - first_tile<M>(a, u);
}
__device__ __forceinline__ int64_t first_stretch(const Q8AttnArgs& a, int u) {
  return (((int64_t)a.b.page_indptr[u] * a.g.S) >> a.chunk_shift) + u;
}
template <int M, Numbered N>
__device__ __forceinline__ bool find_work(const Q8AttnArgs& a, Work& w) {
  constexpr bool kCut = N == Numbered::kKeys || N == Numbered::kBoth, kAllTiles = N == Numbered::kRows || N == Numbered::kBoth;
  const uint32_t place = blockIdx.x / (uint32_t)a.g.H;
  w.h = (int)(blockIdx.x % (uint32_t)a.g.H);
  w.item = blockIdx.x;
  int64_t chunk = 0, qt;
  int u;
  if constexpr (kAllTiles) {
    const int64_t tile = N == Numbered::kBoth ? place % (uint32_t)a.slots : place;
    if constexpr (N == Numbered::kBoth) chunk = place / (uint32_t)a.slots;
    qt = tile_at<M>(a, tile, u);
  } else {
    qt = place % (uint32_t)a.q_tiles;
    const int64_t slot = place / (uint32_t)a.q_tiles;
    u = (int)slot;
    if constexpr (N == Numbered::kKeys) {
      u = find_user(a.b.batch, slot, [&](int s) -> int64_t { return first_stretch(a, s); });
      chunk = slot - first_stretch(a, u);
    }
  }
  w.us = user_span(a.b, a.g.S, u);
  const int64_t rows = (int64_t)w.us.n * a.G;
  if (rows <= a.above || rows > a.upto) return false;        // another launch's
  if constexpr (kAllTiles) qt = (rows + M - 1) / M - 1 - qt;
  const int64_t first = qt * M;
  if (first < 0 || first >= rows || chunk < 0 || chunk > (kMostKeys >> a.chunk_shift)) return false;
  w.row_first = (int)first;
  w.row_last = (int)(first + M < rows ? first + M : rows) - 1;
  w.keys = keys_of(w.us, w.row_last, a.G);
  w.key_first = kCut ? (int)(chunk << a.chunk_shift) : 0;
  if (w.key_first >= w.keys) return false;
  w.partial = kCut && w.keys > (1 << a.chunk_shift);
  w.key_last = w.partial ? min(w.key_first + (1 << a.chunk_shift), w.keys) : w.keys;
  return true;
}
// index of a query row among [total_new][Hq]
__device__ __forceinline__ int64_t row_at(const Q8AttnArgs& a, const Work& w, int row) {
  return ((int64_t)(w.us.row0 + row / a.G) * a.g.H + w.h) * a.G + row % a.G;
}
// Where a user's 16-token sub-blocks lie.  The page ids of 64 neighbouring ones are kept in the lanes: a scalar load each would
// share a counter with the LDS reads, which would then wait for one another.  A sub-block behind the last is the last, a page
// that is none is page 0.
template <int D>
struct SubBlocks {
  const char* head;                // the head's block of page 0
  const int*  pages;
  uint32_t    page_bytes, num_pages;
  int         shift, S, last, have;   // have: the sub-blocks (have, have + 63) are in the lanes
  int         id;
  __device__ __forceinline__ SubBlocks(const Q8AttnArgs& a, const Work& w)
      : head(a.g.layer_base + w.h * q8_head_bytes(a.g.S, D)), pages(a.b.page_indices + w.us.page0), page_bytes((uint32_t)a.g.page_bytes),
        num_pages((uint32_t)a.g.num_pages), shift(a.g.sub_shift), S(a.g.S), last((w.keys + 15) / 16 - 1), have(-64), id(0) {}
  // Both sub-blocks of a tile are among the same 64.
  __device__ __forceinline__ void look_up(int tile) {
    const int from = 2 * tile & ~63;
    if (from == have) return;
    have = from;
    const uint32_t p = (uint32_t)pages[min(from + (int)(threadIdx.x & 63), last) >> shift];
    id = (int)(p < num_pages ? p : 0u);
  }
  struct At { const char *k, *ke; };
  __device__ __forceinline__ At at(int sub) const {
    sub = min(sub, last);
    const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(id, sub & 63);
    const char* h = head + (uint64_t)page * page_bytes;
    const int in_page = sub & ((1 << shift) - 1);
    return {h + in_page * 16 * D, h + 2 * S * D + in_page * 16};
  }
};
template <bool PAST, typename Granule>
__device__ __forceinline__ Granule load_granule(const char* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const Granule*>(p));
  else return *reinterpret_cast<const Granule*>(p);
}
// Four dims, from d on, of a row's result or, `partial`, of its stretch.
template <int D, typename T>
__device__ __forceinline__ void store_sums(const Q8AttnArgs& a, const Work& w, int row, int d, f32x4 v, float inv) {
  if (w.partial) {
    *reinterpret_cast<f32x4*>(a.part_o + (w.item * a.part_rows + (row - w.row_first)) * D + d) = v;
    return;
  }
  v *= inv;
  const int64_t at = row_at(a, w, row) * D + d;
  if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<f32x4*>(a.out + at * 4) = v;
  } else {
    const bf16x2 lo = __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2), hi = __builtin_convertvector((f32x2{v[2], v[3]}), bf16x2);
    *reinterpret_cast<u32x2*>(a.out + at * 2) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

// Few rows: every wavefront has all of them and every fourth tile of the keys, so that the rows' operands stay in registers, K and V
// go there from memory without a barrier, and a tile of one row costs what 16 do (the products are not what bounds it).  PAST: K and V past the caches' retention, where a
// call reads nothing of them twice (kv_past_caches): 32 users x 10 K keys x 8 heads of 128 141 -> 130 us.
template <int D, int MT, typename T, Numbered N, bool PAST>
__global__ __launch_bounds__(256, (MT == 2 || (D == 128 && std::is_same<T, float>::value)) ? 2 : 3) void q8_attn_kernel(Q8AttnArgs a) {
  using A = Attn<D, MT, T>;
  constexpr int M = 16 * MT;
  const int lane = threadIdx.x & 63, grp = lane >> 4, wave = uniform_int(threadIdx.x >> 6);
  Work wk;
  if (!find_work<M, N>(a, wk)) return;
  const int all_see = wk.us.prefix + wk.row_first / a.G;     // the last key that every row sees

  A c;
  c.start();
  int lim[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = min(wk.row_first + 16 * m + (lane & 15), wk.row_last);   // rows behind the last repeat it and are not stored
    lim[m] = wk.us.prefix + row / a.G;
    c.load_queries(m, a.q + row_at(a, wk, row) * D * (int64_t)sizeof(T), grp);
  }

  struct Tile {
    typename A::Granule k[2][A::NJ], v[2][A::NJ];
    uint32_t ke[2], ve[2];
  };
  SubBlocks<D> subs(a, wk);
  // Of 128 dims one tile is in registers: K of the next is asked for when its operands have been made, V when its own have (two
  // tiles, as of fewer dims, take 34 registers more and a third workgroup from a CU; of 64 dims one tile is 4 to 6 % slower).
  constexpr bool kTwo = D <= 64;
  auto load_k = [&](Tile& t, int tile) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const auto at = subs.at(2 * tile + s);
#pragma unroll
      for (int j = 0; j < A::NJ; ++j) t.k[s][j] = load_granule<PAST, typename A::Granule>(at.k + j * 1024 + lane * A::GB);
      t.ke[s] = *reinterpret_cast<const uint8_t*>(at.ke + (lane & 15));
    }
  };
  auto load_v = [&](Tile& t, int tile) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const auto at = subs.at(2 * tile + s);
#pragma unroll
      for (int j = 0; j < A::NJ; ++j)
        t.v[s][j] = load_granule<PAST, typename A::Granule>(at.k + a.g.S * D + j * 1024 + lane * A::GB);
      t.ve[s] = *reinterpret_cast<const uint32_t*>(at.ke + a.g.S + 4 * grp);
    }
  };
  uint32_t nan_seen = 0;
  auto compute = [&](Tile& t, int tile, int next) {
    const int key0 = tile * 32;
    const bool edge = key0 + 31 > all_see;
    const float ks[2] = {__uint_as_float(t.ke[0] << 23), __uint_as_float(t.ke[1] << 23)};
    typename A::Scores s, x;
    typename A::Weights p;
    c.scores([&](int h, int i) { return k_operand(t.k[h][i / A::NE][2 * (i % A::NE)], t.k[h][i / A::NE][2 * (i % A::NE) + 1], ks[h]); }, s);
    if constexpr (!kTwo) {
      subs.look_up(next);
      load_k(t, next);
    }
    if (edge) {
      // what lies behind the last key is anything
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t keep = first_bytes(wk.key_last - (key0 + 16 * s + 4 * grp));
        t.ve[s] = (t.ve[s] & keep) | ((uint32_t)kNoExp * 0x01010101u & ~keep);
#pragma unroll
        for (int j = 0; j < A::NJ; ++j)
#pragma unroll
          for (int w = 0; w < A::W; ++w) {
            const uint32_t v = t.v[s][j][w] & keep, nan = nan_codes(v);
            t.v[s][j][w] = v & ~nan;
            nan_seen |= nan;
          }
      }
    }
    float ef[2][4], iv[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) { ef[s][r] = exp_of(t.ve[s], r); iv[s][r] = inverse_of(t.ve[s], r); }
    c.weigh(s, ef, a.scale, x);
    if (edge) c.hide(key0, lim, grp, x);
    if (c.over(x)) c.move_references(s, ef, key0, edge, lim, a.scale, grp, x);
    c.weights(x, iv, p);
    c.add_products([&](int i) {
      const u32x2 lo = v_values(t.v[0][i / A::W][i % A::W]), hi = v_values(t.v[1][i / A::W][i % A::W]);
      return __builtin_bit_cast(f16x8, (u32x4{lo[0], lo[1], hi[0], hi[1]}));
    }, p);
    if constexpr (!kTwo) load_v(t, next);
  };
  const int tile_end = (wk.key_last + 31) / 32, tile_first = wk.key_first / 32 + wave;
  Tile t0;
  if (tile_first < tile_end) {
    subs.look_up(tile_first);
    load_k(t0, tile_first);
    load_v(t0, tile_first);
    if constexpr (kTwo) {
      Tile t1;
      for (int tile = tile_first;;) {
        const int next = tile + 4;
        subs.look_up(next < tile_end ? next : tile);
        load_k(t1, next < tile_end ? next : tile);
        load_v(t1, next < tile_end ? next : tile);
        compute(t0, tile, next);
        if (next >= tile_end) break;
        tile = next + 4;
        subs.look_up(tile < tile_end ? tile : next);
        load_k(t0, tile < tile_end ? tile : next);
        load_v(t0, tile < tile_end ? tile : next);
        compute(t1, next, tile);
        if (tile >= tile_end) break;
      }
    } else {
      for (int tile = tile_first; tile < tile_end; tile += 4) compute(t0, tile, tile + 4 < tile_end ? tile + 4 : tile);
    }
  }
  if (__any(nan_seen != 0)) {
    for (int again = tile_first; again < tile_end; again += 4)
      if (again * 32 + 31 > all_see) {
        subs.look_up(again);
        load_v(t0, again);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < A::NJ; ++j)
#pragma unroll
            for (int w = 0; w < A::W; ++w) t0.v[s][j][w] &= first_bytes(wk.key_last - (again * 32 + 16 * s + 4 * grp));
        c.add_nan(t0.v, again * 32, lim, grp);
      }
  }

  // The four wavefronts' sums: each takes a quarter of the dims (of 32 dims two take half) from the others.
  constexpr int DT = A::DT, OWNERS = DT < 4 ? DT : 4, OWN = DT / OWNERS;
  __shared__ f32x4 xo[OWNERS * 3 * OWN * MT * 64];
  __shared__ float xy[4][M], xl[4][M], xe[4][M];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const float l = c.total(m);
    if (grp == 0) {
      xy[wave][16 * m + lane] = l == 0.f ? -__builtin_inff() : -c.neg_y[m];   // none of its keys seen
      xl[wave][16 * m + lane] = l;
      xe[wave][16 * m + lane] = c.E[m] - 127.f;
    }
  }
#pragma unroll
  for (int w = 0; w < OWNERS; ++w)
    if (w != wave) {
      const int src = wave - (wave > w);
#pragma unroll
      for (int i = 0; i < OWN; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m) xo[(((w * 3 + src) * OWN + i) * MT + m) * 64 + lane] = c.o[m][w * OWN + i];
    }
  __syncthreads();
  if (wave >= OWNERS) return;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int in_tile = 16 * m + (lane & 15), row = wk.row_first + in_tile;
    float y = xy[0][in_tile];
#pragma unroll
    for (int w = 1; w < 4; ++w) y = fmaxf(y, xy[w][in_tile]);
    const float ref = y > -__builtin_inff() ? y : 0.f;
    float f[4], l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float below = xy[w][in_tile] - ref;
      l = __builtin_fmaf(xl[w][in_tile], exp2_of(below), l);
      f[w] = exp2_of(below + xe[w][in_tile]);
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        f32x4 p;
        if (w == wave) {
          p = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int o = 0; o < OWNERS; ++o)
            if (o == wave) p = c.o[m][o * OWN + i];
        } else {
          p = xo[(((wave * 3 + w - (w > wave)) * OWN + i) * MT + m) * 64 + lane];
        }
        v += p * f[w];
      }
      if (row <= wk.row_last) store_sums<D, T>(a, wk, row, 16 * (wave * OWN + i) + 4 * grp, v, inv);
    }
    if (wk.partial && row <= wk.row_last && wave == 0 && grp == 0)
      *reinterpret_cast<f32x2*>(a.part_ml + (wk.item * a.part_rows + in_tile) * 2) = f32x2{y, l};
  }
}

// Many rows, a wavefront's 32 and its sums, in 32x32x16 products: one query a lane, of each tile the 16 keys 8 b + 4 (lane / 32) + r
// (b, r = 0 .. 3), the lane's accumulators in that order.
template <int D, typename T>
struct Wide {
  static constexpr int KS = D / 16, DT = D / 32;
  static constexpr bool kF32 = std::is_same<T, float>::value;
  static constexpr int QP = kF32 ? 3 : 1, PP = kF32 ? 2 : 1;

  bf16x8 q[KS][QP];
  f32x16 o[DT];
  float  neg_y, neg_r, E, l;       // as Attn's
  bool   first, huge;

  __device__ __forceinline__ void start() {
    neg_y = neg_r = l = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    E = kNoExp;
    first = true;
    huge = false;
  }
  __device__ __forceinline__ void load_queries(const char* row, int hf) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = 16 * s + 8 * hf;
      if constexpr (kF32) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + d * 4), b = *reinterpret_cast<const f32x4*>(row + d * 4 + 16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = j < 4 ? a[j & 3] : b[j & 3];
          const __bf16 h = (__bf16)x;
          const float r = x - (float)h;
          const __bf16 m = (__bf16)r;
          q[s][0][j] = h;
          q[s][1 % QP][j] = m;
          q[s][2 % QP][j] = (__bf16)(r - (float)m);
        }
      } else {
        q[s][0] = *reinterpret_cast<const bf16x8*>(row + d * 2);
      }
    }
  }
  static __device__ __forceinline__ float both_halves_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  __device__ __forceinline__ float total() const {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    return (__uint_as_float(a[0]) + __uint_as_float(a[1])) * exp2_of(E - 127.f);
  }
  static __device__ __forceinline__ int key_of(int r, int hf) { return 8 * (r >> 2) + 4 * hf + (r & 3); }

  // k, v: the tile's operands; ef, iv: e + 127 and 2^-e of its keys of V; `edge`: some row does not see all keys; lim: the last
  // key that this lane's query sees.
  __device__ __forceinline__ void tile(const u32x4 (&k)[KS][64], const u32x4 (&v)[DT][2][64], const float* ef, const float* iv, int key0,
                                       bool edge, int lim, float scale, int lane) {
    const int hf = lane >> 5;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const bf16x8 kk = __builtin_bit_cast(bf16x8, k[i][lane]);
#pragma unroll
      for (int p = QP - 1; p >= 0; --p) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, q[i][p], s, 0, 0, 0);
    }
    float x[16];
    f32x4 e[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) e[b] = *reinterpret_cast<const f32x4*>(ef + 8 * b + 4 * hf);
    auto weigh = [&] {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(s[r], scale, neg_r) + e[r >> 2][r & 3];
    };
    auto hide = [&] {
      if (edge) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = key0 + key_of(r, hf) > lim ? -__builtin_inff() : x[r];
      }
    };
    weigh();
    hide();
    float most = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) most = fmaxf(most, x[r]);
    if (first || huge || __any(most > kMost)) {
      float y = -__builtin_inff();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = edge && key0 + key_of(r, hf) > lim ? -__builtin_inff() : rounded_product(s[r], scale);
        y = fmaxf(y, x[r]);
      }
      y = both_halves_max(y);
      const float was = neg_y, e_was = E;
      const bool seen = y > -__builtin_inff();
      neg_y = seen ? (first ? kRef - y : fminf(was, kRef - y)) : was;
      float e_most = kNoExp;
#pragma unroll
      for (int r = 0; r < 16; ++r) e_most = fmaxf(e_most, (x[r] + neg_y) + (e[r >> 2][r & 3] - kRef));
      e_most = both_halves_max(e_most);
      E = first ? e_most : fmaxf(e_most, e_was + (neg_y - was));
      neg_r = neg_y - E;
      const float f = first ? 0.f : exp2_of((neg_y - was) + (e_was - E));
      l *= f;
#pragma unroll
      for (int c = 0; c < DT; ++c) o[c] *= f;
      huge = __any(__builtin_fabsf(neg_y) > kFused);
      first = false;
      if (huge) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = (rounded_product(s[r], scale) + neg_y) + (e[r >> 2][r & 3] - E);
      } else {
        weigh();
      }
      hide();
    }
    f16x8 p[2][PP];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const f32x4 inv = *reinterpret_cast<const f32x4*>(iv + 8 * b + 4 * hf);
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w[r] = exp2_of(x[4 * b + r]);
        l = __builtin_fmaf(w[r], inv[r], l);
      }
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const f16x2 a = __builtin_convertvector((f32x2{w[r], w[r + 1]}), f16x2);
        p[b >> 1][0][4 * (b & 1) + r] = a[0];
        p[b >> 1][0][4 * (b & 1) + r + 1] = a[1];
        if constexpr (PP == 2) {
          const f16x2 c = __builtin_convertvector((f32x2{w[r] - (float)a[0], w[r + 1] - (float)a[1]}), f16x2);
          p[b >> 1][PP - 1][4 * (b & 1) + r] = c[0];
          p[b >> 1][PP - 1][4 * (b & 1) + r + 1] = c[1];
        }
      }
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        const f16x8 vv = __builtin_bit_cast(f16x8, v[c][sub][lane]);
#pragma unroll
        for (int i = PP - 1; i >= 0; --i) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv, p[sub][i], o[c], 0, 0, 0);
      }
  }

  // As Attn's; v: the codes of V of a 16-token sub-block, of which the first n are keys.
  __device__ __forceinline__ void add_nan(const char* v, int n, int key0, int lim, int lane) {
#pragma unroll 1
    for (int key = 0; key < n; ++key) {
      uint32_t byte[DT], any = 0;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        byte[c] = lane < 32 ? *reinterpret_cast<const uint8_t*>(v + q8_v_sub_index(key, 32 * c + lane, D)) & 0x7fu : 0u;
        any |= byte[c] == 0x7fu;
      }
      if (!__any(any)) continue;
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        const u32x4 a{byte[c] == 0x7fu ? 0x7e00u : 0u, 0u, 0u, 0u}, one{0x3c00u, 0u, 0u, 0u};
        const f32x16 nan = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, one), o[c], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] = key0 + key <= lim ? nan[r] : o[c][r];
      }
    }
  }
};

// Many rows: the wavefronts have 32 rows each and go through the keys together.  Two tiles of 32 keys are converted to operands
// once, K or V of one by each wavefront, into one of two stages in LDS, while the other is multiplied from: codes are converted
// once for 128 rows, and a barrier stands behind 64 keys (behind 32, in 16x16x32 instructions, first visits of 4096 x 8 took 730 us
// where 680).  Of their cycles 51 % are vector instructions, 35 % products.  Workgroups go to the 8
// XCDs in turn, so that with the heads counted first the tiles of a (user, head) meet its keys in one XCD's L2 (8 heads), or two's.
template <int D, typename T, Numbered N>
__global__ __launch_bounds__(256, 2) void q8_attn_wide_kernel(Q8AttnArgs a) {
  using A = Wide<D, T>;
  constexpr int M = 128;
  constexpr int GB = D >= 64 ? 16 : 8, NJ = D >= 64 ? D / 64 : 1, NE = GB / 8, W = GB / 4;   // as Attn's
  using Granule = typename std::conditional<GB == 16, u32x4, u32x2>::type;
  struct Stage {
    u32x4 k[A::KS][64];            // operands, one per lane
    u32x4 v[A::DT][2][64];
    float ef[32], iv[32];
  };
  __shared__ Stage stage[2][2];      // of two tiles each
  __shared__ int nan_seen[2];
  const int lane = threadIdx.x & 63, grp = lane >> 4, wave = uniform_int(threadIdx.x >> 6);
  Work wk;
  if (!find_work<M, N>(a, wk)) return;

  A c;
  c.start();
  const int first_row = wk.row_first + 32 * wave, last_row = min(first_row + 31, wk.row_last);
  const int all_rows_see = wk.us.prefix + wk.row_first / a.G;
  const int all_see = wk.us.prefix + first_row / a.G, some_see = first_row <= wk.row_last ? wk.us.prefix + last_row / a.G : -1;
  const int my_row = first_row + (lane & 31), known_row = min(my_row, wk.row_last);
  const int lim = wk.us.prefix + known_row / a.G;
  c.load_queries(a.q + row_at(a, wk, known_row) * D * (int64_t)sizeof(T), lane >> 5);

  // this wavefront's part of a pair of tiles: K (0, 1) or V (2, 3) of one of the two
  const int my_tile = wave & 1;
  const bool is_v = wave >= 2;
  SubBlocks<D> subs(a, wk);
  struct Raw {
    Granule  g[2][NJ];
    uint32_t e[2];
  };
  const int codes_at = (is_v ? a.g.S * D : 0) + lane * GB, exps_at = (is_v ? a.g.S : 0) + (lane & 15);
  auto load = [&](Raw& r, int pair) {
    const int tile = 2 * pair + my_tile;
    subs.look_up(tile);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const auto at = subs.at(2 * tile + s);
#pragma unroll
      for (int j = 0; j < NJ; ++j) r.g[s][j] = *reinterpret_cast<const Granule*>(at.k + j * 1024 + codes_at);
      r.e[s] = *reinterpret_cast<const uint8_t*>(at.ke + exps_at);
    }
  };
  const int pair_end = (wk.key_last + 63) / 64, pair_first = wk.key_first / 64;
  auto convert = [&](Raw& r, int pair) {
    const int tile = 2 * pair + my_tile;
    Stage& st = stage[(pair - pair_first) & 1][my_tile];
    if (is_v) {
      if (tile * 32 + 31 > all_rows_see) {
        uint32_t any = 0;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int key0 = tile * 32 + 16 * s;
          if (key0 + (lane & 15) >= wk.key_last) r.e[s] = (uint32_t)kNoExp;
          const uint32_t keep = first_bytes(wk.key_last - (key0 + 4 * grp));
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int w = 0; w < W; ++w) {
              const uint32_t v = r.g[s][j][w] & keep, nan = nan_codes(v);
              r.g[s][j][w] = v & ~nan;
              any |= nan;
            }
        }
        if (any) nan_seen[my_tile] = 1;
      }
      // a lane has four keys, group grp of the sub-block, of dim lane % 16 of each 16: of 32 dims' operand half of lane
      // 32 (grp % 2) + the dim
      const int to = 32 * (grp & 1) + (lane & 15);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int w = 0; w < W; ++w)
            reinterpret_cast<u32x2*>(&st.v[j * (W / 2) + w / 2][s][to + 16 * (w & 1)])[grp >> 1] = v_values(r.g[s][j][w]);
        if (lane < 16) {
          st.ef[16 * s + lane] = (float)r.e[s];
          st.iv[16 * s + lane] = inverse_of(r.e[s], 0);
        }
      }
    } else {
      // and of K one token's 8 dims twice, or once
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float scale = __uint_as_float(r.e[s] << 23);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const int eight = (4 * j + grp) * NE + e;        // of the row's eights of dims
            st.k[eight >> 1][32 * (eight & 1) + 16 * s + (lane & 15)] =
                __builtin_bit_cast(u32x4, k_operand(r.g[s][j][2 * e], r.g[s][j][2 * e + 1], scale));
          }
      }
    }
  };
  if (threadIdx.x < 2) nan_seen[threadIdx.x] = 0;
  __syncthreads();
  Raw raw;
  load(raw, pair_first);
  convert(raw, pair_first);
  load(raw, pair_first + 1);
  __syncthreads();
  for (int pair = pair_first; pair < pair_end; ++pair) {
    if (pair + 1 < pair_end) {
      convert(raw, pair + 1);
      load(raw, pair + 2);
    }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      const Stage& st = stage[(pair - pair_first) & 1][i];
      const int key0 = 64 * pair + 32 * i;
      if (key0 <= some_see && key0 < wk.key_last) c.tile(st.k, st.v, st.ef, st.iv, key0, key0 + 31 > all_see, lim, a.scale, lane);
    }
    __syncthreads();
  }
  const int tile_end = (wk.key_last + 31) / 32, tile_first = wk.key_first / 32;
  if (uniform_int(nan_seen[0] | nan_seen[1]) != 0) {
    for (int again = tile_first; again < tile_end; ++again)
      if (again * 32 + 31 > all_rows_see) {
        subs.look_up(again);
#pragma unroll 1
        for (int s = 0; s < 2; ++s)
          c.add_nan(subs.at(2 * again + s).k + a.g.S * D, min(wk.key_last - (again * 32 + 16 * s), 16), again * 32 + 16 * s, lim, lane);
      }
  }
  const float l = c.total(), e = exp2_of(c.E - 127.f);
  if (my_row > wk.row_last) return;
#pragma unroll
  for (int i = 0; i < A::DT; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      store_sums<D, T>(a, wk, my_row, 32 * i + A::key_of(4 * b, lane >> 5),
                       f32x4{c.o[i][4 * b], c.o[i][4 * b + 1], c.o[i][4 * b + 2], c.o[i][4 * b + 3]} * e, 1.f / l);
  if (wk.partial && lane < 32)
    *reinterpret_cast<f32x2*>(a.part_ml + (wk.item * a.part_rows + (my_row - wk.row_first)) * 2) = f32x2{l == 0.f ? -__builtin_inff() : -c.neg_y, l};
}

// Joins the stretches of a row's keys, in an order that only their number decides: one wavefront or four per (user, row, head) of
// few rows (a number that needs no table) or (token, query head) of many, D / 4 lanes to a stretch, so that 2 to 32 of them are
// read at once and a long history's hundreds take no chain of round trips.
template <int D, typename T, int M, Numbered N, int WAVES>
__global__ __launch_bounds__(256) void q8_join_kernel(Q8AttnArgs a) {
  constexpr int L = D / 4, P = 64 / L;                       // lanes of a stretch, stretches of a wavefront
  __shared__ float most[4], xl[4];
  __shared__ f32x4 xo[4][L];
  const int lane = threadIdx.x & 63, wave = uniform_int(threadIdx.x >> 6);
  const int Hq = a.g.H * a.G;
  const uint32_t unit = WAVES == 4 ? blockIdx.x : blockIdx.x * 4 + wave;
  int u, h;
  int64_t row;
  UserSpan us;
  if constexpr (N == Numbered::kKeys) {
    h = (int)(unit % (uint32_t)a.g.H);
    row = unit / (uint32_t)a.g.H % (uint32_t)a.user_rows;
    u = (int)(unit / (uint32_t)a.g.H / (uint32_t)a.user_rows);
    if (u >= a.b.batch) return;
    us = user_span(a.b, a.g.S, u);
  } else {
    const int token = (int)(unit / (uint32_t)Hq), hq = (int)(unit % (uint32_t)Hq);
    if (token >= a.b.total_new) return;
    u = find_user(a.b.batch, token, [&](int s) -> int64_t { return a.b.new_indptr[s]; });
    us = user_span(a.b, a.g.S, u);
    h = hq / a.G;
    row = (int64_t)(token - us.row0) * a.G + hq % a.G;
  }
  const int64_t rows = (int64_t)us.n * a.G;
  if (row < 0 || row >= rows || rows <= a.above || rows > a.upto) return;
  const int64_t qt = row / M, last = (qt + 1) * M < rows ? (qt + 1) * M : rows;
  const int keys = keys_of(us, (int)last - 1, a.G);
  const int chunks = (int)(((int64_t)keys + (1ll << a.chunk_shift) - 1) >> a.chunk_shift);
  if (chunks <= 1) return;
  // the first stretch's place, and places from one to the next
  int64_t place, next;
  if constexpr (N == Numbered::kKeys) {
    const int64_t slot = first_stretch(a, u);
    if (qt >= a.q_tiles || slot < 0 || slot + chunks > a.slots) return;
    place = slot * a.q_tiles + qt;
    next = a.q_tiles;
  } else {
    place = tile_place<M>(a, u, (rows + M - 1) / M - 1 - qt);
    next = a.slots;
    if (place < 0 || place >= a.slots || chunks > a.q_tiles) return;
  }
  const int64_t step = next * a.g.H * a.part_rows;           // rows from a stretch to the next
  const int64_t at = (place * a.g.H + h) * a.part_rows + row % M;
  float y = -__builtin_inff();
  for (int k = WAVES == 4 ? threadIdx.x : lane; k < chunks; k += 64 * WAVES) y = fmaxf(y, a.part_ml[(at + k * step) * 2]);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) y = fmaxf(y, __shfl_xor(y, s));
  if constexpr (WAVES == 4) {
    if (lane == 0) most[wave] = y;
    __syncthreads();
    y = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  }
  const float ref = y > -__builtin_inff() ? y : 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
#pragma unroll 4
  for (int k = (WAVES == 4 ? wave * P : 0) + lane / L; k < chunks; k += WAVES * P) {
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + (at + k * step) * 2);
    const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + (at + k * step) * D + 4 * (lane % L));
    const float f = exp2_of(ml[0] - ref);
    l = __builtin_fmaf(ml[1], f, l);
    acc += v * f;
  }
#pragma unroll
  for (int s = L; s < 64; s <<= 1) {
    l += __shfl_xor(l, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], s);
  }
  if constexpr (WAVES == 4) {
    if (lane < L) xo[wave][lane] = acc;
    if (lane == 0) xl[wave] = l;
    __syncthreads();
    if (wave > 0) return;
    acc = (xo[0][lane % L] + xo[1][lane % L]) + (xo[2][lane % L] + xo[3][lane % L]);
    l = (xl[0] + xl[1]) + (xl[2] + xl[3]);
  }
  if (lane >= L) return;
  const f32x4 v = acc * (1.f / l);
  const int64_t dst = ((us.row0 + row / a.G) * Hq + h * a.G + row % a.G) * D + 4 * lane;
  if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<f32x4*>(a.out + dst * 4) = v;
  } else {
    const bf16x2 lo = __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2), hi = __builtin_convertvector((f32x2{v[2], v[3]}), bf16x2);
    *reinterpret_cast<u32x2*>(a.out + dst * 2) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

}  // namespace

constexpr int kWideRows = 128, kFewRows = 64;

Q8AttnPlan plan_q8_attention(const Q8Geom& g, int32_t num_q_heads, const BatchDev& b, int32_t layers) {
  Q8AttnPlan p{};
  const int64_t G = num_q_heads / g.H, rows = G * b.max_new;
  p.too_large = rows >= (1ll << 30) || b.max_total_len > kMostKeys;
  if (p.too_large || b.total_new <= 0 || b.batch <= 0) return p;
  const int64_t held = (int64_t)b.total_pages * g.S, most = (int64_t)b.batch * b.max_total_len;
  const int64_t keys = held < most ? held : most;
  auto finish = [&](Q8AttnLaunch& l, int64_t places) {
    l.on = true;
    l.items = places * g.H;
    p.too_large |= l.items >= (1ll << 24);             // a launch's threads are counted in 32 bits
    if (l.chunk_shift < 31) {
      const int64_t bytes = (l.items * l.part_rows * (g.D + 2) * (int64_t)sizeof(float) + 255) / 256 * 256;
      if (bytes > p.ws_bytes) p.ws_bytes = bytes;
    }
  };
  const bool wide = rows >= kWideRows;
  if (wide) {
    // Users of many rows.  Where their tiles fill the chip (two workgroups on each of 256 CUs) they are not cut; where they do not,
    // and the longest is not short, or a tile sees so many keys that a stretch's 128 rows (66 KB written and read again at
    // head_dim 128) are little beside them, the keys are.  us a call, cut into stretches of 256 and more / uncut: 8 users of
    // 1588-3176 x 3 heads of 64, fp32 134 / 108; 4 of 284-2279 x 3 (4 query heads each) of 128 156 / 107; 1 of 837 x 5 of 128
    // 41 / 23; of 512 and more / uncut: 2 of 427-3420 x 4 of 32 32 / 42; of 2048 and more / uncut: 28 users of 10-20 tokens behind
    // 8-14 K x 8 (8 query heads each) of 64 230 / 356, 32 of 16-32 behind 4-16 K x 8 (4) of 128 296 / 496.
    Q8AttnLaunch& l = p.wide;
    l.rows = l.part_rows = kWideRows;
    l.above = 0;
    l.upto = INT32_MAX;
    l.chunk_shift = 31;
    l.q_tiles = 1;
    l.slots = (int64_t)b.total_new * G / kWideRows + b.batch;
    // Users of about one length: the long tiles of all of them start first, and what ends last is short.  us, tiles user after
    // user / so: 8 first visits of 4096 x 8 (2 query heads each) of 128 719 / 674, 10 of 1943 x 2 (1) 101 / 74, 8 of 1432 x 16 (1)
    // of 64 90 / 70, 8 of 241-1928 x 3 (3) in fp32 107 / 107.
    const int64_t ranked = (int64_t)b.batch * ((rows + kWideRows - 1) / kWideRows);
    if (ranked <= 2 * l.slots) {
      l.by_rank = true;
      l.slots = ranked;
    }
    const int64_t tiles = l.slots * g.H, seen = (held - b.total_new / 2) / b.batch;   // keys of a tile, about
    const bool few_tiles = tiles < 384 && b.max_total_len > 1024;
    if (few_tiles || (tiles < 2048 && seen >= 4096)) {
      int shift = few_tiles ? 9 : 11;
      while (shift < 30 && (few_tiles ? ((int64_t)b.max_total_len - 1) >> shift : seen >> shift) * tiles > (few_tiles ? 1024 : 2048)) ++shift;
      if ((1ll << shift) < b.max_total_len) {
        l.chunk_shift = shift;
        l.q_tiles = (int)((((int64_t)b.max_total_len - 1) >> shift) + 1);   // stretches of the longest user
      }
    }
    finish(l, l.slots * l.q_tiles);
  }
  // Users of few rows beside them, unless the sizes leave none: a launch of their own, whose wavefronts share out the keys and
  // not the rows.  It costs 4 us, which short histories do not repay.
  const int64_t least = b.total_new - (b.batch - 1ll) * b.max_new;         // of a user, if all others have the most
  if (!wide || (least * G <= kFewRows && b.max_total_len > 1024)) {
    Q8AttnLaunch& l = p.few;
    const int64_t most_rows = wide ? kFewRows : rows;
    if (wide) p.wide.above = kFewRows;
    l.above = 0;
    l.upto = wide ? kFewRows : INT32_MAX;
    l.rows = most_rows > 16 ? 32 : 16;
    l.part_rows = (int)(most_rows < l.rows ? most_rows : l.rows);
    l.user_rows = (int)most_rows;
    l.q_tiles = (int)((most_rows + l.rows - 1) / l.rows);
    l.chunk_shift = 31;
    l.slots = b.batch;
    // Workgroups of at least 256 keys: about 2048, which even out users of unlike length; of little work (keys x heads x tiles)
    // fewer, since each takes some us to begin and to end; of very much 4096.  Two tiles of 128 dims: one full round (two on each
    // of 256 CUs) if some length of stretches gives it.  us a call with 2048 / by this rule: 10 users of 6-48 K keys x 2 heads of 64
    // 20.4 / 17.2, 5 of 9-20 K x 3 27.6 / 21.1, 29 of 0.4-2.6 K x 8 of 128 26.3 / 27.0, 44 of 4-12 K x 1 of 32 15.6 / 14.6, 50 of
    // 11-20 K x 8 82.7 / 77.5; 32 rows each behind 32 x 10 K x 8 of 128 159 / 146, 64 behind 111 x 3.7 K x 2 86.6 / 67.9.  With 1024
    // for 64 x 1.5 K x 8 of 64 28.3 where 27.4, for 32 x 10 K x 8 of 128 141 where 130, with 4096 135.  Short histories are not cut,
    // which saves the second launch and the workgroups' starts: what is short depends on how many tiles there are without cutting.
    // Cut / not, 1 user's 900 keys x 8 heads 9.3 / 7.9, 15 users' 0.6-2.4 K x 2 10.6 / 14.7; 32 of 0.9-1.4 K x 16 of 32 17.9 / 12.1, 44 of
    // 0.4-2.5 K x 8 of 64 23.6 / 17.7, 75 of 0.3-1.1 K x 2 of 128 with 45-90 rows 29.3 / 21.4, 36 of 0.6-3.5 K x 8 16.1 / 16.4; 161 of
    // 0.6-2.3 K x 8 of 64 with 5-55 rows 110.7 / 78.9; from 2048 tiles on always, 172 of 0.3-2.3 K x 16 of 32 68.7 / 56.4.
    const int64_t pairs = (int64_t)l.q_tiles * g.H, uncut = b.batch * pairs;
    if (uncut < 2048 && b.max_total_len > (uncut < 200 ? 1024 : l.rows == 32 && uncut >= 1024 ? 6144 : 2816)) {
      const int64_t work = keys * pairs;
      int64_t most = 2048;
      if (!wide && work < 1 << 19) most = 512;
      else if (!wide && l.rows == 16) most = work < 3 << 18 ? 1024 : work < 1 << 22 ? 2048 : 4096;
      int shift = 8;
      while (shift < 30 && (keys >> shift) * pairs > most) ++shift;
      if (!wide && l.rows == 32 && g.D == 128) {
        auto items = [&](int s) { return ((keys >> s) + b.batch / 2) * pairs; };   // half of a user's last stretch is empty
        int s = shift;
        while (s < 30 && items(s) > 512) ++s;
        if (items(s) >= 384) shift = s;
      }
      if ((1ll << shift) < b.max_total_len) {
        l.chunk_shift = shift;
        l.slots = (held >> shift) + b.batch;
      }
    }
    p.past_caches = l.q_tiles == 1 && kv_past_caches(g.D, keys / g.S * g.page_bytes, layers, keys / b.batch);
    finish(l, l.slots * l.q_tiles);
  }
  return p;
}

template <int D, typename T, int M, Numbered N>
static void launch_join(const Q8AttnArgs& a, hipStream_t stream) {
  // By the stretches of the longest user: a chain of many loads is shared by four wavefronts, a chain of a few too where the
  // rows do not fill the chip.  us a call, one wavefront / four: 70 K keys x 4 heads, 274 stretches 28.7 / 12.6; 55 users' single
  // tokens, 11 stretches, 165 rows 12.6 / 12.0; 2 users' 3 K tokens, 13 stretches, 15 K rows 31 / 50.
  const int64_t rows = (int64_t)a.b.total_new * a.g.H * a.G, units = N == Numbered::kKeys ? (int64_t)a.b.batch * a.user_rows * a.g.H : rows;
  if ((a.b.max_total_len >> a.chunk_shift) >= (rows <= 512 ? 8 : 32)) q8_join_kernel<D, T, M, N, 4><<<dim3((unsigned)units), dim3(256), 0, stream>>>(a);
  else q8_join_kernel<D, T, M, N, 1><<<dim3((unsigned)((units + 3) / 4)), dim3(256), 0, stream>>>(a);
}

template <int D, typename T>
static hipError_t launch(Q8AttnArgs a, const Q8AttnPlan& p, void* workspace, hipStream_t stream) {
  const dim3 block(256);
  auto take = [&](const Q8AttnLaunch& l) {
    a.above = l.above;
    a.upto = l.upto;
    a.q_tiles = l.q_tiles;
    a.by_rank = l.by_rank;
    a.chunk_shift = l.chunk_shift;
    a.part_rows = l.part_rows;
    a.user_rows = l.user_rows;
    a.slots = l.slots;
    a.part_o = (float*)workspace;
    a.part_ml = (float*)workspace + l.items * l.part_rows * D;
    return dim3((unsigned)l.items);
  };
  if (p.wide.on) {
    const dim3 grid = take(p.wide);
    if (a.chunk_shift < 31) {
      q8_attn_wide_kernel<D, T, Numbered::kBoth><<<grid, block, 0, stream>>>(a);
      launch_join<D, T, kWideRows, Numbered::kBoth>(a, stream);
    } else {
      q8_attn_wide_kernel<D, T, Numbered::kRows><<<grid, block, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.few.on) return e;
  }
  const dim3 grid = take(p.few);
  if (p.few.rows == 16) {
    if (a.chunk_shift < 31) {
      if (p.past_caches) q8_attn_kernel<D, 1, T, Numbered::kKeys, true><<<grid, block, 0, stream>>>(a);
      else q8_attn_kernel<D, 1, T, Numbered::kKeys, false><<<grid, block, 0, stream>>>(a);
      launch_join<D, T, 16, Numbered::kKeys>(a, stream);
    } else {
      q8_attn_kernel<D, 1, T, Numbered::kUsers, false><<<grid, block, 0, stream>>>(a);
    }
  } else if (a.chunk_shift < 31) {
    if (p.past_caches) q8_attn_kernel<D, 2, T, Numbered::kKeys, true><<<grid, block, 0, stream>>>(a);
    else q8_attn_kernel<D, 2, T, Numbered::kKeys, false><<<grid, block, 0, stream>>>(a);
    launch_join<D, T, 32, Numbered::kKeys>(a, stream);
  } else {
    q8_attn_kernel<D, 2, T, Numbered::kUsers, false><<<grid, block, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_q8_attn(const Q8Geom& g, const Q8AttnPlan& plan, bool f32, int32_t num_q_heads, const void* q, void* out,
                          const BatchDev& b, float sm_scale, void* workspace, hipStream_t stream) {
  Q8AttnArgs a{};
  a.g = g;
  a.q = (const char*)q;
  a.out = (char*)out;
  a.b = b;
  a.scale = sm_scale * kLog2e;
  a.G = num_q_heads / g.H;
  switch (g.D) {
    case 32: return f32 ? launch<32, float>(a, plan, workspace, stream) : launch<32, uint16_t>(a, plan, workspace, stream);
    case 64: return f32 ? launch<64, float>(a, plan, workspace, stream) : launch<64, uint16_t>(a, plan, workspace, stream);
    default: return f32 ? launch<128, float>(a, plan, workspace, stream) : launch<128, uint16_t>(a, plan, workspace, stream);
  }
}

}  // namespace mts
