// Incremental attention over the 8-bit pool (mts_q8.hpp), query heads sharing key heads:
//   out[i, h] = sum_j softmax_j(sm_scale * q[i, h] . K[j, h / G]) V[j, h / G],  j in [0, prefix + i].
//
// The query rows of a (user, key head) are its new tokens times the G query heads of the key head; a workgroup takes a tile
// of 16 or 32 of them and a stretch of the user's keys, its four wavefronts every fourth tile of 32 keys, each with all the
// rows.  Their sums are joined through LDS, and where the keys are cut into several stretches (a few rows behind a
// long history would leave most of the chip idle) a second kernel joins the stretches.
//
// Operand flow, 16x16x32 matrix instructions: S^T = K Q^T in bf16 and O^T = V^T P^T in fp16.  A code times its row's power of
// two is a bf16 value, so the logits are those of the stored values with fp32 sums; rows of K meet that power
// in the conversion.  S^T leaves a lane with 8 tokens of one query, the ones whose codes of V it holds.
//
// V's power of two varies along the index that P V sums over, so it goes to the weight: with Y a reference of the logits
// (base 2) and E of V's exponents e, both of them per query and wavefront,
//   w_j = 2^(y_j - Y + e_j - E),  O = sum w_j code_j,  l = sum w_j 2^(E - e_j),  out = 2^E O / l.
// w is rounded to fp16 for the product (11 bits, half a step 2^-12: next to it the output's own rounding to bf16, 2^-9, is
// what counts) and taken into l unrounded; weights are scaled so that the references' own is 2^10 and nothing above 2^-24 of it
// is below fp16's normal numbers.  Y and E move only when some w would exceed 2^15, and all sums are then
// scaled.  y_j - Y is one fma; where logits are so large that their rounding is a matter of whole powers of two, the
// product is rounded first, as the reference was, so that the largest logit's weight is the reference's.  fp32 rows: queries as three bf16 parts, weights as two
// fp16 ones, which keep 24 and 22 bits.
//
// Bound: few rows, reading K and V once (2 (D + 1) bytes a token); many, the vector instructions beside the products (per weight
// an fma, an addition, a maximum, an exponential, an fma and half a conversion, and per code of the tile half a conversion
// that the 16 or 32 rows share).
#include <type_traits>

#include "mts_internal.hpp"
#include "mts_q8.hpp"

namespace mts {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kRef = 10.f;       // log2 of the weight of the references
constexpr float kMost = 15.f;      // of the largest weight (fp16 ends below 2^16)
// A reference is a rounded logit, an fma's product is not: up to this size the two differ by 1/4 at most.
constexpr float kFused = 4194304.f;
constexpr float kLog2e = 1.44269504088896340736f;

struct Q8AttnArgs {
  Q8Geom      g;
  const char* q;
  char*       out;
  BatchDev    b;
  float       scale;               // sm_scale * log2(e)
  int32_t     G;                   // query heads of a key head
  int32_t     q_tiles;
  int32_t     chunk_shift;
  int32_t     part_rows;
  int64_t     slots;
  float*      part_o;              // [item][part_rows][D], item = (slot * q_tiles + q tile) * H + head
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

template <int D, int MT, typename T>
struct Attn {
  static constexpr int GB = D >= 64 ? 16 : 8;          // bytes of a lane's granule
  static constexpr int NJ = D >= 64 ? D / 64 : 1;      // granules of a row / 4
  static constexpr int NE = GB / 8;                    // matrix steps of a granule
  static constexpr int W = GB / 4;                     // 16-dim tiles of a granule of V
  static constexpr int DT = D / 16;
  static constexpr bool kF32 = std::is_same<T, float>::value;
  static constexpr int QP = kF32 ? 3 : 1, PP = kF32 ? 2 : 1;
  using Granule = typename std::conditional<GB == 16, u32x4, u32x2>::type;

  struct Tile {
    Granule  k[2][NJ], v[2][NJ];
    uint32_t ke[2], ve[2];
  };

  bf16x8 q[MT][NJ * NE][QP];
  f32x4  o[MT][DT];
  float  neg_y[MT], l[MT];         // -(Y - kRef); sums of this lane's tokens
  int    E;                        // reference of V's exponents, as byte
  bool   huge;                     // some reference is beyond what an fma may be exact to

  static __device__ __forceinline__ bf16x8 k_operand(const Granule& g, int e, float scale) {
    u32x4 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g[2 * e], scale, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g[2 * e], scale, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g[2 * e + 1], scale, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g[2 * e + 1], scale, true));
    return __builtin_bit_cast(bf16x8, w);
  }
  static __device__ __forceinline__ f16x8 v_operand(uint32_t a, uint32_t b) {
    u32x4 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true));
    return __builtin_bit_cast(f16x8, w);
  }

  __device__ __forceinline__ void load_queries(int mt, const char* row, int grp) {
#pragma unroll
    for (int s = 0; s < NJ * NE; ++s) {
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

  // Weights and sums of one tile of 32 keys, the first of them `key0`.  `edge`: some row does not see all of them; lim: the last
  // key that this lane's query sees; key_end: the keys behind it were never written.
  __device__ __forceinline__ void tile(Tile& t, int key0, bool edge, const int (&lim)[MT], int key_end, float scale, bool& first, int grp) {
    f32x4 s[2][MT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int m = 0; m < MT; ++m) s[h][m] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float ks = __uint_as_float(t.ke[h] << 23);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const bf16x8 k = k_operand(t.k[h][j], e, ks);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int p = QP - 1; p >= 0; --p)
              s[h][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[m][j * NE + e][p], s[h][m], 0, 0, 0);
        }
    }
    if (edge) {
      // what lies behind the last key is anything: exponents are given the reference's, codes 0
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = min(max(key_end - (key0 + 16 * h + 4 * grp), 0), 4);
        const uint32_t keep = left == 4 ? ~0u : (1u << (8 * left)) - 1u;
        t.ve[h] = (t.ve[h] & keep) | ((uint32_t)(first ? 67 : E) * 0x01010101u & ~keep);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int w = 0; w < W; ++w) t.v[h][j][w] &= keep;
      }
    }
    int  d[2][4];                              // E - e
    float x[2][MT][4];
    auto differences = [&] {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) d[h][r] = E - (int)((t.ve[h] >> (8 * r)) & 255u);
    };
    auto hidden = [&](int h, int m, int r) { return edge && key0 + 16 * h + 4 * grp + r > lim[m]; };
    auto weigh = [&](auto fused) {             // x: log2 of the weights
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float y = decltype(fused)::value ? __builtin_fmaf(s[h][m][r], scale, neg_y[m]) : rounded_product(s[h][m][r], scale) + neg_y[m];
            x[h][m][r] = hidden(h, m, r) ? -__builtin_inff() : y - (float)d[h][r];
          }
    };
    auto weigh_any = [&] {
      if (huge) weigh(std::false_type{});
      else weigh(std::true_type{});
    };
    bool over = first;
    if (!first) {
      differences();
      weigh_any();
      float most = -__builtin_inff();
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) most = fmaxf(most, x[h][m][r]);
      over = __any(most > kMost);
    }
    if (over) {
      // references that hold for this tile too, the sums scaled to them
      int e_most = first ? 0 : E;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) e_most = max(e_most, (int)((t.ve[h] >> (8 * r)) & 255u));
      e_most = (int)over_groups((float)e_most, [](float a, float b) { return fmaxf(a, b); });
      e_most = uniform_int(e_most);
      const float e_step = __uint_as_float((uint32_t)max(127 + (first ? 0 : E - e_most), 0) << 23);
      E = e_most;
      differences();
      float largest = 0.f;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float y = -__builtin_inff();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) y = fmaxf(y, hidden(h, m, r) ? -__builtin_inff() : rounded_product(s[h][m][r], scale));
        y = over_groups(y, [](float a, float b) { return fmaxf(a, b); });
        // a query that sees none of the tile keeps its reference (0 at first: its sums are 0)
        const float was = neg_y[m];
        const bool seen = y > -__builtin_inff();
        const float now = seen ? (first ? kRef - y : fminf(was, kRef - y)) : was;
        const float f = first ? 0.f : exp2_of(now - was);
        neg_y[m] = now;
        l[m] *= f;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[m][c] *= f * e_step;
        largest = fmaxf(largest, __builtin_fabsf(now));
      }
      huge = __any(largest > kFused);
      weigh_any();
      first = false;
    }
    f16x8 p[MT][PP];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = exp2_of(x[h][m][r]);
          l[m] = __builtin_fmaf(w[r], __uint_as_float((uint32_t)(d[h][r] + 127) << 23), l[m]);
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
    bool poisoned = false;
    if (edge) {
      // a NaN in V of a key that some rows see and others do not must not reach the others through 0 * NaN
      uint32_t nan = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int w = 0; w < W; ++w) nan |= (t.v[h][j][w] & 0x7f7f7f7fu) + 0x01010101u;
      poisoned = __any((nan & 0x80808080u) != 0);
    }
    if (poisoned) {
      // one key at a time: its column alone, and its product only for the queries that see it
#pragma unroll 1
      for (int key = 0; key < 32; ++key) {
        const int h = key >> 4, g = (key >> 2) & 3, r = key & 3;
        const uint32_t keep = grp == g ? 0xffu << (8 * r) : 0u;
        const uint32_t k0 = h == 0 ? keep : 0u, k1 = h == 1 ? keep : 0u;
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          const f16x8 v = v_operand(t.v[0][c / W][c % W] & k0, t.v[1][c / W][c % W] & k1);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            f32x4 n = o[m][c];
#pragma unroll
            for (int i = 0; i < PP; ++i) n = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[m][i], n, 0, 0, 0);
            o[m][c] = key0 + key <= lim[m] ? n : o[m][c];
          }
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        const f16x8 v = v_operand(t.v[0][c / W][c % W], t.v[1][c / W][c % W]);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = PP - 1; i >= 0; --i) o[m][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[m][i], o[m][c], 0, 0, 0);
      }
    }
  }
};

template <int D, int MT, typename T, bool SPLIT>
__global__ __launch_bounds__(256, D == 128 || MT == 2 ? 2 : 3) void q8_attn_kernel(Q8AttnArgs a) {
  using A = Attn<D, MT, T>;
  constexpr int M = 16 * MT;
  const int lane = threadIdx.x & 63, grp = lane >> 4, wave = uniform_int(threadIdx.x >> 6);
  const int h = blockIdx.x % a.g.H;
  const int64_t rest = blockIdx.x / a.g.H;
  const int qt = (int)(rest % a.q_tiles);
  const int64_t slot = rest / a.q_tiles;
  int u = (int)slot, key_first = 0;
  auto base = [&](int s) -> int64_t { return (((int64_t)a.b.page_indptr[s] * a.g.S) >> a.chunk_shift) + s; };
  if constexpr (SPLIT) {
    u = find_user(a.b.batch, slot, base);
    const int64_t chunk = slot - base(u);
    if (chunk < 0 || chunk > (kMostKeys >> a.chunk_shift)) return;
    key_first = (int)(chunk << a.chunk_shift);
  }
  const UserSpan us = user_span(a.b, a.g.S, u);
  const int64_t rows = (int64_t)us.n * a.G, row_first = (int64_t)qt * M;
  if (row_first >= rows) return;
  const int row_last = (int)(row_first + M < rows ? row_first + M : rows) - 1;
  const int keys = keys_of(us, row_last, a.G);
  if (SPLIT && key_first >= keys) return;
  const bool partial = SPLIT && keys > (1 << a.chunk_shift);
  const int key_last = partial ? min(key_first + (1 << a.chunk_shift), keys) : keys;   // one behind
  const int all_see = us.prefix + (int)(row_first / a.G);    // the last key that every row sees

  A c;
  int lim[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t r = row_first + 16 * m + (lane & 15);
    const int row = (int)(r < row_last ? r : row_last);      // rows behind the last repeat it and are not stored
    lim[m] = us.prefix + row / a.G;
    const int64_t at = ((int64_t)(us.row0 + row / a.G) * a.g.H + h) * a.G + row % a.G;
    c.load_queries(m, a.q + at * D * (int64_t)sizeof(T), grp);
    c.neg_y[m] = 0.f;
    c.l[m] = 0.f;
#pragma unroll
    for (int i = 0; i < A::DT; ++i) c.o[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  c.E = 67;
  c.huge = false;
  bool first = true;

  const int64_t head_off = h * q8_head_bytes(a.g.S, D);
  const int sub_mask = (1 << a.g.sub_shift) - 1;
  const int last_sub = (keys + 15) / 16 - 1;
  const int* pages = a.b.page_indices + us.page0;
  auto load = [&](typename A::Tile& t, int tile) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int sub = min(2 * tile + s, last_sub);
      const uint32_t id = (uint32_t)uniform_int(pages[sub >> a.g.sub_shift]);
      const int64_t page = id < (uint32_t)a.g.num_pages ? id : 0;
      const char* head = a.g.layer_base + page * a.g.page_bytes + head_off;
      const int in_page = sub & sub_mask;
      const char* kc = head + in_page * 16 * D;
      const char* vc = kc + a.g.S * D;
      const char* ex = head + 2 * a.g.S * D + in_page * 16;
#pragma unroll
      for (int j = 0; j < A::NJ; ++j) {
        t.k[s][j] = *reinterpret_cast<const typename A::Granule*>(kc + j * 1024 + lane * A::GB);
        t.v[s][j] = *reinterpret_cast<const typename A::Granule*>(vc + j * 1024 + lane * A::GB);
      }
      t.ke[s] = *reinterpret_cast<const uint8_t*>(ex + (lane & 15));
      t.ve[s] = *reinterpret_cast<const uint32_t*>(ex + a.g.S + 4 * grp);
    }
  };
  const int tile_end = (key_last + 31) / 32;
  int tile = key_first / 32 + wave;
  if (tile < tile_end) {
    typename A::Tile t0, t1;
    load(t0, tile);
    for (;;) {
      const int next = tile + 4;
      load(t1, next < tile_end ? next : tile);
      c.tile(t0, tile * 32, tile * 32 + 31 > all_see, lim, key_last, a.scale, first, grp);
      if (next >= tile_end) break;
      tile = next + 4;
      load(t0, tile < tile_end ? tile : next);
      c.tile(t1, next * 32, next * 32 + 31 > all_see, lim, key_last, a.scale, first, grp);
      if (tile >= tile_end) break;
    }
  }

  // The four wavefronts' sums: each takes a quarter of the dims (of 32 dims two take half) from the others.
  constexpr int DT = A::DT, OWNERS = DT < 4 ? DT : 4, OWN = DT / OWNERS;
  __shared__ f32x4 xo[OWNERS * 3 * OWN * MT * 64];
  __shared__ float xy[4][M], xl[4][M], xe[4];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const float l = over_groups(c.l[m], [](float p, float q) { return p + q; });
    if (grp == 0) {
      xy[wave][16 * m + lane] = l == 0.f ? -__builtin_inff() : kRef - c.neg_y[m];   // none of its keys seen
      xl[wave][16 * m + lane] = l;
    }
  }
  if (lane == 0) xe[wave] = (float)(c.E - 127);
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
  const int64_t item = blockIdx.x;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int in_tile = 16 * m + (lane & 15);
    float y = xy[0][in_tile];
#pragma unroll
    for (int w = 1; w < 4; ++w) y = fmaxf(y, xy[w][in_tile]);
    const float ref = y > -__builtin_inff() ? y : 0.f;
    float f[4], l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = exp2_of(xy[w][in_tile] - ref);
      l = __builtin_fmaf(xl[w][in_tile], f[w], l);
      f[w] *= exp2_of(xe[w]);
    }
    const int64_t r = row_first + in_tile;
    const bool live = r <= row_last;
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
          for (int cc = 0; cc < OWNERS; ++cc)
            if (cc == wave) p = c.o[m][cc * OWN + i];
        } else {
          p = xo[(((wave * 3 + w - (w > wave)) * OWN + i) * MT + m) * 64 + lane];
        }
        v += p * f[w];
      }
      const int d = 16 * (wave * OWN + i) + 4 * grp;
      if (live) {
        if (partial) {
          *reinterpret_cast<f32x4*>(a.part_o + (item * a.part_rows + in_tile) * D + d) = v;
        } else {
          v *= inv;
          const int row = (int)r;
          const int64_t at = ((int64_t)(us.row0 + row / a.G) * a.g.H + h) * a.G + row % a.G;
          if constexpr (A::kF32) {
            *reinterpret_cast<f32x4*>(a.out + (at * D + d) * 4) = v;
          } else {
            const bf16x2 lo = __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2), hi = __builtin_convertvector((f32x2{v[2], v[3]}), bf16x2);
            *reinterpret_cast<u32x2*>(a.out + (at * D + d) * 2) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
          }
        }
      }
    }
    if (partial && live && wave == 0 && grp == 0) *reinterpret_cast<f32x2*>(a.part_ml + (item * a.part_rows + in_tile) * 2) = f32x2{y, l};
  }
}

// Joins the stretches of a row's keys, in their order: one wavefront per (token, query head).
template <int D, typename T>
__global__ __launch_bounds__(256) void q8_join_kernel(Q8AttnArgs a, int tile_rows) {
  const int lane = threadIdx.x & 63;
  const int Hq = a.g.H * a.G;
  const int64_t unit = (int64_t)blockIdx.x * 4 + uniform_int(threadIdx.x >> 6);
  const int token = (int)(unit / Hq), hq = (int)(unit % Hq);
  if (token >= a.b.total_new) return;
  const int u = find_user(a.b.batch, token, [&](int s) -> int64_t { return a.b.new_indptr[s]; });
  const UserSpan us = user_span(a.b, a.g.S, u);
  const int i = token - us.row0;
  if (i < 0 || i >= us.n) return;
  const int h = hq / a.G;
  const int64_t row = (int64_t)i * a.G + hq % a.G, rows = (int64_t)us.n * a.G;
  const int qt = (int)(row / tile_rows);
  if (qt >= a.q_tiles) return;
  const int64_t tile_end = (int64_t)(qt + 1) * tile_rows;
  const int keys = keys_of(us, (int)((tile_end < rows ? tile_end : rows) - 1), a.G);
  const int chunks = (int)(((int64_t)keys + (1ll << a.chunk_shift) - 1) >> a.chunk_shift);
  if (chunks <= 1) return;
  const int64_t slot = (((int64_t)a.b.page_indptr[u] * a.g.S) >> a.chunk_shift) + u;
  if (slot < 0 || slot + chunks > a.slots) return;
  const int64_t step = (int64_t)a.q_tiles * a.g.H * a.part_rows;                  // rows from a stretch to the next
  const int64_t at = (slot * a.q_tiles + qt) * a.g.H * a.part_rows + (int64_t)h * a.part_rows + row % tile_rows;
  float y = -__builtin_inff();
  for (int k = lane; k < chunks; k += 64) y = fmaxf(y, a.part_ml[(at + k * step) * 2]);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) y = fmaxf(y, __shfl_xor(y, s));
  const float ref = y > -__builtin_inff() ? y : 0.f;
  constexpr int PER = D >= 64 ? D / 64 : 1;
  const bool mine = lane * PER < D;
  float acc[PER] = {}, l = 0.f;
  for (int k = 0; k < chunks; ++k) {
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + (at + k * step) * 2);
    const float f = exp2_of(ml[0] - ref);
    l = __builtin_fmaf(ml[1], f, l);
    if (mine) {
#pragma unroll
      for (int j = 0; j < PER; ++j) acc[j] = __builtin_fmaf(a.part_o[(at + k * step) * D + lane * PER + j], f, acc[j]);
    }
  }
  if (!mine) return;
  const int64_t dst = ((int64_t)token * Hq + hq) * D + lane * PER;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const float v = acc[j] / l;
    if constexpr (std::is_same<T, float>::value) *reinterpret_cast<float*>(a.out + (dst + j) * 4) = v;
    else *reinterpret_cast<__bf16*>(a.out + (dst + j) * 2) = (__bf16)v;
  }
}

}  // namespace

Q8AttnPlan plan_q8_attention(const Q8Geom& g, int32_t num_q_heads, const BatchDev& b) {
  Q8AttnPlan p{};
  const int64_t G = num_q_heads / g.H, rows = G * b.max_new;
  p.rows = rows > 16 ? 32 : 16;
  p.q_tiles = (int)((rows + p.rows - 1) / p.rows);
  p.chunk_shift = 31;
  p.part_rows = (int)(rows < p.rows ? rows : p.rows);
  p.slots = b.batch;
  p.too_large = rows >= (1ll << 30) || b.max_total_len > kMostKeys;
  if (p.too_large || b.total_new <= 0 || b.batch <= 0) return p;
  const int64_t pairs = (int64_t)p.q_tiles * g.H;
  const int64_t held = (int64_t)b.total_pages * g.S, most = (int64_t)b.batch * b.max_total_len;
  const int64_t keys = held < most ? held : most;
  if (b.batch * pairs < 4096 && b.max_total_len > 256) {
    int shift = 8;
    while (shift < 30 && (keys >> shift) * pairs > 2048) ++shift;
    if ((1ll << shift) < b.max_total_len) {
      p.chunk_shift = shift;
      p.slots = (held >> shift) + b.batch;
    }
  }
  p.items = p.slots * pairs;
  p.too_large = p.items >= (1ll << 31);
  if (p.chunk_shift < 31) p.ws_bytes = (p.items * p.part_rows * (g.D + 2) * (int64_t)sizeof(float) + 255) / 256 * 256;
  return p;
}

template <int D, typename T>
static hipError_t launch(const Q8AttnArgs& a, const Q8AttnPlan& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.items), block(256);
  const bool split = p.chunk_shift < 31;
  if (p.rows == 16) {
    if (split) q8_attn_kernel<D, 1, T, true><<<grid, block, 0, stream>>>(a);
    else q8_attn_kernel<D, 1, T, false><<<grid, block, 0, stream>>>(a);
  } else {
    if (split) q8_attn_kernel<D, 2, T, true><<<grid, block, 0, stream>>>(a);
    else q8_attn_kernel<D, 2, T, false><<<grid, block, 0, stream>>>(a);
  }
  if (split) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t units = (int64_t)a.b.total_new * a.g.H * a.G;
    q8_join_kernel<D, T><<<dim3((unsigned)((units + 3) / 4)), block, 0, stream>>>(a, p.rows);
  }
  return hipGetLastError();
}

hipError_t launch_q8_attn(const Q8Geom& g, const Q8AttnPlan& plan, bool f32, int32_t num_q_heads, const void* q, void* out,
                          const BatchDev& b, float sm_scale, void* workspace, hipStream_t stream) {
  Q8AttnArgs a{g, (const char*)q, (char*)out, b, sm_scale * kLog2e, num_q_heads / g.H, plan.q_tiles, plan.chunk_shift, plan.part_rows,
               plan.slots, (float*)workspace, (float*)workspace + plan.items * plan.part_rows * g.D};
  switch (g.D) {
    case 32: return f32 ? launch<32, float>(a, plan, stream) : launch<32, uint16_t>(a, plan, stream);
    case 64: return f32 ? launch<64, float>(a, plan, stream) : launch<64, uint16_t>(a, plan, stream);
    default: return f32 ? launch<128, float>(a, plan, stream) : launch<128, uint16_t>(a, plan, stream);
  }
}

}  // namespace mts
