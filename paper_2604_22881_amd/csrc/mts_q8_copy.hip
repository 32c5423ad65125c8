// Rows into and out of the 8-bit pool (mts_q8.hpp has the stored form):
//   append - the step's K/V rows behind the prefix, quantised as they are written
//   unpack - contiguous runs (a restored history), quantised as they are written
//   pack   - the inverse: stored rows read back as values into contiguous runs
//
// All three are bound by memory: es + 1 + 1/D bytes per element and a few instructions each (read back, 48 users' 819 MB 145 us,
// 5.6 TB/s; stored and read back, 24 users' 1.47 GB 240 us, 6.1 TB/s).  A wavefront takes a 16-token
// sub-block of one head, K and V.  On the rows' side its lanes take 16 bytes each, whole rows next to one another, on the pool's side
// granules of K and four-token groups of V; codes change sides through 16 rows of the wavefront's own in LDS, 16 bytes longer
// than D so that no access meets a bank twice.  V's [dim][4 tokens] order is a 4x4 transposition of bytes among four
// neighbouring lanes, in registers.
#include <type_traits>

#include "mts_internal.hpp"
#include "mts_q8.hpp"

namespace mts {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

enum { MODE_UNPACK = 0, MODE_APPEND = 1, MODE_PACK = 2 };

struct Q8MoveArgs {
  Q8Geom   g;
  char*    k;            // rows of K and V: of the step (append), of all runs (k alone)
  char*    v;
  int64_t  k_stride;     // bytes from a token's row to the next one's (append)
  int64_t  v_stride;
  BatchDev b;
  SegDev   s;
  int32_t  slots_in_flight;
};

// largest of a row's lanes: 4, 8, 16 or 32 neighbours
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, false));    // quad_perm 1,0,3,2
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, false));    // quad_perm 2,3,0,1
  if constexpr (LANES >= 8) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, false));   // row_half_mirror
  if constexpr (LANES >= 16) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, false));  // row_mirror
  if constexpr (LANES >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)a[0], (uint32_t)a[1]);
  }
  return m;
}

// A lane's 16 bytes of a row: 8 bf16 or 4 float.
template <typename T>
struct Part {
  static constexpr int N = 16 / sizeof(T);
  float x[N];
  __device__ __forceinline__ void take(u32x4 v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (N == 4) {
        x[j] = __uint_as_float(v[j]);
      } else {
        x[2 * j] = __uint_as_float(v[j] << 16);
        x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
      }
    }
  }
};

// Codes of a lane's part of a row, four a word, and the row's exponent byte.
template <int LANES, int N>
__device__ __forceinline__ uint32_t quantise(const float (&x)[N], uint32_t (&codes)[N / 4]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
  uint32_t amax = row_max<LANES>(m);
  const bool odd = __any(amax >= 0x7f800000u);             // an infinity or NaN in some row
  if (odd) {
    m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t a = __float_as_uint(x[j]) & 0x7fffffffu;
      if (a < 0x7f800000u) m = max(m, a);
    }
    amax = row_max<LANES>(m);
  }
  // the exponent of amax, one more where its mantissa is above 1.8125; e + 127 = that - 8
  int32_t e = (int32_t)((amax + 0x17ffffu) >> 23) - 8;
  e = min(max(e, kQ8ExpMin + 127), kQ8ExpMax + 127);
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = __builtin_amdgcn_fmed3f(x[4 * i + j] * inv, -448.f, 448.f);
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    if (odd) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((__float_as_uint(x[4 * i + j]) & 0x7fffffffu) >= 0x7f800000u)
          codes[i] = (codes[i] & ~(0xffu << (8 * j))) | (0x7fu << (8 * j));
    }
  }
  return (uint32_t)e;
}

// the values of a part's codes, rounded to nothing: every one is a value of T
template <typename T>
__device__ __forceinline__ u32x4 values(const uint32_t (&w)[4 / sizeof(T)], float scale) {
  u32x4 v;
  if constexpr (sizeof(T) == 4) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, false);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, true);
    v = u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
      v[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    }
  }
  return v;
}

// PAST: rows go past the caches' retention, those of an unpack and a pack of 128 bytes and more: nothing on the GPU reads them
// again soon (a restore of 120 K tokens x 8 heads of 128 and its read-back: 277 us, 317 the ordinary way).
template <bool PAST>
__device__ __forceinline__ u32x4 load_row(const char* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  else return *reinterpret_cast<const u32x4*>(p);
}
template <bool PAST>
__device__ __forceinline__ void store_row(char* p, u32x4 v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = v;
}

template <int D, typename T, int MODE, bool PAST>
__global__ __launch_bounds__(256) void q8_move_kernel(Q8MoveArgs a) {
  constexpr int N = D / 16, G = D >= 64 ? 16 : 8, W = G / 4;
  constexpr int es = sizeof(T), E = 16 / es, CW = E / 4;     // elements and code words of a lane's part
  constexpr int LPR = D / E, RPI = 64 / LPR, NR = 16 / RPI;  // lanes of a row, rows of an instruction, instructions of a sub-block
  constexpr int NG = D / (4 * G);                            // K granules of a lane
  constexpr int PITCH = D + 16;
  __shared__ __align__(16) char codes[4][2][16][PITCH];
  const int lane = threadIdx.x & 63, r = lane & 3, q = (lane >> 2) & 3, tg = lane >> 4, t16 = 4 * tg + r;
  const int in_block = uniform_int(threadIdx.x >> 6), wave = blockIdx.x * 4 + in_block;
  char (*rows)[16][PITCH] = codes[in_block];
  const int h = wave % a.g.H;
  const int n_runs = MODE == MODE_APPEND ? a.b.batch : a.s.num_segs;
  auto first = [&](int s) -> int64_t { return MODE == MODE_APPEND ? (int64_t)a.b.new_indptr[s] : a.s.seg_tok_indptr[s]; };
  const int64_t none = first(0);                             // rows ahead of the first run
  auto base = [&](int s) -> int64_t { return ((first(s) - none) >> 4) + 2ll * s; };   // slots of the runs before s, or a few more
  const int64_t slots = base(n_runs);
  const int64_t es_stride = (int64_t)a.g.H * D * es, head_row = (int64_t)h * D * es + (lane % LPR) * 16;
  for (int64_t slot = wave / a.g.H; slot < slots; slot += a.slots_in_flight) {
    const int s = find_user(n_runs, slot, base);
    const int64_t row0 = first(s), end = first(s + 1);
    const int64_t n = (MODE == MODE_APPEND && end > a.b.total_new ? a.b.total_new : end) - row0;
    const int u = MODE == MODE_APPEND ? s : a.s.seg_user[s];
    if (n <= 0 || row0 < 0 || u < 0 || u >= a.b.batch) continue;
    const int64_t p0 = MODE == MODE_APPEND ? a.b.prefix_lens[u] : a.s.seg_pos[s];
    const int64_t sub = (p0 >> 4) + slot - base(s);
    if (p0 < 0 || slot < base(s) || 16 * sub >= p0 + n) continue;
    const int64_t page0 = a.b.page_indptr[u], at = page0 + (sub >> a.g.sub_shift);
    if (page0 < 0 || at >= a.b.page_indptr[u + 1] || at >= a.b.total_pages) continue;
    const uint32_t page = (uint32_t)a.b.page_indices[at];
    if (page >= (uint32_t)a.g.num_pages) continue;
    const int in_page = (int)(sub & ((1 << a.g.sub_shift) - 1));
    const int64_t row_of_0 = 16 * sub - p0;                // the run's row that token 0 of the sub-block would be
    const uint32_t lo = row_of_0 < 0 ? (uint32_t)-row_of_0 : 0u, hi = n - row_of_0 < 16 ? (uint32_t)(n - row_of_0) : 16u;
    auto held = [&](int t) { return (uint32_t)t >= lo && (uint32_t)t < hi; };

    char* head = a.g.layer_base + (int64_t)page * a.g.page_bytes + h * q8_head_bytes(a.g.S, D);
    char *kc = head + in_page * 16 * D, *vc = kc + a.g.S * D;
    char *ke = head + 2 * a.g.S * D + in_page * 16, *ve = ke + a.g.S;
    const int64_t k_stride = MODE == MODE_APPEND ? a.k_stride : es_stride, v_stride = MODE == MODE_APPEND ? a.v_stride : es_stride;
    // this lane's part of token 0's rows
    char *k0, *v0;
    if constexpr (MODE == MODE_APPEND) {
      k0 = a.k + (row0 + row_of_0) * k_stride + head_row;
      v0 = a.v + (row0 + row_of_0) * v_stride + head_row;
    } else {
      k0 = a.k + (2 * row0 + row_of_0) * k_stride + head_row;
      v0 = k0 + n * k_stride;
    }
    const int v_at = (tg * 16 + 4 * q + r) * G;            // of dim 4q + r of the first W sixteens; the next W: + 64 G

    if constexpr (MODE == MODE_PACK) {
      const uint32_t kx = *reinterpret_cast<const uint8_t*>(ke + (lane & 15)), vx = *reinterpret_cast<const uint8_t*>(ve + (lane & 15));
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int i = lane + 64 * j;                       // granule of dims G (i / 16) .. of token i % 16
        if constexpr (G == 16) *reinterpret_cast<u32x4*>(&rows[0][i & 15][G * (i >> 4)]) = *reinterpret_cast<const u32x4*>(kc + i * G);
        else *reinterpret_cast<u32x2*>(&rows[0][i & 15][G * (i >> 4)]) = *reinterpret_cast<const u32x2*>(kc + i * G);
      }
#pragma unroll
      for (int c = 0; c < N / W; ++c) {
        uint32_t w[W];
        if constexpr (W == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(vc + v_at + 64 * G * c);
#pragma unroll
          for (int j = 0; j < W; ++j) w[j] = x[j];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2*>(vc + v_at + 64 * G * c);
#pragma unroll
          for (int j = 0; j < W; ++j) w[j] = x[j];
        }
#pragma unroll
        for (int j = 0; j < W; ++j) *reinterpret_cast<uint32_t*>(&rows[1][t16][16 * (c * W + j) + 4 * q]) = transpose_quad(w[j]);
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int t = i * RPI + lane / LPR;
        const float ks = __uint_as_float((uint32_t)__shfl((int)kx, t) << 23), vs = __uint_as_float((uint32_t)__shfl((int)vx, t) << 23);
        uint32_t kw[CW], vw[CW];
#pragma unroll
        for (int j = 0; j < CW; ++j) {
          kw[j] = *reinterpret_cast<const uint32_t*>(&rows[0][t][(lane % LPR) * E + 4 * j]);
          vw[j] = *reinterpret_cast<const uint32_t*>(&rows[1][t][(lane % LPR) * E + 4 * j]);
        }
        if (held(t)) {
          store_row<PAST>(k0 + t * k_stride, values<T>(kw, ks));
          store_row<PAST>(v0 + t * k_stride, values<T>(vw, vs));
        }
      }
      __builtin_amdgcn_wave_barrier();
    } else {
      u32x4 kr[NR], vr[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int t = i * RPI + lane / LPR;
        kr[i] = vr[i] = u32x4{0, 0, 0, 0};
        if (held(t)) {
          kr[i] = load_row<PAST>(k0 + t * k_stride);
          vr[i] = load_row<PAST>(v0 + t * v_stride);
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int t = i * RPI + lane / LPR;
        Part<T> x;
        uint32_t w[CW];
        x.take(kr[i]);
        const uint32_t kx = quantise<LPR>(x.x, w);
#pragma unroll
        for (int j = 0; j < CW; ++j) *reinterpret_cast<uint32_t*>(&rows[0][t][(lane % LPR) * E + 4 * j]) = w[j];
        x.take(vr[i]);
        const uint32_t vx = quantise<LPR>(x.x, w);
#pragma unroll
        for (int j = 0; j < CW; ++j) *reinterpret_cast<uint32_t*>(&rows[1][t][(lane % LPR) * E + 4 * j]) = w[j];
        if (lane % LPR == 0 && held(t)) { ke[t] = (char)kx; ve[t] = (char)vx; }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int i = lane + 64 * j;
        if (held(i & 15)) {
          if constexpr (G == 16) *reinterpret_cast<u32x4*>(kc + i * G) = *reinterpret_cast<const u32x4*>(&rows[0][i & 15][G * (i >> 4)]);
          else *reinterpret_cast<u32x2*>(kc + i * G) = *reinterpret_cast<const u32x2*>(&rows[0][i & 15][G * (i >> 4)]);
        }
      }
      const bool whole = held(4 * tg) && held(4 * tg + 3);
#pragma unroll
      for (int c = 0; c < N / W; ++c) {
        uint32_t w[W];
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = transpose_quad(*reinterpret_cast<const uint32_t*>(&rows[1][t16][16 * (c * W + j) + 4 * q]));
        if (whole) {
          if constexpr (W == 4) *reinterpret_cast<u32x4*>(vc + v_at + 64 * G * c) = u32x4{w[0], w[1], w[2], w[3]};
          else *reinterpret_cast<u32x2*>(vc + v_at + 64 * G * c) = u32x2{w[0], w[1]};
        } else {
          // tokens that are not this run's stay as they are
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (held(4 * tg + t)) {
#pragma unroll
              for (int j = 0; j < W; ++j) vc[v_at + 64 * G * c + 4 * j + t] = (char)(w[j] >> (8 * t));
            }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

int gcd4(int h) { return h % 4 == 0 ? 4 : h % 2 == 0 ? 2 : 1; }

template <int MODE, bool PAST>
hipError_t launch_move(Q8MoveArgs a, bool f32, int64_t slots, hipStream_t stream) {
  // Wavefronts keep their head and go on by whole slots: as many slots in flight as give whole workgroups.  Only calls of more
  // than a million wavefronts go round: a wavefront's sub-block begins with four dependent loads, which a new one overlaps with
  // those before it.  24 users' 120 K tokens x 8 heads of 128 restored and read back, at most 8, 16, 32 K wavefronts and
  // uncapped: 289, 259, 251, 247 us; a run looked up once for four sub-blocks in a row 3 % more.
  const int step = 4 / gcd4(a.g.H);
  int64_t in_flight = (slots + step - 1) / step * step;
  const int64_t most = (1 << 20) / a.g.H / step * step;
  if (in_flight > most) in_flight = most > step ? most : step;
  a.slots_in_flight = (int)in_flight;
  const dim3 grid((unsigned)(in_flight * a.g.H / 4)), block(256);
#define MTS_Q8_MOVE(D)                                                                          \
  if (f32) q8_move_kernel<D, float, MODE, PAST && D * 4 >= 128><<<grid, block, 0, stream>>>(a);  \
  else q8_move_kernel<D, uint16_t, MODE, PAST && D * 2 >= 128><<<grid, block, 0, stream>>>(a);
  switch (a.g.D) {
    case 32: MTS_Q8_MOVE(32) break;
    case 64: MTS_Q8_MOVE(64) break;
    default: MTS_Q8_MOVE(128) break;
  }
#undef MTS_Q8_MOVE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_append(const Q8Geom& g, bool f32, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                            const BatchDev& b, hipStream_t stream) {
  Q8MoveArgs a{g, (char*)k_new, (char*)v_new, k_stride, v_stride, b, SegDev{}, 0};
  return launch_move<MODE_APPEND, false>(a, f32, (int64_t)b.total_new / 16 + 2ll * b.batch, stream);
}

hipError_t launch_q8_unpack(const Q8Geom& g, bool f32, const void* staging, const SegDev& s, const BatchDev& b, hipStream_t stream) {
  Q8MoveArgs a{g, (char*)staging, nullptr, 0, 0, b, s, 0};
  return launch_move<MODE_UNPACK, true>(a, f32, (int64_t)s.num_segs * ((s.max_seg_tokens + 14ll) / 16 + 1), stream);
}

hipError_t launch_q8_pack(const Q8Geom& g, bool f32, void* staging_out, const SegDev& s, const BatchDev& b, hipStream_t stream) {
  Q8MoveArgs a{g, (char*)staging_out, nullptr, 0, 0, b, s, 0};
  return launch_move<MODE_PACK, true>(a, f32, (int64_t)s.num_segs * ((s.max_seg_tokens + 14ll) / 16 + 1), stream);
}

}  // namespace mts
