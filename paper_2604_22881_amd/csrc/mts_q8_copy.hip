// Rows into and out of the 8-bit pool (mts_q8.hpp has the stored form):
//   append - the step's K/V rows behind the prefix, quantised as they are written
//   unpack - contiguous runs (a restored history), quantised as they are written
//   pack   - the inverse: stored rows read back as values into contiguous runs
//
// All three are bound by memory: es + 1 + 1/D bytes per element and a few instructions each.  A wavefront
// takes a 16-token sub-block of one head, K and then V.  Lane (tg, q, r) holds token 4 tg + r and of it the
// dims 16 i + 4 q .. + 3: a row is four lanes of a 16-lane row apart by four, so that its largest value takes
// two rotations, and the four tokens of a group of V are neighbouring lanes, so that V's [dim][4 tokens] order is
// a 4x4 transposition of bytes between them, in registers.
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

// largest magnitude of a row's values, as bits; lanes 4 and 8 apart in a row of 16 hold the same token
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xf, 0xf, false));   // row_ror 4
  return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xf, 0xf, false)); // row_ror 8
}

template <typename T>
__device__ __forceinline__ void load4(const char* p, float x[4]) {
  if constexpr (std::is_same<T, float>::value) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = v[j];
  } else {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      x[2 * j] = __uint_as_float(v[j] << 16);
      x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
  }
}

// Codes of a row's 4 D/16 values that this lane holds, four a word, and the row's exponent byte.
template <int D>
__device__ __forceinline__ uint32_t quantise(const float (&x)[D / 16][4], uint32_t (&codes)[D / 16]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, __float_as_uint(x[i][j]) & 0x7fffffffu);
  uint32_t amax = row_max(m);
  const bool odd = __any(amax >= 0x7f800000u);             // an infinity or NaN in some row
  if (odd) {
    m = 0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t a = __float_as_uint(x[i][j]) & 0x7fffffffu;
        if (a < 0x7f800000u) m = max(m, a);
      }
    amax = row_max(m);
  }
  // the exponent of amax, one more where its mantissa is above 1.8125; e + 127 = that - 8
  int32_t e = (int32_t)((amax + 0x17ffffu) >> 23) - 8;
  e = min(max(e, kQ8ExpMin + 127), kQ8ExpMax + 127);
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = __builtin_amdgcn_fmed3f(x[i][j] * inv, -448.f, 448.f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    if (odd) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((__float_as_uint(x[i][j]) & 0x7fffffffu) >= 0x7f800000u)
          codes[i] = (codes[i] & ~(0xffu << (8 * j))) | (0x7fu << (8 * j));
    }
  }
  return (uint32_t)e;
}

// the values of four codes of one row, rounded to nothing: every one is a value of T
template <typename T>
__device__ __forceinline__ void store4(char* p, uint32_t w, float scale) {
  if constexpr (std::is_same<T, float>::value) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    *reinterpret_cast<f32x4*>(p) = f32x4{a[0], a[1], b[0], b[1]};
  } else {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    *reinterpret_cast<u32x2*>(p) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  }
}

template <int D, typename T, int MODE>
__global__ __launch_bounds__(256) void q8_move_kernel(Q8MoveArgs a) {
  constexpr int N = D / 16, G = D >= 64 ? 16 : 8, W = G / 4;
  const int lane = threadIdx.x & 63, r = lane & 3, q = (lane >> 2) & 3, tg = lane >> 4, t16 = 4 * tg + r;
  const int wave = blockIdx.x * 4 + uniform_int(threadIdx.x >> 6);
  const int h = wave % a.g.H;
  const int n_runs = MODE == MODE_APPEND ? a.b.batch : a.s.num_segs;
  auto first = [&](int s) -> int64_t { return MODE == MODE_APPEND ? (int64_t)a.b.new_indptr[s] : a.s.seg_tok_indptr[s]; };
  auto base = [&](int s) -> int64_t { return (first(s) >> 4) + 2ll * s; };   // slots of the runs before s, or a few more
  const int64_t slots = (first(n_runs) >> 4) + 2ll * n_runs;
  for (int64_t slot = wave / a.g.H; slot < slots; slot += a.slots_in_flight) {
    const int s = find_user(n_runs, slot, base);
    const int64_t row0 = first(s), end = first(s + 1);
    const int64_t n = (MODE == MODE_APPEND && end > a.b.total_new ? a.b.total_new : end) - row0;
    const int u = MODE == MODE_APPEND ? s : a.s.seg_user[s];
    if (n <= 0 || row0 < 0 || u < 0 || u >= a.b.batch) continue;
    const int64_t p0 = MODE == MODE_APPEND ? a.b.prefix_lens[u] : a.s.seg_pos[s];
    const int64_t sub = (p0 >> 4) + slot - base(s);
    if (p0 < 0 || 16 * sub >= p0 + n || 16 * sub + 15 < p0) continue;
    const int64_t at = a.b.page_indptr[u] + (sub >> a.g.sub_shift);
    if (at < 0 || at >= a.b.page_indptr[u + 1] || at >= a.b.total_pages) continue;
    const uint32_t page = (uint32_t)a.b.page_indices[at];
    if (page >= (uint32_t)a.g.num_pages) continue;
    const int in_page = (int)(sub & ((1 << a.g.sub_shift) - 1));
    const int64_t i_row = 16 * sub + t16 - p0;               // this lane's row of the run
    const bool held = i_row >= 0 && i_row < n;
    const uint64_t held_lanes = __ballot(held);
    // the four tokens of this lane's group
    const uint32_t held4 = (uint32_t)(held_lanes >> (16 * tg)) & 15u;

    char* head = a.g.layer_base + (int64_t)page * a.g.page_bytes + h * q8_head_bytes(a.g.S, D);
    char *kc = head + in_page * 16 * D, *vc = kc + a.g.S * D;
    char *ke = head + 2 * a.g.S * D + in_page * 16, *ve = ke + a.g.S;
    const int64_t es = sizeof(T), head_row = (int64_t)h * D * es;
    char *krow, *vrow;                                       // this lane's dims of its token
    if constexpr (MODE == MODE_APPEND) {
      krow = a.k + (row0 + i_row) * a.k_stride + head_row + 4 * q * es;
      vrow = a.v + (row0 + i_row) * a.v_stride + head_row + 4 * q * es;
    } else {
      const int64_t stride = (int64_t)a.g.H * D * es;
      krow = a.k + (2 * row0 + i_row) * stride + head_row + 4 * q * es;
      vrow = krow + n * stride;
    }
    const int k_at = G == 16 ? t16 * 16 + 4 * q : (q >> 1) * 128 + t16 * 8 + (q & 1) * 4;   // of dims 4q; 16 dims on: + 256
    const int v_at = (tg * 16 + 4 * q + r) * G;              // of dim 4q + r of the first W sixteens; the next W: + 64 G

    if constexpr (MODE == MODE_PACK) {
      const float k_scale = __uint_as_float((uint32_t)(uint8_t)ke[t16] << 23), v_scale = __uint_as_float((uint32_t)(uint8_t)ve[t16] << 23);
      uint32_t kw[N], vw[N];
#pragma unroll
      for (int i = 0; i < N; ++i) kw[i] = *reinterpret_cast<const uint32_t*>(kc + k_at + 256 * i);
#pragma unroll
      for (int c = 0; c < N / W; ++c) {
        if constexpr (W == 4) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(vc + v_at + 64 * G * c);
#pragma unroll
          for (int j = 0; j < W; ++j) vw[c * W + j] = w[j];
        } else {
          const u32x2 w = *reinterpret_cast<const u32x2*>(vc + v_at + 64 * G * c);
#pragma unroll
          for (int j = 0; j < W; ++j) vw[c * W + j] = w[j];
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) vw[i] = transpose_quad(vw[i]);
      if (held) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          store4<T>(krow + 16 * es * i, kw[i], k_scale);
          store4<T>(vrow + 16 * es * i, vw[i], v_scale);
        }
      }
    } else {
      float x[N][4], y[N][4];
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = y[i][j] = 0.f;
      if (held) {
#pragma unroll
        for (int i = 0; i < N; ++i) load4<T>(krow + 16 * es * i, x[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) load4<T>(vrow + 16 * es * i, y[i]);
      }
      uint32_t kw[N], vw[N];
      const uint32_t k_exp = quantise<D>(x, kw), v_exp = quantise<D>(y, vw);
      if (held) {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<uint32_t*>(kc + k_at + 256 * i) = kw[i];
        if (q == 0) { ke[t16] = (char)k_exp; ve[t16] = (char)v_exp; }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) vw[i] = transpose_quad(vw[i]);
      if (held4 == 15u) {
#pragma unroll
        for (int c = 0; c < N / W; ++c) {
          if constexpr (W == 4) *reinterpret_cast<u32x4*>(vc + v_at + 64 * G * c) = u32x4{vw[4 * c], vw[4 * c + 1], vw[4 * c + 2], vw[4 * c + 3]};
          else *reinterpret_cast<u32x2*>(vc + v_at + 64 * G * c) = u32x2{vw[2 * c], vw[2 * c + 1]};
        }
      } else {
        // tokens that are not this run's stay as they are
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (held4 >> t & 1u) {
#pragma unroll
            for (int i = 0; i < N; ++i) vc[v_at + 64 * G * (i / W) + 4 * (i % W) + t] = (char)(vw[i] >> (8 * t));
          }
      }
    }
  }
}

int gcd4(int h) { return h % 4 == 0 ? 4 : h % 2 == 0 ? 2 : 1; }

template <int MODE>
hipError_t launch_move(Q8MoveArgs a, bool f32, int64_t slots, hipStream_t stream) {
  // Wavefronts keep their head and go on by whole slots: as many slots in flight as give whole workgroups.
  const int step = 4 / gcd4(a.g.H);
  int64_t in_flight = (slots + step - 1) / step * step;
  const int64_t most = 16384 / a.g.H / step * step;         // 2 rounds of all the wavefronts the chip holds
  if (in_flight > most) in_flight = most > step ? most : step;
  a.slots_in_flight = (int)in_flight;
  const dim3 grid((unsigned)(in_flight * a.g.H / 4)), block(256);
#define MTS_Q8_MOVE(D)                                                                          \
  if (f32) q8_move_kernel<D, float, MODE><<<grid, block, 0, stream>>>(a);                       \
  else q8_move_kernel<D, uint16_t, MODE><<<grid, block, 0, stream>>>(a);
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
  return launch_move<MODE_APPEND>(a, f32, (int64_t)b.total_new / 16 + 2ll * b.batch, stream);
}

hipError_t launch_q8_unpack(const Q8Geom& g, bool f32, const void* staging, const SegDev& s, const BatchDev& b, hipStream_t stream) {
  Q8MoveArgs a{g, (char*)staging, nullptr, 0, 0, b, s, 0};
  return launch_move<MODE_UNPACK>(a, f32, (int64_t)s.num_segs * ((s.max_seg_tokens + 14ll) / 16 + 1), stream);
}

hipError_t launch_q8_pack(const Q8Geom& g, bool f32, void* staging_out, const SegDev& s, const BatchDev& b, hipStream_t stream) {
  Q8MoveArgs a{g, (char*)staging_out, nullptr, 0, 0, b, s, 0};
  return launch_move<MODE_PACK>(a, f32, (int64_t)s.num_segs * ((s.max_seg_tokens + 14ll) / 16 + 1), stream);
}

}  // namespace mts
