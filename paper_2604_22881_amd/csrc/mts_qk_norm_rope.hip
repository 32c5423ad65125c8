// Norm of a step's queries and keys, head by head, and their rotation by position, in one pass:
//   y = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * freq[pair].
//
// Bound by memory: each element is read and written once (39 K tokens x 24 heads of 128 in bf16, 470 MB, 93 us: 5.1 TB/s; one
// token a user, 4 us).  A row of D elements is D / 8 lanes, each with 8 of them such that
// both of a pair are in one lane: dims 4 j .. + 3 of the first and of the second half of the rotated dims, or 8 neighbours.
// The dims behind the rotated ones are shared out in the same way.  A wavefront takes one token and goes through
// heads, so that the angles are found once for several rows.
//
// Angles are turns in 64 bits: position * freq / 2 pi loses its whole turns there, and only the rest is
// rounded to 32 bits (a position of 10^5 times a frequency of 1 in 32 bits is off by up to 0.004).
#include <type_traits>

#include "mts_internal.hpp"
#include "mts_q8.hpp"

namespace mts {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ void load4(const char* p, float* x) {
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

template <typename T>
__device__ __forceinline__ void store4(char* p, const float* x) {
  if constexpr (std::is_same<T, float>::value) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
    const bf16x2 a = __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2), b = __builtin_convertvector((f32x2{x[2], x[3]}), bf16x2);
    *reinterpret_cast<u32x2*>(p) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  }
}

// sum over the row's lanes: 4, 8 or 16 neighbours, the same in each of them
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
  auto add = [&](auto ctrl) {
    v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  add(std::integral_constant<int, 0xB1>{});                        // quad_perm 1,0,3,2
  add(std::integral_constant<int, 0x4E>{});                        // quad_perm 2,3,0,1
  if constexpr (LANES >= 8) add(std::integral_constant<int, 0x141>{});   // row_half_mirror
  if constexpr (LANES >= 16) add(std::integral_constant<int, 0x140>{});  // row_mirror
  return v;
}

template <int D, typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a, BatchDev b, int heads_per_wave) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  constexpr int64_t es = sizeof(T);
  const int lane = threadIdx.x & 63, j = lane % LANES;
  const int heads = a.Hq + a.Hk, parts = (heads + heads_per_wave - 1) / heads_per_wave;
  const int64_t unit = (int64_t)blockIdx.x * 4 + uniform_int(threadIdx.x >> 6);
  const int token = (int)(unit / parts), part = (int)(unit % parts);
  if (token >= b.total_new) return;
  const int u = find_user(b.batch, token, [&](int s) -> int64_t { return b.new_indptr[s]; });
  const int first = b.new_indptr[u];
  if (token < first || token >= b.new_indptr[u + 1]) return;          // a padded step's rows behind the last user stay as they are
  const int64_t pos = (int64_t)b.prefix_lens[u] + (token - first);

  // the lane's two groups of four dims, and its four pairs
  const int rot = a.rot_dim;
  const bool turned = 8 * j < rot;
  int d0 = 8 * j, d1 = 8 * j + 4;
  if (!a.neighbours && turned) { d0 = 4 * j; d1 = rot / 2 + 4 * j; }
  float cs[4], sn[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double turns = (double)pos * (a.freqs[4 * j + i] * 0.15915494309189533577);
      const float rest = (float)(turns - rint(turns));
      sincospif(2.f * rest, &sn[i], &cs[i]);
    }
  }
  float qw[8], kw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) qw[i] = kw[i] = 1.f;
  if (a.q_weight) { load4<T>(a.q_weight + d0 * es, qw); load4<T>(a.q_weight + d1 * es, qw + 4); }
  if (a.k_weight) { load4<T>(a.k_weight + d0 * es, kw); load4<T>(a.k_weight + d1 * es, kw + 4); }

  const int end = min(heads, (part + 1) * heads_per_wave);
  for (int h = part * heads_per_wave + lane / LANES; h < end; h += ROWS) {
    const bool is_q = h < a.Hq;
    const char* src = is_q ? a.q + token * a.q_stride + (int64_t)h * D * es : a.k + token * a.k_stride + (int64_t)(h - a.Hq) * D * es;
    char* dst = is_q ? a.q_out + token * a.q_out_stride + (int64_t)h * D * es : a.k_out + token * a.k_out_stride + (int64_t)(h - a.Hq) * D * es;
    float x[8];
    load4<T>(src + d0 * es, x);
    load4<T>(src + d1 * es, x + 4);
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
      const float f = 1.f / sqrtf(row_sum<LANES>(ss) * (1.f / D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * f * (is_q ? qw[i] : kw[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * (is_q ? qw[i] : kw[i]);
    }
    if (turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float& p = a.neighbours ? x[2 * i] : x[i];
        float& s = a.neighbours ? x[2 * i + 1] : x[4 + i];
        const float first = p * cs[i] - s * sn[i], second = s * cs[i] + p * sn[i];
        p = first;
        s = second;
      }
    }
    store4<T>(dst + d0 * es, x);
    store4<T>(dst + d1 * es, x + 4);
  }
}

template <int D>
hipError_t launch(const QkArgs& a, const BatchDev& b, hipStream_t stream) {
  const int heads = a.Hq + a.Hk, rows = 512 / D;            // rows of a wavefront
  // Few tokens: as many wavefronts as there are rows for; many: all heads of a token to one, which shares its angles
  const int64_t waves = (int64_t)b.total_new * ((heads + rows - 1) / rows);
  const int heads_per_wave = waves <= 8192 ? rows : (heads + rows - 1) / rows * rows;
  const int parts = (heads + heads_per_wave - 1) / heads_per_wave;
  const dim3 grid((unsigned)(((int64_t)b.total_new * parts + 3) / 4)), block(256);
  if (a.f32) qk_norm_rope_kernel<D, float><<<grid, block, 0, stream>>>(a, b, heads_per_wave);
  else qk_norm_rope_kernel<D, uint16_t><<<grid, block, 0, stream>>>(a, b, heads_per_wave);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkArgs& a, const BatchDev& b, hipStream_t stream) {
  switch (a.D) {
    case 32: return launch<32>(a, b, stream);
    case 64: return launch<64>(a, b, stream);
    default: return launch<128>(a, b, stream);
  }
}

}  // namespace mts
