// The 8-bit pool: its geometry, shared by the host entry points and the kernels, and what the kernels
// of this element type have in common.
//
// A row (one token, one head, K or V) of D values is kept as one exponent e and D e4m3 codes: value =
// code * 2^e.  e is the smallest integer with amax <= 464 * 2^e over the row's finite values, held in
// [-60, 60]: the smallest for which amax still rounds to a code (448 and the next step, 480, meet at
// 464).  Scaling by a power of two is exact in fp32, bf16 and fp16, so that codes do not depend on how a
// kernel computes them, every stored value is a bf16 value, and a row that is read back and stored again
// gives the same bytes: its largest value is 448 * 2^e or less, and more than 464 * 2^(e-1), for which the
// smaller exponent would not do (above 232 the codes are 240 and up).
// The exponents' range is held where sums of 2^17 tokens' weights times 2^e, and their inverses, stay
// finite in fp32; values above 448 * 2^60 saturate, below 2^-70 they are 0.
//
// Page: head after head [K codes S*D][V codes S*D][K exponents S][V exponents S], exponents as bytes
// e + 127.  Codes lie in sub-blocks of 16 tokens, 16*D bytes, in which every load of a wavefront is
// one contiguous stretch and already an operand of a 16x16x32 matrix instruction (g = min(16, D/4)):
//   K: [D/g][16 tokens][g dims]: lane (token, group) takes g consecutive dims of its token; the product's
//      k index runs over (group, dim of the lane), in any order that the queries share.
//   V: [D/4g][4 groups of 4 tokens][16 dims][g/4][4 tokens]: lane (dim, group) takes the same four tokens
//      of dims dim, dim + 16, ..: four tokens of two sub-blocks are its 8 of 32 of the k index, the ones whose
//      weights the transposed product of K and Q leaves in that lane.
#pragma once
#include <stdint.h>

#include "mts_layout.hpp"

namespace mts {

constexpr int32_t kQ8ExpMin = -60, kQ8ExpMax = 60;

MTS_HD int32_t q8_granule(int32_t D) { return D >= 64 ? 16 : D / 4; }
// byte index of (token t16 in [0,16), dim d) inside a sub-block
MTS_HD int32_t q8_k_sub_index(int32_t t16, int32_t d, int32_t D) {
  const int32_t g = q8_granule(D);
  return (d / g * 16 + t16) * g + d % g;
}
MTS_HD int32_t q8_v_sub_index(int32_t t16, int32_t d, int32_t D) {
  const int32_t g = q8_granule(D);
  return (((d / (4 * g) * 4 + t16 / 4) * 16 + d % 16) * (g / 4) + d / 16 % (g / 4)) * 4 + t16 % 4;
}
MTS_HD int64_t q8_head_bytes(int32_t S, int32_t D) { return 2ll * S * (D + 1); }
// byte offsets inside a page
MTS_HD int64_t q8_code_offset(int32_t kv, int32_t h, int32_t slot, int32_t d, int32_t S, int32_t D) {
  const int32_t in_sub = kv == 0 ? q8_k_sub_index(slot & 15, d, D) : q8_v_sub_index(slot & 15, d, D);
  return h * q8_head_bytes(S, D) + (int64_t)kv * S * D + (int64_t)(slot >> 4) * 16 * D + in_sub;
}
MTS_HD int64_t q8_exp_offset(int32_t kv, int32_t h, int32_t slot, int32_t S, int32_t D) {
  return h * q8_head_bytes(S, D) + 2ll * S * D + (int64_t)kv * S + slot;
}

#if defined(__HIPCC__)

__device__ __forceinline__ int uniform_int(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Largest u in [0, n) with base(u) <= x, for a base that never falls and base(0) <= x: 64 places are looked
// at a time, one per lane, so that up to 64 users cost one round trip, 4096 two.  All lanes take part.
template <typename F>
__device__ __forceinline__ int find_user(int n, int64_t x, F base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  for (;;) {
    const int step = (len + 63) >> 6;
    const int at = lo + lane * step;
    const bool below = at < lo + len && base(at) <= x;
    const int k = __popcll(__ballot(below));
    const int skip = k > 0 ? (k - 1) * step : 0;
    lo += skip;
    len = min(step, len - skip);
    if (step == 1) return uniform_int(lo);
  }
}

// byte j of the result: the quad's lane j's byte number (lane & 3)
__device__ __forceinline__ uint32_t transpose_quad(uint32_t v) {
  const int lane = threadIdx.x;
  const uint32_t a = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);           // quad_perm 1,0,3,2
  // bytes 0-3 of a perm's selector are its second operand, 4-7 its first
  v = __builtin_amdgcn_perm(a, v, (lane & 1) ? 0x03070105u : 0x06020400u);
  const uint32_t b = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);           // quad_perm 2,3,0,1
  return __builtin_amdgcn_perm(b, v, (lane & 2) ? 0x03020706u : 0x05040100u);
}

#endif

}  // namespace mts
