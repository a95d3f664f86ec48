// What the grouped-query decode kernels share: the walk of a wave through its
// range's chunks, the online softmax of one chunk, and the operands made of
// the codes of an 8-bit cache.
#pragma once

#include <math.h>

#include "device_common.h"

namespace flexattn {

// The running max of a row moves only when a chunk raises it by more than
// this many log2 units; in between, probabilities are taken against the
// stale max (so they stay below 2^8) and the accumulators are left alone.
constexpr float kRescaleThreshold = 8.0f;

__device__ __forceinline__ bool wave_any(bool pred) { return __builtin_amdgcn_ballot_w64(pred) != 0; }

// Position in a wave's chunk stream: piece i (plan item), chunk ci of it, and
// the piece's first entry in the LDS page window. Wave-uniform.
struct DecodeCursor {
  int i, ci, seq, k0, k1, poff;
};

__device__ __forceinline__ int pages_in(int k0, int k1, int P) { return (k1 - 1) / P - k0 / P + 1; }

// Online-softmax step of one 16-row block over one chunk of NB 16-key blocks.
// s[b][r]: raw score q.k of key kc0 + 16b + 4gq + r for this lane's row; with
// `masked`, keys at or past `limit` are excluded (one code path: a second
// inlined copy for the unmasked case costs registers). The scale is folded
// into the exponent: p = 2^(s * scale_log2 - m). Updates the row's max m
// (log2 units, lazily), the lane's partial sum l and the accumulators o
// (rows 4gq + r), and gives the probabilities as bf16 A operands of P V, one
// per 32 keys.
template <int NB, int NACC>
__device__ __forceinline__ void softmax_chunk(const f32x4 (&s)[NB], bool masked, int kc0, int limit, int gq,
                                              float scale_log2, float& m, float& l, f32x4 (&o)[NACC],
                                              u32x4 (&pop)[NB / 2]) {
  float x[4 * NB];
#pragma unroll
  for (int e = 0; e < 4 * NB; ++e) x[e] = s[e >> 2][e & 3];
  if (masked) {
#pragma unroll
    for (int e = 0; e < 4 * NB; ++e) x[e] = kc0 + chunk_key(e, gq) < limit ? x[e] : -INFINITY;
  }
  float bmax[NB / 2];
#pragma unroll
  for (int h = 0; h < NB / 2; ++h)
    bmax[h] = fmaxf(fmaxf(fmaxf(x[8 * h], x[8 * h + 1]), fmaxf(x[8 * h + 2], x[8 * h + 3])),
                    fmaxf(fmaxf(x[8 * h + 4], x[8 * h + 5]), fmaxf(x[8 * h + 6], x[8 * h + 7])));
  float cmax = bmax[0];
#pragma unroll
  for (int h = 1; h < NB / 2; ++h) cmax = fmaxf(cmax, bmax[h]);
  cmax = group_max(cmax) * scale_log2;
  const bool need = cmax > m + kRescaleThreshold;
  if (wave_any(need)) {
    const float m_new = need ? cmax : m;
    const float alpha = fast_exp2(m - m_new);   // 1 if unchanged, 0 from -inf
    l *= alpha;
    m = m_new;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float ar = shfl_f(alpha, 4 * gq + r);
#pragma unroll
      for (int a = 0; a < NACC; ++a) o[a][r] *= ar;
    }
  }
  const float neg_m = m == -INFINITY ? 0.f : -m;
  float psum = 0.f;
#pragma unroll
  for (int e2 = 0; e2 < 2 * NB; ++e2) {
    const float p0 = fast_exp2(fmaf(x[2 * e2], scale_log2, neg_m));
    const float p1 = fast_exp2(fmaf(x[2 * e2 + 1], scale_log2, neg_m));
    psum += p0 + p1;
    pop[e2 >> 2][e2 & 3] = pack_bf16x2(p0, p1);
  }
  l += psum;
}

// A block scale byte (e8m0) as the float whose exponent it is.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float((byte & 0xFFu) << 23); }

// Two e4m3 codes (the low or high half of w) times a power of two, as two bf16
// in one dword: exact, a code has 4 significant bits.
template <bool HI>
__device__ __forceinline__ uint32_t codes_bf16x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Eight codes as eight bf16, the first four by one scale and the others by another.
__device__ __forceinline__ u32x4 codes_bf16x8(uint32_t w0, uint32_t w1, float scale0, float scale1) {
  return u32x4{codes_bf16x2<false>(w0, scale0), codes_bf16x2<true>(w0, scale0), codes_bf16x2<false>(w1, scale1),
               codes_bf16x2<true>(w1, scale1)};
}

// ds_read_b64_tr_b8: within each group of 16 lanes, lane j supplies the LDS
// address of 8 consecutive bytes; lane i receives byte i % 8 of the lanes
// i / 8, 2 + i / 8, .. 14 + i / 8. With lane j pointing at row R(j / 2), column
// c + 8 (j % 2), lane i gets column c + i of rows R(0 .. 7).
typedef int32_t v2i32 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 lds_read_tr8(const uint8_t* lds_addr) {
  typedef __attribute__((address_space(3))) v2i32* lds_v2i32_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i32_ptr)(lds_addr)));
}

}  // namespace flexattn
