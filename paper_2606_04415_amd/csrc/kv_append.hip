// KV append: the write side of the paged KV pool that prefill and decode of
// one device share (Sec. 3.4, "Memory Locality": co-located phases extend and
// read one pool instead of moving KV caches between workers). Each new token's
// key row, and value row unless values alias keys, goes to its slot
// (page = slot / P, row = slot % P) of the paged caches: copied
// (kv_append_kernel), with queries and keys turned by their positions on the
// way (rope_append_kernel), or turned and quantised into an 8-bit cache
// (kv8_append_kernel). All read each new value once and write it once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.h"
#include "kernels.h"

// Rotated values are rounded product by product (see below), never fused.
#pragma clang fp contract(off)

namespace flexattn {

namespace {

// ---------------------------------------------------------------------------
// Copies. HBM-bound: one thread per 16-byte chunk of a token's row, so a wave
// reads 1 KB of consecutive new-token data and writes it to consecutive
// bytes of one cache row (heads of a slot are contiguous when the head stride
// equals the head dimension). Out-of-range slots are skipped and counted.
// ---------------------------------------------------------------------------
struct alignas(16) Chunk {
  uint32_t w[4];
};

__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams a) {
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t per_tok = a.ck + a.cv;   // 16-byte chunks of one token (K then V)
  if (i >= a.n_tokens * per_tok) return;
  const int64_t t = i / per_tok;
  int64_t c = i - t * per_tok;
  const int32_t slot = a.slot_mapping[t];
  if (slot < 0) return;                      // padding token
  if (int64_t(slot) >= a.num_slots) {        // outside the pool: skipped, counted once per token
    if (c == 0 && a.bad_count) atomicAdd(a.bad_count, 1);
    return;
  }
  const int64_t page = slot / a.P, row = slot - page * a.P;
  const bool is_v = c >= a.ck;
  if (is_v) c -= a.ck;
  const int d = is_v ? a.dv : a.dk;
  const int cpd = d / 8;                     // chunks per head
  const int64_t h = c / cpd, x = 8 * (c - h * cpd);
  const uint16_t* src = (is_v ? a.v_new + t * a.v_new_stride : a.k_new + t * a.k_new_stride) + h * d + x;
  const CacheRef& dst_ref = is_v ? a.vc : a.kc;
  uint16_t* dst = const_cast<uint16_t*>(dst_ref.base) + page * dst_ref.sp + row * dst_ref.ss + h * dst_ref.sh + x;
  *reinterpret_cast<Chunk*>(dst) = *reinterpret_cast<const Chunk*>(src);
}

// ---------------------------------------------------------------------------
// Rotation of pair (x, y) by the angle of its position: (x c - y s, y c + x s),
// the products and the sum each rounded to fp32 (no contraction, so that the
// codes of an 8-bit cache do not depend on which sums a compiler fuses), then
// one rounding to bf16 or e4m3.
//
// A thread's unit is 8 pairs of one head of one token: two 16-byte chunks, with
// their 8 cosines and 8 sines. Pairs half a part apart lie in chunks half a
// part apart, neighbouring pairs in one 32-byte piece; either way consecutive
// threads read and write consecutive chunks.
// ---------------------------------------------------------------------------
// Positions of one token on its axes; ok: all inside the table (the others are
// taken as 0, so that the table can be read before the token is given up).
// AXES: more than one (kernels for one axis are a third of the code of those
// for several, which costs short calls instruction fetches).
template <bool AXES>
struct Positions {
  int32_t p[AXES ? kRopeMaxAxes : 1] = {};
  bool ok = true;
};

template <bool AXES>
__device__ __forceinline__ void check_position(const RopeParams& r, Positions<AXES>& x, int a, int32_t pos) {
  const bool ok = pos >= 0 && pos < r.max_position;
  x.p[a] = ok ? pos : 0;
  x.ok = x.ok && ok;
}

template <bool AXES>
__device__ __forceinline__ Positions<AXES> read_positions(const RopeParams& r, int64_t t) {
  Positions<AXES> x;
#pragma unroll
  for (int a = 0; a < (AXES ? kRopeMaxAxes : 1); ++a)
    if (!AXES || a < r.n_axes) check_position(r, x, a, r.positions[a * r.positions_stride + t]);
  return x;
}

// The one position of a token that has no row of positions.
template <bool AXES>
__device__ __forceinline__ Positions<AXES> position_at(const RopeParams& r, int32_t pos) {
  Positions<AXES> x;
  check_position(r, x, 0, pos);
  return x;
}

__device__ __forceinline__ int axis_of(const RopeParams& r, int i) {
  if (r.dealt) {
    const int a = i % r.n_axes;
    const int n = a == 1 ? r.sections[1] : a == 2 ? r.sections[2] : r.sections[3];
    return a != 0 && i < r.n_axes * n ? a : 0;
  }
  const int s1 = r.sections[0], s2 = s1 + r.sections[1], s3 = s2 + r.sections[2];
  return (r.n_axes > 1 && i >= s1 ? 1 : 0) + (r.n_axes > 2 && i >= s2 ? 1 : 0) + (r.n_axes > 3 && i >= s3 ? 1 : 0);
}

__device__ __forceinline__ int32_t pick(const Positions<true>& x, int a) {
  return a == 0 ? x.p[0] : a == 1 ? x.p[1] : a == 2 ? x.p[2] : x.p[3];
}

// Cosines and sines of pairs 8 j .. 8 j + 7 at a token's positions: from one
// table row when one axis has them all, from two when sections meet in the
// unit, else pair by pair.
struct Turn {
  float c[8], s[8];
};

__device__ __forceinline__ Turn read_row(const RopeParams& r, int32_t pos, int j) {
  const float* row = r.cos_sin + int64_t(pos) * r.rot_dim + 8 * j;
  Turn t;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(row + 4 * v);
    const f32x4 s = *reinterpret_cast<const f32x4*>(row + r.rot_dim / 2 + 4 * v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      t.c[4 * v + e] = c[e];
      t.s[4 * v + e] = s[e];
    }
  }
  return t;
}

__device__ __forceinline__ Turn read_turn(const RopeParams& r, const Positions<false>& x, int j) {
  return read_row(r, x.p[0], j);
}
__device__ __forceinline__ Turn read_turn(const RopeParams& r, const Positions<true>& x, int j) {
  const int half = r.rot_dim / 2;
  if (!r.dealt) {
    const int a0 = axis_of(r, 8 * j), a1 = axis_of(r, 8 * j + 7);
    if (a1 <= a0 + 1) {
      Turn t = read_row(r, pick(x, a0), j);
      if (a1 != a0) {
        const Turn u = read_row(r, pick(x, a1), j);
#pragma unroll
        for (int e = 1; e < 8; ++e) {
          const bool next = axis_of(r, 8 * j + e) != a0;
          t.c[e] = next ? u.c[e] : t.c[e];
          t.s[e] = next ? u.s[e] : t.s[e];
        }
      }
      return t;
    }
  }
  Turn t;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float* row = r.cos_sin + int64_t(pick(x, axis_of(r, 8 * j + e))) * r.rot_dim + 8 * j + e;
    t.c[e] = row[0];
    t.s[e] = row[half];
  }
  return t;
}

__device__ __forceinline__ void unpack8(const u32x4& v, float (&x)[8]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    x[2 * w] = __uint_as_float(v[w] << 16);
    x[2 * w + 1] = __uint_as_float(v[w] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// The two chunks of a unit, as columns of the head: units 0 .. rot_dim / 16 - 1
// hold the pairs, the others the columns that pass unchanged, in order.
__device__ __forceinline__ void unit_columns(const RopeParams& r, int j, int& c0, int& c1) {
  const int turned = r.rot_dim / 16;
  if (j < turned) {
    c0 = r.rot_begin + (r.neighbours ? 16 * j : 8 * j);
    c1 = r.neighbours ? c0 + 8 : c0 + r.rot_dim / 2;
  } else {
    c0 = 16 * (j - turned);
    c1 = c0 + 8;
    if (c0 >= r.rot_begin) c0 += r.rot_dim;
    if (c1 >= r.rot_begin) c1 += r.rot_dim;
  }
}

// Turn a unit's 16 values, a the first chunk's and b the second's.
__device__ __forceinline__ void turn_unit(const RopeParams& r, const Turn& t, float (&a)[8], float (&b)[8]) {
  if (r.neighbours) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x0 = a[2 * e], y0 = a[2 * e + 1], x1 = b[2 * e], y1 = b[2 * e + 1];
      a[2 * e] = x0 * t.c[e] - y0 * t.s[e];
      a[2 * e + 1] = y0 * t.c[e] + x0 * t.s[e];
      b[2 * e] = x1 * t.c[4 + e] - y1 * t.s[4 + e];
      b[2 * e + 1] = y1 * t.c[4 + e] + x1 * t.s[4 + e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = a[e], y = b[e];
      a[e] = x * t.c[e] - y * t.s[e];
      b[e] = y * t.c[e] + x * t.s[e];
    }
  }
}

// Heads that one thread takes: it reads the cosines and sines of its unit once
// for all of them, and their loads are in flight together. (1, 2 and 4 heads,
// kernel times: 2176 tokens of 28/4 heads of 128 10.5, 9.9 and 9.9 us; 5648
// tokens of 32/8 heads of 64 on three axes 21.2, 18.4 and 20.0; a 4096-token
// latent prompt 257, 242 and 240; 64 tokens 3.6, 4.0 and 4.9.)
constexpr int kHeadsPerThread = 2;

// Unit j of heads h .. h + kHeadsPerThread - 1 of a token's n_heads rows, from
// src(head) to dst(head) (a row's first column), written if live(); heads past
// the last repeat it and are not written.
template <bool AXES, typename Live, typename Src, typename Dst>
__device__ __forceinline__ void move_units(const RopeParams& r, const Positions<AXES>& x, int j, int h, int n_heads, Live&& live,
                                           Src&& src, Dst&& dst) {
  int c0, c1;
  unit_columns(r, j, c0, c1);
  u32x4 v0[kHeadsPerThread], v1[kHeadsPerThread];
#pragma unroll
  for (int k = 0; k < kHeadsPerThread; ++k) {
    const uint16_t* s = src(min(h + k, n_heads - 1));
    v0[k] = load16(s + c0);
    v1[k] = load16(s + c1);
  }
  if (j < r.rot_dim / 16) {
    const Turn t = read_turn(r, x, j);
#pragma unroll
    for (int k = 0; k < kHeadsPerThread; ++k) {
      float a[8], b[8];
      unpack8(v0[k], a);
      unpack8(v1[k], b);
      turn_unit(r, t, a, b);
      v0[k] = pack8(a);
      v1[k] = pack8(b);
    }
  }
  if (!live()) return;
#pragma unroll
  for (int k = 0; k < kHeadsPerThread; ++k) {
    if (h + k >= n_heads) break;
    uint16_t* d = dst(h + k);
    *reinterpret_cast<u32x4*>(d + c0) = v0[k];
    *reinterpret_cast<u32x4*>(d + c1) = v1[k];
  }
}

// ---------------------------------------------------------------------------
// Into the bf16 cache: a work-group takes `per_wg` tokens, or a part of one; a
// thread takes one unit of two consecutive heads (queries, then keys), or 32
// bytes of values. Bound by HBM: a latent prompt of 4096 tokens 241 us, 5.0 TB/s
// read and written. (With the parts of a token in turn in one work-group, 16
// latent tokens of 128 heads took 9.2 us, now 4.0, 256 16.3, now 15.6.)
// ---------------------------------------------------------------------------
template <int DK, int DV, bool AXES>
__global__ __launch_bounds__(512) void rope_append_kernel(RopeAppendParams p) {
  constexpr int UK = DK / 16, UV = DV / 16;
  const AppendParams& a = p.kv;
  const int heads = p.Hq + p.Hkv;
  const int nqk = (heads + kHeadsPerThread - 1) / kHeadsPerThread * UK, nv = a.cv ? p.Hkv * UV : 0;
  const int per_tok = nqk + nv, page_bits = __builtin_ctz(a.P);   // (pages of 16 or 64)
  const int64_t t0 = int64_t(blockIdx.x) * p.per_wg;
  const int n = int(min(int64_t(p.per_wg), a.n_tokens - t0)) * per_tok;
  const int i = blockIdx.y * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int dt = p.per_wg == 1 ? 0 : i / per_tok;
  const int u = i - dt * per_tok;
  const int64_t t = t0 + dt;
  const int32_t slot = a.slot_mapping[t];
  const auto x = read_positions<AXES>(p.rope, t);
  // A negative slot is padding; another fault is counted once a token.
  const bool inside = slot >= 0 && int64_t(slot) < a.num_slots, live = inside && x.ok;
  const int64_t page = inside ? slot >> page_bits : 0, row = inside ? slot & (a.P - 1) : 0;
  if (u < nqk) {
    const int g = u / UK;
    move_units(
        p.rope, x, u - g * UK, g * kHeadsPerThread, heads, [&] { return live; },
        [&](int h) { return h < p.Hq ? p.q + t * p.q_stride + h * DK : a.k_new + t * a.k_new_stride + (h - p.Hq) * DK; },
        [&](int h) {
          return h < p.Hq ? p.q_out + (t * p.Hq + h) * DK
                          : const_cast<uint16_t*>(a.kc.base) + page * a.kc.sp + row * a.kc.ss + (h - p.Hq) * a.kc.sh;
        });
  } else {
    const int v = u - nqk, h = v / UV, c = 16 * (v - h * UV);
    const uint16_t* src = a.v_new + t * a.v_new_stride + h * DV + c;
    const u32x4 v0 = load16(src), v1 = load16(src + 8);
    if (!live) return;   // (never a token's unit 0)
    uint16_t* dst = const_cast<uint16_t*>(a.vc.base) + page * a.vc.sp + row * a.vc.ss + h * a.vc.sh + c;
    *reinterpret_cast<u32x4*>(dst) = v0;
    *reinterpret_cast<u32x4*>(dst + 8) = v1;
  }
  if (u == 0 && slot >= 0 && !live && a.bad_count) atomicAdd(a.bad_count, 1);
}

// ---------------------------------------------------------------------------
// Into the 8-bit cache. One, two or four waves take a new token: they find the
// token's sequence, turn its query, and take their part of the token's block: a
// task is the block's new rows of one KV head, K or V, for one wave, and the
// waves of the block's new tokens (which are consecutive) share them out.
// A wave holds its rows in registers between the maximum that gives the scale
// and the conversion, so they are read once. (With all tasks of a block in the
// work-group of its first token, a 2048-token chunk beside 128 decodes took
// 33.6 us, now 12.8. The rotation of that step into the bf16 cache takes 8.8 in
// 5808 waves; the 8704 here last as long each, waiting for 64% of it (62%
// there). Which of the chain of search, page, rows, maximum and codes costs what
// is not measured apart; the search in one round instead of two changed nothing.)
// ---------------------------------------------------------------------------

// The sequence that holds new token t: the largest s with query_start_loc[s]
// <= t (0 also where there is none, B behind the last), its first and end token
// and its length. 63 probes at a time; the last round, over 64 neighbours,
// brings the rest along. No sequence holds a token outside [start, end).
struct Sequence {
  int s, start, end, L;
};

__device__ __forceinline__ Sequence find_sequence(const int32_t* qsl, const int32_t* seq_lens, int B, int64_t t, int lane) {
  int base = 0, len = B;                 // s lies in base .. base + len
  while (len > 62) {
    const int step = (len + 62) / 63;
    const int64_t at = base + int64_t(lane + 1) * step;
    const bool below = lane < 63 && at <= base + len && int64_t(qsl[min(at, int64_t(B))]) <= t;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
    const int end = base + len;
    base += n * step;
    len = min(step - 1, end - base);
  }
  const int v = qsl[min(base + lane, B)], held = seq_lens[min(base + lane, B - 1)];
  const bool below = lane > 0 && lane <= len && int64_t(v) <= t;
  const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
  return Sequence{__builtin_amdgcn_readfirstlane(base + n), __builtin_amdgcn_readlane(v, n),
                  __builtin_amdgcn_readlane(v, n + 1), __builtin_amdgcn_readlane(held, n)};
}

// Least k >= -117 with a <= 448 * 2^k, from the bits of a >= 0. 448 = 1.75 *
// 2^8; -117 keeps the scaled value of the smallest code, 2^-9, a normal number.
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
  const int k = int(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(k, -117);
}

__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float(uint32_t(min(max(k + 127, 0), 254)) << 23); }

// Four values as e4m3 codes, rounded to nearest even; infinities and NaN become
// NaN (finite values are at most 448 here, by the choice of the scale).
__device__ __forceinline__ uint32_t encode4(float x0, float x1, float x2, float x3) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
  return uint32_t(w);
}

// Four codes times f as codes again.
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), true);
  return encode4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// Maximum over the wave: rotations within rows of 16 lanes, then swaps of rows.
template <int N>
__device__ __forceinline__ uint32_t row_ror(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x120 + N, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, row_ror<8>(v));
  v = max(v, row_ror<4>(v));
  v = max(v, row_ror<2>(v));
  v = max(v, row_ror<1>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return uint32_t(__builtin_amdgcn_readfirstlane(int(max(b[0], b[1]))));
}

// The `count` new rows of one block for one KV head, keys or values, in a wave's
// registers: those of new tokens t, t + 1, ... Lane l holds unit l % U of row
// l / U of each pass. All loads are issued before the first value is used, lanes
// past the last row reading it again.
template <int D, int PASSES, bool AXES>
struct Block {
  static constexpr int U = D / 16;              // units of a row
  static constexpr int RPP = 64 / U;            // rows of a pass
  int c0, c1;
  float a[PASSES][8], b[PASSES][8];             // a unit's two chunks
  bool mine[PASSES];                            // the lane has a row to write

  __device__ __forceinline__ void read(const Kv8AppendParams& p, bool turn, const uint16_t* src, int64_t stride, int64_t t,
                                       int32_t pos, int count, int lane) {
    const RopeParams& r = p.rope;
    const int j = lane % U;
    c0 = 16 * j;
    c1 = c0 + 8;
    if (turn) unit_columns(r, j, c0, c1);
    u32x4 v0[PASSES], v1[PASSES];
    Positions<AXES> x[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int at = min(i * RPP + lane / U, count - 1);
      v0[i] = load16(src + (t + at) * stride + c0);
      v1[i] = load16(src + (t + at) * stride + c1);
      if (r.cos_sin) x[i] = r.positions ? read_positions<AXES>(r, t + at) : position_at<AXES>(r, pos + at);
      mine[i] = at == i * RPP + lane / U && x[i].ok;
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      unpack8(v0[i], a[i]);
      unpack8(v1[i], b[i]);
      if (turn && j < r.rot_dim / 16) turn_unit(r, read_turn(r, x[i], j), a[i], b[i]);
    }
  }

  // codes: the block's row 0 at this head, ss bytes from row to row; scale: its
  // byte. The new rows are r0, r0 + 1, ..; earlier rows of the sequence are
  // there iff r0 > 0.
  __device__ __forceinline__ void write(uint8_t* codes, int64_t ss, uint8_t* scale, int r0, int lane) const {
    bool any = false;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) any = any || mine[i];
    if (__builtin_amdgcn_ballot_w64(any) == 0) return;   // all rows skipped: the block keeps its scale too
    const int old = r0 > 0 ? int(*scale) - 127 : -128;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t ua = __float_as_uint(a[i][e]) & 0x7FFFFFFFu, ub = __float_as_uint(b[i][e]) & 0x7FFFFFFFu;
        most = max(most, max(ua < 0x7F800000u ? ua : 0u, ub < 0x7F800000u ? ub : 0u));
      }
      top = max(top, mine[i] ? most : 0u);
    }
    const int k = max(scale_exponent(wave_max(top)), old);
    if (r0 > 0 && k > old) {   // a power of two: codes stay exact down to the subnormal ones
      const float f = power_of_two(old - k);
      for (int i = lane; i < r0 * U; i += 64) {
        u32x4* at = reinterpret_cast<u32x4*>(codes + (i / U) * ss + 16 * (i % U));
        u32x4 v = *at;
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] = rescale4(v[w], f);
        *at = v;
      }
    }
    // 2^-k. (The append's own scales end at k = 120; a block that a caller
    // filled may hold 2^127 or NaN, whose inverses, 2^-128 for the latter, are
    // subnormal.)
    const float inv = __uint_as_float(k < 127 ? uint32_t(127 - k) << 23 : 0x400000u >> (k - 127));
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      if (!mine[i]) continue;
      uint8_t* row = codes + (r0 + i * RPP + lane / U) * ss;
      const auto code = [&](const float (&y)[8]) {
        return u32x2{encode4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                     encode4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
      };
      *reinterpret_cast<u32x2*>(row + c0) = code(a[i]);
      *reinterpret_cast<u32x2*>(row + c1) = code(b[i]);
    }
    if (lane == 0) *scale = uint8_t(k + 127);
  }
};

constexpr int kAppendWaves = 4;   // of a work-group

template <int D, bool AXES>
__global__ __launch_bounds__(64 * kAppendWaves) void kv8_append_kernel(Kv8AppendParams p) {
  constexpr int U = D / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = 1 << p.log_waves, w = wave & (waves - 1);   // of the token
  const int64_t t = (int64_t(blockIdx.x) * kAppendWaves + wave) >> p.log_waves;
  if (t >= p.n_tokens) return;
  const bool rope = p.rope.cos_sin != nullptr;
  Positions<AXES> x;
  if (rope && p.rope.positions) x = read_positions<AXES>(p.rope, t);
  const Sequence q = find_sequence(p.qsl, p.seq_lens, p.num_seqs, t, lane);
  // Padding: behind the last sequence or before the first one. (The token's rank
  // among its block's new rows, below, is the first head that it takes: negative
  // for a token before its sequence's first.)
  if (q.s >= p.num_seqs || t < q.start || t >= q.end) return;
  const int64_t q1 = min(int64_t(q.end), p.n_tokens);
  const int32_t pos = int32_t(q.L - (q.end - t));
  if (rope && !p.rope.positions) x = position_at<AXES>(p.rope, pos);
  // The page is loaded here and waited for where something is written: rows,
  // positions and table come in the meantime.
  const int32_t page_at = pos >> __builtin_ctz(p.P);
  const bool in_row = pos >= 0 && page_at < p.bt_stride;
  const int32_t page = p.bt[int64_t(q.s) * p.bt_stride + (in_row ? page_at : 0)];
  if (rope) {
    for (int u = 64 * w + lane; u < (p.Hq + kHeadsPerThread - 1) / kHeadsPerThread * U; u += 64 * waves) {
      const int g = u / U;
      move_units(
          p.rope, x, u - g * U, g * kHeadsPerThread, p.Hq, [&] { return x.ok && in_row && page >= 0 && page < p.num_pages; },
          [&](int h) { return p.q + t * p.q_stride + h * D; }, [&](int h) { return p.q_out + (t * p.Hq + h) * D; });
    }
  }
  // The token's block holds `count` of the call's new rows, from row r0 on, and
  // this token's is the `rank`-th: its waves take every count-th task (a KV
  // head, or its K or V), from the last wave down (the first ones turn queries).
  const int32_t first = max(pos & ~15, q.L - (q.end - max(q.start, 0)));   // position of the block's first new row
  const int r0 = first & 15, rank = pos - first;
  const int64_t tf = t - rank;
  const int count = int(min(int64_t(16 - r0), q1 - tf));   // at least rank + 1
  const int64_t row0 = pos & (p.P - 1) & ~15;         // the block's first slot in its page
  const auto read = [&](auto& b, int h, int kv) {
    b.read(p, rope && !kv, (kv ? p.v_new : p.k_new) + h * D, kv ? p.v_new_stride : p.k_new_stride, tf, first, count, lane);
  };
  const auto write = [&](const auto& b, int h, int kv) {
    b.write(kv ? p.v + page * p.v_sp + row0 * p.v_ss + h * p.v_sh : p.k + page * p.k_sp + row0 * p.k_ss + h * p.k_sh,
            kv ? p.v_ss : p.k_ss, p.scales + page * p.scale_sp + (row0 / 16 * p.Hkv + h) * 2 + kv, r0, lane);
  };
  const auto paged = [&] { return in_row && page >= 0 && page < p.num_pages; };
  const int mine = rank + (waves - 1 - w) * count;
  constexpr int RPP = 64 / U;
  if (count <= RPP) {          // one pass holds the rows: keys and values of a head side by side
    for (int h = mine; h < p.Hkv; h += waves * count) {
      Block<D, 1, AXES> k, v;
      read(k, h, 0);
      read(v, h, 1);
      if (!paged()) break;
      write(k, h, 0);
      write(v, h, 1);
    }
  } else {
    for (int task = mine; task < 2 * p.Hkv; task += waves * count) {
      Block<D, 16 / RPP, AXES> b;
      read(b, task >> 1, task & 1);
      if (!paged()) break;
      write(b, task >> 1, task & 1);
    }
  }
  if (w == 0 && lane == 0 && !(x.ok && paged()) && p.bad_count) atomicAdd(p.bad_count, 1);
}

template <int DK, int DV, bool AXES>
hipError_t launch_rope_append_t(RopeAppendParams p, hipStream_t stream) {
  // Work-groups of up to 512 threads, a unit each: those of as many tokens as
  // 512 threads cover, or of one, in as few equal parts as take them.
  const int units = (p.Hq + p.Hkv + kHeadsPerThread - 1) / kHeadsPerThread * (DK / 16) + (p.kv.cv ? p.Hkv * (DV / 16) : 0);
  p.per_wg = int32_t(std::min<int64_t>(std::max(1, 512 / units), p.kv.n_tokens));
  const int n = units * p.per_wg, parts = (n + 511) / 512;
  const int threads = ((n + parts - 1) / parts + 63) / 64 * 64;
  const int64_t blocks = (p.kv.n_tokens + p.per_wg - 1) / p.per_wg;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((rope_append_kernel<DK, DV, AXES>), dim3(uint32_t(blocks), parts), dim3(threads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const AppendParams& a, hipStream_t stream) {
  const int64_t total = a.n_tokens * (a.ck + a.cv);
  if (total == 0) return hipSuccess;
  const int64_t blocks = (total + 255) / 256;
  if (blocks > int64_t(INT32_MAX)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kv_append_kernel, dim3(uint32_t(blocks)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_rope_append(const RopeAppendParams& p, hipStream_t stream) {
  if (p.kv.n_tokens == 0) return hipSuccess;
  const bool axes = p.rope.n_axes > 1;
  switch (p.kv.dk) {
    case 64: return axes ? launch_rope_append_t<64, 64, true>(p, stream) : launch_rope_append_t<64, 64, false>(p, stream);
    case 128: return axes ? launch_rope_append_t<128, 128, true>(p, stream) : launch_rope_append_t<128, 128, false>(p, stream);
    case 192: return axes ? launch_rope_append_t<192, 128, true>(p, stream) : launch_rope_append_t<192, 128, false>(p, stream);
    case 576: return axes ? launch_rope_append_t<576, 512, true>(p, stream) : launch_rope_append_t<576, 512, false>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_kv8_append(Kv8AppendParams p, int head_dim, hipStream_t stream) {
  if (p.n_tokens == 0 || p.num_seqs == 0) return hipSuccess;
  if (p.n_tokens > INT32_MAX) return hipErrorInvalidValue;
  if (head_dim != 64 && head_dim != 128) return hipErrorInvalidValue;
  const bool axes = p.rope.n_axes > 1;
  const auto kern = head_dim == 128 ? (axes ? kv8_append_kernel<128, true> : kv8_append_kernel<128, false>)
                                    : (axes ? kv8_append_kernel<64, true> : kv8_append_kernel<64, false>);
  // Waves of a token: four where calls are short, where a single token's tasks
  // follow each other in fewer; fewer where tokens fill the machine many times
  // over, most of all those of prompts, which share their block's tasks, with
  // little to turn. One, two and four waves, us: 64 decode tokens of 28/4 heads
  // of 128 12.3, 8.2, 6.0, 2048 of a prompt beside 128 19.2, 14.8, 13.8; prompts
  // of 1 x 1024 9.3, 8.6, 7.5, 1 x 2048 11.7, 11.6, 11.5, 8 x 2048 65.5, 65.7,
  // 68.9, on three axes 89.7, 103, 132; 8 x 2048 of 8/8 heads of 64 25.6, 28.4,
  // 36.9, of 32/8 50.5, 48.0, 51.9, of 4/1 17.3, 22.4, 35.5; 4 x 2048 beside 128
  // decodes, 28/4 of 128, 41.5, 39.2, 42.6.
  const bool prompts = p.n_tokens >= int64_t(64) * p.num_seqs || p.Hkv == 1;   // or one task a token
  const int units = (p.Hq + kHeadsPerThread - 1) / kHeadsPerThread * (head_dim / 16);
  if (prompts && p.n_tokens >= 4096) p.log_waves = axes || units <= 32 ? 0 : 1;
  else p.log_waves = p.n_tokens >= (prompts ? 2048 : 8192) ? 1 : 2;
  const int64_t blocks = ((p.n_tokens << p.log_waves) + kAppendWaves - 1) / kAppendWaves;
  hipLaunchKernelGGL(kern, dim3(uint32_t(blocks)), dim3(64 * kAppendWaves), 0, stream, p);
  return hipGetLastError();
}

}  // namespace flexattn
