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
// Positions of one token on its axes.
struct Positions {
  int32_t p[kRopeMaxAxes];
  bool ok;
};

__device__ __forceinline__ Positions read_positions(const RopeParams& r, int64_t t) {
  Positions x;
  x.ok = true;
#pragma unroll
  for (int a = 0; a < kRopeMaxAxes; ++a) {
    x.p[a] = a < r.n_axes ? r.positions[a * r.positions_stride + t] : 0;
    x.ok = x.ok && x.p[a] >= 0 && x.p[a] < r.max_position;
  }
  return x;
}

// The one position of a token that has no table of positions of its own.
__device__ __forceinline__ Positions position_at(const RopeParams& r, int32_t pos) {
  return Positions{{pos, 0, 0, 0}, pos >= 0 && pos < r.max_position};
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

__device__ __forceinline__ int32_t pick(const Positions& x, int a) {
  return a == 0 ? x.p[0] : a == 1 ? x.p[1] : a == 2 ? x.p[2] : x.p[3];
}

// Cosines and sines of pairs 8 j .. 8 j + 7 at a token's positions: from one
// table row when one axis has them all, else pair by pair.
struct Turn {
  float c[8], s[8];
};

__device__ __forceinline__ Turn read_turn(const RopeParams& r, const Positions& x, int j) {
  Turn t;
  const int half = r.rot_dim / 2;
  const int a0 = r.n_axes == 1 ? 0 : axis_of(r, 8 * j);
  if (r.n_axes == 1 || (!r.dealt && axis_of(r, 8 * j + 7) == a0)) {
    const float* row = r.cos_sin + int64_t(pick(x, a0)) * r.rot_dim + 8 * j;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const f32x4 c = *reinterpret_cast<const f32x4*>(row + 4 * v);
      const f32x4 s = *reinterpret_cast<const f32x4*>(row + half + 4 * v);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        t.c[4 * v + e] = c[e];
        t.s[4 * v + e] = s[e];
      }
    }
    return t;
  }
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

// One unit of a head's row from src to dst (both at the head's first column).
__device__ __forceinline__ void move_unit(const RopeParams& r, const Positions& x, int j, const uint16_t* src,
                                          uint16_t* dst) {
  int c0, c1;
  unit_columns(r, j, c0, c1);
  u32x4 v0 = load16(src + c0), v1 = load16(src + c1);
  if (j < r.rot_dim / 16) {
    const Turn t = read_turn(r, x, j);
    float a[8], b[8];
    unpack8(v0, a);
    unpack8(v1, b);
    turn_unit(r, t, a, b);
    v0 = pack8(a);
    v1 = pack8(b);
  }
  *reinterpret_cast<u32x4*>(dst + c0) = v0;
  *reinterpret_cast<u32x4*>(dst + c1) = v1;
}

// ---------------------------------------------------------------------------
// Into the bf16 cache: a work-group takes `per_wg` tokens and walks their
// units (queries, keys, values). Bound by HBM; the table rows are read by every
// head of a token and come from the caches.
// ---------------------------------------------------------------------------
template <int DK, int DV>
__global__ __launch_bounds__(512) void rope_append_kernel(RopeAppendParams p) {
  constexpr int UK = DK / 16, UV = DV / 16;
  const AppendParams& a = p.kv;
  const int nq = p.Hq * UK, nk = p.Hkv * UK, nv = a.cv ? p.Hkv * UV : 0;
  const int per_tok = nq + nk + nv;
  const int64_t t0 = int64_t(blockIdx.x) * p.per_wg;
  const int n = int(min(int64_t(p.per_wg), a.n_tokens - t0)) * per_tok;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int dt = p.per_wg == 1 ? 0 : i / per_tok;
    int u = i - dt * per_tok;
    const int64_t t = t0 + dt;
    const int32_t slot = a.slot_mapping[t];
    if (slot < 0) continue;                    // padding token
    const Positions x = read_positions(p.rope, t);
    if (!x.ok || int64_t(slot) >= a.num_slots) {
      if (u == 0 && a.bad_count) atomicAdd(a.bad_count, 1);
      continue;
    }
    if (u < nq) {
      const int h = u / UK;
      move_unit(p.rope, x, u - h * UK, p.q + t * p.q_stride + h * DK, p.q_out + (t * p.Hq + h) * DK);
      continue;
    }
    u -= nq;
    const int64_t page = slot / a.P, row = slot - page * a.P;
    if (u < nk) {
      const int h = u / UK;
      move_unit(p.rope, x, u - h * UK, a.k_new + t * a.k_new_stride + h * DK,
                const_cast<uint16_t*>(a.kc.base) + page * a.kc.sp + row * a.kc.ss + h * a.kc.sh);
    } else {
      u -= nk;
      const int h = u / UV, c = 16 * (u - h * UV);
      const uint16_t* src = a.v_new + t * a.v_new_stride + h * DV + c;
      uint16_t* dst = const_cast<uint16_t*>(a.vc.base) + page * a.vc.sp + row * a.vc.ss + h * a.vc.sh + c;
      const u32x4 v0 = load16(src), v1 = load16(src + 8);
      *reinterpret_cast<u32x4*>(dst) = v0;
      *reinterpret_cast<u32x4*>(dst + 8) = v1;
    }
  }
}

// ---------------------------------------------------------------------------
// Into the 8-bit cache. Work-group t takes new token t: it finds the token's
// sequence, turns its query, and, when the token is the first of its block in
// this call, quantises the block's new rows, one wave for each KV head and K or
// V (the rows of a block are consecutive new tokens, so no two work-groups
// touch a block). A wave holds its rows in registers between the maximum that
// gives the scale and the conversion, so they are read once.
// ---------------------------------------------------------------------------

// The sequence that holds new token t (B: none): the largest s with
// query_start_loc[s] <= t, 64 probes at a time.
__device__ __forceinline__ int find_sequence(const int32_t* qsl, int B, int64_t t, int lane) {
  int base = 0, len = B;
  while (len > 0) {
    const int step = (len + 63) / 64;
    const int64_t x = base + int64_t(lane + 1) * step;
    const bool below = x <= base + len && int64_t(qsl[x]) <= t;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
    const int end = base + len;
    base += n * step;
    len = min(step - 1, end - base);
  }
  return __builtin_amdgcn_readfirstlane(base);
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

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v = max(v, uint32_t(__shfl_xor(int(v), m, 64)));
  return v;
}

// Rows r0 .. r1 - 1 of one block for one KV head, keys or values: row r is new
// token t + r - r0. codes: the block's row 0 at this head; scale: its byte.
template <int D>
__device__ __forceinline__ void quantise_block(const Kv8AppendParams& p, bool turn, const uint16_t* src, int64_t stride,
                                               int64_t t, int32_t pos, int r0, int r1, uint8_t* codes, int64_t ss,
                                               uint8_t* scale, int lane) {
  constexpr int U = D / 16;              // units of a row
  constexpr int RPP = 64 / U;            // rows of a pass
  constexpr int PASSES = 16 / RPP;
  const RopeParams& r = p.rope;
  const bool kept = r0 > 0;              // the block holds earlier rows of the sequence
  const int old = kept ? int(*scale) - 127 : -128;
  const int j = lane % U;
  int c0 = 16 * j, c1 = c0 + 8;
  if (turn) unit_columns(r, j, c0, c1);
  float a[PASSES][8], b[PASSES][8];
  bool write[PASSES];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = i * RPP + lane / U;
    write[i] = row >= r0 && row < r1;
    if (!write[i]) continue;
    const int64_t tok = t + row - r0;
    Positions x{{0, 0, 0, 0}, true};
    if (r.cos_sin) x = r.positions ? read_positions(r, tok) : position_at(r, pos + row - r0);
    if (!x.ok) {
      write[i] = false;
      continue;
    }
    unpack8(load16(src + tok * stride + c0), a[i]);
    unpack8(load16(src + tok * stride + c1), b[i]);
    if (turn && j < r.rot_dim / 16) turn_unit(r, read_turn(r, x, j), a[i], b[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t ua = __float_as_uint(a[i][e]) & 0x7FFFFFFFu, ub = __float_as_uint(b[i][e]) & 0x7FFFFFFFu;
      top = max(top, max(ua < 0x7F800000u ? ua : 0u, ub < 0x7F800000u ? ub : 0u));
    }
  }
  const int k = max(scale_exponent(wave_max(top)), old);
  if (kept && k > old) {   // a power of two: codes stay exact down to the subnormal ones
    const float f = power_of_two(old - k);
    for (int i = lane; i < r0 * U; i += 64) {
      u32x4* at = reinterpret_cast<u32x4*>(codes + (i / U) * ss + 16 * (i % U));
      u32x4 v = *at;
#pragma unroll
      for (int w = 0; w < 4; ++w) v[w] = rescale4(v[w], f);
      *at = v;
    }
  }
  const float inv = __uint_as_float(uint32_t(max(127 - k, 1)) << 23);
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    if (!write[i]) continue;
    uint8_t* row = codes + (i * RPP + lane / U) * ss;
    const auto code = [&](const float (&x)[8]) {
      return u32x2{encode4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                   encode4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
    };
    *reinterpret_cast<u32x2*>(row + c0) = code(a[i]);
    *reinterpret_cast<u32x2*>(row + c1) = code(b[i]);
  }
  if (lane == 0) *scale = uint8_t(k + 127);
}

template <int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8AppendParams p) {
  constexpr int U = D / 16;
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = find_sequence(p.qsl, p.num_seqs, t, lane);
  if (s >= p.num_seqs) return;           // padding token
  const int64_t q0 = p.qsl[s], q1 = min(int64_t(p.qsl[s + 1]), p.n_tokens);
  const int32_t pos = int32_t(p.seq_lens[s] - (p.qsl[s + 1] - t));
  const int32_t page_at = pos / p.P;
  int32_t page = -1;
  if (pos >= 0 && page_at < p.bt_stride) page = p.bt[int64_t(s) * p.bt_stride + page_at];
  const bool paged = page >= 0 && int64_t(page) < p.num_pages;
  const bool rope = p.rope.cos_sin != nullptr;
  Positions x{{0, 0, 0, 0}, true};
  if (rope) x = p.rope.positions ? read_positions(p.rope, t) : position_at(p.rope, pos);
  if (!paged || !x.ok) {
    if (threadIdx.x == 0 && p.bad_count) atomicAdd(p.bad_count, 1);
  } else if (rope) {
    for (int u = threadIdx.x; u < p.Hq * U; u += blockDim.x) {
      const int h = u / U;
      move_unit(p.rope, x, u - h * U, p.q + t * p.q_stride + h * D, p.q_out + (t * p.Hq + h) * D);
    }
  }
  const int r0 = pos & 15;
  if (!paged || (t != q0 && r0 != 0)) return;   // the block is an earlier token's
  const int r1 = int(min(int64_t(16), r0 + (q1 - t)));
  const int64_t row0 = pos % p.P - r0;          // the block's first slot in its page
  for (int task = w; task < 2 * p.Hkv; task += blockDim.x / 64) {
    const int kv = task & 1, h = task >> 1;
    uint8_t* codes = kv ? p.v + page * p.v_sp + row0 * p.v_ss + h * p.v_sh : p.k + page * p.k_sp + row0 * p.k_ss + h * p.k_sh;
    uint8_t* scale = p.scales + page * p.scale_sp + (row0 / 16 * p.Hkv + h) * 2 + kv;
    quantise_block<D>(p, rope && !kv, (kv ? p.v_new : p.k_new) + h * D, kv ? p.v_new_stride : p.k_new_stride, t, pos, r0,
                      r1, codes, kv ? p.v_ss : p.k_ss, scale, lane);
  }
}

template <int DK, int DV>
hipError_t launch_rope_append_t(RopeAppendParams p, hipStream_t stream) {
  // Work-groups of up to 512 threads: a token's units, or those of as many
  // tokens as 512 threads cover at one unit each; when a token has more, as
  // few threads as take them in the same number of rounds.
  const int units = (p.Hq + p.Hkv) * (DK / 16) + (p.kv.cv ? p.Hkv * (DV / 16) : 0);
  p.per_wg = int32_t(std::min<int64_t>(std::max(1, 512 / units), p.kv.n_tokens));
  const int n = units * p.per_wg, rounds = (n + 511) / 512;
  const int threads = ((n + rounds - 1) / rounds + 63) / 64 * 64;
  const int64_t blocks = (p.kv.n_tokens + p.per_wg - 1) / p.per_wg;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((rope_append_kernel<DK, DV>), dim3(uint32_t(blocks)), dim3(threads), 0, stream, p);
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
  switch (p.kv.dk) {
    case 64: return launch_rope_append_t<64, 64>(p, stream);
    case 128: return launch_rope_append_t<128, 128>(p, stream);
    case 192: return launch_rope_append_t<192, 128>(p, stream);
    case 576: return launch_rope_append_t<576, 512>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_kv8_append(const Kv8AppendParams& p, int head_dim, hipStream_t stream) {
  if (p.n_tokens == 0 || p.num_seqs == 0) return hipSuccess;
  if (p.n_tokens > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid(uint32_t(p.n_tokens)), threads(256);
  if (head_dim == 128) hipLaunchKernelGGL(kv8_append_kernel<128>, grid, threads, 0, stream, p);
  else if (head_dim == 64) hipLaunchKernelGGL(kv8_append_kernel<64>, grid, threads, 0, stream, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace flexattn
