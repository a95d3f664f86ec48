// Decode over an 8-bit cache (e4m3 codes, a power-of-two scale for each 16
// keys, KV head and K / V), grouped-query heads of 64 or 128.
//
// The work is laid out as for the bf16 cache: work-group (range r, column c)
// owns one balanced page range and some KV heads, its waves walk the range
// as one stream of chunks with the next chunk's loads in flight, and a piece's
// end writes an output or a partial. What differs:
//
//  - A wave serves 128 bytes of a slot's row, the unit that HBM reads: one head
//    of 128, or two of 64 (a wave for each head of 64 fetched every line
//    twice: 128 sequences of 1000 to 8000 keys, 8 heads, 166 us; with
//    the second half served by L2 134).
//  - A chunk is 64 keys, 16 KB of codes, the bytes in flight that the bf16
//    kernel has with 32.
//  - Codes become bf16 on their way from LDS into the matrix operands
//    (v_cvt_scalef32_pk_bf16_fp8 with the block's scale, exact), so all products
//    are bf16 and nothing is rounded that a bf16 cache would not round.
//  - V passes through the wave's LDS buffer like K: the transposing read
//    gives a lane the 8 keys of one column as 8 bytes, which is the operand
//    once converted.
//
// Bound by HBM: 256 sequences of 2000 keys, 28/4 heads of 128, 83.6 us with
// the merge, 6.3 TB/s; 64 of 4000 47.7, 5.5 TB/s; 128 of 1000 to 8000, 32/8 of
// 64, 105. One sequence of 1000: 10.9, of which the merge takes 3. Memory counters:
// 64 of 512 to 4096 keys, 28/4 heads of 128, fetch 152.5 MB of the 149.7 that
// there are, the 128 sequences 630.6 of 628.4.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "decode_walk.h"
#include "kernels.h"

namespace flexattn {

namespace {

constexpr int kChunk = 64;                       // keys
constexpr int kWaves = 4;                        // of a work-group (the planner gives it at most 4 * kRow bytes of a row)
constexpr int kRow = 128;                        // bytes of a slot's row that a wave serves
constexpr int kStage = 2 * kChunk * kRow;        // a wave's LDS buffer: K rows, then V rows
constexpr int kOutRow = 132;                     // floats from row to row of outputs in the buffer
static_assert(16 * kOutRow * 4 <= kStage, "outputs fit the buffer");

// Physical 16-byte chunk of logical chunk x in row r. K: reads of one chunk by
// the 16 lanes of a lane group hit distinct banks. V: the transposing reads of
// one 16-byte column by two lane groups, rows 4g + i and 16 + 4g + i (i < 4, g
// even and odd), hit distinct banks. Writes of whole rows do in both.
__device__ __forceinline__ int swz_k8(int x, int r) { return x ^ ((r >> 1) & 7); }
__device__ __forceinline__ int swz_v8(int x, int r) { return x ^ (((r >> 1) & 1) | ((r >> 3) & 2) | (r & 4)); }

struct Chunk8 {
  u32x4 k[4][2], v[4][2];   // 16-key block b, load t: row 8t + lane / 8, 16-byte chunk lane % 8
  uint32_t page;            // lane l: page of block l & 3
  uint32_t scales[2];       // lane l: scale bytes (K, V) of block l & 3, of the wave's heads
};

// One decode work-group's work, as decode_gqa_body. COMBINE: several waves serve
// the same heads.
template <int D, int P, bool COMBINE>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(1, 8)))
void decode_kv8_kernel(AttnParams p) {
  static_assert(D == 64 || D == 128, "head dim");
  constexpr int HPW = kRow / D;            // heads of a wave
  constexpr int DC = D / 32;               // 32-dim slices of a head's contraction
  constexpr int CBH = 8 / HPW;             // 16-column blocks of a head
  extern __shared__ __attribute__((aligned(16))) uint8_t s_dyn[];
  __shared__ float s_m[COMBINE ? kWaves : 1][HPW][16], s_l[COMBINE ? kWaves : 1][HPW][16];
  int* const s_pt = reinterpret_cast<int*>(s_dyn + kWaves * kStage);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, gq = lane >> 4;
  const int range = blockIdx.x, col = blockIdx.y, W = gridDim.y;
  const int G = p.G;
  const int HW = p.rows_per_wg / G;                  // KV heads of this work-group
  const int units = (HW + HPW - 1) / HPW;            // and the waves that serve them
  const int WPH = COMBINE ? kWaves / units : 1;
  const int unit = w / WPH, u = w % WPH;
  const int g = col * HW + unit * HPW;               // this wave's first KV head
  const bool active = unit < units && g < p.Hkv;
  // Heads of this wave that exist.
  const int heads = !active ? 0 : min(HPW, min(HW - unit * HPW, p.Hkv - g));
  const int i_begin = p.ranges[range], i_end = p.ranges[range + 1];
  const int g0 = active ? g : 0;
  const uint8_t* kbase = reinterpret_cast<const uint8_t*>(p.kc.base) + int64_t(g0) * p.kc.sh;
  const uint8_t* vbase = reinterpret_cast<const uint8_t*>(p.vc.base) + int64_t(g0) * p.vc.sh;
  const uint32_t ksp = uint32_t(p.kc.sp), kss = uint32_t(p.kc.ss), vsp = uint32_t(p.vc.sp), vss = uint32_t(p.vc.ss);
  // Byte offsets of a block's loads from its first row: row 8t + q8, chunk x8
  // (of the second head from its fourth on; when it does not exist, past every
  // resource, which reads zeros). The heads of a slot are not necessarily side
  // by side, but fewer than 2^31 bytes apart (the host checks it).
  const int q8 = lane >> 3, x8 = lane & 7;
  const bool second = HPW == 2 && x8 >= 4, gone = second && heads < 2;
  const uint32_t kx = second ? uint32_t(p.kc.sh) + 16u * (x8 - 4) : 16u * x8;
  const uint32_t vx = second ? uint32_t(p.vc.sh) + 16u * (x8 - 4) : 16u * x8;
  const uint32_t past_k = heads == 2 ? uint32_t(p.kc.sh) : 0u, past_v = heads == 2 ? uint32_t(p.vc.sh) : 0u;
  uint32_t k_lane[2], v_lane[2], k_wr[2], k_rd[2];
  uint8_t* const stage = s_dyn + w * kStage;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = 8 * t + q8;
    k_lane[t] = gone ? 0x80000000u : uint32_t(row) * kss + kx;
    v_lane[t] = gone ? 0x80000000u : uint32_t(row) * vss + vx;
    k_wr[t] = uint32_t(row * kRow + 16 * swz_k8(x8, row));
    k_rd[t] = uint32_t(n * kRow + 16 * swz_k8(4 * t + gq, n));
  }
  // V writes: row q8 of an even block; 8 rows on the chunk is the same, 16 rows
  // on (odd blocks) bit 1 of the chunk turns. V reads: column block 0 of the
  // lane's key in a 32-key half; column block cb turns the chunk by cb.
  const uint32_t v_wr = uint32_t(kChunk * kRow + q8 * kRow + 16 * swz_v8(x8, q8));
  const int v_row = 16 * (n >> 3) + 4 * gq + ((n >> 1) & 3);
  const uint32_t v_rd = uint32_t(kChunk * kRow + v_row * kRow + 16 * swz_v8(0, v_row) + 8 * (n & 1));

  // The range's block-table entries, piece after piece.
  {
    int poff = 0;
    for (int i = i_begin; i < i_end; ++i) {
      const int k0 = scalar_word(p.items, 8 * i + 3), k1 = scalar_word(p.items, 8 * i + 4);
      const int32_t* bt_row = p.bt + int64_t(scalar_word(p.items, 8 * i)) * p.bt_stride + k0 / P;
      const int npg = pages_in(k0, k1, P);
      for (int t = tid; t < npg; t += kWaves * 64) s_pt[poff + t] = bt_row[t];
      poff += npg;
    }
  }

  auto open = [&](DecodeCursor& c, int i, int poff) {
    for (; active && i < i_end; ++i) {
      const int k0 = scalar_word(p.items, 8 * i + 3), k1 = scalar_word(p.items, 8 * i + 4);
      if (u * kChunk < k1 - k0) {
        c = DecodeCursor{i, u, scalar_word(p.items, 8 * i), k0, k1, poff};
        return;
      }
      poff += pages_in(k0, k1, P);
    }
    c.i = i_end;
  };
  auto advance = [&](DecodeCursor& c) {
    c.ci += WPH;
    if (c.k0 + kChunk * c.ci >= c.k1) open(c, c.i + 1, c.poff + pages_in(c.k0, c.k1, P));
  };

  // Loads of one chunk through buffer resources on each 16-key block (its rows
  // lie in one page). A block's resource ends with the piece's last key in the
  // wave's last head: later rows may be read, within the page, where a cache
  // keeps heads apart, and compute() drops them. As in the bf16 kernel, a
  // cursor past the range issues the same loads, of nothing.
  auto load = [&](Chunk8& c, const DecodeCursor& cur) {
    const bool live = cur.i < i_end;
    const int kc0 = cur.k0 + kChunk * cur.ci;
    const int key = min(kc0 + 16 * (lane & 3), cur.k1 - 1);
    c.page = live ? uint32_t(s_pt[cur.poff + key / P - cur.k0 / P]) : 0u;
    const int64_t at = live ? int64_t(c.page) * p.scale_sp + (key % P / 16 * p.Hkv + g0) * 2 : 0;
    c.scales[0] = *reinterpret_cast<const uint16_t*>(p.kv_scales + at);
    if constexpr (HPW == 2) c.scales[1] = *reinterpret_cast<const uint16_t*>(p.kv_scales + at + (heads == 2 ? 2 : 0));
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const uint32_t rows = uint32_t(__builtin_amdgcn_readfirstlane(live ? min(max(cur.k1 - (kc0 + 16 * b), 0), 16) : 0));
      const uint32_t pg = uint32_t(__builtin_amdgcn_readlane(int(c.page), P == 16 ? b : 0));
      const uint32_t slot = P == 16 ? 0u : uint32_t(kc0 % P + 16 * b);
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(kbase + (uint64_t(pg) * ksp + slot * kss)), 0,
          __builtin_amdgcn_readfirstlane(int(rows ? (rows - 1) * kss + past_k + D : 0u)), kBufferFlags);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(vbase + (uint64_t(pg) * vsp + slot * vss)), 0,
          __builtin_amdgcn_readfirstlane(int(rows ? (rows - 1) * vss + past_v + D : 0u)), kBufferFlags);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        c.k[b][t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, int(k_lane[t]), 0, 2));
#pragma unroll
      for (int t = 0; t < 2; ++t)
        c.v[b][t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, int(v_lane[t]), 0, 2));
    }
  };

  // Q as the B operand of S^T = K Q^T: column n = query head (g + e) * G + n of
  // the piece's token; operand 2t + h of a head holds dims 16 (4t + gq) + 8h ..,
  // as the codes of the row's chunk 4t + gq do.
  u32x4 qop[HPW][DC];
  int q_piece = -1;
  auto load_q = [&](int i) {
    const int tok = scalar_word(p.items, 8 * i + 6);
#pragma unroll
    for (int e = 0; e < HPW; ++e) {
      const bool ok = n < G && e < heads;
      const uint16_t* qr = p.q + (int64_t(tok) * p.Hq + (ok ? (g + e) * G + n : 0)) * D + 16 * gq;
#pragma unroll
      for (int c = 0; c < DC; ++c) qop[e][c] = ok ? load16(qr + 64 * (c >> 1) + 8 * (c & 1)) : zero4();
    }
    q_piece = i;
  };

  float m[HPW], l[HPW];
  f32x4 o[HPW][CBH];
  auto reset = [&]() {
#pragma unroll
    for (int e = 0; e < HPW; ++e) {
      m[e] = -INFINITY;
      l[e] = 0.f;
#pragma unroll
      for (int a = 0; a < CBH; ++a) o[e][a] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  reset();

  auto compute = [&](Chunk8& c, const DecodeCursor& cur) {
    const int kc0 = cur.k0 + kChunk * cur.ci;
    if (kc0 + kChunk > cur.k1) {   // slots past the last key may hold NaN, which a probability of 0 does not remove
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (kc0 + 16 * b + 8 * t + q8 >= cur.k1) c.v[b][t] = zero4();
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        *reinterpret_cast<u32x4*>(stage + k_wr[t] + 16 * kRow * b) = c.k[b][t];
        *reinterpret_cast<u32x4*>(stage + (b & 1 ? v_wr ^ 32u : v_wr) + 16 * kRow * b + 8 * kRow * t) = c.v[b][t];
      }
    wave_lds_sync();
    f32x4 s[HPW][4];
    u32x4 x[4][2];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t) x[b][t] = *reinterpret_cast<const u32x4*>(stage + k_rd[t] + 16 * kRow * b);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
      for (int e = 0; e < HPW; ++e) s[e][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 2; ++t) {      // a head of 128 has both of the lane's chunks, one of 64 its own
        const int e = HPW == 2 ? t : 0, c0 = HPW == 2 ? 0 : 2 * t;
        const float f = scale_of(uint32_t(__builtin_amdgcn_readlane(int(c.scales[e]), b)));
        s[e][b] = mfma_16x16x32(codes_bf16x8(x[b][t][0], x[b][t][1], f, f), qop[e][c0], s[e][b]);
        s[e][b] = mfma_16x16x32(codes_bf16x8(x[b][t][2], x[b][t][3], f, f), qop[e][c0 + 1], s[e][b]);
      }
    }
    u32x4 pop[HPW][2];
#pragma unroll
    for (int e = 0; e < HPW; ++e)
      softmax_chunk(s[e], kc0 + kChunk > cur.k1, kc0, cur.k1, gq, p.scale_log2, m[e], l[e], o[e], pop[e]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 0; e < HPW; ++e) {
        const float f0 = scale_of(uint32_t(__builtin_amdgcn_readlane(int(c.scales[e]), 2 * h)) >> 8);
        const float f1 = scale_of(uint32_t(__builtin_amdgcn_readlane(int(c.scales[e]), 2 * h + 1)) >> 8);
#pragma unroll
        for (int a = 0; a < CBH; ++a) {
          const u32x2 y = lds_read_tr8(stage + (v_rd ^ uint32_t(16 * (e * CBH + a))) + 32 * kRow * h);
          o[e][a] = mfma_16x16x32(pop[e][h], codes_bf16x8(y[0], y[1], f0, f1), o[e][a]);
        }
      }
    }
    wave_lds_sync();
  };

  // Write piece i's result: the output of a whole sequence or the partial of a
  // split one. Lane (n, gq) holds columns 16a + n of rows 4gq + r; they pass
  // through the wave's buffer so that a lane writes 8 columns of a row.
  auto finish = [&](int i) {
    const int nspl = scalar_word(p.items, 8 * i + 2);
    const int tok = scalar_word(p.items, 8 * i + 6);
    const int64_t slot = int64_t(scalar_word(p.items, 8 * i + 7)) * W + col;   // this piece's workspace slot
    float* const s_o = reinterpret_cast<float*>(stage);
#pragma unroll
    for (int e = 0; e < HPW; ++e)
#pragma unroll
      for (int a = 0; a < CBH; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) s_o[(4 * gq + r) * kOutRow + 16 * (e * CBH + a) + n] = o[e][a][r];
    auto put = [&](int head, int row, int d, const f32x4& v0, const f32x4& v1, float mr, float lr) {
      if (nspl == 1) {
        const float inv = 1.f / lr;
        *reinterpret_cast<u32x4*>(p.out + (int64_t(tok) * p.Hq + head * G + row) * D + d) =
            u32x4{pack_bf16x2(v0[0] * inv, v0[1] * inv), pack_bf16x2(v0[2] * inv, v0[3] * inv),
                  pack_bf16x2(v1[0] * inv, v1[1] * inv), pack_bf16x2(v1[2] * inv, v1[3] * inv)};
        if (d == 0 && p.lse) p.lse[int64_t(tok) * p.Hq + head * G + row] = (mr + log2f(lr)) * kLn2;
      } else {
        const int64_t srow = slot * p.rows_per_wg + (head - col * HW) * G + row;
        *reinterpret_cast<f32x4*>(p.ws_o + srow * D + d) = v0;
        *reinterpret_cast<f32x4*>(p.ws_o + srow * D + d + 4) = v1;
        if (d == 0) {
          p.ws_stats[srow * 2] = mr;
          p.ws_stats[srow * 2 + 1] = lr;
        }
      }
    };
    float lt[HPW];
#pragma unroll
    for (int e = 0; e < HPW; ++e) lt[e] = group_sum(l[e]);
    if constexpr (!COMBINE) {
      wave_lds_sync();
      const int e = 8 * n / D, d = 8 * n % D;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 4 * r + gq;
        float mr = shfl_f(m[0], row), lr = shfl_f(lt[0], row);
        if constexpr (HPW == 2) {
          const float m1 = shfl_f(m[1], row), l1 = shfl_f(lt[1], row);
          mr = e ? m1 : mr;
          lr = e ? l1 : lr;
        }
        const float* src = s_o + row * kOutRow + 8 * n;
        if (row < G && e < heads)
          put(g + e, row, d, *reinterpret_cast<const f32x4*>(src), *reinterpret_cast<const f32x4*>(src + 4), mr, lr);
      }
      wave_lds_sync();
    } else {
      // Several waves per head: their states meet in LDS.
      if (gq == 0) {
#pragma unroll
        for (int e = 0; e < HPW; ++e) {
          s_m[w][e][n] = m[e];
          s_l[w][e][n] = lt[e];
        }
      }
      lds_barrier();
      for (int idx = tid; idx < units * G * 16; idx += kWaves * 64) {
        const int un = idx / (G * 16), row = idx / 16 % G, c = 8 * (idx % 16);
        const int e = c / D, head = col * HW + un * HPW + e;
        if (un * HPW + e >= HW || head >= p.Hkv) continue;
        float M = -INFINITY;
        for (int ww = 0; ww < WPH; ++ww) M = fmaxf(M, s_m[un * WPH + ww][e][row]);
        float den = 0.f;
        f32x4 v0 = {0.f, 0.f, 0.f, 0.f}, v1 = v0;
        for (int ww = 0; ww < WPH; ++ww) {
          const float mw = s_m[un * WPH + ww][e][row];
          const float f = mw == -INFINITY ? 0.f : fast_exp2(mw - M);
          const float* src = reinterpret_cast<const float*>(s_dyn + (un * WPH + ww) * kStage) + row * kOutRow + c;
          den += f * s_l[un * WPH + ww][e][row];
          v0 += f * *reinterpret_cast<const f32x4*>(src);
          v1 += f * *reinterpret_cast<const f32x4*>(src + 4);
        }
        put(head, row, c % D, v0, v1, M, den);
      }
      lds_barrier();   // the buffers are free again
    }
    reset();
  };

  // Finish every piece before i, then make sure Q is piece i's (every wave
  // finishes every piece of the range in order: several waves per head meet in
  // each).
  int fin = i_begin;
  auto enter = [&](int i) {
    for (; fin < i; ++fin) finish(fin);
    if (q_piece != i) load_q(i);
  };

  DecodeCursor c{i_end, 0, 0, 0, 0, 0};
  open(c, i_begin, 0);
  if (c.i < i_end) load_q(c.i);
  wait_vmem_all();
  lds_barrier();   // the page window is complete

  // Two fixed chunk buffers, the loop unrolled by two (see the bf16 kernel for
  // the order: everything a chunk waits for is issued before the next one's
  // loads).
  Chunk8 A, B;
  load(A, c);
  while (c.i < i_end) {
    enter(c.i);
    DecodeCursor c2 = c;
    advance(c2);
    load(B, c2);
    compute(A, c);
    if (c2.i >= i_end) break;
    enter(c2.i);
    DecodeCursor c3 = c2;
    advance(c3);
    load(A, c3);
    compute(B, c2);
    c = c3;
  }
  for (; fin < i_end; ++fin) finish(fin);
}

// Split-K merge of sequences with many pieces: a work-group per output row, its
// threads in PG groups over the pieces (group j takes j, j + PG, ..), four
// loads each in flight, joined through LDS in group order. The merge with one
// thread per four columns walks the pieces alone, eight at a time: one sequence
// of 16,000 keys in 250 pieces took 41 us with its decode, now 15.
template <int DV>
__global__ __launch_bounds__(256) void merge_many_kernel(AttnParams p) {
  constexpr int CT = DV / 4, PG = 256 / CT, KB = 4;
  __shared__ float s_m[PG], s_l[PG];
  __shared__ f32x4 s_o[PG][CT];
  const int32_t* it = p.items + 8 * p.merge[blockIdx.x];   // the sequence's first piece
  const int col = blockIdx.y, W = gridDim.y, i = blockIdx.z;
  const int rows = p.rows_per_wg, head = col * rows + i;
  if (head >= p.Hq) return;
  const int nspl = it[2], slot0 = it[5];
  const int c = threadIdx.x % CT, pg = threadIdx.x / CT;
  float M = -INFINITY, den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = pg; j0 < nspl; j0 += KB * PG) {
    float mj[KB], lj[KB];
    f32x4 vj[KB];
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int j = j0 + k * PG;
      const int64_t r = (int64_t(slot0 + min(j, nspl - 1)) * W + col) * rows + i;
      mj[k] = j < nspl ? p.ws_stats[r * 2] : -INFINITY;
      lj[k] = p.ws_stats[r * 2 + 1];
      vj[k] = *reinterpret_cast<const f32x4*>(p.ws_o + r * DV + 4 * c);
    }
    float Mn = M;
#pragma unroll
    for (int k = 0; k < KB; ++k) Mn = fmaxf(Mn, mj[k]);
    const float sc = M == -INFINITY ? 0.f : fast_exp2(M - Mn);
    den *= sc;
    acc *= sc;
    M = Mn;
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const float f = mj[k] == -INFINITY ? 0.f : fast_exp2(mj[k] - M);
      den += f * lj[k];
      acc += f * vj[k];
    }
  }
  if (c == 0) {
    s_m[pg] = M;
    s_l[pg] = den;
  }
  s_o[pg][c] = acc;
  __syncthreads();
  if (pg != 0) return;
  float top = s_m[0];
  for (int k = 1; k < PG; ++k) top = fmaxf(top, s_m[k]);
  den = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < PG; ++k) {
    const float f = s_m[k] == -INFINITY ? 0.f : fast_exp2(s_m[k] - top);
    den += f * s_l[k];
    acc += f * s_o[k][c];
  }
  const float inv = 1.f / den;
  const int64_t row = int64_t(it[6]) * p.Hq + head;
  *reinterpret_cast<u32x2*>(p.out + row * DV + 4 * c) =
      u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
  if (c == 0 && p.lse) p.lse[row] = (top + log2f(den)) * kLn2;
}

template <int D, int P>
hipError_t launch_t(const AttnParams& p, hipStream_t stream) {
  const dim3 grid(p.n_ranges, p.grid_y);
  const size_t window = size_t(std::max(p.range_pages, 1)) * 4;
  const int hw = p.rows_per_wg / p.G, units = (hw * D + kRow - 1) / kRow;
  auto go = [&](auto kern) {
    const size_t lds = size_t(kWaves) * kStage + window;
    const hipError_t attr = set_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, grid, dim3(kWaves * 64), lds, stream, p);
    return hipGetLastError();
  };
  // One wave per 128 bytes of a slot; when that is one or two, four share them.
  return units <= 2 ? go(decode_kv8_kernel<D, P, true>) : go(decode_kv8_kernel<D, P, false>);
}

}  // namespace

hipError_t launch_merge_many(const AttnParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.n_merge, p.grid_y, p.rows_per_wg);
  if (head_dim == 128) hipLaunchKernelGGL(merge_many_kernel<128>, grid, dim3(256), 0, stream, p);
  else if (head_dim == 64) hipLaunchKernelGGL(merge_many_kernel<64>, grid, dim3(256), 0, stream, p);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_decode_kv8(const AttnParams& p, int head_dim, hipStream_t stream) {
  if (p.P != 16 && p.P != 64) return hipErrorInvalidValue;
  if (head_dim == 128) return p.P == 16 ? launch_t<128, 16>(p, stream) : launch_t<128, 64>(p, stream);
  if (head_dim == 64) return p.P == 16 ? launch_t<64, 16>(p, stream) : launch_t<64, 64>(p, stream);
  return hipErrorInvalidValue;
}

}  // namespace flexattn
