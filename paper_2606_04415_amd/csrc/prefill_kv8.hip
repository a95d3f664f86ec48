// Prefill over an 8-bit cache (e4m3 codes, a power-of-two scale for each 16
// keys, KV head and K / V), grouped-query heads of 64 or 128.
//
// Tiles of 128 rows, a row being a (token, query head) pair of one KV head, as
// for the bf16 cache: four waves of 32 rows walk the tile's keys 32 at a time
// with a running maximum and sum for each row. What differs:
//
//  - Codes come by DMA into a ring of two raw tiles, and each wave converts the
//    part that it loaded into the bf16 tile of a stage (exact, a code has 4
//    significant bits), once for the work-group. All products are bf16.
//  - Products of 32x32x16: a wave's 32 rows are one operand, a row's running
//    maximum and sum sit in one lane (and its other half's), and half as many
//    instructions as of 16x16x32 leave issue slots to the softmax. 28/4 heads
//    of 128, us: a prompt of 2048 on 4096 keys 215 with 16x16x32 and 197 so, 32/8
//    of 64 146 and 135.
//  - One group of waves, or KG = 2 that take the key tiles in turn and join
//    their states at the end, where the longest tile would outlast the rest
//    (the rule is in plan.cpp).
//  - A tile's keys may be cut into pieces (plan.cpp); merge_tiles_kernel joins
//    them.
//
// Measured: eight prompts of 2048, 28/4 heads of 128, 275 to 302 us by box and
// clock, 797 to 875 TFLOP/s (the first 60 launches of a process 322 in the mean);
// 159 MB fetched, of which the keys and values 2.5 times over. With
// the machine full the clock gives way: against 16x16x32 it takes 6% fewer
// clocks and 2% more time, at 2.1 GHz instead of 2.25, and vector work, operand
// reads and products each fill less than two thirds of the clocks.
#include <float.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "decode_walk.h"
#include "kernels.h"

namespace flexattn {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kKeys = 32;      // of a tile
constexpr int kWaves = 4;      // of a key group
constexpr int kTileRows = 128;

// Lane l = 32h + n supplies row n of A and column n of B, 8 contraction slots
// of half h each, and receives D[8i + 4h + r][n] in register 4i + r.
__device__ __forceinline__ f32x16 mfma_32x32x16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Physical 16-byte chunk of logical chunk x in row r of a stage's K and V: the
// rows that one operand read touches at a time fall into distinct banks.
template <int D>
__device__ __forceinline__ int swizzle_k(int x, int r) {
  return x ^ (D == 128 ? r & 15 : (r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int swizzle_v(int x, int r) {
  return x ^ (4 * (D == 128 ? r & 3 : (r >> 1) & 1));
}

template <int D, int P, int KG>
struct Layout {
  static constexpr int ROW = 2 * D;                 // bytes of a bf16 row
  static constexpr int V_OFF = kKeys * ROW, STAGE = 2 * V_OFF;
  static constexpr int RAW = 2 * kKeys * D;         // bytes of a raw tile
  static constexpr int WIN = P == 16 ? 512 : 256;   // block-table entries of a window
  static constexpr int BPP = P / 16;                // blocks of a page
  // LDS: each group's two stages and two raw tiles, the window's pages, its
  // blocks' scale bytes; at the end, the states of all groups but the first.
  static constexpr int REGION = 2 * STAGE + 2 * RAW, PT_OFF = KG * REGION, SC_OFF = PT_OFF + 4 * WIN;
  static constexpr int STATE = kWaves * 64 * (2 * D + 16);   // of a group: accumulators, maxima and sums
  static constexpr size_t LDS_BYTES = std::max<size_t>(SC_OFF + 2 * WIN * BPP, (KG - 1) * STATE);
  static_assert(REGION % 256 == 0 && V_OFF % 256 == 0, "operand columns enter their addresses by exclusive or");
};

// Loads and conversion. A load covers 64 16-byte chunks, whole rows of K or of
// V, which all lie in one block of 16 keys: page, resource and scale are
// wave-uniform.
template <int D, int P, int KG>
struct Loader {
  using L = Layout<D, P, KG>;
  static constexpr int CPR = D / 16;         // 16-byte chunks of codes in a row
  static constexpr int RPL = 64 / CPR;       // rows of a load
  static constexpr int NL = 2 * kKeys * CPR / 256;   // loads of a wave per tile: K then V (head dim 128), or K or V (64)

  uint8_t* lds;                              // the group's region
  const int* s_pt;
  const uint16_t* s_sc;
  const uint8_t* base[NL];
  uint32_t sp[NL], ss[NL], ld_off[NL], st_off[NL][2];
  int key_end, row0, lane, w;                // row0: first row of the wave's loads
  bool is_v[NL];
  u32x4 x[NL];                               // read_raw() to convert()
  uint32_t scale;

  __device__ __forceinline__ Loader(const AttnParams& p, int head, uint8_t* lds_, int w_, int lane_, int key_end_,
                                    int group)
      : lds(lds_ + group * L::REGION), s_pt(reinterpret_cast<const int*>(lds_ + L::PT_OFF)),
        s_sc(reinterpret_cast<const uint16_t*>(lds_ + L::SC_OFF)), key_end(key_end_), lane(lane_), w(w_) {
    row0 = RPL * (w % (kKeys / RPL));
    const int row = row0 + lane / CPR, c = lane % CPR;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      is_v[j] = NL == 2 ? j == 1 : w >= 2;
      const CacheRef& r = is_v[j] ? p.vc : p.kc;
      base[j] = reinterpret_cast<const uint8_t*>(r.base) + int64_t(head) * r.sh;
      sp[j] = uint32_t(r.sp);
      ss[j] = uint32_t(r.ss);
      ld_off[j] = uint32_t(lane / CPR) * ss[j] + 16u * uint32_t(lane % CPR);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        st_off[j][h] = is_v[j] ? uint32_t(L::V_OFF + row * L::ROW + 16 * swizzle_v<D>(2 * c + h, row))
                               : uint32_t(row * L::ROW + 16 * swizzle_k<D>(2 * c + h, row));
    }
  }
  __device__ __forceinline__ uint8_t* raw(int slot, int j) const {
    return lds + 2 * L::STAGE + slot * L::RAW + (w * NL + j) * 1024;
  }
  // Page of the wave's loads of the tile at kb.
  __device__ __forceinline__ int first_page(int kb, int pt_base) const {
    return s_pt[uint32_t(min(kb + row0, key_end - 1)) / P - uint32_t(pt_base)];
  }
  // Start the loads of the tile at kb into a raw slot. Rows past key_end repeat
  // the last key's (masked later). (A tile starts on a multiple of 32 keys, so
  // at page 16 the wave's first slot in its page is the same in every tile.)
  __device__ __forceinline__ void fetch(int kb, int slot, int first) const {
    const uint32_t page = uint32_t(__builtin_amdgcn_readfirstlane(first));
    const bool whole = kb + row0 + RPL <= key_end;
    const int key = min(kb + row0, key_end - 1);
    const uint32_t in_page = P == 16 && whole ? uint32_t(row0) % 16 : uint32_t(key) % P;
    i32x4 r[NL];
#pragma unroll
    for (int j = 0; j < NL; ++j)
      r[j] = uniform_rsrc(base[j] + (uint64_t(page) * sp[j] + in_page * ss[j]), uint32_t(RPL) * ss[j]);
    if (whole) {
#pragma unroll
      for (int j = 0; j < NL; ++j) dma16_buf(r[j], ld_off[j], raw(slot, j));
    } else {
      const uint32_t row = uint32_t(min(lane / CPR, key_end - 1 - key));
#pragma unroll
      for (int j = 0; j < NL; ++j) dma16_buf(r[j], row * ss[j] + 16u * uint32_t(lane % CPR), raw(slot, j));
    }
  }
  // The wave's part of the raw tile at kb, whose loads have landed, into
  // registers; then as bf16 into a stage.
  __device__ __forceinline__ void read_raw(int kb, int slot, int pt_base) {
    uint32_t block = uint32_t(min(kb + row0, key_end - 1)) / 16 - uint32_t(pt_base * L::BPP);
    asm volatile("" : "+v"(block));   // read into a vector register: a scalar one would be waited for here
    scale = s_sc[block];
#pragma unroll
    for (int j = 0; j < NL; ++j) x[j] = *reinterpret_cast<const u32x4*>(raw(slot, j) + 16 * lane);
  }
  __device__ __forceinline__ void convert(int st) const {
    uint8_t* stage = lds + st * L::STAGE;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const float f = scale_of(is_v[j] ? scale >> 8 : scale);
      *reinterpret_cast<u32x4*>(stage + st_off[j][0]) = codes_bf16x8(x[j][0], x[j][1], f, f);
      *reinterpret_cast<u32x4*>(stage + st_off[j][1]) = codes_bf16x8(x[j][2], x[j][3], f, f);
    }
  }
};

template <int D, int P, int KG, int WPE>
__global__ __launch_bounds__(64 * kWaves * KG) __attribute__((amdgpu_waves_per_eu(WPE)))
void prefill_kv8_kernel(AttnParams p) {
  using L = Layout<D, P, KG>;
  constexpr int NQ = D / 16, NC = D / 32;   // 16-column parts of the scores' products; 32-column blocks of an output
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];

  // Work-group -> (item, KV head): when the head count divides 8, the tiles of
  // a head run on the same XCDs (work-group b runs on XCD b % 8), whose L2 then
  // holds that head's keys only.
  int item = int(blockIdx.x), head = int(blockIdx.y);
  if (p.xcd_remap) {
    const int x = int(blockIdx.x) & 7, j = int(blockIdx.x) >> 3;
    head = x % p.grid_y;
    item = j * (8 / p.grid_y) + x / p.grid_y;
    if (item >= p.n_items) return;
  }

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = KG > 1 ? wave % kWaves : wave, group = KG > 1 ? wave / kWaves : 0;
  const int32_t* it = p.items + 8 * item;
  const int seq = it[0], r0 = it[2], r1 = it[3], key_end = it[4], key_begin = it[5];
  const int q0 = p.qsl[seq], nq = p.qsl[seq + 1] - q0, before = p.seq_lens[seq] - nq;   // keys before the chunk's first token
  const int32_t* bt_row = p.bt + int64_t(seq) * p.bt_stride;
  const int G = p.G, wr0 = r0 + 32 * w;             // first row of the wave
  const bool wave_on = wr0 < r1;
  const int rfirst = wave_on ? wr0 : r0;
  const int row = rfirst + n < r1 ? rfirst + n : rfirst, tok = row / G;   // lanes past the tile repeat a row
  const int row_limit = before + tok + 1;           // keys that the lane's row sees
  const int wave_limit = wave_on ? before + (min(r1, wr0 + 32) - 1) / G + 1 : 0;
  const int wave_full = before + rfirst / G + 1;    // keys that all rows of the wave see

  // Q as the B operand of S^T = K Q^T.
  u32x4 qop[NQ];
  {
    const uint16_t* qr = p.q + (int64_t(q0 + tok) * p.Hq + head * G + (row - tok * G)) * D + 8 * h;
#pragma unroll
    for (int c = 0; c < NQ; ++c) qop[c] = load16(qr + 16 * c);
  }

  // A row's maximum starts at the lowest finite float rather than -inf: -m then
  // enters the exponent with no guard. Scores of masked keys are -inf, so a row
  // whose keys are all masked in a tile keeps this floor and adds zeros. The
  // sums add the probabilities before they are rounded: the log-sum-exp is good
  // to fp32, and the outputs' roundings average out.
  float m = -FLT_MAX, lpart = 0.f;   // lpart: the lane's keys
  f32x16 o[NC];
#pragma unroll
  for (int a = 0; a < NC; ++a)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[a][i] = 0.f;

  Loader<D, P, KG> loader(p, head, lds, w, lane, key_end, group);

  // Lane offsets of the operand reads in a stage. K: row n, columns 16c + 8h on;
  // V (transposing reads): rows 4h + i / 4 of a 16-lane group's lane i, column
  // 16 (group % 2) on. Rows start on multiples of their size, so columns and
  // swizzle meet in an exclusive or.
  const int vi = lane & 15, vg = (lane >> 4) & 1, v_row = 4 * h + (vi >> 2);
  const uint32_t k_off = uint32_t(n * L::ROW + 16 * swizzle_k<D>(h, n));
  const uint32_t v_off = uint32_t(L::V_OFF + v_row * L::ROW + 16 * swizzle_v<D>(2 * vg + ((vi & 3) >> 1), v_row) + 8 * (vi & 1));
  const uint32_t region = uint32_t(reinterpret_cast<uintptr_t>((lds_byte_ptr)lds)) + uint32_t(group * L::REGION);
  auto k_read = [&](uint32_t at, int c) {
    typedef const __attribute__((address_space(3))) u32x4* ptr;
    return *reinterpret_cast<ptr>(at ^ uint32_t(32 * c));
  };
  auto v_read = [&](uint32_t at, int i) {   // i: 16 keys, then 32-column block, fastest first
    typedef __attribute__((address_space(3))) v4i16* ptr;
    const uint32_t a = (at ^ uint32_t(64 * (i >> 1))) + uint32_t(16 * (i & 1) * L::ROW);
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(a)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(a + 8 * L::ROW)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };

  // One key tile: S^T = K Q^T, masking (only when the tile crosses a row's
  // limit), the tile's maximum of each row, lazy rescale, then probabilities
  // and O += P V. scored() runs behind the scores' products, for work that
  // hides there. Operands are read some products ahead, held in place by the
  // scheduling barriers. A wave's products go before the other waves' vector
  // work, which then fills the gaps of the matrix pipe (28/4 heads of 128, us: a
  // prompt of 2048 on 4096 keys 190.8 without and 186.2, of 2048 56.7 and 54.7,
  // eight of 2048 286.3 and 284.2; the softmax first instead 194, 56.6 and 288).
  // Heads of 64, with half the products, keep the turn up to the maxima (32/8:
  // 2048 on 4096 keys 128.1 and 125.5, 7 of 170 on 6000 110.7 and 107.0, eight
  // of 2048 192.6 and 190.8; with heads of 128 16 of 300 on 300 55.0 and 58.3).
  auto compute_tile = [&](bool masked, int st, int kc0, auto&& scored) {
    const uint32_t stage = uint32_t(__builtin_amdgcn_readfirstlane(region + uint32_t(st * L::STAGE)));
    const uint32_t k_at = stage + k_off, v_at = stage + v_off;
    constexpr int KD = 4, VD = 2;
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    {
      u32x4 kb[KD];
#pragma unroll
      for (int c = 0; c < KD; ++c) kb[c] = k_read(k_at, c);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int c = 0; c < NQ; ++c) {
        s = mfma_32x32x16(kb[c % KD], qop[c], s);
        if (c + KD < NQ) kb[c % KD] = k_read(k_at, c + KD);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (D == 128) __builtin_amdgcn_s_setprio(0);
    scored();
    u32x4 vb[VD];
#pragma unroll
    for (int i = 0; i < VD; ++i) vb[i] = v_read(v_at, i);
    __builtin_amdgcn_sched_barrier(0);

    // s[4j + r] is the score of key kc0 + 8j + 4h + r for row n.
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = kc0 + 8 * (i >> 2) + 4 * h + (i & 3) < row_limit ? s[i] : -INFINITY;
    }
    float mx = s[0];   // one chain, which the compiler pairs into three-input maxima
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = swap32_combine_max(mx) * p.scale_log2;

    if constexpr (D == 64) __builtin_amdgcn_s_setprio(0);
    // Lazy rescale: a row's maximum moves only when the tile's exceeds it by
    // more than the threshold.
    const bool need = mx > m + kRescaleThreshold;
    if (wave_any(need)) {
      const float m_new = need ? mx : m;
      const float alpha = fast_exp2(m - m_new);   // 1 if unchanged, 0 from the floor
      m = m_new;
      lpart *= alpha;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float ar = shfl_f(alpha, 8 * (i >> 2) + 4 * h + (i & 3));
#pragma unroll
        for (int a = 0; a < NC; ++a) o[a][i] *= ar;
      }
    }

    // Probabilities 2^(s * scale_log2 - m) as the bf16 A operands of P V (each
    // rounded once: the products take bf16).
    u32x4 pop[2];
    const float neg_m = -m;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p0 = fast_exp2(fmaf(s[2 * e], p.scale_log2, neg_m));
      const float p1 = fast_exp2(fmaf(s[2 * e + 1], p.scale_log2, neg_m));
      pop[e >> 2][e & 3] = pack_bf16x2(p0, p1);
      lpart += p0 + p1;
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < 2 * NC; ++i) {
      o[i >> 1] = mfma_32x32x16(pop[i & 1], vb[i % VD], o[i >> 1]);
      if (i + VD < 2 * NC) vb[i % VD] = v_read(v_at, i + VD);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // Past the barrier of step kt (every wave has written its part of the group's
  // tile and is done with the one before) the group's next tile is converted to
  // where the last one was, behind this one's scores, and the loads of the
  // third one on start into its raw slot; those of the second are in flight.
  // Pages and scales are staged in windows of block-table entries.
  int* const pt = reinterpret_cast<int*>(lds + L::PT_OFF);
  uint16_t* const sc = reinterpret_cast<uint16_t*>(lds + L::SC_OFF);
  constexpr int NL = Loader<D, P, KG>::NL, NT = 64 * kWaves * KG;
  const int last = key_end > 0 ? (key_end - 1) / P : 0;
  for (int wk0 = key_begin; wk0 < key_end; wk0 += L::WIN * P) {
    const int wk1 = min(key_end, wk0 + L::WIN * P), pt_base = wk0 / P, tiles = (wk1 - wk0 + kKeys - 1) / kKeys;
    const int pages = min(L::WIN, last + 1 - pt_base);
    const int ntiles = (tiles - group + KG - 1) / KG, steps = (tiles + KG - 1) / KG;   // the group's; the longest group's
    auto key_of = [&](int kt) { return wk0 + (kt * KG + group) * kKeys; };
    lds_barrier();
    for (int i = tid; i < pages; i += NT) pt[i] = bt_row[pt_base + i];
    wait_vmem_all();   // Q too, the first time: in the loops vmcnt counts only the tile loads
    lds_barrier();
    if (ntiles > 0) loader.fetch(key_of(0), 0, loader.first_page(key_of(0), pt_base));
    if (ntiles > 1) loader.fetch(key_of(1), 1, loader.first_page(key_of(1), pt_base));
    for (int i = tid; i < pages * L::BPP; i += NT)
      sc[i] = *reinterpret_cast<const uint16_t*>(p.kv_scales + int64_t(pt[i / L::BPP]) * p.scale_sp +
                                                 (i % L::BPP * p.Hkv + head) * 2);
    wait_vmem_all();
    lds_barrier();
    if (ntiles > 0) {
      loader.read_raw(key_of(0), 0, pt_base);
      loader.convert(0);
    }
    if (ntiles > 2) loader.fetch(key_of(2), 0, loader.first_page(key_of(2), pt_base));
    // Tiles that no row of the wave masks and that have three more behind them.
    const int steady = wave_on ? min(max(0, wave_full - wk0) / kKeys - group + KG - 1, tiles) / KG : 0;
    int kt = 0;
    for (; kt < min(steady, ntiles - 3); ++kt) {
      lds_barrier();
      wait_vmem<NL>();
      __atomic_signal_fence(__ATOMIC_SEQ_CST);   // the reads of the raw tile stay behind the wait
      const int page = loader.first_page(key_of(kt + 3), pt_base);
      loader.read_raw(key_of(kt + 1), (kt + 1) & 1, pt_base);
      compute_tile(false, kt & 1, key_of(kt), [&] {
        loader.convert((kt + 1) & 1);
        loader.fetch(key_of(kt + 3), (kt + 1) & 1, page);
      });
    }
    for (; kt < steps; ++kt) {
      const int kc = key_of(kt);
      lds_barrier();
      if (kt + 1 < ntiles) {
        if (kt + 2 < ntiles) wait_vmem<NL>();
        else wait_vmem<0>();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        loader.read_raw(key_of(kt + 1), (kt + 1) & 1, pt_base);
        loader.convert((kt + 1) & 1);
        if (kt + 3 < ntiles) loader.fetch(key_of(kt + 3), (kt + 1) & 1, loader.first_page(key_of(kt + 3), pt_base));
      }
      if (kt < ntiles && wave_on && kc < wave_limit) compute_tile(kc + kKeys > wave_full, kt & 1, kc, [] {});
    }
  }

  // The groups' states meet in the first: row maxima and sums, accumulators
  // scaled to the common maximum, in group order.
  if constexpr (KG > 1) {
    lds_barrier();
    auto state = [&](int g) { return lds + (g - 1) * L::STATE + w * (L::STATE / kWaves) + 16 * lane; };
    if (group > 0) {
      uint8_t* at = state(group);
#pragma unroll
      for (int a = 0; a < NC; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(at + (4 * a + i) * 1024) = f32x4{o[a][4 * i], o[a][4 * i + 1], o[a][4 * i + 2], o[a][4 * i + 3]};
      *reinterpret_cast<f32x4*>(at + 4 * NC * 1024) = f32x4{m, lpart, 0.f, 0.f};
    }
    lds_barrier();
    if (group > 0) return;
#pragma unroll 1
    for (int g = 1; g < KG; ++g) {
      const uint8_t* at = state(g);
      const f32x4 ml = *reinterpret_cast<const f32x4*>(at + 4 * NC * 1024);
      const float M = fmaxf(m, ml[0]), f0 = fast_exp2(m - M), f1 = fast_exp2(ml[0] - M);
      m = M;
      lpart = lpart * f0 + ml[1] * f1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a0[4], a1[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          a0[r] = shfl_f(f0, 8 * i + 4 * h + r);
          a1[r] = shfl_f(f1, 8 * i + 4 * h + r);
        }
#pragma unroll
        for (int a = 0; a < NC; ++a) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(at + (4 * a + i) * 1024);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[a][4 * i + r] = o[a][4 * i + r] * a0[r] + v[r] * a1[r];
        }
      }
    }
  }
  if (!wave_on) return;

  // Register 4i + r of block a is row 8i + 4h + r, column 32a + n.
  const float ltot = lpart + shfl_xor_f(lpart, 32);
  if (it[6] > 1) {   // a piece of the tile's keys: its state, for the merge
    const int64_t slot0 = (int64_t(it[7]) * p.Hkv + head) * kTileRows + 32 * w;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ri = 8 * (i >> 2) + 4 * h + (i & 3);
      if (wr0 + ri >= r1) continue;
      float* dst = p.pre_o + (slot0 + ri) * D + n;
#pragma unroll
      for (int a = 0; a < NC; ++a) dst[32 * a] = o[a][i];
    }
    if (h == 0 && wr0 + n < r1) {
      p.pre_stats[(slot0 + n) * 2] = m;
      p.pre_stats[(slot0 + n) * 2 + 1] = ltot;
    }
    return;
  }
  const float inv = 1.f / ltot;
  const int tok0 = r0 / G;
  const int64_t out0 = int64_t(q0 + tok0) * p.Hq + head * G;
  const int out_row = (tok - tok0) * p.Hq + (row - tok * G);   // of the lane's row, from out0
  if (p.lse && h == 0 && wr0 + n < r1) p.lse[out0 + out_row] = (m + log2f(ltot)) * kLn2;
  // Neighbouring lanes trade one of two rows' values, so that each stores two
  // columns of one row.
  const int odd = n & 1;
  const uint32_t sel = odd ? 0x03020706u : 0x05040100u;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const int ri = 8 * (i >> 2) + 4 * h + (i & 3);
    const float inv0 = shfl_f(inv, ri), inv1 = shfl_f(inv, ri + 1);
    const int dst_row = __shfl(out_row, ri + odd, 64);
    if (wr0 + ri + odd >= r1 && wr0 + ri >= r1) continue;
    uint16_t* dst = p.out + (out0 + dst_row) * D + (n & ~1);
#pragma unroll
    for (int a = 0; a < NC; ++a) {
      const uint32_t mine = pack_bf16x2(o[a][i] * inv0, o[a][i + 1] * inv1);
      const uint32_t theirs = __builtin_amdgcn_update_dpp(0, mine, 0xB1, 0xF, 0xF, false);   // lane ^ 1
      if (wr0 + ri + odd < r1) *reinterpret_cast<uint32_t*>(dst + 32 * a) = __builtin_amdgcn_perm(theirs, mine, sel);
    }
  }
}

// Joins the pieces of a prefill tile whose keys were cut: work-group (cut tile,
// KV head, slice of 8 or 16 rows), a thread per four columns of a row, the
// pieces in order, four loads in flight. A piece in which a row sees no key
// holds a sum of 0 and the lowest maximum, which weighs 0: every row sees key 0.
template <int DV>
__global__ __launch_bounds__(256) void merge_tiles_kernel(AttnParams p) {
  constexpr int CT = DV / 4, RPW = 256 / CT, KB = 4;
  const int32_t* it = p.items + 8 * p.cut_tiles[blockIdx.x];
  const int pieces = it[6], h = blockIdx.y;
  const int c = threadIdx.x % CT, i = blockIdx.z * RPW + threadIdx.x / CT, r = it[2] + i;
  if (r >= it[3]) return;
  const int64_t step = int64_t(p.Hkv) * 128, row0 = (int64_t(it[7]) * p.Hkv + h) * 128 + i;
  float M = -INFINITY, den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < pieces; j0 += KB) {
    float mj[KB], lj[KB];
    f32x4 vj[KB];
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int64_t at = row0 + min(j0 + k, pieces - 1) * step;
      mj[k] = j0 + k < pieces ? p.pre_stats[at * 2] : -INFINITY;
      lj[k] = p.pre_stats[at * 2 + 1];
      vj[k] = *reinterpret_cast<const f32x4*>(p.pre_o + at * DV + 4 * c);
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
  const float inv = 1.f / den;
  const int tok = r / p.G;
  const int64_t row = int64_t(p.qsl[it[0]] + tok) * p.Hq + h * p.G + (r - tok * p.G);
  *reinterpret_cast<u32x2*>(p.out + row * DV + 4 * c) =
      u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
  if (c == 0 && p.lse) p.lse[row] = (M + log2f(den)) * kLn2;
}

template <int D, int P, int KG, int WPE>
hipError_t launch_t(const AttnParams& p, dim3 grid, hipStream_t stream) {
  auto kern = prefill_kv8_kernel<D, P, KG, WPE>;
  constexpr size_t lds = Layout<D, P, KG>::LDS_BYTES;
  const hipError_t attr = set_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, grid, dim3(64 * kWaves * KG), lds, stream, p);
  return hipGetLastError();
}

template <int D, int P>
hipError_t launch_p(const AttnParams& p, hipStream_t stream) {
  AttnParams q = p;
  dim3 grid(p.n_items, p.grid_y);
  if (8 % p.grid_y == 0) {
    q.xcd_remap = 1;
    grid = dim3((p.n_items * p.grid_y + 7) / 8 * 8, 1);
  }
  const hipError_t e = p.key_groups == 2 ? launch_t<D, P, 2, 2>(q, grid, stream) : launch_t<D, P, 1, D == 128 ? 3 : 4>(q, grid, stream);
  if (e != hipSuccess || p.n_cut_tiles == 0) return e;
  hipLaunchKernelGGL(merge_tiles_kernel<D>, dim3(p.n_cut_tiles, p.Hkv, kTileRows / (1024 / D)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefill_kv8(const AttnParams& p, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return p.P == 16 ? launch_p<128, 16>(p, stream) : p.P == 64 ? launch_p<128, 64>(p, stream) : hipErrorInvalidValue;
  if (head_dim == 64) return p.P == 16 ? launch_p<64, 16>(p, stream) : p.P == 64 ? launch_p<64, 64>(p, stream) : hipErrorInvalidValue;
  return hipErrorInvalidValue;
}

}  // namespace flexattn
