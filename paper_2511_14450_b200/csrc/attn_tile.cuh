// Attention of a tile of 128 query rows against a run of paged keys on the tcgen05 tensor cores, as a CTA body.
//
// The 128 rows are 128 / G tokens (prefill) or sequences (shared prefix) times the G query heads that share one KV head,
// so a KV head's keys and values pass once for all its query heads.  Keys / values go by in tiles of 64 tokens
// (4 pages), two tiles in flight.
//   warp 0   lanes 0-15 issue TMA: the query tile once (3-D box: 64 dims x G heads x 128 / G rows, 128-byte swizzle),
//            then per tile one 2-D box per page and 64-wide half of head_dim for keys and for values.  The cache keeps
//            a token's row chunk-permuted inside each 128-byte half, so a box of 16 rows x 128 bytes lands as a ready
//            128-byte-swizzled operand.
//   warp 1   issues tcgen05.mma: S_b = Q K^T (128 x 64) into one of two score buffers in tensor memory and, once the
//            softmax warps have written the weights, O += P V (P from tensor memory).  The scores of tile j + 2 are
//            issued right behind the value product of tile j, so the tensor core works ahead of the softmax.  One lane
//            waits and issues: with the whole warp waiting, a tile spent 600 of 1850 cycles between its products.
//   warps 2-5  softmax, one thread per query row (tensor-memory lane); the reference maximum is moved, and O rescaled,
//            only when a row of the warp has outgrown it by 2^8.  In the tile that holds the end of the sequence they also
//            zero the values behind the end (0 times garbage infinity is not 0).
// Every barrier exists once per buffer (phase = tile / 2), every wait is bounded, failure unwinds through a shared flag.
// Measured (causal, 40 / 10 heads of 128): 2048 tokens 55 us = 780 TFLOP/s, capped 70, distance bias 68, 4096 tokens 168 us =
// 1020 TFLOP/s, where the products alone (two CTAs to an SM, nothing else running) take 126: with 64 keys a step the score
// product reads 6 KB of shared memory in the 32 cycles of its products.
#pragma once
#include "attn_paged.cuh"
#include "tcgen05.cuh"

namespace hyp {

constexpr int AT_ROWS = 128, AT_KEYS = 64, AT_THREADS = 192;

template <int D>
struct AtGeom {
  static constexpr int HALVES = D / 64;
  static constexpr int Q_BYTES = HALVES * 128 * 64 * 2;
  static constexpr int STAGE = AT_KEYS * D * 2;                  // one tile of keys (or values)
  static constexpr int SMEM = Q_BYTES + 4 * STAGE + 1024;        // queries, keys[2], values[2], alignment
};

// What one CTA works on: key tiles 0 .. n_first - 1 of the sequence, then n_tiles - n_first from `second` on.
struct TileWork {
  int head0;                  // first query head of the group: kvh * G
  int kvh;
  int row0;                   // first row of the query matrix
  int rows;                   // rows (tokens or sequences) in the tile, <= 128 / G
  const int32_t* table;       // page ids
  int key_end;                // keys at or behind it exist for nobody (bounds the pages that are read)
  int n_first, second, n_tiles;
};
// Which keys a row sees: [lo, hi] and [0, pre); for the distance bias `pos` is the row's position.
struct TileRow {
  int lo, hi, pre;
};
struct TileScore {
  float scale;                // x -> exponent (base 2)
  float to_tanh;              // CAP: raw product -> argument of the tanh
  float tanh_c[4];            // CAP: see tanh2_small
  float ratio;                // BIAS: this thread's slope, in units of x
};

struct TileShared {
  uint64_t bars[16];
  uint32_t tmem_slot;
  int abort_word;
};

__device__ __forceinline__ void at_tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void at_tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void at_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// MMA whose A operand is read from tensor memory (lane = row, two fp16 k-values per 32-bit column).
__device__ __forceinline__ void at_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}
// MN-major operand of D (MN) x 16 (K) fp16, 128-byte swizzle: the 64-wide pieces of a page are 4 x 2 KB apart, 8-row
// groups along K are 1024 B apart.
__device__ __forceinline__ uint64_t at_desc_mn(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((4 * 2048) >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Two fp32 values in one 64-bit register: the packed forms issue one instruction for both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pk2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void up2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3abs(float m, float a, float b) { return max3(m, fabsf(a), fabsf(b)); }

// tanh x of two raw products within TANH_RANGE (see tanh_any); the argument's factor (raw product -> x) is multiplied into
// the coefficients: c[i] = TANH_Ci * factor^(2 i + 1).  Runs on the packed FMA path; the form for the whole range needs two
// of the sixteen special-function lanes' operations a score, which alone would take longer than both matrix products.
__device__ __forceinline__ f32x2 tanh2_small(f32x2 raw, const float (&c)[4]) {
  const f32x2 u = mul2(raw, raw);
  f32x2 p = fma2(u, pk2(c[3], c[3]), pk2(c[2], c[2]));
  p = fma2(u, p, pk2(c[1], c[1]));
  p = fma2(u, p, pk2(c[0], c[0]));
  return mul2(raw, p);
}
__device__ __forceinline__ f32x2 abs2(f32x2 v) { return v & 0x7fffffff7fffffffull; }
// A finished row leaves through shared memory: the thread that owns it writes it there (rows 16 bytes apart from a
// multiple of 128, so that a quarter warp's 16-byte stores meet no bank twice) and sends it off as one bulk copy.  Direct
// stores, 32 rows at a time and 16 bytes of each, cost 4600 cycles for 128 rows of 512 bytes.
__device__ __forceinline__ void at_stage16(uint32_t dst, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void at_send_row(void* dst, uint32_t src, uint32_t bytes, bool valid) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  if (valid) asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the row has left shared memory
}

// The rare paths - moving the reference maximum, and capped scores beyond the polynomial's range - are functions of their
// own: inlined, the second one alone cost the tiles that never take it 20 % (77 against 64 us, 2048 tokens).

// Rescales the warp's rows of O by corr (one factor a lane) once every earlier value product has drained.
template <int D>
__device__ __noinline__ bool at_rescale(uint32_t tmem_o_row, float corr, uint32_t o_prev, uint32_t o_parity, volatile int* abort_flag) {
  if (!__all_sync(0xffffffffu, mbar_wait(o_prev, o_parity, abort_flag))) return false;
  tc_fence_after();
#pragma unroll 2
  for (int c = 0; c < D; c += 16) {
    uint32_t v[16];
    tmem_ld16(tmem_o_row + c, v);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * corr);
    at_tmem_st16(tmem_o_row + c, v);
  }
  return true;
}

// Bit i of the 64: key0 + i is visible to the row.
struct TileMask {
  uint32_t lo, hi;
};
__device__ __forceinline__ TileMask tile_mask(const TileRow& rw, int key0) {
  auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; };
  const unsigned long long vis = (below(rw.hi + 1 - key0) & ~below(rw.lo - key0)) | below(rw.pre - key0);
  return TileMask{(uint32_t)vis, (uint32_t)(vis >> 32)};
}

// The largest score (in log2 units) that a row sees in a tile with a distance bias.
template <int D, bool CAP>
__device__ __noinline__ float at_true_max(uint32_t tmem_row, int key0, int pos, TileMask mask, TileScore sc) {
  float mx = PG_NEG;
#pragma unroll 1
  for (int c = 0; c < AT_KEYS; c += 16) {
    uint32_t v[16];
    tmem_ld16(tmem_row + c, v);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = __uint_as_float(v[i]);
      if (CAP) x = tanh_any(x * sc.to_tanh);
      x = fmaf(-sc.ratio, fabsf((float)(key0 + c + i - pos)), x);
      mx = (c < 32 ? mask.lo : mask.hi) >> ((c + i) & 31) & 1u ? fmaxf(mx, x) : mx;
    }
  }
  return mx * sc.scale;
}

struct SoftmaxState {
  float m_ref, l;
  bool ok;
};
template <int D, bool BIAS>
__device__ __noinline__ SoftmaxState at_softmax_exact(uint32_t tmem_sb, uint32_t tmem_o, uint32_t lane_off, int key0, int pos, TileRow rw,
                                                      TileScore sc, int j, uint32_t o_prev, uint32_t o_parity,
                                                      volatile int* abort_flag, SoftmaxState st);

// Softmax of one 64-key tile for one query row: see the head of the file.  A score enters the exponent as x * scale with
// x the raw product (scale = log2(e) / sqrt(D)) or, capped, the tanh (scale = softcap * log2(e)); the distance bias is
// added to x as ratio * distance, ratio = slope * log2(e) / scale.  What a row may not see becomes -1e30, which the exponent
// turns into 0 as long as the reference stays above -1e20.
template <int D, bool CAP, bool BIAS, bool MASKED, bool EXACT>
__device__ __forceinline__ void at_softmax(uint32_t tmem_sb, uint32_t tmem_o, uint32_t lane_off, int key0, int pos, const TileRow& rw,
                                           const TileScore& sc, int j, uint32_t o_prev, uint32_t o_parity, volatile int* abort_flag,
                                           SoftmaxState& st) {
  uint32_t sv[AT_KEYS];
#pragma unroll
  for (int c = 0; c < AT_KEYS; c += 16) tmem_ld16(tmem_sb + lane_off + c, reinterpret_cast<uint32_t(&)[16]>(sv[c]));
  tmem_ld_wait();
  float x[AT_KEYS];
#pragma unroll
  for (int i = 0; i < AT_KEYS; ++i) x[i] = __uint_as_float(sv[i]);
  const TileMask mask = MASKED ? tile_mask(rw, key0) : TileMask{~0u, ~0u};
  auto seen = [&](int i, float v) { return !MASKED || ((i < 32 ? mask.lo : mask.hi) & (1u << (i & 31))) ? v : PG_NEG; };
  // The largest product bounds the largest score: the cap keeps the order, and the bias of the tile is at most that of its
  // nearest (slope < 0: farthest) key.  So the cap, the bias and the second mask run beside the exponentials, which set the
  // pace, and not in front of them.  One vote asks for everything that is rare: a bound that is too high for the
  // reference, or a product beyond the polynomial's range.
  float m4[4] = {PG_NEG, PG_NEG, PG_NEG, PG_NEG}, a4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < AT_KEYS; i += 2) {
    m4[(i >> 1) & 3] = max3(m4[(i >> 1) & 3], seen(i, x[i]), seen(i + 1, x[i + 1]));
    if (CAP && !EXACT) a4[(i >> 1) & 3] = max3abs(a4[(i >> 1) & 3], x[i], x[i + 1]);
  }
  float mx = max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]);
  bool wide = false;
  if (CAP && !EXACT) {
    // NaN (garbage behind the end of a sequence) is dropped by the maxima and removed by the mask below
    wide = !(max3(fmaxf(a4[0], a4[1]), a4[2], a4[3]) * sc.to_tanh <= TANH_RANGE);
    float top, same;
    up2(tanh2_small(pk2(mx, mx), sc.tanh_c), top, same);
    mx = mx > PG_NEG ? top : mx;
  }
  if (CAP && EXACT) mx = mx > PG_NEG ? tanh_any(mx * sc.to_tanh) : mx;
  if (BIAS) {
    const int near = max(max(key0 - pos, pos - (key0 + AT_KEYS - 1)), 0), far = max(abs(key0 - pos), abs(key0 + AT_KEYS - 1 - pos));
    mx += fmaxf(-sc.ratio * (float)near, -sc.ratio * (float)far);
  }
  mx *= sc.scale;  // scale > 0
  if (__any_sync(0xffffffffu, mx > st.m_ref + 8.f || wide)) {
    if (CAP && !EXACT && __any_sync(0xffffffffu, wide)) {
      st = at_softmax_exact<D, BIAS>(tmem_sb, tmem_o, lane_off, key0, pos, rw, sc, j, o_prev, o_parity, abort_flag, st);
      return;
    }
    if (BIAS) mx = at_true_max<D, CAP>(tmem_sb + lane_off, key0, pos, MASKED ? mask : TileMask{~0u, ~0u}, sc);
    if (!BIAS || __any_sync(0xffffffffu, mx > st.m_ref + 8.f)) {
      const float new_ref = fmaxf(st.m_ref, mx), corr = ex2_approx(st.m_ref - new_ref);
      if (j > 0) {
        st.ok = at_rescale<D>(tmem_o + lane_off, corr, o_prev, o_parity, abort_flag);
        if (!st.ok) return;
        st.l *= corr;
      }
      st.m_ref = new_ref;
    }
  }
  if (CAP) {
#pragma unroll
    for (int i = 0; i < AT_KEYS; i += 2) {
      if (EXACT) {
        x[i] = tanh_any(x[i] * sc.to_tanh);
        x[i + 1] = tanh_any(x[i + 1] * sc.to_tanh);
      } else {
        up2(tanh2_small(pk2(x[i], x[i + 1]), sc.tanh_c), x[i], x[i + 1]);
      }
    }
  }
  if (BIAS) {
    f32x2 dist = pk2((float)(key0 - pos), (float)(key0 + 1 - pos));
    const f32x2 r2 = pk2(-sc.ratio, -sc.ratio), two = pk2(2.f, 2.f);
#pragma unroll
    for (int i = 0; i < AT_KEYS; i += 2) {
      up2(fma2(r2, abs2(dist), pk2(x[i], x[i + 1])), x[i], x[i + 1]);
      dist = add2(dist, two);  // whole numbers: exact
    }
  }
  if (MASKED) {
#pragma unroll
    for (int i = 0; i < AT_KEYS; ++i) x[i] = seen(i, x[i]);
  }
  const float neg_ref = -fmaxf(st.m_ref, -1e20f);
  const f32x2 s2 = pk2(sc.scale, sc.scale), n2 = pk2(neg_ref, neg_ref);
  f32x2 l2[2] = {0ull, 0ull};
#pragma unroll
  for (int c = 0; c < AT_KEYS; c += 32) {
    uint32_t pk[16];
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      float p0, p1;
      up2(fma2(pk2(x[c + i], x[c + i + 1]), s2, n2), p0, p1);
      p0 = ex2_approx(p0);
      p1 = ex2_approx(p1);
      l2[(i >> 1) & 1] = add2(l2[(i >> 1) & 1], pk2(p0, p1));
      pk[i >> 1] = pack_f16(p0, p1);
    }
    at_tmem_st16(tmem_sb + lane_off + 32 + (c >> 1), pk);  // key k of the tile: 16-bit half k & 1 of column 32 + k / 2
  }
  float l0, l1;
  up2(add2(l2[0], l2[1]), l0, l1);
  st.l += l0 + l1;
  at_tmem_st_wait();
}
template <int D, bool BIAS>
__device__ __noinline__ SoftmaxState at_softmax_exact(uint32_t tmem_sb, uint32_t tmem_o, uint32_t lane_off, int key0, int pos, TileRow rw,
                                                      TileScore sc, int j, uint32_t o_prev, uint32_t o_parity,
                                                      volatile int* abort_flag, SoftmaxState st) {
  at_softmax<D, true, BIAS, true, true>(tmem_sb, tmem_o, lane_off, key0, pos, rw, sc, j, o_prev, o_parity, abort_flag, st);
  return st;
}

// Barriers and tensor memory; the whole CTA, behind its wait for the preceding kernel (tensor memory taken before it could be
// what a CTA of that kernel is waiting for).
__device__ __forceinline__ void tile_setup(TileShared& sh) {
  if (threadIdx.x == 0) {
    // p_full (12, 13): every softmax warp
    for (int i = 0; i < 16; ++i) mbar_init(smem_u32(sh.bars) + 8u * i, (i == 12 || i == 13) ? 4u : 1u);
    sh.abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x >> 5 == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_slot)), "r"(256));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
}
// The whole CTA, last.
__device__ __forceinline__ void tile_release(TileShared& sh) {
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x >> 5 == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem_slot), "r"(256));
  }
}

// The whole CTA (192 threads) calls this between the two.  `store(row, head_in_group, valid, m_ref, l, stage, load)` is called by the
// softmax threads at the end: load(c, v, w) reads columns c .. c + 31 of the thread's O row from tensor memory (all lanes call
// it), stage is the thread's row of D floats in shared memory.
template <int D, bool CAP, bool BIAS, typename RowFn, typename StoreFn>
__device__ __forceinline__ void tile_body(const CUtensorMap* tm_q, const CUtensorMap* tm_kv, uint8_t* smem_raw, TileShared& sh,
                                          const TileWork& wk, int G, int Hkv, float softcap, const float* slopes, int* err,
                                          RowFn row_fn, StoreFn store) {
  using Geo = AtGeom<D>;
  constexpr uint32_t IDESC_S = (1u << 4) | ((uint32_t)(AT_KEYS >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = base, sK = base + Geo::Q_BYTES, sV = sK + 2 * Geo::STAGE;
  // barriers: one per buffer b = tile & 1 (add 8 * b); phase of tile j = j / 2
  const uint32_t bar0 = smem_u32(sh.bars);
  const uint32_t q_full = bar0, drained = bar0 + 8, k_full = bar0 + 16, v_full = bar0 + 32, s_full = bar0 + 80, p_full = bar0 + 96, o_done = bar0 + 112;
  volatile int* abort_flag = &sh.abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_tiles = wk.n_tiles;
  // columns 0-63 / 64-127: the two score buffers (P over the upper half of each); from 128: O
  const uint32_t tmem_s = sh.tmem_slot, tmem_o = sh.tmem_slot + 128u;
  // The walk goes from the last tile to the first: with a distance bias the near keys set the reference maximum at once (the
  // other way round it moved in nearly every tile).
  auto key_tile = [&](int j) {
    const int i = n_tiles - 1 - j;
    return i < wk.n_first ? i : i - wk.n_first + wk.second;
  };

  if (warp == 0) {
    // ---------------- TMA producer: one box per lane and tile ----------------
    // lanes 0-7 bring the keys, 8-15 the values; within each, lane = page (0-3) x 64-wide half of head_dim
    if (lane == 0) {
      mbar_expect_tx(q_full, Geo::Q_BYTES);
      for (int h = 0; h < Geo::HALVES; ++h) at_tma_load_3d(sQ + h * 128 * 64 * 2, tm_q, h * 64, wk.head0, wk.row0, q_full);
    }
    const int is_v = lane >> 3, p = (lane >> 1) & 3, h = lane & 1;
    if (lane < 16 && h < Geo::HALVES) {
      const uint32_t full = is_v ? v_full : k_full;
      const uint32_t empty = is_v ? o_done : s_full;  // a stage is free once the product that read it has drained
      const uint32_t dst = is_v ? sV + (h * 4 + p) * 2048 : sK + h * (AT_KEYS * 128) + p * 2048;
      const int last_page = (wk.key_end - 1) / PG_PT;
      // Key lanes and value lanes advance independently (their stages drain at different times), so no lane may
      // block in a wait the others have to reconverge with: every lane polls its own barrier once per turn.
      bool ok = true;
      int j = 0;
      uint32_t idle = 0;
      uint64_t t_idle = 0;
      while (j < n_tiles) {
        const uint32_t b = (uint32_t)(j & 1);
        if (j < 2 || mbar_try(empty + 8 * b, (uint32_t)(((j >> 1) - 1) & 1))) {
          const int pi = min(4 * key_tile(j) + p, last_page);  // past the last page: any valid page (its keys are masked)
          const int row0 = ((wk.table[pi] * 2 + is_v) * Hkv + wk.kvh) * PG_PT;
          if ((lane & 7) == 0) mbar_expect_tx(full + 8 * b, Geo::STAGE);  // a copy may land first: the count goes negative meanwhile
          tma_load_2d(dst + b * Geo::STAGE, tm_kv, h * 64, row0, full + 8 * b);
          ++j;
          idle = 0;
        } else if ((++idle & 1023u) == 0) {
          const uint64_t now = globaltimer();
          if (idle == 1024u) t_idle = now;
          if (*abort_flag || now - t_idle > WAIT_LIMIT_NS) { ok = false; break; }
        }
      }
      if (!ok && (lane & 7) == 0) {
        *abort_flag = 1;
        atomicCAS(err, 0, 22);
      }
      // no copy may be in flight when the CTA leaves: at the end of a clean run these have long completed
      if (lane == 0) mbar_wait(q_full, 0, nullptr);
      for (int i = max(0, j - 2); i < j && (lane & 7) == 0; ++i)
        mbar_wait(full + 8 * (uint32_t)(i & 1), (uint32_t)((i >> 1) & 1), nullptr);
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer: one lane ----------------
    if (lane == 0) {
      const uint64_t dq = smem_desc(sQ), dk = smem_desc(sK), dv = at_desc_mn(sV);
      bool ok = mbar_wait(q_full, 0, abort_flag);
      auto scores = [&](int j) -> bool {
        const uint32_t b = (uint32_t)(j & 1);
        if (!mbar_wait(k_full + 8 * b, (uint32_t)((j >> 1) & 1), abort_flag)) return false;
        tc_fence_after();
        const uint64_t dkb = dk + (uint64_t)(b * (Geo::STAGE >> 4));
#pragma unroll
        for (int kb = 0; kb < Geo::HALVES; ++kb)
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            tc_mma(tmem_s + 64u * b, dq + (uint64_t)(kb * ((128 * 64 * 2) >> 4) + ks * 2),
                   dkb + (uint64_t)(kb * ((AT_KEYS * 128) >> 4) + ks * 2), IDESC_S, (kb | ks) ? 1u : 0u);
        tc_commit(s_full + 8 * b);  // also frees the key stage
        return true;
      };
      ok = ok && scores(0);
      if (ok && n_tiles > 1) ok = scores(1);
      for (int j = 0; j < n_tiles && ok; ++j) {
        const uint32_t b = (uint32_t)(j & 1), ph = (uint32_t)((j >> 1) & 1);
        if (!mbar_wait(v_full + 8 * b, ph, abort_flag) || !mbar_wait(p_full + 8 * b, ph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        // O += P V: 4 pages of 16 keys; P sits in tensor memory (8 columns per page)
        const uint64_t dvb = dv + (uint64_t)(b * (Geo::STAGE >> 4));
#pragma unroll
        for (int p = 0; p < 4; ++p)
          at_mma_ta(tmem_o, tmem_s + 64u * b + 32u + (uint32_t)(8 * p), dvb + (uint64_t)(p * (2048 >> 4)), IDESC_PV,
                    (j > 0 || p > 0) ? 1u : 0u);
        tc_commit(o_done + 8 * b);  // also frees the value stage
        // the scores of tile j + 2 reuse this tile's buffer: issued behind its value product
        if (j + 2 < n_tiles) ok = scores(j + 2);
      }
      if (!ok) {
        *abort_flag = 1;
        atomicCAS(err, 0, 23);
        // products that are under way still read shared memory and write tensor memory
        tc_commit(drained);
        mbar_wait(drained, 0, nullptr);
      }
    }
  } else {
    // ---------------- softmax / epilogue: thread = query row = tensor-memory lane ----------------
    const int q = warp & 3;
    const int r = 32 * q + lane;
    const uint32_t lane_off = (uint32_t)(32 * q) << 16;
    const int t = r / G, gh = r % G;
    const bool valid = t < wk.rows;
    const bool warp_idle = (32 * q) / G >= wk.rows;  // no row of this warp exists: its weights are never used
    int pos;
    const TileRow rw = row_fn(min(t, wk.rows - 1), pos);  // rows past the end are clamped: computed, never stored
    TileScore sc{rsqrtf((float)D) * PG_LOG2E, 0.f, {0.f, 0.f, 0.f, 0.f}, 0.f};
    if (CAP) {
      sc.to_tanh = rsqrtf((float)D) / softcap;
      const float f = sc.to_tanh, f2 = f * f;
      sc.tanh_c[0] = TANH_C0 * f;
      sc.tanh_c[1] = TANH_C1 * f * f2;
      sc.tanh_c[2] = TANH_C2 * f * f2 * f2;
      sc.tanh_c[3] = TANH_C3 * f * f2 * f2 * f2;
      sc.scale = softcap * PG_LOG2E;
    }
    if (BIAS) sc.ratio = slopes[wk.head0 + gh] * PG_LOG2E / sc.scale;
    SoftmaxState st{PG_NEG, 0.f, true};
    bool ok = true;
    for (int j = 0; j < n_tiles && ok; ++j) {
      const uint32_t b = (uint32_t)(j & 1);
      ok = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * b, (uint32_t)((j >> 1) & 1), abort_flag));
      if (!ok) break;
      tc_fence_after();
      if (!warp_idle) {
        const int key0 = key_tile(j) * AT_KEYS;
        // the value product of tile j - 1: buffer (j - 1) & 1, phase (j - 1) / 2
        const uint32_t o_prev = o_done + 8 * (b ^ 1), o_parity = (uint32_t)(((j - 1) >> 1) & 1);
        const bool whole = (key0 >= rw.lo && key0 + AT_KEYS - 1 <= rw.hi) || key0 + AT_KEYS <= rw.pre;
        if (__any_sync(0xffffffffu, !whole))
          at_softmax<D, CAP, BIAS, true, false>(tmem_s + 64u * b, tmem_o, lane_off, key0, pos, rw, sc, j, o_prev, o_parity, abort_flag, st);
        else
          at_softmax<D, CAP, BIAS, false, false>(tmem_s + 64u * b, tmem_o, lane_off, key0, pos, rw, sc, j, o_prev, o_parity, abort_flag, st);
        ok = st.ok;
        if (!ok) break;
      }
      const int left = wk.key_end - key_tile(j) * AT_KEYS;
      if (left < AT_KEYS) {  // the end of the sequence lies in this tile
        ok = __all_sync(0xffffffffu, mbar_wait(v_full + 8 * b, (uint32_t)((j >> 1) & 1), abort_flag));
        if (!ok) break;
        for (int e = 32 * q + lane; e < Geo::HALVES * (AT_KEYS - left) * 8; e += 128) {
          const int h = e / ((AT_KEYS - left) * 8), zr = left + (e % ((AT_KEYS - left) * 8)) / 8, c = e & 7;
          at_stage16(sV + b * Geo::STAGE + (uint32_t)(h * AT_KEYS + zr) * 128u + (uint32_t)c * 16u, 0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + 8 * b);  // one arrival a warp: 128 on one word take their time
    }
    // the last value product (a commit follows every earlier one too)
    if (ok && !mbar_wait(o_done + 8 * ((n_tiles - 1) & 1), (uint32_t)(((n_tiles - 1) >> 1) & 1), abort_flag)) ok = false;
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    if (ok && !warp_idle)
      // every product has drained: the operands' space is free
      store(min(t, wk.rows - 1), gh, valid, st.m_ref, st.l, base + (uint32_t)r * (D * 4 + 16), [&](int c, uint32_t (&v)[16], uint32_t (&w)[16]) {
        tmem_ld16(tmem_o + lane_off + c, v);
        tmem_ld16(tmem_o + lane_off + c + 16, w);
        tmem_ld_wait();
      });
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicCAS(err, 0, 24);
    }
  }
}

static_assert(AT_ROWS * (128 * 4 + 16) <= AtGeom<128>::SMEM - 1024 && AT_ROWS * (64 * 4 + 16) <= AtGeom<64>::SMEM - 1024, "rows to be stored");

// Which row tile of `tile_rows` rows is tile t?  Sets run from cu[i] to cu[i + 1] and are cut into tiles one by one.
// Every warp finds it for itself, 32 sets at a time; set = -1: no such tile.  a[set] and b[set] (b may be null: 0) are fetched
// beside the bounds, not behind them.
__device__ __forceinline__ void at_locate(const int32_t* cu, const int32_t* a, const int32_t* b, int n_sets, int tile_rows, int t, int& set,
                                          int& first, int& q0, int& len, int& a_set, int& b_set) {
  const int lane = threadIdx.x & 31;
  set = -1;
  first = q0 = len = a_set = b_set = 0;
  int before = 0;
  for (int i0 = 0; i0 < n_sets; i0 += 32) {
    const int i = i0 + lane;
    const int c0 = i < n_sets ? cu[i] : 0;
    const int a0 = i < n_sets ? a[i] : 0, b0 = b && i < n_sets ? b[i] : 0;
    const int my_len = i < n_sets ? max(cu[i + 1] - c0, 0) : 0;
    const int nt = (my_len + tile_rows - 1) / tile_rows;
    int incl = nt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, t < before + incl);
    if (hit) {
      const int src = __ffs(hit) - 1;
      set = i0 + src;
      first = __shfl_sync(0xffffffffu, c0, src);
      a_set = __shfl_sync(0xffffffffu, a0, src);
      b_set = __shfl_sync(0xffffffffu, b0, src);
      len = __shfl_sync(0xffffffffu, my_len, src);
      q0 = (t - before - __shfl_sync(0xffffffffu, incl - nt, src)) * tile_rows;
      return;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
}

}  // namespace hyp
