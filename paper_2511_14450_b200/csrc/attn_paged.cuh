// Split decode attention over the paged cache, as a CTA body shared by the operators that need one query row per
// sequence: attention with modified scores, attention that keeps its scores, and the sequences' own part of
// shared-prefix attention.
//
// A CTA takes one (split, KV head, sequence): the visible pages of the sequence go round-robin over the splits and,
// inside the CTA, over the warps; every warp streams its pages through its own ring of bulk copies (16 keys and 16 values of
// one head are contiguous in the cache and already chunk-permuted for ldmatrix), forms the scores of the page's 16
// keys for the G query heads that share the KV head (rows of one mma.sync.m16n8k16 operand), keeps its own running
// maximum and denominator and its own O += P V.  No CTA-wide synchronisation inside the loop.  Bound by HBM: a page
// of one head is 8 KB (head_dim 128) for 32 MMAs.
// Measured: 4 x 32768 tokens, 40 / 10 heads of 128: 6.1 TB/s of cache, 0.95 of the copy bandwidth; 8 x 1024 tokens 11.5 us, one
// wave of start-up latencies (length and page ids, first pages) for 42 MB.
// The CTA's result is one partial row per query head: sum of weighted values (fp32), maximum (log2 units), denominator.
#pragma once
#include "attn_common.cuh"
#include "sm100_common.cuh"

namespace hyp {

constexpr int PG_PT = 16;           // tokens per page
constexpr float PG_NEG = -1e30f;    // "no key seen yet": below every score that finite fp16 operands can form
constexpr float PG_LOG2E = 1.4426950408889634f;

// PAGED_FLAT: the sequence's own pages behind those of its group's prefix
enum PagedMode : int { PAGED_PLAIN = 0, PAGED_SCORED = 1, PAGED_MOD = 2, PAGED_FLAT = 3 };

struct PagedArgs {
  const __half* q;            // row b at q + b * q_stride, head h at + h * D
  long long q_stride;
  const __half* pool;         // one block's page pool
  const int32_t* table;       // [n_seqs, table_stride] page ids
  int table_stride;
  const int32_t* ctx;         // [n_seqs] tokens before the new one; -1 = nothing to see
  int Hq, Hkv;
  float* acc;                 // partial rows: ((b * Hq + h) * n_slots + slot0 + split) * D
  float* ml;                  // the same rows' (maximum, denominator)
  int n_slots, slot0;
  int wave_splits;            // splits of a (sequence, KV head) that make one wave of the batch
  int* err;
  float* scores;              // PAGED_SCORED: [n_seqs * Hq][score_stride] scores in log2 units
  int score_stride;
  float softcap;              // PAGED_MOD: 0 = none
  int window;                 // PAGED_MOD: 0 = none
  const float* slopes;        // PAGED_MOD: [Hq] or null
  const int32_t* prefix;      // PAGED_MOD: [n_seqs] or null
  const int32_t* cu_group;    // PAGED_FLAT: groups of sequences, their prefixes' pages and lengths
  const int32_t* prefix_table;
  const int32_t* prefix_lens;
  int prefix_stride, n_groups;
  // one split, or a cluster: the result is the operator's (out non-null); PAGED_SCORED (one split) then finishes the running
  // sums as well
  __half* out;                // [n_seqs, Hq * D]
  float decay;
  const float* w_in;
  float* w_out;
  long long w_stride;
};

// Tokens of a sequence, the new one at position ctx included, as far as its table row can name them; any ctx (the row holds at
// most 2^30 tokens, and the clamp comes before the sum).
__device__ __forceinline__ int paged_total(int ctx, int table_stride) { return min(max(ctx, -1), table_stride * PG_PT - 1) + 1; }

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh x for |x| <= TANH_RANGE is x times a polynomial in x^2 (four coefficients, least absolute error of tanh x over the
// range, fitted by reweighted least squares): off by 1.3e-7 at most, by 2.4e-6 of the value near 0.  Beyond the range
// 1 - 2 / (1 + e^(2x)), which saturates cleanly but near 0 would leave an error of 2^-23, times the cap, in every
// small score.  (The hardware tanh, 2^-11, would put a capped score of 50 off by 0.02 and its weight off by 2 %.)
constexpr float TANH_RANGE = 0.5f;
constexpr float TANH_C0 = 0.9999976761797865f, TANH_C1 = -0.33320655167817165f, TANH_C2 = 0.13145145181299145f, TANH_C3 = -0.04337247117084689f;
__device__ __forceinline__ float tanh_any(float x) {
  const float u = x * x;
  const float small = x * fmaf(u, fmaf(u, fmaf(u, TANH_C3, TANH_C2), TANH_C1), TANH_C0);
  const float large = fmaf(-2.f, rcp_approx(1.f + ex2_approx(2.f * PG_LOG2E * x)), 1.f);
  return fabsf(x) <= TANH_RANGE ? small : large;
}

// Contiguous bulk copy of data that is not read again soon: first to leave the L2.
__device__ __forceinline__ void bulk_load_once(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy)
               : "memory");
}

template <int D, int WARPS>
constexpr int paged_smem_bytes(int slots) { return WARPS * slots * 2 * PG_PT * D * 2; }

// `smem`: 128-byte aligned shared memory, paged_smem_bytes<D, WARPS>(SLOTS) bytes; `bars`: WARPS * SLOTS mbarriers.
// WARPS warps of the CTA call this (warp = 0 .. WARPS - 1); `bar_sync` joins exactly those warps.
// CLUSTER: the n_splits (2 .. 8) CTAs of a (sequence, KV head) are a thread-block cluster and join their results through
// distributed shared memory; every one of them must call this.
template <int D, int G, int MODE, int WARPS, int SLOTS, bool CLUSTER, typename Sync>
__device__ __forceinline__ void paged_body(const PagedArgs& a, uint8_t* smem, uint64_t* bars, int split, int n_splits, int kvh,
                                           int b, int tid, Sync bar_sync) {
  constexpr int KS = D / 16, DN = D / 8, CPR = D / 8;
  constexpr int PAGE_BYTES = PG_PT * D * 2;
  constexpr int SLOT_BYTES = 2 * PAGE_BYTES;  // keys, then values
  constexpr int THREADS = WARPS * 32;
  static_assert(paged_smem_bytes<D, WARPS>(SLOTS) >= (2 * WARPS * 8 + WARPS * G * D + 16 + 16 + G * D + 128) * 4, "the combine buffers reuse the ring");
  const int warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, tq = lane & 3;

  const int32_t* bt = a.table + (long long)b * a.table_stride;
  const bool early = MODE == PAGED_PLAIN || MODE == PAGED_SCORED || (MODE == PAGED_MOD && a.window == 0 && a.prefix == nullptr);
  int32_t ids_cur = 0;
  if (early) {
    const int v = split + n_splits * (warp + WARPS * lane);
    if (v < a.table_stride) ids_cur = bt[v];
  }
  // Visible keys: [lo, total) behind the query, and [0, pre).  PAGED_FLAT: [0, pre) is the prefix, in pages of its own, and
  // its keys are numbered from -16 * (its pages) on.
  const int total = paged_total(a.ctx[b], a.table_stride);
  int lo = 0, pre = 0;
  const int32_t* pt = nullptr;
  if (MODE == PAGED_MOD) {
    if (a.window > 0) lo = max(total - a.window, 0);
    if (a.prefix) pre = min(max(a.prefix[b], 0), total);
  }
  if (MODE == PAGED_FLAT) {
    int g = 0;  // groups that end at or before b
    for (int i0 = 0; i0 < a.n_groups; i0 += 32) g += __popc(__ballot_sync(0xffffffffu, i0 + lane < a.n_groups && a.cu_group[i0 + lane + 1] <= b));
    if (g < a.n_groups) {
      pre = min(max(a.prefix_lens[g], 0), a.prefix_stride * PG_PT);
      pt = a.prefix_table + (long long)g * a.prefix_stride;
    }
  }
  const int n_pages = (total + PG_PT - 1) / PG_PT;
  const int n_pre = MODE == PAGED_MOD || MODE == PAGED_FLAT ? (pre + PG_PT - 1) / PG_PT : 0;
  const int p_lo = MODE == PAGED_MOD ? max(lo / PG_PT, n_pre) : 0;
  const int n_vis = n_pre + max(n_pages - p_lo, 0);
  // The splits were planned for the length that the table could hold; a shorter sequence uses no more of them than the same
  // rule gives for its own length (see paged_splits), and the CTAs left over say that they have seen nothing.
  const int fair = max(a.wave_splits, (n_vis + 15) / 16);  // a large batch still evens out over CTAs of 16 pages
  const int used = n_vis > 64 * a.wave_splits ? n_splits : max(min(min(n_splits, fair), (n_vis + WARPS - 1) / WARPS), 1);
  if (!CLUSTER && split >= used) {  // the whole CTA
    if (tid < G) *reinterpret_cast<float2*>(a.ml + (((size_t)b * a.Hq + kvh * G + tid) * a.n_slots + a.slot0 + split) * 2) = make_float2(PG_NEG, 0.f);
    return;
  }
  auto page_index = [&](int i) {  // this warp's i-th page
    const int v = split + used * (warp + WARPS * i);
    return MODE == PAGED_MOD ? (v < n_pre ? v : v - n_pre + p_lo) : MODE == PAGED_FLAT ? v - n_pre : v;
  };
  const int first = split + used * warp, stride_p = used * WARPS;
  const int my_n = split < used && first < n_vis ? (n_vis - first + stride_p - 1) / stride_p : 0;

  const size_t page_elems = kv_page_elems(a.Hkv, PG_PT, D);
  const size_t v_off = (size_t)a.Hkv * PG_PT * D;
  const uint32_t my_bars = smem_u32(bars) + 8u * (warp * SLOTS);
  const uint32_t my_ring = smem_u32(smem) + (uint32_t)(warp * SLOTS) * SLOT_BYTES;
  // page ids: lane l holds the id of this warp's page base + l, for the 32 pages being issued and the 32 after them.  Where
  // the walk does not depend on the length (no window, no prefix, all splits used) the first ids are fetched together with it.
  auto load_ids = [&](int base) {
    if (base + lane >= my_n) return 0;
    const int p = page_index(base + lane);
    return MODE == PAGED_FLAT && p < 0 ? pt[p + n_pre] : bt[p];
  };
  if (!early || used != n_splits) ids_cur = load_ids(0);
  int32_t ids_next = load_ids(32);
  auto issue = [&](int i, int slot) {  // all lanes call, i ascending
    if (i > 0 && (i & 31) == 0) {
      ids_cur = ids_next;
      ids_next = load_ids(i + 32);
    }
    const int page = __shfl_sync(0xffffffffu, ids_cur, i & 31);
    if (lane == 0) {
      const __half* src = a.pool + (size_t)page * page_elems + (size_t)kvh * PG_PT * D;
      const uint32_t dst = my_ring + slot * SLOT_BYTES, bar = my_bars + 8u * slot;
      mbar_expect_tx(bar, SLOT_BYTES);
      if (MODE == PAGED_SCORED) {  // the pages pass through; the scores, written now and read by the next kernel, should stay in the L2
        bulk_load_once(dst, src, PAGE_BYTES, bar);
        bulk_load_once(dst + PAGE_BYTES, src + v_off, PAGE_BYTES, bar);
      } else {
        bulk_load(dst, src, PAGE_BYTES, bar);
        bulk_load(dst + PAGE_BYTES, src + v_off, PAGE_BYTES, bar);
      }
    }
  };
  if (lane == 0) {
    for (int s = 0; s < SLOTS; ++s) mbar_init(my_bars + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  for (int s = 0; s < SLOTS && s < my_n; ++s) issue(s, s);

  // query heads kvh*G .. kvh*G+G-1 as operand rows 0..G-1 (rows G..15 are zero)
  uint32_t qf[KS][2];  // [k step][k half]; only the "row g" halves of the fragment are non-zero
  {
    const __half* qrow = a.q + (long long)b * a.q_stride + (size_t)(kvh * G + (g < G ? g : 0)) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks][0] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + 16 * ks + 2 * tq) : 0u;
      qf[ks][1] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + 16 * ks + 8 + 2 * tq) : 0u;
    }
  }
  const float sl2 = rsqrtf((float)D) * PG_LOG2E;
  float cap_l2 = 0.f, to_tanh = 0.f, slope_l2 = 0.f;
  if (MODE == PAGED_MOD) {
    if (a.softcap > 0.f) {
      cap_l2 = a.softcap * PG_LOG2E;
      to_tanh = rsqrtf((float)D) / a.softcap;
    }
    if (a.slopes && g < G) slope_l2 = a.slopes[kvh * G + g] * PG_LOG2E;
  }
  float* srow = MODE == PAGED_SCORED ? a.scores + ((size_t)b * a.Hq + kvh * G + (g < G ? g : 0)) * a.score_stride : nullptr;

  float o[DN][2];  // row g of each 8-wide output column tile (rows 8..15 are padding and dropped)
#pragma unroll
  for (int i = 0; i < DN; ++i) o[i][0] = o[i][1] = 0.f;
  float m_run = PG_NEG, l_run = 0.f;

  bool ok = true;
  int slot = 0;
  uint32_t phase = 0;
  for (int i = 0; i < my_n; ++i) {
    if (!mbar_wait(my_bars + 8u * slot, phase, nullptr)) { ok = false; break; }
    const uint32_t kt = my_ring + slot * SLOT_BYTES, vt = kt + PAGE_BYTES;
    const int k0 = page_index(i) * PG_PT;
    auto visible = [&](int key) {
      if (MODE == PAGED_MOD) return key < total && (key >= lo || key < pre);
      if (MODE == PAGED_FLAT) return key < 0 ? key + n_pre * PG_PT < pre : key < total;
      return key < total;
    };
    // slots that nobody may see can hold anything: their values are zeroed (a weight of 0 times infinity is not 0)
    const bool partial = MODE == PAGED_FLAT && k0 < 0 ? k0 + PG_PT == 0 && (pre & (PG_PT - 1)) != 0
                                                      : k0 + PG_PT > total || (MODE == PAGED_MOD && k0 < lo && k0 + PG_PT > pre);
    if (partial) {
      for (int e = lane; e < PG_PT * CPR; e += 32)
        if (!visible(k0 + e / CPR))
          asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vt + (uint32_t)e * 16u), "r"(0u) : "memory");
      __syncwarp();
    }

    // scores of the page's 16 keys: two 8-key column tiles
    float s[2][4];
    s[0][0] = s[0][1] = s[0][2] = s[0][3] = 0.f;
    s[1][0] = s[1][1] = s[1][2] = s[1][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int r = (lane & 7) + ((lane >> 4) << 3);
      const int c = 2 * ks + ((lane >> 3) & 1);
      uint32_t b0, b1, b2, b3;
      ldsm_x4(kt + tile_off<D>(r, c), b0, b1, b2, b3);
      mma_f16_16816(s[0], qf[ks][0], 0u, qf[ks][1], 0u, b0, b1);
      mma_f16_16816(s[1], qf[ks][0], 0u, qf[ks][1], 0u, b2, b3);
    }
    const int key0 = k0 + 2 * tq;
    float mx = m_run;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = key0 + 8 * nt + e;
        float v;
        if (MODE == PAGED_MOD) {
          v = a.softcap > 0.f ? tanh_any(s[nt][e] * to_tanh) * cap_l2 : s[nt][e] * sl2;
          v = fmaf(slope_l2, (float)(key - (total - 1)), v);
        } else {
          v = s[nt][e] * sl2;
        }
        v = visible(key) ? v : PG_NEG;
        s[nt][e] = v;
        mx = fmaxf(mx, v);
      }
    if (MODE == PAGED_SCORED && g < G) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
        *reinterpret_cast<float2*>(srow + key0 + 8 * nt) = make_float2(s[nt][0], s[nt][1]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float corr = ex2_approx(m_run - mx);
    m_run = mx;
    float p[2][2];
    float sum = 0.f;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        p[nt][e] = visible(key0 + 8 * nt + e) ? ex2_approx(s[nt][e] - mx) : 0.f;
        sum += p[nt][e];
      }
    l_run = l_run * corr + sum;
    const uint32_t pa0 = pack_f16(p[0][0], p[0][1]), pa2 = pack_f16(p[1][0], p[1][1]);
#pragma unroll
    for (int dp = 0; dp < DN / 2; ++dp) {
      const int r = (lane & 7) + (((lane >> 3) & 1) << 3);
      const int c = 2 * dp + (lane >> 4);
      uint32_t b0, b1, b2, b3;
      ldsm_x4_t(vt + tile_off<D>(r, c), b0, b1, b2, b3);
      float c0[4] = {o[2 * dp][0] * corr, o[2 * dp][1] * corr, 0.f, 0.f};
      float c1[4] = {o[2 * dp + 1][0] * corr, o[2 * dp + 1][1] * corr, 0.f, 0.f};
      mma_f16_16816(c0, pa0, 0u, pa2, 0u, b0, b1);
      mma_f16_16816(c1, pa0, 0u, pa2, 0u, b2, b3);
      o[2 * dp][0] = c0[0]; o[2 * dp][1] = c0[1];
      o[2 * dp + 1][0] = c1[0]; o[2 * dp + 1][1] = c1[1];
    }
    __syncwarp();  // every lane's reads of the slot are done; hand it back to the copy engine
    if (i + SLOTS < my_n) {
      if (partial) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      issue(i + SLOTS, slot);
    }
    if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
  }
  if (!ok) {
    if (lane == 0) atomicCAS(a.err, 0, 21);
    for (int s = 0; s < SLOTS; ++s) mbar_wait(my_bars + 8u * s, 0, nullptr), mbar_wait(my_bars + 8u * s, 1, nullptr);
  }
  bar_sync();  // every warp is done with its ring: the space is reused below

  // combine the warps: (m, l) per head, then rescaled O
  l_run += __shfl_xor_sync(0xffffffffu, l_run, 1);
  l_run += __shfl_xor_sync(0xffffffffu, l_run, 2);
  float* sm_m = reinterpret_cast<float*>(smem);  // [WARPS][8]
  float* sm_l = sm_m + WARPS * 8;                // [WARPS][8]
  float* sm_o = sm_l + WARPS * 8;                // [WARPS][G][D]
  float *fin_m = sm_o + WARPS * G * D, *fin_inv = fin_m + 8;  // PAGED_SCORED, one split: the heads' maxima, reciprocal denominators
  float *ex_m = fin_inv + 8, *ex_l = ex_m + 8, *ex_o = ex_l + 8;  // CLUSTER: this CTA's result, read by its peers
  float *all_m = ex_o + G * D, *all_l = all_m + 64;               // CLUSTER: every CTA's maxima and denominators, [head][split]
  if (g < G) {
    if (tq == 0) {
      sm_m[warp * 8 + g] = m_run;
      sm_l[warp * 8 + g] = l_run;
    }
#pragma unroll
    for (int dn = 0; dn < DN; ++dn)
      *reinterpret_cast<float2*>(sm_o + (warp * G + g) * D + 8 * dn + 2 * tq) = make_float2(o[dn][0], o[dn][1]);
  }
  bar_sync();
  for (int e = tid; e < G * D; e += THREADS) {
    const int gq = e / D, dd = e % D;
    float mx = PG_NEG;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) mx = fmaxf(mx, sm_m[w * 8 + gq]);
    float l = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float wgt = ex2_approx(sm_m[w * 8 + gq] - mx);
      l += wgt * sm_l[w * 8 + gq];
      acc += wgt * sm_o[(w * G + gq) * D + dd];
    }
    if (CLUSTER) {
      ex_o[e] = acc;
      if (dd == 0) {
        ex_m[gq] = mx;
        ex_l[gq] = l;
      }
    } else if (a.out) {
      a.out[((size_t)b * a.Hq + kvh * G + gq) * D + dd] = __float2half_rn(l != 0.f ? acc / l : 0.f);
      if (MODE == PAGED_SCORED && dd == 0) {
        fin_m[gq] = mx;
        fin_inv[gq] = l != 0.f ? 1.f / l : 0.f;
      }
    } else {
      const size_t row = ((size_t)b * a.Hq + kvh * G + gq) * a.n_slots + a.slot0 + split;
      a.acc[row * D + dd] = acc;
      if (dd == 0) *reinterpret_cast<float2*>(a.ml + row * 2) = make_float2(mx, l);
    }
  }
  if (CLUSTER) {
    bar_sync();
    cluster_barrier();
    // loads from a peer have a long latency: every thread asks for all of its own at once
    if (tid < G * n_splits) {
      const int gq = tid / n_splits, sp = tid % n_splits;
      const float mv = ld_cluster_f32(smem_u32(ex_m + gq), sp), lv = ld_cluster_f32(smem_u32(ex_l + gq), sp);
      all_m[gq * 8 + sp] = mv;
      all_l[gq * 8 + sp] = lv;
    }
    bar_sync();
    const int per = (G * D + n_splits - 1) / n_splits, e1 = min(G * D, (split + 1) * per);
    for (int e = split * per + tid; e < e1; e += THREADS) {
      const int gq = e / D;
      float ov[8];
#pragma unroll
      for (int sp = 0; sp < 8; ++sp) ov[sp] = sp < n_splits ? ld_cluster_f32(smem_u32(ex_o + e), sp) : 0.f;
      float mx = PG_NEG, l = 0.f, acc = 0.f;
#pragma unroll
      for (int sp = 0; sp < 8; ++sp)
        if (sp < n_splits) mx = fmaxf(mx, all_m[gq * 8 + sp]);
#pragma unroll
      for (int sp = 0; sp < 8; ++sp)
        if (sp < n_splits) {
          const float wgt = ex2_approx(all_m[gq * 8 + sp] - mx);
          l += wgt * all_l[gq * 8 + sp];
          acc += wgt * ov[sp];
        }
      a.out[((size_t)b * a.Hq + kvh * G) * D + e] = __float2half_rn(l != 0.f ? acc / l : 0.f);
    }
  }
  if (MODE == PAGED_SCORED && a.out) {
    bar_sync();  // the scores in global memory are this CTA's own
    const float* sc = a.scores + ((size_t)b * a.Hq + kvh * G) * a.score_stride;
    const long long wrow = ((long long)b * a.Hkv + kvh) * a.w_stride;
    for (int i = lane >> 4; i < my_n; i += 2) {  // a warp takes two of its pages at a time
      const int k = page_index(i) * PG_PT + (lane & 15);
      if (k < total) {
        float w = 0.f;
#pragma unroll
        for (int gq = 0; gq < G; ++gq) w += ex2_approx(sc[(size_t)gq * a.score_stride + k] - fin_m[gq]) * fin_inv[gq];
        a.w_out[wrow + k] = a.w_in && k < total - 1 ? fmaf(a.decay, a.w_in[wrow + k], w) : w;  // the new token's sum starts here
      }
    }
  }
  if (CLUSTER) cluster_barrier();  // nobody leaves while a peer may still read its result
}

// Joins the n_slots (at most 96) partial rows that start at row0 and writes the query head's D fp16 results.  A CTA of
// MERGE_THREADS; every warp derives the slots' weights for itself, takes every fourth slot's values, and the warps meet in
// shared memory.  A slot whose denominator is 0 has seen nothing: its values are not read.  A query with nothing to see
// gives zeros.
constexpr int MERGE_THREADS = 128, MERGE_SLOTS = 96;
template <int D>
__device__ __forceinline__ void paged_merge_row(const float* acc, const float* ml, size_t row0, int n_slots, __half* out, float* sm) {
  constexpr int V = D / 32, WARPS = MERGE_THREADS / 32;  // values per lane
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float m[3], l[3], w[3];
  float mx = PG_NEG;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int s = lane + 32 * k;
    const float2 x = s < n_slots ? *reinterpret_cast<const float2*>(ml + (row0 + s) * 2) : make_float2(PG_NEG, 0.f);
    m[k] = x.x;
    l[k] = x.y;
    mx = fmaxf(mx, x.x);
  }
  mx = warp_max(mx);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    w[k] = l[k] != 0.f ? ex2_approx(m[k] - mx) : 0.f;  // NaN is carried on
    sum += l[k] != 0.f ? w[k] * l[k] : 0.f;
  }
  sum = warp_sum(sum);
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll 4
    for (int s = warp; s < 32; s += WARPS) {
      if (32 * k + s >= n_slots) break;
      const float ws = __shfl_sync(0xffffffffu, w[k], s), ls = __shfl_sync(0xffffffffu, l[k], s);
      if (ls != 0.f) {
        const float* src = acc + (row0 + 32 * k + s) * D + V * lane;
        if (V == 4) {
          const float4 x = *reinterpret_cast<const float4*>(src);
          v[0] += ws * x.x; v[1] += ws * x.y; v[2] += ws * x.z; v[V - 1] += ws * x.w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(src);
          v[0] += ws * x.x; v[1] += ws * x.y;
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) sm[warp * D + V * lane + i] = v[i];
  __syncthreads();
  if ((int)threadIdx.x < D) {
    float x = 0.f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) x += sm[k * D + threadIdx.x];
    out[threadIdx.x] = __float2half_rn(sum != 0.f ? x / sum : 0.f);
  }
}

}  // namespace hyp
