// Decode attention of one new token per sequence over the 8-bit paged cache.
//
// A CTA takes one (split, KV head, sequence); the pages go round-robin over the splits and, inside the CTA, over the warps.  Every warp
// streams its pages through a ring of bulk copies (a half page of one head is one run: codes and scales) and forms, with no CTA-wide
// step, S^T = K Q^T and O^T += V^T P^T on mma.sync.m16n8k16: the page's 16 keys, or 16 of the head's dimensions, are the operand of 16
// rows and the (up to eight) query heads of the KV head that of eight columns, so that no row of an instruction is idle.
//   Codes become fp16 on their way to the operand registers: offset codes by a byte permute that puts them below the exponent of
//   1024 and one packed subtraction, E4M3 by the hardware conversion; both exact.  The order of the dimensions inside a product is that
//   in which a lane reads 16 bytes of a key's row; the queries are fetched in the same order.
//   A key's scale multiplies its score in fp32.  A value's scale goes into its weight: w = p * scale * 2^(m - m2), with references m for
//   the scores and m2 for score + log2(scale), so that the fp16 weights are relative to the largest one, whatever the scales are.  What is kept
//   is m2 - m: beside a score of 1e9 and more m2 itself would have lost log2(scale) to rounding.
//   Both references move only when a weight outgrows 2^15 (one vote a step instead of shuffles and a rescaled O).
// A warp takes two pages a step: their chains of products run side by side (8 x 1024 tokens 9.9 -> 8.7 us).
// Weights are rounded to fp16 (2^-11 of each, or 2^-32 of the warp's largest so far); sums, references and O are fp32.  Bound by HBM: 4 x 32768 tokens of 10 KV heads of 128 5.7 TB/s
// of cache, where the same copies without the arithmetic reach 5.8; 64 ragged sequences of up to 8192 5.6 (6.0); 8 x 1024 one wave of
// latencies, 8.7 us (6.4).  Neither more CTAs (six of 80 registers) nor the conversions taken out changed the long ones.
#include "attn_paged.cuh"
#include "cache_ops.cuh"
#include "kv8.cuh"
#include "mx4.cuh"

namespace hyp {

namespace {

constexpr int K8_WARPS = 4, K8_THREADS = K8_WARPS * 32;
constexpr int K8_STEP = 2, K8_SLOTS = 2;    // pages that a warp takes at a time; ring slots of that many
constexpr int K8_PER_SM = 3, K8_WAVES = 5;  // resident CTAs; waves that a long context is cut for
// The value reference moves so that the largest weight times scale is 2^K8_HEAD, and a weight may grow to 2^15 (fp16 ends at 2^16) before it moves again:
// what lies 2^21 below the largest is still a normal fp16 number and steps of 2^-31 of it are left below that.  With the largest at 1 a million small weights beside a
// large one could lose, or count twice, 3 % of the result.
constexpr float K8_HEAD = 7.f, K8_GROWN = 32768.f;
// "No key seen yet".  A key's fp32 scale takes scores down to -FLT_MAX, so nothing finite is below every one of them; at the bottom itself a
// reference that has not moved is as good as one that has.
constexpr float K8_NONE = -3.402823466e38f;

struct Kv8Args {
  const __half* q;  // row b at q + b * q_stride
  long long q_stride;
  const uint8_t* pool;
  const int32_t* table;
  int table_stride;
  const int32_t* ctx;
  int Hq, Hkv;
  float* acc;  // partial rows ((b * Hq + h) * n_slots + split) * D, their (maximum, denominator) in ml
  float* ml;
  int n_slots, wave_splits;
  __half* out;  // one split, or a cluster: the result itself
  int* err;
};

template <int D>
constexpr int kv8_smem() { return K8_WARPS * K8_SLOTS * K8_STEP * 2 * kv8_half_page(D); }

// Four codes of one row to two operand registers: (0, 1) and (2, 3).
template <int FMT>
__device__ __forceinline__ void key_pair(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FMT == HYP_KV8_INT8) {
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
    uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), bias), y = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  } else {
    lo = e4m3x2_to_half2(w & 0xffffu);
    hi = e4m3x2_to_half2(w >> 16);
  }
}
// Two dimensions of two tokens, bytes (t0 d0, t0 d1, t1 d0, t1 d1), to the token pairs of d0 and of d1.
template <int FMT>
__device__ __forceinline__ void value_pair(uint32_t w, uint32_t& d0, uint32_t& d1) {
  if (FMT == HYP_KV8_INT8) {
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));
    uint32_t a = __byte_perm(w, 0x64646464u, 0x4240), b = __byte_perm(w, 0x64646464u, 0x4341);
    const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), bias), y = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
    d0 = *reinterpret_cast<const uint32_t*>(&x);
    d1 = *reinterpret_cast<const uint32_t*>(&y);
  } else {
    const uint32_t t = __byte_perm(w, 0u, 0x3120);
    d0 = e4m3x2_to_half2(t & 0xffffu);
    d1 = e4m3x2_to_half2(t >> 16);
  }
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ float lds32(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

template <int D, int G, int FMT, bool CLUSTER>
__global__ void __launch_bounds__(K8_THREADS, K8_PER_SM) attn_kv8_kernel(const Kv8Args a) {
  constexpr int KS = D / 16, HALF = kv8_half_page(D), PAGE = 2 * HALF, SLOT = K8_STEP * PAGE, T = K8_STEP;
  static_assert(T == 2, "page ids come in pairs");
  extern __shared__ __align__(128) uint8_t k8_smem[];
  __shared__ uint64_t bars[K8_WARPS * K8_SLOTS];
  static_assert(kv8_smem<D>() >= (2 * K8_WARPS * 8 + K8_WARPS * G * D + 16 + G * D + 128) * 4, "the combine buffers reuse the ring");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, tq = lane & 3;
  const int split = blockIdx.x, n_splits = gridDim.x, kvh = blockIdx.y, b = blockIdx.z;
  pdl_wait();     // queries, lengths and cache rows may come from the kernel launched just before
  pdl_trigger();

  const int32_t* bt = a.table + (long long)b * a.table_stride;
  // Ids of this warp's next 32 steps of two pages, one step a lane; the first ones do not wait for the length.
  int2 ids_cur = make_int2(0, 0);
  auto two_ids = [&](int step, int limit) {
    return make_int2(T * step < limit ? bt[T * step] : 0, T * step + 1 < limit ? bt[T * step + 1] : 0);
  };
  ids_cur = two_ids(split + n_splits * (warp + K8_WARPS * lane), a.table_stride);
  const int total = paged_total(a.ctx[b], a.table_stride), n_pages = (total + PG_PT - 1) / PG_PT, n_steps = (n_pages + T - 1) / T;
  // a shorter sequence uses no more splits than the plan's rule gives for its own length
  const int fair = max(a.wave_splits, (n_pages + 15) / 16);
  const int used = n_pages > 64 * a.wave_splits ? n_splits : max(min(min(n_splits, fair), (n_steps + K8_WARPS - 1) / K8_WARPS), 1);
  if (!CLUSTER && split >= used) {
    if (tid < G) *reinterpret_cast<float2*>(a.ml + (((size_t)b * a.Hq + kvh * G + tid) * a.n_slots + split) * 2) = make_float2(K8_NONE, 0.f);
    return;
  }
  const int first = split + used * warp, stride_s = used * K8_WARPS;
  const int my_n = split < used && first < n_steps ? (n_steps - first + stride_s - 1) / stride_s : 0;
  auto load_ids = [&](int base) { return base + lane < my_n ? two_ids(first + stride_s * (base + lane), n_pages) : make_int2(0, 0); };
  if (used != n_splits) ids_cur = load_ids(0);
  int2 ids_next = load_ids(32);
  const uint32_t my_bars = smem_u32(bars) + 8u * (warp * K8_SLOTS), my_ring = smem_u32(k8_smem) + (uint32_t)(warp * K8_SLOTS) * SLOT;
  const uint32_t page_bytes = 2u * a.Hkv * HALF, v_off = (uint32_t)a.Hkv * HALF;
  const uint8_t* head_base = a.pool + (size_t)kvh * HALF;
  auto issue = [&](int i, int slot) {  // all lanes call, i ascending
    if (i > 0 && (i & 31) == 0) {
      ids_cur = ids_next;
      ids_next = load_ids(i + 32);
    }
    const int page0 = __shfl_sync(0xffffffffu, ids_cur.x, i & 31), page1 = __shfl_sync(0xffffffffu, ids_cur.y, i & 31);
    if (lane == 0) {
      const uint32_t dst = my_ring + slot * SLOT, bar = my_bars + 8u * slot;
      const bool both = T * (first + stride_s * i) + 1 < n_pages;  // the last step may hold one page
      mbar_expect_tx(bar, both ? SLOT : PAGE);
      const uint8_t* src = head_base + (uint64_t)(uint32_t)page0 * page_bytes;
      bulk_load(dst, src, HALF, bar);
      bulk_load(dst + HALF, src + v_off, HALF, bar);
      if (both) {
        src = head_base + (uint64_t)(uint32_t)page1 * page_bytes;
        bulk_load(dst + PAGE, src, HALF, bar);
        bulk_load(dst + PAGE + HALF, src + v_off, HALF, bar);
      }
    }
  };
  if (lane == 0) {
    for (int s = 0; s < K8_SLOTS; ++s) mbar_init(my_bars + 8u * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  for (int s = 0; s < K8_SLOTS && s < my_n; ++s) issue(s, s);

  // queries: column g of the operand, four dimensions a product in the order of the keys' bytes
  uint32_t qf[KS][2];
  {
    const __half* qrow = a.q + (long long)b * a.q_stride + (size_t)(kvh * G + (g < G ? g : 0)) * D;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const uint2 x = *reinterpret_cast<const uint2*>(qrow + 64 * (j / 4) + 16 * tq + 4 * (j % 4));
      qf[j][0] = g < G ? x.x : 0u;
      qf[j][1] = g < G ? x.y : 0u;
    }
  }
  const float sl2 = rsqrtf((float)D) * PG_LOG2E;
  float o[KS][4];  // 16-byte chunk c of the head: (dims 16c + 2g, + 1) x (heads 2tq, 2tq + 1)
#pragma unroll
  for (int c = 0; c < KS; ++c) o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;
  float m[2] = {K8_NONE, K8_NONE}, d2[2] = {0.f, 0.f}, f[2] = {1.f, 1.f}, l[2] = {0.f, 0.f};  // of heads 2tq, 2tq + 1; d2 = m2 - m, f = 2^-d2

  bool ok = true;
  int slot = 0;
  uint32_t phase = 0;
  for (int i = 0; i < my_n; ++i) {
    if (!__all_sync(0xffffffffu, mbar_wait(my_bars + 8u * slot, phase, nullptr))) { ok = false; break; }
    const uint32_t at0 = my_ring + slot * SLOT;
    const int k0 = T * (first + stride_s * i) * PG_PT;
    const bool partial = k0 + T * PG_PT > total;
    if (FMT == HYP_KV8_E4M3 && partial) {  // a code behind the end may be a NaN, and a weight of 0 times NaN is not 0
      for (int e = lane; e < T * D; e += 32)
        if (k0 + e / (D / 16) >= total)
          asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at0 + HALF + (uint32_t)(e / D * PAGE + e % D * 16)), "r"(0u) : "memory");
      __syncwarp();
    }
    // scores of keys g and g + 8 of every page for heads 2tq, 2tq + 1
    float s[T][4];
#pragma unroll
    for (int t = 0; t < T; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const uint32_t at = at0 + t * PAGE + g * D + kv8_chunk<D>(tq + 4 * h, g);  // slots g and g + 8 have the same parity
        const uint4 x = lds128(at), y = lds128(at + 8 * D);
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t a0, a1, a2, a3;
          key_pair<FMT>(xw[j], a0, a2);
          key_pair<FMT>(yw[j], a1, a3);
          mma_f16_16816(s[t], a0, a1, a2, a3, qf[4 * h + j][0], qf[4 * h + j][1]);
        }
      }
    }
    // [page][(key g, head 2tq), (g, 2tq + 1), (g + 8, 2tq), (g + 8, 2tq + 1)]
    float v[T][4], p[T][4], w[T][4], vs[T][2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const uint32_t sc = at0 + t * PAGE + 16 * D + 4 * g;
      const float ks0 = lds32(sc) * sl2, ks1 = lds32(sc + 32) * sl2;
      vs[t][0] = lds32(sc + HALF);
      vs[t][1] = lds32(sc + HALF + 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[t][e] = s[t][e] * (e < 2 ? ks0 : ks1);
    }
    if (partial) {  // keys behind the end: no weight, whatever their slots hold
#pragma unroll
      for (int t = 0; t < T; ++t) {
        if (k0 + t * PG_PT + g >= total) v[t][0] = v[t][1] = -INFINITY, vs[t][0] = 0.f;
        if (k0 + t * PG_PT + g + 8 >= total) v[t][2] = v[t][3] = -INFINITY, vs[t][1] = 0.f;
      }
    }
    float most = 0.f;
    auto weigh = [&] {  // (a scale times a reference may leave fp32: 0 times infinity would be NaN)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[t][e] = ex2_approx(v[t][e] - m[e & 1]);
          w[t][e] = p[t][e] * min_nan(vs[t][e >> 1] * f[e & 1], 3e38f);
          most = fmaxf(most, fmaxf(p[t][e], w[t][e]));
        }
    };
    weigh();
    if (__any_sync(0xffffffffu, most > K8_GROWN)) {  // new references: the largest score, the largest score + log2(scale)
      float corr2[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = m[h];
#pragma unroll
        for (int t = 0; t < T; ++t) top = fmaxf(top, fmaxf(v[t][h], v[t][2 + h]));
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float down = m[h] - top;  // (may leave fp32 to -infinity: the old sums are nothing then)
        float d = down + d2[h];
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int k = 0; k < 2; ++k) d = fmaxf(d, v[t][2 * k + h] - top + (fmaxf(lg2_approx(vs[t][k]), -64.f) - K8_HEAD));  // (values whose scale is below 2^-64 are zeros in fp16)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) d = fmaxf(d, __shfl_xor_sync(0xffffffffu, d, x));
        l[h] *= ex2_approx(down);
        corr2[h] = ex2_approx(down + d2[h] - d);
        m[h] = top;
        d2[h] = d;
        f[h] = ex2_approx(-d);
      }
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        o[c][0] *= corr2[0]; o[c][2] *= corr2[0];
        o[c][1] *= corr2[1]; o[c][3] *= corr2[1];
      }
      weigh();
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      l[0] += p[t][0] + p[t][2];
      l[1] += p[t][1] + p[t][3];
      const uint32_t b0 = transpose_8x8(pack_f16(w[t][0], w[t][1])), b1 = transpose_8x8(pack_f16(w[t][2], w[t][3]));
      const uint32_t vt = at0 + t * PAGE + HALF;
#pragma unroll
      for (int c2 = 0; c2 < KS / 2; ++c2) {
        const int row = lane & 15;  // slots 0-7 and 8-15 of chunk 2 c2, then of the next one
        uint32_t r0, r1, r2, r3, a0, a1, a2, a3;
        ldsm_x4_t(vt + row * D + kv8_chunk<D>(2 * c2 + (lane >> 4), row), r0, r1, r2, r3);
        value_pair<FMT>(r0, a0, a1);
        value_pair<FMT>(r1, a2, a3);
        mma_f16_16816(o[2 * c2], a0, a1, a2, a3, b0, b1);
        value_pair<FMT>(r2, a0, a1);
        value_pair<FMT>(r3, a2, a3);
        mma_f16_16816(o[2 * c2 + 1], a0, a1, a2, a3, b0, b1);
      }
    }
    __syncwarp();  // every lane's reads of the slot are done; hand it back to the copy engine
    if (i + K8_SLOTS < my_n) issue(i + K8_SLOTS, slot);
    if (++slot == K8_SLOTS) { slot = 0; phase ^= 1u; }
  }
  if (!ok) {
    if (lane == 0) atomicCAS(a.err, 0, 34);
    for (int s = 0; s < K8_SLOTS; ++s) mbar_wait(my_bars + 8u * s, 0, nullptr), mbar_wait(my_bars + 8u * s, 1, nullptr);
  }
  __syncthreads();  // every warp is done with its ring: the space is reused below

  float* sm_m = reinterpret_cast<float*>(k8_smem);  // [warps][8]
  float* sm_l = sm_m + K8_WARPS * 8;
  float* sm_o = sm_l + K8_WARPS * 8;                // [warps][G][D]
  float *ex_m = sm_o + K8_WARPS * G * D, *ex_l = ex_m + 8, *ex_o = ex_l + 8;  // CLUSTER: this CTA's result, read by its peers
  float *all_m = ex_o + G * D, *all_l = all_m + 64;                           // CLUSTER: every CTA's, [head][split]
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
    const float back = ex2_approx(d2[h]);  // O in units of 2^m
    const int head = 2 * tq + h;
    if (head < G) {
      if (g == 0) {
        sm_m[warp * 8 + head] = m[h];
        sm_l[warp * 8 + head] = l[h];
      }
#pragma unroll
      for (int c = 0; c < KS; ++c)
        *reinterpret_cast<float2*>(sm_o + (warp * G + head) * D + 16 * c + 2 * g) = make_float2(o[c][h] * back, o[c][2 + h] * back);
    }
  }
  __syncthreads();
  for (int e = tid; e < G * D; e += K8_THREADS) {
    const int gq = e / D, dd = e % D;
    float mx = K8_NONE;
#pragma unroll
    for (int w = 0; w < K8_WARPS; ++w) mx = fmaxf(mx, sm_m[w * 8 + gq]);
    float lsum = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < K8_WARPS; ++w) {
      const float wgt = ex2_approx(sm_m[w * 8 + gq] - mx);
      lsum += wgt * sm_l[w * 8 + gq];
      acc += wgt * sm_o[(w * G + gq) * D + dd];
    }
    if (CLUSTER) {
      ex_o[e] = acc;
      if (dd == 0) {
        ex_m[gq] = mx;
        ex_l[gq] = lsum;
      }
    } else if (a.out) {
      a.out[((size_t)b * a.Hq + kvh * G + gq) * D + dd] = __float2half_rn(lsum != 0.f ? acc / lsum : 0.f);
    } else {
      const size_t row = ((size_t)b * a.Hq + kvh * G + gq) * a.n_slots + split;
      a.acc[row * D + dd] = acc;
      if (dd == 0) *reinterpret_cast<float2*>(a.ml + row * 2) = make_float2(mx, lsum);
    }
  }
  if (CLUSTER) {
    __syncthreads();
    cluster_barrier();
    if (tid < G * n_splits) {  // loads from a peer have a long latency: every thread asks for all of its own at once
      const int gq = tid / n_splits, sp = tid % n_splits;
      const float mv = ld_cluster_f32(smem_u32(ex_m + gq), sp), lv = ld_cluster_f32(smem_u32(ex_l + gq), sp);
      all_m[gq * 8 + sp] = mv;
      all_l[gq * 8 + sp] = lv;
    }
    __syncthreads();
    const int per = (G * D + n_splits - 1) / n_splits, e1 = min(G * D, (split + 1) * per);
    for (int e = split * per + tid; e < e1; e += K8_THREADS) {
      const int gq = e / D;
      float ov[8];
#pragma unroll
      for (int sp = 0; sp < 8; ++sp) ov[sp] = sp < n_splits ? ld_cluster_f32(smem_u32(ex_o + e), sp) : 0.f;
      float mx = K8_NONE, lsum = 0.f, acc = 0.f;
#pragma unroll
      for (int sp = 0; sp < 8; ++sp)
        if (sp < n_splits) mx = fmaxf(mx, all_m[gq * 8 + sp]);
#pragma unroll
      for (int sp = 0; sp < 8; ++sp)
        if (sp < n_splits) {
          const float wgt = ex2_approx(all_m[gq * 8 + sp] - mx);
          lsum += wgt * all_l[gq * 8 + sp];
          acc += wgt * ov[sp];
        }
      a.out[((size_t)b * a.Hq + kvh * G) * D + e] = __float2half_rn(lsum != 0.f ? acc / lsum : 0.f);
    }
    cluster_barrier();  // nobody leaves while a peer may still read its result
  }
}

// Joins the partial rows of one (sequence, query head), at most 64.  Every warp derives the weights for itself and takes every fourth row,
// eight loads on their way at a time; a row that has seen nothing (denominator 0) holds anything and counts as zeros.
template <int D>
__global__ void __launch_bounds__(K8_THREADS) kv8_merge_kernel(const float* __restrict__ acc, const float* __restrict__ ml, int n_slots,
                                                               __half* __restrict__ out) {
  constexpr int V = D / 32, BATCH = 8;
  __shared__ float sm[K8_WARPS * D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const size_t row = blockIdx.x, row0 = row * n_slots;  // row = b * Hq + h
  pdl_wait();
  pdl_trigger();
  float m[2], l[2], w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = lane + 32 * k;
    const float2 x = s < n_slots ? *reinterpret_cast<const float2*>(ml + (row0 + s) * 2) : make_float2(K8_NONE, 0.f);
    m[k] = x.x;
    l[k] = x.y;
  }
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
  const float mx = warp_max(fmaxf(m[0], m[1]));
#pragma unroll
  for (int k = 0; k < 2; ++k) w[k] = l[k] != 0.f ? ex2_approx(m[k] - mx) : 0.f;  // NaN is carried on
  const float sum = warp_sum((l[0] != 0.f ? w[0] * l[0] : 0.f) + (l[1] != 0.f ? w[1] * l[1] : 0.f));
  for (int s0 = warp; s0 < n_slots; s0 += K8_WARPS * BATCH) {
    float r[BATCH][V];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int s = s0 + K8_WARPS * i;
      const float* src = acc + (row0 + (s < n_slots ? s : s0)) * D + V * lane;
      if (V == 4) {
        const float4 x = *reinterpret_cast<const float4*>(src);
        r[i][0] = x.x; r[i][1] = x.y; r[i][2] = x.z; r[i][V - 1] = x.w;
      } else {
        const float2 x = *reinterpret_cast<const float2*>(src);
        r[i][0] = x.x; r[i][1] = x.y;
      }
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int s = s0 + K8_WARPS * i;
      const float w0 = __shfl_sync(0xffffffffu, w[0], s & 31), w1 = __shfl_sync(0xffffffffu, w[1], s & 31);
      const float l0 = __shfl_sync(0xffffffffu, l[0], s & 31), l1 = __shfl_sync(0xffffffffu, l[1], s & 31);
      const float ws = s < 32 ? w0 : w1;
      if (s < n_slots && (s < 32 ? l0 : l1) != 0.f) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = fmaf(ws, r[i][j], v[j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) sm[warp * D + V * lane + i] = v[i];
  __syncthreads();
  if ((int)threadIdx.x < D) {
    float x = 0.f;
#pragma unroll
    for (int k = 0; k < K8_WARPS; ++k) x += sm[k * D + threadIdx.x];
    out[row * D + threadIdx.x] = __float2half_rn(sum != 0.f ? x / sum : 0.f);
  }
}

// The same for up to K8_FEW rows of each of n_rows (sequence, query head): a warp joins them, all its loads on their way at once.
constexpr int K8_FEW = 8;
template <int D>
__global__ void __launch_bounds__(K8_THREADS) kv8_merge_few_kernel(const float* __restrict__ acc, const float* __restrict__ ml, int n_slots,
                                                                   int n_rows, __half* __restrict__ out) {
  constexpr int V = D / 32;
  const int lane = threadIdx.x & 31, row = blockIdx.x * K8_WARPS + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (row >= n_rows) return;
  const size_t first = (size_t)row * n_slots;
  float r[K8_FEW][V];
  float2 x[K8_FEW];
#pragma unroll
  for (int i = 0; i < K8_FEW; ++i) {
    const size_t at = first + (i < n_slots ? i : 0);
    x[i] = *reinterpret_cast<const float2*>(ml + at * 2);
    const float* src = acc + at * D + V * lane;
    if (V == 4) {
      const float4 y = *reinterpret_cast<const float4*>(src);
      r[i][0] = y.x; r[i][1] = y.y; r[i][2] = y.z; r[i][V - 1] = y.w;
    } else {
      const float2 y = *reinterpret_cast<const float2*>(src);
      r[i][0] = y.x; r[i][1] = y.y;
    }
  }
  float mx = K8_NONE, sum = 0.f, v[V];
#pragma unroll
  for (int i = 0; i < K8_FEW; ++i) mx = fmaxf(mx, x[i].x);
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = 0.f;
#pragma unroll
  for (int i = 0; i < K8_FEW; ++i) {
    if (i >= n_slots || x[i].y == 0.f) continue;  // NaN is carried on
    const float w = ex2_approx(x[i].x - mx);
    sum = fmaf(w, x[i].y, sum);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = fmaf(w, r[i][j], v[j]);
  }
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  __half* to = out + (size_t)row * D + V * lane;
  if (V == 4)
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_f16(v[0] * inv, v[1] * inv), pack_f16(v[2] * inv, v[V - 1] * inv));
  else
    *reinterpret_cast<uint32_t*>(to) = pack_f16(v[0] * inv, v[1] * inv);
}

template <int D, int G, int FMT, bool CLUSTER>
int launch_one(const Kv8Args& a, int n_splits, int n_seqs, cudaStream_t st) {
  constexpr int smem = kv8_smem<D>();
  const int rc = allow_smem<attn_kv8_kernel<D, G, FMT, CLUSTER>>(smem);
  if (rc) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_splits, a.Hkv, n_seqs);
  cfg.blockDim = dim3(K8_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = pdl_level() >= 2;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_splits;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CLUSTER ? 2 : 1;
  HYP_CUDA_TRY(cudaLaunchKernelEx(&cfg, attn_kv8_kernel<D, G, FMT, CLUSTER>, a));
  return 1;
}

template <int D, int G, int FMT>
int launch_joined(Kv8Args a, int n_splits, int n_seqs, __half* out, cudaStream_t st) {
  const bool cluster = n_splits >= 2 && n_splits <= 8 && (long long)n_splits * a.Hkv * n_seqs <= (long long)K8_PER_SM * sm_count();
  if (n_splits == 1 || cluster) a.out = out;
  else if ((long long)n_seqs * a.Hq > 0x7fffffffll) return HYP_ECAPACITY;  // rows to join
  if (cluster) return launch_one<D, G, FMT, true>(a, n_splits, n_seqs, st);
  const int rc = launch_one<D, G, FMT, false>(a, n_splits, n_seqs, st);
  if (rc < 0 || n_splits == 1) return rc;
  const int rows = n_seqs * a.Hq;
  if (a.n_slots <= K8_FEW)
    HYP_CUDA_TRY(launch_pdl<2>(kv8_merge_few_kernel<D>, dim3((unsigned)((rows + K8_WARPS - 1) / K8_WARPS)), dim3(K8_THREADS), (size_t)0, st, a.acc, a.ml,
                               a.n_slots, rows, out));
  else
    HYP_CUDA_TRY(launch_pdl<2>(kv8_merge_kernel<D>, dim3((unsigned)rows), dim3(K8_THREADS), (size_t)0, st, a.acc, a.ml, a.n_slots, out));
  return rc + 1;
}

template <int D, int G>
int launch_fmt(const Kv8Args& a, int fmt, int n_splits, int n_seqs, __half* out, cudaStream_t st) {
  return fmt == HYP_KV8_INT8 ? launch_joined<D, G, HYP_KV8_INT8>(a, n_splits, n_seqs, out, st)
                             : launch_joined<D, G, HYP_KV8_E4M3>(a, n_splits, n_seqs, out, st);
}

int wave_splits(int n_seqs, int Hkv) {
  const int want = (int)((long long)K8_PER_SM * sm_count() / ((long long)n_seqs * Hkv));
  return want < 1 ? 1 : want;
}

}  // namespace

int kv8_splits(int n_seqs, int Hkv, int max_pages) {
  // Up to 16 pages: one CTA per sequence and KV head, which writes the result itself (the join is a launch of its own).  Short contexts, and
  // long ones of few heads: one wave of CTAs, or just below (4 x 32768 tokens, 10 KV heads: 60.5 us in one wave, 62.7 / 65 / 67.3 in two to
  // four).  Long contexts of more heads than a fourth of a wave: about five waves, so that ragged batches even out (64 ragged sequences of up to
  // 8192, 8 heads: 111 us in one wave, 107.7 in three, 103 in five).  At least one step of two pages per warp.
  const long long groups = (long long)n_seqs * Hkv;
  if (max_pages <= 4 * K8_WARPS) return 1;
  int want = wave_splits(n_seqs, Hkv);
  if (want < 4 && max_pages > 64 * want) want = (int)(K8_WAVES * K8_PER_SM * sm_count() / groups);
  if (want < 1) want = 1;
  const int cap = (max_pages + K8_STEP * K8_WARPS - 1) / (K8_STEP * K8_WARPS);
  if (want > cap) want = cap;
  return want > 64 ? 64 : want;
}

int launch_attn_kv8(const Kv8View& c, const __half* q, long long q_stride, const int32_t* ctx, float* scratch, __half* out, int* err,
                    cudaStream_t st) {
  const int ns = kv8_splits(c.n_seqs, c.Hkv, c.table_stride), G = c.Hq / c.Hkv;
  Kv8Args a{};
  a.q = q; a.q_stride = q_stride; a.pool = c.pool; a.table = c.table; a.table_stride = c.table_stride; a.ctx = ctx;
  a.Hq = c.Hq; a.Hkv = c.Hkv;
  a.acc = scratch; a.ml = scratch + (size_t)c.n_seqs * c.Hq * ns * c.D; a.n_slots = ns;
  a.wave_splits = wave_splits(c.n_seqs, c.Hkv);
  a.err = err;
#define HYP_F(DD, GG) if (c.D == DD && G == GG) return launch_fmt<DD, GG>(a, c.fmt, ns, c.n_seqs, out, st);
  HYP_F(128, 1) HYP_F(128, 2) HYP_F(128, 4) HYP_F(128, 8) HYP_F(64, 1) HYP_F(64, 2) HYP_F(64, 4) HYP_F(64, 8)
#undef HYP_F
  return HYP_EINVAL;
}

}  // namespace hyp
