// Product of activations and microscaled 4-bit weights: out[m, n] (+)= sum_k a[m, k] * w[n, k].
//
// The tensor cores multiply E2M1 by E4M3 operands, each under a power of two per row and block of 32 k
// (tcgen05.mma.kind::mxf8f6f4.block_scale), with fp32 sums.  So nothing of the weights is converted by the CUDA cores: the copy
// engine spreads the packed codes to the operand's byte containers on their way to shared memory, the scales go from there to
// tensor memory.  (The CUDA cores would have 45 codes a cycle and SM to convert to keep up with HBM.)  The activations, 16-bit values,
// become one to three E4M3 terms: the first is a rounded to four bits under its block's power of two, the next is what is left, under a
// power of two of its own.  Two terms hold a bf16 value, three an fp16 value (what they leave is below 2^-25 of the block's largest).  The
// terms of a token are more columns of the same operand (they share the weights' pass through shared memory) and are added in the epilogue.
// The products are exact in the tensor cores' fp32 sums; the sums are not: measured against fp64 6e-8 of the result for 8 x 7680 x 5120 with K in
// four shares (a fp32 matrix product 1.0e-7), 2.3e-7 for 512 x 5120 x 17920, where one accumulator runs over 140 blocks (8.5e-8).
//
// A CTA owns two tiles of 128 weight rows (the M operand, two accumulators; SwiGLU: gate rows and the matching up rows; or one tile) and a
// tile of tokens (the N operand, terms x tokens columns, at most 256).  Where there are few such tiles K is split over a cluster of up to eight CTAs:
// each leaves its sums in shared memory, and every one of them finishes a share of the tokens, adding the others' in rank order
// through distributed shared memory: deterministic.
//   warp 0     one lane fills the ring with weight codes (a TMA box), one of warp 2 with weight scales, one of warp 3 with terms;
//   warp 1     one lane copies the scales to tensor memory and issues the MMAs;
//   warps 2-9  epilogue, lane = weight row.
// Few tokens: bound by the weights' way: from HBM for large matrices (32 rows, gate and up 17920 x 5120: 98 MB in 16 us of main loop, 23.4 us in
// all), through shared memory, where the spread weights are written and read at twice their size, for small ones (8 rows, 7680 x 5120:
// 9.6 us, 5 of them launches, terms, start and end).  Many tokens: by the operands' way from the L2 (512 x 5120 x 17920, one term: 51 us =
// 1.85 PFLOP/s, tensor pipe 62 % busy during the product; 2048 x 7680 x 5120: 82 us = 1.97; 2048 x 5120 x 17920: 170 us = 2.2).
// Every mbarrier wait is bounded; the cluster barriers are reached by every thread of every CTA.
#include <cuda.h>
#include <math.h>

#include <mutex>

#include "cache_ops.cuh"
#include "gemm_tc.cuh"
#include "mx4.cuh"
#include "tcgen05.cuh"

namespace hyp {

namespace {

constexpr int MX_EPI_WARPS = 8, MX_THREADS = 64 + 32 * MX_EPI_WARPS, MX_MAX_STAGES = 12, MX_A_BYTES = MX_ROWS * MX_BK;

// How a product is cut.
struct Plan {
  int a_tiles;         // weight row tiles of a CTA (SwiGLU: gate and up)
  int row_units;       // CTAs across the weight rows
  int tiles, tt, nb;   // token tiles of tt tokens, nb operand rows each (terms x tokens, filled up to a multiple of 16)
  int ksplit, sf_bytes;
  size_t block_bytes;  // terms of one (token tile, 128 k) with their scales
};
constexpr int MX_MAX_DYN = 216 * 1024, MX_MORE_TILES = 3;
constexpr int OWN_TERMS = 4, OWN_BYTES = 64 * 1024;  // see launch_for
// Tensor memory: one accumulator of 256 columns beside the scales, or two of 240.
int row_cap(int a_tiles) { return a_tiles == 2 ? 240 : 256; }
bool cut(Plan& p, int M, int N, int terms, int a_tiles, bool swiglu, int tiles) {
  p.a_tiles = a_tiles;
  p.row_units = (N + (swiglu ? 1 : a_tiles) * MX_ROWS - 1) / ((swiglu ? 1 : a_tiles) * MX_ROWS);
  p.tt = ((M + tiles - 1) / tiles + 7) / 8 * 8;
  p.tiles = (M + p.tt - 1) / p.tt;
  p.nb = (p.tt * terms + 15) / 16 * 16;
  p.sf_bytes = (p.nb + MX_ROWS - 1) / MX_ROWS * MX_SF_BYTES;
  p.block_bytes = (size_t)p.nb * MX_BK + p.sf_bytes;
  return p.nb <= row_cap(a_tiles);
}
// The fewest token tiles that M can be cut into.
int least_tiles(int M, int terms, int cap) {
  const int most = cap / terms / 8 * 8;
  return (M + most - 1) / most;
}
// CTAs that are on the GPU at once, one to an SM, in clusters of ks = 1 .. 8 (which do not fill every group of SMs that shares a cluster's
// paths); of the current device.
const int* slots_by_ks();
int tmem_columns(int a_tiles, int nb) {
  int cols = 32;
  while (cols < a_tiles * (nb + 4) + 8) cols <<= 1;
  return cols;
}
// The cheapest cut by a count of cycles.  A stage of 128 k takes the longest of: its operands' way into the SM (about 53 bytes a cycle from the
// L2), the ring's round trip (about 3300 for all stages that fit), the issuing warp (450, for two row tiles 700), the MMAs, and the
// weights' way from HBM (3300 bytes a cycle for all).  A CTA takes about 5000 to start and end, and its results; shares of K meet in a cluster.
// Measured against every cut of one or two row tiles, four token counts and one to six shares: within 5 % of the best of 512 x 5120 x 17920
// (one row tile 50.4 us, two 54.3), 512 x 7680 x 5120 (24.5, 27.1), 600 x 4096 x 4096, 128 x 5120 x 17920 (27.7, 30.5), 64 x 7680 x 5120 of three
// terms (14.2, 16.0), 8 x 7680 x 5120 (10.2, 9.5), 8 x 5120 x 17920 (16.1, 15.8) and eight others.
Plan plan_for(int M, int N, int KB, int terms, bool swiglu) {
  Plan best{}, p{};
  double least = 0.0;
  const int* slots_of = slots_by_ks();
  for (int a = swiglu ? 2 : 1; a <= 2; ++a) {
    const int t0 = least_tiles(M, terms, row_cap(a));
    for (int t = t0; t <= t0 + MX_MORE_TILES; ++t) {
      if (!cut(p, M, N, terms, a, swiglu, t)) continue;
      for (int ks = 1; ks <= 8; ++ks) {
        if (ks > 1 && (ks > KB / 4 || a * p.tt * MX_ROWS * 4 > MX_MAX_DYN - 1024)) break;
        const double ctas = (double)p.row_units * p.tiles * ks, slots = slots_of[ks], block = (double)p.block_bytes;
        const double on_sm = ctas > slots && tmem_columns(a, p.nb) <= 256 ? 2.0 : 1.0;  // CTAs of an SM (see launch_for)
        const double ring = fmin(floor((MX_MAX_DYN / on_sm - 1024.0) / (a * (MX_A_BYTES + MX_SF_BYTES) + block)), MX_MAX_STAGES);
        const double stage = fmax(fmax(on_sm * (a * MX_PACK_BYTES + block) / 53.0, 3300.0 / fmax(ring, 2.0)),
                                  fmax(on_sm * fmax(a == 2 ? 700.0 : 450.0, 2.0 * a * p.nb),
                                       a * (double)MX_PACK_BYTES * fmin(ctas, on_sm * slots) / p.tiles / 3300.0));
        const double cta = (double)((KB + ks - 1) / ks) * stage + 5000.0 + a * p.tt * 30.0 + (ks > 1 ? 1500.0 + a * p.tt * 40.0 : a == 2 ? 1500.0 : 0.0);
        const double cost = ceil(ctas / (on_sm * slots)) * cta;
        if (least == 0.0 || cost < least) {
          least = cost;
          best = p;
          best.ksplit = ks;
        }
      }
    }
  }
  return best;
}

// ---------------------------------------------------------------------------------------------
// activations to terms: four lanes take a block of 32 k of one token, eight values each
// ---------------------------------------------------------------------------------------------
// The largest magnitude of a block's 32 values, as fp32 bits, from the 16-bit values of its four lanes, two at a time.
__device__ __forceinline__ uint32_t block_top(uint4 raw, bool f16) {
  constexpr uint32_t ABS = 0x7fff7fffu;
  uint32_t m = __vmaxu2(__vmaxu2(raw.x & ABS, raw.y & ABS), __vmaxu2(raw.z & ABS, raw.w & ABS));
  m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
  m = max(m & 0xffffu, m >> 16);
  return f16 ? __float_as_uint(__half2float(__ushort_as_half((unsigned short)m))) : m << 16;
}
// U chunks at a time, their blocks' largest magnitudes in `tops`; calls put(chunk, term, codes, scale).  Every lane of the warp calls this.  Issue
// slots count where there are many (108 instructions a chunk; with fp32 maxima and a loop over the terms 205: 128 rows of two terms 17.3 instead of 16.6 us
// in all), so the power of two is formed from the bits: 0x1fffff more carries into the exponent exactly where the mantissa passes 1.75 (448 = 1.75 * 2^8).
template <int U, typename Put>
__device__ __forceinline__ void make_terms(float (&v)[U][8], const uint32_t (&tops)[U], int terms, Put put) {
  bool bad[U];
#pragma unroll
  for (int j = 0; j < U; ++j) bad[j] = tops[j] >= 0x7f800000u;
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    if (t >= terms) break;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      uint32_t top = tops[j];
      if (t > 0) {
        top = __float_as_uint(absmax_nan(v[j]));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      }
      const int byte = max((int)((top + 0x1fffffu) >> 23) - 8, 0);  // exponent + 127 of the least power of two p with top <= 448 p
      const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t q0 = to_e4m3x2(v[j][4 * h] * inv, v[j][4 * h + 1] * inv), q1 = to_e4m3x2(v[j][4 * h + 2] * inv, v[j][4 * h + 3] * inv);
        w[h] = __byte_perm(q0, q1, 0x5410);
        if (t + 1 < terms) {
          const float scale = __uint_as_float(byte ? (uint32_t)byte << 23 : 0x00400000u);
          const float2 f = half2_values(e4m3x2_to_half2(q0)), g = half2_values(e4m3x2_to_half2(q1));
          v[j][4 * h] = fmaf(-f.x, scale, v[j][4 * h]);  // exact: what is left has fewer bits
          v[j][4 * h + 1] = fmaf(-f.y, scale, v[j][4 * h + 1]);
          v[j][4 * h + 2] = fmaf(-g.x, scale, v[j][4 * h + 2]);
          v[j][4 * h + 3] = fmaf(-g.y, scale, v[j][4 * h + 3]);
        }
      }
      put(j, t, make_uint2(w[0], w[1]), bad[j] ? 255 : (uint8_t)byte);  // under a NaN scale the codes do not matter
    }
  }
}
// Where chunk c (eight k) of operand row r goes in a block of terms, and the scale of its 32 k.
__device__ __forceinline__ uint32_t term_at(int r, int c) { return (uint32_t)(r * MX_BK + (((c >> 1) ^ (r & 7)) << 4) + 8 * (c & 1)); }
__device__ __forceinline__ uint32_t term_scale_at(int nb, int r, int c) {
  return (uint32_t)(nb * MX_BK + (r >> 7) * MX_SF_BYTES + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (c >> 2));
}

constexpr int TERM_THREADS = 128;
// grid (M, segments of 128 U chunks of eight values).  512 x 17920, one term: 8 us of the product's 51 (9.6 on cold caches: read 18 MB, write 9).
template <int TYPE, int U, int TERMS>
__global__ void __launch_bounds__(TERM_THREADS) mx_terms_kernel(const uint8_t* __restrict__ a, long long stride, int K8, int KB, int tt,
                                                                int nb, size_t block_bytes, uint8_t* __restrict__ out) {
  const int m = blockIdx.x, c0 = blockIdx.y * (TERM_THREADS * U) + threadIdx.x;
  uint4 raw[U];
  pdl_wait();
  pdl_trigger();
  const uint4* src = reinterpret_cast<const uint4*>(a + m * stride * 2) + c0;
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = c0 + u * TERM_THREADS < K8 ? src[u * TERM_THREADS] : make_uint4(0u, 0u, 0u, 0u);
  float v[U][8];
  uint32_t tops[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    unpack8(raw[u], TYPE == HYP_TYPE_F16, v[u]);
    tops[u] = block_top(raw[u], TYPE == HYP_TYPE_F16);
  }
  const int tile = m / tt, row = m - tile * tt;
  uint8_t* blk0 = out + (size_t)tile * KB * block_bytes;
  make_terms<U>(v, tops, TERMS, [&](int u, int t, uint2 codes, uint8_t scale) {
    const int c = c0 + u * TERM_THREADS;
    if (c >= 16 * KB) return;
    const int r = t * tt + row;
    uint8_t* blk = blk0 + (size_t)(c >> 4) * block_bytes;
    *reinterpret_cast<uint2*>(blk + term_at(r, c & 15)) = codes;
    if ((c & 3) == 0) blk[term_scale_at(nb, r, c & 15)] = scale;
  });
}

// ---------------------------------------------------------------------------------------------
// product
// ---------------------------------------------------------------------------------------------
// Bytes from one block of a CTA's own terms to the next (operands start on 1024 bytes).
__host__ __device__ __forceinline__ uint32_t own_place(size_t block_bytes) { return ((uint32_t)block_bytes + 1023u) & ~1023u; }

struct MxArgs {
  const uint8_t* packed;  // weights, for the scales
  const uint8_t* terms;   // activations in terms; OWN: as they are
  const uint8_t* act;
  long long act_stride;
  size_t block_bytes;
  int M, N, K8, KB, ldo;
  int tiles, row_units, token_tiles, tt, nb, n_terms;
  int stages, stage_bytes, ksplit, tmem_cols;
  uint32_t idesc;
  bool f16, vec;          // vec: four results at a time may be stored
  void* out;
  int* err;
};

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// The issuing threads run alone, at about five cycles an instruction: what they do for a stage is kept to additions.
template <bool ACC>
__device__ __forceinline__ void mx_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb) {
  if (ACC)
    asm volatile("tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], 1;"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb) : "memory");
  else
    asm volatile("tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], 0;"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb) : "memory");
}
// 512 bytes of scales (32 lines of 16 bytes) to four columns of tensor memory, the same in every quarter of the lanes.
__device__ __forceinline__ void mx_copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// Their shared-memory descriptor: eight lines are 128 bytes, no swizzle.
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// without the wait: several loads share one
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t local_addr, uint32_t rank) {
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local_addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
  return v;
}
__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + __expf(-g)) * u; }

// Four results of token m, columns n .. n + 3.
template <int EPI>
__device__ __forceinline__ void mx_store(const MxArgs& p, int m, int n, float4 y) {
  const size_t o = (size_t)m * p.ldo + n;
  const float e[4] = {y.x, y.y, y.z, y.w};
  if (EPI == EPI_STORE_BF16 || EPI == EPI_SWIGLU_BF16) {
    uint16_t* to = reinterpret_cast<uint16_t*>(p.out) + o;
    const uint32_t lo = p.f16 ? half2_sat(y.x, y.y) : pack_bf16(y.x, y.y), hi = p.f16 ? half2_sat(y.z, y.w) : pack_bf16(y.z, y.w);
    if (p.vec && n + 3 < p.N) {
      *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
    } else {
      const uint16_t h[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < p.N) to[i] = h[i];
    }
  } else {
    float* to = reinterpret_cast<float*>(p.out) + o;
    if (p.vec && n + 3 < p.N) {
      if (EPI == EPI_RESID_F32) {
        const float4 x = *reinterpret_cast<const float4*>(to);
        y.x += x.x; y.y += x.y; y.z += x.z; y.w += x.w;
      }
      *reinterpret_cast<float4*>(to) = y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < p.N) to[i] = EPI == EPI_RESID_F32 ? to[i] + e[i] : e[i];
    }
  }
}

// The terms of a CTA's tokens m0 .. m0 + mt - 1 for its n_kb blocks of 128 k; 32 MX_EPI_WARPS threads, a chunk of eight k at a time, the next
// one's values on their way.
__device__ __forceinline__ void own_terms(const MxArgs& p, uint8_t* to, int kb0, int n_kb, int m0, int mt, int t) {
  constexpr int STEP = 32 * MX_EPI_WARPS;
  const int all = 16 * mt * n_kb;  // blocks of four lanes; rows behind the last token hold anything, their columns are not read
  auto fetch = [&](int i) {
    const int c = i & 15, row = (i >> 4) % mt, ck = 16 * (kb0 + (i >> 4) / mt) + c;
    return i < all && ck < p.K8 ? *reinterpret_cast<const uint4*>(p.act + ((long long)(m0 + row) * p.act_stride + 8ll * ck) * 2) : make_uint4(0, 0, 0, 0);
  };
  uint4 raw = fetch(t);
  for (int i = t; (i & ~31) < all; i += STEP) {  // the warp's lanes stay together
    float v[1][8];
    unpack8(raw, p.f16, v[0]);
    const uint32_t tops[1] = {block_top(raw, p.f16)};
    raw = fetch(i + STEP);
    const int c = i & 15, row = (i >> 4) % mt;
    uint8_t* blk = to + (i >> 4) / mt * own_place(p.block_bytes);
    make_terms<1>(v, tops, p.n_terms, [&](int, int term, uint2 codes, uint8_t scale) {
      if (i >= all) return;
      const int r = term * p.tt + row;
      *reinterpret_cast<uint2*>(blk + term_at(r, c)) = codes;
      if ((c & 3) == 0) blk[term_scale_at(p.nb, r, c)] = scale;
    });
  }
}

// A_TILES 2 without SwiGLU: two neighbouring row tiles, so that the terms' way from the L2 serves twice the products.
// OWN: a CTA's share of K is so small that it makes its terms itself, in a place of their own beside the ring: a launch less.
template <int EPI, int A_TILES, bool OWN>
__global__ void __launch_bounds__(MX_THREADS, 1)
gemm_mx4_kernel(const __grid_constant__ CUtensorMap tm_w, const MxArgs p) {
  constexpr bool SWIGLU = EPI == EPI_SWIGLU_BF16, DUAL = A_TILES == 2;
  static_assert(!SWIGLU || DUAL, "gate and up");
  extern __shared__ uint8_t mx_smem[];
  __shared__ uint64_t bars[2 * MX_MAX_STAGES + 2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  const uint32_t base = (smem_u32(mx_smem) + 1023u) & ~1023u;
  uint8_t* ring = mx_smem + (base - smem_u32(mx_smem));
  float* sums = reinterpret_cast<float*>(ring);  // behind the main loop: [accumulator][token][128 rows]
  const int S = p.stages;
  // a stage: weights, terms with their scales (OWN: behind the ring), weight scales
  const uint32_t b_off = A_TILES * MX_A_BYTES, sfa_off = b_off + (OWN ? 0u : (uint32_t)p.block_bytes);
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (MX_MAX_STAGES + s); };
  const uint32_t tfull_bar = bar0 + 8u * (2 * MX_MAX_STAGES), terms_bar = tfull_bar + 8;
  volatile int* abort_flag = &abort_word;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x % (unsigned)p.ksplit);
  const int unit = (int)(blockIdx.x / (unsigned)p.ksplit);
  const int tile = unit / p.token_tiles * (DUAL && !SWIGLU ? 2 : 1), tok = unit % p.token_tiles;  // the token tiles of a weight tile run side by side
  const int kb0 = (int)((long long)p.KB * rank / p.ksplit), kb1 = (int)((long long)p.KB * (rank + 1) / p.ksplit);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), OWN ? 2 : 3);  // codes, weight scales, terms
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(tfull_bar, 1);
    mbar_init(terms_bar, MX_EPI_WARPS);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const uint8_t* terms = OWN ? nullptr : p.terms + ((size_t)tok * p.KB + kb0) * p.block_bytes;
  // What a producing thread adds to the ring: `src` steps by `step` from k-block to k-block, `dst` and `bar` from stage to stage.
  const int n_kb = kb1 - kb0, n_first = min(S, n_kb);
  const int line0 = (int)(((long long)tile * p.KB + kb0) * (MX_PACK_BYTES / 64)), up_lines = (SWIGLU ? p.tiles : tile + 1 < p.tiles ? 1 : 0) * p.KB * (MX_PACK_BYTES / 64);  // to the second row tile (behind the last: itself)
  auto load_w = [&](int line, uint32_t dst, uint32_t bar) {
    mbar_expect_tx(bar, A_TILES * MX_CODE_BYTES);  // a box counts by what it reads
    tma_load_2d(dst, &tm_w, 0, line, bar);
    if (DUAL) tma_load_2d(dst + MX_A_BYTES, &tm_w, 0, line + up_lines, bar);
  };
  auto load_s = [&](const uint8_t* src, uint32_t dst, uint32_t bar) {
    mbar_expect_tx(bar, A_TILES * MX_SF_BYTES);
    bulk_load(dst + sfa_off, src, MX_SF_BYTES, bar);
    if (DUAL) bulk_load(dst + sfa_off + MX_SF_BYTES, src + 64ll * up_lines, MX_SF_BYTES, bar);
  };
  const uint32_t term_bytes = (uint32_t)p.block_bytes;
  auto load_t = [&](const uint8_t* src, uint32_t dst, uint32_t bar) {
    mbar_expect_tx(bar, term_bytes);
    bulk_load(dst + b_off, src, term_bytes, bar);
  };
  // A whole warp walks the CTA's stages from `from` (at most S) on, one lane issues.
  auto produce = [&](auto load, auto src, auto step, int from) {
    src += step * from;
    int stage = from == S ? 0 : from;
    uint32_t phase = from == S ? 0u : 1u;  // of the "empty" phase waited for; the first pass over the ring waits for nothing
    uint32_t dst = base + stage * p.stage_bytes;
    for (int i = from; i < n_kb; ++i) {
      if (i >= S && !__all_sync(0xffffffffu, mbar_wait(empty_bar(stage), phase, abort_flag))) {
        if (lane == 0) {
          *abort_flag = 1;
          atomicCAS(p.err, 0, 31);
        }
        return false;
      }
      if (elect_one()) load(src, dst, full_bar(stage));
      __syncwarp();
      src += step;
      dst += p.stage_bytes;
      if (++stage == S) {
        stage = 0;
        phase ^= 1u;
        dst = base;
      }
    }
    return true;
  };
  auto first_w = [&] {
    if (threadIdx.x == 0)
      for (int i = 0; i < n_first; ++i) load_w(line0 + i * (MX_PACK_BYTES / 64), base + i * p.stage_bytes, full_bar(i));
  };
  __syncwarp();
  // The kernel before this one is the one that made the terms (its own wait has seen the end of whatever wrote the weights): the first weights go
  // out before the wait.  OWN: it may be any kernel.
  if (!OWN) first_w();
  __syncwarp();
  pdl_wait();
  if (OWN) first_w();
  __syncwarp();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(p.tmem_cols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_trigger();

  const int m0 = tok * p.tt, mt = min(p.tt, p.M - m0);
  if (warp == 0) {
    if (OWN) {
      // scales along with the codes: the other warps make terms
      if (elect_one())
        for (int i = 0; i < n_first; ++i) load_s(p.packed + 64ll * line0 + MX_CODE_BYTES + (size_t)i * MX_PACK_BYTES, base + i * p.stage_bytes, full_bar(i));
      __syncwarp();
      produce([&](int line, uint32_t dst, uint32_t bar) {
        load_w(line, dst, bar);
        load_s(p.packed + 64ll * line + MX_CODE_BYTES, dst, bar);
      }, line0, MX_PACK_BYTES / 64, n_first);
    } else {
      produce(load_w, line0, MX_PACK_BYTES / 64, n_first);
    }
  } else if (warp == 1) {
    // The whole warp walks the loop and one lane issues: so the operands stay in uniform registers (a lane on its own moves each of them there
    // for every instruction: 800 cycles a stage).
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0), ub = __shfl_sync(0xffffffffu, base, 0);
    const uint32_t sfa = tm + (uint32_t)(A_TILES * p.nb), sfb = sfa + 4 * A_TILES, step = (uint32_t)p.stage_bytes >> 4;
    const uint32_t ut = OWN ? ub + S * p.stage_bytes : ub + b_off, t_step = OWN ? own_place(p.block_bytes) >> 4 : step;
    const uint64_t da0 = smem_desc(ub), db0 = smem_desc(ut), dsa0 = scales_desc(ub + sfa_off), dsb0 = scales_desc(ut + p.nb * MX_BK);
    const uint32_t id0 = p.idesc, id1 = id0 | 1u << 29 | 1u << 4, id2 = id0 | 2u << 29 | 2u << 4, id3 = id0 | 3u << 29 | 3u << 4;  // byte of a scale word
    const uint32_t acc2 = tm + (uint32_t)p.nb;
    const bool two_sf = p.nb > MX_ROWS;
    int stage = 0;
    uint32_t phase = 0, at = 0, t_at = 0;  // the places of the stage and of its terms, in descriptor units
    bool ok = !OWN || __all_sync(0xffffffffu, mbar_wait(terms_bar, 0, abort_flag));
    for (int i = 0; i < n_kb && ok; ++i) {
      ok = __all_sync(0xffffffffu, mbar_wait(full_bar(stage), phase, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const uint64_t da = da0 + at, db = db0 + t_at;
      if (elect_one()) {
        // scales of this stage: in order behind the MMAs that still read the ones before
        mx_copy_scales(sfa, dsa0 + at);
        if (DUAL) mx_copy_scales(sfa + 4, dsa0 + at + MX_SF_BYTES / 16);
        mx_copy_scales(sfb, dsb0 + t_at);
        if (two_sf) mx_copy_scales(sfb + 4, dsb0 + t_at + MX_SF_BYTES / 16);
        if (i == 0) {
          mx_mma<false>(tm, da, db, id0, sfa, sfb);
          if (DUAL) mx_mma<false>(acc2, da + MX_A_BYTES / 16, db, id0, sfa + 4, sfb);
        } else {
          mx_mma<true>(tm, da, db, id0, sfa, sfb);
          if (DUAL) mx_mma<true>(acc2, da + MX_A_BYTES / 16, db, id0, sfa + 4, sfb);
        }
        mx_mma<true>(tm, da + 2, db + 2, id1, sfa, sfb);
        if (DUAL) mx_mma<true>(acc2, da + MX_A_BYTES / 16 + 2, db + 2, id1, sfa + 4, sfb);
        mx_mma<true>(tm, da + 4, db + 4, id2, sfa, sfb);
        if (DUAL) mx_mma<true>(acc2, da + MX_A_BYTES / 16 + 4, db + 4, id2, sfa + 4, sfb);
        mx_mma<true>(tm, da + 6, db + 6, id3, sfa, sfb);
        if (DUAL) mx_mma<true>(acc2, da + MX_A_BYTES / 16 + 6, db + 6, id3, sfa + 4, sfb);
        tc_commit(empty_bar(stage));
        if (i == n_kb - 1) tc_commit(tfull_bar);
      }
      __syncwarp();
      at += step;
      t_at += t_step;
      if (++stage == S) {
        stage = 0;
        phase ^= 1u;
        at = 0;
        if (!OWN) t_at = 0;
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicCAS(p.err, 0, 32);
    }
  } else {
    bool ok = true;
    // two of these warps issue copies first
    if (!OWN && warp == 2) ok = produce(load_s, p.packed + 64ll * line0 + MX_CODE_BYTES, MX_PACK_BYTES, 0);
    if (!OWN && warp == 3) ok = produce(load_t, terms, term_bytes, 0);
    if (OWN) own_terms(p, ring + S * p.stage_bytes, kb0, n_kb, m0, mt, threadIdx.x - 64);
    if (OWN) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(terms_bar);
    }
    ok = mbar_wait(tfull_bar, 0, abort_flag) && ok;
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicCAS(p.err, 0, 33);
    }
  }
  // Results by way of shared memory: the accumulators with their terms added up (lane = weight row), then a warp to a token, four columns a
  // lane, 512 bytes of a row at a time.  Shares of K leave all they have there and finish a part of the tokens each.
  __syncthreads();
  tc_fence_after();
  auto leave = [&](int h, float* to, bool both) {  // accumulator h, or SwiGLU of both
    const int row = 32 * (warp & 3) + lane;
    const uint32_t t0 = tmem_base + ((uint32_t)(32 * (warp & 3)) << 16) + h * p.nb;
    constexpr int B = 2;  // groups of eight tokens in flight
    for (int c = 8 * B * ((warp - 2) / 4); c < mt; c += 8 * B * (MX_EPI_WARPS / 4)) {  // two warps share a quarter of the lanes
      float v[B][8], u[B][8];
      for (int t = 0; t < p.n_terms; ++t) {
        float w[B][8], x[B][8];
#pragma unroll
        for (int i = 0; i < B; ++i) {
          if (c + 8 * i < p.tt) {
            tmem_ld8(t0 + t * p.tt + c + 8 * i, w[i]);
            if (SWIGLU && both) tmem_ld8(t0 + p.nb + t * p.tt + c + 8 * i, x[i]);
          }
        }
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[i][j] = t == 0 ? w[i][j] : v[i][j] + w[i][j];
            if (SWIGLU) u[i][j] = t == 0 ? x[i][j] : u[i][j] + x[i][j];
          }
      }
#pragma unroll
      for (int i = 0; i < B; ++i) {
        if (c + 8 * i < p.tt) {
#pragma unroll
          for (int j = 0; j < 8; ++j) to[(c + 8 * i + j) * MX_ROWS + row] = SWIGLU && both ? swiglu(v[i][j], u[i][j]) : v[i][j];
        }
      }
    }
  };
  if (p.ksplit == 1) {
#pragma unroll
    for (int h = 0; h < (SWIGLU ? 1 : A_TILES); ++h) {
      if (warp >= 2 && !abort_word) leave(h, sums, true);
      __syncthreads();
      const int n = (tile + h) * MX_ROWS + 4 * lane;
      if (n < p.N && !abort_word)
        for (int m = warp; m < mt; m += MX_THREADS / 32) mx_store<EPI>(p, m0 + m, n, *reinterpret_cast<const float4*>(sums + m * MX_ROWS + 4 * lane));
      if (h + 1 < A_TILES) __syncthreads();
    }
  } else {
    if (warp >= 2 && !abort_word) {
      leave(0, sums, false);
      if (DUAL) leave(1, sums + p.tt * MX_ROWS, false);
    }
    __syncthreads();
    cluster_barrier();
    const int n = tile * MX_ROWS + 4 * lane;
    if (n < p.N && !abort_word) {
      const uint32_t at = smem_u32(sums) + 16u * lane;
      for (int m = rank + p.ksplit * warp; m < mt; m += p.ksplit * (MX_THREADS / 32)) {
        float4 v[8], u[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          v[r] = u[r] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (r < p.ksplit) {
            v[r] = ld_cluster_v4(at + 512u * m, r);
            if (DUAL) u[r] = ld_cluster_v4(at + 512u * (p.tt + m), r);
          }
        }
        float4 y = v[0], z = u[0];
#pragma unroll
        for (int r = 1; r < 8; ++r) {
          if (r < p.ksplit) {
            y.x += v[r].x; y.y += v[r].y; y.z += v[r].z; y.w += v[r].w;
            z.x += u[r].x; z.y += u[r].y; z.z += u[r].z; z.w += u[r].w;
          }
        }
        if (SWIGLU) y = make_float4(swiglu(y.x, z.x), swiglu(y.y, z.y), swiglu(y.z, z.z), swiglu(y.w, z.w));
        mx_store<EPI>(p, m0 + m, n, y);
        if (DUAL && !SWIGLU && n + MX_ROWS < p.N) mx_store<EPI>(p, m0 + m, n + MX_ROWS, z);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && abort_word)  // given up: let the copies in flight land
    for (int s = 0; s < S; ++s) mbar_wait(full_bar(s), 0, nullptr, 50000000), mbar_wait(full_bar(s), 1, nullptr, 50000000);
  if (p.ksplit > 1) cluster_barrier();  // nobody leaves while a peer may still read its sums
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols));
  }
}

// What a launch needs beside the cut.
struct Launch {
  Plan plan;
  long long ctas;
  int tmem_cols, stages, stage_bytes, smem;
  bool own, many;  // the CTAs make their terms; else the terms' launch takes two chunks a thread
};

template <int EPI, int A_TILES, bool OWN>
int launch_own(const CUtensorMap& map, const MxArgs& p, const Launch& l, cudaStream_t st) {
  const int rc = allow_smem<gemm_mx4_kernel<EPI, A_TILES, OWN>>(MX_MAX_DYN);
  if (rc) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)l.ctas);
  cfg.blockDim = dim3(MX_THREADS);
  cfg.dynamicSmemBytes = l.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int na = 0;
  if (pdl_level() >= 2) {
    attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
  }
  if (p.ksplit > 1) {
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = (unsigned)p.ksplit;
    attr[na].val.clusterDim.y = 1;
    attr[na].val.clusterDim.z = 1;
    ++na;
  }
  cfg.attrs = attr;
  cfg.numAttrs = na;
  HYP_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_mx4_kernel<EPI, A_TILES, OWN>, map, p));
  return 1;
}

int current_device() {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 64 ? dev : 0;
}

const int* slots_by_ks() {
  static int known[64][9];
  static std::once_flag asked[64];  // a second thread's first call waits: a plan weighed by half of the table would cut K another way
  const int dev = current_device();
  std::call_once(asked[dev], [dev] {
    for (int ks = 1; ks <= 8; ++ks) {
      int n = 0;
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute attr;
      cfg.gridDim = dim3((unsigned)ks * 64);
      cfg.blockDim = dim3(MX_THREADS);
      cfg.dynamicSmemBytes = 200 * 1024;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = (unsigned)ks;
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if (ks > 1 && (allow_smem<gemm_mx4_kernel<EPI_STORE_F32, 1, false>>(MX_MAX_DYN) != HYP_OK ||
                     cudaOccupancyMaxActiveClusters(&n, gemm_mx4_kernel<EPI_STORE_F32, 1, false>, &cfg) != cudaSuccess)) {
        n = 0;
        cudaGetLastError();  // the question was refused: no error of the launch that asks
      }
      if (n < 1) n = sm_count() / ks;
      known[dev][ks] = n * ks;
    }
  });
  return known[dev];
}

template <int EPI, int A_TILES>
int launch_epi(const CUtensorMap& map, const MxArgs& p, const Launch& l, cudaStream_t st) {
  return l.own ? launch_own<EPI, A_TILES, true>(map, p, l, st) : launch_own<EPI, A_TILES, false>(map, p, l, st);
}

int launch_by_epi(int epi, const CUtensorMap& map, const MxArgs& p, const Launch& l, cudaStream_t st) {
  const bool dual = l.plan.a_tiles == 2;
  switch (epi) {
    case EPI_STORE_BF16: return dual ? launch_epi<EPI_STORE_BF16, 2>(map, p, l, st) : launch_epi<EPI_STORE_BF16, 1>(map, p, l, st);
    case EPI_RESID_F32: return dual ? launch_epi<EPI_RESID_F32, 2>(map, p, l, st) : launch_epi<EPI_RESID_F32, 1>(map, p, l, st);
    case EPI_SWIGLU_BF16: return launch_epi<EPI_SWIGLU_BF16, 2>(map, p, l, st);
    case EPI_STORE_F32: return dual ? launch_epi<EPI_STORE_F32, 2>(map, p, l, st) : launch_epi<EPI_STORE_F32, 1>(map, p, l, st);
    default: return HYP_EINVAL;
  }
}

// A program calls with a few sizes again and again, and weighing the cuts takes 1-2 us of the host.
Plan known_plan(int M, int N, int KB, int terms, bool swiglu) {
  struct Entry {
    int M, N, KB, terms, dev;
    bool swiglu;
    Plan plan;
  };
  static thread_local Entry table[16] = {};
  Entry& e = table[((unsigned)M * 31u + (unsigned)N / 16u + (unsigned)KB * 7u + (unsigned)terms) % 16u];
  const int dev = current_device();
  if (e.M != M || e.N != N || e.KB != KB || e.terms != terms || e.dev != dev || e.swiglu != swiglu)
    e = Entry{M, N, KB, terms, dev, swiglu, plan_for(M, N, KB, terms, swiglu)};
  return e.plan;
}

// 0 stages: no room (no plan asks for it)
Launch launch_for(int M, int N, int KB, int terms, bool swiglu) {
  Launch l{};
  l.plan = known_plan(M, N, KB, terms, swiglu);
  const Plan& t = l.plan;
  l.ctas = (long long)t.row_units * t.tiles * t.ksplit;
  // Up to OWN_TERMS terms a thread (of a chunk each) the CTAs make their terms themselves (one token, 512 x 256 of three: 3.6 instead of 4.4 us, 7680 x 5120
  // 8.9, 9.3; three tokens, 1000 x 2000 of two: 4.8, 5.7); with more, a launch of their own is faster (two tokens, 7680 x 5120 of three: 9.3
  // instead of 9.6).
  const int share = (KB + t.ksplit - 1) / t.ksplit, own_threads = 32 * MX_EPI_WARPS;
  l.own = t.tiles == 1 && (16ll * M * share + own_threads - 1) / own_threads * terms <= OWN_TERMS &&
          share * (long long)own_place(t.block_bytes) <= OWN_BYTES && (long long)t.row_units * t.ksplit <= sm_count();
  l.many = !l.own && 16ll * M * KB > 1 << 18;  // two chunks a thread: half the CTAs (512 x 5120 x 17920 51 us, one chunk 55, four 51; 128 rows 28, 29, 31)
  l.tmem_cols = tmem_columns(t.a_tiles, t.nb);
  l.stage_bytes = (t.a_tiles * (MX_A_BYTES + MX_SF_BYTES) + (l.own ? 0 : (int)t.block_bytes) + 1023) / 1024 * 1024;
  const int own_bytes = l.own ? share * (int)own_place(t.block_bytes) : 0;
  const int sum_bytes = (t.ksplit > 1 ? t.a_tiles : 1) * t.tt * MX_ROWS * 4;
  // two CTAs to an SM where there are more than SMs and tensor memory has room for both
  const int budget = l.ctas > sm_count() && l.tmem_cols <= 256 ? 112 * 1024 : MX_MAX_DYN;
  l.stages = (budget - 1024 - own_bytes) / l.stage_bytes;
  if (l.stages > MX_MAX_STAGES) l.stages = MX_MAX_STAGES;
  if (l.stages < 2) l.stages = 2;
  const int ring = l.stages * l.stage_bytes + own_bytes;
  l.smem = (ring > sum_bytes ? ring : sum_bytes) + 1024;  // the sums reuse the ring
  if (l.smem > MX_MAX_DYN) l.stages = 0;
  // never more CTAs on an SM than tensor memory holds: one that waits for it would hold up its cluster
  const int least = 228 * 1024 / (512 / l.tmem_cols + 1);
  if (l.smem < least) l.smem = least;
  return l;
}

}  // namespace

size_t mx4_scratch_bytes(int M, int K, int terms) {
  // whatever the plan: t tiles of at most M / t + 8 tokens, their operand rows filled up by 15 at most
  const long long t = least_tiles(M, terms, 240) + MX_MORE_TILES, rows = (long long)M * terms + t * (8 * terms + 15);
  return (size_t)mx_kb(K) * (rows * MX_BK + (rows / MX_ROWS + t) * MX_SF_BYTES);
}

void mx4_plan(int M, int N, int K, int terms, bool swiglu, int32_t (&plan)[8]) {
  const Launch l = launch_for(M, N, mx_kb(K), terms, swiglu);
  const int32_t v[8] = {l.plan.a_tiles, l.plan.tiles, l.plan.ksplit, (int32_t)(l.ctas > 0x7fffffffll ? 0x7fffffff : l.ctas), l.stages,
                        228 * 1024 / (l.smem + 1024), l.own, l.own ? 0 : l.many ? 2 : 1};
  for (int i = 0; i < 8; ++i) plan[i] = v[i];
}

int launch_gemm_mx4(const void* a, int a_type, long long a_stride, const uint8_t* packed, int M, int N, int K, int terms, int epi,
                    void* out, int ldo, uint8_t* scratch, cudaStream_t st) {
  const bool swiglu = epi == EPI_SWIGLU_BF16, wide = epi == EPI_STORE_F32 || epi == EPI_RESID_F32;
  const Launch l = launch_for(M, N, mx_kb(K), terms, swiglu);
  const Plan& t = l.plan;
  if (l.stages == 0) return HYP_EINVAL;
  MxArgs p{};
  p.packed = packed; p.terms = scratch; p.block_bytes = t.block_bytes;
  p.M = M; p.N = N; p.KB = mx_kb(K); p.ldo = ldo;
  p.tiles = mx_row_tiles(N); p.row_units = t.row_units; p.token_tiles = t.tiles; p.tt = t.tt; p.nb = t.nb; p.n_terms = terms;
  p.ksplit = t.ksplit; p.stages = l.stages; p.stage_bytes = l.stage_bytes; p.tmem_cols = l.tmem_cols;
  p.f16 = a_type == HYP_TYPE_F16; p.out = out; p.err = tc_err_flag_ptr();
  p.vec = ldo % 4 == 0 && ((uintptr_t)out & (wide ? 15 : 7)) == 0;
  p.idesc = (5u << 7) | (0u << 10) | ((uint32_t)(t.nb >> 3) << 17) | (1u << 23) | ((uint32_t)(MX_ROWS >> 4) << 24);  // E2M1 x E4M3, power-of-two scales
  if (l.ctas > 0x7fffffffll) return HYP_ECAPACITY;
  CUtensorMap map;
  int rc = tc_make_mx4_map(&map, packed, (long long)(swiglu ? 2 : 1) * p.tiles * p.KB * (MX_PACK_BYTES / 64));
  if (rc) return rc;
  if (l.own) {
    p.act = (const uint8_t*)a; p.act_stride = a_stride; p.K8 = K / 8;
    return launch_by_epi(epi, map, p, l, st);
  }
  const long long chunks = 16ll * p.KB;  // of a row: its segments fit the grid (K is at most 2^25)
  const long long segments = (chunks + TERM_THREADS * (l.many ? 2 : 1) - 1) / (TERM_THREADS * (l.many ? 2 : 1));
  auto go = [&](auto kernel) {
    return launch_pdl<2>(kernel, dim3((unsigned)M, (unsigned)segments), dim3(TERM_THREADS), (size_t)0, st, (const uint8_t*)a, a_stride, K / 8, p.KB,
                         t.tt, t.nb, t.block_bytes, scratch);
  };
  auto by_chunks = [&](auto two, auto one) { return l.many ? go(two) : go(one); };
#define HYP_F(T, N) \
  if (a_type == T && terms == N) HYP_CUDA_TRY(by_chunks(mx_terms_kernel<T, 2, N>, mx_terms_kernel<T, 1, N>));
  HYP_F(HYP_TYPE_F16, 1) HYP_F(HYP_TYPE_F16, 2) HYP_F(HYP_TYPE_F16, 3) HYP_F(HYP_TYPE_BF16, 1) HYP_F(HYP_TYPE_BF16, 2) HYP_F(HYP_TYPE_BF16, 3)
#undef HYP_F
  rc = launch_by_epi(epi, map, p, l, st);
  return rc < 0 ? rc : rc + 1;
}

}  // namespace hyp
