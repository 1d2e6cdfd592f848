// Product of activations and microscaled 4-bit weights: out[m, n] (+)= sum_k a[m, k] * w[n, k].
//
// The tensor cores multiply E2M1 by E4M3 operands, each under a power of two per row and block of 32 k
// (tcgen05.mma.kind::mxf8f6f4.block_scale), with fp32 sums.  So nothing of the weights is converted by the CUDA cores: the copy
// engine spreads the packed codes to the operand's byte containers on their way to shared memory, the scales go from there to
// tensor memory, and a CTA keeps up with HBM.  The activations, 16-bit values, become one to three E4M3 terms: the first is a
// rounded to four bits under its block's power of two, the next is what is left, under a power of two of its own.  Two terms hold
// a bf16 value, three an fp16 value (what they leave is below 2^-25 of the block's largest).  The terms of a token are more columns of the same operand (they share the
// weights' pass through shared memory) and are added in the epilogue.
//
// A CTA owns 128 weight rows (the M operand; SwiGLU: gate rows and the matching up rows, two accumulators) and a tile of tokens (the
// N operand, terms x tokens columns, at most 256).  Where there are few such tiles K is split over a cluster of up to eight CTAs:
// each leaves its sums in shared memory, and every one of them finishes a share of the tokens, adding the others' in rank order
// through distributed shared memory: deterministic.
//   warp 0     one lane fills the ring: weight codes (a TMA box), weight scales, terms with their scales (bulk copies);
//   warp 1     one lane copies the scales to tensor memory and issues the MMAs;
//   warps 2-5  epilogue, lane = weight row.
// Every mbarrier wait is bounded; the cluster barriers are reached by every thread of every CTA.
#include <cuda.h>

#include "cache_ops.cuh"
#include "gemm_tc.cuh"
#include "mx4.cuh"
#include "tcgen05.cuh"

namespace hyp {

namespace {

constexpr int MX_THREADS = 192, MX_MAX_STAGES = 12, MX_A_BYTES = MX_ROWS * MX_BK;

// How M tokens are cut: tiles of `tt` tokens, `nb` operand rows (terms x tokens, filled up to a multiple of 16).  `cap`: most rows.
struct TokenTiles {
  int tiles, tt, nb, sf_bytes;
  size_t block_bytes;  // terms of one (token tile, 128 k) with their scales
};
TokenTiles token_tiles(int M, int terms, int cap) {
  TokenTiles t;
  const int most = cap / terms / 8 * 8;
  t.tiles = (M + most - 1) / most;
  t.tt = ((M + t.tiles - 1) / t.tiles + 7) / 8 * 8;
  t.tiles = (M + t.tt - 1) / t.tt;
  t.nb = (t.tt * terms + 15) / 16 * 16;
  t.sf_bytes = (t.nb + MX_ROWS - 1) / MX_ROWS * MX_SF_BYTES;
  t.block_bytes = (size_t)t.nb * MX_BK + t.sf_bytes;
  return t;
}
// SwiGLU keeps two accumulators beside the scales in 512 columns of tensor memory.
int row_cap(int epi) { return epi == EPI_SWIGLU_BF16 ? 240 : 256; }

// ---------------------------------------------------------------------------------------------
// activations to terms: four threads take a block of 32 k of one token, eight values each
// ---------------------------------------------------------------------------------------------
constexpr int TERM_THREADS = 128;
// grid (M, segments of 128 chunks of eight values)
template <int TYPE>
__global__ void __launch_bounds__(TERM_THREADS) mx_terms_kernel(const uint8_t* __restrict__ a, long long stride, int M, int K8, int KB, int terms,
                                                                int tt, int nb, size_t block_bytes, uint8_t* __restrict__ out) {
  const int m = blockIdx.x, c = blockIdx.y * TERM_THREADS + threadIdx.x;
  const bool row_in = c < 16 * KB;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  pdl_wait();
  pdl_trigger();
  if (c < K8) load8<TYPE>(a + (m * stride + 8 * c) * 2, v);
  const int kb = c >> 4, chunk = (c & 15) >> 1;  // 16-byte chunk of the 128-byte operand row
  uint8_t* blk = out + ((size_t)(m / tt) * KB + kb) * block_bytes;
  bool bad = false;
  for (int t = 0; t < terms; ++t) {
    uint32_t top = absmax_bits(v);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    bad = bad || top >= 0x7f800000u;
    const int e = bad ? 0 : e4m3_exponent(top);
    const float inv = pow2(-e), scale = pow2(e);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t q = bad ? 0u : to_e4m3x2(v[2 * p] * inv, v[2 * p + 1] * inv);
      w[p >> 1] |= q << (16 * (p & 1));
      const float2 f = half2_values(e4m3x2_to_half2(q));
      v[2 * p] -= f.x * scale;
      v[2 * p + 1] -= f.y * scale;
    }
    if (row_in) {
      const int r = t * tt + m % tt;
      *reinterpret_cast<uint2*>(blk + r * MX_BK + ((chunk ^ (r & 7)) << 4) + 8 * (c & 1)) = make_uint2(w[0], w[1]);
      if ((c & 3) == 0)
        blk[nb * MX_BK + (r >> 7) * MX_SF_BYTES + (r & 31) * 16 + ((r >> 5) & 3) * 4 + ((c >> 2) & 3)] = bad ? 255 : (uint8_t)(e + 127);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// product
// ---------------------------------------------------------------------------------------------
struct MxArgs {
  const uint8_t* packed;  // weights, for the scales
  const uint8_t* terms;   // activations
  size_t block_bytes;
  int M, N, KB, ldo;
  int tiles, token_tiles, tt, nb, n_terms, sf_bytes;
  int stages, stage_bytes, ksplit, tmem_cols;
  uint32_t idesc;
  bool f16;
  void* out;
  int* err;
};

__device__ __forceinline__ void mx_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc)
      : "memory");
}
// 512 bytes of scales (32 lines of 16 bytes) to four columns of tensor memory, the same in every quarter of the lanes.
__device__ __forceinline__ void mx_copy_scales(uint32_t tmem, uint32_t smem) {
  uint64_t d = (uint64_t)((smem & 0x3FFFFu) >> 4);
  d |= (uint64_t)1 << 16;           // not used: one 16-byte column
  d |= (uint64_t)(128 >> 4) << 32;  // eight lines on
  d |= (uint64_t)1 << 46;
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(d) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

template <int EPI>
__device__ __forceinline__ void mx_store(const MxArgs& p, int m, int n, float a, float b) {
  const size_t o = (size_t)m * p.ldo + n;
  if (EPI == EPI_STORE_BF16 || EPI == EPI_SWIGLU_BF16) {
    const float y = EPI == EPI_SWIGLU_BF16 ? a / (1.f + __expf(-a)) * b : a;
    if (p.f16)
      reinterpret_cast<__half*>(p.out)[o] = __float2half_rn(y != y ? y : fminf(fmaxf(y, -65504.f), 65504.f));
    else
      reinterpret_cast<__nv_bfloat16*>(p.out)[o] = __float2bfloat16_rn(y);
  } else if (EPI == EPI_RESID_F32) {
    reinterpret_cast<float*>(p.out)[o] += a;
  } else {
    reinterpret_cast<float*>(p.out)[o] = a;
  }
}

template <int EPI>
__global__ void __launch_bounds__(MX_THREADS)
gemm_mx4_kernel(const __grid_constant__ CUtensorMap tm_w, const MxArgs p) {
  constexpr bool SWIGLU = EPI == EPI_SWIGLU_BF16;
  constexpr int A_TILES = SWIGLU ? 2 : 1;
  extern __shared__ uint8_t mx_smem[];
  __shared__ uint64_t bars[2 * MX_MAX_STAGES + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  const uint32_t base = (smem_u32(mx_smem) + 1023u) & ~1023u;
  float* dump = reinterpret_cast<float*>(mx_smem + (base - smem_u32(mx_smem)));  // [accumulator][token][128 rows]
  const int S = p.stages;
  const uint32_t b_off = A_TILES * MX_A_BYTES, sfa_off = b_off + (uint32_t)p.block_bytes;  // terms, their scales, weight scales
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (MX_MAX_STAGES + s); };
  const uint32_t tfull_bar = bar0 + 8u * (2 * MX_MAX_STAGES);
  volatile int* abort_flag = &abort_word;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x % (unsigned)p.ksplit);
  const int unit = (int)(blockIdx.x / (unsigned)p.ksplit);
  const int tile = unit / p.token_tiles, tok = unit % p.token_tiles;  // the token tiles of a weight tile run side by side
  const int kb0 = (int)((long long)p.KB * rank / p.ksplit), kb1 = (int)((long long)p.KB * (rank + 1) / p.ksplit);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(tfull_bar, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const uint8_t* terms = p.terms + (size_t)tok * p.KB * p.block_bytes;
  auto load_w = [&](int kb, int s) {
    const uint32_t st = base + s * p.stage_bytes;
    mbar_expect_tx(full_bar(s), (uint32_t)(A_TILES * MX_PACK_BYTES + p.block_bytes));  // the box counts by what it reads
#pragma unroll
    for (int h = 0; h < A_TILES; ++h) {
      const long long blk = (long long)(h * p.tiles + tile) * p.KB + kb;
      tma_load_2d(st + h * MX_A_BYTES, &tm_w, 0, (int)(blk * (MX_PACK_BYTES / 64)), full_bar(s));
      bulk_load(st + sfa_off + h * MX_SF_BYTES, p.packed + blk * MX_PACK_BYTES + MX_CODE_BYTES, MX_SF_BYTES, full_bar(s));
    }
  };
  auto load_t = [&](int kb, int s) {
    bulk_load(base + s * p.stage_bytes + b_off, terms + (size_t)kb * p.block_bytes, (uint32_t)p.block_bytes, full_bar(s));
  };
  const int n_first = min(S, kb1 - kb0);
  __syncwarp();
  if (threadIdx.x == 0)  // weights are no kernel's output: their first boxes go out before the wait
    for (int i = 0; i < n_first; ++i) load_w(kb0 + i, i);
  __syncwarp();
  pdl_wait();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(p.tmem_cols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_trigger();

  int issued = n_first;  // stages that the producer has filled
  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < n_first; ++i) load_t(kb0 + i, i);
      int stage = n_first == S ? 0 : n_first;
      uint32_t phase = n_first == S ? 1 : 0;
      bool ok = true;
      for (int kb = kb0 + n_first; kb < kb1; ++kb) {
        if (!mbar_wait(empty_bar(stage), phase ^ 1, abort_flag)) { ok = false; break; }
        load_w(kb, stage);
        load_t(kb, stage);
        issued = kb + 1 - kb0;
        if (++stage == S) { stage = 0; phase ^= 1; }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicCAS(p.err, 0, 31);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t t_sfa = tmem_base + (uint32_t)(A_TILES * p.nb), t_sfb = t_sfa + 4 * A_TILES;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(full_bar(stage), phase, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = base + stage * p.stage_bytes;
        // scales of this stage: in order behind the MMAs that still read the ones before
#pragma unroll
        for (int h = 0; h < A_TILES; ++h) mx_copy_scales(t_sfa + 4 * h, sa + sfa_off + h * MX_SF_BYTES);
        for (int h = 0; h < p.sf_bytes; h += MX_SF_BYTES) mx_copy_scales(t_sfb + h / (MX_SF_BYTES / 4), sa + b_off + p.nb * MX_BK + h);
        const uint64_t da = smem_desc(sa), db = smem_desc(sa + b_off);
#pragma unroll
        for (int k = 0; k < MX_BK / 32; ++k) {
          const uint32_t accum = (kb > kb0 || k > 0) ? 1u : 0u;
          const uint32_t idesc = p.idesc | (uint32_t)k << 29 | (uint32_t)k << 4;  // which byte of a scale word
          mx_mma(tmem_base, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, t_sfa, t_sfb, accum);
          if (SWIGLU)
            mx_mma(tmem_base + (uint32_t)p.nb, da + (uint64_t)(MX_A_BYTES / 16 + k * 2), db + (uint64_t)(k * 2), idesc, t_sfa + 4, t_sfb, accum);
        }
        tc_commit(empty_bar(stage));
        if (++stage == S) { stage = 0; phase ^= 1; }
      }
      if (ok) {
        tc_commit(tfull_bar);
      } else {
        *abort_flag = 1;
        atomicCAS(p.err, 0, 32);
      }
    }
  }

  // ---------------- epilogue warps ----------------
  const int row = 32 * (warp & 3) + lane;  // the quarter of the lanes that this warp may read
  const uint32_t t0 = tmem_base + ((uint32_t)(32 * (warp & 3)) << 16);
  const int n = tile * MX_ROWS + row, m0 = tok * p.tt, mt = min(p.tt, p.M - m0);
  bool acc_ok = true;
  // eight tokens' sums over the terms, `acc` = accumulator
  auto sums = [&](int acc, int c, float (&v)[8]) {
    tmem_ld8(t0 + acc * p.nb + c, v);
    for (int t = 1; t < p.n_terms; ++t) {
      float w[8];
      tmem_ld8(t0 + acc * p.nb + t * p.tt + c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
  };
  if (warp >= 2) {
    acc_ok = mbar_wait(tfull_bar, 0, abort_flag);
    tc_fence_after();
    if (!acc_ok && lane == 0) {
      *abort_flag = 1;
      atomicCAS(p.err, 0, 33);
    }
    if (acc_ok) {
      for (int c = 0; c < mt; c += 8) {
        float v[8], u[8];
        sums(0, c, v);
        if (SWIGLU) sums(1, c, u);
        if (p.ksplit > 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dump[(c + i) * MX_ROWS + row] = v[i];
            if (SWIGLU) dump[(p.tt + c + i) * MX_ROWS + row] = u[i];
          }
        } else if (n < p.N) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < mt) mx_store<EPI>(p, m0 + c + i, n, v[i], SWIGLU ? u[i] : 0.f);
        }
      }
    }
  }
  if (p.ksplit > 1) {
    __syncthreads();
    cluster_barrier();
    if (warp >= 2 && acc_ok && n < p.N) {
      const uint32_t at = smem_u32(dump) + 4u * row;
      for (int c = rank; c < mt; c += p.ksplit) {
        float v[8], u[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          v[r] = r < p.ksplit ? ld_cluster_f32(at + 4u * (c * MX_ROWS), r) : 0.f;
          u[r] = SWIGLU && r < p.ksplit ? ld_cluster_f32(at + 4u * ((p.tt + c) * MX_ROWS), r) : 0.f;
        }
        float a = v[0], b = u[0];
#pragma unroll
        for (int r = 1; r < 8; ++r) {
          if (r < p.ksplit) {
            a += v[r];
            b += u[r];
          }
        }
        mx_store<EPI>(p, m0 + c, n, a, b);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && abort_word)  // given up: let the copies in flight land
    for (int i = max(issued - S, 0); i < issued; ++i) mbar_wait(full_bar(i % S), (uint32_t)(i / S) & 1u, nullptr);
  if (p.ksplit > 1) cluster_barrier();  // nobody leaves while a peer may still read its sums
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols));
  }
}

template <int EPI>
int launch_epi(const CUtensorMap& map, MxArgs& p, cudaStream_t st) {
  constexpr int A_TILES = EPI == EPI_SWIGLU_BF16 ? 2 : 1;
  constexpr int MAX_DYN = 216 * 1024;
  const int rc = allow_smem<gemm_mx4_kernel<EPI>>(MAX_DYN);
  if (rc) return rc;
  // K shares: about 1.5 CTAs per SM in all, at least four k-blocks each
  const int sms = sm_count();
  const long long units = (long long)p.tiles * p.token_tiles;
  long long ks = (3ll * sms / 2 + units / 2) / units;
  if (ks > p.KB / 4) ks = p.KB / 4;
  if (ks > 8) ks = 8;
  if (ks < 1) ks = 1;
  p.ksplit = (int)ks;
  if (units * ks > 0x7fffffffll) return HYP_ECAPACITY;
  int cols = 32;
  while (cols < A_TILES * (p.nb + 4) + 8) cols <<= 1;
  p.tmem_cols = cols;
  p.stage_bytes = A_TILES * (MX_A_BYTES + MX_SF_BYTES) + (int)p.block_bytes;
  p.stage_bytes = (p.stage_bytes + 1023) / 1024 * 1024;
  const int dump_bytes = ks > 1 ? A_TILES * p.tt * MX_ROWS * 4 : 0;
  // two CTAs to an SM where there are that many and tensor memory has room for both
  const bool two = units * ks > sms && cols <= 256;
  const int budget = two ? 110 * 1024 : MAX_DYN;
  int stages = (budget - 1024) / p.stage_bytes;
  if (stages > MX_MAX_STAGES) stages = MX_MAX_STAGES;
  while (stages * p.stage_bytes < dump_bytes) ++stages;  // the sums reuse the ring
  if (stages < 2) stages = 2;
  if (stages > MX_MAX_STAGES || stages * p.stage_bytes + 1024 > MAX_DYN) return HYP_EINVAL;
  p.stages = stages;
  // never more CTAs on an SM than tensor memory holds: one that waits for it would hold up its cluster
  int smem = stages * p.stage_bytes + 1024;
  const int least = 228 * 1024 / (512 / cols + 1);
  if (smem < least) smem = least;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * ks));
  cfg.blockDim = dim3(MX_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int na = 0;
  if (pdl_level() >= 2) {
    attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
  }
  if (ks > 1) {
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = (unsigned)ks;
    attr[na].val.clusterDim.y = 1;
    attr[na].val.clusterDim.z = 1;
    ++na;
  }
  cfg.attrs = attr;
  cfg.numAttrs = na;
  HYP_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_mx4_kernel<EPI>, map, p));
  return 1;
}

}  // namespace

size_t mx4_scratch_bytes(int M, int K, int terms) {
  // the two row caps cut the tokens differently: the larger of both
  size_t most = 0;
  for (int cap : {240, 256}) {
    const TokenTiles t = token_tiles(M, terms, cap);
    const size_t n = (size_t)t.tiles * mx_kb(K) * t.block_bytes;
    if (n > most) most = n;
  }
  return most;
}

int launch_gemm_mx4(const void* a, int a_type, long long a_stride, const uint8_t* packed, int M, int N, int K, int terms, int epi,
                    void* out, int ldo, uint8_t* scratch, cudaStream_t st) {
  const TokenTiles t = token_tiles(M, terms, row_cap(epi));
  MxArgs p{};
  p.packed = packed; p.terms = scratch; p.block_bytes = t.block_bytes;
  p.M = M; p.N = N; p.KB = mx_kb(K); p.ldo = ldo;
  p.tiles = mx_row_tiles(N); p.token_tiles = t.tiles; p.tt = t.tt; p.nb = t.nb; p.n_terms = terms; p.sf_bytes = t.sf_bytes;
  p.f16 = a_type == HYP_TYPE_F16; p.out = out; p.err = tc_err_flag_ptr();
  p.idesc = (5u << 7) | (0u << 10) | ((uint32_t)(t.nb >> 3) << 17) | (1u << 23) | ((uint32_t)(MX_ROWS >> 4) << 24);  // E2M1 x E4M3, power-of-two scales
  CUtensorMap map;
  int rc = tc_make_mx4_map(&map, packed, (long long)(epi == EPI_SWIGLU_BF16 ? 2 : 1) * p.tiles * p.KB * (MX_PACK_BYTES / 64));
  if (rc) return rc;
  const int segments = (16 * p.KB + TERM_THREADS - 1) / TERM_THREADS;
  if (segments > 65535) return HYP_ECAPACITY;
  auto go = [&](auto kernel) {
    return launch_pdl<2>(kernel, dim3((unsigned)M, (unsigned)segments), dim3(TERM_THREADS), (size_t)0, st, (const uint8_t*)a, a_stride, M, K / 8, p.KB, terms,
                         t.tt, t.nb, t.block_bytes, scratch);
  };
  HYP_CUDA_TRY(a_type == HYP_TYPE_F16 ? go(mx_terms_kernel<HYP_TYPE_F16>) : go(mx_terms_kernel<HYP_TYPE_BF16>));
  switch (epi) {
    case EPI_STORE_BF16: rc = launch_epi<EPI_STORE_BF16>(map, p, st); break;
    case EPI_RESID_F32: rc = launch_epi<EPI_RESID_F32>(map, p, st); break;
    case EPI_SWIGLU_BF16: rc = launch_epi<EPI_SWIGLU_BF16>(map, p, st); break;
    case EPI_STORE_F32: rc = launch_epi<EPI_STORE_F32>(map, p, st); break;
    default: return HYP_EINVAL;
  }
  return rc < 0 ? rc : rc + 1;
}

}  // namespace hyp
