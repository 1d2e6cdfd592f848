// Decode attention with modified scores, decode attention that sums the weights each cached position receives, and
// shared-prefix decode attention (see attn_paged.cuh and attn_tile.cuh for the two CTA bodies).
#include <math.h>

#include "attn_tile.cuh"
#include "cache_ops.cuh"
#include "gemm_tc.cuh"

namespace hyp {

namespace {

constexpr int PD_WARPS = 4;      // decode kernels
// Bytes of prefix that the sequences of a batch may read again, each for itself, and prefix pages below which they always
// do; measured on 2 to 128 sequences of three head layouts: at 21 MB 9.9-12.5 us against 12.4 with row tiles, at 42 MB equal,
// at 84 MB 14.1-17.2 against 12.3-16.1; behind 128 tokens 10.4-19.1 against 12.5-27.8 whatever the batch.
constexpr double FLAT_BYTES = 32e6;
constexpr int FLAT_PAGES = 8;
template <int D>
constexpr int pd_slots() { return D == 128 ? 2 : 4; }  // 64 KB of ring: three CTAs per SM

template <int D, int G, int MODE, bool CLUSTER>
__global__ void __launch_bounds__(PD_WARPS * 32) paged_decode_kernel(PagedArgs a) {
  extern __shared__ __align__(128) uint8_t pd_smem[];
  __shared__ uint64_t bars[PD_WARPS * pd_slots<D>()];
  pdl_wait();     // queries, lengths and cache rows may come from the kernel launched just before
  pdl_trigger();  // after the wait: nothing of this operator runs before its inputs exist
  paged_body<D, G, MODE, PD_WARPS, pd_slots<D>(), CLUSTER>(a, pd_smem, bars, blockIdx.x, gridDim.x, blockIdx.y, blockIdx.z, threadIdx.x,
                                                           [] { __syncthreads(); });
}

// Joins the partial rows of one (sequence, query head) and writes fp16.
template <int D>
__global__ void __launch_bounds__(MERGE_THREADS)
paged_merge_kernel(const float* __restrict__ acc, const float* __restrict__ ml, int n_slots, __half* __restrict__ out) {
  __shared__ float sm[MERGE_THREADS / 32 * D];
  pdl_wait();
  pdl_trigger();
  const size_t row = blockIdx.x;  // b * Hq + h
  paged_merge_row<D>(acc, ml, row * n_slots, n_slots, out + row * D, sm);
}

// Second kernel of the scored operator.  grid (G + key chunks, Hkv, n_seqs): the first G CTAs of a (sequence, KV head) join
// the value sums of one query head each; every other one joins the splits' (maximum, denominator) of the G heads, turns
// its chunk of scores into weights and adds them to the running sums.
constexpr int SC_PER = 4, SC_KEYS = MERGE_THREADS * SC_PER;
template <int D, int G>
__global__ void __launch_bounds__(MERGE_THREADS)
scored_finish_kernel(PagedArgs a, __half* __restrict__ out) {
  __shared__ float sm[MERGE_THREADS / 32 * D];
  pdl_wait();
  pdl_trigger();
  const int kvh = blockIdx.y, b = blockIdx.z;
  const size_t row0 = (size_t)b * a.Hq + kvh * G;
  if (blockIdx.x < G) {
    const size_t row = row0 + blockIdx.x;
    paged_merge_row<D>(a.acc, a.ml, row * a.n_slots, a.n_slots, out + row * D, sm);
    return;
  }
  const int total = paged_total(a.ctx[b], a.table_stride);
  const int k0 = (blockIdx.x - G) * SC_KEYS + SC_PER * threadIdx.x;  // this thread's four keys
  if (k0 - SC_PER * (int)threadIdx.x >= total) return;
  const float* wi = a.w_in ? a.w_in + ((long long)b * a.Hkv + kvh) * a.w_stride : nullptr;
  float* wo = a.w_out + ((long long)b * a.Hkv + kvh) * a.w_stride;
  // everything this thread needs from memory is asked for before the maxima are joined
  float4 s[G];
  float old[SC_PER];
#pragma unroll
  for (int gq = 0; gq < G; ++gq)
    s[gq] = k0 < total ? *reinterpret_cast<const float4*>(a.scores + (row0 + gq) * a.score_stride + k0) : make_float4(PG_NEG, PG_NEG, PG_NEG, PG_NEG);
#pragma unroll
  for (int i = 0; i < SC_PER; ++i) old[i] = wi && k0 + i < total - 1 ? wi[k0 + i] : 0.f;  // the new token's sum starts here
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float *s_m = sm, *s_inv = sm + G;
  for (int gq = warp; gq < G; gq += MERGE_THREADS / 32) {
    const float* ml = a.ml + (row0 + gq) * a.n_slots * 2;
    float mx = PG_NEG, l = 0.f;
    for (int i = lane; i < a.n_slots; i += 32) {
      const float2 x = *reinterpret_cast<const float2*>(ml + 2 * i);
      const float top = fmaxf(mx, x.x);
      l = l * ex2_approx(mx - top) + x.y * ex2_approx(x.x - top);
      mx = top;
    }
    const float top = warp_max(mx);
    l = warp_sum(l * ex2_approx(mx - top));
    if (lane == 0) {
      s_m[gq] = top;
      s_inv[gq] = l != 0.f ? 1.f / l : 0.f;
    }
  }
  __syncthreads();
  float w[SC_PER] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int gq = 0; gq < G; ++gq) {
    w[0] += ex2_approx(s[gq].x - s_m[gq]) * s_inv[gq];
    w[1] += ex2_approx(s[gq].y - s_m[gq]) * s_inv[gq];
    w[2] += ex2_approx(s[gq].z - s_m[gq]) * s_inv[gq];
    w[3] += ex2_approx(s[gq].w - s_m[gq]) * s_inv[gq];
  }
#pragma unroll
  for (int i = 0; i < SC_PER; ++i)
    if (k0 + i < total) wo[k0 + i] = fmaf(a.decay, old[i], w[i]);
}

// ---------------------------------------------------------------------------------------------
// shared prefix: the prefixes' row tiles and the sequences' own pages, then a join of the partial rows.  Where both parts fit
// two waves of CTAs, one launch holds them: the own pages stream through the slots that the row tiles leave (20.2 instead of
// 23.7 us for 32 sequences behind 2048 tokens).  Larger batches stream their own pages in a launch of their own, with three
// smaller CTAs to an SM.
// ---------------------------------------------------------------------------------------------
struct SharedArgs {
  PagedArgs own;              // slots prefix_splits ..
  const int32_t* cu_group;
  const int32_t* prefix_table;
  int prefix_stride;
  const int32_t* prefix_lens;
  int n_groups, prefix_splits, own_splits, prefix_ctas;
  bool even;                  // see prefix_cut_even
};

// How the prefixes are cut: every (row tile, KV head) of group g is shared by `splits` CTAs of `per` key tiles each.
struct PrefixCut {
  int group, first, q0, len, plen, split, splits, per, kvh;
};
// Up to 32 groups, one lane each: the prefix CTAs (at most two per SM) are handed out so that all get about the same number of
// key tiles, whatever the lengths of the prefixes and the sizes of the groups.  (A fixed number of splits made 1.3
// waves of unequal CTAs of five prefixes of 4096 to 8192 tokens: 53 us.)
__device__ __forceinline__ bool prefix_cut_even(const SharedArgs& a, int T, PrefixCut& c) {
  const int lane = threadIdx.x & 31;
  const bool in = lane < a.n_groups;
  const int c0 = in ? a.cu_group[lane] : 0, c1 = in ? a.cu_group[lane + 1] : 0;
  const int plen = in ? min(max(a.prefix_lens[lane], 0), a.prefix_stride * PG_PT) : 0;
  const int units = (max(c1 - c0, 0) + T - 1) / T * a.own.Hkv, tiles = (plen + AT_KEYS - 1) / AT_KEYS;
  // lane i tries `per` = low + i * step: low is what an even share without rounding would be
  const int all = __reduce_add_sync(0xffffffffu, units * tiles), most = max(__reduce_max_sync(0xffffffffu, tiles), 1);
  int low = max((all + a.prefix_ctas - 1) / a.prefix_ctas, 1);
  low = max(low, (most + a.prefix_splits - 1) / a.prefix_splits);  // no prefix in more shares than there are slots
  const int step = max(low / 16, 1), mine = min(low + lane * step, most);
  int total = 0;
  for (int g = 0; g < a.n_groups; ++g) {
    const int ug = __shfl_sync(0xffffffffu, units, g), tg = __shfl_sync(0xffffffffu, tiles, g);
    total += ug * max((tg + mine - 1) / mine, 1);
  }
  const uint32_t fits = __ballot_sync(0xffffffffu, total <= a.prefix_ctas);
  c.per = fits ? __shfl_sync(0xffffffffu, mine, __ffs(fits) - 1) : most;  // one share each always fits
  const int splits = max((tiles + c.per - 1) / c.per, 1), count = units * splits;
  int incl = count;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  const uint32_t hit = __ballot_sync(0xffffffffu, (int)blockIdx.x < incl);
  if (!hit) return false;
  const int src = __ffs(hit) - 1;
  const int i = (int)blockIdx.x - __shfl_sync(0xffffffffu, incl - count, src);
  c.group = src;
  c.first = __shfl_sync(0xffffffffu, c0, src);
  c.len = __shfl_sync(0xffffffffu, c1, src) - c.first;
  c.plen = __shfl_sync(0xffffffffu, plen, src);
  c.splits = __shfl_sync(0xffffffffu, splits, src);
  c.split = i % c.splits;
  c.kvh = i / c.splits % a.own.Hkv;
  c.q0 = i / (c.splits * a.own.Hkv) * T;
  return true;
}
// More groups, or more row tiles than CTAs fit at once: prefix_splits shares for every (row tile, KV head).
__device__ __forceinline__ bool prefix_cut_fixed(const SharedArgs& a, int T, PrefixCut& c) {
  c.splits = a.prefix_splits;
  c.split = blockIdx.x % c.splits;
  c.kvh = blockIdx.x / c.splits % a.own.Hkv;
  int plen, none;
  at_locate(a.cu_group, a.prefix_lens, nullptr, a.n_groups, T, blockIdx.x / (c.splits * a.own.Hkv), c.group, c.first, c.q0, c.len, plen, none);
  if (c.group < 0) return false;
  c.plen = min(max(plen, 0), a.prefix_stride * PG_PT);
  c.per = ((c.plen + AT_KEYS - 1) / AT_KEYS + c.splits - 1) / c.splits;
  return true;
}

constexpr int SH_WARPS = AT_THREADS / 32;
template <int D>
constexpr int sh_slots() { return D == 128 ? 2 : 4; }
template <int D>
constexpr int sh_smem() {
  return AtGeom<D>::SMEM > paged_smem_bytes<D, SH_WARPS>(sh_slots<D>()) ? AtGeom<D>::SMEM : paged_smem_bytes<D, SH_WARPS>(sh_slots<D>());
}

template <int D, int G>
__global__ void __launch_bounds__(AT_THREADS, 2)
shared_decode_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kv, SharedArgs a) {
  extern __shared__ __align__(128) uint8_t sh_smem_raw[];
  __shared__ TileShared ts;
  __shared__ uint64_t bars[SH_WARPS * sh_slots<D>()];
  pdl_wait();
  if ((int)blockIdx.x >= a.prefix_ctas) {
    pdl_trigger();
    const int i = blockIdx.x - a.prefix_ctas;
    paged_body<D, G, PAGED_PLAIN, SH_WARPS, sh_slots<D>(), false>(a.own, sh_smem_raw, bars, i % a.own_splits, a.own_splits,
                                                          (i / a.own_splits) % a.own.Hkv, i / (a.own_splits * a.own.Hkv),
                                                          threadIdx.x, [] { __syncthreads(); });
    return;
  }
  tile_setup(ts);
  pdl_trigger();  // only now: a kernel that starts early must not find tensor memory free that this CTA still has to take
  constexpr int T = AT_ROWS / G;
  PrefixCut cut;
  if (!(a.even ? prefix_cut_even(a, T, cut) : prefix_cut_fixed(a, T, cut))) {
    tile_release(ts);
    return;
  }
  const int kvh = cut.kvh, split = cut.split, plen = cut.plen;
  const int all_tiles = (plen + AT_KEYS - 1) / AT_KEYS;
  TileWork wk;
  wk.head0 = kvh * G;
  wk.kvh = kvh;
  wk.row0 = cut.first + cut.q0;
  wk.rows = min(T, cut.len - cut.q0);
  wk.table = a.prefix_table + (long long)cut.group * a.prefix_stride;
  wk.key_end = plen;
  wk.n_first = 0;
  wk.second = split * cut.per;
  wk.n_tiles = max(0, min(cut.per, all_tiles - split * cut.per));
  auto slot_of = [&](int t, int gh) { return ((size_t)(wk.row0 + t) * a.own.Hq + wk.head0 + gh) * a.own.n_slots + split; };
  // shares that are empty, or that this group does not have, still have to say so
  for (int s = split + (wk.n_tiles > 0); s < (split == cut.splits - 1 ? a.prefix_splits : split + 1); ++s) {
    const int t = threadIdx.x / G, gh = threadIdx.x % G;
    if (threadIdx.x < AT_ROWS && t < wk.rows) *reinterpret_cast<float2*>(a.own.ml + (slot_of(t, gh) + s - split) * 2) = make_float2(PG_NEG, 0.f);
  }
  if (wk.n_tiles == 0) {  // the whole CTA
    tile_release(ts);
    return;
  }
  tile_body<D, false, false>(
      &tm_q, &tm_kv, sh_smem_raw, ts, wk, G, a.own.Hkv, 0.f, nullptr, a.own.err,
      [&](int, int& pos) {
        pos = plen - 1;
        return TileRow{0, plen - 1, 0};
      },
      [&](int t, int gh, bool valid, float m_ref, float l, uint32_t stage, auto load) {
        const size_t row = slot_of(t, gh);
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint32_t v[16], w[16];
          load(c, v, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            at_stage16(stage + 4 * c + 16 * i, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            at_stage16(stage + 4 * c + 64 + 16 * i, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          }
        }
        at_send_row(a.own.acc + row * D, stage, D * 4, valid);
        if (valid) *reinterpret_cast<float2*>(a.own.ml + row * 2) = make_float2(m_ref, l);
      });
  tile_release(ts);
}

// ---------------------------------------------------------------------------------------------
// prefill with modified scores
// ---------------------------------------------------------------------------------------------
struct PrefillModArgs {
  __half* out;
  const int32_t* cu_q;
  const int32_t* ctx;
  const int32_t* table;
  int table_stride, n_seqs, Hq, Hkv, G;
  float softcap;
  int window;
  const float* slopes;
  const int32_t* prefix;
  int* err;
};

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(AT_THREADS, 2)
prefill_mod_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kv, PrefillModArgs a) {
  extern __shared__ __align__(128) uint8_t pm_smem[];
  __shared__ TileShared ts;
  pdl_wait();
  tile_setup(ts);
  pdl_trigger();  // only now: a kernel that starts early must not find tensor memory free that this CTA still has to take
  const int T = AT_ROWS / a.G;
  const int kvh = blockIdx.x % a.Hkv;  // heads vary fastest: every head's heaviest tile is scheduled before any lighter one
  int seq, first, q0, len, ctx, pre;
  // the last tiles of a sequence see the most keys: they go first
  at_locate(a.cu_q, a.ctx, a.prefix, a.n_seqs, T, (int)(gridDim.x / a.Hkv) - 1 - (int)(blockIdx.x / a.Hkv), seq, first, q0, len, ctx, pre);
  if (seq < 0) {
    tile_release(ts);
    return;
  }
  ctx = min(max(ctx, 0), 1 << 30);  // no table names more; a position, and a position plus a tile, stay within 32 bits
  const int have = min(ctx + len, a.table_stride * PG_PT);  // tokens in the cache, the new rows included
  pre = min(max(pre, 0), have);
  const int window = a.window > 0 ? a.window : 0x7fffffff;
  TileWork wk;
  wk.head0 = kvh * a.G;
  wk.kvh = kvh;
  wk.row0 = first + q0;
  wk.rows = min(T, len - q0);
  wk.table = a.table + (long long)seq * a.table_stride;
  wk.key_end = have;
  const int lo = max(ctx + q0 - window + 1, 0), hi = min(ctx + q0 + wk.rows, have);  // keys of the tile's rows: [lo, hi), [0, pre)
  wk.n_first = (pre + AT_KEYS - 1) / AT_KEYS;
  wk.second = max(lo / AT_KEYS, wk.n_first);
  wk.n_tiles = wk.n_first + max((hi + AT_KEYS - 1) / AT_KEYS - wk.second, 0);
  if (wk.n_tiles == 0) {  // a window that lies wholly behind what the table can name: rows that see nothing
    const int per = a.G * D / 8;  // 16-byte pieces of a token's G heads
    for (int e = threadIdx.x; e < wk.rows * per; e += AT_THREADS)
      *reinterpret_cast<uint4*>(a.out + ((size_t)(wk.row0 + e / per) * a.Hq + wk.head0) * D + (size_t)(e % per) * 8) = make_uint4(0u, 0u, 0u, 0u);
    tile_release(ts);
    return;
  }
  tile_body<D, CAP, BIAS>(
      &tm_q, &tm_kv, pm_smem, ts, wk, a.G, a.Hkv, a.softcap, a.slopes, a.err,
      [&](int t, int& pos) {
        pos = ctx + q0 + t;
        return TileRow{max(pos - window + 1, 0), min(pos, have - 1), pre};
      },
      [&](int t, int gh, bool valid, float, float l, uint32_t stage, auto load) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
        __half* orow = a.out + ((size_t)(wk.row0 + t) * a.Hq + wk.head0 + gh) * D;
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint32_t v[16], w[16];
          load(c, v, w);
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            pk[i] = pack_f16(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
            pk[8 + i] = pack_f16(__uint_as_float(w[2 * i]) * inv, __uint_as_float(w[2 * i + 1]) * inv);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) at_stage16(stage + 2 * c + 16 * i, pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
        }
        at_send_row(orow, stage, D * 2, valid);
      });
  tile_release(ts);
}

int wave_splits(int n_seqs, int Hkv) {  // three CTAs per SM
  const int want = (int)(3 * sm_count() / ((long long)n_seqs * Hkv));
  return want < 1 ? 1 : want;
}

PagedArgs paged_args(const CacheView& c, const __half* q, long long q_stride, float* scratch, int n_slots, int slot0, int* err) {
  PagedArgs a{};
  a.q = q; a.q_stride = q_stride;
  a.pool = c.pool; a.table = c.table; a.table_stride = c.table_stride; a.ctx = c.ctx;
  a.Hq = c.Hq; a.Hkv = c.Hkv;
  a.acc = scratch;
  a.ml = scratch + (size_t)c.n_seqs * c.Hq * n_slots * c.D;
  a.n_slots = n_slots; a.slot0 = slot0;
  a.wave_splits = wave_splits(c.n_seqs, c.Hkv);
  a.err = err;
  return a;
}

template <int D, int G, int MODE, bool CLUSTER>
int launch_paged(const PagedArgs& a, int n_splits, int n_seqs, cudaStream_t st) {
  constexpr int smem = paged_smem_bytes<D, PD_WARPS>(pd_slots<D>());
  const int rc = allow_smem<paged_decode_kernel<D, G, MODE, CLUSTER>>(smem);
  if (rc) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_splits, a.Hkv, n_seqs);
  cfg.blockDim = dim3(PD_WARPS * 32);
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
  HYP_CUDA_TRY(cudaLaunchKernelEx(&cfg, paged_decode_kernel<D, G, MODE, CLUSTER>, a));
  return 1;
}
// Up to eight splits of a batch that is on the GPU all at once join inside the kernel.  In more than one wave a cluster's CTAs
// also have to find room together: 64 ragged sequences of up to 8192 tokens took 56 instead of 49 us that way.
bool joins_in_cluster(int n_splits, int Hkv, int n_seqs) {
  return n_splits >= 2 && n_splits <= 8 && (long long)n_splits * Hkv * n_seqs <= 3ll * sm_count();
}

template <int D>
int launch_merge(const PagedArgs& a, int n_seqs, __half* out, cudaStream_t st) {
  HYP_CUDA_TRY(launch_pdl<2>(paged_merge_kernel<D>, dim3(n_seqs * a.Hq), dim3(MERGE_THREADS), (size_t)0, st, a.acc, a.ml, a.n_slots, out));
  return 1;
}

#define HYP_DG_DISPATCH(F)                                                            \
  do {                                                                                \
    const int G_ = c.Hq / c.Hkv;                                                      \
    if (c.D == 128 && G_ == 1) return F(128, 1);                                      \
    if (c.D == 128 && G_ == 2) return F(128, 2);                                      \
    if (c.D == 128 && G_ == 4) return F(128, 4);                                      \
    if (c.D == 128 && G_ == 8) return F(128, 8);                                      \
    if (c.D == 64 && G_ == 1) return F(64, 1);                                        \
    if (c.D == 64 && G_ == 2) return F(64, 2);                                        \
    if (c.D == 64 && G_ == 4) return F(64, 4);                                        \
    if (c.D == 64 && G_ == 8) return F(64, 8);                                        \
    return HYP_EINVAL;                                                                \
  } while (0)

template <int D, int G, int MODE>
int decode_joined_dg(PagedArgs a, int n_splits, int n_seqs, __half* out, cudaStream_t st) {
  // (the running sums gain nothing from it: their weights would wait for the join, 14.1 instead of 13.2 us)
  const bool cluster = MODE != PAGED_SCORED && joins_in_cluster(n_splits, a.Hkv, n_seqs);
  if (n_splits == 1 || cluster) a.out = out;
  if constexpr (MODE != PAGED_SCORED)
    if (cluster) return launch_paged<D, G, MODE, true>(a, n_splits, n_seqs, st);
  const int rc = launch_paged<D, G, MODE, false>(a, n_splits, n_seqs, st);
  if (rc < 0 || n_splits == 1) return rc;
  if (MODE == PAGED_SCORED) {
    const int chunks = (a.table_stride * PG_PT + SC_KEYS - 1) / SC_KEYS;
    HYP_CUDA_TRY(launch_pdl<2>(scored_finish_kernel<D, G>, dim3(G + chunks, a.Hkv, n_seqs), dim3(MERGE_THREADS), (size_t)0, st, a, out));
    return 2;
  }
  const int rc2 = launch_merge<D>(a, n_seqs, out, st);
  return rc2 < 0 ? rc2 : rc + rc2;
}

template <int D, int G>
int decode_shared_dg(const CUtensorMap& mq, const CUtensorMap& mkv, const SharedArgs& a, int n_seqs, __half* out, cudaStream_t st) {
  constexpr int smem = sh_smem<D>();
  int rc = allow_smem<shared_decode_kernel<D, G>>(smem);
  if (rc) return rc;
  const long long own_ctas = (long long)a.own_splits * a.own.Hkv * n_seqs;
  const bool together = a.prefix_ctas + own_ctas <= 4ll * sm_count();
  HYP_CUDA_TRY(launch_pdl<2>(shared_decode_kernel<D, G>, dim3((unsigned)(a.prefix_ctas + (together ? own_ctas : 0))), dim3(AT_THREADS),
                             (size_t)smem, st, mq, mkv, a));
  if (!together) {
    rc = launch_paged<D, G, PAGED_PLAIN, false>(a.own, a.own_splits, n_seqs, st);
    if (rc < 0) return rc;
  }
  rc = launch_merge<D>(a.own, n_seqs, out, st);
  return rc < 0 ? rc : together ? 2 : 3;
}

template <int D, bool CAP, bool BIAS>
int prefill_mod_launch(const CUtensorMap& mq, const CUtensorMap& mkv, const PrefillModArgs& a, int M, cudaStream_t st) {
  constexpr int smem = AtGeom<D>::SMEM;
  const int rc = allow_smem<prefill_mod_kernel<D, CAP, BIAS>>(smem);
  if (rc) return rc;
  const int T = AT_ROWS / a.G;
  const long long tiles = (long long)M / T + a.n_seqs;  // every sequence adds at most one ragged tile
  if (tiles * a.Hkv > 0x7fffffffll) return HYP_ECAPACITY;
  HYP_CUDA_TRY(launch_pdl<2>(prefill_mod_kernel<D, CAP, BIAS>, dim3((unsigned)(tiles * a.Hkv)), dim3(AT_THREADS), (size_t)smem, st, mq, mkv, a));
  return 1;
}

}  // namespace

int paged_splits(int n_seqs, int Hkv, int max_pages) {
  // Up to 16 pages (four per warp): one CTA per sequence and KV head, which then writes the result itself (the join is a
  // launch of its own, ~2.5 us).  Short contexts: one wave of three CTAs per SM.  Longer ones (more than 64 pages a CTA
  // that way): about four waves, so that ragged batches even out.  At least one page per warp.
  const long long groups = (long long)n_seqs * Hkv;
  if (max_pages <= 4 * PD_WARPS) return 1;
  int want = wave_splits(n_seqs, Hkv);
  if (max_pages > 64 * want) want = (int)((12 * sm_count() + groups - 1) / groups);
  const int cap = (max_pages + PD_WARPS - 1) / PD_WARPS;
  if (want > cap) want = cap;
  return want > 64 ? 64 : want;
}

size_t paged_scratch_floats(int n_seqs, int Hq, int D, int n_slots) { return (size_t)n_seqs * Hq * n_slots * (D + 2); }
size_t scored_scores_offset(int n_seqs, int Hq, int Hkv, int D, int max_pages) {
  return (paged_scratch_floats(n_seqs, Hq, D, paged_splits(n_seqs, Hkv, max_pages)) + 3) / 4 * 4;
}

int launch_decode_mod(const CacheView& c, const hyp_attn_mod& mod, const __half* q, long long q_stride, float* scratch,
                      __half* out, int* err, cudaStream_t st) {
  // A window bounds what is read, whatever the table could hold; a prefix, whose length is only known on the device, is taken for
  // 16 pages.  Against a plan by the table's width where there is a prefix (window 128, prefix 256 / 2048 / 8192, 32 / 8 heads of
  // 128): 8 sequences 8.4 / 17 / 47 us, by the table 10.6 / 21 / 55; 32 sequences 12.4 / 48 / 164 against 16.9 / 55 / 170; one sequence
  // 8.5 / 9.0 / 20 against 10.2 / 10.3 / 14.  Fewer pages never mean more splits, so the scratch for the whole table suffices.
  int pages = c.table_stride;
  if (mod.window > 0) pages = (int)fmin((double)pages, mod.window / 16.0 + 2.0 + (mod.prefix_lens ? 16.0 : 0.0));
  const int ns = paged_splits(c.n_seqs, c.Hkv, pages);
  PagedArgs a = paged_args(c, q, q_stride, scratch, ns, 0, err);
  a.softcap = mod.softcap; a.window = mod.window; a.slopes = mod.slopes; a.prefix = mod.prefix_lens;
#define HYP_F(DD, GG) decode_joined_dg<DD, GG, PAGED_MOD>(a, ns, c.n_seqs, out, st)
  HYP_DG_DISPATCH(HYP_F);
#undef HYP_F
}

int launch_decode_scored(const CacheView& c, const __half* q, long long q_stride, float decay, const float* w_in, float* w_out,
                         long long w_stride, float* scratch, __half* out, int* err, cudaStream_t st) {
  const int ns = paged_splits(c.n_seqs, c.Hkv, c.table_stride);
  PagedArgs a = paged_args(c, q, q_stride, scratch, ns, 0, err);
  a.score_stride = c.table_stride * PG_PT;
  a.scores = scratch + scored_scores_offset(c.n_seqs, c.Hq, c.Hkv, c.D, c.table_stride);
  a.decay = decay; a.w_in = w_in; a.w_out = w_out; a.w_stride = w_stride;
#define HYP_F(DD, GG) decode_joined_dg<DD, GG, PAGED_SCORED>(a, ns, c.n_seqs, out, st)
  HYP_DG_DISPATCH(HYP_F);
#undef HYP_F
}

SharedPlan shared_plan(int n_seqs, int Hq, int Hkv, int D, int n_groups, int prefix_pages, int own_pages) {
  SharedPlan p{};
  const int T = AT_ROWS / (Hq / Hkv);
  p.row_tiles = n_seqs / T + n_groups;  // every group adds at most one ragged tile
  // Where the prefixes are short or the batch is small, every sequence walks its prefix for itself: what it reads again
  // comes from the L2, and a whole launch and the row tiles' set-up fall away.
  const double again = (double)n_seqs * Hkv * prefix_pages * (2 * PG_PT * 2) * D;
  p.flat = again <= FLAT_BYTES || prefix_pages <= FLAT_PAGES;
  if (p.flat) {
    p.prefix_splits = 0;
    p.own_splits = paged_splits(n_seqs, Hkv, prefix_pages + own_pages);
    return p;
  }
  const int slots = 2 * sm_count();  // resident CTAs (half of them: 107 instead of 96 us for 128 sequences behind five prefixes)
  // at least four key tiles each (two: 24.8 instead of 23.7 us for 32 sequences behind 2048 tokens, and twice the partial rows)
  const int most = (prefix_pages * PG_PT + 4 * AT_KEYS - 1) / (4 * AT_KEYS);
  p.even = n_groups <= 32 && (long long)p.row_tiles * Hkv <= slots;
  if (p.even) {
    p.prefix_splits = most < 16 ? most : 16;
    const int need = p.row_tiles * Hkv * p.prefix_splits;
    p.prefix_ctas = need < slots ? need : slots;
  } else {
    const int full = (n_seqs + T - 1) / T > n_groups ? (n_seqs + T - 1) / T : n_groups;
    p.prefix_splits = (int)(slots / ((long long)full * Hkv));
    if (p.prefix_splits > most) p.prefix_splits = most;
    if (p.prefix_splits > MERGE_SLOTS - 64) p.prefix_splits = MERGE_SLOTS - 64;
    if (p.prefix_splits < 1) p.prefix_splits = 1;
    p.prefix_ctas = (int)fmin((double)p.prefix_splits * Hkv * p.row_tiles, 2147483647.0);  // too many are refused by the caller
  }
  p.own_splits = paged_splits(n_seqs, Hkv, own_pages);
  return p;
}

int launch_decode_shared(const CacheView& c, const __half* q, long long q_stride, int n_groups, const int32_t* cu_group,
                         const int32_t* prefix_table, int prefix_stride, const int32_t* prefix_lens, float* scratch,
                         __half* out, int* err, cudaStream_t st) {
  const SharedPlan p = shared_plan(c.n_seqs, c.Hq, c.Hkv, c.D, n_groups, prefix_stride, c.table_stride);
  SharedArgs a{};
  a.own = paged_args(c, q, q_stride, scratch, p.prefix_splits + p.own_splits, p.prefix_splits, err);
  a.cu_group = cu_group; a.prefix_table = prefix_table; a.prefix_stride = prefix_stride; a.prefix_lens = prefix_lens;
  a.n_groups = n_groups; a.prefix_splits = p.prefix_splits; a.own_splits = p.own_splits;
  a.even = p.even; a.prefix_ctas = p.prefix_ctas;
  if (p.flat) {
    PagedArgs f = a.own;
    f.cu_group = cu_group; f.prefix_table = prefix_table; f.prefix_lens = prefix_lens;
    f.prefix_stride = prefix_stride; f.n_groups = n_groups;
#define HYP_F(DD, GG) decode_joined_dg<DD, GG, PAGED_FLAT>(f, p.own_splits, c.n_seqs, out, st)
    HYP_DG_DISPATCH(HYP_F);
#undef HYP_F
  }
  CUtensorMap mq, mkv;
  int rc = tc_make_q_map(&mq, q, c.n_seqs, q_stride, c.Hq, c.Hq / c.Hkv, c.D);
  if (!rc) rc = tc_make_pool_map(&mkv, c.pool, c.D);
  if (rc) return rc;
#define HYP_F(DD, GG) decode_shared_dg<DD, GG>(mq, mkv, a, c.n_seqs, out, st)
  HYP_DG_DISPATCH(HYP_F);
#undef HYP_F
}

int launch_prefill_mod(const CacheView& c, const hyp_attn_mod& mod, int M, const __half* q, long long q_stride,
                       const int32_t* cu_q, __half* out, int* err, cudaStream_t st) {
  PrefillModArgs a{};
  a.out = out; a.cu_q = cu_q; a.ctx = c.ctx; a.table = c.table; a.table_stride = c.table_stride;
  a.n_seqs = c.n_seqs; a.Hq = c.Hq; a.Hkv = c.Hkv; a.G = c.Hq / c.Hkv;
  a.softcap = mod.softcap; a.window = mod.window; a.slopes = mod.slopes; a.prefix = mod.prefix_lens;
  a.err = err;
  CUtensorMap mq, mkv;
  int rc = tc_make_q_map(&mq, q, M, q_stride, c.Hq, a.G, c.D);
  if (!rc) rc = tc_make_pool_map(&mkv, c.pool, c.D);
  if (rc) return rc;
  const bool cap = mod.softcap > 0.f, bias = mod.slopes != nullptr;
#define HYP_F(DD)                                                                        \
  if (c.D == DD) {                                                                       \
    if (cap && bias) return prefill_mod_launch<DD, true, true>(mq, mkv, a, M, st);       \
    if (cap) return prefill_mod_launch<DD, true, false>(mq, mkv, a, M, st);              \
    if (bias) return prefill_mod_launch<DD, false, true>(mq, mkv, a, M, st);             \
    return prefill_mod_launch<DD, false, false>(mq, mkv, a, M, st);                      \
  }
  HYP_F(128) HYP_F(64)
#undef HYP_F
  return HYP_EINVAL;
}

}  // namespace hyp
