// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) the first n_sink tokens, the
// last n_recent tokens and the heaviest of the others stay, in their order, n_keep in all.
//
//   select kernel: grid (Hkv, n_seqs), 1024 threads.  The weights between the protected ends stand for order-preserving
//   32-bit keys, held in shared memory (up to 32768, read again from L2 for longer contexts).  The threshold, the m-th
//   largest key, is found digit by digit (11, 11 and 10 bits): a histogram in shared memory of the keys that agree with the
//   digits found so far, scanned from the top.  Counts do not depend on the order of the additions, so the result is the
//   same on every run.  The kept indexes and weights are then written at the places that a scan over (stripe, warp)
//   counts gives; among keys equal to the threshold the lowest indexes win.  (40 heads of 4096
//   tokens: 21 us searching bit pairs with block-wide counts, 16 us with the weights in registers - every CTA then runs
//   straight through 32-fold unrolled code once, and waits for its instructions.)
//   Then the kept rows move, re-permuted for their new slots.  To other pages: a warp for 32 rows.  In place a row moves down
//   or stays, so one CTA per (sequence, KV head, keys or values) goes up the rows and reads each batch completely before it
//   writes it: a batch writes at or below its own sources, never at a later one's.  A few rows of a few heads are moved by
//   the selecting CTA.
// Every kept row is read and written once: 13.4 us for 84 MB (4 x 4096 -> 2048, 40 / 10 heads of 128; HBM reads 42 MB and sees 2 of the 42 MB
// written, the rest stays in the L2), 40.5 us for 264 MB (32 ragged sequences).  The selection is bound by its block-wide steps
// (10 us for 40 heads of 4096 tokens, 22 us for 256 of up to 8191).  In place the same 84 MB take 35 us: 80 CTAs, each a chain of
// batches.
#include "cache_ops.cuh"
#include "hyperion.h"

namespace hyp {

namespace {

constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32, EV_STRIPES = 32;  // stripes of EV_THREADS candidates in shared memory

// Keys ascend with the weight; -0 equals +0, NaN counts as -infinity.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) w = __int_as_float(0xff800000);
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int EV_BINS = 2048;

// Inclusive sum over the block's threads, one value each.  `tmp`: EV_WARPS words.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* tmp) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 31) tmp[warp] = v;
  __syncthreads();
  return v + __reduce_add_sync(0xffffffffu, lane < warp ? tmp[lane] : 0u);
}

// One key into the histogram.  All lanes call; where the whole warp has the same bin, one lane adds for all.
__device__ __forceinline__ void count_bin(uint32_t* hist, bool valid, uint32_t bin) {
  if (!valid) bin = ~0u;
  const uint32_t first = __shfl_sync(0xffffffffu, bin, 0);
  if (__all_sync(0xffffffffu, bin == first)) {
    if (valid && (threadIdx.x & 31) == 0) atomicAdd(hist + first, 32u);
  } else if (valid) {
    atomicAdd(hist + bin, 1u);
  }
}

// Few rows and at most one CTA per SM (MOVES): the selecting CTA moves them itself, keys and values, all read before any is written - in place or
// not - and a launch falls away (13.0 -> 10.8 us for 4 x 1000 -> 200; 320 CTAs, two to an SM without this, 31.8 -> 40).
constexpr int MH_UNROLL = 8;
__host__ __device__ constexpr int move_here_rows(int D) { return MH_UNROLL * EV_THREADS / (2 * (D / 8)); }
__device__ __forceinline__ void move_rows(const EvictArgs& a, int kvh, int b, int len, const int32_t* kept) {
  const int lg = a.D == 128 ? 4 : 3;  // 16-byte chunks of a row: 1 << lg
  const int32_t* bt = a.table + (long long)b * a.table_stride;
  const int32_t* dt = a.dst_table + (long long)b * a.dst_stride;
  auto at = [&](int32_t page, int kind, int slot, int c) {
    return ((((size_t)page * 2 + kind) * a.Hkv + kvh) * 16 + slot) * a.D + ((c ^ (slot & 7)) << 3);
  };
  uint4 v[MH_UNROLL];
#pragma unroll
  for (int u = 0; u < MH_UNROLL; ++u) {
    const int e = u * EV_THREADS + threadIdx.x, i = e >> (lg + 1);
    if (i < len) {
      const int s = kept[i];
      v[u] = *reinterpret_cast<const uint4*>(a.pool + at(bt[s >> 4], (e >> lg) & 1, s & 15, e & ((1 << lg) - 1)));
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < MH_UNROLL; ++u) {
    const int e = u * EV_THREADS + threadIdx.x, i = e >> (lg + 1);
    if (i < len) *reinterpret_cast<uint4*>(a.dst + at(dt[i >> 4], (e >> lg) & 1, i & 15, e & ((1 << lg) - 1))) = v[u];
  }
}

// STAGED: the candidates fit shared memory (chosen by what the table's row can name).
template <bool STAGED, bool MOVES>
__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(EvictArgs a) {
  extern __shared__ float sw[];  // STAGED: the candidates' weights
  __shared__ uint32_t hist[EV_BINS];
  __shared__ uint32_t tmp[EV_WARPS];
  __shared__ uint32_t found[3];  // bin, keys above it, keys in it
  pdl_wait();
  pdl_trigger();
  const int kvh = blockIdx.x, b = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t = min(max(a.cached[b], 0), a.table_stride * 16);
  const long long head = (long long)b * a.Hkv + kvh;
  const float* w = a.w_in + head * a.w_stride;
  float* wo = a.w_out + head * a.w_out_stride;
  int32_t* kept = a.kept + head * a.n_keep;
  if (kvh == 0 && tid == 0) a.new_lens[b] = min(t, a.n_keep);
  if (t <= a.n_keep) {
    for (int i = tid; i < a.n_keep; i += EV_THREADS) {
      kept[i] = i < t ? i : -1;
      if (i < t) wo[i] = w[i];
    }
    if (MOVES) {
      __syncthreads();  // the kept slots are this CTA's own
      move_rows(a, kvh, b, t, kept);
    }
    return;
  }
  const int r0 = a.n_sink, n = t - a.n_sink - a.n_recent;  // candidates w[r0 .. r0 + n), of which m stay; n > m
  const int m = a.n_keep - a.n_sink - a.n_recent;
  if (STAGED)  // every thread reads back its own, so nothing has to be waited for yet
    for (int k = tid; k < n; k += EV_THREADS) sw[k] = w[r0 + k];
  auto weight = [&](int k) { return STAGED ? sw[k] : w[r0 + k]; };
  // threshold: the m-th largest key.  need: how many of the keys that agree with the digits found so far stay.
  uint32_t thr = 0, known = 0;
  int need = m;
  bool all = m == 0;  // every key that agrees stays (or nothing does)
  for (int shift = 21; shift >= 0 && !all; shift = shift == 21 ? 10 : shift == 10 ? 0 : -1) {
    const uint32_t digit = shift == 0 ? 1023u : 2047u;
    for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    auto add = [&](int k, float x) {
      const uint32_t key = weight_key(x);
      count_bin(hist, k < n && (key & known) == thr, (key >> shift) & digit);
    };
    for (int s = 0; s < n; s += EV_THREADS) add(s + tid, s + tid < n ? weight(s + tid) : 0.f);
    __syncthreads();
    // thread i has bins 2047 - 2i and 2046 - 2i: keys in the bins above a bin, from the top
    const uint32_t hi = hist[EV_BINS - 1 - 2 * tid], lo = hist[EV_BINS - 2 - 2 * tid];
    const uint32_t upto = block_scan(hi + lo, tmp), before = upto - hi - lo;
    if ((int)before < need && (int)(before + hi) >= need) {
      found[0] = EV_BINS - 1 - 2 * tid;
      found[1] = before;
      found[2] = hi;
    } else if ((int)(before + hi) < need && (int)upto >= need) {
      found[0] = EV_BINS - 2 - 2 * tid;
      found[1] = before + hi;
      found[2] = lo;
    }
    __syncthreads();
    thr |= found[0] << shift;
    known |= digit << shift;
    need -= (int)found[1];
    all = need == (int)found[2];
    __syncthreads();  // the histogram is cleared and `found` rewritten by the next digit
  }
  // A key stays if the digits found are above the threshold's, or equal to them and it is among the first `need` of those.
  const int limit = all ? (m == 0 ? 0 : n) : need;

  if (STAGED) {
    // (stripe, warp) counts, greater in the low half, equal in the high half: at most 32768 each
    uint32_t* cnt = hist;
    const int stripes = m > 0 ? (n + EV_THREADS - 1) / EV_THREADS : 0;
    for (int i = 0; i < stripes; ++i) {
      const int k = i * EV_THREADS + tid;
      const uint32_t key = k < n ? weight_key(sw[k]) & known : 0u;
      const uint32_t mg = __ballot_sync(0xffffffffu, k < n && key > thr), me = __ballot_sync(0xffffffffu, k < n && key == thr);
      if (lane == 0) cnt[i * EV_WARPS + warp] = __popc(mg) | (__popc(me) << 16);
    }
    __syncthreads();  // all weights have been read: from here on they may be overwritten
    const uint32_t mine = tid < stripes * EV_WARPS ? cnt[tid] : 0u;
    const uint32_t upto = block_scan(mine, tmp);
    cnt[tid] = upto - mine;
    __syncthreads();
    for (int i = 0; i < stripes; ++i) {
      const int k = i * EV_THREADS + tid;
      const float x = k < n ? sw[k] : 0.f;
      const uint32_t key = weight_key(x) & known;
      const bool gt = k < n && key > thr, eq = k < n && key == thr;
      const uint32_t below = (1u << lane) - 1u, base = cnt[i * EV_WARPS + warp];
      const int e_before = (int)(base >> 16) + __popc(__ballot_sync(0xffffffffu, eq) & below);
      const int g_before = (int)(base & 0xffffu) + __popc(__ballot_sync(0xffffffffu, gt) & below);
      if (gt || (eq && e_before < limit)) {
        const int pos = r0 + g_before + min(e_before, limit);
        kept[pos] = r0 + k;
        wo[pos] = x;
      }
    }
  } else {
    // stripes of 1024 candidates, each read before any of it is written
    __shared__ uint2 totals[2][EV_WARPS];
    uint32_t gt_base = 0, eq_base = 0;
    int turn = 0;
    for (int s = 0; s < n && m > 0; s += EV_THREADS, turn ^= 1) {
      const int k = s + tid;
      const float x = k < n ? w[r0 + k] : 0.f;
      const uint32_t key = weight_key(x) & known;
      const bool gt = k < n && key > thr, eq = k < n && key == thr;
      const uint32_t mg = __ballot_sync(0xffffffffu, gt), me = __ballot_sync(0xffffffffu, eq);
      if (lane == 0) totals[turn][warp] = make_uint2(__popc(mg), __popc(me));
      __syncthreads();
      const uint2 tl = totals[turn][lane];
      const uint32_t before_g = __reduce_add_sync(0xffffffffu, lane < warp ? tl.x : 0u);
      const uint32_t before_e = __reduce_add_sync(0xffffffffu, lane < warp ? tl.y : 0u);
      const uint32_t below = (1u << lane) - 1u;
      const int g_before = (int)(gt_base + before_g) + __popc(mg & below), e_before = (int)(eq_base + before_e) + __popc(me & below);
      if (gt || (eq && e_before < limit)) {
        const int pos = r0 + g_before + min(e_before, limit);
        kept[pos] = r0 + k;
        wo[pos] = x;
      }
      gt_base += __reduce_add_sync(0xffffffffu, tl.x);
      eq_base += __reduce_add_sync(0xffffffffu, tl.y);
    }
  }
  // the protected ends; the first tokens stay where they are, the last move down
  for (int i = tid; i < a.n_sink; i += EV_THREADS) {
    kept[i] = i;
    wo[i] = w[i];
  }
  for (int s = 0; s < a.n_recent; s += EV_THREADS) {
    const int i = s + tid;
    const float x = i < a.n_recent ? w[t - a.n_recent + i] : 0.f;
    __syncthreads();
    if (i < a.n_recent) {
      kept[a.n_keep - a.n_recent + i] = t - a.n_recent + i;
      wo[a.n_keep - a.n_recent + i] = x;
    }
  }
  if (MOVES) {
    __syncthreads();
    move_rows(a, kvh, b, a.n_keep, kept);
  }
}

// Rows to other pages: grid (segments, 2 * Hkv, n_seqs).  A warp takes 32 kept rows: each lane looks up one row's source and
// destination (the chain kept index -> page -> row is walked once for 32 rows), then the warp copies the rows, four
// 512-byte pieces in flight at a time and six CTAs to an SM.  (With every thread walking the chain for its own chunks: 40 us
// for 4 x 4096 -> 2048 with the selection; eight pieces in flight and three CTAs, one and a half waves: 31.2; this: 26.5.)
constexpr int MV_THREADS = 256, MV_ROWS = MV_THREADS;
template <int D>
__global__ void __launch_bounds__(MV_THREADS, 6) evict_move_kernel(EvictArgs a) {
  constexpr int CPR = D / 8, RPI = 32 / CPR, UNROLL = 4;  // 16-byte chunks per row, rows per warp-wide access
  pdl_wait();
  pdl_trigger();
  const int kind = blockIdx.y & 1, kvh = blockIdx.y >> 1, b = blockIdx.z;
  const int lane = threadIdx.x & 31;
  const int len = min(min(max(a.cached[b], 0), a.table_stride * 16), a.n_keep);
  const int i = blockIdx.x * MV_ROWS + (threadIdx.x & ~31) + lane;
  const int rows = min(32, len - (i - lane));
  if (rows <= 0) return;
  // rows are numbered through the pool: 2^32 of them are more than any pool has
  uint32_t from = 0, to = 0;
  if (i < len) {
    const int s = a.kept[((long long)b * a.Hkv + kvh) * a.n_keep + i];
    const int32_t src_page = a.table[(long long)b * a.table_stride + (s >> 4)], dst_page = a.dst_table[(long long)b * a.dst_stride + (i >> 4)];
    from = (((uint32_t)src_page * 2 + kind) * a.Hkv + kvh) * 16 + (s & 15);
    to = (((uint32_t)dst_page * 2 + kind) * a.Hkv + kvh) * 16 + (i & 15);
  }
  const int c = lane % CPR, sub = lane / CPR;
#pragma unroll 1
  for (int it = 0; it < 32; it += UNROLL * RPI) {
    if (it >= rows) return;
    uint4 v[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int r = it + u * RPI + sub;
      const uint32_t row = __shfl_sync(0xffffffffu, from, r);
      if (r < rows) v[u] = __ldcs(reinterpret_cast<const uint4*>(a.pool + (size_t)row * D + ((c ^ (row & 7)) << 3)));
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int r = it + u * RPI + sub;
      const uint32_t row = __shfl_sync(0xffffffffu, to, r);
      if (r < rows) *reinterpret_cast<uint4*>(a.dst + (size_t)row * D + ((c ^ (row & 7)) << 3)) = v[u];
    }
  }
}

// In place: grid (2 * Hkv, n_seqs); the CTA goes up the rows and reads each batch completely before it writes it.
constexpr int MI_THREADS = 512, MI_UNROLL = 4;
template <int D>
__global__ void __launch_bounds__(MI_THREADS) evict_move_in_place_kernel(EvictArgs a) {
  constexpr int CPR = D / 8, STEP = MI_THREADS / CPR;  // 16-byte chunks per row, rows per pass
  pdl_wait();
  pdl_trigger();
  const int kind = blockIdx.x & 1, kvh = blockIdx.x >> 1, b = blockIdx.y;
  const int len = min(min(max(a.cached[b], 0), a.table_stride * 16), a.n_keep);
  const int32_t* kept = a.kept + ((long long)b * a.Hkv + kvh) * a.n_keep;
  const int32_t* bt = a.table + (long long)b * a.table_stride;
  const int c = threadIdx.x % CPR, r = threadIdx.x / CPR;
  auto row_at = [&](int32_t page, int slot) { return ((((size_t)page * 2 + kind) * a.Hkv + kvh) * 16 + slot) * D; };
  for (int i0 = 0; i0 < len; i0 += STEP * MI_UNROLL) {
    uint4 v[MI_UNROLL];
    int src[MI_UNROLL];
#pragma unroll
    for (int u = 0; u < MI_UNROLL; ++u) {
      const int i = i0 + u * STEP + r;
      src[u] = i < len ? kept[i] : -1;
      if (src[u] == i) src[u] = -1;  // the row stays where it is
    }
#pragma unroll
    for (int u = 0; u < MI_UNROLL; ++u)
      if (src[u] >= 0) v[u] = *reinterpret_cast<const uint4*>(a.pool + row_at(bt[src[u] >> 4], src[u] & 15) + ((c ^ (src[u] & 7)) << 3));
    __syncthreads();  // the whole batch is read before any of it is written
#pragma unroll
    for (int u = 0; u < MI_UNROLL; ++u) {
      const int i = i0 + u * STEP + r;
      if (src[u] >= 0) *reinterpret_cast<uint4*>(a.dst + row_at(bt[i >> 4], i & 15) + ((c ^ (i & 7)) << 3)) = v[u];
    }
  }
}

template <int D>
int launch_move(const EvictArgs& a, cudaStream_t st) {
  if (a.in_place)
    HYP_CUDA_TRY(launch_pdl<2>(evict_move_in_place_kernel<D>, dim3(2 * a.Hkv, a.n_seqs), dim3(MI_THREADS), (size_t)0, st, a));
  else
    HYP_CUDA_TRY(launch_pdl<2>(evict_move_kernel<D>, dim3((a.n_keep + MV_ROWS - 1) / MV_ROWS, 2 * a.Hkv, a.n_seqs), dim3(MV_THREADS),
                               (size_t)0, st, a));
  return 1;
}

}  // namespace

int launch_kv_evict(const EvictArgs& a, cudaStream_t st) {
  if (a.D != 64 && a.D != 128) return HYP_EINVAL;
  const long long most = (long long)a.table_stride * 16 - a.n_sink - a.n_recent;  // candidates a sequence can have
  if (most <= EV_STRIPES * EV_THREADS) {
    const size_t smem = most > 0 ? (size_t)most * sizeof(float) : 0;
    constexpr int most_smem = EV_STRIPES * EV_THREADS * (int)sizeof(float);
    const bool moves = a.n_keep <= move_here_rows(a.D) && (long long)a.n_seqs * a.Hkv <= sm_count();
    const int rc = moves ? allow_smem<evict_select_kernel<true, true>>(most_smem) : allow_smem<evict_select_kernel<true, false>>(most_smem);
    if (rc) return rc;
    HYP_CUDA_TRY(launch_pdl<2>(moves ? evict_select_kernel<true, true> : evict_select_kernel<true, false>, dim3(a.Hkv, a.n_seqs), dim3(EV_THREADS),
                               smem, st, a));
    if (moves) return 1;
  } else {
    HYP_CUDA_TRY(launch_pdl<2>(evict_select_kernel<false, false>, dim3(a.Hkv, a.n_seqs), dim3(EV_THREADS), (size_t)0, st, a));
  }
  const int rc = a.D == 128 ? launch_move<128>(a, st) : launch_move<64>(a, st);
  return rc < 0 ? rc : 1 + rc;
}

}  // namespace hyp
