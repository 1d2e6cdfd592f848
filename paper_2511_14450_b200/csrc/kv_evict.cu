// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) the first n_sink tokens, the
// last n_recent tokens and the heaviest of the others stay, in their order, n_keep in all.
//
//   select kernel: grid (Hkv, n_seqs), 1024 threads.  The weights between the protected ends become order-preserving
//   32-bit keys, held in registers (up to 32 per thread, read again from L2 for longer contexts), and the threshold -
//   the m-th largest key - is found bit pair by bit pair with three block-wide counts a step: no histogram, no atomics,
//   the same result on every run.  One ordered pass then writes the kept indexes and their weights; among keys equal to the
//   threshold the lowest indexes win.
//   move kernel: copies the kept rows, 16-byte chunks, re-permuted for their new slot.  Other pages: every row at its
//   own pace.  In place a row moves down or stays, so one CTA per (sequence, KV head, keys or values) goes up the rows and
//   reads each batch completely before it writes it: a batch writes at or below its own sources, never at a later one's.
// The move is bound by HBM (every kept row read and written once), the selection by its block-wide steps.
#include "cache_ops.cuh"
#include "hyperion.h"

namespace hyp {

namespace {

constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32, EV_NPT = 32;

// Keys ascend with the weight; -0 equals +0, NaN counts as -infinity.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) w = __int_as_float(0xff800000);
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Number of the block's keys >= each of three bounds.  buf: [2][EV_WARPS][3], alternating, so one barrier a call is enough.
struct Counts {
  int a, b, c;
};
__device__ __forceinline__ Counts block_counts(int a, int b, int c, int (*buf)[3]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  a = __reduce_add_sync(0xffffffffu, a);
  b = __reduce_add_sync(0xffffffffu, b);
  c = __reduce_add_sync(0xffffffffu, c);
  if (lane == 0) {
    buf[warp][0] = a;
    buf[warp][1] = b;
    buf[warp][2] = c;
  }
  __syncthreads();
  Counts r;
  r.a = __reduce_add_sync(0xffffffffu, buf[lane][0]);
  r.b = __reduce_add_sync(0xffffffffu, buf[lane][1]);
  r.c = __reduce_add_sync(0xffffffffu, buf[lane][2]);
  return r;
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(EvictArgs a) {
  __shared__ int counts[2][EV_WARPS][3];
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
    return;
  }
  const int r0 = a.n_sink, n = t - a.n_sink - a.n_recent;  // candidates w[r0 .. r0 + n), of which m stay; n > m
  const int m = a.n_keep - a.n_sink - a.n_recent;

  // threshold: the m-th largest key; `all`: exactly m keys are >= it
  uint32_t thr = 0;
  bool all = false;
  int greater = 0;
  if (m > 0) {
    uint32_t key[EV_NPT];
    const bool in_regs = n <= EV_NPT * EV_THREADS;
    if (in_regs) {
#pragma unroll
      for (int i = 0; i < EV_NPT; ++i) {
        const int k = i * EV_THREADS + tid;
        key[i] = k < n ? weight_key(w[r0 + k]) : 0u;  // 0 is below every key of a number
      }
    }
    int turn = 0;
    auto count3 = [&](uint32_t c1, uint32_t c2, uint32_t c3) {  // c1 <= c2 <= c3, all > 0
      int n1 = 0, n2 = 0, n3 = 0;
      if (in_regs) {
#pragma unroll
        for (int i = 0; i < EV_NPT; ++i)
          if (i * EV_THREADS < n) {
            n1 += key[i] >= c1;
            n2 += key[i] >= c2;
            n3 += key[i] >= c3;
          }
      } else {
        for (int k = tid; k < n; k += EV_THREADS) {
          const uint32_t v = weight_key(w[r0 + k]);
          n1 += v >= c1;
          n2 += v >= c2;
          n3 += v >= c3;
        }
      }
      turn ^= 1;
      return block_counts(n1, n2, n3, counts[turn]);
    };
    for (int bit = 30; bit >= 0 && !all; bit -= 2) {
      const uint32_t c1 = thr | (1u << bit), c2 = thr | (2u << bit), c3 = thr | (3u << bit);
      const Counts r = count3(c1, c2, c3);
      if (r.c >= m) thr = c3, all = r.c == m;
      else if (r.b >= m) thr = c2, all = r.b == m;
      else if (r.a >= m) thr = c1, all = r.a == m;
    }
    if (!all) {
      const Counts r = count3(thr + 1, thr + 1, thr + 1);  // thr < 0xffffffff: that pattern is no number's key
      greater = r.a;
    }
  }
  const int need_eq = all ? n : m - greater;  // how many of the keys equal to the threshold stay

  // ordered pass: stripes of 1024 candidates; (greater, equal) counts in one word
  for (int i = tid; i < a.n_sink; i += EV_THREADS) {
    kept[i] = i;
    wo[i] = w[i];
  }
  __syncthreads();
  __shared__ uint2 totals[2][EV_WARPS];
  uint32_t gt_base = 0, eq_base = 0;
  int turn = 0;
  for (int s = 0; s < n && m > 0; s += EV_THREADS, turn ^= 1) {
    const int k = s + tid;
    const float v = k < n ? w[r0 + k] : 0.f;
    const uint32_t key = k < n ? weight_key(v) : 0u;
    const bool gt = k < n && key > thr, eq = k < n && key == thr;
    const uint32_t mg = __ballot_sync(0xffffffffu, gt), me = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) totals[turn][warp] = make_uint2(__popc(mg), __popc(me));
    __syncthreads();  // also: this stripe has been read before any of it is written
    const uint2 tl = totals[turn][lane];
    const uint32_t before_g = __reduce_add_sync(0xffffffffu, lane < warp ? tl.x : 0u);
    const uint32_t before_e = __reduce_add_sync(0xffffffffu, lane < warp ? tl.y : 0u);
    const uint32_t below = (1u << lane) - 1u;
    const int g_before = (int)(gt_base + before_g + __popc(mg & below)), e_before = (int)(eq_base + before_e + __popc(me & below));
    if (gt || (eq && e_before < need_eq)) {
      const int pos = r0 + g_before + min(e_before, need_eq);
      kept[pos] = r0 + k;
      wo[pos] = v;
    }
    gt_base += __reduce_add_sync(0xffffffffu, tl.x);
    eq_base += __reduce_add_sync(0xffffffffu, tl.y);
  }
  for (int s = 0; s < a.n_recent; s += EV_THREADS) {
    const int i = s + tid;
    const float v = i < a.n_recent ? w[t - a.n_recent + i] : 0.f;
    __syncthreads();
    if (i < a.n_recent) {
      kept[a.n_keep - a.n_recent + i] = t - a.n_recent + i;
      wo[a.n_keep - a.n_recent + i] = v;
    }
  }
}

// grid (segments, 2 * Hkv, n_seqs)
constexpr int MV_THREADS = 512, MV_UNROLL = 4;
template <int D, bool IN_PLACE>
__global__ void __launch_bounds__(MV_THREADS) evict_move_kernel(EvictArgs a, int rows_per_cta) {
  constexpr int CPR = D / 8, STEP = MV_THREADS / CPR;  // 16-byte chunks per row, rows per pass
  pdl_wait();
  pdl_trigger();
  const int kind = blockIdx.y & 1, kvh = blockIdx.y >> 1, b = blockIdx.z;
  const int len = min(min(max(a.cached[b], 0), a.table_stride * 16), a.n_keep);
  const int begin = blockIdx.x * rows_per_cta, end = min(len, begin + rows_per_cta);
  const int32_t* kept = a.kept + ((long long)b * a.Hkv + kvh) * a.n_keep;
  const int32_t* bt = a.table + (long long)b * a.table_stride;
  const int32_t* dt = a.dst_table + (long long)b * a.dst_stride;
  const int c = threadIdx.x % CPR, r = threadIdx.x / CPR;
  auto row_at = [&](int32_t page, int slot) {
    return ((((size_t)page * 2 + kind) * a.Hkv + kvh) * 16 + slot) * D;
  };
  for (int i0 = begin; i0 < end; i0 += STEP * MV_UNROLL) {
    uint4 v[MV_UNROLL];
    int src[MV_UNROLL];
#pragma unroll
    for (int u = 0; u < MV_UNROLL; ++u) {
      const int i = i0 + u * STEP + r;
      src[u] = i < end ? kept[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < MV_UNROLL; ++u)
      if (src[u] >= 0) v[u] = *reinterpret_cast<const uint4*>(a.pool + row_at(bt[src[u] >> 4], src[u] & 15) + ((c ^ (src[u] & 7)) << 3));
    if (IN_PLACE) __syncthreads();  // the whole batch is read before any of it is written
#pragma unroll
    for (int u = 0; u < MV_UNROLL; ++u) {
      const int i = i0 + u * STEP + r;
      if (src[u] >= 0 && !(IN_PLACE && src[u] == i))
        *reinterpret_cast<uint4*>(a.dst + row_at(dt[i >> 4], i & 15) + ((c ^ (i & 7)) << 3)) = v[u];
    }
  }
}

template <int D>
int launch_move(const EvictArgs& a, cudaStream_t st) {
  constexpr int BATCH = MV_THREADS / (D / 8) * MV_UNROLL;
  if (a.in_place) {
    HYP_CUDA_TRY(launch_pdl<2>(evict_move_kernel<D, true>, dim3(1, 2 * a.Hkv, a.n_seqs), dim3(MV_THREADS), (size_t)0, st, a, a.n_keep));
  } else {
    HYP_CUDA_TRY(launch_pdl<2>(evict_move_kernel<D, false>, dim3((a.n_keep + BATCH - 1) / BATCH, 2 * a.Hkv, a.n_seqs),
                               dim3(MV_THREADS), (size_t)0, st, a, BATCH));
  }
  return 1;
}

}  // namespace

int launch_kv_evict(const EvictArgs& a, cudaStream_t st) {
  if (a.D != 64 && a.D != 128) return HYP_EINVAL;
  HYP_CUDA_TRY(launch_pdl<2>(evict_select_kernel, dim3(a.Hkv, a.n_seqs), dim3(EV_THREADS), (size_t)0, st, a));
  const int rc = a.D == 128 ? launch_move<128>(a, st) : launch_move<64>(a, st);
  return rc < 0 ? rc : 1 + rc;
}

}  // namespace hyp
