// Writing the 8-bit paged cache and reading it back.
#include "kv8.cuh"
#include "mx4.cuh"
#include "sm100_common.cuh"

namespace hyp {

namespace {

constexpr float KV8_LEAST = 0x1p-118f;  // rows whose largest magnitude is below this count as zeros: their scales would leave fp32's normal range

// Four consecutive values of a row as fp32.
template <int TYPE>
__device__ __forceinline__ void load4(const void* p, float (&v)[4]) {
  if (TYPE == HYP_TYPE_F32) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  } else {
    const uint2 r = *reinterpret_cast<const uint2*>(p);
    if (TYPE == HYP_TYPE_F16) {
      const float2 a = half2_values(r.x), b = half2_values(r.y);
      v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    } else {
      v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
    }
  }
}

// The sequence that owns row `row`: the last i with cu[i] <= row (all lanes give the same).  32 places at a time.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int n, int row, int lane) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int below = __popc(__ballot_sync(0xffffffffu, at < hi && cu[at] <= row));
    lo += max(below - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// Scale of a row from its largest magnitude.  int8: amax / 127 rounded to fp32 once.  The product with the rounded 1 / 127 is less than a step
// of fp64 off the quotient, which never lies that near to the middle of two fp32 numbers for a 24-bit amax, but does for one in 2^27 or so of
// 53 bits: a product that came out as a middle goes a step to where the quotient lies.  e4m3: the least power of two p with amax <= 448 p.
template <int FMT>
__device__ __forceinline__ float row_scale(double amax) {
  if (FMT == HYP_KV8_INT8) {
    double q = amax * (1.0 / 127.0);
    if ((__double2loint(q) & 0x1fffffff) == 0x10000000) {
      const double rest = fma(-127.0, q, amax);  // its sign is exact
      q = __longlong_as_double(__double_as_longlong(q) + (rest > 0.0 ? 1 : rest < 0.0 ? -1 : 0));
    }
    return (float)q;
  }
  const long long b = __double_as_longlong(amax);
  return pow2((int)(b >> 52) - 1023 - 8 + ((b & 0xfffffffffffffll) > 0xc000000000000ll ? 1 : 0));
}
template <int FMT>
__device__ __forceinline__ float row_scale(float amax) {  // of values that were not rotated
  if (FMT == HYP_KV8_INT8) return (float)((double)amax * (1.0 / 127.0));
  return pow2(e4m3_exponent(__float_as_uint(amax)));
}
// x times an exact power of two, to fp32 rounded to odd, so that the rounding to E4M3 behind it is the only one.
__device__ __forceinline__ float odd_product(double x, double inv) {
  const double y = x * inv;
  const float f = __double2float_rz(y);
  return (double)f != y ? __uint_as_float(__float_as_uint(f) | 1u) : f;
}

// Four codes of values x[i] under scale s > 0; the values are off by at most `tol` from those meant (0: exact).  Returns false where some
// code hangs on what lies within tol: next to a border between two codes.
constexpr float ROUND_INT = 12582912.f;  // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
template <int FMT>
__device__ __forceinline__ bool fast_codes(const float (&x)[4], float tol, float s, uint32_t& w) {
  if (FMT == HYP_KV8_INT8) {
    float inv;  // near enough: the rest decides
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const float most = fmaf(0.5f, s, -tol);
    uint32_t q[4];
    bool sure = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = fmaf(x[i], inv, ROUND_INT + 128.f);
      const float r = fmaf(-(t - (ROUND_INT + 128.f)), s, x[i]);  // without rounding: the code has 8 bits, s 24, the rest is at most s
      sure = sure && fabsf(r) < most;
      q[i] = __float_as_uint(t);
    }
    w = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    return sure;
  }
  const float inv = __uint_as_float(0x7f000000u - __float_as_uint(s));  // 1 / s, a power of two in [2^-121, 2^126]
  w = to_e4m3x2(x[0] * inv, x[1] * inv) | to_e4m3x2(x[2] * inv, x[3] * inv) << 16;
  if (tol == 0.f) return true;
  const uint32_t lo = to_e4m3x2((x[0] - tol) * inv, (x[1] - tol) * inv) | to_e4m3x2((x[2] - tol) * inv, (x[3] - tol) * inv) << 16;
  const uint32_t hi = to_e4m3x2((x[0] + tol) * inv, (x[1] + tol) * inv) | to_e4m3x2((x[2] + tol) * inv, (x[3] + tol) * inv) << 16;
  return lo == hi;
}
// The same from fp64 values, exactly: nearest, ties to even.
template <int FMT>
__device__ __noinline__ uint32_t exact_codes(double x0, double x1, double x2, double x3, float s) {
  const double x[4] = {x0, x1, x2, x3}, inv = 1.0 / (double)s;
  if (FMT == HYP_KV8_INT8) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int q = __double2int_rn(x[i] * inv);
      const double r = fma((double)-q, (double)s, x[i]), twice = 2.0 * fabs(r);
      if (twice > (double)s || (twice == (double)s && (q & 1))) q += r < 0.0 ? -1 : 1;
      w |= (uint32_t)(q + 128) << (8 * i);
    }
    return w;
  }
  return to_e4m3x2(odd_product(x[0], inv), odd_product(x[1], inv)) | to_e4m3x2(odd_product(x[2], inv), odd_product(x[3], inv)) << 16;
}

struct WriteArgs {
  const uint8_t* qkv;
  long long stride;
  const float* rope;  // [positions][D / 2] (cos, sin), or null
  int rope_positions;
  uint8_t* pool;
  const int32_t* table;
  int table_stride;
  const int32_t* cu;
  const int32_t* ctx;
  __half* q_out;      // or null
  int n_seqs, M, Hq, Hkv;
  int per;            // heads of a CTA, a multiple of 128 / D
  int* err;
};

// grid (M, shares of the heads); ROPE: rotates.  One bulk copy brings a CTA's heads of a row to shared memory while the warps look up the row's sequence, page
// and angles; then D / 4 lanes take a head, four values each.
//   Bound by HBM for prompts (4096 fp32 rows of 60 heads of 128: 179 MB in 31-32 us, 5.6-5.8 TB/s), by latency for single tokens (8 rows: 2.5 us).
// Loads by the warps themselves, one head ahead, had 24 KB on their way on an SM: 46 us.  Warps hide a head's chain of steps: a rotation that
// is decided at run time costs 7-10 % (34 us; rows that are not rotated 9.9 instead of 8.1 for 2500), a CTA that walks over rows with the next one's
// look-ups ahead (64 registers) 55-80 %.  Six CTAs to an SM (rotating; eight otherwise) leave 40 (32) registers, for which most rotating forms, and the int8 ones at
// D = 64, spill 8 or 16 bytes.  With five (seven) append and read of 4096 rows of 60 heads, fp32, take 42.3 instead of 41.6 us in int8, 40.1 instead of 41.8 in
// e4m3, bf16 in int8 40.3, 40.9; 4096 rows of 40 heads of 64, bf16 in int8, 22.4, 20.7.
//   Codes have to be those of the exact value.  Exact arithmetic on every value costs more than the memory (in fp64 76 us for 4096 rows of 60
// heads, issue slots 84 % busy), so values are rotated and rounded in fp32, and fp64, in which products of fp32 numbers are exact, is
// used for the largest value of a row and where a code hangs on the rotation's roundings.  Those are two of half a step each, of a term and of
// the sum; as both members of the row's pairs are kept, neither exceeds 1.42 times the row's largest magnitude: 2^-22 of it covers them.
template <int D, int FMT, int TYPE, bool ROPE>
__global__ void __launch_bounds__(256, ROPE ? 6 : 8) kv8_write_kernel(const WriteArgs a) {
  constexpr int LANES = D / 4, PER = 32 / LANES, SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  extern __shared__ __align__(128) uint8_t wr_smem[];
  __shared__ uint64_t bar_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LANES, sub = lane / LANES;
  const uint32_t mine = LANES == 32 ? 0xffffffffu : 0xffffu << (16 * sub);  // the lanes of this head
  const int row = blockIdx.x, heads = a.Hq + 2 * a.Hkv;
  const int h_lo = (a.q_out ? 0 : a.Hq) + blockIdx.y * a.per, h_hi = min(h_lo + a.per, heads);
  const uint32_t bar = smem_u32(&bar_word);
  pdl_wait();
  pdl_trigger();
  if (row >= a.cu[a.n_seqs]) return;
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    const uint32_t bytes = (uint32_t)(h_hi - h_lo) * (D * SIZE);
    mbar_expect_tx(bar, bytes);
    bulk_load(smem_u32(wr_smem), a.qkv + ((long long)row * a.stride + (long long)h_lo * D) * SIZE, bytes, bar);
  }
  const int seq = sequence_of(a.cu, a.n_seqs, row, lane);
  const long long pos = (long long)a.ctx[seq] + (row - a.cu[seq]);
  const bool kept = row >= a.cu[seq] && pos >= 0 && pos < (long long)a.table_stride * 16;
  const int slot = (int)(pos & 15);
  uint8_t* page = a.pool + (kept ? (size_t)a.table[(long long)seq * a.table_stride + (pos >> 4)] * 2 * a.Hkv * kv8_half_page(D) : 0);
  float cs[8];  // (cos, sin) of this lane's four pairs, the sine with the sign of its term
  if (ROPE) {
    const long long at = min(max(pos, 0ll), (long long)a.rope_positions - 1);
    const float4* t = reinterpret_cast<const float4*>(a.rope + (at * (D / 2) + 4 * (l % (LANES / 2))) * 2);
    const float4 t0 = t[0], t1 = t[1];
    const float sign = l < LANES / 2 ? -1.f : 1.f;
    cs[0] = t0.x; cs[1] = t0.y * sign; cs[2] = t0.z; cs[3] = t0.w * sign; cs[4] = t1.x; cs[5] = t1.y * sign; cs[6] = t1.z; cs[7] = t1.w * sign;
  }
  const int code_at = slot * D + kv8_chunk<D>(l >> 2, slot) + 4 * (l & 3);
  __syncthreads();  // the barrier is set up
  if (!__all_sync(0xffffffffu, mbar_wait(bar, 0, nullptr))) {  // the lanes go on together, or not at all
    if (lane == 0) atomicCAS(a.err, 0, 35);
    if (threadIdx.x == 0) mbar_wait(bar, 0, nullptr);
    return;
  }
  const uint8_t* mine_at = wr_smem + 4 * l * SIZE;
  const int other = (l < LANES / 2 ? D / 2 : -D / 2) * SIZE;
  __half* q_to = a.q_out + (long long)row * a.Hq * D + 4 * l;
  for (int h0 = h_lo + warp * PER; h0 < h_hi; h0 += 8 * PER) {  // the warp's lanes stay together
    const int head = h0 + sub;
    const bool in = head < h_hi;
    const bool any_turn = ROPE && h0 < a.Hq + a.Hkv, turn = any_turn && head < a.Hq + a.Hkv;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f};  // own values and the other members of their pairs, D / 2 away
    if (in) load4<TYPE>(mine_at + (head - h_lo) * (D * SIZE), v);
    if (turn && in) load4<TYPE>(mine_at + (head - h_lo) * (D * SIZE) + other, o);
    float x[4] = {v[0], v[1], v[2], v[3]};
    if (turn) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = fmaf(v[i], cs[2 * i], o[i] * cs[2 * i + 1]);
    }
    if (head < a.Hq) *reinterpret_cast<uint2*>(q_to + (size_t)head * D) = make_uint2(half2_sat(x[0], x[1]), half2_sat(x[2], x[3]));
    if (h0 + PER <= a.Hq) continue;  // the whole warp holds queries
    const uint32_t own_top = max(max(__float_as_uint(x[0]) & 0x7fffffffu, __float_as_uint(x[1]) & 0x7fffffffu),
                                 max(__float_as_uint(x[2]) & 0x7fffffffu, __float_as_uint(x[3]) & 0x7fffffffu));
    const uint32_t top = __reduce_max_sync(mine, own_top);
    const bool bad = top >= 0x7f800000u;
    // the largest magnitude exactly: among the values whose fp32 form is within its error of the largest one
    float s = 0.f;
    bool some = __uint_as_float(top) >= KV8_LEAST;
    if (!any_turn) {
      s = row_scale<FMT>(__uint_as_float(top));
    } else {
      const float close = __uint_as_float(top) * (1.f - 0x1p-20f);
      double m = 0.0;
      if (turn && __uint_as_float(own_top) >= close) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (fabsf(x[i]) >= close) m = fmax(m, fabs(fma((double)v[i], (double)cs[2 * i], (double)o[i] * (double)cs[2 * i + 1])));
      }
      const uint32_t owners = __ballot_sync(0xffffffffu, m > 0.0) & mine;
      double best = __shfl_sync(0xffffffffu, m, owners ? __ffs(owners) - 1 : lane);  // every lane takes part, zeros among them
      if (__any_sync(0xffffffffu, __popc(owners) > 1)) {
        best = m;
#pragma unroll
        for (int k = LANES / 2; k > 0; k >>= 1) best = fmax(best, __shfl_xor_sync(0xffffffffu, best, k));
      }
      const double amax = turn ? best : (double)__uint_as_float(top);
      some = amax >= (double)KV8_LEAST;
      s = row_scale<FMT>(amax);
    }
    uint32_t w = FMT == HYP_KV8_INT8 ? 0x80808080u : 0u;
    if (bad || !some) {
      s = 0.f;
    } else {
      if (!fast_codes<FMT>(x, turn ? __uint_as_float(top) * 0x1p-22f : 0.f, s, w)) {
        double xd[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) xd[i] = turn ? fma((double)v[i], (double)cs[2 * i], (double)o[i] * (double)cs[2 * i + 1]) : (double)x[i];
        w = exact_codes<FMT>(xd[0], xd[1], xd[2], xd[3], s);
      }
    }
    if (head >= a.Hq && in && kept) {
      uint8_t* half_page = page + (size_t)(head - a.Hq) * kv8_half_page(D);  // value heads follow the key heads
      *reinterpret_cast<uint32_t*>(half_page + code_at) = w;
      if (l == 0) *reinterpret_cast<float*>(half_page + 16 * D + 4 * slot) = bad ? __uint_as_float(0x7fffffffu) : s;
    }
  }
}

// A warp takes half pages in turn: 16-byte chunks of codes, times their slot's scale, to two chunks of fp16.  Bound by HBM (4096 tokens of 10
// heads of 128: 53 MB in 10 us), small ones by latency (2.4 us).
template <int D, int FMT>
__global__ void __launch_bounds__(256) kv8_read_kernel(const uint8_t* __restrict__ pool, const int32_t* __restrict__ table, int table_stride,
                                                       const int32_t* __restrict__ first, const int32_t* __restrict__ lens, int Hkv,
                                                       __half* __restrict__ dst, const int32_t* __restrict__ dst_table, int dst_stride) {
  constexpr int CPR = D / 16, STEPS = 16 * CPR / 32;
  const int lane = threadIdx.x & 31, seq = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  const int most = min(table_stride, dst_stride) * 16;
  const int n = min(max(lens[seq], 0), most), n0 = first ? min(max(first[seq], 0), n) : 0;
  const int p0 = n0 / 16, pages = (n + 15) / 16 - p0;
  if (n0 >= n) return;
  const int units = pages * 2 * Hkv;
  for (int u = blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += gridDim.x * 8) {
    const int p = p0 + u / (2 * Hkv), hh = u % (2 * Hkv);
    const uint8_t* src = pool + kv8_half_offset(table[(long long)seq * table_stride + p], 0, hh, Hkv, D);
    __half* to = dst + ((size_t)dst_table[(long long)seq * dst_stride + p] * 2 * Hkv + hh) * 16 * D;
    uint4 r[STEPS];
    float s[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int at = i * 32 + lane, t = at / CPR;
      r[i] = *reinterpret_cast<const uint4*>(src + 16 * at);
      s[i] = *reinterpret_cast<const float*>(src + 16 * D + 4 * t);
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int at = i * 32 + lane, t = at / CPR, c = kv8_chunk<D>(at % CPR, t) >> 4;
      if (16 * p + t < n0 || 16 * p + t >= n) continue;
      const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
      uint32_t h[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float2 lo, hi;
        if (FMT == HYP_KV8_INT8) {  // a code below the exponent of 2^23, which then goes
          lo = make_float2(__uint_as_float(__byte_perm(w[k], 0x4b000000u, 0x7440)) - 8388736.f, __uint_as_float(__byte_perm(w[k], 0x4b000000u, 0x7441)) - 8388736.f);
          hi = make_float2(__uint_as_float(__byte_perm(w[k], 0x4b000000u, 0x7442)) - 8388736.f, __uint_as_float(__byte_perm(w[k], 0x4b000000u, 0x7443)) - 8388736.f);
        } else {
          lo = half2_values(e4m3x2_to_half2(w[k] & 0xffffu));
          hi = half2_values(e4m3x2_to_half2(w[k] >> 16));
        }
        h[2 * k] = half2_sat(lo.x * s[i], lo.y * s[i]);
        h[2 * k + 1] = half2_sat(hi.x * s[i], hi.y * s[i]);
      }
      uint4* row = reinterpret_cast<uint4*>(to + t * D);
      row[kv_chunk_pos(2 * c, t)] = make_uint4(h[0], h[1], h[2], h[3]);
      row[kv_chunk_pos(2 * c + 1, t)] = make_uint4(h[4], h[5], h[6], h[7]);
    }
  }
}

constexpr int WR_SMEM = 32 * 1024;  // of a row in a CTA
template <int D, int FMT, int TYPE>
int write_go(WriteArgs a, cudaStream_t st) {
  constexpr int PER = 128 / D, HEAD = D * (TYPE == HYP_TYPE_F32 ? 4 : 2);
  const int heads = (a.q_out ? a.Hq : 0) + 2 * a.Hkv;
  // few rows: down to a head (a pair at D = 64) for every warp; many: as much of a row as a CTA holds
  int y = (8 * sm_count() + a.M - 1) / a.M;
  const int most = (heads + 8 * PER - 1) / (8 * PER), least = (heads * HEAD + WR_SMEM - 1) / WR_SMEM;
  if (y > most) y = most;
  if (y < least) y = least;
  a.per = ((heads + y - 1) / y + PER - 1) / PER * PER;
  y = (heads + a.per - 1) / a.per;
  const dim3 grid((unsigned)a.M, (unsigned)y);
  HYP_CUDA_TRY((a.rope ? launch_pdl<2>(kv8_write_kernel<D, FMT, TYPE, true>, grid, dim3(256), (size_t)a.per * HEAD, st, a)
                       : launch_pdl<2>(kv8_write_kernel<D, FMT, TYPE, false>, grid, dim3(256), (size_t)a.per * HEAD, st, a)));
  return 1;
}
template <int D, int FMT>
int write_type(const WriteArgs& a, int type, cudaStream_t st) {
  if (type == HYP_TYPE_F32) return write_go<D, FMT, HYP_TYPE_F32>(a, st);
  if (type == HYP_TYPE_F16) return write_go<D, FMT, HYP_TYPE_F16>(a, st);
  return write_go<D, FMT, HYP_TYPE_BF16>(a, st);
}

}  // namespace

int launch_kv8_write(const Kv8View& c, int M, const void* qkv, int type, long long stride, const float* rope, int rope_positions,
                     const int32_t* cu_q, const int32_t* ctx, __half* q_out, int* err, cudaStream_t st) {
  WriteArgs a{};
  a.err = err;
  a.qkv = (const uint8_t*)qkv; a.stride = stride; a.rope = rope; a.rope_positions = rope_positions;
  a.pool = c.pool; a.table = c.table; a.table_stride = c.table_stride; a.cu = cu_q; a.ctx = ctx; a.q_out = q_out;
  a.n_seqs = c.n_seqs; a.M = M; a.Hq = c.Hq; a.Hkv = c.Hkv;
  if (c.D == 128) return c.fmt == HYP_KV8_INT8 ? write_type<128, HYP_KV8_INT8>(a, type, st) : write_type<128, HYP_KV8_E4M3>(a, type, st);
  return c.fmt == HYP_KV8_INT8 ? write_type<64, HYP_KV8_INT8>(a, type, st) : write_type<64, HYP_KV8_E4M3>(a, type, st);
}

int launch_kv8_read(const Kv8View& c, const int32_t* first, const int32_t* lens, __half* dst, const int32_t* dst_table, int dst_stride,
                    cudaStream_t st) {
  // The lengths are on the device: about eight CTAs to an SM share a sequence's half pages, whatever the table could hold.
  const long long units = (long long)(c.table_stride < dst_stride ? c.table_stride : dst_stride) * 2 * c.Hkv;
  long long x = (units + 7) / 8, most = (8ll * sm_count() + c.n_seqs - 1) / c.n_seqs;
  if (x > most) x = most;
  const dim3 grid((unsigned)x, (unsigned)c.n_seqs);
  auto go = [&](auto kernel) {
    return launch_pdl<2>(kernel, grid, dim3(256), (size_t)0, st, (const uint8_t*)c.pool, c.table, c.table_stride, first, lens, c.Hkv, dst,
                         dst_table, dst_stride);
  };
  if (c.D == 128)
    HYP_CUDA_TRY(c.fmt == HYP_KV8_INT8 ? go(kv8_read_kernel<128, HYP_KV8_INT8>) : go(kv8_read_kernel<128, HYP_KV8_E4M3>));
  else
    HYP_CUDA_TRY(c.fmt == HYP_KV8_INT8 ? go(kv8_read_kernel<64, HYP_KV8_INT8>) : go(kv8_read_kernel<64, HYP_KV8_E4M3>));
  return 1;
}

}  // namespace hyp
