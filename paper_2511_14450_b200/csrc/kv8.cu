// Writing the 8-bit paged cache and reading it back.
#include "kv8.cuh"
#include "mx4.cuh"

namespace hyp {

namespace {

constexpr float KV8_LEAST = 0x1p-118f;  // rows whose largest magnitude is below this count as zeros: their scales would leave fp32's normal range

__device__ __forceinline__ __half half_sat(float x) { return __float2half_rn(x != x ? x : fminf(fmaxf(x, -65504.f), 65504.f)); }
__device__ __forceinline__ uint32_t half2_sat(float a, float b) {
  const __half2 h = __halves2half2(half_sat(a), half_sat(b));
  return *reinterpret_cast<const uint32_t*>(&h);
}

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

// Scale of a row from its largest magnitude, in the arithmetic T of its values (fp32 as they came, fp64 where they were rotated).
// int8: amax / 127 rounded to fp32.  e4m3: the least power of two p with amax <= 448 p.
template <int FMT>
__device__ __forceinline__ float row_scale(float amax) {
  if (FMT == HYP_KV8_INT8) return __fdiv_rn(amax, 127.f);
  return pow2(e4m3_exponent(__float_as_uint(amax)));
}
template <int FMT>
__device__ __forceinline__ float row_scale(double amax) {
  if (FMT == HYP_KV8_INT8) return (float)(amax / 127.0);
  const long long b = __double_as_longlong(amax);
  return pow2((int)(b >> 52) - 1023 - 8 + ((b & 0xfffffffffffffll) > 0xc000000000000ll ? 1 : 0));
}

// The integer nearest to x / s, ties to even, exactly: the estimate from the product is off by one at most next to a border, and
// the remainder x - q s is formed without rounding (q has 8 bits, s 24; the difference is at most s).
__device__ __forceinline__ int to_int(float x) { return __float2int_rn(x); }
__device__ __forceinline__ int to_int(double x) { return __double2int_rn(x); }
template <typename T>
__device__ __forceinline__ int nearest_code(T x, float s, float inv) {
  int q = to_int(x * (T)inv);
  const T r = fma((T)-q, (T)s, x), twice = r < 0 ? -2 * r : 2 * r;
  if (twice > (T)s || (twice == (T)s && (q & 1))) q += r < 0 ? -1 : 1;
  return q;
}
// x times an exact power of two, to E4M3 (nearest, ties to even); fp64 goes to fp32 rounded to odd, so that it is not rounded twice.
__device__ __forceinline__ float e4m3_input(float x, float inv) { return x * inv; }
__device__ __forceinline__ float e4m3_input(double x, float inv) {
  const double y = x * (double)inv;
  const float f = __double2float_rz(y);
  return (double)f != y ? __uint_as_float(__float_as_uint(f) | 1u) : f;
}
template <int FMT, typename T>
__device__ __forceinline__ uint32_t four_codes(const T (&x)[4], float s) {
  if (FMT == HYP_KV8_INT8) {
    const float inv = s > 0.f ? 1.f / s : 0.f;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)(nearest_code(x[i], s, inv) + 128) << (8 * i);
    return w;
  }
  const float inv = s > 0.f ? 1.f / s : 0.f;  // exact: a power of two
  return to_e4m3x2(e4m3_input(x[0], inv), e4m3_input(x[1], inv)) | to_e4m3x2(e4m3_input(x[2], inv), e4m3_input(x[3], inv)) << 16;
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
};

// D / 4 lanes take a head of a row, four values each.
template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(256) kv8_write_kernel(const WriteArgs a) {
  constexpr int LANES = D / 4, PER = 32 / LANES, SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LANES;
  const int row = blockIdx.x;
  const int h0 = a.q_out ? 0 : a.Hq, heads = a.Hq + 2 * a.Hkv;
  const int head = h0 + (blockIdx.y * 8 + warp) * PER + lane / LANES;
  pdl_wait();
  pdl_trigger();
  if (row >= a.cu[a.n_seqs]) return;
  const bool in = head < heads;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (in) load4<TYPE>(a.qkv + ((long long)row * a.stride + (long long)head * D + 4 * l) * SIZE, v);
  const int seq = sequence_of(a.cu, a.n_seqs, row, lane);
  const long long pos = (long long)a.ctx[seq] + (row - a.cu[seq]);
  const bool turn = a.rope && in && head < a.Hq + a.Hkv;
  float cs[8];  // (cos, sin) of this lane's four pairs
  if (turn) {
    const long long at = min(max(pos, 0ll), (long long)a.rope_positions - 1);
    const float4* t = reinterpret_cast<const float4*>(a.rope + (at * (D / 2) + 4 * (l % (LANES / 2))) * 2);
    const float4 t0 = t[0], t1 = t[1];
    cs[0] = t0.x; cs[1] = t0.y; cs[2] = t0.z; cs[3] = t0.w; cs[4] = t1.x; cs[5] = t1.y; cs[6] = t1.z; cs[7] = t1.w;
  }
  float o[4];  // the other member of each pair, D / 2 away
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __shfl_xor_sync(0xffffffffu, v[i], LANES / 2);
  const float sign = l < LANES / 2 ? -1.f : 1.f;

  if (in && head < a.Hq) {
    if (turn) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], cs[2 * i], sign * o[i] * cs[2 * i + 1]);
    }
    *reinterpret_cast<uint2*>(a.q_out + ((long long)row * a.Hq + head) * D + 4 * l) = make_uint2(half2_sat(v[0], v[1]), half2_sat(v[2], v[3]));
  }
  // A warp may hold heads of both kinds: everybody takes part in the reductions.  Rotated keys are formed in fp64: the two products are
  // exact there, so a code does not depend on how a sum was rounded.
  const bool wide = __any_sync(0xffffffffu, turn && head >= a.Hq);
  double x[4];
  float m = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
  bool bad = !(isfinite(v[0]) && isfinite(v[1]) && isfinite(v[2]) && isfinite(v[3]));
  double md = 0.0;
  if (wide) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = turn ? fma((double)v[i], (double)cs[2 * i], (double)(sign * o[i]) * (double)cs[2 * i + 1]) : (double)v[i];
      md = fmax(md, fabs(x[i]));
      bad = bad || !isfinite(x[i]);
    }
  }
#pragma unroll
  for (int k = LANES / 2; k > 0; k >>= 1) {
    if (wide)
      md = fmax(md, __shfl_xor_sync(0xffffffffu, md, k));
    else
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    bad = (__shfl_xor_sync(0xffffffffu, (int)bad, k) != 0) || bad;
  }
  if (!in || head < a.Hq || pos < 0 || pos >= (long long)a.table_stride * 16) return;
  const int kvh = (head - a.Hq) % a.Hkv, kind = (head - a.Hq) / a.Hkv, slot = (int)(pos & 15);
  uint32_t w = FMT == HYP_KV8_INT8 ? 0x80808080u : 0u;
  float s = 0.f;
  if (!bad && (wide ? md >= (double)KV8_LEAST : m >= KV8_LEAST)) {
    s = wide ? row_scale<FMT>(md) : row_scale<FMT>(m);
    w = wide ? four_codes<FMT>(x, s) : four_codes<FMT>(v, s);
  }
  uint8_t* half_page = a.pool + kv8_half_offset(a.table[(long long)seq * a.table_stride + (pos >> 4)], kind, kvh, a.Hkv, D);
  *reinterpret_cast<uint32_t*>(half_page + slot * D + kv8_chunk<D>(l >> 2, slot) + 4 * (l & 3)) = w;
  if (l == 0) *reinterpret_cast<float*>(half_page + 16 * D + 4 * slot) = bad ? __uint_as_float(0x7fffffffu) : s;
}

// A warp takes half pages in turn: 16-byte chunks of codes, times their slot's scale, to two chunks of fp16.
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
        if (FMT == HYP_KV8_INT8) {
          lo = make_float2((float)((int)(w[k] & 255u) - 128), (float)((int)(w[k] >> 8 & 255u) - 128));
          hi = make_float2((float)((int)(w[k] >> 16 & 255u) - 128), (float)((int)(w[k] >> 24) - 128));
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

template <int D, int FMT, int TYPE>
int write_go(const WriteArgs& a, cudaStream_t st) {
  const int units = (a.q_out ? a.Hq : 0) + 2 * a.Hkv, per_cta = 8 * (128 / D);
  HYP_CUDA_TRY(launch_pdl<2>(kv8_write_kernel<D, FMT, TYPE>, dim3((unsigned)a.M, (unsigned)((units + per_cta - 1) / per_cta)), dim3(256),
                             (size_t)0, st, a));
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
                     const int32_t* cu_q, const int32_t* ctx, __half* q_out, cudaStream_t st) {
  WriteArgs a{};
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
