// Microscaled 4-bit floating point: a matrix to codes and block exponents, back, and to the packed form of the product.
//
// A warp takes a run of a row, a lane eight values at a time, so that four lanes hold a block of 32: the block's largest magnitude by
// two shuffles, the exponent floor(log2 amax) - 2 from its bits (amax lands in [4, 8), where 6 is the largest code: what lies above
// saturates), every value times the exact inverse power, rounded to E2M1 by the hardware conversion (nearest, ties to even).
// Bound by HBM: 17920 x 5120 bf16 values to codes and back, 464 MB in 79 us = 5.9 TB/s (one pass, 16-byte loads, up to four in flight a lane); next
// by issue slots: with a division by the row length in every thread and eight values to a thread it took 114 us.
#include "mx4.cuh"

namespace hyp {

namespace {

constexpr int QT = 256, QW = QT / 32;

// grid (rows / 8, segments of 32 U chunks); a chunk is eight values
template <int TYPE, int U>
__global__ void __launch_bounds__(QT) mx4_quantize_kernel(const uint8_t* __restrict__ x, int N, int K8, long long x_stride,
                                                          uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, int blocks) {
  constexpr int SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  const int lane = threadIdx.x & 31, row = blockIdx.x * QW + (threadIdx.x >> 5), c0 = blockIdx.y * (32 * U) + lane;
  pdl_wait();
  pdl_trigger();
  if (row >= N) return;
  const uint8_t* src = x + (row * x_stride + 8ll * c0) * SIZE;
  uint32_t* to = codes + (long long)row * K8 + c0;
  uint8_t* sc = scales + (long long)row * blocks + (c0 >> 2);
  float v[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (c0 + 32 * u < K8) {
      load8<TYPE>(src + 32 * u * 8 * SIZE, v[u]);
    } else {  // behind K: zeros
#pragma unroll
      for (int k = 0; k < 8; ++k) v[u][k] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t m = __float_as_uint(absmax_nan(v[u]));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const bool bad = m >= 0x7f800000u;
    const int e = max((int)(m >> 23) - 127 - 2, -127);  // amax below 2^-126 included: it is far below 4 * 2^-127
    const float inv = bad ? 0.f : pow2(-e);
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = v[u][k] * inv;
    const int c = c0 + 32 * u;
    if (c < K8) to[32 * u] = bad ? 0u : to_e2m1x8(y);
    if (c < K8 && (c & 3) == 0) sc[8 * u] = bad ? 255 : (uint8_t)(m == 0u ? 0 : e + 127);
  }
}

template <int TYPE, int U>
__global__ void __launch_bounds__(QT) mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int N,
                                                            int K8, int blocks, uint8_t* __restrict__ out, long long out_stride) {
  constexpr int SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  const int lane = threadIdx.x & 31, row = blockIdx.x * QW + (threadIdx.x >> 5), c0 = blockIdx.y * (32 * U) + lane;
  pdl_wait();
  pdl_trigger();
  if (row >= N) return;
  const uint32_t* src = codes + (long long)row * K8 + c0;
  const uint8_t* sc = scales + (long long)row * blocks + (c0 >> 2);
  uint8_t* to = out + (row * out_stride + 8ll * c0) * SIZE;
  uint32_t q[U];
  int s[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool in = c0 + 32 * u < K8;
    q[u] = in ? src[32 * u] : 0u;
    s[u] = in ? sc[8 * u] : 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (c0 + 32 * u >= K8) continue;
    const float f = s[u] == 255 ? __uint_as_float(0x7fffffffu) : pow2(s[u] - 127);
    uint32_t h[4], w[4];
    e2m1x8_to_half2(q[u], h);
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 t = half2_values(h[k]);
      v[2 * k] = t.x * f;
      v[2 * k + 1] = t.y * f;
    }
    uint8_t* o = to + 32 * u * 8 * SIZE;
    if (TYPE == HYP_TYPE_F32) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = TYPE == HYP_TYPE_BF16 ? pack_bf16(v[2 * k], v[2 * k + 1]) : half2_sat(v[2 * k], v[2 * k + 1]);
      *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// One thread for a row's 32 k of a block: 16 bytes of codes and their scale.
__global__ void __launch_bounds__(QT) mx4_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int N, int K,
                                                      int KB, int tiles, long long total, uint8_t* __restrict__ packed) {
  const long long i = (long long)blockIdx.x * QT + threadIdx.x;
  if (i >= total) return;
  const int j = (int)(i & 3), r = (int)(i >> 2) & (MX_ROWS - 1);
  const long long blk = i / (4 * MX_ROWS);
  const int kb = (int)(blk % KB);
  const long long tile = blk / KB;                     // gate tiles, then up tiles
  const int half = (int)(tile / tiles), n = (int)(tile % tiles) * MX_ROWS + r;
  const int b = 4 * kb + j, k0 = MX_BLOCK * b;
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  uint8_t s = 127;
  if (n < N && k0 < K) {
    const long long row = (long long)half * N + n;
    const uint8_t* src = codes + row * (K / 2) + k0 / 2;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (k0 + 8 * q < K) w[q] = *reinterpret_cast<const uint32_t*>(src + 4 * q);
    s = scales[row * ((K + MX_BLOCK - 1) / MX_BLOCK) + b];
  }
  uint8_t* dst = packed + blk * MX_PACK_BYTES;
  *reinterpret_cast<uint4*>(dst + 64 * r + 16 * j) = make_uint4(w[0], w[1], w[2], w[3]);
  dst[MX_CODE_BYTES + (r & 31) * 16 + (r >> 5) * 4 + j] = s;
}

// Long rows: four chunks a lane; short ones: one.
template <template <int, int> class F, int U, typename... A>
cudaError_t by_type(int type, A... a) {
  return type == HYP_TYPE_F32 ? F<HYP_TYPE_F32, U>::go(a...) : type == HYP_TYPE_F16 ? F<HYP_TYPE_F16, U>::go(a...) : F<HYP_TYPE_BF16, U>::go(a...);
}
dim3 matrix_grid(int N, int K8, int u) { return dim3((unsigned)((N - 1) / QW + 1), (unsigned)((K8 + 32 * u - 1) / (32 * u))); }
template <int TYPE, int U>
struct Quantize {
  static cudaError_t go(const void* x, int N, int K, long long stride, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
    return launch_pdl<2>(mx4_quantize_kernel<TYPE, U>, matrix_grid(N, K / 8, U), dim3(QT), (size_t)0, st, (const uint8_t*)x, N, K / 8, stride,
                         (uint32_t*)codes, scales, (K + MX_BLOCK - 1) / MX_BLOCK);
  }
};
template <int TYPE, int U>
struct Dequantize {
  static cudaError_t go(const uint8_t* codes, const uint8_t* scales, int N, int K, void* out, long long stride, cudaStream_t st) {
    return launch_pdl<2>(mx4_dequantize_kernel<TYPE, U>, matrix_grid(N, K / 8, U), dim3(QT), (size_t)0, st, (const uint32_t*)codes, scales, N,
                         K / 8, (K + MX_BLOCK - 1) / MX_BLOCK, (uint8_t*)out, stride);
  }
};
bool wide_rows(int K) { return K > 1024; }

}  // namespace

int launch_mx4_quantize(const void* x, int type, int N, int K, long long x_stride, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  HYP_CUDA_TRY((wide_rows(K) ? by_type<Quantize, 4>(type, x, N, K, x_stride, codes, scales, st)
                            : by_type<Quantize, 1>(type, x, N, K, x_stride, codes, scales, st)));
  return 1;
}

int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int N, int K, int type, void* out, long long out_stride, cudaStream_t st) {
  HYP_CUDA_TRY((wide_rows(K) ? by_type<Dequantize, 4>(type, codes, scales, N, K, out, out_stride, st)
                            : by_type<Dequantize, 1>(type, codes, scales, N, K, out, out_stride, st)));
  return 1;
}

int launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int N, int K, int halves, uint8_t* packed, cudaStream_t st) {
  const int tiles = mx_row_tiles(N), KB = mx_kb(K);
  const long long total = (long long)halves * tiles * KB * 4 * MX_ROWS, ctas = (total + QT - 1) / QT;
  if (ctas > 0x7fffffffll) return HYP_ECAPACITY;
  mx4_pack_kernel<<<(unsigned)ctas, QT, 0, st>>>(codes, scales, N, K, KB, tiles, total, packed);
  return 1;
}

}  // namespace hyp
