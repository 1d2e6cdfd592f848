// Microscaled 4-bit floating point: a matrix to codes and block exponents, back, and to the packed form of the product.
//
// Four threads take a block of 32 values, eight each: the block's largest magnitude by two shuffles, the exponent
// floor(log2 amax) - 2 from its bits (so that amax lands in [4, 8), where 6 is the largest code: what lies above 6 saturates),
// every value times the exact inverse power, rounded to E2M1 by the hardware conversion (nearest, ties to even).  Bound by HBM: one
// pass, 16-byte loads.
#include "mx4.cuh"

namespace hyp {

namespace {

constexpr int QT = 256;

template <int TYPE>
__global__ void __launch_bounds__(QT) mx4_quantize_kernel(const void* __restrict__ x, int N, int K8, long long x_stride,
                                                          uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, int blocks) {
  constexpr int SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  const int per_row = 4 * blocks;  // threads of a row; those behind K take zeros
  const long long i = (long long)blockIdx.x * QT + threadIdx.x;
  const long long row = i / per_row;
  const int c = (int)(i - row * per_row);
  const bool in = row < N && c < K8;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  pdl_wait();
  if (in) load8<TYPE>(reinterpret_cast<const uint8_t*>(x) + (row * x_stride + 8 * c) * SIZE, v);
  uint32_t m = absmax_bits(v);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const bool bad = m >= 0x7f800000u;
  const int e = max((int)(m >> 23) - 127 - 2, -127);  // amax below 2^-126 included: it is far below 2^-127 * 4
  const float inv = pow2(-e);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = bad ? 0.f : v[k] * inv;
  if (in) codes[row * K8 + c] = to_e2m1x8(v);
  if (row < N && (c & 3) == 0) scales[row * blocks + (c >> 2)] = bad ? 255 : (uint8_t)(m == 0u ? 0 : e + 127);
  pdl_trigger();
}

template <int TYPE>
__global__ void __launch_bounds__(QT) mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int N,
                                                            int K8, int blocks, void* __restrict__ out, long long out_stride) {
  constexpr int SIZE = TYPE == HYP_TYPE_F32 ? 4 : 2;
  const long long i = (long long)blockIdx.x * QT + threadIdx.x;
  pdl_wait();
  if (i < (long long)N * K8) {
    const long long row = i / K8;
    const int c = (int)(i - row * K8);
    const int s = scales[row * blocks + (c >> 2)];
    const float f = s == 255 ? __uint_as_float(0x7fffffffu) : pow2(s - 127);
    uint32_t h[4], w[4];
    e2m1x8_to_half2(codes[i], h);
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 t = half2_values(h[k]);
      v[2 * k] = t.x * f;
      v[2 * k + 1] = t.y * f;
    }
    uint8_t* o = reinterpret_cast<uint8_t*>(out) + (row * out_stride + 8 * c) * SIZE;
    if (TYPE == HYP_TYPE_F32) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = TYPE == HYP_TYPE_BF16 ? pack_bf16(v[2 * k], v[2 * k + 1])
               : s == 255            ? 0x7fff7fffu
                                     : pack_f16_sat(v[2 * k], v[2 * k + 1]);
      *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  pdl_trigger();
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

}  // namespace

int launch_mx4_quantize(const void* x, int type, int N, int K, long long x_stride, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int blocks = (K + MX_BLOCK - 1) / MX_BLOCK;
  const long long ctas = ((long long)N * 4 * blocks + QT - 1) / QT;
  if (ctas > 0x7fffffffll) return HYP_ECAPACITY;
  auto go = [&](auto kernel) { return launch_pdl<2>(kernel, dim3((unsigned)ctas), dim3(QT), (size_t)0, st, x, N, K / 8, x_stride, (uint32_t*)codes, scales, blocks); };
  HYP_CUDA_TRY(type == HYP_TYPE_F32 ? go(mx4_quantize_kernel<HYP_TYPE_F32>)
               : type == HYP_TYPE_F16 ? go(mx4_quantize_kernel<HYP_TYPE_F16>) : go(mx4_quantize_kernel<HYP_TYPE_BF16>));
  return 1;
}

int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int N, int K, int type, void* out, long long out_stride, cudaStream_t st) {
  const int blocks = (K + MX_BLOCK - 1) / MX_BLOCK;
  const long long ctas = ((long long)N * (K / 8) + QT - 1) / QT;
  if (ctas > 0x7fffffffll) return HYP_ECAPACITY;
  auto go = [&](auto kernel) { return launch_pdl<2>(kernel, dim3((unsigned)ctas), dim3(QT), (size_t)0, st, (const uint32_t*)codes, scales, N, K / 8, blocks, out, out_stride); };
  HYP_CUDA_TRY(type == HYP_TYPE_F32 ? go(mx4_dequantize_kernel<HYP_TYPE_F32>)
               : type == HYP_TYPE_F16 ? go(mx4_dequantize_kernel<HYP_TYPE_F16>) : go(mx4_dequantize_kernel<HYP_TYPE_BF16>));
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
