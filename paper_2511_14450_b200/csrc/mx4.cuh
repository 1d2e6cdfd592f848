// Microscaled 4-bit weights: the packed form that the product reads, E4M3 / E2M1 conversions, launchers.
//
// A matrix w[n, k] in microscaled 4-bit floating point: blocks of 32 along k share a power of two 2^(s - 127) (one byte s, 255 =
// NaN), the values are E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the even k in the low half.
//
// Packed for the product: blocks of 128 rows x 128 k, all k-blocks of a row tile one after the other.  A block is 128 rows of 64
// bytes of codes, then the 512 bytes of its scales in the order in which they go to tensor memory: row r's scale of the 32-k block
// j at (r % 32) * 16 + (r / 32) * 4 + j.  So a CTA streams one run of memory.  Rows and k beyond the matrix are zeros under a
// scale of 1.  SwiGLU: the gate rows' tiles, then the up rows'.
#pragma once
#include "common.cuh"
#include "hyperion_ops.h"

namespace hyp {

constexpr int MX_ROWS = 128, MX_BK = 128, MX_BLOCK = 32;
constexpr int MX_CODE_BYTES = MX_ROWS * MX_BK / 2, MX_SF_BYTES = 512;
constexpr int MX_PACK_BYTES = MX_CODE_BYTES + MX_SF_BYTES;  // 136 lines of 64 bytes
inline int mx_row_tiles(int N) { return (N - 1) / MX_ROWS + 1; }
inline int mx_kb(int K) { return (K - 1) / MX_BK + 1; }
inline size_t mx4_packed_bytes(int N, int K, int halves) { return (size_t)halves * mx_row_tiles(N) * mx_kb(K) * MX_PACK_BYTES; }

// Exponent e of the least power of two with amax <= 448 * 2^e, by amax's bits (finite, not negative); -127 at least.
__device__ __forceinline__ int e4m3_exponent(uint32_t bits) {
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return bits == 0u || e < -127 ? -127 : e;
}
// 2^e for -127 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 0x00400000u); }
// two E4M3 codes, `lo` in the low byte
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
  return r;
}
// eight values to eight E2M1 codes, the first in the lowest bits
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// eight E2M1 codes to four pairs of fp16
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t v, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(v));
}
__device__ __forceinline__ float2 half2_values(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// fp32 -> fp16 pair, saturating at +-65504; NaN stays NaN
__device__ __forceinline__ uint32_t half2_sat(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Eight consecutive values of a matrix row as fp32 (16-byte loads; p aligned to 16 bytes).
template <int TYPE>
__device__ __forceinline__ void load8(const void* p, float (&v)[8]) {
  if (TYPE == HYP_TYPE_F32) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (TYPE == HYP_TYPE_F16) {
        const float2 f = half2_values(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      } else {
        v[2 * i] = bf16_lo(w[i]);
        v[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  }
}
__device__ __forceinline__ void unpack8(uint4 r, bool f16, float (&v)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = f16 ? half2_values(w[i]) : make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
// Largest magnitude of eight values, NaN if one is.
__device__ __forceinline__ float absmax_nan(const float (&v)[8]) {
  float m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) m[i] = fabsf(v[i]);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m[i]) : "f"(m[i + o]));
  return m[0];
}

int launch_mx4_quantize(const void* x, int type, int N, int K, long long x_stride, uint8_t* codes, uint8_t* scales, cudaStream_t st);
int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int N, int K, int type, void* out, long long out_stride, cudaStream_t st);
int launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int N, int K, int halves, uint8_t* packed, cudaStream_t st);

size_t mx4_scratch_bytes(int M, int K, int terms);
void mx4_plan(int M, int N, int K, int terms, bool swiglu, int32_t (&plan)[8]);  // as hyp_op_gemm_mx4_plan
int launch_gemm_mx4(const void* a, int a_type, long long a_stride, const uint8_t* packed, int M, int N, int K, int terms, int epi,
                    void* out, int ldo, uint8_t* scratch, cudaStream_t st);

}  // namespace hyp
