// 8-bit MFMA GEMM: C = act(A W^T + bias), A [M,K] and W [N,K] e4m3, both K-contiguous, with a power-of-two scale for each
// 1 x 128 block of A and each 128 x 128 block of W; fp32 accumulate.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes the scales as operands: a lane gives one for its row and half of k (A fragment:
// lane holds row lane%32, 32 consecutive k starting at 32*(lane/32); B likewise for column lane%32; accumulator register
// i of a lane is row 8*(i/4) + 4*(lane/32) + i%4, column lane%32).  A block of 128 is two such steps, so
// scaling costs no instruction of its own and changes no bit of the products.  The waves accumulate C^T blocks (operands
// swapped), so a lane owns one row m and four consecutive columns n per accumulator quad.
#include "fp8_device.h"
#include "hero_kernels.h"

namespace {

// One wave a workgroup, 32 rows x 128 columns, fragments straight from memory: right for every size.
template <bool QUANT>
__global__ __launch_bounds__(64) void gemm_fp8_direct_kernel(GemmFp8Args g) {
  const int lane = threadIdx.x, lr = lane & 31, lh = lane >> 5;
  const int n0 = blockIdx.x * 128, m0 = blockIdx.y * 32;
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.a), 0, (uint32_t)g.m * (uint32_t)g.k, 0x00020000);
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.w), 0, (uint32_t)g.n * (uint32_t)g.k, 0x00020000);
  const int pitch = fp8_scale_pitch(g.k);
  const uint8_t* sa = g.a_scales + (int64_t)min(m0 + lr, g.m - 1) * pitch;
  const uint8_t* sw = g.w_scales + (int64_t)blockIdx.x * pitch;
  auto frag = [&](__amdgpu_buffer_rsrc_t rs, int row, int k0) {
    i32x8_t f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 32 * lh + 16 * h;
      const uint32_t off = k < g.k ? (uint32_t)row * (uint32_t)g.k + (uint32_t)k : 0xFFFFFFF0u;   // (past the buffer: zero)
      const auto t = __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * h + e] = (int)t[e];
    }
    return f;
  };
  floatx16_t acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
  for (int k = 0; k < g.k; k += 64) {
    const int scale_a = sa[k >> 7], scale_w = sw[k >> 7];
    const i32x8_t a = frag(ra, m0 + lr, k);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc[j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(rw, n0 + 32 * j + lr, k), a, acc[j], 0, 0, 0, scale_w, 0, scale_a);
  }
  const int m = m0 + lr;
  float largest = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = n0 + 32 * j + 8 * q + 4 * lh;
      u32x2_t bias = {0u, 0u};
      if (g.bias && n < g.n) bias = *reinterpret_cast<const u32x2_t*>(g.bias + n);
      float* v = reinterpret_cast<float*>(&acc[j]) + 4 * q;
      v[0] += unpack_lo(bias[0]); v[1] += unpack_hi(bias[0]);
      v[2] += unpack_lo(bias[1]); v[3] += unpack_hi(bias[1]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (g.gelu) v[e] = gelu_tanh(v[e]);
        largest = fmaxf(largest, n < g.n ? finite_size(v[e]) : 0.f);
      }
      if (!QUANT && m < g.m && n < g.n) {
        const u32x2_t out = {pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3])};
        *reinterpret_cast<u32x2_t*>(g.c + (int64_t)m * g.n + n) = out;
      }
    }
  if (!QUANT) return;
  const uint32_t byte = fp8_scale_of(fmaxf(largest, __shfl_xor(largest, 32, 64)));
  const float inv = fp8_inverse_scale(byte);
  if (m >= g.m) return;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = n0 + 32 * j + 8 * q + 4 * lh;
      const float* v = reinterpret_cast<const float*>(&acc[j]) + 4 * q;
      if (n < g.n) *reinterpret_cast<uint32_t*>(g.out.q + (int64_t)m * g.n + n) = pack_fp8x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    }
  if (lh == 0) {
    const int out_pitch = fp8_scale_pitch(g.n), last = blockIdx.x == gridDim.x - 1 ? out_pitch : (int)blockIdx.x + 1;
    for (int b = blockIdx.x; b < last; ++b) g.out.scales[(int64_t)m * out_pitch + b] = (uint8_t)(b == (int)blockIdx.x ? byte : FP8_SCALE_ONE);
  }
}

}  // namespace

hipError_t launch_gemm_fp8(const GemmFp8Args& g, hipStream_t st) {
  if (g.m <= 0 || g.n <= 0) return hipSuccess;
  if (g.k <= 0 || g.k % 16 != 0 || g.n % 16 != 0) return hipErrorInvalidValue;
  const dim3 grid((g.n + 127) / 128, (g.m + 31) / 32);
  if (grid.y > 65535) return hipErrorInvalidValue;
  if (g.out.q) hipLaunchKernelGGL(gemm_fp8_direct_kernel<true>, grid, dim3(64), 0, st, g);
  else hipLaunchKernelGGL(gemm_fp8_direct_kernel<false>, grid, dim3(64), 0, st, g);
  return hipGetLastError();
}
