// Rows and weights in 8 bits (e4m3 elements, a power-of-two scale for each block of 128), by themselves or out of a
// root-mean-square norm that also adds the residual branch.
//
// A wave takes 512 neighbouring elements of a row at a time, eight a lane: 16 lanes hold a block, whose largest magnitude
// they find with four lane rotations, and the four scale bytes of the piece are one 32-bit word.  Everything here is
// bound by HBM: one pass, every byte read and written once.  Elements and sums are stored past the caches (nontemporal):
// 17776 x 1920 of bf16 with add and sum 50.5 -> 45.2 us, weight blocks 7680 x 1920 10.5 -> 9.1; nontemporal loads are
// slower (the same rms over 4485 listed rows 12.4 -> 14.1 us).  A float32 copy of 137 MB runs at 5.9 to 6.3 TB/s here.
#include <algorithm>

#include "fp8_device.h"
#include "hero_kernels.h"

namespace {

constexpr int PIECE = 512;                // elements of a wave's piece: four blocks

template <typename T>
__device__ __forceinline__ void store_past(T v, void* p) { __builtin_nontemporal_store(v, static_cast<T*>(p)); }

__device__ __forceinline__ void store8_past(float* p, const float* v) {
  store_past(floatx4_t{v[0], v[1], v[2], v[3]}, p);
  store_past(floatx4_t{v[4], v[5], v[6], v[7]}, p + 4);
}
__device__ __forceinline__ void store8_past(bf16_t* p, const float* v) {
  store_past(u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])}, p);
}

// A lane's eight elements (zeros past the end of the row) into out_q; the piece's scale word is stored by lane 0.
__device__ __forceinline__ void store_piece(const float* v, uint8_t* q, bool in_row, uint8_t* scale_word, int lane) {
  float largest = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) largest = fmaxf(largest, finite_size(v[e]));
  const uint32_t byte = fp8_scale_of(max_of_16_lanes(largest));
  if (in_row) {
    const u32x2_t out = {pack_fp8x4(v[0], v[1], v[2], v[3], byte),
                         pack_fp8x4(v[4], v[5], v[6], v[7], byte)};
    store_past(out, q);
  }
  uint32_t word = 0;
#pragma unroll
  for (int b = 0; b < 4; ++b) word |= (uint32_t)__builtin_amdgcn_readlane((int)byte, 16 * b) << (8 * b);
  if (lane == 0) *reinterpret_cast<uint32_t*>(scale_word) = word;
}

// One wave a row for rows of one piece (four rows to a workgroup), else one workgroup a row, ITERS pieces to each of its WAVES
// waves, and the sum of squares goes through LDS.  One piece a wave, as few registers and as many rows in flight as there can
// be, beats two (17776 x 1920 of float32 with add and sum 73 -> 68 us, 5.5 TB/s; 4000 x 6000 55 -> 50 us, 5.4 TB/s) and a wave
// for the whole row (78 us); workgroups that walk over rows with the next row's loads on their way came to 71 to 76.
template <typename XT, int ITERS, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void rms_fp8_kernel(RmsFp8Args a, int pitch) {
  __shared__ float red[2 * WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (r >= a.n_rows) return;
  const int64_t src = a.rows ? (int64_t)a.rows[r] : r;
  const XT* xr = static_cast<const XT*>(a.x) + src * a.hidden;
  const bf16_t* ar = a.add ? a.add + src * a.hidden : nullptr;
  const int first = (WAVES == 1 ? 0 : wave * ITERS) * PIECE;         // this wave's first element
  float v[ITERS][8];
  u32x4_t gain[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int c = first + it * PIECE + lane * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[it][e] = 0.f;
    gain[it] = u32x4_t{0u, 0u, 0u, 0u};
    if (c < a.hidden) {
      ResidIO<XT>::load8(xr + c, v[it]);
      if (ar) {
        float b[8];
        ResidIO<bf16_t>::load8(ar + c, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[it][e] += b[e];
      }
      gain[it] = *reinterpret_cast<const u32x4_t*>(a.gain + c);
    }
  }
  // mean of (scale * h)^2; `words`: LDS that no other sum uses
  auto mean_square = [&](float scale, float* words) {
    float sq = 0.f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
      for (int e = 0; e < 8; ++e) sq += (v[it][e] * scale) * (v[it][e] * scale);
    sq = wave_sum(sq);
    if (WAVES > 1) {
      if (lane == 0) words[wave] = sq;
      __syncthreads();
      sq = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) sq += words[i];
    }
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(sq / (float)a.hidden)));
  };
  // Below 2^-96 squares may have lost bits or all of them, and a sum may have passed the type's largest: such a row (the
  // same choice for all waves that hold it) is scaled by a power of two that takes its squares and their sum into range.
  // (17776 x 1920 of float32 68.1 us with and without this test, one row 3.08 and 2.95.)
  float scale = 1.f, square = mean_square(1.f, red) + a.eps;
  if (!(square >= 0x1p-96f && square < __builtin_inff())) {
    scale = square < 0x1p-96f ? 0x1p100f : 0x1p-80f;
    square = mean_square(scale, red + WAVES) + a.eps * scale * scale;
  }
  const float rstd = rsqrtf(square);
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int piece = first + it * PIECE, c = piece + lane * 8;
    if (piece >= a.hidden) break;
    if (a.sum && c < a.hidden) store8_past(static_cast<XT*>(a.sum) + r * a.hidden + c, v[it]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[it][2 * e] = v[it][2 * e] * scale * rstd * unpack_lo(gain[it][e]);
      v[it][2 * e + 1] = v[it][2 * e + 1] * scale * rstd * unpack_hi(gain[it][e]);
    }
    // (past the end of a row the zeros may meet an infinite rstd)
    if (c >= a.hidden) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[it][e] = 0.f;
    }
    store_piece(v[it], a.out.q + r * a.hidden + c, c < a.hidden, a.out.scales + r * pitch + piece / PIECE * 4, lane);
  }
}

// A piece to a wave (17776 x 1920 of bf16: 19.2 us, 5.3 TB/s; four pieces a wave 25 us)
template <typename XT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const XT* __restrict__ x, int64_t pieces, int columns,
                                                            int row_pieces, Fp8Out out) {
  const int lane = threadIdx.x & 63;
  const int64_t p = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (p >= pieces) return;
  const int64_t row = p / row_pieces;
  const int i = (int)(p - row * row_pieces), c = i * PIECE + lane * 8;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (c < columns) ResidIO<XT>::load8(x + row * columns + c, v);
  store_piece(v, out.q + row * columns + c, c < columns, out.scales + p * 4, lane);
}

// 128 x 128 blocks: a workgroup a block, 16 rows of it at a time, all of it in registers until its largest magnitude is known
// (7680 x 1920 of bf16: 9.1 us, 4.8 TB/s; 5760 x 1920 of fp32 10.4 us, 5.3 TB/s)
template <typename XT>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const XT* __restrict__ x, int n_rows, int columns,
                                                              int pitch, Fp8Out out) {
  __shared__ float red[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 128 + (threadIdx.x & 15) * 8, r0 = blockIdx.y * 128 + (threadIdx.x >> 4);
  float v[8][8], largest = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (c < columns && r0 + 16 * i < n_rows) ResidIO<XT>::load8(x + (int64_t)(r0 + 16 * i) * columns + c, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = fmaxf(largest, finite_size(v[i][e]));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) largest = fmaxf(largest, __shfl_xor(largest, o, 64));
  if (lane == 0) red[wave] = largest;
  __syncthreads();
  largest = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const uint32_t byte = fp8_scale_of(largest);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (c >= columns || r0 + 16 * i >= n_rows) continue;
    const float* t = v[i];
    const u32x2_t o = {pack_fp8x4(t[0], t[1], t[2], t[3], byte),
                       pack_fp8x4(t[4], t[5], t[6], t[7], byte)};
    store_past(o, out.q + (int64_t)(r0 + 16 * i) * columns + c);
  }
  // the last block of a row of blocks also writes the bytes that fill the word
  const int b = blockIdx.x + threadIdx.x;
  if (threadIdx.x == 0 || (blockIdx.x == gridDim.x - 1 && b < pitch))
    out.scales[(int64_t)blockIdx.y * pitch + b] = (uint8_t)(threadIdx.x == 0 ? byte : FP8_SCALE_ONE);
}

template <typename XT>
hipError_t rms_dispatch(const RmsFp8Args& a, hipStream_t st) {
  const int pitch = fp8_scale_pitch(a.hidden), pieces = pitch / 4;
#define LAUNCH(I, W)                                                                                               \
  hipLaunchKernelGGL((rms_fp8_kernel<XT, I, W>), dim3(W == 1 ? (a.n_rows + 3) / 4 : a.n_rows), dim3(W == 1 ? 256 : 64 * W), 0, \
                     st, a, pitch)
  if (pieces <= 1) LAUNCH(1, 1);
  else if (pieces <= 2) LAUNCH(1, 2);
  else if (pieces <= 4) LAUNCH(1, 4);
  else if (pieces <= 6) LAUNCH(1, 6);
  else if (pieces <= 8) LAUNCH(1, 8);
  else if (pieces <= 12) LAUNCH(1, 12);
  else if (pieces <= 16) LAUNCH(1, 16);
  else if (pieces <= 32) LAUNCH(2, 16);
  else return hipErrorInvalidValue;
#undef LAUNCH
  return hipGetLastError();
}

template <typename XT>
hipError_t quantize_dispatch(const XT* x, int n_rows, int columns, int block_rows, const Fp8Out& out, hipStream_t st) {
  const int pitch = fp8_scale_pitch(columns);
  if (block_rows == 1) {
    const int64_t pieces = (int64_t)n_rows * (pitch / 4);
    hipLaunchKernelGGL(quantize_rows_kernel<XT>, dim3((unsigned)((pieces + 3) / 4)), dim3(256), 0, st, x, pieces, columns,
                       pitch / 4, out);
  } else {
    hipLaunchKernelGGL(quantize_blocks_kernel<XT>, dim3(columns / 128 + (columns % 128 != 0), (n_rows + 127) / 128), dim3(256), 0, st, x,
                       n_rows, columns, pitch, out);
  }
  return hipGetLastError();
}

// A launch has fewer than 2^32 threads in x and 2^16 workgroups in y: more rows than these go to several launches.
constexpr int LAUNCH_ROWS = 1 << 21;       // (of 1024 threads at most, or 2^14 rows of blocks)

}  // namespace

hipError_t launch_gather_rms_fp8(const RmsFp8Args& all, hipStream_t st) {
  if (all.hidden <= 0 || all.hidden % 16 != 0) return hipErrorInvalidValue;
  hipError_t e = hipSuccess;
  for (int r = 0; r < all.n_rows && e == hipSuccess; r += std::min(LAUNCH_ROWS, all.n_rows - r)) {
    RmsFp8Args a = all;
    const int64_t done = (int64_t)r * a.hidden, x_bytes = done * (a.x_fp32 ? 4 : 2);
    a.n_rows = std::min(LAUNCH_ROWS, all.n_rows - r);
    if (a.rows) a.rows += r;
    else {
      a.x = static_cast<const char*>(a.x) + x_bytes;
      if (a.add) a.add += done;
    }
    if (a.sum) a.sum = static_cast<char*>(a.sum) + x_bytes;
    a.out.q += done;
    a.out.scales += (int64_t)r * fp8_scale_pitch(a.hidden);
    e = a.x_fp32 ? rms_dispatch<float>(a, st) : rms_dispatch<bf16_t>(a, st);
  }
  return e;
}

hipError_t launch_quantize_fp8(const void* x, bool x_fp32, int n_rows, int columns, int block_rows, const Fp8Out& out,
                               hipStream_t st) {
  if (columns <= 0 || columns % 16 != 0) return hipErrorInvalidValue;
  const int pitch = fp8_scale_pitch(columns);
  // (64 threads a piece: 2^31 a launch)
  const int most = block_rows == 1 ? std::max(1, std::min(LAUNCH_ROWS, (1 << 25) / (pitch / 4))) : LAUNCH_ROWS;
  hipError_t e = hipSuccess;
  for (int r = 0; r < n_rows && e == hipSuccess; r += std::min(most, n_rows - r)) {
    const int64_t done = (int64_t)r * columns;
    const int rows = std::min(most, n_rows - r);
    const Fp8Out o = {out.q + done, out.scales + (int64_t)(r / block_rows) * pitch};
    e = x_fp32 ? quantize_dispatch(static_cast<const float*>(x) + done, rows, columns, block_rows, o, st)
               : quantize_dispatch(static_cast<const bf16_t*>(x) + done, rows, columns, block_rows, o, st);
  }
  return e;
}
