// 8-bit MFMA GEMM: C = act(A W^T + bias), A [M,K] and W [N,K] e4m3, both K-contiguous, with a power-of-two scale for each
// 1 x 128 block of A and each 128 x 128 block of W; fp32 accumulate.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes the scales as operands: a lane gives one for its row and half of k (A fragment:
// lane holds row lane%32, 32 consecutive k starting at 32*(lane/32); B likewise for column lane%32; accumulator register
// i of a lane is row 8*(i/4) + 4*(lane/32) + i%4, column lane%32).  A block of 128 is two such steps, so
// scaling costs no instruction of its own and changes no bit of the products.  The waves accumulate C^T blocks (operands
// swapped), so a lane owns one row m and four consecutive columns n per accumulator quad.
#include <algorithm>
#include <atomic>
#include <type_traits>

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

// ------------------------------------------------------------------------------------------
// Large problems: 256 x 256 tile, eight waves (two per SIMD) of 64 x 128, K walked in stages of 128 (one scale block, one
// 128-byte line per row) through LDS rings of three A slots and two W slots (all 160 KB of a CU) that are filled by direct
// global -> LDS loads, W one stage and A two stages ahead; LDS rows of 128 B whose eight 16-byte chunks are
// XOR-swizzled with (row/2)%8.  One barrier a stage.  In bytes a stage is that of a bf16 kernel with k steps of 64, and takes
// the matrix pipe as long (16 MFMAs of 64 cycles a wave), at twice the flops.
//  * A wave's 128 columns are one scale block of the weight and, in 8-bit results, one block of the output row: its scale is
//    found without leaving the wave.
//  * The four MFMAs of a stage's last two W fragments run after the next barrier, while the first fragments of the new stage
//    arrive; within a stage a fragment is read four MFMAs ahead of its use, so four W fragments and two pairs of A
//    fragments are all that is held (64 registers beside 128 accumulators).
//  * Scale bytes of GROUP stages lie in registers, shifted down a byte a stage; those of the next group are asked for at the
//    start of a group, since the wait for them is a wait for every fill in flight.
// ------------------------------------------------------------------------------------------
constexpr int BK = 128;
constexpr int STAGE_BYTES = 256 * BK;              // one operand, one stage: 32 KB
constexpr int RING_B_OFF = 3 * STAGE_BYTES;        // the W ring starts after the A ring
constexpr int CST = 272;                           // bf16 staging: bytes per 128-column row (+16 pad)
constexpr int CST8 = 144;                          // 8-bit staging
constexpr int STAGE_REGION = 64 * CST;             // per-wave staging region (17408 B)
constexpr int GEMM256_LDS = 5 * STAGE_BYTES;
static_assert(8 * STAGE_REGION <= GEMM256_LDS, "staging");
constexpr int GROUP = 12;                          // stages whose scale bytes are held: a multiple of 6 (ring slots) and 4
constexpr int WORDS = GROUP / 4;

// Tile slots 0 .. full_items-1 are whole work items; every later slot is cut into `split` chunks along k whose fp32 sums
// go to a workspace (256 KB a chunk, in accumulator order) and are added up by the fix-up kernel.
struct Split {
  int32_t full_items, split;
  float* ws;
};

// chunks begin on whole scale words
__device__ __forceinline__ int chunk_begin(int chunk, int n_chunks, int n_stages) {
  return chunk == n_chunks ? n_stages : chunk * n_stages / n_chunks / 4 * 4;
}

// A wave's 64 x 128 sums, acc[i][j][4q+e] = C[mw + 32i + lr][nw + 32j + 8q + 4lh + e], to the result; region: LDS of this wave
template <bool QUANT, bool GELU>
__device__ __forceinline__ void store_tile(const GemmFp8Args& g, floatx16_t (&acc)[2][4], int mw, int nw, int lane, char* region) {
  const int lr = lane & 31, lh = lane >> 5;
  const int out_pitch = fp8_scale_pitch(g.n), block = nw >> 7, blocks = (g.n + 127) >> 7;
  const bf16_t* bias = g.bias != nullptr ? g.bias : reinterpret_cast<const bf16_t*>(g.w);   // (any readable place)
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float largest = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // (columns past N: no weights and no bias, so 0, which counts for no scale and is not stored)
        const int n = nw + 32 * j + 8 * q + 4 * lh;
        u32x2_t b = *reinterpret_cast<const u32x2_t*>(bias + min(n, g.n - 4));
        if (g.bias == nullptr || n >= g.n) b = u32x2_t{0u, 0u};
        float v[4] = {acc[i][j][4 * q] + unpack_lo(b[0]), acc[i][j][4 * q + 1] + unpack_hi(b[0]),
                      acc[i][j][4 * q + 2] + unpack_lo(b[1]), acc[i][j][4 * q + 3] + unpack_hi(b[1])};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (GELU) v[e] = gelu_tanh(v[e]);
          if (QUANT) {
            acc[i][j][4 * q + e] = v[e];
            largest = fmaxf(largest, finite_size(v[e]));
          }
        }
        if (!QUANT) {
          const u32x2_t pk = {pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3])};
          *reinterpret_cast<u32x2_t*>(region + (32 * i + lr) * CST + (32 * j + 8 * q + 4 * lh) * 2) = pk;
        }
      }
    if (QUANT) {
      const uint32_t byte = fp8_scale_of(fmaxf(largest, __shfl_xor(largest, 32, 64)));
      const float inv = fp8_inverse_scale(byte);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint32_t*>(region + (32 * i + lr) * CST8 + 32 * j + 8 * q + 4 * lh) =
              pack_fp8x4(acc[i][j][4 * q] * inv, acc[i][j][4 * q + 1] * inv, acc[i][j][4 * q + 2] * inv, acc[i][j][4 * q + 3] * inv);
      const int m = mw + 32 * i + lr;
      if (lh == 0 && m < g.m && nw < g.n) {
        uint8_t* s = g.out.scales + (int64_t)m * out_pitch;
        s[block] = (uint8_t)byte;
        if (block == blocks - 1)
          for (int x = blocks; x < out_pitch; ++x) s[x] = (uint8_t)FP8_SCALE_ONE;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (!QUANT) {
    // 64 rows x 16 pieces of 8 columns: two 128-byte lines per row
#pragma unroll 4
    for (int it = 0; it < 16; ++it) {
      const int rl = it * 4 + (lane >> 4), piece = lane & 15;
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(region + rl * CST + piece * 16);
      const int m = mw + rl, n = nw + piece * 8;
      if (m < g.m && n < g.n) *reinterpret_cast<u32x4_t*>(g.c + (int64_t)m * g.n + n) = v;
    }
  } else {
    // 64 rows x 8 pieces of 16 columns
#pragma unroll 4
    for (int it = 0; it < 8; ++it) {
      const int rl = it * 8 + (lane >> 3), piece = lane & 7;
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(region + rl * CST8 + piece * 16);
      const int m = mw + rl, n = nw + piece * 16;
      if (m < g.m && n < g.n) *reinterpret_cast<u32x4_t*>(g.out.q + (int64_t)m * g.n + n) = v;
    }
  }
}

template <bool QUANT, bool GELU>
__global__ __launch_bounds__(512) void gemm256_fp8_kernel(GemmFp8Args g, int tiles_m, int tiles_n, int per_xcd, int group_m, Split sk) {
  int slot = blockIdx.x, chunk = 0, n_chunks = 1;
  if (slot >= sk.full_items) {
    const int r = slot - sk.full_items;
    slot = sk.full_items + r / sk.split;
    chunk = r - (r / sk.split) * sk.split;
    n_chunks = sk.split;
  }
  int m0, n0;
  if (!tile_origin(slot, 256, 256, tiles_m, tiles_n, per_xcd, group_m, m0, n0)) return;

  extern __shared__ u32x4_t smem[];
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)smem;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave & 3) * 64, wn0 = (wave >> 2) * 128;
  const int lr = lane & 31, lh = lane >> 5;

  // ---- fills: per stage this wave brings blocks wave+8i (8 rows each) of A and of W, i = 0..3; lane l fetches, for row l/8
  //      of the block, the chunk that belongs in slot l%8.  Chunks past K are asked for past the buffer and arrive as zero. ----
  const uint32_t row_bytes = (uint32_t)g.k;
  const u32x4_t rsA = rsrc_words(g.a, (uint32_t)g.m * row_bytes);
  const u32x4_t rsB = rsrc_words(g.w, (uint32_t)g.n * row_bytes);
  const int row = wave * 8 + (lane >> 3);
  const uint32_t fill_chunk = (lane & 7) ^ ((row >> 1) & 7);            // (the same for rows 64 apart)
  const uint32_t voffA = (uint32_t)(m0 + row) * row_bytes + fill_chunk * 16, voffB = (uint32_t)(n0 + row) * row_bytes + fill_chunk * 16;
  const uint32_t step64 = 64u * row_bytes;
  const uint32_t fillA = lds0 + wave * 1024, fillB = lds0 + RING_B_OFF + wave * 1024;
  const int n_stages = (g.k + BK - 1) / BK;
  const int stage_begin = chunk_begin(chunk, n_chunks, n_stages), stage_end = chunk_begin(chunk + 1, n_chunks, n_stages);
  const uint32_t past = fill_chunk * 16 >= (uint32_t)(g.k - (n_stages - 1) * BK) ? 0xFFFFFFF0u : 0u;
  auto voff = [&](uint32_t base, int stage, int q) {
    return (base + (uint32_t)q * step64) | (stage == n_stages - 1 ? past : 0u);
  };
  auto fill_a = [&](int slot, int stage, int q) {
    lds_fill(rsA, fillA + (uint32_t)slot * STAGE_BYTES + q * 8192, voff(voffA, stage, q), (uint32_t)stage * BK);
  };
  auto fill_b = [&](int slot, int stage, int q) {
    lds_fill(rsB, fillB + (uint32_t)slot * STAGE_BYTES + q * 8192, voff(voffB, stage, q), (uint32_t)stage * BK);
  };

  // ---- scale bytes: of rows wm0 + 32i + lr, and of the wave's columns ----
  const int pitch = fp8_scale_pitch(g.k);
  const __amdgpu_buffer_rsrc_t rsSA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.a_scales), 0, (uint32_t)g.m * (uint32_t)pitch, 0x00020000);
  const __amdgpu_buffer_rsrc_t rsSW = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.w_scales), 0, (uint32_t)((g.n + 127) / 128) * (uint32_t)pitch, 0x00020000);
  const uint32_t offSA = (uint32_t)(m0 + wm0 + lr) * (uint32_t)pitch, offSW = (uint32_t)((n0 + wn0) / 128) * (uint32_t)pitch;
  uint32_t wordA[2][WORDS], wordW[WORDS], nextA[2][WORDS], nextW[WORDS];
  auto ask_scales = [&](int stage) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      nextA[0][w] = __builtin_amdgcn_raw_buffer_load_b32(rsSA, offSA, stage + 4 * w, 0);
      nextA[1][w] = __builtin_amdgcn_raw_buffer_load_b32(rsSA, offSA + 32u * (uint32_t)pitch, stage + 4 * w, 0);
      nextW[w] = __builtin_amdgcn_raw_buffer_load_b32(rsSW, offSW, stage + 4 * w, 0);
    }
  };

  // ---- fragment reads: row R, chunk c of a stage sits at R*128 + (c ^ ((R/2)%8))*16.  A fragment of 64 k is the four
  //      chunks 4s .. 4s+3, the even ones to lanes 0-31: both operands take k in this order ----
  uint32_t first = (uint32_t)(lr * 128 + ((lh ^ ((lr >> 1) & 7)) * 16));        // chunk lh of row lr
  const uint32_t baseA = lds0 + wm0 * 128, baseB = lds0 + RING_B_OFF + wn0 * 128;
  auto frag = [&](uint32_t base, int slice, int slot, int i) {
    typedef const __attribute__((address_space(3))) u32x4_t* lds_t;
    const uint32_t at = base + slot * STAGE_BYTES + i * 4096;
    const u32x4_t lo = *(lds_t)(size_t)((first ^ (uint32_t)(64 * slice)) + at), hi = *(lds_t)(size_t)((first ^ (uint32_t)(64 * slice + 32)) + at);
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  floatx16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  i32x8_t fa[2][2], fb[4];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    fa[1][0][e] = fa[1][1][e] = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) fb[u][e] = 0;
  }
  int scaleA[2] = {(int)FP8_SCALE_ONE, (int)FP8_SCALE_ONE}, scaleW = (int)FP8_SCALE_ONE;
  // MFMA x of a stage: W fragment x/2 (slice x/8), A fragment x%2
  auto mma = [&](int x) {
    const int i = x & 1, u = (x >> 1) & 7, j = u & 3;
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[u & 3], fa[u >> 2][i], acc[i][j], 0, 0, 0, scaleW, 0, scaleA[i]);
  };
  auto stage = [&](auto SLOT_A, auto SLOT_B, int t) {
    constexpr int SA = decltype(SLOT_A)::value, SB = decltype(SLOT_B)::value;
    // All but the four newest fills (A of stage t+1) have landed: A and W of stage t are in LDS, and every wave's reads of
    // stage t-1 are complete: its slots are free.
    asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int y = 0; y < 16; ++y) {
      // (past the last stage it is fetched once more into the idle slot: in bounds, never read)
      if (y < 4) fill_b(SB ^ 1, min(t + 1, stage_end - 1), y);
      else if (y < 8) fill_a((SA + 2) % 3, min(t + 2, stage_end - 1), y - 4);
      if (y == 4) {
        // the stage's own scales: byte 0 of the words, which move down by one
#pragma unroll
        for (int i = 0; i < 2; ++i) scaleA[i] = (int)wordA[i][0];
        scaleW = (int)wordW[0];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            wordA[i][w] = w + 1 < WORDS ? __builtin_amdgcn_alignbit(wordA[i][w + 1], wordA[i][w], 8) : wordA[i][w] >> 8;
          wordW[w] = w + 1 < WORDS ? __builtin_amdgcn_alignbit(wordW[w + 1], wordW[w], 8) : wordW[w] >> 8;
        }
      }
      const int s = y >> 3, u = y >> 1;
      if ((y & 7) == 0) asm volatile("" : "+v"(first));     // (its sums are formed here again, not held through the loop)
      if ((y & 7) == 0) fa[s][0] = frag(baseA, s, SA, 0);
      if ((y & 1) == 0) fb[u & 3] = frag(baseB, s, SB, u & 3);
      if ((y & 7) == 1) fa[s][1] = frag(baseA, s, SA, 1);
      mma(y < 4 ? y + 12 : y - 4);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  ask_scales(stage_begin);
#pragma unroll
  for (int q = 0; q < 4; ++q) fill_a(0, stage_begin, q);
#pragma unroll
  for (int q = 0; q < 4; ++q) fill_b(0, stage_begin, q);
#pragma unroll
  for (int q = 0; q < 4; ++q) fill_a(1, min(stage_begin + 1, stage_end - 1), q);
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  for (int t0 = stage_begin; t0 < stage_end; t0 += GROUP) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      wordA[0][w] = nextA[0][w]; wordA[1][w] = nextA[1][w];
      wordW[w] = __builtin_amdgcn_readfirstlane(nextW[w]);
      asm volatile("" : "+v"(wordA[0][w]), "+v"(wordA[1][w]));
    }
    if (t0 + GROUP < stage_end) ask_scales(t0 + GROUP);
    const int group_end = min(t0 + GROUP, stage_end);
    for (int t = t0; t < group_end; t += 6) {
      stage(I0{}, I0{}, t);
      if (t + 1 < stage_end) stage(I1{}, I1{}, t + 1);
      if (t + 2 < stage_end) stage(I2{}, I0{}, t + 2);
      if (t + 3 < stage_end) stage(I0{}, I1{}, t + 3);
      if (t + 4 < stage_end) stage(I1{}, I0{}, t + 4);
      if (t + 5 < stage_end) stage(I2{}, I1{}, t + 5);
    }
  }
#pragma unroll
  for (int x = 12; x < 16; ++x) mma(x);

  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (n_chunks > 1) {
    float* part = sk.ws + ((size_t)(slot - sk.full_items) * sk.split + chunk) * 65536 + tid * 4;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          floatx4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          *reinterpret_cast<floatx4_t*>(part + ((i * 4 + j) * 4 + q) * 2048) = v;
        }
    return;
  }
  __syncthreads();                       // every wave is done with the rings
  store_tile<QUANT, GELU>(g, acc, m0 + wm0, n0 + wn0, lane, reinterpret_cast<char*>(smem) + wave * STAGE_REGION);
}

// Adds up the chunks of the cut tiles and stores the result: a one-wave workgroup to each 64 x 128 part of a tile.
template <bool QUANT, bool GELU>
__global__ __launch_bounds__(64) void gemm256_fp8_fixup_kernel(GemmFp8Args g, int tiles_m, int tiles_n, int per_xcd, int group_m, Split sk) {
  const int tile = blockIdx.x >> 3, wave = blockIdx.x & 7, lane = threadIdx.x;
  int m0, n0;
  if (!tile_origin(sk.full_items + tile, 256, 256, tiles_m, tiles_n, per_xcd, group_m, m0, n0)) return;
  extern __shared__ u32x4_t smem[];
  floatx16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  const float* part = sk.ws + (size_t)tile * sk.split * 65536 + (wave * 64 + lane) * 4;
  for (int c = 0; c < sk.split; ++c, part += 65536) {
    floatx4_t v[32];
#pragma unroll
    for (int x = 0; x < 32; ++x) v[x] = __builtin_nontemporal_load(reinterpret_cast<const floatx4_t*>(part + x * 2048));
#pragma unroll
    for (int x = 0; x < 32; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[x >> 4][(x >> 2) & 3][4 * (x & 3) + e] += v[x][e];
  }
  store_tile<QUANT, GELU>(g, acc, m0 + (wave & 3) * 64, n0 + (wave >> 2) * 128, lane, reinterpret_cast<char*>(smem));
}

template <bool QUANT, bool GELU>
hipError_t launch_gemm256_fp8(const GemmFp8Args& g, int split, hipStream_t st) {
  static std::atomic<uint64_t> lds_allowed{0};
  auto kern = gemm256_fp8_kernel<QUANT, GELU>;
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), GEMM256_LDS, lds_allowed);
  if (e != hipSuccess) return e;
  const int tiles_m = (g.m + 255) / 256, tiles_n = (g.n + 255) / 256;
  const int per_xcd = (tiles_m * tiles_n + 7) / 8, slots = per_xcd * 8;
  const int group_m = (g.k >= 8192 || tiles_m <= 24) ? 4 : 8;
  const Split sk = {split > 1 ? slots / 256 * 256 : slots, split, g.scratch};
  const int cut = slots - sk.full_items;
  hipLaunchKernelGGL(kern, dim3(sk.full_items + cut * sk.split), dim3(512), GEMM256_LDS, st, g, tiles_m, tiles_n, per_xcd, group_m, sk);
  if (cut > 0)
    hipLaunchKernelGGL((gemm256_fp8_fixup_kernel<QUANT, GELU>), dim3(cut * 8), dim3(64), STAGE_REGION, st, g, tiles_m, tiles_n, per_xcd, group_m, sk);
  return hipGetLastError();
}


// The chip runs 256 workgroups at a time: the tiles of a last, partly filled round are cut along k where that pays (the round
// then takes ceil(n * s / 256) / s of a tile's time) and the sums fit the scratch.
int choose_split(const GemmFp8Args& g) {
  const int slots = ((g.m + 255) / 256 * ((g.n + 255) / 256) + 7) / 8 * 8, n_rem = slots % 256;
  if (n_rem == 0 || g.scratch == nullptr) return 1;
  const int stages = (g.k + BK - 1) / BK;
  const int s_max = (int)std::min<size_t>((size_t)std::min(stages / 16, 8), g.scratch_bytes / ((size_t)n_rem * 262144));
  double best = 1.0;
  int split = 1;
  for (int s = 2; s <= s_max; ++s) {
    const double t = (double)((n_rem * s + 255) / 256) / s + 0.1 * n_rem / stages * s;
    if (t < best - 0.02) { best = t; split = s; }
  }
  return split;
}

}  // namespace

hipError_t launch_gemm_fp8(const GemmFp8Args& g, hipStream_t st) {
  if (g.m <= 0 || g.n <= 0) return hipSuccess;
  if (g.k <= 0 || g.k % 16 != 0 || g.n % 16 != 0) return hipErrorInvalidValue;
  // operands are addressed with 32-bit byte offsets
  if (((int64_t)g.m + 512) * g.k >= (int64_t)1 << 32 || ((int64_t)g.n + 512) * g.k >= (int64_t)1 << 32) return hipErrorInvalidValue;
  if (g.m > 128) {
    const int split = choose_split(g);
    if (g.out.q) return g.gelu ? launch_gemm256_fp8<true, true>(g, split, st) : launch_gemm256_fp8<true, false>(g, split, st);
    return g.gelu ? launch_gemm256_fp8<false, true>(g, split, st) : launch_gemm256_fp8<false, false>(g, split, st);
  }
  const dim3 grid((g.n + 127) / 128, (g.m + 31) / 32);
  if (g.out.q) hipLaunchKernelGGL(gemm_fp8_direct_kernel<true>, grid, dim3(64), 0, st, g);
  else hipLaunchKernelGGL(gemm_fp8_direct_kernel<false>, grid, dim3(64), 0, st, g);
  return hipGetLastError();
}
