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

// ------------------------------------------------------------------------------------------
// Large problems: 256 x 256 tile, eight waves (two per SIMD) of 64 x 128, K walked in stages of 128 (one scale block, one
// 128-byte line per row) through LDS rings of three A slots and two W slots (all 160 KB of a CU) that are filled by direct
// global -> LDS loads, A two stages ahead, W in halves of a stage of which three are on their way; LDS rows of 128 B whose eight
// 16-byte chunks are XOR-swizzled with (row/2)%8.  A barrier each half stage.  In bytes a stage is that of a bf16 kernel with
// k steps of 64, and takes the matrix pipe as long (16 MFMAs of 64 cycles a wave), at twice the flops.
// Bound by the matrix pipes at the clock that the chip's power allows: 8192^3 runs at 2.73 PFLOP/s on random data and at 3.9
// on zeros (a loop of these MFMAs on registers: 3.2 to 3.8 and 4.6).  17776 x 7680 x 1920 takes 225 to 258 us on
// different cards (2.0 to 2.3 PFLOP/s; with GELU into 8 bits 254 to 286, whose epilogues the pipes wait for), 17776 x 1920 x 7680 222 to 249.
//  * A wave's 128 columns are one scale block of the weight and, in 8-bit results, one block of the output row: its scale is
//    found without leaving the wave.
//  * The last four MFMAs of a half stage run after the next barrier, while the first fragments behind it arrive; a fragment is
//    read four MFMAs ahead of its use, so four W fragments and two pairs of A fragments are all that is held (64 registers
//    beside 128 accumulators).
//  * Workgroups walk over the tiles: the next tile's first fills go out before a result is stored.  (17776 x 7680 x 1920 on one card: 264 us
//    with W filled a whole stage ahead, 249 in halves, 241 with sums that begin with the bias and tile places found without
//    divisions, the rest from the last round's quarters.)
//  * Scale bytes of GROUP stages lie in registers, shifted down a byte a stage; those of the next group are asked for at the
//    start of a group, since the wait for them is a wait for every fill in flight.
// ------------------------------------------------------------------------------------------
constexpr int BK = 128;
constexpr int STAGE_BYTES = 256 * BK;              // one operand, one stage: 32 KB
constexpr int RING_B_OFF = 3 * STAGE_BYTES;        // the W ring starts after the A ring
constexpr int GEMM256_LDS = 5 * STAGE_BYTES;
constexpr int GROUP = 12;                          // stages whose scale bytes are held: a multiple of 6 (ring slots) and 4
constexpr int WORDS = GROUP / 4;

// Division by a number that the host knows: exact while the dividend times the divisor stays below 2^32 (quick; the plain
// division of a uniform value takes some 40 dependent instructions, 0.2 us, and there are three to a tile)
struct Divisor {
  uint32_t d = 1, mul = 0;             // mul 0: too large for that
};
inline Divisor divisor(uint32_t d, uint64_t most) {
  return {d, (uint64_t)d * most < ((uint64_t)1 << 32) && d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0u};
}
__device__ __forceinline__ uint32_t divide(uint32_t x, const Divisor& by) {
  if (by.d == 1) return x;
  return by.mul != 0 ? __umulhi(x, by.mul) : x / by.d;
}

// The tiles of a problem: slots are dealt so that each XCD owns a contiguous range of tiles, walked in groups of group_m row
// tiles; some slots that pad the range to a multiple of 8 are empty.
struct Grid {
  int32_t tiles_m, tiles_n, per_xcd, group_m;
  Divisor group, rows, last_rows;      // tiles of a group; row tiles of a group, of the last one
};
Grid make_grid(const GemmFp8Args& g, int bm, int bn) {
  Grid t;
  t.tiles_m = (g.m + bm - 1) / bm;
  t.tiles_n = (g.n + bn - 1) / bn;
  t.per_xcd = (t.tiles_m * t.tiles_n + 7) / 8;
  // (operand panels of a long-k problem are several MB each, and a problem with few row tiles gives each XCD few groups)
  t.group_m = (g.k >= 8192 || t.tiles_m <= 24) ? 4 : 8;
  const uint64_t most = (uint64_t)t.per_xcd * 8;
  t.group = divisor((uint32_t)(t.group_m * t.tiles_n), most);
  t.rows = divisor((uint32_t)t.group_m, most);
  t.last_rows = divisor((uint32_t)((t.tiles_m - 1) % t.group_m + 1), most);
  return t;
}
// slot -> origin of its bm x bn tile; false for an empty one
__device__ __forceinline__ bool origin(const Grid& t, int slot, int bm, int bn, int& m0, int& n0) {
  const uint32_t p = (uint32_t)((slot % 8) * t.per_xcd + slot / 8);
  if (p >= (uint32_t)(t.tiles_m * t.tiles_n)) return false;
  const uint32_t group = divide(p, t.group), first_m = group * t.group_m;
  const uint32_t in_group = p - group * t.group.d;
  const bool last = first_m + t.group_m > (uint32_t)t.tiles_m;
  const uint32_t rows = last ? t.last_rows.d : t.rows.d, column = last ? divide(in_group, t.last_rows) : divide(in_group, t.rows);
  m0 = (int)(first_m + in_group - column * rows) * bm;
  n0 = (int)column * bn;
  return true;
}

// Tile slots 0 .. full_items-1 are whole work items; every later slot is cut into `split` chunks along k whose fp32 sums
// go to a workspace (256 KB a chunk, in accumulator order) and are added up by the fix-up kernel.
struct Split {
  int32_t full_items, split;
  float* ws;
  Divisor by;                          // by split
};

// chunks begin on whole scale words
__device__ __forceinline__ int chunk_begin(int chunk, int n_chunks, const Divisor& by, int n_stages) {
  return chunk == n_chunks ? n_stages : (int)divide((uint32_t)(chunk * n_stages), by) / 4 * 4;
}

// Scale words of a weight's block of rows are the same for a whole wave: scalar loads (word clamped to the row's last)
__device__ __forceinline__ uint32_t weight_scale_word(const GemmFp8Args& g, int n, int pitch, int word) {
  typedef const __attribute__((address_space(4))) uint32_t* scalar_t;
  const uint32_t row = (uint32_t)min(n, g.n - 1) / 128u;
  const uint64_t at = (uint64_t)g.w_scales + (uint64_t)(row * (uint32_t)pitch) + (uint32_t)fp8_scale_word_offset(word, pitch);
  return *(scalar_t)at;
}

// Bias of a wave's 128 columns, two a lane; past the end of the buffer (columns past N, or no bias) zeros
__device__ __forceinline__ uint32_t load_bias(const GemmFp8Args& g, int nw, int lane, bool none) {
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(g.bias), 0, g.bias != nullptr && !none ? (uint32_t)g.n * 2u : 0u, 0x00020000);
  return __builtin_amdgcn_raw_buffer_load_b32(rs, (uint32_t)(nw + 2 * lane) * 2u, 0, 0);
}

// The sums begin with it: acc[i][j][4q+e] belongs to column nw + 32j + 8q + 4lh + e
__device__ __forceinline__ void begin_with(uint32_t bias, int lane, floatx16_t (&acc)[2][4]) {
  const bool high = lane >= 32;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      auto word = [&](int w) {
        const uint32_t lo = __builtin_amdgcn_readlane((int)bias, 16 * j + 4 * q + w), hi = __builtin_amdgcn_readlane((int)bias, 16 * j + 4 * q + 2 + w);
        return high ? hi : lo;
      };
      const uint32_t a = word(0), b = word(1);
      const float v[4] = {unpack_lo(a), unpack_hi(a), unpack_lo(b), unpack_hi(b)};
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[0][j][4 * q + e] = acc[1][j][4 * q + e] = v[e];
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A wave's 64 x 128 sums, acc[i][j][4q+e] = C[m0 + wm0 + 32i + lr][nw + 32j + 8q + 4lh + e], to the result, staged in two
// quarters (8-bit results: halves) through 4 KB of this wave's LDS.  What lies outside the matrix is sent past the end of the buffer.
constexpr int STAGING = 4096;
template <bool QUANT, bool GELU>
__device__ __forceinline__ void store_tile(const GemmFp8Args& g, floatx16_t (&acc)[2][4], int m0, int wm0, int nw,
                                           int lane, char* region) {
  const int out_pitch = fp8_scale_pitch(g.n), block = nw >> 7, blocks = (g.n + 127) >> 7;
  const uint32_t row_bytes = (uint32_t)g.n * (QUANT ? 1u : 2u);
  char* base = (QUANT ? reinterpret_cast<char*>(g.out.q) : reinterpret_cast<char*>(g.c)) + (int64_t)m0 * row_bytes;
  const uint32_t rows = (uint32_t)min(g.m - m0, 256);
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(base, 0, rows * row_bytes, 0x00020000);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    forget(lane);                          // (what follows from it is formed again, not held from the first half)
    const int lr = lane & 31, lh = lane >> 5;
    float largest = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // (columns past N: no weights and no bias, so 0, which counts for no scale and is not stored)
        float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (GELU) v[e] = gelu_tanh(v[e]);
          if (QUANT) {
            acc[i][j][4 * q + e] = v[e];
            largest = fmaxf(largest, __builtin_fabsf(v[e]));       // (NaN does not count; infinities below)
          }
        }
        if (!QUANT) {
          const u32x2_t pk = {pack_bf16x2_hw(v[0], v[1]), pack_bf16x2_hw(v[2], v[3])};
          *reinterpret_cast<u32x2_t*>(region + lr * 128 + (((4 * (j & 1) + q) ^ ((lr >> 1) & 7)) * 16) + lh * 8) = pk;
        }
      }
      if (!QUANT && (j & 1)) {
        // 32 rows x 8 pieces of 8 columns: one 128-byte line per row
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int rl = it * 8 + (lane >> 3), piece = lane & 7, n = nw + 64 * (j >> 1) + piece * 8;
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(region + rl * 128 + ((piece ^ ((rl >> 1) & 7)) * 16));
          __builtin_amdgcn_raw_buffer_store_b128(v, rs, n < g.n ? (uint32_t)(wm0 + 32 * i + rl) * row_bytes + (uint32_t)n * 2u : 0xFFFFFFF0u, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (QUANT) {
      if (__any(largest == __builtin_inff())) {
        largest = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) largest = fmaxf(largest, finite_size(acc[i][j][e]));
      }
      const uint32_t byte = fp8_scale_of(fmaxf(largest, __shfl_xor(largest, 32, 64)));
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint32_t*>(region + lr * 128 + (((2 * j + (q >> 1)) ^ ((lr >> 1) & 7)) * 16) + (q & 1) * 8 + lh * 4) =
              pack_fp8x4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3], byte);
      const int m = m0 + wm0 + 32 * i + lr;
      if (lh == 0 && m < g.m && nw < g.n) {
        uint8_t* s = g.out.scales + (int64_t)m * out_pitch;
        s[block] = (uint8_t)byte;
        if (block == blocks - 1)
          for (int x = blocks; x < out_pitch; ++x) s[x] = (uint8_t)FP8_SCALE_ONE;
      }
      // 32 rows x 8 pieces of 16 columns
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int rl = it * 8 + (lane >> 3), piece = lane & 7, n = nw + piece * 16;
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(region + rl * 128 + ((piece ^ ((rl >> 1) & 7)) * 16));
        __builtin_amdgcn_raw_buffer_store_b128(v, rs, n < g.n ? (uint32_t)(wm0 + 32 * i + rl) * row_bytes + (uint32_t)n : 0xFFFFFFF0u, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

struct Args256 {
  GemmFp8Args g;
  Grid grid;
  Split sk;
};
// The kernel's arguments, read again where they are used: between tiles, so that no register holds them in the main loop
__device__ __forceinline__ const Args256& args_again() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  forget_scalar(p);
  return *(const Args256*)p;
}

template <bool QUANT, bool GELU>
__global__ __launch_bounds__(512) void gemm256_fp8_kernel(Args256 args) {
  const GemmFp8Args& g = args.g;
  // ---- the work items of this workgroup: blockIdx.x, then every gridDim.x-th; a whole tile or a chunk of one ----
  const int n_stages = (g.k + BK - 1) / BK;
  struct Item {
    int index, m0, n0, part, begin, end;         // part: the chunk's place among the partial sums; -1: a whole tile
  };
  auto item_from = [&](int index) {              // the first one from `index` on that is a tile (some slots are empty)
    const Args256 now = args_again();
    const Grid& grid = now.grid;
    const Split& sk = now.sk;
    const int n_items = sk.full_items + (8 * grid.per_xcd - sk.full_items) * sk.split;
    for (; index < n_items; index += gridDim.x) {
      const bool cut = index >= sk.full_items && sk.split > 1;
      const int r = index - sk.full_items, tile = cut ? (int)divide((uint32_t)r, sk.by) : 0, chunk = r - tile * sk.split;
      int m0, n0;
      if (origin(grid, cut ? sk.full_items + tile : index, 256, 256, m0, n0))
        return Item{index, m0, n0, cut ? r : -1, cut ? chunk_begin(chunk, sk.split, sk.by, n_stages) : 0,
                    cut ? chunk_begin(chunk + 1, sk.split, sk.by, n_stages) : n_stages};
    }
    return Item{-1, 0, 0, -1, 0, 0};
  };
  Item it = item_from(blockIdx.x);
  if (it.index < 0) return;

  extern __shared__ u32x4_t smem[];
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)smem;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave & 3) * 64, wn0 = (wave >> 2) * 128;
  const int lr = lane & 31, lh = lane >> 5;

  // ---- fills: per stage this wave brings blocks wave+8q (8 rows each) of A, q = 0..3, and of each half of W, q = 0, 1; lane l
  //      fetches, for row l/8 of the block, the chunk that belongs in slot l%8.  Half `hh` of W: rows 64*hh .. +63 and
  //      128 + 64*hh .. +63 of the tile.  Chunks past K are asked for past the buffer and arrive as zero. ----
  const uint32_t row_bytes = (uint32_t)g.k;
  const u32x4_t rsA = rsrc_words(g.a, (uint32_t)g.m * row_bytes);
  const u32x4_t rsB = rsrc_words(g.w, (uint32_t)g.n * row_bytes);
  uint32_t voffA, voffB;
  const uint32_t step64 = 64u * row_bytes;
  uint32_t fillA = lds0 + wave * 1024, fillB = lds0 + RING_B_OFF + wave * 1024;
  const uint32_t past = (uint32_t)((lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7)) * 16u >= (uint32_t)(g.k - (n_stages - 1) * BK) ? 0xFFFFFFF0u : 0u;
  auto fill_a = [&](int slot, int stage, int q) {
    lds_fill(rsA, fillA + (uint32_t)slot * STAGE_BYTES + q * 8192, (voffA + (uint32_t)q * step64) | (stage == n_stages - 1 ? past : 0u), (uint32_t)stage * BK);
  };
  auto fill_b = [&](int slot, int hh, int stage, int q) {
    lds_fill(rsB, fillB + (uint32_t)slot * STAGE_BYTES + hh * (STAGE_BYTES / 2) + q * 8192,
             (voffB + (uint32_t)(2 * q + hh) * step64) | (stage == n_stages - 1 ? past : 0u), (uint32_t)stage * BK);
  };

  // ---- scale bytes: of rows wm0 + 32i + lr, and of the wave's columns ----
  const int pitch = fp8_scale_pitch(g.k);
  const __amdgpu_buffer_rsrc_t rsSA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.a_scales), 0, (uint32_t)g.m * (uint32_t)pitch, 0x00020000);
  uint32_t wordA[2][WORDS], wordW[WORDS], nextA[2][WORDS], nextW[WORDS];
  auto ask_scales = [&](int m0, int n0, int stage) {
    int l = lane;
    forget(l);
    const uint32_t at = (uint32_t)(m0 + wm0 + (l & 31)) * (uint32_t)pitch;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const int word = fp8_scale_word_offset(stage / 4 + w, pitch);
      nextA[0][w] = __builtin_amdgcn_raw_buffer_load_b32(rsSA, at, word, 0);
      nextA[1][w] = __builtin_amdgcn_raw_buffer_load_b32(rsSA, at + 32u * (uint32_t)pitch, word, 0);
      nextW[w] = weight_scale_word(g, n0 + wn0, pitch, stage / 4 + w);
    }
  };
  auto take_scales = [&]() {               // (pinned here: waiting for them is waiting for every fill before them)
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      wordA[0][w] = nextA[0][w]; wordA[1][w] = nextA[1][w];
      wordW[w] = nextW[w];
      forget(wordA[0][w]); forget(wordA[1][w]);
    }
  };

  // ---- fragment reads: row R, chunk c of a stage sits at R*128 + (c ^ ((R/2)%8))*16.  A fragment of 64 k is the four
  //      chunks 4s .. 4s+3, the even ones to lanes 0-31: both operands take k in this order ----
  uint32_t firstA = lds0 + (uint32_t)(lr * 128 + ((lh ^ ((lr >> 1) & 7)) * 16)), firstB = firstA;      // chunk lh of row lr
  firstA += wm0 * 128;
  firstB += RING_B_OFF + (wn0 / 2) * 128;
  auto frag = [&](uint32_t from, int slice, uint32_t offset) {
    typedef const __attribute__((address_space(3))) u32x4_t* lds_t;
    const u32x4_t lo = *(lds_t)(size_t)((from ^ (uint32_t)(64 * slice)) + offset), hi = *(lds_t)(size_t)((from ^ (uint32_t)(64 * slice + 32)) + offset);
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  floatx16_t acc[2][4];
  i32x8_t fa[2][2], fb[4];                 // A fragments [slice][32 rows]; W fragments of a half stage
  int scaleA[2], scaleW;
  // Half `hh` of stage t: MFMA x = 0..7 has slice x/4, W fragment x/2 (columns 64*hh + 32*(x/2%2)), A fragment x%2; each runs
  // four steps after its first fragment was asked for, the last four of a half after the next barrier.
  auto mma = [&](int x, int h) {
    const int sl = x >> 2, j = 2 * (h & 1) + ((x >> 1) & 1), i = x & 1;
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[x >> 1], fa[sl][i], acc[i][j], 0, 0, 0, scaleW, 0, scaleA[i]);
  };
  auto half_stage = [&](auto H, int t) {         // H: of the twelve halves after which slots and registers come round again
    constexpr int h = decltype(H)::value, SA = h / 2 % 3, SB = h / 2 % 2, hh = h % 2;
    // All but the eight newest fills have landed: this half of W, and at the first half all of A; every wave's reads of
    // the half before are complete: its slot of W (at the first half: A's slot of stage t-1 too) is free.
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    // (what follows from these is formed here again and not held in registers through the loop)
    forget(firstA); forget(firstB); forget(voffA); forget(voffB);
    forget_scalar(fillA); forget_scalar(fillB);
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      // the half of W three halves on, half of A two stages on (past the last stage it is fetched once more into the idle
      // slot: in bounds, never read)
      if (y < 2) fill_b(hh == 0 ? SB ^ 1 : SB, hh ^ 1, min(t + 1 + hh, it.end - 1), y);
      else if (y < 4) fill_a((SA + 2) % 3, min(t + 2, it.end - 1), 2 * hh + y - 2);
      if (hh == 0 && y == 4) {
        // the stage's own scales: byte 0 of the words, which move down by one
#pragma unroll
        for (int i = 0; i < 2; ++i) scaleA[i] = (int)wordA[i][0];
        scaleW = (int)wordW[0];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            wordA[i][w] = w + 1 < WORDS ? __builtin_amdgcn_alignbit(wordA[i][w + 1], wordA[i][w], 8) : wordA[i][w] >> 8;
          wordW[w] = w + 1 < WORDS ? (wordW[w] >> 8 | wordW[w + 1] << 24) : wordW[w] >> 8;
        }
      }
      if (hh == 0 && (y & 3) < 2) fa[y >> 2][y & 1] = frag(firstA, y >> 2, SA * STAGE_BYTES + (y & 1) * 4096);
      if ((y & 1) == 0) fb[y >> 1] = frag(firstB, y >> 2, SB * STAGE_BYTES + hh * (STAGE_BYTES / 2) + ((y >> 1) & 1) * 4096);
      if (y >= 4) mma(y - 4, h);
      else if (h != 0 || t != it.begin) mma(y + 4, h + 11);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto stage = [&](auto S, int t) {
    half_stage(std::integral_constant<int, 2 * decltype(S)::value>{}, t);
    half_stage(std::integral_constant<int, 2 * decltype(S)::value + 1>{}, t);
  };
  // what an item's main loop needs first: A and W of its first stage, A of the second
  auto start_item = [&]() {
    int l = lane;
    forget(l);
    const uint32_t at = (uint32_t)(wave * 8 + (l >> 3)) * row_bytes + (uint32_t)((l & 7) ^ ((wave * 4 + (l >> 4)) & 7)) * 16u;
    voffA = (uint32_t)it.m0 * row_bytes + at;
    voffB = (uint32_t)it.n0 * row_bytes + at;
    const int second = min(it.begin + 1, it.end - 1);
#pragma unroll
    for (int q = 0; q < 4; ++q) fill_a(0, it.begin, q);
#pragma unroll
    for (int q = 0; q < 2; ++q) fill_b(0, 0, it.begin, q);
    // (the eight that the first barrier need not wait for, in the order in which later ones do)
#pragma unroll
    for (int q = 0; q < 2; ++q) fill_b(0, 1, it.begin, q);
#pragma unroll
    for (int q = 0; q < 2; ++q) fill_a(1, second, q);
#pragma unroll
    for (int q = 0; q < 2; ++q) fill_b(1, 0, second, q);
#pragma unroll
    for (int q = 2; q < 4; ++q) fill_a(1, second, q);
  };
  uint32_t bias = load_bias(g, it.n0 + wn0, lane, it.part >= 0);           // (cut tiles: added by the fix-up kernel)
  ask_scales(it.m0, it.n0, it.begin);
  start_item();
  take_scales();
  for (;;) {
    begin_with(bias, lane, acc);
    for (int t0 = it.begin;;) {
      const int group_end = min(t0 + GROUP, it.end);
      if (group_end < it.end) ask_scales(it.m0, it.n0, group_end);
      for (int t = t0; t < group_end; t += 6) {
        stage(std::integral_constant<int, 0>{}, t);
        if (t + 1 < group_end) stage(std::integral_constant<int, 1>{}, t + 1);
        if (t + 2 < group_end) stage(std::integral_constant<int, 2>{}, t + 2);
        if (t + 3 < group_end) stage(std::integral_constant<int, 3>{}, t + 3);
        if (t + 4 < group_end) stage(std::integral_constant<int, 4>{}, t + 4);
        if (t + 5 < group_end) stage(std::integral_constant<int, 5>{}, t + 5);
      }
      t0 = group_end;
      if (t0 >= it.end) break;
      take_scales();
    }
#pragma unroll
    for (int x = 4; x < 8; ++x) mma(x, 1);

    // Every wave is done with the rings, and no fill is in flight.  The next item's first fills go out before this one's
    // result is stored: they arrive, and the stores drain, behind other work.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const Item done = it;
    it = item_from(it.index + gridDim.x);
    if (it.index >= 0) {
      bias = load_bias(args_again().g, it.n0 + wn0, lane, it.part >= 0);
      ask_scales(it.m0, it.n0, it.begin);
      start_item();
    }
    int l = lane;
    forget(l);                             // (addresses are formed here, not held in registers through the loop)
    if (done.part >= 0) {
      float* part = args_again().sk.ws + (size_t)done.part * 65536 + wave * 256 + l * 4;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            floatx4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            *reinterpret_cast<floatx4_t*>(part + ((i * 4 + j) * 4 + q) * 2048) = v;
          }
    } else {
      // staging lies in the slot that the next item fills after its first barrier: the third of A
      char* region = reinterpret_cast<char*>(smem) + 2 * STAGE_BYTES + wave * STAGING;
      store_tile<QUANT, GELU>(args_again().g, acc, done.m0, wm0, done.n0 + wn0, l, region);
    }
    if (it.index < 0) return;
    take_scales();
  }
}

// Adds up the chunks of the cut tiles and stores the result: a one-wave workgroup to each 64 x 128 part of a tile.  Bound by the
// partial sums, read once and past the caches, 0.26 us a MB.
template <bool QUANT, bool GELU>
__global__ __launch_bounds__(64) void gemm256_fp8_fixup_kernel(GemmFp8Args g, Grid grid, Split sk) {
  const int tile = blockIdx.x >> 3, wave = blockIdx.x & 7, lane = threadIdx.x;
  int m0, n0;
  if (!origin(grid, sk.full_items + tile, 256, 256, m0, n0)) return;
  extern __shared__ u32x4_t smem[];
  floatx16_t acc[2][4];
  const int nw = n0 + (wave >> 2) * 128;
  begin_with(load_bias(g, nw, lane, false), lane, acc);
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
  store_tile<QUANT, GELU>(g, acc, m0, (wave & 3) * 64, nw, lane, reinterpret_cast<char*>(smem));
}

template <bool QUANT, bool GELU>
hipError_t launch_quarters(const GemmFp8Args& g, const Grid& grid, hipStream_t st);

// quarters: the tiles of the last, partly filled round go to a second kernel, four workgroups to a tile
template <bool QUANT, bool GELU>
hipError_t launch_gemm256_fp8(const GemmFp8Args& g, int split, bool quarters, hipStream_t st) {
  static std::atomic<uint64_t> lds_allowed{0};
  auto kern = gemm256_fp8_kernel<QUANT, GELU>;
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), GEMM256_LDS, lds_allowed);
  if (e != hipSuccess) return e;
  const Grid grid = make_grid(g, 256, 256);
  const int slots = grid.per_xcd * 8;
  const int whole = slots / 256 * 256;
  if (quarters) {
    // (no item after the whole ones)
    if (whole > 0) hipLaunchKernelGGL(kern, dim3(256), dim3(512), GEMM256_LDS, st, Args256{g, grid, Split{whole, 0, nullptr, Divisor()}});
    return whole < slots ? launch_quarters<QUANT, GELU>(g, grid, st) : hipGetLastError();
  }
  const Split sk = {split > 1 ? whole : slots, split, g.scratch, divisor((uint32_t)split, 1u << 28)};
  const int cut = slots - sk.full_items;
  if ((size_t)cut * sk.split * 262144 > (cut > 0 ? g.scratch_bytes : 0)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kern, dim3(std::min(sk.full_items + cut * sk.split, 256)), dim3(512), GEMM256_LDS, st, Args256{g, grid, sk});
  if (cut > 0)
    hipLaunchKernelGGL((gemm256_fp8_fixup_kernel<QUANT, GELU>), dim3(cut * 8), dim3(64), STAGING, st, g, grid, sk);
  return hipGetLastError();
}


// ------------------------------------------------------------------------------------------
// Smaller problems.  Their kernels end in stream_tile, which takes the fp32 sums row by row.
// ------------------------------------------------------------------------------------------

// BM x BN sums at (m0, n0), eight neighbouring ones from load(row, column, v), to the result, by NT threads.  In 8 bits a row
// of 128 columns lies in 16 neighbouring lanes, which find its scale (BN = 128, and whole rounds of all threads of a wave).
template <bool QUANT, bool GELU, int BM, int BN, int NT, typename Load>
__device__ __forceinline__ void stream_tile(const GemmFp8Args& g, int m0, int n0, int tid, Load load) {
  constexpr int PIECES = BN / 8;
  static_assert(!QUANT || (BN == 128 && BM * PIECES % 64 == 0), "a row's block lies in 16 lanes");
  const int out_pitch = fp8_scale_pitch(g.n), block = n0 >> 7, blocks = (g.n + 127) >> 7;
  const bf16_t* bias = g.bias != nullptr ? g.bias : reinterpret_cast<const bf16_t*>(g.w);   // (any readable place)
  for (int p = tid; p < BM * PIECES; p += NT) {
    const int ml = p / PIECES, nl = (p - ml * PIECES) * 8, m = m0 + ml, n = n0 + nl;
    float v[8];
    load(ml, nl, v);
    u32x4_t b = *reinterpret_cast<const u32x4_t*>(bias + min(n, g.n - 8));
    if (g.bias == nullptr) b = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] += unpack_lo(b[e]); v[2 * e + 1] += unpack_hi(b[e]); }
    if (GELU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = gelu_tanh(v[e]);
    }
    if (!QUANT) {
      u32x4_t out;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = pack_bf16x2_hw(v[2 * e], v[2 * e + 1]);
      if (m < g.m && n < g.n) *reinterpret_cast<u32x4_t*>(g.c + (int64_t)m * g.n + n) = out;
    } else {
      float largest = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) largest = fmaxf(largest, n < g.n ? finite_size(v[e]) : 0.f);
      const uint32_t byte = fp8_scale_of(max_of_16_lanes(largest));
      if (m < g.m && n < g.n) {
        const u32x2_t out = {pack_fp8x4(v[0], v[1], v[2], v[3], byte),
                             pack_fp8x4(v[4], v[5], v[6], v[7], byte)};
        *reinterpret_cast<u32x2_t*>(g.out.q + (int64_t)m * g.n + n) = out;
      }
      if (m < g.m && nl == 0) {
        uint8_t* s = g.out.scales + (int64_t)m * out_pitch;
        s[block] = (uint8_t)byte;
        if (block == blocks - 1)
          for (int x = blocks; x < out_pitch; ++x) s[x] = (uint8_t)FP8_SCALE_ONE;
      }
    }
  }
}

// Tiles of less than 256 x 256 cut along k: slots 0 .. full_items - 1 are whole work items, the `tiles` slots after them are cut
// in `chunks`, whose sums ([BM][BN] floats a chunk) the fix-up kernel adds up.  All first chunks, then all second ones, ..., so
// that the chunks of a tile stay on the XCD that owns its range of tiles (slots are a multiple of 8).
struct Cut {
  int32_t full_items, tiles, chunks;
  float* parts;
  Divisor by_tiles, by_chunks;
};
// QUARTERS: the tiles after full_items are 256 x 256, of which a "chunk" is a quarter of 128 x 128 with all of k.
struct CutItem { int slot, chunk, n_chunks; };
template <bool QUARTERS>
__device__ __forceinline__ CutItem cut_item(const Cut& cut) {
  const int r = QUARTERS ? (int)blockIdx.x : (int)blockIdx.x - cut.full_items;      // (a kernel for quarters has nothing else)
  if (r < 0) return {(int)blockIdx.x, 0, 1};
  const int chunk = (int)divide((uint32_t)r, cut.by_tiles);
  return {cut.full_items + r - chunk * cut.tiles, chunk, cut.chunks};
}

// BM x BN tile, eight waves: 2 x 2 sub-tiles, each computed by two waves that take one half of every stage of 128 k.  The
// sub-tile is then large (few LDS reads a flop) with two waves on every SIMD.  Stages go global -> LDS into a ring of RING
// slots, filled RING - 1 stages ahead, one barrier a stage; a slot holds the BM rows of A, then the BN rows of W.  As in the
// 256 x 256 kernel the MFMAs of a stage's last W fragment run after the next barrier, while the first fragments arrive.
// Bound by what a CU takes in, 65 to 75 KB/us by such fills: 128 x 128 takes 4 us and 0.48 us a stage of 32 KB (with all 256 CUs
// at work 0.7), 192 x 192 7 and 0.78 to 1.03 of 48 KB.  4485 x 1920 x 7680, 240 tiles of 192 x 192: 66 us, 2.0 PFLOP/s.
template <int BM, int BN>
struct HalfK {
  static constexpr int STAGE = (BM + BN) * 128;                          // bytes
  static constexpr int RING = 163840 / STAGE < 4 ? 163840 / STAGE : 4;
  static constexpr int TILE_BYTES = BM * (BN + 4) * 4;
  static constexpr int LDS = RING * STAGE > TILE_BYTES ? RING * STAGE : TILE_BYTES;
  static constexpr int WORDS = BM <= 128 ? 6 : BM + BN <= 320 ? 4 : 2;   // scale words of a row that are held: what the registers allow
};

template <int BM, int BN, bool QUARTERS, bool QUANT, bool GELU>
__global__ __launch_bounds__(512) void gemm_fp8_halfk_kernel(GemmFp8Args g, Grid grid, Cut cut) {
  using C = HalfK<BM, BN>;
  constexpr int MB = BM / 64, NB = BN / 64;            // 32 x 32 blocks of a wave's BM/2 x BN/2 sub-tile
  constexpr int NF = (BM + BN) / 64;                   // 1 KB fills of a wave per stage
  constexpr int RING = C::RING, STAGE = C::STAGE, WORDS = C::WORDS, GROUP = 4 * WORDS;
  constexpr int STEPS = MB * NB, NW = BN == 128 ? 1 : NB;              // scale blocks among a wave's columns
  static_assert(BM % 64 == 0 && BN % 64 == 0 && RING >= 3 && NB >= 2, "tile shape");
  CutItem it = cut_item<QUARTERS>(cut);
  int m0, n0;
  if (QUARTERS) {
    if (!origin(grid, it.slot, 256, 256, m0, n0)) return;
    m0 += (it.chunk & 1) * 128;
    n0 += (it.chunk >> 1) * 128;
    if (m0 >= g.m || n0 >= g.n) return;
    it.n_chunks = 1;
  } else if (!origin(grid, it.slot, BM, BN, m0, n0)) {
    return;
  }

  extern __shared__ u32x4_t smem[];
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)smem;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);             // waves w and w+4 share a SIMD
  const int wm0 = (wave & 1) * (BM / 2), wn0 = ((wave >> 1) & 1) * (BN / 2), kg = wave >> 2;
  const int lr = lane & 31, lh = lane >> 5;

  // fills: this wave's blocks of eight rows are wave + 8i of the slot's (BM + BN) / 8
  const uint32_t row_bytes = (uint32_t)g.k;
  const u32x4_t rsA = rsrc_words(g.a, (uint32_t)g.m * row_bytes);
  const u32x4_t rsB = rsrc_words(g.w, (uint32_t)g.n * row_bytes);
  const int row = wave * 8 + (lane >> 3);
  const uint32_t fill_chunk = (lane & 7) ^ ((row >> 1) & 7);
  const uint32_t voffA = (uint32_t)(m0 + row) * row_bytes + fill_chunk * 16, voffB = (uint32_t)(n0 + row) * row_bytes + fill_chunk * 16;
  const uint32_t step64 = 64u * row_bytes;
  const int n_stages = (g.k + BK - 1) / BK;
  const int stage_begin = it.n_chunks == 1 ? 0 : chunk_begin(it.chunk, it.n_chunks, cut.by_chunks, n_stages);
  const int stage_end = it.n_chunks == 1 ? n_stages : chunk_begin(it.chunk + 1, it.n_chunks, cut.by_chunks, n_stages);
  const uint32_t past = fill_chunk * 16 >= (uint32_t)(g.k - (n_stages - 1) * BK) ? 0xFFFFFFF0u : 0u;
  auto fill = [&](int slot, int want, int i) {
    const int stage = min(want, stage_end - 1);        // (past the end: the last stage again, unread)
    const uint32_t v = i < BM / 64 ? voffA + (uint32_t)i * step64 : voffB + (uint32_t)(i - BM / 64) * step64;
    lds_fill(i < BM / 64 ? rsA : rsB, lds0 + wave * 1024 + i * 8192 + (uint32_t)slot * STAGE, v | (stage == n_stages - 1 ? past : 0u),
             (uint32_t)stage * BK);
  };

  const int pitch = fp8_scale_pitch(g.k);
  const __amdgpu_buffer_rsrc_t rsSA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.a_scales), 0, (uint32_t)g.m * (uint32_t)pitch, 0x00020000);
  const uint32_t offSA = (uint32_t)(m0 + wm0 + lr) * (uint32_t)pitch;
  uint32_t wordA[MB][WORDS], nextA[MB][WORDS], wordW[NW][WORDS], nextW[NW][WORDS];
  auto ask_scales = [&](int stage) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
        nextA[i][w] = __builtin_amdgcn_raw_buffer_load_b32(rsSA, offSA + 32u * i * (uint32_t)pitch, fp8_scale_word_offset(stage / 4 + w, pitch), 0);
#pragma unroll
      for (int j = 0; j < NW; ++j) nextW[j][w] = weight_scale_word(g, n0 + wn0 + 32 * j, pitch, stage / 4 + w);
    }
  };

  uint32_t first = (uint32_t)(lr * 128 + ((lh ^ ((lr >> 1) & 7)) * 16)) ^ (uint32_t)(64 * kg);
  const uint32_t baseA = lds0 + wm0 * 128, baseB = lds0 + (BM + wn0) * 128;
  auto frag = [&](uint32_t base, int i) {
    typedef const __attribute__((address_space(3))) u32x4_t* lds_t;
    const u32x4_t lo = *(lds_t)(size_t)(first + base + i * 4096), hi = *(lds_t)(size_t)((first ^ 32u) + base + i * 4096);
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  floatx16_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  i32x8_t fa[2][MB], fb[NB];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int i = 0; i < MB; ++i) fa[1][i][e] = fa[0][i][e] = 0;
#pragma unroll
    for (int j = 0; j < NB; ++j) fb[j][e] = 0;
  }
  int scaleA[MB], scaleW[NW];
#pragma unroll
  for (int i = 0; i < MB; ++i) scaleA[i] = (int)FP8_SCALE_ONE;
#pragma unroll
  for (int j = 0; j < NW; ++j) scaleW[j] = (int)FP8_SCALE_ONE;
  auto mma = [&](int set, int x) {
    const int i = x % MB, j = x / MB;
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[set][i], acc[i][j], 0, 0, 0, scaleW[NW == 1 ? 0 : j], 0, scaleA[i]);
  };
  int slot = 0;
  auto stage = [&](auto SET, int t) {
    constexpr int P = decltype(SET)::value;
    // all but the fills of the RING - 2 newest stages have landed: stage t is in LDS; every wave's fragment reads of stage
    // t-1 are complete, so its slot can be filled again
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((RING - 2) * NF) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    forget(first);
    const uint32_t so = (uint32_t)slot * STAGE;
    const int refill = slot == 0 ? RING - 1 : slot - 1;
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      if (y < NF) fill(refill, t + RING - 1, y);
      if (y == STEPS - 1) {
#pragma unroll
        for (int z = STEPS; z < NF; ++z) fill(refill, t + RING - 1, z);
      }
      if (y == MB) {
#pragma unroll
        for (int i = 0; i < MB; ++i) scaleA[i] = (int)wordA[i][0];
#pragma unroll
        for (int j = 0; j < NW; ++j) scaleW[j] = (int)wordW[j][0];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
#pragma unroll
          for (int i = 0; i < MB; ++i) wordA[i][w] = w + 1 < WORDS ? __builtin_amdgcn_alignbit(wordA[i][w + 1], wordA[i][w], 8) : wordA[i][w] >> 8;
#pragma unroll
          for (int j = 0; j < NW; ++j) wordW[j][w] = w + 1 < WORDS ? (wordW[j][w] >> 8 | wordW[j][w + 1] << 24) : wordW[j][w] >> 8;
        }
      }
      if (y < MB) fa[P][y] = frag(baseA + so, y);
      if (y % MB == 0) fb[y / MB] = frag(baseB + so, y / MB);
      if (y < MB) mma(P ^ 1, STEPS - MB + y);
      else mma(P, y - MB);
      __builtin_amdgcn_sched_barrier(0);
    }
    slot = slot == RING - 1 ? 0 : slot + 1;
  };
  ask_scales(stage_begin);
#pragma unroll
  for (int s = 0; s < RING - 1; ++s)
#pragma unroll
    for (int i = 0; i < NF; ++i) fill(s, stage_begin + s, i);
  for (int t0 = stage_begin; t0 < stage_end; t0 += GROUP) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        wordA[i][w] = nextA[i][w];
        forget(wordA[i][w]);
      }
#pragma unroll
      for (int j = 0; j < NW; ++j) wordW[j][w] = nextW[j][w];
    }
    if (t0 + GROUP < stage_end) ask_scales(t0 + GROUP);
    const int group_end = min(t0 + GROUP, stage_end);
    for (int t = t0; t < group_end; t += 2) {
      stage(std::integral_constant<int, 0>{}, t);
      if (t + 1 < group_end) {
        stage(std::integral_constant<int, 1>{}, t + 1);
      } else {
        // an odd number of stages: the next set to be read is the other one again
#pragma unroll
        for (int i = 0; i < MB; ++i) fa[1][i] = fa[0][i];
      }
    }
  }
#pragma unroll
  for (int y = 0; y < MB; ++y) mma(1, STEPS - MB + y);

  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();                       // every wave is done with the ring, and no fill is in flight
  float* tile = reinterpret_cast<float*>(smem);
  constexpr int LDT = BN + 4;
  float* mine = tile + (wm0 + lr) * LDT + wn0 + 4 * lh;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (kg == half) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            floatx4_t* p = reinterpret_cast<floatx4_t*>(mine + 32 * i * LDT + 32 * j + 8 * q);
            floatx4_t v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            if (half == 1) {
              const floatx4_t o = *p;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += o[e];
            }
            *p = v;
          }
    }
    __syncthreads();
  }
  if (it.n_chunks > 1) {
    float* part = cut.parts + ((size_t)(it.slot - cut.full_items) * it.n_chunks + it.chunk) * (BM * BN);
    for (int p = tid; p < BM * BN / 4; p += 512)
      __builtin_nontemporal_store(*reinterpret_cast<const floatx4_t*>(tile + p / (BN / 4) * LDT + p % (BN / 4) * 4), reinterpret_cast<floatx4_t*>(part + p * 4));
    return;
  }
  stream_tile<QUANT, GELU, BM, BN, 512>(g, m0, n0, tid, [&](int ml, int nl, float* v) { ResidIO<float>::load8(tile + ml * LDT + nl, v); });
}

// Adds up the chunks of cut tiles and stores the result; 16 rows of a tile to a workgroup, so that small problems have some
// 256 of them (226 x 1920 x 7680 in six chunks, 12 MB: 4.2 us).
template <int BM, int BN, bool QUANT, bool GELU>
__global__ __launch_bounds__(256) void gemm_fp8_fixup_kernel(GemmFp8Args g, Grid grid, Cut cut) {
  constexpr int ROWS = 16;
  const int tile = blockIdx.x / (BM / ROWS), r0 = blockIdx.x % (BM / ROWS) * ROWS;
  int m0, n0;
  if (!origin(grid, cut.full_items + tile, BM, BN, m0, n0)) return;
  const float* part = cut.parts + (size_t)tile * cut.chunks * (BM * BN) + r0 * BN;
  stream_tile<QUANT, GELU, ROWS, BN, 256>(g, m0 + r0, n0, threadIdx.x, [&](int ml, int nl, float* v) {
    const float* p = part + ml * BN + nl;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 4
    for (int c = 0; c < cut.chunks; ++c) {
      float w[8];
      ResidIO<float>::load8(p + (size_t)c * (BM * BN), w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
  });
}

// Few tiles: what counts is that operands are asked for early, many at once, and taken in by every CU.  A workgroup has 16 * R rows and
// 16 * C columns (8-bit results: 128, a block) and its waves share k, each with a ring of RING slots of its own, so there is no
// barrier until the sums meet in LDS.  v_mfma_scale_f32_16x16x128_f8f6f4 (A fragment: lane holds row lane%16 and a quarter of
// 128 k; accumulator register i of a lane is row 4*(lane/16) + i, column lane%16): a stage of 128 k is one step.
// Bound by what a CU takes in, 80 to 90 KB/us, after a start of 2 to 3 us: 226 x 1920 x 1920 in tiles of 32 x 64 takes 5.4 us (tiles
// of 128 x 128 11.8, of 32 x 16 10.2), 128 x 4096 x 4096 8.2 (17.3 cut along k, 16.7), 226 x 1920 x 7680 11.7 (17.2, 22.2);
// 1 x 7680 x 1920 in tiles of 16 x 16 3.7 us back to back, 4 TB/s of weights.  A slot each for eight waves is as good as three
// each for four.  Operands loaded straight into registers took twice as long: such a load touches 16 lines where one into LDS
// touches eight.
template <int R, int C, int WAVES, int RING>
struct SharedK {
  static constexpr int STAGE = 16 * (R + C) * 128;                        // bytes: the rows of A, then those of W
  static constexpr int WAVE = RING * STAGE + (R + 1) * 1024;               // and scale bytes of 64 stages: of the rows of A, of W
  static constexpr int LDT = 16 * C + 4, SUMS = WAVES * 16 * R * LDT * 4;
  static constexpr int LDS = WAVES * WAVE > SUMS ? WAVES * WAVE : SUMS;
};

constexpr int SHARED_STAGES = 60;    // most stages of a wave: 64, as its scale bytes begin on a whole word

template <int R, int C, int WAVES, int RING, bool QUANT, bool GELU>
__global__ __launch_bounds__(64 * WAVES) void gemm_fp8_shared_kernel(GemmFp8Args g, Grid grid) {
  using S = SharedK<R, C, WAVES, RING>;
  constexpr int STAGE = S::STAGE, NF = 2 * (R + C), LDT = S::LDT;
  int m0, n0;
  if (!origin(grid, blockIdx.x, 16 * R, 16 * C, m0, n0)) return;
  extern __shared__ u32x4_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) void*)smem) + wave * S::WAVE;
  const uint32_t scales = ring + RING * STAGE;
  const uint32_t row_bytes = (uint32_t)g.k;
  const u32x4_t rsA = rsrc_words(g.a, (uint32_t)g.m * row_bytes);
  const u32x4_t rsB = rsrc_words(g.w, (uint32_t)g.n * row_bytes);
  const int n_stages = (g.k + BK - 1) / BK;
  const int begin = wave * n_stages / WAVES, end = (wave + 1) * n_stages / WAVES;
  // scale bytes: lane l brings those of row l/4, stages 16 * (l%4) .. +15 from the word of `begin` on; W's one row in lanes 0-3
  const int pitch = fp8_scale_pitch(g.k), scale_begin = begin & ~3;
  {
    const u32x4_t rsSA = rsrc_words(g.a_scales, (uint32_t)g.m * (uint32_t)pitch);
    const u32x4_t rsSW = rsrc_words(g.w_scales, (uint32_t)((g.n + 127) / 128) * (uint32_t)pitch);
    const uint32_t at = (uint32_t)(scale_begin + (lane & 3) * 16);
#pragma unroll
    for (int i = 0; i < R; ++i) lds_fill(rsSA, scales + i * 1024, (uint32_t)(m0 + 16 * i + (lane >> 2)) * (uint32_t)pitch + at);
    lds_fill(rsSW, scales + R * 1024, lane < 4 ? (uint32_t)(n0 / 128) * (uint32_t)pitch + at : 0xFFFFFFF0u);
  }
  auto fill = [&](int slot, int stage) {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int row = i * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
      const uint32_t past = stage * BK + chunk * 16 >= g.k ? 0xFFFFFFF0u : 0u;
      const uint32_t v = (uint32_t)(i < 2 * R ? m0 + row : n0 + row - 16 * R) * row_bytes + chunk * 16;
      lds_fill(i < 2 * R ? rsA : rsB, ring + (uint32_t)slot * STAGE + i * 1024, v | past, (uint32_t)stage * BK);
    }
  };
  floatx4_t acc[R][C];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[i][j] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < RING; ++s)
    if (begin + s < end) fill(s, begin + s);
  // chunks lq and lq + 4 of a row; both operands take k in this order
  const uint32_t first = (uint32_t)(lr * 128 + ((lq ^ ((lr >> 1) & 7)) * 16));
  typedef const __attribute__((address_space(3))) u32x4_t* lds_t;
  typedef const __attribute__((address_space(3))) uint8_t* lds_byte_t;
  auto frag = [&](uint32_t base) {
    const u32x4_t lo = *(lds_t)(size_t)(base + first), hi = *(lds_t)(size_t)(base + (first ^ 64u));
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  int slot = 0;
  for (int t = begin; t < end; ++t) {
    // the fills of the stages after this one may still be in flight
    const int newer = min(RING - 1, end - 1 - t);
    if (RING > 3 && newer == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(RING > 3 ? 3 * NF : 0) : "memory");
    else if (RING > 2 && newer == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(RING > 2 ? 2 * NF : 0) : "memory");
    else if (RING > 1 && newer == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(RING > 1 ? NF : 0) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    static_assert(RING <= 4 && (RING - 1) * NF < 64, "counts above");
    const uint32_t base = ring + (uint32_t)slot * STAGE, s = scales + (uint32_t)(t - scale_begin);
    const int scale_w = *(lds_byte_t)(size_t)(s + R * 1024);
    i32x8_t a[R], w[C];
    int scale_a[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      a[i] = frag(base + 2048 * i);
      scale_a[i] = *(lds_byte_t)(size_t)(s + i * 1024 + lr * 64);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) w[j] = frag(base + 2048 * (R + j));
    if (t + RING < end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                  // the slot has been read
      __builtin_amdgcn_sched_barrier(0);
      fill(slot, t + RING);
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < C; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j], a[i], acc[i][j], 0, 0, 0, scale_w, 0, scale_a[i]);
    slot = slot == RING - 1 ? 0 : slot + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                        // (a wave without stages has scale bytes on their way)
  __syncthreads();                       // every wave has read its last stage: no fill is in flight
  // acc[i][j][e] = C[m0 + 16i + lr][n0 + 16j + 4lq + e]
  float* tile = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j)
      *reinterpret_cast<floatx4_t*>(tile + (wave * 16 * R + 16 * i + lr) * LDT + 16 * j + 4 * lq) = acc[i][j];
  __syncthreads();
  stream_tile<QUANT, GELU, 16 * R, 16 * C, 64 * WAVES>(g, m0, n0, tid, [&](int ml, int nl, float* v) {
    ResidIO<float>::load8(tile + ml * LDT + nl, v);
#pragma unroll
    for (int c = 1; c < WAVES; ++c) {
      float w[8];
      ResidIO<float>::load8(tile + (c * 16 * R + ml) * LDT + nl, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
  });
}

template <int R, int C, int WAVES, int RING, bool QUANT, bool GELU>
hipError_t launch_shared(const GemmFp8Args& g, hipStream_t st) {
  static std::atomic<uint64_t> lds_allowed{0};
  constexpr int LDS = SharedK<R, C, WAVES, RING>::LDS;
  static_assert(LDS <= 163840, "LDS of a CU");
  if (((g.k + BK - 1) / BK + WAVES - 1) / WAVES > SHARED_STAGES) return hipErrorInvalidValue;
  auto kern = gemm_fp8_shared_kernel<R, C, WAVES, RING, QUANT, GELU>;
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), LDS, lds_allowed);
  if (e != hipSuccess) return e;
  const Grid grid = make_grid(g, 16 * R, 16 * C);
  hipLaunchKernelGGL(kern, dim3(grid.per_xcd * 8), dim3(64 * WAVES), LDS, st, g, grid);
  return hipGetLastError();
}

template <int BM, int BN, bool QUANT, bool GELU>
hipError_t launch_halfk(const GemmFp8Args& g, int chunks, hipStream_t st) {
  static std::atomic<uint64_t> lds_allowed{0};
  auto kern = gemm_fp8_halfk_kernel<BM, BN, false, QUANT, GELU>;
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), HalfK<BM, BN>::LDS, lds_allowed);
  if (e != hipSuccess) return e;
  const Grid grid = make_grid(g, BM, BN);
  const int slots = grid.per_xcd * 8, full = chunks > 1 ? slots / 256 * 256 : slots;
  const Cut cut = {full, slots - full, chunks, g.scratch, divisor((uint32_t)(slots - full), 4096), divisor((uint32_t)chunks, 1u << 28)};
  if ((size_t)cut.tiles * chunks * (BM * BN * 4) > (cut.tiles > 0 ? g.scratch_bytes : 0)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kern, dim3(full + (slots - full) * chunks), dim3(512), (HalfK<BM, BN>::LDS), st, g, grid, cut);
  if (slots > full)
    hipLaunchKernelGGL((gemm_fp8_fixup_kernel<BM, BN, QUANT, GELU>), dim3((slots - full) * (BM / 16)), dim3(256), 0, st, g, grid, cut);
  return hipGetLastError();
}

template <bool QUANT, bool GELU>
hipError_t launch_quarters(const GemmFp8Args& g, const Grid& grid, hipStream_t st) {
  static std::atomic<uint64_t> lds_allowed{0};
  auto kern = gemm_fp8_halfk_kernel<128, 128, true, QUANT, GELU>;
  constexpr int LDS = HalfK<128, 128>::LDS;
  hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), LDS, lds_allowed);
  if (e != hipSuccess) return e;
  const int slots = grid.per_xcd * 8, whole = slots / 256 * 256;
  const Cut cut = {whole, slots - whole, 4, nullptr, divisor((uint32_t)(slots - whole), 4096), Divisor()};
  hipLaunchKernelGGL(kern, dim3((slots - whole) * 4), dim3(512), LDS, st, g, grid, cut);
  return hipGetLastError();
}

// TILE_16 to TILE_64x128: whose waves share k; 8-bit results: 16 x 128, 32 x 128 and 64 x 128
enum TileKind { TILE_16, TILE_32, TILE_32x64, TILE_64, TILE_64x128, TILE_128, TILE_192x128, TILE_192, TILE_256 };

constexpr int TWO_SLOTS = 16;        // stages of 16 x 16 tiles that eight waves hold in two slots each

template <bool QUANT, bool GELU>
hipError_t launch_kind(const GemmFp8Args& g, TileKind kind, int chunks, hipStream_t st) {
  const int stages = (g.k + BK - 1) / BK;
  switch (kind) {
    case TILE_16:
      // one tile's weights: two slots a wave, and two workgroups to a CU, where they hold all its stages (1 x 7680 x 1920: 5.1 us with three
      // inputs in turns, 6.6 with four slots), else four (149 x 816 x 3008 8.2 -> 6.8).  A block of 128 columns: four waves with two
      // slots for the fewest stages (8160 columns, two stages: 3.9 us, eight waves with a slot 4.2), else eight (5 x 304 x 7344: 11.1, 12.8)
      if constexpr (QUANT) return stages <= 4 ? launch_shared<1, 8, 4, 2, QUANT, GELU>(g, st) : launch_shared<1, 8, 8, 1, QUANT, GELU>(g, st);
      else return stages <= TWO_SLOTS ? launch_shared<1, 1, 8, 2, QUANT, GELU>(g, st) : launch_shared<1, 1, 8, 4, QUANT, GELU>(g, st);
    case TILE_32:
      if constexpr (QUANT) return launch_shared<2, 8, 6, 1, QUANT, GELU>(g, st);
      else return launch_shared<2, 2, 8, 2, QUANT, GELU>(g, st);
    case TILE_32x64:
      if constexpr (QUANT) return hipErrorInvalidValue;
      else return launch_shared<2, 4, 8, 1, QUANT, GELU>(g, st);
    case TILE_64:
      if constexpr (QUANT) return hipErrorInvalidValue;
      else return launch_shared<4, 4, 4, 2, QUANT, GELU>(g, st);
    case TILE_64x128: return launch_shared<4, 8, 4, 1, QUANT, GELU>(g, st);
    case TILE_128: return launch_halfk<128, 128, QUANT, GELU>(g, chunks, st);
    case TILE_192x128: return launch_halfk<192, 128, QUANT, GELU>(g, chunks, st);
    case TILE_192:
      if constexpr (QUANT) return hipErrorInvalidValue;                  // a block of 128 columns would lie in two tiles
      else return launch_halfk<192, 192, QUANT, GELU>(g, chunks, st);
    case TILE_256: return launch_gemm256_fp8<QUANT, GELU>(g, chunks, chunks < 0, st);
  }
  return hipErrorInvalidValue;
}

// chunks: along k, of the tiles of the last round (1: not cut); -1 (256 x 256): they are computed in quarters
struct TileChoice { TileKind kind; int chunks; };

// Expected times (us), fitted to timings of every kind, cut and not, in both result types, those near the fastest weighing
// most: the tiles from 128 x 128 on to 1900 at 48 sizes (1 .. 17776 rows, n 96 .. 7680, k 64 .. 8192), those whose waves share k to
// 1000 at 72 (1 .. 2553 rows, n 16 .. 8160, k 192 .. 7872).  At the latter the kind chosen takes 2.4 % longer than the best of all
// kinds on average, 26 % at most (2 x 416 x 7168 in 8 bits: seven chunks where 16 x 128 tiles are better).  At 80 other sizes, drawn
// afterwards, with 64 MiB of scratch: 1.2 and 27 % at 30 of 1 .. 600 rows, 0.1 and 1.3 % at 30 of 600 .. 17776 rows (all of these
// with n and k to 8192), 3.7 and 14 % at 20 with k from 8192 to 16384, past what was fitted (1 x 8864 x 11024: 29.0 us, 25.4).
//
// Tiles: a round of at most 256 of them, one a CU, takes fixed + stages * rate; the rate rises from `low` to `high` as the last
// CUs come to work and the chip lowers its clock.  Per round at k = 1920: 128 x 128 14.5, 192 x 128 17.4, 192 x 192 22.4,
// 256 x 256 29.4 us.  [1]: results in 8 bits.
struct TileCost { int bm, bn; float fixed, low, high; };
constexpr TileCost TILE_COST[][2] = {{{128, 128, 4.0f, 0.48f, 0.70f}, {128, 128, 5.0f, 0.42f, 0.63f}},
                                     {{192, 128, 5.3f, 0.70f, 0.81f}, {192, 128, 6.7f, 0.51f, 0.76f}},
                                     {{192, 192, 7.0f, 0.78f, 1.03f}, {0, 0, 0.f, 0.f, 0.f}},
                                     {{256, 256, 5.7f, 1.11f, 1.58f}, {256, 256, 5.0f, 1.12f, 1.55f}}};
// Tiles whose waves share k: the stages of a wave, a share for each workgroup of a CU, and the bytes that a CU takes in, some 85 a ns.
struct SharedCost { int bm, bn, waves; float fixed, stage, group, per_mb; };
constexpr SharedCost SHARED_COST[][2] = {{{16, 16, 8, 2.4f, 0.f, 0.42f, 13.1f}, {16, 128, 8, 1.1f, 0.f, 2.2f, 11.1f}},
                                         {{32, 32, 8, 1.3f, 0.12f, 1.7f, 10.5f}, {32, 128, 6, 0.8f, 0.f, 3.3f, 11.6f}},
                                         {{32, 64, 8, 1.1f, 0.f, 2.2f, 11.6f}, {0, 0, 0, 0.f, 0.f, 0.f, 0.f}},
                                         {{64, 64, 4, 0.4f, 0.24f, 3.0f, 12.3f}, {0, 0, 0, 0.f, 0.f, 0.f, 0.f}},
                                         {{64, 128, 4, 0.f, 0.53f, 4.2f, 10.9f}, {64, 128, 4, 0.f, 0.44f, 5.3f, 9.6f}}};
constexpr double FIXUP = 3.7, FIXUP_PER_MB = 0.26, SECOND_LAUNCH = 2.8;

double rounds_cost(const TileCost& c, int64_t items, double stages) {
  const double rem = (double)(items % 256) / 256.0;
  return (double)(items / 256) * (c.fixed + stages * c.high) +
         (rem > 0 ? c.fixed + stages * (c.low + rem * rem * rem * (c.high - c.low)) : 0.0);
}

// stages a chunk of a cut tile has at least: fewer do not cover the start of its pipeline
constexpr int LEAST_STAGES = 8, MOST_CHUNKS = 8;

TileChoice choose_tile(const GemmFp8Args& g) {
  const int quant = g.out.q != nullptr ? 1 : 0, stages = (g.k + BK - 1) / BK;
  TileChoice choice = {TILE_256, 1};
  double best = 1e30;
  auto consider = [&](TileKind kind, int chunks, double t) {
    if (t < best) { best = t; choice = {kind, chunks}; }
  };
  for (int kind = TILE_16; kind <= TILE_64x128; ++kind) {
    const SharedCost& c = SHARED_COST[kind][quant];
    if (c.bm == 0 || (stages + c.waves - 1) / c.waves > SHARED_STAGES) continue;
    // (up to 16 rows: no tile that is half empty, where 16 x 16 has two workgroups to a CU: 1 x 7680 x 1920 5.2 us, in tiles of 32 x 32 5.6;
    // 5 x 5488 x 1136 3.7, 4.0.  From 17 stages on the prices are right: 1 x 8192 x 8192 13.7 us in 16 x 16, 12.2 in 32 x 32, 12.7 in
    // 32 x 64; 1 x 7680 x 2304 7.2, 6.3, 6.4; 16 x 14336 x 4096 15.4, 13.0, 11.9; 1 x 1920 x 7680 5.8, 7.4, 9.9)
    if (quant == 0 && kind > TILE_16 && g.m <= 16 && stages <= TWO_SLOTS) continue;
    const int64_t tiles = (int64_t)((g.m + c.bm - 1) / c.bm) * ((g.n + c.bn - 1) / c.bn), a_cu = (tiles + 255) / 256;
    if (tiles > (1 << 20)) continue;
    consider((TileKind)kind, 1, c.fixed + c.stage * ((stages + c.waves - 1) / c.waves) + c.group * a_cu +
             c.per_mb * 1e-6 * (double)a_cu * stages * (c.bm + c.bn) * BK);
  }
  for (int kind = TILE_128; kind <= TILE_256; ++kind) {
    const TileCost& c = TILE_COST[kind - TILE_128][quant];
    if (c.bm == 0) continue;
    const int64_t tiles = (int64_t)((g.m + c.bm - 1) / c.bm) * ((g.n + c.bn - 1) / c.bn);
    const int64_t slots = (tiles + 7) / 8 * 8, whole = slots / 256 * 256, rem = slots - whole;
    consider((TileKind)kind, 1, rounds_cost(c, tiles, stages));
    if (rem == 0) continue;
    const double before = rounds_cost(c, whole, stages);
    if (kind == TILE_256)
      consider(TILE_256, -1, before + (whole > 0 ? SECOND_LAUNCH : 0.0) + rounds_cost(TILE_COST[0][quant], 4 * (tiles - whole), stages));
    if (g.scratch == nullptr || before + c.fixed + FIXUP >= best) continue;
    for (int s = 2; s <= MOST_CHUNKS && stages / s >= LEAST_STAGES; ++s) {
      const size_t bytes = (size_t)rem * s * c.bm * c.bn * 4;
      if (bytes > g.scratch_bytes) break;
      consider((TileKind)kind, s, before + rounds_cost(c, rem * s, (double)stages / s) + FIXUP + FIXUP_PER_MB * 1e-6 * (double)bytes);
    }
  }
  return choice;
}

}  // namespace

hipError_t launch_gemm_fp8(const GemmFp8Args& g, hipStream_t st) {
  if (g.m <= 0 || g.n <= 0) return hipSuccess;
  if (g.k <= 0 || g.k % 16 != 0 || g.n % 16 != 0) return hipErrorInvalidValue;
  // operands, and 256 rows of a result, are addressed with 32-bit byte offsets
  if (((int64_t)g.m + 512) * g.k >= (int64_t)1 << 32 || ((int64_t)g.n + 512) * g.k >= (int64_t)1 << 32 || g.n >= 1 << 23) return hipErrorInvalidValue;
  const TileChoice t = choose_tile(g);
  if (g.out.q) return g.gelu ? launch_kind<true, true>(g, t.kind, t.chunks, st) : launch_kind<true, false>(g, t.kind, t.chunks, st);
  return g.gelu ? launch_kind<false, true>(g, t.kind, t.chunks, st) : launch_kind<false, false>(g, t.kind, t.chunks, st);
}

void gemm_fp8_route(const GemmFp8Args& g, int* tile_m, int* tile_n, int* last) {
  const TileChoice t = choose_tile(g);
  const int quant = g.out.q != nullptr ? 1 : 0;
  *tile_m = t.kind < TILE_128 ? SHARED_COST[t.kind][quant].bm : TILE_COST[t.kind - TILE_128][quant].bm;
  *tile_n = t.kind < TILE_128 ? SHARED_COST[t.kind][quant].bn : TILE_COST[t.kind - TILE_128][quant].bn;
  *last = t.chunks;
}
