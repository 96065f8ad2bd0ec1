// The product of 8-bit scaled tensors,
//   C[m, n] = sum over blocks b of 128:  sa[b, m] sw[n / 128, b]  sum over k in b:  A[m, k] W[n, k].
//
// v_mfma_f32_16x16x128_f8f6f4 multiplies 16 rows of W by 16 rows of A over one whole scale block: lane l supplies 32 codes of
// row l % 16 of either operand, and gets D[n = 4 (l / 16) + e][m = l % 16], e < 4.  Which 32 of the 128 a lane holds does not
// matter as long as both operands agree: here the 16 at 16 (l / 16) and the 16 at 64 + 16 (l / 16), so that a load of 16
// bytes a lane takes 64 consecutive bytes of a row.  The product of a block starts from zero and is added to the fp32 sum
// with its scale, sum += d * (sa sw), in fp32.  Inside a block the instruction itself keeps less (measured, the same for the
// 16x16x32 form): it takes eight consecutive codes of a lane at a time and drops what their products have below 2^-13 of
// the power of two of the largest.  On activations with a few large channels that is 2.5e-5 of the result's size, 70 times
// below the rounding of a bf16 result and 1000 times below that of an 8-bit one; there is no fp32 result for that reason.
// Lane l needs the activation scale of its own row m only, and the weight scale is the
// same for all of a wave's columns.
#include <cstdio>
#include <type_traits>

#include "scaled.h"

namespace svdmlp {

struct MmP {
  const char *a, *w;
  const __bf16* sa;
  const float* sw;
  void* c;
  __bf16* c_scales;
  float* part;        // [ranges][M][N] partial sums
  int64_t a_ld, w_ld, sa_ld, c_ld, c_scales_ld;
  int M, N, K, KB;
  int out_type;
  int tiles;                  // of the result
  int band;                   // k_mm_tile: row tiles of a band of banded_tile; k_mm_ring: tiles of a strip
  int ranges, range_blocks;   // ranges of the contraction, blocks of 128 in each (the last may be shorter)
};

// Workgroups sum range after range of the contraction.  A division is 0.1 us before a workgroup's first load: left out where it can be.
__device__ __forceinline__ int range_of(int id, const MmP& p) {
  return p.ranges == 1 ? 0 : __builtin_amdgcn_readfirstlane(id / p.tiles);
}

__device__ __forceinline__ f32x4 mfma_f8(const i32x8& w, const i32x8& a, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, 0, 0, 0);
}

// codes c .. c + 15 of a row, those from K on zero.  Rows start on 16 bytes, so the 16 bytes that hold a code lie together.
__device__ __forceinline__ u32x4 codes16_to(const char* row, int c, int K) {
  const int last = (K - 1) & ~15;
  u32x4 v = *(const u32x4*)(row + (c < last ? c : last));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = K - c - 4 * i;   // codes of this word
    v[i] = left >= 4 ? v[i] : left <= 0 ? 0u : v[i] & (0xffffffffu >> (32 - 8 * left));
  }
  return v;
}
__device__ __forceinline__ i32x8 join16(const u32x4& lo, const u32x4& hi) {
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}
// this lane's 32 codes of block b of a row; FULL: the block ends before K
template <bool FULL>
__device__ __forceinline__ i32x8 block_codes(const char* row, int b, int g, int K) {
  const int c = b * SCALE_BLOCK + 16 * g;
  if (FULL) return join16(*(const u32x4*)(row + c), *(const u32x4*)(row + c + 64));
  return join16(codes16_to(row, c, K), codes16_to(row, c + 64, K));
}

// ---- up to 16 rows ------------------------------------------------------------------------------------
// The weights go from HBM straight into registers, once.  A workgroup has 16 columns and a range of the contraction, whose
// blocks go to its eight waves in turn, four at a time, all loads before the first product; the waves' sums meet in LDS.  One
// row by W[4096, 4096] takes 6.2 us in a graph, by W[8192, 4096] 8.7 us (5.4 TB/s without the 2.5 us of a launch with one
// load in it); two column tiles a workgroup 7.6 and 8.4 us, sixteen waves 6.3 and 8.5 us.
constexpr int FEW_WAVES = 8;
__global__ __launch_bounds__(64 * FEW_WAVES) void k_mm_few(MmP p) {
  __shared__ f32x4 red[FEW_WAVES][64];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int z = range_of(blockIdx.x, p), n0 = (blockIdx.x - z * p.tiles) * 16;
  const char* wr = p.w + (int64_t)min(n0 + r, p.N - 1) * p.w_ld;
  const char* ar = p.a + min(r, p.M - 1) * p.a_ld;
  const __bf16* sa = p.sa + min(r, p.M - 1);
  const float* sw = p.sw + (int64_t)(n0 / SCALE_BLOCK) * p.KB;
  f32x4 acc = {};
  // U blocks of this wave from b on
  auto blocks = [&](auto full, auto u, int b) {
    constexpr bool FULL = decltype(full)::value;
    constexpr int U = decltype(u)::value;
    i32x8 fw[U], fa[U];
    float s[U];
#pragma unroll
    for (int x = 0; x < U; ++x) {
      fw[x] = block_codes<FULL>(wr, b + x * FEW_WAVES, g, p.K);
      fa[x] = block_codes<FULL>(ar, b + x * FEW_WAVES, g, p.K);
      s[x] = (float)sa[(b + x * FEW_WAVES) * p.sa_ld] * sw[b + x * FEW_WAVES];
    }
#pragma unroll
    for (int x = 0; x < U; ++x) {
      const f32x4 d = mfma_f8(fw[x], fa[x], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += d[e] * s[x];
    }
  };
  constexpr std::true_type whole_block{};
  constexpr std::integral_constant<int, 1> one{};
  constexpr std::integral_constant<int, 2> two{};
  constexpr std::integral_constant<int, 4> four{};
  const int b0 = z * p.range_blocks, b1 = min(b0 + p.range_blocks, p.KB);
  const int whole = min(b1, p.K / SCALE_BLOCK);
  int b = b0 + wave;
  for (; b + 3 * FEW_WAVES < whole; b += 4 * FEW_WAVES) blocks(whole_block, four, b);
  if (b + FEW_WAVES < whole) {
    blocks(whole_block, two, b);
    b += 2 * FEW_WAVES;
  }
  if (b < whole) blocks(whole_block, one, b);
  if (whole < b1 && (whole - b0) % FEW_WAVES == wave) blocks(std::false_type{}, one, whole);
  red[wave][lane] = acc;
  __syncthreads();
  if (wave > 0 || r >= p.M) return;
  f32x4 v = red[0][lane];
#pragma unroll
  for (int w = 1; w < FEW_WAVES; ++w) v += red[w][lane];
  const int n = n0 + 4 * g;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= p.N) return;
    if (p.part) p.part[((int64_t)z * p.M + r) * p.N + n + e] = v[e];
    else ((__bf16*)p.c)[r * p.c_ld + n + e] = (__bf16)v[e];
  }
}

// ---- a wave's piece of the result ---------------------------------------------------------------------
// 16 MT rows from m0 and 16 NT columns from n0 on: lane l has, of its MT rows m0 + MT (l % 16) + i, the columns 16 j + 4 (l / 16) +
// 0..3, to be rounded or (PARTS, where there is a buffer for them) added up later.  It passes through LDS (MmResult::BYTES for
// each wave, free to use) so that rows leave in pieces of 32 NT bytes.
template <int MT, int NT>
struct MmResult {
  static constexpr int ROWS = MT < 4 ? 16 * MT : 64, LD = 32 * NT + 16;       // rows at a time, bytes per row
  static constexpr int BYTES = ROWS * LD + 64 * MT;
};

template <int MT, int NT, bool PARTS>
__device__ __forceinline__ void mm_result(const MmP& p, const f32x4 (&acc)[NT][MT], int z, int m0, int n0, int wave, char* lds) {
  using T = MmResult<MT, NT>;
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  if (PARTS && p.part) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = m0 + MT * r + i;
      if (m >= p.M) continue;
      float* q = p.part + ((int64_t)z * p.M + m) * p.N;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int n = n0 + 16 * j + 4 * g;
        if (n + 4 <= p.N) {
          __builtin_memcpy(q + n, &acc[j][i], 16);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < p.N) q[n + e] = acc[j][i][e];
        }
      }
    }
    return;
  }
  char* mine = lds + wave * T::BYTES;
  constexpr int IR = T::ROWS / 16;     // row tiles that pass through LDS at a time
  if (16 * NT == SCALE_BLOCK / 2 && p.out_type == SVDMLP_F8) {
    // largest magnitude of the block of 128 columns of which this wave and its neighbour hold half each
    float inv[MT];
    float* largest = (float*)(mine + T::ROWS * T::LD);
    const float* others = (const float*)(lds + (wave ^ 1) * T::BYTES + T::ROWS * T::LD);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float x = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n0 + 16 * j + 4 * g + e < p.N) x = fmaxf(x, fabsf(acc[j][i][e]));
      x = fmaxf(x, __shfl_xor(x, 16));
      x = fmaxf(x, __shfl_xor(x, 32));
      if (g == 0) largest[16 * i + r] = x;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = m0 + MT * r + i;
      const __bf16 s = scale_of(fmaxf(largest[16 * i + r], others[16 * i + r]));
      inv[i] = 1.f / (float)s;
      if (g == 0 && wave % 2 == 0 && m < p.M && n0 < p.N) p.c_scales[(int64_t)(n0 / SCALE_BLOCK) * p.c_scales_ld + m] = s;
    }
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += IR) {
#pragma unroll
      for (int i = i0; i < i0 + IR; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const f32x4 v = acc[j][i];
          *(unsigned*)(mine + (16 * (i - i0) + r) * T::LD + 16 * j + 4 * g) = codes4(v[0] * inv[i], v[1] * inv[i], v[2] * inv[i], v[3] * inv[i]);
        }
      // LDS accesses of a wave are done in order
#pragma unroll
      for (int k = 0; k < T::ROWS / (64 / NT); ++k) {
        const int row = 64 / NT * k + lane / NT, m = m0 + MT * (row % 16) + i0 + row / 16, n = n0 + 16 * (lane % NT);
        if (m >= p.M || n >= p.N) continue;
        const u32x4 v = *(const u32x4*)(mine + row * T::LD + 16 * (lane % NT));
        unsigned char* c = (unsigned char*)p.c + m * p.c_ld + n;
        if (n + 16 <= p.N) {
          *(u32x4*)c = v;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (n + e < p.N) c[e] = (unsigned char)(v[e / 4] >> (8 * (e % 4)));
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i0 = 0; i0 < MT; i0 += IR) {
#pragma unroll
    for (int i = i0; i < i0 + IR; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const f32x4 v = acc[j][i];
        *(bf16x4*)(mine + (16 * (i - i0) + r) * T::LD + 2 * (16 * j + 4 * g)) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
      }
    constexpr int L = 2 * NT;            // lanes a row
#pragma unroll
    for (int k = 0; k < T::ROWS / (64 / L); ++k) {
      const int row = 64 / L * k + lane / L, m = m0 + MT * (row % 16) + i0 + row / 16, n = n0 + 8 * (lane % L);
      if (m >= p.M || n >= p.N) continue;
      const u32x4 v = *(const u32x4*)(mine + row * T::LD + 16 * (lane % L));
      __bf16* c = (__bf16*)p.c + m * p.c_ld + n;
      if (n + 8 <= p.N) {
        __builtin_memcpy(c, &v, 16);
      } else {
        const bf16x8 x = as_bf16x8(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < p.N) c[e] = x[e];
      }
    }
  }
}

// sums <- SiLU(gate) sums
template <int MT, int NT>
__device__ __forceinline__ void gate_sums(f32x4 (&sums)[NT][MT], const f32x4 (&gate)[NT][MT]) {
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = gate[j][i][e];
        sums[j][i][e] *= g * __builtin_amdgcn_rcpf(1.f + __expf(-g));
      }
}

// ---- tiles through LDS ------------------------------------------------------------------------------
// C times 16 bytes a lane, global -> LDS, if t < steps: a wave-uniform base and a 32-bit offset per lane; lane l lands at
// lds_dst + 16 l, each copy STRIDE bytes after the one before.  The branch is inside so that the compiler sees none in the
// middle of a step, where it would move registers about.
template <int STRIDE>
__device__ __forceinline__ void copies(const char* sbase, const unsigned (&v)[4], unsigned lds_dst, int t, int steps) {
  asm volatile(
      "s_cmp_ge_i32 %6, %7\n\ts_cbranch_scc1 .Lskip%=\n\t"
      "s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %0\n"
      ".Lskip%=:" ::"s"(sbase), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(lds_dst), "s"(t), "s"(steps), "n"(STRIDE)
      : "memory", "m0", "scc");
}
template <int STRIDE>
__device__ __forceinline__ void copies(const char* sbase, const unsigned (&v)[2], unsigned lds_dst, int t, int steps) {
  asm volatile(
      "s_cmp_ge_i32 %4, %5\n\ts_cbranch_scc1 .Lskip%=\n\t"
      "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0\n\t"
      "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %0\n"
      ".Lskip%=:" ::"s"(sbase), "v"(v[0]), "v"(v[1]), "s"(lds_dst), "s"(t), "s"(steps), "n"(STRIDE) : "memory", "m0", "scc");
}

// Waits until at most N of this wave's copies are on their way, or none unless t < steps.
template <int N>
__device__ __forceinline__ void wait_copies(int t, int steps) {
  asm volatile("s_cmp_lt_i32 %0, %1\n\ts_cbranch_scc1 .Lsome%=\n\ts_waitcnt vmcnt(0)\n.Lsome%=:\n\ts_waitcnt vmcnt(%2)"
               ::"s"(t), "s"(steps), "n"(N) : "memory", "scc");
}

// WM x WN waves, each with 16 MT rows x 16 NT columns.  A step is one block of the contraction: the tile's rows of A and of W,
// 128 bytes each, lie in LDS row by row, the eight 16-byte pieces of row r in the order piece ^ (r % 8), which spreads the
// reads of sixteen rows over the banks.  A wave reads its rows of W into registers first, then its rows of A tile by tile.
//
// The two halves of the workgroup (the upper rows of the tile and the lower) run half a step apart, with a barrier every half
// step, so that of the two waves of a SIMD (eight waves) one is in the middle of its products while the other one waits
// for its first reads.  Half h starts step t in phase 2 t + h.  It then copies its rows of A of step t + 1 (two buffers: it
// has read those of step t - 1 itself) and its share of the rows of W of step t + 2 (three buffers: the second half read those
// of step t - 1 in phase 2 t - 1).  Before a step it waits for its A, in the middle of one for its share of the next W,
// which the first half reads in the next phase.
//
// That is what the order needs; what is waited for is more.  The scales of step t + 1 are loads into registers, for which the
// compiler waits at the end of step t with vmcnt(0), since it does not count the copies issued after them: A of step t + 1 and W of
// step t + 2 have landed by then too, so a copy of W has one step to do so, not one and a half.  Where the matrix ends inside a
// lane's MT rows those loads are single ones, waited for before the step's copies are issued (1777 and 1776 rows x 2687 x 7301:
// 40.9 and 40.5 us).
//
// 4096 x 8192 x 16384 (rows, contraction, columns) takes 416-450 us by the card (2.4-2.6 PFLOP/s), the same on zeros 336-364; in
// step, without the half step between them, 486 us.  Its matrix units work in 0.68 of a busy CU's clocks: what bounds it are the
// waits of a step and the clock that power leaves.  4096 x 4096 x 4096, one tile a CU, takes 60 us = 2.29 PFLOP/s: a tile's first
// copies and its result, 5 us, stand alone there.
// PARTS: the workgroup sums a range of the contraction, where tiles are fewer than CUs and the contraction is long.
// GATED: the sums of the contraction's first half wait in registers while the second half is summed, then SiLU(first) second is
// the result: 4096 x (512 + 512) x 14336 into 8 bits 97-107 us, where two products into bf16 and the gated quantiser take 153 (in a
// graph; 117 MB each that are not written and read), 128 rows 9.9 and 16.4, one 7.0 and 10.3.  Its contraction is not cut, so a
// narrow result of a long one leaves most CUs without work at few rows: 16 x (4096 + 4096) x 1400 31 us, those three 16.  The 256 x 256 tile has no registers for two sums, the smaller ones of
// k_mm_ring not the 128 columns of a scale.
template <int MT, int NT, int WM, int WN>
struct MmTile {
  static constexpr int TM = 16 * MT * WM, TN = 16 * NT * WN, WAVES = WM * WN, HALF = WAVES / 2;
  static constexpr int CA = TM / 8 / WAVES, CW = TN / 8 / WAVES;      // copies of a wave per step, eight rows each
  static constexpr int A_UNIT = TM * SCALE_BLOCK, W_UNIT = TN * SCALE_BLOCK;      // rows of a step
  static constexpr int W_AT = 2 * A_UNIT, LDS = W_AT + 3 * W_UNIT;
  static_assert(WAVES * MmResult<MT, NT>::BYTES <= LDS, "the result passes through the same memory");
};

template <int MT, int NT, int WM, int WN, bool PARTS, bool GATED>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mm_tile(MmP p) {
  using T = MmTile<MT, NT, WM, WN>;
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / WN, wn = wave % WN, half = wave / T::HALF;
  const int mtiles = (p.M + T::TM - 1) / T::TM, ntiles = (p.N + T::TN - 1) / T::TN;
  const int id = xcd_contiguous_id(blockIdx.x, gridDim.x), z = PARTS ? range_of(id, p) : 0;
  int mt, nt;
  banded_tile(id - z * p.tiles, mtiles, ntiles, p.band, mt, nt);
  // divisions are done by the vector unit; copies take their addresses from scalar registers
  const int m0 = __builtin_amdgcn_readfirstlane(mt) * T::TM, n0 = __builtin_amdgcn_readfirstlane(nt) * T::TN;
  const unsigned lds0 = lds_offset_of(lds);
  // A block that ends inside comes first, so that only the prologue has to clear what lies behind it.
  const int b0 = PARTS ? z * p.range_blocks : 0, b1 = PARTS ? min(b0 + p.range_blocks, p.KB) : p.KB;
  const int steps = b1 - b0, tail = b1 == p.KB ? p.K % SCALE_BLOCK : 0;
  auto block_of = [&](int t) { return !tail ? b0 + t : t == 0 ? b1 - 1 : b0 + t - 1; };

  // Which row of A is which row of LDS: a lane has row r of each of a wave's MT tiles of 16, and those are MT consecutive rows of
  // the matrix, so that it gets their scales in one load.
  auto arow_of = [&](int x) { return x / (16 * MT) * (16 * MT) + x % 16 * MT + x % (16 * MT) / 16; };
  // copies: lane l brings piece (l % 8) ^ (l / 8) of row l / 8 of eight rows; rows beyond the matrix repeat its last one
  const int cr = lane / 8, cp = (lane % 8) ^ cr;
  const char *abase = p.a + m0 * p.a_ld, *wbase = p.w + n0 * p.w_ld;
  unsigned aoff[T::CA], woff[T::CW];
  const int a8 = half * (T::TM / 16) + wave % T::HALF;       // eight rows of A: a8 + HALF c, of this wave's half; of W: wave + WAVES c
#pragma unroll
  for (int c = 0; c < T::CA; ++c) aoff[c] = (unsigned)min(arow_of(8 * (a8 + T::HALF * c) + cr), p.M - 1 - m0) * (unsigned)p.a_ld + 16 * cp;
#pragma unroll
  for (int c = 0; c < T::CW; ++c) woff[c] = (unsigned)min(8 * (wave + T::WAVES * c) + cr, p.N - 1 - n0) * (unsigned)p.w_ld + 16 * cp;
  auto issue_a = [&](const unsigned (&off)[T::CA], int t, int unit) {
    copies<1024 * T::HALF>(abase + (int64_t)block_of(t) * SCALE_BLOCK, off, lds0 + unit * T::A_UNIT + 1024 * a8, t, steps);
  };
  auto issue_w = [&](const unsigned (&off)[T::CW], int t, int unit) {
    copies<1024 * T::WAVES>(wbase + (int64_t)block_of(t) * SCALE_BLOCK, off, lds0 + T::W_AT + unit * T::W_UNIT + 1024 * wave, t, steps);
  };
  auto clear8 = [&](int at) {      // what this lane brought beyond the end of the contraction
    u32x4* q = (u32x4*)(lds + at + lane * 16);
    u32x4 v = *q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int l = tail - 16 * cp - 4 * i;
      v[i] = l >= 4 ? v[i] : l <= 0 ? 0u : v[i] & (0xffffffffu >> (32 - 8 * l));
    }
    *q = v;
  };

  // this lane's pieces g and 4 + g of row r of a 16-row tile
  const int at0 = r * SCALE_BLOCK + 16 * (g ^ (r % 8)), at1 = r * SCALE_BLOCK + 16 * ((4 + g) ^ (r % 8));
  const int arow = 16 * MT * wm, wrow = 16 * NT * wn;
  auto frag = [&](int at, int row) {
    const char* q = lds + at + row * SCALE_BLOCK;
    return join16(*(const u32x4*)(q + at0), *(const u32x4*)(q + at1));
  };
  // scales of a block: those of this lane's MT rows, as they lie in memory (where the matrix ends among them, one by one), and
  // the wave's weights'
  const unsigned short* sa = (const unsigned short*)p.sa + m0;
  const int srow = arow + MT * r, sleft = p.M - m0;
  const float* sw = p.sw + (int64_t)min((n0 + wrow) / SCALE_BLOCK, (p.N - 1) / SCALE_BLOCK) * p.KB;
  typedef __attribute__((ext_vector_type(MT / 2))) unsigned pairs;
  pairs s_next;
  float sw_next;
  auto load_scales = [&](int t) {
    const unsigned short* q = sa + block_of(t) * p.sa_ld;
    if (srow + MT <= sleft) {
      __builtin_memcpy(&s_next, q + srow, sizeof(s_next));
    } else {
#pragma unroll
      for (int i = 0; i < MT / 2; ++i) s_next[i] = q[min(srow + 2 * i, sleft - 1)] | (unsigned)q[min(srow + 2 * i + 1, sleft - 1)] << 16;
    }
    sw_next = sw[block_of(t)];
  };
  auto scale_next = [&](int i) {
    return __builtin_bit_cast(float, i % 2 ? s_next[i / 2] & 0xffff0000u : s_next[i / 2] << 16) * sw_next;
  };

  // The product of tile q of a step (row q / NT, column q % NT) is scaled and added LAG products later, when it is there; the
  // last ones of a step under the next step's first.
  constexpr int LAG = 3, Q = MT * NT;
  f32x4 acc[NT][MT] = {}, d[LAG + 1] = {}, gate[GATED ? NT : 1][GATED ? MT : 1];
  float s_last = 0.f;     // (a product that is NaN stays NaN times zero: its element is NaN then already)
  auto add = [&](int q, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[q % NT][q / NT][e] += d[q % (LAG + 1)][e] * s;
  };
  load_scales(0);
  if (!tail) {
    issue_w(woff, 0, 0);
    issue_a(aoff, 0, 0);
  } else {
    // how far this lane's piece lies behind the last one that holds codes
    const unsigned back = (unsigned)max(0, 16 * cp - ((tail - 1) & ~15));
    unsigned av[T::CA], wv[T::CW];
#pragma unroll
    for (int c = 0; c < T::CA; ++c) av[c] = aoff[c] - back;
#pragma unroll
    for (int c = 0; c < T::CW; ++c) wv[c] = woff[c] - back;
    issue_w(wv, 0, 0);
    issue_a(av, 0, 0);
    wait_vmcnt<0>();
    for (int c = 0; c < T::CA; ++c) clear8(1024 * (a8 + T::HALF * c));
    for (int c = 0; c < T::CW; ++c) clear8(T::W_AT + 1024 * (wave + T::WAVES * c));
  }
  issue_w(woff, 1, 1);
  if (half == 1) {     // half a step behind
    wait_copies<T::CW>(1, steps);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    lds_barrier();
  }
  int wu = 0;          // unit of the step's rows of W
  // steps t .. end - 1
  auto run = [&](int t, int end) {
    for (; t < end; ++t) {
      const int at_a = t % 2 * T::A_UNIT, at_w = T::W_AT + wu * T::W_UNIT;
      // this wave's copies of the step's A have landed, its LDS accesses are done
      wait_copies<T::CW>(t + 1, steps);
      __builtin_amdgcn_s_waitcnt(0xC07F);
      lds_barrier();
      float s[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) s[i] = scale_next(i);
      if (t + 1 < steps) load_scales(t + 1);
      issue_a(aoff, t + 1, (t + 1) % 2);
      issue_w(woff, t + 2, wu > 0 ? wu - 1 : 2);
      i32x8 fw[NT], fa[2];
      fa[0] = frag(at_a, arow);
#pragma unroll
      for (int j = 0; j < NT; ++j) fw[j] = frag(at_w, wrow + 16 * j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if (i == MT / 2) {
          wait_copies<T::CA + T::CW>(t + 2, steps);
          lds_barrier();
        }
        if (i + 1 < MT) fa[(i + 1) % 2] = frag(at_a, arow + 16 * (i + 1));
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          __builtin_amdgcn_sched_barrier(0);
          const int q = i * NT + j;
          d[q % (LAG + 1)] = mfma_f8(fw[j], fa[i % 2], f32x4{0.f, 0.f, 0.f, 0.f});
          __builtin_amdgcn_sched_barrier(0);
          if (q < LAG) add(Q + q - LAG, s_last);
          else add(q - LAG, s[(q - LAG) / NT]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      s_last = s[MT - 1];
      wu = wu < 2 ? wu + 1 : 0;
    }
  };
  auto flush = [&] {
#pragma unroll
    for (int q = Q - LAG; q < Q; ++q) add(q, s_last);
  };
  if constexpr (GATED) {
    for (int part = 0; part < 2; ++part) {
      run(part * (steps / 2), (part + 1) * (steps / 2));
      flush();
      if (part) break;
      s_last = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) gate[j][i] = acc[j][i], acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  } else {
    run(0, steps);
    flush();
  }
  if (half == 0) lds_barrier();    // as many as the other half
  lds_barrier();      // everyone has read the last step
  if constexpr (GATED) gate_sums<MT, NT>(acc, gate);
  mm_result<MT, NT, PARTS>(p, acc, z, m0 + arow, n0 + wrow, wave, lds);
}

// ---- small tiles, three steps in LDS ------------------------------------------------------------------
// Once 16 bytes a lane, global -> LDS, as above; copy_word: 4 bytes (2: BYTES = 2, into the low half of 4), lane l at lds_dst + 4 l.
__device__ __forceinline__ void copy1(const char* sbase, unsigned v, unsigned lds_dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" ::"s"(sbase), "v"(v), "s"(lds_dst) : "memory", "m0");
}
template <int BYTES>
__device__ __forceinline__ void copy_word(const char* sbase, unsigned v, unsigned lds_dst) {
  if (BYTES == 4)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, %0" ::"s"(sbase), "v"(v), "s"(lds_dst) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %0" ::"s"(sbase), "v"(v), "s"(lds_dst) : "memory", "m0");
}
// Four waves, 2 x 2, each with 16 MT rows x 16 NT columns, for results of few tiles, where a CU has one to three workgroups and what
// counts is a step's chain: wait, barrier, LDS, products.  So a step's operands go from LDS to registers while the step before
// is multiplied, the copies of two more are on their way (three to seven made no difference), addresses are advanced and not
// computed, and the scales come by copies as well (4 bytes for each row of A, the weights' scale 64 times), since a wait for a
// load into a register would wait for the copies issued before it.  Rows x contraction x columns in a graph: 32 x 4096 x 14336
// 11.3 us (6.7 TB/s of weights without the 2.5 us of a launch), 128 x 2048 x 8192 8.5 us, 256 x 4096 x 4096 13.0 us.
constexpr int STAGES = 3;
template <int MT, int NT>
struct MmRing {
  static constexpr int TM = 32 * MT, TN = 32 * NT;
  static constexpr int W_AT = TM * SCALE_BLOCK, SA_AT = W_AT + TN * SCALE_BLOCK, SW_AT = SA_AT + 256, STAGE = SW_AT + 256;
  static constexpr int CA = TM / 32, CW = TN / 32, COPIES = CA + CW + 1;     // of a wave per step
  static constexpr int LDS = STAGES * STAGE;
  static_assert(4 * MmResult<MT, NT>::BYTES <= LDS && TM <= 64 && TN <= SCALE_BLOCK, "one load of scales");
};

template <int MT, int NT, bool GATED>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mm_ring(MmP p) {
  using T = MmRing<MT, NT>;
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
  // The tiles that share a strip of the larger operand run side by side on an XCD, whose L2 then serves it to all but the first.
  const int id = xcd_contiguous_id(blockIdx.x, gridDim.x), z = range_of(id, p), in_z = id - z * p.tiles;
  const int strip = __builtin_amdgcn_readfirstlane(in_z / p.band), at = in_z - strip * p.band;
  const int m0 = (p.M > p.N ? strip : at) * T::TM, n0 = (p.M > p.N ? at : strip) * T::TN;
  const int b0 = z * p.range_blocks, b1 = min(b0 + p.range_blocks, p.KB);
  const unsigned lds0 = lds_offset_of(lds);
  const int steps = b1 - b0, tail = b1 == p.KB ? p.K % SCALE_BLOCK : 0;
  auto arow_of = [&](int x) { return x / (16 * MT) * (16 * MT) + x % 16 * MT + x % (16 * MT) / 16; };
  const int cr = lane / 8, cp = (lane % 8) ^ cr;
  // what the next copies read
  const int first = tail ? b1 - 1 : b0;
  const char* anext = p.a + m0 * p.a_ld + (int64_t)first * SCALE_BLOCK;
  const char* wnext = p.w + n0 * p.w_ld + (int64_t)first * SCALE_BLOCK;
  const char* snext = wn == 0 ? (const char*)(p.sa + first * p.sa_ld + m0) : (const char*)(p.sw + (int64_t)(n0 / SCALE_BLOCK) * p.KB + first);
  const int64_t s_step = wn == 0 ? 2 * p.sa_ld : 4;
  unsigned aoff[T::CA], woff[T::CW];
#pragma unroll
  for (int c = 0; c < T::CA; ++c) aoff[c] = (unsigned)min(arow_of(8 * (wave + 4 * c) + cr), p.M - 1 - m0) * (unsigned)p.a_ld + 16 * cp;
#pragma unroll
  for (int c = 0; c < T::CW; ++c) woff[c] = (unsigned)min(8 * (wave + 4 * c) + cr, p.N - 1 - n0) * (unsigned)p.w_ld + 16 * cp;
  const unsigned soff = 2 * min(lane, p.M - 1 - m0);
  auto issue = [&](int stage, unsigned back) {
    const unsigned at = lds0 + stage * T::STAGE;
#pragma unroll
    for (int c = 0; c < T::CA; ++c) copy1(anext, aoff[c] - back, at + 1024 * (wave + 4 * c));
#pragma unroll
    for (int c = 0; c < T::CW; ++c) copy1(wnext, woff[c] - back, at + T::W_AT + 1024 * (wave + 4 * c));
    if (wn == 0) copy_word<2>(snext, soff, at + T::SA_AT);
    else copy_word<4>(snext, 0, at + T::SW_AT);
    anext += SCALE_BLOCK;
    wnext += SCALE_BLOCK;
    snext += s_step;
  };
  issue(0, tail ? (unsigned)max(0, 16 * cp - ((tail - 1) & ~15)) : 0u);
  if (tail) {
    anext += (b0 - b1) * SCALE_BLOCK;      // back to the first block
    wnext += (b0 - b1) * SCALE_BLOCK;
    snext += (b0 - b1) * s_step;
    wait_vmcnt<0>();
    for (int c = 0; c < T::CA + T::CW; ++c) {       // clear what this lane brought beyond the end of the contraction
      u32x4* q = (u32x4*)(lds + 1024 * (wave + 4 * c) + lane * 16);
      u32x4 v = *q;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int l = tail - 16 * cp - 4 * i;
        v[i] = l >= 4 ? v[i] : l <= 0 ? 0u : v[i] & (0xffffffffu >> (32 - 8 * l));
      }
      *q = v;
    }
  }
#pragma unroll
  for (int t = 1; t < STAGES; ++t)
    if (t < steps) issue(t, 0);

  const int at0 = r * SCALE_BLOCK + 16 * (g ^ (r % 8)), at1 = r * SCALE_BLOCK + 16 * ((4 + g) ^ (r % 8));
  const int arow = 16 * MT * wm, wrow = 16 * NT * wn;
  auto frag = [&](int at) { return join16(*(const u32x4*)(lds + at + at0), *(const u32x4*)(lds + at + at1)); };
  // A step's operands are read from LDS while the step before is multiplied; its place in LDS is then free.
  struct Step {
    i32x8 w[NT], a[MT];
    unsigned sa[MT];
    float sw;
  };
  auto read = [&](Step& x, int stage) {
    const int at = stage * T::STAGE;
#pragma unroll
    for (int i = 0; i < MT; ++i) x.a[i] = frag(at + (arow + 16 * i) * SCALE_BLOCK);
#pragma unroll
    for (int j = 0; j < NT; ++j) x.w[j] = frag(at + T::W_AT + (wrow + 16 * j) * SCALE_BLOCK);
#pragma unroll
    for (int i = 0; i < MT; ++i) x.sa[i] = *(const unsigned*)(lds + at + T::SA_AT + 4 * (arow + MT * r + i));
    x.sw = *(const float*)(lds + at + T::SW_AT + 4 * lane);
  };
  f32x4 acc[NT][MT] = {};
  int stage = 0;                      // of step t
  auto step = [&](int t, const Step& now, Step& next) {
    wait_copies<T::COPIES>(t + 2, steps);      // those of step t + 1 have landed
    __builtin_amdgcn_s_waitcnt(0xC07F);
    lds_barrier();
    if (t + STAGES < steps) issue(stage, 0);
    stage = stage + 1 < STAGES ? stage + 1 : 0;
    read(next, stage);                // past the last step: not used
    __builtin_amdgcn_sched_barrier(0);
    f32x4 d[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) d[j][i] = mfma_f8(now.w[j], now.a[i], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const float s = __builtin_bit_cast(float, now.sa[i] << 16) * now.sw;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][i][e] += d[j][i][e] * s;
      }
    __builtin_amdgcn_sched_barrier(0);
  };
  Step even, odd;
  wait_copies<2 * T::COPIES>(2, steps);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  lds_barrier();
  read(even, 0);
  f32x4 gate[GATED ? NT : 1][GATED ? MT : 1];
  auto turn = [&](int done) {
    if constexpr (GATED) {
      if (done != steps / 2) return;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) gate[j][i] = acc[j][i], acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  for (int t = 0; t < steps; t += 2) {
    step(t, even, odd);
    turn(t + 1);
    if (t + 1 < steps) step(t + 1, odd, even);
    turn(t + 2);
  }
  if constexpr (GATED) gate_sums<MT, NT>(acc, gate);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  lds_barrier();      // everyone has read the last step
  mm_result<MT, NT, true>(p, acc, z, m0 + arow, n0 + wrow, wave, lds);
}

// Adds the ranges' partial sums in their order and rounds: 16 lanes hold 128 columns of a row, a workgroup 16 rows of them.
template <int JOIN, RowEnd END>      // JOIN: ranges whose loads are issued together
__global__ __launch_bounds__(256) void k_mm_join(MmP p) {
  const int lane = threadIdx.x % 16, nb = (p.N + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const int m = (int)(blockIdx.x / nb) * 16 + threadIdx.x / 16, b = (int)(blockIdx.x % nb);
  if (m >= p.M) return;
  const Cols<END> k(b * SCALE_BLOCK + 8 * lane, p.N);
  float v[8] = {};
  for (int z = 0; z < p.ranges; z += JOIN) {
    Raw8<float> x[JOIN];
#pragma unroll
    for (int i = 0; i < JOIN; ++i) x[i] = z + i < p.ranges ? load8(p.part + ((int64_t)(z + i) * p.M + m) * p.N, k) : Raw8<float>{};
#pragma unroll
    for (int i = 0; i < JOIN; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[i].get(e);
  }
  if (p.out_type == SVDMLP_F8) {
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = k.own(e) ? fmaxf(amax, fabsf(v[e])) : amax;
    const __bf16 s = scale_of(max16(amax));
    if (k.any()) store_codes8((unsigned char*)p.c + m * p.c_ld, k, v, 1.f / (float)s);
    if (lane == 0) p.c_scales[b * p.c_scales_ld + m] = s;
  } else if (k.any()) {
    store8((__bf16*)p.c + m * p.c_ld, k, v);
  }
}

// ---- host -------------------------------------------------------------------------------------------
// Which kernel, and into how many ranges the contraction is cut: the least time by a model of the compute units.  A
// workgroup's steps take `step` us where it has a CU to itself (its own chain of waits), `pair` where it shares it with another,
// `share` each where more do (the CU's copies and matrix products; below one a CU, the chip's share of them), a tile besides
// `tile` us for its first copies and its result, a launch LAUNCH_US; cut contractions and 8-bit results of 64-column tiles add
// a second launch that reads the partial sums.  The figures are fitted to 8700 random sizes of 1 - 8192 rows, 100 - 16384 columns
// and contractions, every kernel with the model's ranges and the next to them, in a graph; over 9400 others the times of the chosen
// over those of the fastest were 1.006 in the geometric mean, 1.27 at most.  Model / measured us of the chosen and of others, rows x
// contraction x columns:
//   16 x 4096 x 14336   ring 32x64 10.9 / 11.3, few 16.5 / 17.9         256 x 4096 x 4096   ring 32x64 12.4 / 13.0, ring 64x64 13.7 / 14.1
//   1024 x 4096 x 4096  ring 64x128 22.9 / 26.0, tile 128x256 in 2 ranges 37.8 / 32.3
//   2048 x 4096 x 4096  tile 128x256 38.4 / 37.0, tile 256x256 53.7 / 47.4
//   4096 x 4096 x 4096  tile 256x256 59.1 / 60.0, tile 128x256 69.8 / 72.9
//   4096 x 8192 x 16384 tile 256x256 434 / 446, tile 128x256 540 / 560
//   286 x 13184 x 7424  tile 256x256 in 4 ranges 62 / 58, in one 148 / 143
//   4096 x 14336 x 512  ring 64x64 45 / 50, tile 128x256 in 4 ranges 50 / 44, in one 105 / 93 (the model misses the fastest here)
// Gated, into 8 bits: 1 x 1024 x 14336  ring 32x128 7.3 / 7.4, ring 64x128 9.4 / 9.6;  512 x 1024 x 14336  tile 128x256 15.5 / 16.4, ring
// 64x128 26 / 22;  4096 x 1024 x 14336  tile 128x256 93 / 96, ring 64x128 167 / 129.
// (Further tiles measured and not kept: 128 x 128 with four waves, 256 x 128, 128 x 64: level or behind one of these.)
enum { MM_FEW = 0, MM_RING_32, MM_RING_64, MM_RING_64_128, MM_TILE_128_256, MM_TILE_256, MM_RING_32_128, MM_KINDS };
struct MmKind {
  const char* name;
  int rows, cols, max_rows;      // of a tile; rows of A that it takes (0: any)
  double step, pair, share, tile;
};
constexpr MmKind MM_KIND[MM_KINDS] = {
    {"k_mm_few[tile=16x16", 16, 16, 16, 0.57 / FEW_WAVES, 1.09 / FEW_WAVES, 0.545 / FEW_WAVES, 0.},
    {"k_mm_ring[tile=32x64", 32, 64, 0, 0.24, 0.28, 0.174, 0.46},
    {"k_mm_ring[tile=64x64", 64, 64, 0, 0.33, 0.366, 0.268, 0.65},
    {"k_mm_ring[tile=64x128", 64, 128, 0, 0.485, 0.577, 0.393, 0.98},
    {"k_mm_tile[tile=128x256", 128, 256, 0, 1.02, 1.9, 1.0, 3.25},
    {"k_mm_tile[tile=256x256", 256, 256, 0, 1.43, 3.1, 1.6, 5.4},
    {"k_mm_ring[tile=32x128", 32, 128, 0, 0.45, 0.57, 0.255, 0.8},     // gated only: level with the others or behind them elsewhere
};
constexpr double LAUNCH_US = 2.5, JOIN_US = 2.6, JOIN_RANGE_US = 0.1, HBM_BYTES_PER_US = 7.05e6, PART_BYTES_PER_US = 5.2e6;
constexpr int MM_CUS = 256;      // the model's device, so that a result's order of sums goes by the extents alone

struct MmPlan {
  int kind, ranges, range_blocks;
  bool join;                  // partial sums that k_mm_join adds and rounds
  int64_t tiles;
  double est_us;
};

static int plan_mm(int64_t M, int64_t N, int64_t K, int out_type, int gated, MmPlan* best) {
  if (M < 0 || N <= 0 || K <= 0) return SVDMLP_INVALID_ARGUMENT;
  if (out_type != SVDMLP_F8 && out_type != SVDMLP_BF16) return SVDMLP_INVALID_ARGUMENT;
  if (gated != 0 && (gated != 1 || K % (2 * SCALE_BLOCK))) return SVDMLP_INVALID_ARGUMENT;
  if (M >= int64_t(1) << 24 || N > int64_t(1) << 22 || K > int64_t(1) << 22) return SVDMLP_UNSUPPORTED;
  const int KB = (int)scale_blocks(K);
  best->kind = -1;
  for (int k = 0; k < MM_KINDS; ++k) {
    const MmKind& kind = MM_KIND[k];
    if (kind.max_rows && M > kind.max_rows) continue;
    if (k == MM_RING_32_128 ? !gated : gated && k != MM_RING_64_128 && k != MM_TILE_128_256) continue;      // 128 columns in a workgroup, registers for two sums
    const int64_t tiles = ((M + kind.rows - 1) / kind.rows) * ((N + kind.cols - 1) / kind.cols);
    const bool large = k == MM_TILE_128_256 || k == MM_TILE_256;
    for (int r = 1; r <= (gated ? 1 : large ? 8 : 32) && r <= KB; r += !large ? r : r < 4 ? 1 : 2) {
      MmPlan q;
      q.kind = k;
      q.tiles = tiles;
      q.range_blocks = (KB + r - 1) / r;
      q.ranges = (KB + q.range_blocks - 1) / q.range_blocks;
      if (q.ranges != r && r > 1) continue;
      if (tiles * r >= int64_t(1) << 22) continue;        // a grid of 512 lanes each, below 2^31
      q.join = r > 1 || (out_type == SVDMLP_F8 && kind.cols < SCALE_BLOCK);
      const int64_t per_cu = (tiles * r + MM_CUS - 1) / MM_CUS;
      const bool on_lines = k == MM_FEW || (K + 15) / 16 % 8 == 0;     // packed rows begin on lines; else 128 bytes take two
      double step = per_cu < 2 ? kind.share * tiles * r / MM_CUS : per_cu == 2 && on_lines ? kind.pair : kind.share * per_cu;
      if (step < kind.step) step = kind.step;
      int steps = q.range_blocks;
      double hbm = ((double)N * K + (double)M * K + (double)M * N * (out_type == SVDMLP_F8 ? 1 : 2)) / HBM_BYTES_PER_US;
      if (k == MM_FEW) {          // eight waves take a block each; every workgroup reads the rows of A
        steps = (steps + FEW_WAVES - 1) / FEW_WAVES * FEW_WAVES;
        step += 0.0205 / FEW_WAVES * M * per_cu;
      }
      if (gated && k == MM_RING_64_128) step *= 1.4;     // registers for two sums: fewer waves
      if (!on_lines) {
        step *= k == MM_TILE_256 ? 1.07 : 1.28;
        hbm *= 1.84;
      }
      double t = kind.tile * (gated ? 1.5 : 1.) * per_cu + steps * step;      // SiLU of the tile
      if (t < hbm) t = hbm;
      q.est_us = LAUNCH_US + t + (q.join ? JOIN_US + JOIN_RANGE_US * r + 8. * M * N * r / PART_BYTES_PER_US : 0.);
      if (best->kind < 0 || q.est_us < best->est_us) *best = q;
    }
  }
  return best->kind < 0 ? SVDMLP_UNSUPPORTED : SVDMLP_OK;
}

static size_t part_bytes(const MmPlan& q, int64_t M, int64_t N) { return q.join ? (size_t)q.ranges * M * N * 4 : 0; }

template <RowEnd END>
static hipError_t launch_join(const MmP& p, hipStream_t st) {
  const unsigned wgs = (unsigned)((p.M + 15) / 16 * scale_blocks(p.N));
  if (p.ranges == 1) return launch(k_mm_join<1, END>, wgs, 256, p, st);
  if (p.ranges <= 4) return launch(k_mm_join<4, END>, wgs, 256, p, st);
  if (p.ranges <= 8) return launch(k_mm_join<8, END>, wgs, 256, p, st);
  return launch(k_mm_join<16, END>, wgs, 256, p, st);
}
static hipError_t launch_join(const MmP& p, hipStream_t st) {
  switch (row_end(p.N)) {
    case WHOLE: return launch_join<WHOLE>(p, st);
    case OVERLAP: return launch_join<OVERLAP>(p, st);
    default: return launch(k_mm_join<4, SHORT>, (unsigned)((p.M + 15) / 16), 256, p, st);
  }
}

template <int MT>
static hipError_t launch_tile(const MmP& p, unsigned wgs, hipStream_t st) {
  if (p.part) return launch(k_mm_tile<MT, 4, 2, 4, true, false>, wgs, 512, p, st);
  return launch(k_mm_tile<MT, 4, 2, 4, false, false>, wgs, 512, p, st);
}
static hipError_t launch_mm(MmP& p, const MmPlan& q, bool gated, hipStream_t st) {
  const unsigned wgs = (unsigned)(q.tiles * q.ranges);
  const MmKind& kind = MM_KIND[q.kind];
  const int mtiles = (p.M + kind.rows - 1) / kind.rows, ntiles = (p.N + kind.cols - 1) / kind.cols;
  p.tiles = (int)q.tiles;
  p.band = q.kind == MM_TILE_128_256 || q.kind == MM_TILE_256 ? band_height(mtiles, wgs) : p.M > p.N ? ntiles : mtiles;
  switch (q.kind) {
    case MM_FEW: return launch(k_mm_few, wgs, 64 * FEW_WAVES, p, st);
    case MM_RING_32: return launch(k_mm_ring<1, 2, false>, wgs, 256, p, st);
    case MM_RING_64: return launch(k_mm_ring<2, 2, false>, wgs, 256, p, st);
    case MM_RING_64_128:
      if (gated) return launch(k_mm_ring<2, 4, true>, wgs, 256, p, st);
      return launch(k_mm_ring<2, 4, false>, wgs, 256, p, st);
    case MM_TILE_128_256:
      if (gated) return launch(k_mm_tile<4, 4, 2, 4, false, true>, wgs, 512, p, st);
      return launch_tile<4>(p, wgs, st);
    case MM_RING_32_128: return launch(k_mm_ring<1, 4, true>, wgs, 256, p, st);
    default: return launch_tile<8>(p, wgs, st);
  }
}

}  // namespace svdmlp

using namespace svdmlp;

extern "C" {

size_t svdmlp_scaled_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t out_type) {
  MmPlan q;
  return plan_mm(M, N, K, out_type, 0, &q) == SVDMLP_OK ? part_bytes(q, M, N) : 0;
}

int svdmlp_scaled_matmul_describe(int64_t M, int64_t N, int64_t K, int32_t out_type, int32_t gated, char* buf, size_t buf_bytes) {
  if (!buf || buf_bytes == 0) return SVDMLP_INVALID_ARGUMENT;
  buf[0] = 0;
  MmPlan q;
  if (const int st = plan_mm(M, N, K, out_type, gated, &q)) return st;
  const int n = std::snprintf(buf, buf_bytes, "%s tiles=%lld ranges=%d est_us=%.1f]%s", MM_KIND[q.kind].name, (long long)q.tiles, q.ranges,
                              q.est_us, q.join ? " k_mm_join" : "");
  return n > 0 && (size_t)n < buf_bytes ? SVDMLP_OK : SVDMLP_INVALID_ARGUMENT;
}

int svdmlp_scaled_matmul(const svdmlp_scaled_matmul_args* a, void* hip_stream) {
  if (!a) return SVDMLP_INVALID_ARGUMENT;
  MmPlan q;
  if (const int st = plan_mm(a->M, a->N, a->K, a->out_type, a->gated, &q)) return st;
  if (const int st = check_codes(a->a, a->a_ld, a->K)) return st;
  if (const int st = check_codes(a->w, a->w_ld, a->K)) return st;
  if (!a->a_scales || !a->w_scales || !aligned_to(a->a_scales, 2) || !aligned_to(a->w_scales, 4) || a->a_scales_ld < a->M)
    return SVDMLP_INVALID_ARGUMENT;
  if (a->out_type == SVDMLP_F8) {
    if (const int st = check_codes(a->c, a->c_ld, a->N)) return st;
    if (!a->c_scales || !aligned_to(a->c_scales, 2) || a->c_scales_ld < a->M) return SVDMLP_INVALID_ARGUMENT;
  } else if (!a->c || a->c_ld < a->N || !aligned_to(a->c, 2)) {
    return SVDMLP_INVALID_ARGUMENT;
  }
  if (a->c == a->a || a->c == a->w) return SVDMLP_INVALID_ARGUMENT;
  if (a->M == 0) return SVDMLP_OK;
  if (q.join) {
    if (a->workspace_bytes < part_bytes(q, a->M, a->N)) return SVDMLP_WORKSPACE_TOO_SMALL;
    if (!a->workspace || !aligned_to(a->workspace, 16)) return SVDMLP_INVALID_ARGUMENT;
  }
  const bool f8 = a->out_type == SVDMLP_F8;
  if (outputs_overlap({rows_of(a->c, a->M, a->N, a->c_ld, f8 ? 1 : 2), activation_scales(f8 ? a->c_scales : nullptr, a->M, a->N, a->c_scales_ld),
                       rows_of(q.join ? a->workspace : nullptr, 1, (int64_t)part_bytes(q, a->M, a->N), 0, 1)},
                      {rows_of(a->a, a->M, a->K, a->a_ld, 1), activation_scales(a->a_scales, a->M, a->K, a->a_scales_ld),
                       rows_of(a->w, a->N, a->K, a->w_ld, 1), weight_scales(a->w_scales, a->N, a->K)}))
    return SVDMLP_INVALID_ARGUMENT;
  MmP p;
  p.a = (const char*)a->a; p.w = (const char*)a->w; p.sa = (const __bf16*)a->a_scales; p.sw = a->w_scales;
  p.c = a->c; p.c_scales = (__bf16*)a->c_scales; p.part = q.join ? (float*)a->workspace : nullptr;
  p.a_ld = a->a_ld; p.w_ld = a->w_ld; p.sa_ld = a->a_scales_ld; p.c_ld = a->c_ld; p.c_scales_ld = a->c_scales_ld;
  p.M = (int)a->M; p.N = (int)a->N; p.K = (int)a->K; p.KB = (int)scale_blocks(a->K);
  p.out_type = a->out_type;
  p.ranges = q.ranges; p.range_blocks = q.range_blocks;
  hipStream_t st = (hipStream_t)hip_stream;
  hipError_t e = launch_mm(p, q, a->gated != 0, st);
  if (e == hipSuccess && q.join) e = launch_join(p, st);
  return status_of(e);
}

}  // extern "C"
