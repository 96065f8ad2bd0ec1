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
  int band;                   // row tiles of a band of banded_tile
  int ranges, range_blocks;   // ranges of the contraction, blocks of 128 in each (the last may be shorter)
};

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

__device__ __forceinline__ void store4(const MmP& p, int m, int n, const f32x4& v) {
  if (m >= p.M || n >= p.N) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= p.N) return;
    ((__bf16*)p.c)[m * p.c_ld + n + e] = (__bf16)v[e];
  }
}

// Few rows, up to 16 MT: the weights go from HBM straight into registers, once.  A workgroup has 16 NT columns and a range
// of the contraction, whose blocks go to its waves in turn; the waves' sums meet in LDS.
template <int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_mm_few(MmP p) {
  __shared__ f32x4 red[WAVES][MT * NT][64];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int ntiles = (p.N + 16 * NT - 1) / (16 * NT), z = blockIdx.x / ntiles;
  const int n0 = (blockIdx.x - z * ntiles) * 16 * NT;
  const char *wr[NT], *ar[MT];
  const __bf16* sa[MT];
#pragma unroll
  for (int j = 0; j < NT; ++j) wr[j] = p.w + (int64_t)min(n0 + 16 * j + r, p.N - 1) * p.w_ld;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(16 * i + r, p.M - 1);
    ar[i] = p.a + m * p.a_ld;
    sa[i] = p.sa + m;
  }
  const float* sw = p.sw + (int64_t)(n0 / SCALE_BLOCK) * p.KB;
  f32x4 acc[NT][MT] = {};
  // U blocks of this wave from b on, all loads before the first product
  auto blocks = [&](auto full, auto u, int b) {
    constexpr bool FULL = decltype(full)::value;
    constexpr int U = decltype(u)::value;
    i32x8 fw[U][NT], fa[U][MT];
    float s[U][MT];
#pragma unroll
    for (int x = 0; x < U; ++x) {
#pragma unroll
      for (int j = 0; j < NT; ++j) fw[x][j] = block_codes<FULL>(wr[j], b + x * WAVES, g, p.K);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        fa[x][i] = block_codes<FULL>(ar[i], b + x * WAVES, g, p.K);
        s[x][i] = (float)sa[i][(b + x * WAVES) * p.sa_ld] * sw[b + x * WAVES];
      }
    }
#pragma unroll
    for (int x = 0; x < U; ++x)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const f32x4 d = mfma_f8(fw[x][j], fa[x][i], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][i][e] += d[e] * s[x][i];
        }
  };
  constexpr std::true_type whole_block{};
  constexpr std::integral_constant<int, 1> one{};
  constexpr std::integral_constant<int, 2> two{};
  constexpr std::integral_constant<int, (MT + NT <= 3 ? 4 : 2)> most{};
  const int b0 = z * p.range_blocks, b1 = min(b0 + p.range_blocks, p.KB);
  const int whole = min(b1, p.K / SCALE_BLOCK);
  int b = b0 + wave;
  for (; b + (most - 1) * WAVES < whole; b += most * WAVES) blocks(whole_block, most, b);
  if (most > 2 && b + WAVES < whole) {
    blocks(whole_block, two, b);
    b += 2 * WAVES;
  }
  if (b < whole) blocks(whole_block, one, b);
  if (whole < b1 && (whole - b0) % WAVES == wave) blocks(std::false_type{}, one, whole);
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) red[wave][j * MT + i][lane] = acc[j][i];
  __syncthreads();
  for (int x = threadIdx.x; x < MT * NT * 64; x += 64 * WAVES) {
    f32x4 v = red[0][x / 64][x % 64];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += red[w][x / 64][x % 64];
    const int j = x / 64 / MT, i = x / 64 % MT, m = 16 * i + x % 16, n = n0 + 16 * j + 4 * (x % 64 / 16);
    if (!p.part) {
      store4(p, m, n, v);
    } else if (m < p.M) {
      float* q = p.part + ((int64_t)z * p.M + m) * p.N + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < p.N) q[e] = v[e];
    }
  }
}

// ---- tiles through LDS ------------------------------------------------------------------------------
// Four times 16 bytes a lane, global -> LDS, if t < steps: a wave-uniform base and a 32-bit offset per lane; lane l lands at
// lds_dst + 16 l, each copy STRIDE bytes after the one before.  The branch is inside so that the compiler sees none in the
// middle of a step, where it would move registers about.
template <int STRIDE>
__device__ __forceinline__ void copy4(const char* sbase, const unsigned (&v)[4], unsigned lds_dst, int t, int steps) {
  asm volatile(
      "s_cmp_ge_i32 %6, %7\n\ts_cbranch_scc1 .Lskip%=\n\t"
      "s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %0\n\t"
      "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %0\n"
      ".Lskip%=:" ::"s"(sbase), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(lds_dst), "s"(t), "s"(steps), "n"(STRIDE)
      : "memory", "m0", "scc");
}

// Waits until at most N of this wave's copies are on their way, or none unless t < steps.
template <int N>
__device__ __forceinline__ void wait_copies(int t, int steps) {
  asm volatile("s_cmp_lt_i32 %0, %1\n\ts_cbranch_scc1 .Lsome%=\n\ts_waitcnt vmcnt(0)\n.Lsome%=:\n\ts_waitcnt vmcnt(%2)"
               ::"s"(t), "s"(steps), "n"(N) : "memory", "scc");
}

// 2 x WN waves, each with 16 MT rows x 16 NT columns.  A step is one block of the contraction: the tile's rows of W and of A,
// 128 bytes each, lie in LDS row by row, the eight 16-byte pieces of row r in the order piece ^ (r % 8), which spreads the
// reads of sixteen rows over the banks.  A wave reads its rows of W into registers first, then its rows of A tile by tile.
//
// The two halves of the workgroup (rows 0 .. ROWS / 2 - 1 and the others) run half a step apart, with a barrier every half
// step, so that of the two waves of a SIMD (256 x 256 tile) one is in the middle of its products while the other one waits
// for its first reads.  Half h starts step t in phase 2 t + h.  It then copies its rows of A of step t + 1 (two buffers: it
// has read those of step t - 1 itself) and its share of the rows of W of step t + 2 (three buffers: the second half read those
// of step t - 1 in phase 2 t - 1).  Before a step it waits for its A, in the middle of one for its share of the next W,
// which the first half reads in the next phase.
template <int MT, int NT, int WM, int WN>
struct MmTile {
  static constexpr int ROWS = 16 * MT * WM, WAVES = WM * WN;     // of the tile, and columns
  static_assert(WM == 2 && 16 * NT * WN == ROWS && ROWS == 32 * WAVES, "units of equal size, four copies a wave");
  static constexpr int UNIT = ROWS * SCALE_BLOCK;                // rows of A or W of a step
  static constexpr int W_AT = 2 * UNIT;                          // two units for A, then three for W
  static constexpr int OUT_ROWS = 64, OUT_LD = 32 * NT + 16;     // a wave's piece of the result in LDS, bytes per row
  static constexpr int OUT = WAVES * OUT_ROWS * OUT_LD, LDS = 5 * UNIT;
  static_assert(OUT + 4 * WN * ROWS <= LDS, "the result passes through the same memory");
};

template <int MT, int NT, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mm_tile(MmP p) {
  using T = MmTile<MT, NT, WM, WN>;
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / WN, wn = wave % WN;
  const int mtiles = (p.M + T::ROWS - 1) / T::ROWS, ntiles = (p.N + T::ROWS - 1) / T::ROWS, tiles = mtiles * ntiles;
  int mt, nt;
  const int id = xcd_contiguous_id(blockIdx.x, gridDim.x), z = __builtin_amdgcn_readfirstlane(id / tiles);
  banded_tile(id - z * tiles, mtiles, ntiles, p.band, mt, nt);
  // divisions are done by the vector unit; copies take their addresses from scalar registers
  const int m0 = __builtin_amdgcn_readfirstlane(mt) * T::ROWS, n0 = __builtin_amdgcn_readfirstlane(nt) * T::ROWS;
  const int b0 = z * p.range_blocks, b1 = min(b0 + p.range_blocks, p.KB);
  const unsigned lds0 = lds_offset_of(lds);
  // The steps of the range.  A block that ends inside comes first, so that only the prologue has to clear what lies behind it.
  const int steps = b1 - b0, tail = b1 == p.KB ? p.K % SCALE_BLOCK : 0;
  auto block_of = [&](int t) { return !tail ? b0 + t : t == 0 ? b1 - 1 : b0 + t - 1; };

  // Which row of A is which row of LDS: a lane has row r of each of a wave's MT tiles of 16, and those are MT consecutive rows of
  // the matrix, so that it gets their scales in one load.
  auto arow_of = [&](int x) { return x / (16 * MT) * (16 * MT) + x % 16 * MT + x % (16 * MT) / 16; };
  // copies: lane l brings piece (l % 8) ^ (l / 8) of row l / 8 of eight rows; rows beyond the matrix repeat its last one
  const int cr = lane / 8, cp = (lane % 8) ^ cr;
  const char *abase = p.a + m0 * p.a_ld, *wbase = p.w + n0 * p.w_ld;
  unsigned aoff[4], woff[4];
  const int a8 = wm * (T::ROWS / 16) + wn;       // eight rows of A: a8 + WN c, in this wave's half; of W: wave + WAVES c
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    aoff[c] = (unsigned)min(arow_of(8 * (a8 + WN * c) + cr), p.M - 1 - m0) * (unsigned)p.a_ld + 16 * cp;
    woff[c] = (unsigned)min(8 * (wave + T::WAVES * c) + cr, p.N - 1 - n0) * (unsigned)p.w_ld + 16 * cp;
  }
  auto issue_a = [&](const unsigned (&off)[4], int t, int unit) {
    copy4<1024 * WN>(abase + (int64_t)block_of(t) * SCALE_BLOCK, off, lds0 + unit * T::UNIT + 1024 * a8, t, steps);
  };
  auto issue_w = [&](const unsigned (&off)[4], int t, int unit) {
    copy4<1024 * T::WAVES>(wbase + (int64_t)block_of(t) * SCALE_BLOCK, off, lds0 + T::W_AT + unit * T::UNIT + 1024 * wave, t, steps);
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
  f32x4 acc[NT][MT] = {}, d[LAG + 1] = {};
  float s_last = 0.f;
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
    const unsigned wv[4] = {woff[0] - back, woff[1] - back, woff[2] - back, woff[3] - back};
    const unsigned av[4] = {aoff[0] - back, aoff[1] - back, aoff[2] - back, aoff[3] - back};
    issue_w(wv, 0, 0);
    issue_a(av, 0, 0);
    wait_vmcnt<0>();
    for (int c = 0; c < 4; ++c) {
      clear8(1024 * (a8 + WN * c));
      clear8(T::W_AT + 1024 * (wave + T::WAVES * c));
    }
  }
  issue_w(woff, 1, 1);
  if (wm == 1) {       // half a step behind
    wait_copies<4>(1, steps);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    lds_barrier();
  }
  int wu = 0;          // unit of the step's rows of W
  for (int t = 0; t < steps; ++t) {
    const int at_a = t % 2 * T::UNIT, at_w = T::W_AT + wu * T::UNIT;
    // this wave's copies of the step's A have landed, its LDS accesses are done
    wait_copies<4>(t + 1, steps);
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
        wait_copies<8>(t + 2, steps);
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
  if (wm == 0) lds_barrier();      // as many as the other half
#pragma unroll
  for (int q = Q - LAG; q < Q; ++q) add(q, s_last);

  // ---- result: lane has columns n + 0..3 of row m of every 16 x 16 tile
  const int mw = m0 + arow, nw = n0 + 16 * NT * wn;
  if (p.part) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = mw + MT * r + i;
      if (m < p.M) {
        float* q = p.part + ((int64_t)z * p.M + m) * p.N;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int n = nw + 16 * j + 4 * g;
          if (n + 4 <= p.N) __builtin_memcpy(q + n, &acc[j][i], 16);
          else
            for (int e = 0; e < 4; ++e)
              if (n + e < p.N) q[n + e] = acc[j][i][e];
        }
      }
    }
    return;
  }
  lds_barrier();      // everyone has read the last step
  const bool f8 = p.out_type == SVDMLP_F8;
  float* amax_of = (float*)(lds + T::OUT);
  float inv[MT];
  if (f8) {
    // largest magnitude of the block of 128 columns that this wave and its neighbour hold half of each
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float x = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (nw + 16 * j + 4 * g + e < p.N) x = fmaxf(x, fabsf(acc[j][i][e]));
      x = fmaxf(x, __shfl_xor(x, 16));
      x = fmaxf(x, __shfl_xor(x, 32));
      if (g == 0) amax_of[wn * T::ROWS + arow + 16 * i + r] = x;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int row = arow + 16 * i + r, m = mw + MT * r + i;
      const __bf16 s = scale_of(fmaxf(amax_of[wn * T::ROWS + row], amax_of[(wn ^ 1) * T::ROWS + row]));
      inv[i] = 1.f / (float)s;
      if (g == 0 && wn % 2 == 0 && m < p.M && nw < p.N) p.c_scales[(int64_t)(nw / SCALE_BLOCK) * p.c_scales_ld + m] = s;
    }
  }
  char* mine = lds + wave * T::OUT_ROWS * T::OUT_LD;
  static_assert(16 * NT == 64, "two waves hold a block of 128 columns; 128 bytes of bf16 in a row's piece");
  constexpr int IR = T::OUT_ROWS / 16;     // row tiles that pass through LDS at a time
#pragma unroll
  for (int i0 = 0; i0 < MT; i0 += IR) {
#pragma unroll
    for (int i = i0; i < i0 + IR; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        char* q = mine + (16 * (i - i0) + r) * T::OUT_LD;
        const f32x4 v = acc[j][i];
        if (f8) *(unsigned*)(q + 16 * j + 4 * g) = codes4(v[0] * inv[i], v[1] * inv[i], v[2] * inv[i], v[3] * inv[i]);
        else *(bf16x4*)(q + 2 * (16 * j + 4 * g)) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
      }
    // LDS of the same wave: in order
    if (f8) {
#pragma unroll
      for (int k = 0; k < T::OUT_ROWS / 16; ++k) {
        const int row = 16 * k + lane / 4, m = mw + MT * (row % 16) + i0 + row / 16, n = nw + 16 * (lane % 4);
        if (m >= p.M || n >= p.N) continue;
        const u32x4 v = *(const u32x4*)(mine + row * T::OUT_LD + 16 * (lane % 4));
        unsigned char* c = (unsigned char*)p.c + m * p.c_ld + n;
        if (n + 16 <= p.N) *(u32x4*)c = v;
        else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (n + e < p.N) c[e] = (unsigned char)(v[e / 4] >> (8 * (e % 4)));
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < T::OUT_ROWS / 8; ++k) {
        const int row = 8 * k + lane / 8, m = mw + MT * (row % 16) + i0 + row / 16, n = nw + 8 * (lane % 8);
        if (m >= p.M || n >= p.N) continue;
        const u32x4 v = *(const u32x4*)(mine + row * T::OUT_LD + 16 * (lane % 8));
        __bf16* c = (__bf16*)p.c + m * p.c_ld + n;
        if (n + 8 <= p.N) __builtin_memcpy(c, &v, 16);
        else {
          const bf16x8 x = as_bf16x8(v);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (n + e < p.N) c[e] = x[e];
        }
      }
    }
  }
}

// Adds the ranges' partial sums in their order and rounds: 16 lanes hold 128 columns of a row, a workgroup 16 rows of them.
__global__ __launch_bounds__(256) void k_mm_join(MmP p) {
  const int lane = threadIdx.x % 16, nb = (p.N + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const int m = (int)(blockIdx.x / nb) * 16 + threadIdx.x / 16, b = (int)(blockIdx.x % nb), n = b * SCALE_BLOCK + 8 * lane;
  if (m >= p.M) return;
  float v[8] = {};
  if (n < p.N)
    for (int z = 0; z < p.ranges; ++z) {
      const Raw8<float> x = load8(p.part + ((int64_t)z * p.M + m) * p.N, n, p.N);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x.get(e);
    }
  if (p.out_type == SVDMLP_F8) {
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
    const __bf16 s = scale_of(max16(amax));
    if (n < p.N) store_codes8((unsigned char*)p.c + m * p.c_ld, n, p.N, v, 1.f / (float)s);
    if (lane == 0) p.c_scales[b * p.c_scales_ld + m] = s;
  } else if (n < p.N) {
    store8((__bf16*)p.c + m * p.c_ld, n, p.N, v);
  }
}

// ---- host -------------------------------------------------------------------------------------------
enum { MM_FEW = 0, MM_TILE_128 = 1, MM_TILE_256 = 2 };
struct MmPlan {
  int kernel;
  int mt, nt, waves;          // MM_FEW
  int ranges, range_blocks;
  bool join;                  // partial sums that k_mm_join adds and rounds
  int64_t tiles;
};


static int plan_mm(int64_t M, int64_t N, int64_t K, int out_type, MmPlan* q) {
  if (M < 0 || N <= 0 || K <= 0) return SVDMLP_INVALID_ARGUMENT;
  if (out_type != SVDMLP_F8 && out_type != SVDMLP_BF16) return SVDMLP_INVALID_ARGUMENT;
  if (M >= int64_t(1) << 24 || N > int64_t(1) << 22 || K > int64_t(1) << 22) return SVDMLP_UNSUPPORTED;
  const int KB = (int)scale_blocks(K);
  *q = MmPlan{};
  int ranges = 1;
  int few_max = 64;
  if (M <= few_max) {
    q->kernel = MM_FEW;
    q->mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    q->nt = 4;
    while (q->nt > 1 && (N + 16 * q->nt - 1) / (16 * q->nt) < 256) q->nt /= 2;
    q->tiles = (N + 16 * q->nt - 1) / (16 * q->nt);
    q->waves = q->tiles <= 256 && KB >= 32 && q->mt * q->nt <= 8 ? 16 : 8;
    if (out_type == SVDMLP_F8) {
      while (q->tiles * ranges < 256 && ranges * 2 * q->waves <= KB) ranges *= 2;
      q->join = true;
    }
  } else {
    const int64_t t256 = (M + 255) / 256 * ((N + 255) / 256), t128 = (M + 127) / 128 * ((N + 127) / 128);
    q->kernel = t256 >= 200 ? MM_TILE_256 : MM_TILE_128;
    q->tiles = q->kernel == MM_TILE_256 ? t256 : t128;
    const int slots = q->kernel == MM_TILE_256 ? 256 : 512;
    while (q->tiles * ranges * 2 <= slots && KB / (ranges * 2) >= 4) ranges *= 2;
  }
  q->range_blocks = (KB + ranges - 1) / ranges;
  q->ranges = (KB + q->range_blocks - 1) / q->range_blocks;
  if (q->ranges > 1) q->join = true;
  if (q->tiles * q->ranges >= int64_t(1) << 22) return SVDMLP_UNSUPPORTED;    // a grid of 1024 lanes each, below 2^32
  return SVDMLP_OK;
}

static size_t part_bytes(const MmPlan& q, int64_t M, int64_t N) { return q.join ? (size_t)q.ranges * M * N * 4 : 0; }

template <int MT, int NT>
static void run_few(const MmP& p, const MmPlan& q, hipStream_t st) {
  const unsigned wgs = (unsigned)(q.tiles * q.ranges);
  if (q.waves == 16) {
    if constexpr (MT * NT <= 8) k_mm_few<MT, NT, 16><<<wgs, 1024, 0, st>>>(p);
  }
  else if (q.waves == 8) k_mm_few<MT, NT, 8><<<wgs, 512, 0, st>>>(p);
  else k_mm_few<MT, NT, 4><<<wgs, 256, 0, st>>>(p);
}
template <int MT>
static void run_few(const MmP& p, const MmPlan& q, hipStream_t st) {
  if (q.nt == 1) run_few<MT, 1>(p, q, st);
  else if (q.nt == 2) run_few<MT, 2>(p, q, st);
  else run_few<MT, 4>(p, q, st);
}

static void launch_mm(MmP& p, const MmPlan& q, hipStream_t st) {
  if (q.kernel == MM_FEW) {
    if (q.mt == 1) run_few<1>(p, q, st);
    else if (q.mt == 2) run_few<2>(p, q, st);
    else run_few<4>(p, q, st);
    return;
  }
  const unsigned wgs = (unsigned)(q.tiles * q.ranges);
  const int rows = q.kernel == MM_TILE_256 ? 256 : 128;
  p.band = band_height((p.M + rows - 1) / rows, wgs);
  if (q.kernel == MM_TILE_256) k_mm_tile<8, 4, 2, 4><<<wgs, 512, 0, st>>>(p);
  else k_mm_tile<4, 4, 2, 2><<<wgs, 256, 0, st>>>(p);
}

}  // namespace svdmlp

using namespace svdmlp;

extern "C" {

size_t svdmlp_scaled_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t out_type) {
  MmPlan q;
  return plan_mm(M, N, K, out_type, &q) == SVDMLP_OK ? part_bytes(q, M, N) : 0;
}

int svdmlp_scaled_matmul_describe(int64_t M, int64_t N, int64_t K, int32_t out_type, char* buf, size_t buf_bytes) {
  if (!buf || buf_bytes == 0) return SVDMLP_INVALID_ARGUMENT;
  buf[0] = 0;
  MmPlan q;
  if (const int st = plan_mm(M, N, K, out_type, &q)) return st;
  int n;
  if (q.kernel == MM_FEW)
    n = std::snprintf(buf, buf_bytes, "k_mm_few[tile=%dx%d tiles=%lld waves=%d ranges=%d]%s", 16 * q.mt, 16 * q.nt, (long long)q.tiles,
                      q.waves, q.ranges, q.join ? " k_mm_join" : "");
  else
    n = std::snprintf(buf, buf_bytes, "k_mm_tile[tile=%s tiles=%lld ranges=%d]%s", q.kernel == MM_TILE_256 ? "256x256" : "128x128",
                      (long long)q.tiles, q.ranges, q.join ? " k_mm_join" : "");
  return n > 0 && (size_t)n < buf_bytes ? SVDMLP_OK : SVDMLP_INVALID_ARGUMENT;
}

int svdmlp_scaled_matmul(const svdmlp_scaled_matmul_args* a, void* hip_stream) {
  if (!a || a->reserved != 0) return SVDMLP_INVALID_ARGUMENT;
  MmPlan q;
  if (const int st = plan_mm(a->M, a->N, a->K, a->out_type, &q)) return st;
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
  MmP p;
  p.a = (const char*)a->a; p.w = (const char*)a->w; p.sa = (const __bf16*)a->a_scales; p.sw = a->w_scales;
  p.c = a->c; p.c_scales = (__bf16*)a->c_scales; p.part = q.join ? (float*)a->workspace : nullptr;
  p.a_ld = a->a_ld; p.w_ld = a->w_ld; p.sa_ld = a->a_scales_ld; p.c_ld = a->c_ld; p.c_scales_ld = a->c_scales_ld;
  p.M = (int)a->M; p.N = (int)a->N; p.K = (int)a->K; p.KB = (int)scale_blocks(a->K);
  p.out_type = a->out_type;
  p.ranges = q.ranges; p.range_blocks = q.range_blocks;
  hipStream_t st = (hipStream_t)hip_stream;
  launch_mm(p, q, st);
  if (q.join) k_mm_join<<<(unsigned)((p.M + 15) / 16 * scale_blocks(p.N)), 256, 0, st>>>(p);
  return launch_status();
}

}  // extern "C"
