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
// this lane's 32 codes of block b of a row
__device__ __forceinline__ i32x8 block_codes(const char* row, int b, int g, int K) {
  const int c = b * SCALE_BLOCK + 16 * g;
  if (K - b * SCALE_BLOCK >= SCALE_BLOCK) return join16(*(const u32x4*)(row + c), *(const u32x4*)(row + c + 64));
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

// Tiles of 16 MT rows x 16 NT columns; the blocks of the contraction go to the waves in turn, whose sums meet in LDS.
template <int MT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_mm_few(MmP p) {
  __shared__ f32x4 red[WAVES][MT * NT][64];
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
  const char *wr[NT], *ar[MT];
  const __bf16* sa[MT];
#pragma unroll
  for (int j = 0; j < NT; ++j) wr[j] = p.w + (int64_t)min(n0 + 16 * j + r, p.N - 1) * p.w_ld;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(m0 + 16 * i + r, p.M - 1);
    ar[i] = p.a + m * p.a_ld;
    sa[i] = p.sa + m;
  }
  const float* sw = p.sw + (int64_t)(n0 / SCALE_BLOCK) * p.KB;
  f32x4 acc[NT][MT] = {};
  const int b0 = blockIdx.z * p.range_blocks, b1 = min(b0 + p.range_blocks, p.KB);
  for (int b = b0 + wave; b < b1; b += WAVES) {
    i32x8 fw[NT], fa[MT];
    float s[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) fw[j] = block_codes(wr[j], b, g, p.K);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      fa[i] = block_codes(ar[i], b, g, p.K);
      s[i] = (float)sa[i][b * p.sa_ld] * sw[b];
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const f32x4 d = mfma_f8(fw[j], fa[i], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][i][e] += d[e] * s[i];
      }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) red[wave][j * MT + i][lane] = acc[j][i];
  __syncthreads();
  for (int x = threadIdx.x; x < MT * NT * 64; x += 64 * WAVES) {
    f32x4 v = red[0][x / 64][x % 64];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += red[w][x / 64][x % 64];
    const int j = x / 64 / MT, i = x / 64 % MT, m = m0 + 16 * i + x % 16, n = n0 + 16 * j + 4 * (x % 64 / 16);
    if (!p.part) {
      store4(p, m, n, v);
    } else if (m < p.M) {
      float* q = p.part + ((int64_t)blockIdx.z * p.M + m) * p.N + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < p.N) q[e] = v[e];
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
struct MmPlan {
  int ranges, range_blocks;
  bool join;
};

static int plan_mm(int64_t M, int64_t N, int64_t K, int out_type, MmPlan* q) {
  if (M < 0 || N <= 0 || K <= 0) return SVDMLP_INVALID_ARGUMENT;
  if (out_type != SVDMLP_F8 && out_type != SVDMLP_BF16) return SVDMLP_INVALID_ARGUMENT;
  if (M >= int64_t(1) << 24 || N > int64_t(1) << 22 || K > int64_t(1) << 22) return SVDMLP_UNSUPPORTED;
  if (M > int64_t(65535) * 64) return SVDMLP_UNSUPPORTED;   // a grid's second dimension
  const int KB = (int)scale_blocks(K);
  q->ranges = 1;
  q->range_blocks = KB;
  q->join = out_type == SVDMLP_F8;
  return SVDMLP_OK;
}

static size_t part_bytes(const MmPlan& q, int64_t M, int64_t N) { return q.join ? (size_t)q.ranges * M * N * 4 : 0; }

static void launch_mm(const MmP& p, hipStream_t st) {
  k_mm_few<4, 4, 4><<<dim3((p.N + 63) / 64, (p.M + 63) / 64, p.ranges), 256, 0, st>>>(p);
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
  const int n = std::snprintf(buf, buf_bytes, "k_mm_few[tile=64x64 ranges=%d]%s", q.ranges, q.join ? " k_mm_join" : "");
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
  launch_mm(p, st);
  if (q.join) k_mm_join<<<(unsigned)((p.M + 15) / 16 * scale_blocks(p.N)), 256, 0, st>>>(p);
  return launch_status();
}

}  // extern "C"
