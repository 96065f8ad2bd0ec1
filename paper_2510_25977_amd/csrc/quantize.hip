// Quantiser to e4m3 codes with a scale per block: scale = max(amax / 448, 2^-100), code = nearest even of v / scale.
// Bounded by HBM: 2 (gated 4) bytes of bf16 read and one written per element, about twenty vector instructions on it;
// 4096 x 14336 gated 294 MB in 56 us (5.2 TB/s; a copy of 2 GiB moves 4.8), not gated 177 MB in 34 us (in a graph, over as many
// sets of tensors as no cache holds); weights of 28672 x 4096, once, 353 MB in 65 us (by the profiler).
#include "scaled.h"

namespace svdmlp {

struct QuantP {
  const void *x, *gated;
  unsigned char* codes;
  void* scales;        // bf16, weights: fp32
  int64_t x_ld, gated_ld, codes_ld, scales_ld;
  int64_t rows;
  int cols;
};

// A group of 16 lanes holds the 128 columns of one row's block, eight a lane.  A workgroup takes 16 rows x QB blocks: the
// scales of 16 rows lie side by side, and a row's piece is QB * 256 bytes of bf16.
template <class T, bool GATED, int QB, RowEnd END>
__global__ __launch_bounds__(256) void k_quantize(QuantP p) {
  const int g = threadIdx.x / 16, lane = threadIdx.x % 16;
  const int nb = (p.cols + SCALE_BLOCK - 1) / SCALE_BLOCK, strips = (nb + QB - 1) / QB;
  const int64_t row = (int64_t)(blockIdx.x / strips) * 16 + g;
  const int b0 = (int)(blockIdx.x % strips) * QB;
  if (row >= p.rows) return;
  const T* x = (const T*)p.x + row * p.x_ld;
  const T* u = GATED ? (const T*)p.gated + row * p.gated_ld : nullptr;
  Raw8<T> rx[QB], ru[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    const Cols<END> k((b0 + i) * SCALE_BLOCK + lane * 8, p.cols);
    rx[i] = load8(x, k);
    if (GATED) ru[i] = load8(u, k);
  }
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    const Cols<END> k((b0 + i) * SCALE_BLOCK + lane * 8, p.cols);
    float v[8], amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = rx[i].get(e);
      if (GATED) v[e] *= __builtin_amdgcn_rcpf(1.f + __expf(-v[e])) * ru[i].get(e);
      amax = END == WHOLE || k.own(e) ? fmaxf(amax, fabsf(v[e])) : amax;
    }
    const __bf16 s = scale_of(max16(amax));
    if (k.any()) store_codes8(p.codes + row * p.codes_ld, k, v, 1.f / (float)s);
    if (lane == 0 && b0 + i < nb) ((__bf16*)p.scales)[(int64_t)(b0 + i) * p.scales_ld + row] = s;
  }
}

// Weights, once: a workgroup per 128 x 128 block.
template <class T, RowEnd END>
__global__ __launch_bounds__(256) void k_quantize_block(QuantP p) {
  __shared__ float part[4];
  const int g = threadIdx.x / 16, lane = threadIdx.x % 16;
  const int kb = (p.cols + SCALE_BLOCK - 1) / SCALE_BLOCK;
  const int64_t r0 = (int64_t)(blockIdx.x / kb) * SCALE_BLOCK;
  const Cols<END> k((int)(blockIdx.x % kb) * SCALE_BLOCK + lane * 8, p.cols);
  Raw8<T> r[8];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + g + 16 * i;
    r[i] = row < p.rows ? load8((const T*)p.x + row * p.x_ld, k) : Raw8<T>{};
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = END == WHOLE || k.own(e) ? fmaxf(amax, fabsf(r[i].get(e))) : amax;
  amax = max16(amax);
  amax = fmaxf(amax, __shfl_xor(amax, 16));
  amax = fmaxf(amax, __shfl_xor(amax, 32));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = amax;
  __syncthreads();
  const float s = weight_scale_of(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + g + 16 * i;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r[i].get(e);
    if (row < p.rows && k.any()) store_codes8(p.codes + row * p.codes_ld, k, v, 1.f / s);
  }
  if (threadIdx.x == 0) ((float*)p.scales)[blockIdx.x] = s;
}

// Blocks a group: 1 / 2 / 4 take, in a graph over several sets, 53.2 / 54.4 / 56.0 us at 4096 x 14336 gated, 34.1 / 32.2 / 33.7 not
// gated, 13.0 / 12.2 / 12.4 at 4096 x 4096, 17.7 / 17.0 / 17.9 at 1777 x 7301 gated: within 5 %.  At few rows, where workgroups are
// few, four are the slowest: 2.4 / 2.7 / 3.4 us at 16 x 14336 gated, of the 4.2 us that a call takes the host.  Rows of less than
// eight columns have one block.
template <class T, bool GATED, int QB, RowEnd END>
static hipError_t run_quantize(const QuantP& p, hipStream_t st) {
  const int64_t strips = (p.rows + 15) / 16, nb = scale_blocks(p.cols);
  return launch(k_quantize<T, GATED, QB, END>, (unsigned)(strips * ((nb + QB - 1) / QB)), 256, p, st);
}
template <class T, RowEnd END>
static hipError_t launch_quantize(const QuantP& p, bool weights, hipStream_t st) {
  constexpr int QB = END == SHORT ? 1 : 4;
  if (weights) return launch(k_quantize_block<T, END>, (unsigned)(scale_blocks(p.rows) * scale_blocks(p.cols)), 256, p, st);
  if (p.gated) return run_quantize<T, true, QB, END>(p, st);
  return run_quantize<T, false, QB, END>(p, st);
}
template <class T>
static hipError_t launch_quantize(const QuantP& p, bool weights, hipStream_t st) {
  switch (row_end(p.cols)) {
    case WHOLE: return launch_quantize<T, WHOLE>(p, weights, st);
    case OVERLAP: return launch_quantize<T, OVERLAP>(p, weights, st);
    default: return launch_quantize<T, SHORT>(p, weights, st);
  }
}

}  // namespace svdmlp

using namespace svdmlp;

extern "C" int svdmlp_quantize(const svdmlp_quantize_args* a, void* hip_stream) {
  if (!a || a->rows < 0 || a->cols <= 0 || !is_float_type(a->type)) return SVDMLP_INVALID_ARGUMENT;
  if (a->block_rows != 1 && a->block_rows != SCALE_BLOCK) return SVDMLP_INVALID_ARGUMENT;
  const bool weights = a->block_rows == SCALE_BLOCK;
  if (weights && a->gated) return SVDMLP_INVALID_ARGUMENT;
  if (!a->x || a->x_ld < a->cols || (a->gated && a->gated_ld < a->cols)) return SVDMLP_INVALID_ARGUMENT;
  const int64_t t = type_bytes(a->type);
  if (!aligned_to(a->x, t) || !aligned_to(a->gated, t)) return SVDMLP_INVALID_ARGUMENT;
  if (const int st = check_codes(a->codes, a->codes_ld, a->cols)) return st;
  if (!a->scales || !aligned_to(a->scales, weights ? 4 : 2) || (!weights && a->scales_ld < a->rows)) return SVDMLP_INVALID_ARGUMENT;
  if (a->codes == a->x || a->codes == a->gated) return SVDMLP_INVALID_ARGUMENT;
  if (a->rows >= int64_t(1) << 24 || a->cols > int64_t(1) << 22) return SVDMLP_UNSUPPORTED;
  if ((a->rows + 15) / 16 * scale_blocks(a->cols) >= int64_t(1) << 23) return SVDMLP_UNSUPPORTED;   // grid of 256 lanes below 2^31
  if (a->rows == 0) return SVDMLP_OK;
  if (outputs_overlap({rows_of(a->codes, a->rows, a->cols, a->codes_ld, 1),
                       weights ? weight_scales(a->scales, a->rows, a->cols) : activation_scales(a->scales, a->rows, a->cols, a->scales_ld)},
                      {rows_of(a->x, a->rows, a->cols, a->x_ld, t), rows_of(a->gated, a->rows, a->cols, a->gated_ld, t)}))
    return SVDMLP_INVALID_ARGUMENT;
  const QuantP p = {a->x, a->gated, (unsigned char*)a->codes, a->scales, a->x_ld, a->gated_ld, a->codes_ld, a->scales_ld,
                    a->rows, (int)a->cols};
  if (a->type == SVDMLP_F32) return status_of(launch_quantize<float>(p, weights, (hipStream_t)hip_stream));
  return status_of(launch_quantize<__bf16>(p, weights, (hipStream_t)hip_stream));
}
