// The norms around a block of the residual stream, with the residual, the gate and the scales, in one pass:
//   b = [norm(branch) (weight + plus) + bias] branch_scale act(gate)    h = residual_scale residual + b    out = norm(h) ..
// A row lies in the registers of its threads in fp32 from its first load to its last store, so every input is read once and
// every result written once, and HBM bounds it (in a graph, over as many sets of tensors as no cache holds): 4096 x 4096 with a
// residual into 8 bits 118 MB in 24.9 us (4.7 TB/s; a copy of 2 GiB moves 4.8), 8192 x 5120 with an fp32 residual 503 MB in 91 us
// (5.5 TB/s), with a tanh gate and scale 108 us.
#include "scaled.h"

namespace svdmlp {

struct NormP {
  const void *residual, *branch, *weight, *bias, *branch_scale, *gate, *next_weight, *next_bias;
  void *h, *out;
  __bf16* out_scales;
  int64_t residual_ld, branch_ld, gate_ld, h_ld, out_ld, out_scales_ld;
  int64_t rows;
  unsigned gate_rows;
  int d, kind, next_kind, gate_act, out_f8;
  float eps, next_eps, weight_plus, residual_scale, inv_d;
};

// Sum over the TPR threads of a row.  part: one float per wave, a buffer of its own for every call of a kernel.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* part) {
  x = sum64(x);
  if constexpr (TPR > 64) {
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) x += part[w];
  }
  return x;
}

// v <- its norm, without weight.  What is not a thread's own holds zeros and is left out of the second sum of a LAYER norm.
template <int TPR, int NV, RowEnd END>
__device__ __forceinline__ void normalize(float (&v)[NV][8], int kind, float eps, const NormP& p, int t, float* part) {
  if (kind == SVDMLP_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[i][e];
    const float mean = row_sum<TPR>(s, part) * p.inv_d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = Cols<END>((i * TPR + t) * 8, p.d).own(e) ? v[i][e] - mean : 0.f;
    part += TPR / 64;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[i][e] * v[i][e];
  const float scale = 1.f / sqrtf(row_sum<TPR>(s, part) * p.inv_d + eps);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] *= scale;
}

// tanh to a few units in the last place: its series up to x^9 below 0.25, from exp(2 |x|) above
__device__ __forceinline__ float tanh_f32(float x) {
  const float y = fabsf(x), y2 = y * y;
  const float series = y * (1.f + y2 * (-1.f / 3 + y2 * (2.f / 15 + y2 * (-17.f / 315 + y2 * (62.f / 2835)))));
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(__expf(2.f * y) + 1.f);
  return copysignf(y < 0.25f ? series : t, x);
}
__device__ __forceinline__ float activated(float g, int act) {
  return act == SVDMLP_GATE_SIGMOID ? __builtin_amdgcn_rcpf(1.f + __expf(-g)) : act == SVDMLP_GATE_TANH ? tanh_f32(g) : g;
}

// TPR threads hold a row, thread t columns 8 (i TPR + t) .. + 7, i < NV: 16 lanes hold a block of 128 columns.  Weights come with the
// row up to two vectors a thread (4096 x 4096 24.9 us, 25.4 after the row's sum), with four they come when they are needed: the
// registers allow half the waves otherwise (2048 x 16384 with every input and an fp32 residual 120 us, 143; fp32 RMS norm of 2048 x
// 32768 123, 237).  At one vector of bf16 the biases, the scale and the gate come along too (3616 x 3968 with all of them 32.7 us,
// 35.0 later).
template <class T, class S, int TPR, int NV, RowEnd END>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void k_norm(NormP p) {
  constexpr int WAVES = TPR / 64;
  constexpr bool EARLY = NV < 4;                         // weights loaded with the row,
  constexpr bool ALL_EARLY = NV == 1 && sizeof(T) == 2;  // and whatever else there is
  __shared__ float part[4 * WAVES];
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (TPR == 64 ? 4 : 1) + threadIdx.x / TPR;
  if (row >= p.rows) return;   // whole waves, and whole workgroups where they meet at a barrier
  Raw8<T> rb[NV], w[NV], nw[NV], bias[NV], bscale[NV], gate[NV], nbias[NV];
  Raw8<S> rr[NV];
  const T* gate_row = (const T*)p.gate + (int64_t)((unsigned)row / p.gate_rows) * p.gate_ld;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Cols<END> k((i * TPR + t) * 8, p.d);
    rb[i] = p.branch ? load8((const T*)p.branch + row * p.branch_ld, k) : Raw8<T>{};
    rr[i] = p.residual ? load8((const S*)p.residual + row * p.residual_ld, k) : Raw8<S>{};
    if (EARLY) {
      w[i] = p.weight ? load8((const T*)p.weight, k) : Raw8<T>{};
      nw[i] = p.next_weight ? load8((const T*)p.next_weight, k) : Raw8<T>{};
    }
    if (ALL_EARLY) {
      bias[i] = p.bias ? load8((const T*)p.bias, k) : Raw8<T>{};
      bscale[i] = p.branch_scale ? load8((const T*)p.branch_scale, k) : Raw8<T>{};
      gate[i] = p.gate ? load8(gate_row, k) : Raw8<T>{};
      nbias[i] = p.next_bias ? load8((const T*)p.next_bias, k) : Raw8<T>{};
    }
  }
  float v[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Cols<END> k((i * TPR + t) * 8, p.d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = END == WHOLE || k.own(e) ? rb[i].get(e) : 0.f;
  }
  if (p.kind != SVDMLP_NORM_NONE) normalize<TPR, NV, END>(v, p.kind, p.eps, p, t, part);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Cols<END> k((i * TPR + t) * 8, p.d);
    if (!k.any()) continue;
    if (p.weight) {
      if (!EARLY) w[i] = load8((const T*)p.weight, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= w[i].get(e) + p.weight_plus;
    }
    if (p.bias) {
      if (!ALL_EARLY) bias[i] = load8((const T*)p.bias, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] += bias[i].get(e);
    }
    if (p.branch_scale) {
      if (!ALL_EARLY) bscale[i] = load8((const T*)p.branch_scale, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= bscale[i].get(e);
    }
    if (p.gate) {
      if (!ALL_EARLY) gate[i] = load8(gate_row, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= activated(gate[i].get(e), p.gate_act);
    }
    if (p.residual) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] += p.residual_scale * rr[i].get(e);
    }
    if (p.h) store8((S*)p.h + row * p.h_ld, k, v[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (END != WHOLE && !k.own(e)) v[i][e] = 0.f;
  }
  if (p.next_kind == SVDMLP_NORM_NONE) return;
  normalize<TPR, NV, END>(v, p.next_kind, p.next_eps, p, t, part + 2 * WAVES);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Cols<END> k((i * TPR + t) * 8, p.d);
    if (p.next_weight) {
      if (!EARLY) nw[i] = load8((const T*)p.next_weight, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= nw[i].get(e) + p.weight_plus;
    }
    if (p.next_bias) {
      if (!ALL_EARLY) nbias[i] = load8((const T*)p.next_bias, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] += nbias[i].get(e);
    }
    if (!p.out_f8) {
      if (k.any()) store8((T*)p.out + row * p.out_ld, k, v[i]);
      continue;
    }
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = END == WHOLE || k.own(e) ? fmaxf(amax, fabsf(v[i][e])) : amax;
    const __bf16 s = scale_of(max16(amax));
    if (k.any()) {
      store_codes8((unsigned char*)p.out + row * p.out_ld, k, v[i], 1.f / (float)s);
      if (t % 16 == 0) p.out_scales[(int64_t)((i * TPR + t) / 16) * p.out_scales_ld + row] = s;
    }
  }
}

template <class T, class S, int TPR, int NV, RowEnd END>
static hipError_t run_norm(const NormP& p, hipStream_t st) {
  constexpr int per = TPR == 64 ? 4 : 1;
  return launch(k_norm<T, S, TPR, NV, END>, (unsigned)((p.rows + per - 1) / per), TPR * per, p, st);
}
template <class T, class S, int TPR, int NV>
static hipError_t run_norm(const NormP& p, hipStream_t st) {
  if (p.d % 8 == 0) return run_norm<T, S, TPR, NV, WHOLE>(p, st);
  return run_norm<T, S, TPR, NV, OVERLAP>(p, st);
}

// As few vectors a thread as a workgroup's size allows: a row's chain (loads, sums over the workgroup, stores) is what a CU has
// four of at 512 threads.  us in a graph over several sets, 1024 / 512 / 256 / 128 threads for the row: 4096 x 4096 in 8 bits with
// a residual 26.4 / 24.9 / 25.6 / 29.3, one such row 3.1 / 2.8 / 3.4 / 4.6, 8192 x 5120 with every input and an fp32 residual 166 /
// 120 / 126 / -; 5359 x 562 with all inputs 13.4 with 128 threads, 16.8 with 256.
static int row_threads(int64_t d) { return d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 16384 ? 512 : 1024; }

template <class T, class S>
static hipError_t launch_norm(const NormP& p, hipStream_t st) {
  if (row_end(p.d) == SHORT) return run_norm<T, S, 64, 1, SHORT>(p, st);
  switch (row_threads(p.d)) {
    case 64: return run_norm<T, S, 64, 1>(p, st);
    case 128: return run_norm<T, S, 128, 1>(p, st);
    case 256: return run_norm<T, S, 256, 1>(p, st);
    case 512: break;
    default: return run_norm<T, S, 1024, 4>(p, st);
  }
  if (p.d <= 4096) return run_norm<T, S, 512, 1>(p, st);
  if (p.d <= 8192) return run_norm<T, S, 512, 2>(p, st);
  return run_norm<T, S, 512, 4>(p, st);
}

static bool known_norm(int k) { return k == SVDMLP_NORM_NONE || k == SVDMLP_NORM_RMS || k == SVDMLP_NORM_LAYER; }

}  // namespace svdmlp

using namespace svdmlp;

extern "C" int svdmlp_norm(const svdmlp_norm_args* a, void* hip_stream) {
  if (!a || a->rows < 0 || a->d <= 0 || !is_float_type(a->type) || !is_float_type(a->stream_type)) return SVDMLP_INVALID_ARGUMENT;
  if (a->out_type != a->type && a->out_type != SVDMLP_F8) return SVDMLP_INVALID_ARGUMENT;
  if (!known_norm(a->kind) || !known_norm(a->next_kind)) return SVDMLP_INVALID_ARGUMENT;
  if (a->gate_act < SVDMLP_GATE_PLAIN || a->gate_act > SVDMLP_GATE_TANH) return SVDMLP_INVALID_ARGUMENT;
  if (!a->residual && !a->branch) return SVDMLP_INVALID_ARGUMENT;
  const bool next = a->next_kind != SVDMLP_NORM_NONE;
  if (next != (a->out != nullptr) || (!next && !a->h)) return SVDMLP_INVALID_ARGUMENT;
  if (!a->branch && (a->kind != SVDMLP_NORM_NONE || a->branch_scale || a->gate)) return SVDMLP_INVALID_ARGUMENT;
  if ((a->kind != SVDMLP_NORM_NONE && !(a->eps > 0.f)) || (next && !(a->next_eps > 0.f))) return SVDMLP_INVALID_ARGUMENT;
  if ((a->kind == SVDMLP_NORM_NONE && (a->weight || a->bias)) || (!next && (a->next_weight || a->next_bias))) return SVDMLP_INVALID_ARGUMENT;
  if (a->gate && (a->gate_rows < 1 || a->gate_ld < a->d)) return SVDMLP_INVALID_ARGUMENT;
  if ((a->residual && a->residual_ld < a->d) || (a->branch && a->branch_ld < a->d) || (a->h && a->h_ld < a->d)) return SVDMLP_INVALID_ARGUMENT;
  const int64_t t = type_bytes(a->type), s = type_bytes(a->stream_type), o = type_bytes(a->out_type);
  for (const void* q : {a->branch, a->weight, a->bias, a->branch_scale, a->gate, a->next_weight, a->next_bias})
    if (!aligned_to(q, t)) return SVDMLP_INVALID_ARGUMENT;
  if (!aligned_to(a->residual, s) || !aligned_to(a->h, s)) return SVDMLP_INVALID_ARGUMENT;
  if (next && a->out_type == SVDMLP_F8) {
    if (const int st = check_codes(a->out, a->out_ld, a->d)) return st;
    if (!a->out_scales || !aligned_to(a->out_scales, 2) || a->out_scales_ld < a->rows) return SVDMLP_INVALID_ARGUMENT;
  } else if (next && (a->out_ld < a->d || !aligned_to(a->out, t))) {
    return SVDMLP_INVALID_ARGUMENT;
  }
  // h may take the place of the residual, element for element; nothing else may share a buffer
  if (a->h && a->h == a->residual && a->h_ld != a->residual_ld) return SVDMLP_INVALID_ARGUMENT;
  if ((a->h && (a->h == a->branch || a->h == a->out)) || (a->out && (a->out == a->residual || a->out == a->branch))) return SVDMLP_INVALID_ARGUMENT;
  if (a->type == SVDMLP_F32 && a->stream_type == SVDMLP_BF16) return SVDMLP_UNSUPPORTED;
  if (a->d > 32768 || a->rows >= (int64_t(1) << 31) / row_threads(a->d)) return SVDMLP_UNSUPPORTED;   // registers; lanes of a grid
  if (a->rows == 0) return SVDMLP_OK;
  auto vec = [&](const void* q) { return rows_of(q, 1, a->d, 0, t); };
  if (outputs_overlap({rows_of(a->h, a->rows, a->d, a->h_ld, s), rows_of(a->out, a->rows, a->d, a->out_ld, o),
                       activation_scales(next && o == 1 ? a->out_scales : nullptr, a->rows, a->d, a->out_scales_ld)},
                      {rows_of(a->residual == a->h ? nullptr : a->residual, a->rows, a->d, a->residual_ld, s),
                       rows_of(a->branch, a->rows, a->d, a->branch_ld, t), vec(a->weight), vec(a->bias), vec(a->branch_scale),
                       rows_of(a->gate, a->gate ? (a->rows - 1) / a->gate_rows + 1 : 0, a->d, a->gate_ld, t), vec(a->next_weight), vec(a->next_bias)}))
    return SVDMLP_INVALID_ARGUMENT;
  NormP p;
  p.residual = a->residual; p.branch = a->branch; p.weight = a->weight; p.bias = a->bias;
  p.branch_scale = a->branch_scale; p.gate = a->gate; p.next_weight = a->next_weight; p.next_bias = a->next_bias;
  p.h = a->h; p.out = a->out; p.out_scales = (__bf16*)a->out_scales;
  p.residual_ld = a->residual_ld; p.branch_ld = a->branch_ld; p.gate_ld = a->gate_ld; p.h_ld = a->h_ld; p.out_ld = a->out_ld;
  p.out_scales_ld = a->out_scales_ld; p.gate_rows = (unsigned)(a->gate_rows < 1 ? 1 : a->gate_rows < a->rows ? a->gate_rows : a->rows);
  p.rows = a->rows; p.d = (int)a->d; p.kind = a->kind; p.next_kind = a->next_kind; p.gate_act = a->gate_act;
  p.out_f8 = next && a->out_type == SVDMLP_F8;
  p.eps = a->eps; p.next_eps = a->next_eps; p.weight_plus = a->weight_plus; p.residual_scale = a->residual_scale;
  p.inv_d = (float)(1.0 / (double)a->d);
  hipStream_t st = (hipStream_t)hip_stream;
  if (a->type == SVDMLP_F32) return status_of(launch_norm<float, float>(p, st));
  if (a->stream_type == SVDMLP_F32) return status_of(launch_norm<__bf16, float>(p, st));
  return status_of(launch_norm<__bf16, __bf16>(p, st));
}
