// What the operators around an 8-bit factored layer share: vectors of a row that may start and end anywhere, e4m3 codes,
// reductions over lanes, and the host's argument checks.
#pragma once
#include "common.h"
#include "rows.h"

namespace svdmlp {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

constexpr int SCALE_BLOCK = 128;              // columns (weights: rows too) that share a scale
constexpr float F8_LARGEST = 448.f;           // e4m3
constexpr float F8_SMALLEST_SCALE = 0x1p-100f;  // keeps 1 / scale finite; an all-zero block gets it
constexpr int64_t MAX_CODE_LD = int64_t(1) << 23;   // 256 rows of codes stay within a 32-bit offset

inline int64_t scale_blocks(int64_t n) { return (n + SCALE_BLOCK - 1) / SCALE_BLOCK; }
inline bool is_float_type(int t) { return t == SVDMLP_BF16 || t == SVDMLP_F32; }
inline int64_t type_bytes(int t) { return t == SVDMLP_F32 ? 4 : t == SVDMLP_F8 ? 1 : 2; }
inline bool aligned_to(const void* q, size_t a) { return (reinterpret_cast<uintptr_t>(q) & (a - 1)) == 0; }
// Rows of codes: 16-byte aligned, stride a multiple of 16
inline int check_codes(const void* codes, int64_t ld, int64_t cols) {
  if (!codes || ld < cols) return SVDMLP_INVALID_ARGUMENT;
  if (!aligned_to(codes, 16) || ld % 16) return SVDMLP_INVALID_ARGUMENT;
  return ld < MAX_CODE_LD ? SVDMLP_OK : SVDMLP_UNSUPPORTED;
}
inline Rows rows_of(const void* at, int64_t rows, int64_t cols, int64_t ld, int64_t bytes) {
  return Rows(at, rows, cols * bytes, rows > 1 ? ld * bytes : 0);
}
inline Rows activation_scales(const void* at, int64_t rows, int64_t cols, int64_t ld) { return rows_of(at, scale_blocks(cols), rows, ld, 2); }
inline Rows weight_scales(const void* at, int64_t rows, int64_t cols) { return rows_of(at, 1, scale_blocks(rows) * scale_blocks(cols), 0, 4); }
inline int status_of(hipError_t e) { return e == hipSuccess ? SVDMLP_OK : SVDMLP_HIP_ERROR; }

#ifdef __HIPCC__
// One launch and its own error: the thread's last error may be one that an earlier call of the program left there.
template <class P>
hipError_t launch(void (*kernel)(P), unsigned workgroups, unsigned threads, const P& p, hipStream_t st) {
  void* args[] = {const_cast<P*>(&p)};
  const hipError_t e = hipLaunchKernel((const void*)kernel, dim3(workgroups), dim3(threads), args, 0, st);
  if (e != hipSuccess) (void)hipGetLastError();      // reported by the status
  return e;
}

// Eight consecutive elements of a row as they lie in memory, from any element's address (the hardware takes 16-byte
// accesses at any alignment).
template <class T>
struct Raw8;
template <>
struct Raw8<__bf16> {
  u32x4 v;
  __device__ __forceinline__ float get(int e) const {
    const unsigned w = v[e / 2];
    return __builtin_bit_cast(float, e % 2 ? w & 0xffff0000u : w << 16);
  }
};
template <>
struct Raw8<float> {
  f32x4 v[2];
  __device__ __forceinline__ float get(int e) const { return v[e / 4][e % 4]; }
};

// How rows of n columns end, for kernels whose lanes hold eight consecutive columns each, from a multiple of 8 on.  WHOLE: n is a
// multiple of 8.  OVERLAP: the last vector that begins inside is read from column n - 8 on, and its first columns, which the lane
// before it has too, are left out of sums and stores; so no lane loads element by element, and waits for that, while the others
// wait for it at the row's next barrier (fp32 RMS norm of 4096 x 4091: 37 us that way, 28.7 this; 4096 x 4096 27.0).  SHORT: rows
// of less than eight columns, element by element.
enum RowEnd { WHOLE, OVERLAP, SHORT };
inline RowEnd row_end(int64_t n) { return n % 8 == 0 ? WHOLE : n > 8 ? OVERLAP : SHORT; }

// The columns c .. c + 7 of a lane whose own begin at col; the first `skip` are not its own (8: it has none).
template <RowEnd END>
struct Cols {
  int c, skip;
  __device__ __forceinline__ Cols(int col, int n)
      : c(END == WHOLE ? col : min(col, n - 8)), skip(END == WHOLE ? (col < n ? 0 : 8) : max(0, min(8, col + 8 - n))) {}
  __device__ __forceinline__ bool any() const { return skip < 8; }
  __device__ __forceinline__ bool own(int e) const { return END == WHOLE ? any() : e >= skip; }
};

template <class T, RowEnd END>
__device__ __forceinline__ Raw8<T> load8(const T* row, const Cols<END>& k) {
  Raw8<T> r = {};
  if (END != SHORT) {
    if (k.any()) __builtin_memcpy(&r, row + k.c, sizeof(r));
  } else {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k.own(i) ? row[k.c + i] : (T)0.f;
    __builtin_memcpy(&r, e, sizeof(r));
  }
  return r;
}
// Behind element-wise stores: the compiler would make one store of the last of them and the vector store's last element, and cut
// the vector store up for it (fp32 RMS norm of 4096 x 4091 36.3 us, 28.7).
__device__ __forceinline__ void apart() { asm volatile("" ::: "memory"); }
template <class T, RowEnd END>
__device__ __forceinline__ void store8(T* row, const Cols<END>& k, const float (&x)[8]) {
  T e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = (T)x[i];
  if (k.skip == 0) {
    __builtin_memcpy(row + k.c, e, sizeof(e));
  } else if (END != WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k.own(i)) row[k.c + i] = e[i];
    apart();
  }
}

// x of another lane of the same 16, by a DPP control: 0xB1 lane ^ 1, 0x4E lane ^ 2, 0x141 mirrored in 8, 0x140 in 16
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float max16(float x) {   // over aligned groups of 16 lanes
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  x = fmaxf(x, dpp<0x141>(x));
  return fmaxf(x, dpp<0x140>(x));
}
__device__ __forceinline__ float sum64(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  x += dpp<0x141>(x);
  x += dpp<0x140>(x);
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The scale of a block whose largest magnitude is amax.  Activations: rounded to bf16 (a scale rounded down leaves at most
// 449.75 for a code, which rounds to 448), half the bytes and the same scale whatever the last bits of a sum were.
__device__ __forceinline__ float weight_scale_of(float amax) { return fmaxf(amax * (1.f / F8_LARGEST), F8_SMALLEST_SCALE); }
__device__ __forceinline__ __bf16 scale_of(float amax) { return (__bf16)weight_scale_of(amax); }
// four values, already divided by their scale, as e4m3 codes, round to nearest even
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Codes of a lane's own columns (rows of codes 16-byte aligned)
template <RowEnd END>
__device__ __forceinline__ void store_codes8(unsigned char* row, const Cols<END>& k, const float (&x)[8], float inv) {
  u32x2 w;
  w[0] = codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  w[1] = codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
  if (k.skip == 0) {
    *(u32x2*)(row + k.c) = w;
  } else if (END != WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k.own(i)) row[k.c + i] = (unsigned char)(w[i / 4] >> (8 * (i % 4)));
    apart();
  }
}
#endif

}  // namespace svdmlp
