// What the layer operators share (layer.cu, layer_gather*, layer_sample.cu, layer_slope.cu): value types, activations, the
// row view of a matrix. A layer is Z = A.B + bias, C = f(Z) + residual, with A sparse and everything else dense and row-major.
// Internal: not part of the C ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace comet {

// A matrix by rows: row i holds the entries pos[i] .. pos[i+1].
struct RowView {
  const int32_t *pos, *crd;
  const void *val;
  int64_t rows, cols, nnz;
};

// The products' arithmetic. `acc`: products and short sums; `sum`: what the short sums (at most 128 terms) are added to. fp32
// keeps 128-term sums in fp32 and adds them in double, so that a row of any length stays within 128 * 2^-24 of the sum of
// its terms' magnitudes; 16-bit results are rounded to 2^-9 or 2^-12 anyway and take fp32 for both.
template <class T> struct Num;
template <> struct Num<double> { using acc = double; using sum = double; };
template <> struct Num<float> { using acc = float; using sum = double; };
template <> struct Num<__nv_bfloat16> { using acc = float; using sum = float; };
template <> struct Num<__half> { using acc = float; using sum = float; };

__device__ __forceinline__ double widen(double x) { return x; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

// One rounding from the wide type (the 16-bit types come from fp32).
template <class T, class W> __device__ __forceinline__ T narrow(W x) { return (T)x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16, float>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half narrow<__half, float>(float x) { return __float2half_rn(x); }

// 16 bytes of a row as wide values, and back.
template <class T> struct Piece {
  static constexpr int kValues = 16 / sizeof(T);
  union { uint4 raw; T at[kValues]; };
  __device__ __forceinline__ Piece() {}
};

// ---- activations and their slopes, in the wide type (fp32 or fp64)
__device__ __forceinline__ float f_exp(float x) { return expf(x); }
__device__ __forceinline__ double f_exp(double x) { return exp(x); }
__device__ __forceinline__ float f_erf(float x) { return erff(x); }
__device__ __forceinline__ double f_erf(double x) { return erf(x); }
__device__ __forceinline__ float f_tanh(float x) { return tanhf(x); }
__device__ __forceinline__ double f_tanh(double x) { return tanh(x); }

constexpr double kSqrtHalf = 0.70710678118654752440, kSqrtTwoOverPi = 0.79788456080286535588, kInvSqrtTwoPi = 0.39894228040143267794;
constexpr double kGeluCubic = 0.044715;

template <class W> __device__ __forceinline__ W activate(int act, W z) {
  switch (act) {
    case COMET_ACT_RELU: return z > (W)0 ? z : (z == z ? (W)0 : z);                   // NaN stays NaN
    case COMET_ACT_GELU: return (W)0.5 * z * ((W)1 + f_erf(z * (W)kSqrtHalf));
    case COMET_ACT_GELU_TANH: return (W)0.5 * z * ((W)1 + f_tanh((W)kSqrtTwoOverPi * (z + (W)kGeluCubic * z * z * z)));
    case COMET_ACT_SILU: return z / ((W)1 + f_exp(-z));
    default: return z;
  }
}

template <class W> __device__ __forceinline__ W activate_slope(int act, W z) {
  switch (act) {
    case COMET_ACT_RELU: return z > (W)0 ? (W)1 : (W)0;
    case COMET_ACT_GELU: return (W)0.5 * ((W)1 + f_erf(z * (W)kSqrtHalf)) + z * f_exp((W)-0.5 * z * z) * (W)kInvSqrtTwoPi;
    case COMET_ACT_GELU_TANH: {
      const W t = f_tanh((W)kSqrtTwoOverPi * (z + (W)kGeluCubic * z * z * z));
      const W rise = (W)kSqrtTwoOverPi * ((W)1 + (W)(3 * kGeluCubic) * z * z);
      return (W)0.5 * ((W)1 + t) + ((W)1 - t * t == (W)0 ? (W)0 : (W)0.5 * z * ((W)1 - t * t) * rise);
    }
    case COMET_ACT_SILU: {
      const W g = (W)1 / ((W)1 + f_exp(-z));
      return g * ((W)1 + z * ((W)1 - g));
    }
    default: return (W)1;
  }
}

// ---- launchers

// One of the up to two products of a call: its matrix, its dense operand, and, for its own pre-activation, bias and place to keep it.
struct GatherSource {
  RowView A;
  const void *B;
  int64_t ldb;
  const void *bias;        // NULL: none
  void *pre;               // NULL: not kept
};
enum GatherMode { kLayer, kGated, kSumOfTwo };   // f(Z) + residual; f(Z0) * Z1; Z0 + Z1 (no bias, no activation)
struct GatherCall {
  GatherMode mode;
  GatherSource src[2];     // kLayer uses the first only
  int64_t R;
  int act, bias_along;
  const void *residual;
  int64_t ldr, ldz;
  void *C;
  int64_t ldc;
};
comet_status_t layer_gather(Context *ctx, int dtype, const GatherCall &call, cudaStream_t s);

// out[p] = sum over r of P[row of p, r] * Q[crd[p], r]
comet_status_t layer_sample(Context *ctx, int dtype, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R,
                            void *out, cudaStream_t s);

// Gradients of the pre-activations and of the biases. One source: dz0 = dC * f'(z0). Two: dz0 = dC * z1 * f'(z0), dz1 = dC * f(z0).
// dz* (rows x R, contiguous) and bias* may be NULL.
struct SlopeCall {
  int64_t rows, R;
  int act, bias_along, sources;
  const void *dC;
  int64_t lddc;
  const void *z[2];
  int64_t ldz;
  void *dz[2], *bias[2];
};
comet_status_t layer_slope(Context *ctx, int dtype, const SlopeCall &call, cudaStream_t s);

// out[p] = val[index[p]] for the transposed matrix's entries
comet_status_t layer_pick(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, void *out, cudaStream_t s);

inline size_t layer_elem_size(int dtype) { return dtype == COMET_F64 ? 8 : dtype == COMET_F32 ? 4 : 2; }
inline bool layer_dtype(int dtype) { return dtype >= COMET_F64 && dtype <= COMET_F16; }

}  // namespace comet
