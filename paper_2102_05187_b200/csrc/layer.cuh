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
  bool ordered;            // a row's columns ascend and are distinct (compressed levels); of a caller's [CN,S] nothing is known about them
};

// The products' arithmetic. `acc`: products and short sums; `sum`: what the short sums (at most 128 terms) are added to. fp32
// keeps 128-term sums in fp32 and adds them in double, so that a row of any length stays within 128 * 2^-24 of the sum of
// its terms' magnitudes; 16-bit results are rounded to 2^-9 or 2^-12 anyway and take fp32 for both.
template <class T> struct Num;
template <> struct Num<double> { using acc = double; using sum = double; };
template <> struct Num<float> { using acc = float; using sum = double; };
template <> struct Num<__nv_bfloat16> { using acc = float; using sum = float; static constexpr bool is_bf16 = true; };
template <> struct Num<__half> { using acc = float; using sum = float; static constexpr bool is_bf16 = false; };

__device__ __forceinline__ double widen(double x) { return x; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

// One rounding from the wide type (the 16-bit types come from fp32).
template <class T, class W> __device__ __forceinline__ T narrow(W x) { return (T)x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16, float>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half narrow<__half, float>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ uint32_t narrow2(float low, float high, __nv_bfloat16) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(low, high);
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ uint32_t narrow2(float low, float high, __half) {
  const __half2 x = __floats2half2_rn(low, high);
  return *reinterpret_cast<const uint32_t *>(&x);
}

// 16 bytes of a row.
template <class T> struct Piece {
  static constexpr int kValues = 16 / sizeof(T);
  union { uint4 raw; T at[kValues]; };
  __device__ __forceinline__ Piece() {}
};

// N neighbouring values read or written at once (2 to 16 bytes, aligned to their size).
template <int Bytes> struct Word;
template <> struct Word<2> { using type = unsigned short; };
template <> struct Word<4> { using type = unsigned int; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };
template <class T, int N> struct Values {
  using word = typename Word<(int)sizeof(T) * N>::type;
  union { word raw; T at[N]; };
  __device__ __forceinline__ Values() {}
  __device__ __forceinline__ void read(const T *p) { raw = __ldcs(reinterpret_cast<const word *>(p)); }
  __device__ __forceinline__ void write(T *p) const { *reinterpret_cast<word *>(p) = raw; }
};

// ---- activations and their slopes, in the wide type (fp32 or fp64). Fast: for results that are rounded to 16 bits, exp and the quotient from the
// special function unit (relative errors of 2^-21 or so).
template <bool Fast> __device__ __forceinline__ float f_exp(float x) { return Fast ? __expf(x) : expf(x); }
template <bool Fast> __device__ __forceinline__ double f_exp(double x) { return exp(x); }
__device__ __forceinline__ float f_erf(float x) { return erff(x); }
__device__ __forceinline__ double f_erf(double x) { return erf(x); }
template <bool Fast> __device__ __forceinline__ float f_quotient(float x, float y) { return Fast ? __fdividef(x, y) : x / y; }
template <bool Fast> __device__ __forceinline__ double f_quotient(double x, double y) { return x / y; }

constexpr double kSqrtHalf = 0.70710678118654752440, kSqrtTwoOverPi = 0.79788456080286535588, kInvSqrtTwoPi = 0.39894228040143267794;
constexpr double kGeluCubic = 0.044715;

// 1 / (1 + exp(-x)) as (s, 1 - s), both to full relative accuracy: the exponential is taken of -|x|, which neither overflows nor cancels.
template <bool Fast, class W> __device__ __forceinline__ void logistic(W x, W &s, W &rest) {
  const W e = f_exp<Fast>(x > (W)0 ? -x : x), big = f_quotient<Fast>((W)1, (W)1 + e), small = e * big;
  s = x > (W)0 ? big : small;
  rest = x > (W)0 ? small : big;
}

template <bool Fast, class W> __device__ __forceinline__ W activate(int act, W z) {
  W s, rest;
  switch (act) {
    case COMET_ACT_RELU: return z > (W)0 ? z : (z == z ? (W)0 : z);                   // NaN stays NaN
    case COMET_ACT_GELU: return (W)0.5 * z * ((W)1 + f_erf(z * (W)kSqrtHalf));
    case COMET_ACT_GELU_TANH:                                                         // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
      logistic<Fast>((W)(2 * kSqrtTwoOverPi) * (z + (W)kGeluCubic * z * z * z), s, rest);
      return z * s;
    case COMET_ACT_SILU:
      logistic<Fast>(z, s, rest);
      return z * s;
    default: return z;
  }
}

// The same on N values: what is chosen by `act` is chosen once.
template <bool Fast, int N, class W> __device__ __forceinline__ void activate_all(int act, W (&z)[N]) {
  if (act == COMET_ACT_NONE) return;
  if (act == COMET_ACT_RELU) {
#pragma unroll
    for (int v = 0; v < N; ++v) z[v] = activate<Fast>(COMET_ACT_RELU, z[v]);
  } else if (act == COMET_ACT_GELU) {
#pragma unroll
    for (int v = 0; v < N; ++v) z[v] = activate<Fast>(COMET_ACT_GELU, z[v]);
  } else if (act == COMET_ACT_GELU_TANH) {
#pragma unroll
    for (int v = 0; v < N; ++v) z[v] = activate<Fast>(COMET_ACT_GELU_TANH, z[v]);
  } else {
#pragma unroll
    for (int v = 0; v < N; ++v) z[v] = activate<Fast>(COMET_ACT_SILU, z[v]);
  }
}

template <bool Fast, class W> __device__ __forceinline__ W activate_slope(int act, W z) {
  W s, rest;
  switch (act) {
    case COMET_ACT_RELU: return z > (W)0 ? (W)1 : (W)0;
    case COMET_ACT_GELU: return (W)0.5 * ((W)1 + f_erf(z * (W)kSqrtHalf)) + z * f_exp<Fast>((W)-0.5 * z * z) * (W)kInvSqrtTwoPi;
    case COMET_ACT_GELU_TANH: {
      logistic<Fast>((W)(2 * kSqrtTwoOverPi) * (z + (W)kGeluCubic * z * z * z), s, rest);
      const W bend = s * rest;
      return s + (bend == (W)0 ? (W)0 : z * bend * (W)(2 * kSqrtTwoOverPi) * ((W)1 + (W)(3 * kGeluCubic) * z * z));
    }
    case COMET_ACT_SILU:
      logistic<Fast>(z, s, rest);
      return s * ((W)1 + z * rest);
    default: return (W)1;
  }
}

// ---- launchers
inline size_t layer_elem_size(int dtype) { return dtype == COMET_F64 ? 8 : dtype == COMET_F32 ? 4 : 2; }
inline bool layer_dtype(int dtype) { return dtype >= COMET_F64 && dtype <= COMET_F16; }
inline bool layer_aligned(int dtype, const void *p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && ld * (int64_t)layer_elem_size(dtype) % 16 == 0); }

// One of the up to two products of a call: its matrix, its dense operand, and, for its own pre-activation, bias and place to keep it.
struct GatherSource {
  RowView A;
  const int32_t *pick;     // entry p's value is val[pick[p]]; NULL: val[p]. Tensor-core form only: the others get values in order
  const void *B;
  int64_t ldb;
  const void *bias;        // NULL: none
  void *pre;               // NULL: not kept
};
enum GatherMode { kLayer, kGated, kSumOfTwo };   // f(Z) + residual; f(Z0) * Z1; Z0 + Z1 (no bias, no activation)
constexpr int kPanelSmem = 200 * 1024;         // most shared memory of a panel of B's rows (layer_panel.cuh)
// Rows of so many bytes that a panel holds beside the row of zeros, in steps of 16.
constexpr int panel_capacity(int row_bytes) { return (kPanelSmem / row_bytes - 1) / 16 * 16; }

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

constexpr int kLayerStatusWord = 63;           // of Context::h_pinned: set by a tensor-core kernel that gave up (layer_tile.cuh), read by the next layer call
int64_t wait_patience();                       // cycles that a wait of those kernels may take

// out[p] = sum over r of P[row of p, r] * Q[crd[p], r]
comet_status_t layer_sample(Context *ctx, int dtype, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R,
                            void *out, cudaStream_t s);

// A matrix's entries by tiles of 128 x 64 (layer_tile_list.cu; its rows have to be ordered): words of tile (t, b) at words + bases[t * (blocks + 1) + b] up to the next base.
struct TileList { const uint32_t *words; const int32_t *bases; };
bool tile_lists_fit(const RowView &A);
size_t tile_list_bytes(const RowView &A);
comet_status_t tile_lists(Context *ctx, const RowView *A, const int32_t *const *pick, int sources, char *const *mem, TileList *lists, cudaStream_t s);

// The same two on the tensor cores (layer_tile_product.cu, layer_tile_sample.cu), and whether a call is one for them.
bool tile_product_fits(int dtype, const GatherCall &call);
comet_status_t tile_product(Context *ctx, int dtype, const GatherCall &call, const TileList *lists, cudaStream_t s);
// (These two want dense operands that start on 16 bytes with rows that are a whole number of 16 bytes apart.)
bool tile_sample_fits(int dtype, const RowView &A, int64_t R);
comet_status_t tile_sample(Context *ctx, int dtype, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R, void *out,
                           cudaStream_t s);

// Gradients of the pre-activations and of the biases. One source: dz0 = dC * f'(z0). Two: dz0 = dC * z1 * f'(z0), dz1 = dC * f(z0).
// dz* (rows x R, leading dimension lddz) and bias* may be NULL.
struct SlopeCall {
  int64_t rows, R;
  int act, bias_along, sources;
  const void *dC;
  int64_t lddc;
  const void *z[2];
  int64_t ldz;
  void *dz[2], *bias[2];
  int64_t lddz;
};
comet_status_t layer_slope(Context *ctx, int dtype, const SlopeCall &call, cudaStream_t s);

// The epilogue on products that are there already (rows x R each, fp64 for COMET_F64, else fp32): one source z0 gives f(z0 + bias0) + residual, two give f(z0 + bias0) * (z1 + bias1),
// or, `sum`, z0 + z1. Pre-activations of fp64 and fp32 may be kept where they are read.
struct FinishCall {
  int64_t rows, R;
  int act, bias_along, sources;
  bool sum;
  const void *z[2];
  int64_t ldzin;
  const void *bias[2];
  void *pre[2];
  int64_t ldz;
  const void *residual;
  int64_t ldr;
  void *C;
  int64_t ldc;
};
comet_status_t layer_finish(Context *ctx, int dtype, const FinishCall &call, cudaStream_t s);

// A copy of a rows x R matrix with rows layer_padded values apart (the padding is not written): a whole number of 16 bytes, of 128 where the
// tensor-core forms take 16-bit rows of 64 values and more (a tile's row is then one line).
inline int64_t layer_padded(int dtype, int64_t R) {
  const int64_t v = dtype == COMET_F64 ? 2 : dtype == COMET_F32 ? 4 : R > 32 ? 64 : 8;
  return (R + v - 1) / v * v;
}
comet_status_t layer_pad(Context *ctx, int dtype, const void *in, int64_t rows, int64_t R, int64_t ld, void *out, cudaStream_t s);

// 16-bit values as fp32: a rows x R matrix with rows layer_padded(COMET_F32, R) values apart; n values, by number where index is not NULL.
comet_status_t layer_widen(Context *ctx, int dtype, const void *in, int64_t rows, int64_t R, int64_t ld, float *out, cudaStream_t s);
comet_status_t layer_widen_values(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, float *out, cudaStream_t s);

// out[p] = val[index[p]] for the transposed matrix's entries
comet_status_t layer_pick(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, void *out, cudaStream_t s);


}  // namespace comet
