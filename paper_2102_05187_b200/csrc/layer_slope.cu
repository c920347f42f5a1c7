// Gradients of the pre-activations and of the biases of a layer, and the pass that picks a transposed matrix's values.
//
//   one source:   dz0 = dC * f'(z0)                          two (gated):  dz0 = dC * z1 * f'(z0),  dz1 = dC * f(z0)
//   bias along the rows: sum of dz over r;  along the columns: sum of dz over i
//
// One pass over dC and the kept pre-activations writes dz and the sums: bound by memory. A warp per row, 32 (or, with 16-byte pieces,
// 32 * 16 / size) columns a round, joins the row's sum by shuffles; a column's sum is taken over blocks of rows first and the blocks are added by a
// second launch in their order. Sums are held in fp32 within a lane (at most 64 terms) and in double beyond, and are taken of the
// slopes before dz is rounded to its type.
#include "kernels.cuh"
#include "layer.cuh"

namespace comet {
namespace {

constexpr int kSlopeThreads = 256;

template <class T> struct SlopeArgs {
  const T *dC, *z[2];
  T *dz[2];
  T *row_bias[2];
  int64_t rows, R, lddc, ldz, lddz;
  int act, sources;
};

template <class T> __device__ __forceinline__ void slopes(const SlopeArgs<T> &a, typename Num<T>::acc g, typename Num<T>::acc z0, typename Num<T>::acc z1,
                                                          typename Num<T>::acc (&d)[2]) {
  if (a.sources == 1) {
    d[0] = a.act == COMET_ACT_NONE ? g : g * activate_slope<sizeof(T) == 2>(a.act, z0);
  } else {
    d[0] = a.act == COMET_ACT_NONE ? g * z1 : g * z1 * activate_slope<sizeof(T) == 2>(a.act, z0);
    d[1] = g * activate<sizeof(T) == 2>(a.act, z0);
  }
}

template <class T, int V> __global__ void __launch_bounds__(kSlopeThreads) layer_slope_kernel(const SlopeArgs<T> a) {
  using acc_t = typename Num<T>::acc;
  const int lane = threadIdx.x & 31;
  const int64_t step = (int64_t)gridDim.x * (kSlopeThreads / 32);
  for (int64_t i = (int64_t)blockIdx.x * (kSlopeThreads / 32) + (threadIdx.x >> 5); i < a.rows; i += step) {
    double sum[2] = {0.0, 0.0};
    for (int64_t col = (int64_t)lane * V; col < a.R; col += 32 * V) {
      Piece<T> g, z[2], out[2];
      const bool full = V > 1 && col + V <= a.R;
      if (full) {
        g.raw = __ldcs(reinterpret_cast<const uint4 *>(a.dC + i * a.lddc + col));
        if (a.z[0]) z[0].raw = __ldcs(reinterpret_cast<const uint4 *>(a.z[0] + i * a.ldz + col));
        if (a.sources == 2) z[1].raw = __ldcs(reinterpret_cast<const uint4 *>(a.z[1] + i * a.ldz + col));
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (col + v >= a.R) continue;
          g.at[v] = a.dC[i * a.lddc + col + v];
          if (a.z[0]) z[0].at[v] = a.z[0][i * a.ldz + col + v];
          if (a.sources == 2) z[1].at[v] = a.z[1][i * a.ldz + col + v];
        }
      }
      acc_t part[2] = {(acc_t)0, (acc_t)0};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!full && col + v >= a.R) continue;
        acc_t d[2] = {(acc_t)0, (acc_t)0};
        slopes(a, widen(g.at[v]), a.z[0] ? widen(z[0].at[v]) : (acc_t)0, a.sources == 2 ? widen(z[1].at[v]) : (acc_t)0, d);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          part[q] += d[q];
          out[q].at[v] = narrow<T, acc_t>(d[q]);
        }
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (q >= a.sources) continue;
        sum[q] += (double)part[q];
        if (!a.dz[q]) continue;
        T *to = a.dz[q] + i * a.lddz + col;
        if (full) *reinterpret_cast<uint4 *>(to) = out[q].raw;
        else {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (col + v < a.R) to[v] = out[q].at[v];
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (q >= a.sources || !a.row_bias[q]) continue;
      for (int off = 16; off >= 1; off >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], off);
      if (lane == 0) a.row_bias[q][i] = narrow<T, acc_t>((acc_t)sum[q]);
    }
  }
}

// part[block of rows, r] = the block's column sums (source 0): a thread per column
template <class T> __global__ void __launch_bounds__(kSlopeThreads) column_sums_kernel(const SlopeArgs<T> a, int64_t rows_per_block, double *__restrict__ part) {
  using acc_t = typename Num<T>::acc;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ double joined[kSlopeThreads / 32][33];
  const int64_t col = (int64_t)blockIdx.y * 32 + lane;
  const int64_t from = (int64_t)blockIdx.x * rows_per_block, to = min(a.rows, from + rows_per_block);
  double sum = 0.0;
  if (col < a.R) {
#pragma unroll 4
    for (int64_t i = from + warp; i < to; i += kSlopeThreads / 32) {
      acc_t d[2];
      slopes(a, widen(a.dC[i * a.lddc + col]), a.z[0] ? widen(a.z[0][i * a.ldz + col]) : (acc_t)0, (acc_t)0, d);
      sum += (double)d[0];
    }
  }
  joined[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && col < a.R) {
    for (int w = 1; w < kSlopeThreads / 32; ++w) sum += joined[w][lane];
    part[(int64_t)blockIdx.x * a.R + col] = sum;
  }
}

template <class T> __global__ void __launch_bounds__(kSlopeThreads) column_join_kernel(const double *__restrict__ part, int64_t blocks, int64_t R, T *__restrict__ out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ double joined[kSlopeThreads / 32][33];
  const int64_t col = (int64_t)blockIdx.x * 32 + lane;
  double sum = 0.0;
  if (col < R)
    for (int64_t b = warp; b < blocks; b += kSlopeThreads / 32) sum += part[b * R + col];
  joined[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && col < R) {
    for (int w = 1; w < kSlopeThreads / 32; ++w) sum += joined[w][lane];
    out[col] = narrow<T, typename Num<T>::acc>((typename Num<T>::acc)sum);
  }
}

template <class T> comet_status_t slope_typed(Context *ctx, const SlopeCall &c, cudaStream_t s) {
  SlopeArgs<T> a{};
  a.dC = (const T *)c.dC;
  a.rows = c.rows; a.R = c.R; a.lddc = c.lddc; a.ldz = c.ldz; a.lddz = c.lddz;
  a.act = c.act; a.sources = c.sources;
  constexpr int V = 16 / sizeof(T);
  const auto ok = [](const void *p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && (ld * (int64_t)sizeof(T)) % 16 == 0); };
  bool vec = c.R >= V && ok(c.dC, c.lddc), rows_pass = false;
  for (int q = 0; q < c.sources; ++q) {
    a.z[q] = (const T *)c.z[q];
    a.dz[q] = (T *)c.dz[q];
    if (c.bias_along == COMET_BIAS_ROWS) a.row_bias[q] = (T *)c.bias[q];
    vec = vec && ok(c.z[q], c.ldz) && ok(c.dz[q], c.lddz);
    rows_pass = rows_pass || a.dz[q] || a.row_bias[q];
  }
  if (rows_pass) {
    const int64_t blocks = ceil_div(c.rows, kSlopeThreads / 32);
    const unsigned grid = (unsigned)(blocks < 16 * kSmCount ? blocks : 16 * kSmCount);
    if (vec) layer_slope_kernel<T, V><<<grid, kSlopeThreads, 0, s>>>(a);
    else layer_slope_kernel<T, 1><<<grid, kSlopeThreads, 0, s>>>(a);
    COMET_LAUNCH_CHECK(ctx);
  }
  if (c.bias_along == COMET_BIAS_COLS && c.bias[0]) {
    int64_t blocks = ceil_div(c.rows, 64);
    const int64_t most = 8 * kSmCount;
    if (blocks > most) blocks = most;
    const int64_t per = ceil_div(c.rows, blocks);
    blocks = ceil_div(c.rows, per);
    double *part = (double *)ctx_alloc(ctx, (size_t)blocks * (size_t)c.R * sizeof(double), s);
    if (!part) return COMET_ERR_ALLOC;
    cudaError_t e = cudaSuccess;
    for (int64_t first = 0; first < c.R && e == cudaSuccess; first += 65535 * 32) {       // blockIdx.y counts 32 columns
      SlopeArgs<T> b = a;
      b.dC += first;
      if (b.z[0]) b.z[0] += first;
      b.R = c.R - first < 65535 * 32 ? c.R - first : 65535 * 32;
      column_sums_kernel<T><<<dim3((unsigned)blocks, (unsigned)ceil_div(b.R, 32)), kSlopeThreads, 0, s>>>(b, per, part);
      column_join_kernel<T><<<(unsigned)ceil_div(b.R, 32), kSlopeThreads, 0, s>>>(part, blocks, b.R, (T *)c.bias[0] + first);
      ctx->launches += 2;
      e = cudaGetLastError();
    }
    ctx_free(ctx, part, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
  }
  return COMET_OK;
}

template <class V> __global__ void __launch_bounds__(kBlockThreads) layer_pick_kernel(const V *__restrict__ val, const int32_t *__restrict__ index, int64_t n,
                                                                                      V *__restrict__ out) {
  const int64_t p = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x;
  if (p < n) out[p] = __ldg(val + ld_stream(index + p));
}

// A warp per row and run of 1,024 values.
template <class V> __global__ void __launch_bounds__(kBlockThreads) layer_pad_kernel(const V *__restrict__ in, int64_t rows, int64_t R, int64_t ld, int64_t ldo,
                                                                                     V *__restrict__ out) {
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * (kBlockThreads / 32) + (threadIdx.x >> 5);
  if (i >= rows) return;
  for (int64_t first = (int64_t)blockIdx.y * 1024; first < R; first += (int64_t)gridDim.y * 1024) {
    const V *from = in + i * ld;
    V *to = out + i * ldo;
#pragma unroll 8
    for (int64_t col = first + lane; col < min(R, first + 1024); col += 32) to[col] = __ldg(from + col);
  }
}

}  // namespace

comet_status_t layer_pad(Context *ctx, int dtype, const void *in, int64_t rows, int64_t R, int64_t ld, void *out, cudaStream_t s) {
  if (rows == 0) return COMET_OK;
  const int64_t runs = ceil_div(R, 1024);
  const dim3 grid((unsigned)ceil_div(rows, kBlockThreads / 32), (unsigned)(runs < 65535 ? runs : 65535));
  const int64_t ldo = layer_padded(dtype, R);
  switch (layer_elem_size(dtype)) {
    case 8: layer_pad_kernel<<<grid, kBlockThreads, 0, s>>>((const unsigned long long *)in, rows, R, ld, ldo, (unsigned long long *)out); break;
    case 4: layer_pad_kernel<<<grid, kBlockThreads, 0, s>>>((const unsigned int *)in, rows, R, ld, ldo, (unsigned int *)out); break;
    default: layer_pad_kernel<<<grid, kBlockThreads, 0, s>>>((const unsigned short *)in, rows, R, ld, ldo, (unsigned short *)out);
  }
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

comet_status_t layer_slope(Context *ctx, int dtype, const SlopeCall &c, cudaStream_t s) {
  if (c.rows == 0) {                                       // no row: a column's sum is empty
    if (c.bias_along == COMET_BIAS_COLS && c.bias[0]) COMET_CUDA_TRY(ctx, cudaMemsetAsync(c.bias[0], 0, (size_t)c.R * layer_elem_size(dtype), s));
    return COMET_OK;
  }
  switch (dtype) {
    case COMET_F64: return slope_typed<double>(ctx, c, s);
    case COMET_F32: return slope_typed<float>(ctx, c, s);
    case COMET_BF16: return slope_typed<__nv_bfloat16>(ctx, c, s);
    default: return slope_typed<__half>(ctx, c, s);
  }
}

comet_status_t layer_pick(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, void *out, cudaStream_t s) {
  if (n == 0) return COMET_OK;
  const unsigned blocks = (unsigned)ceil_div(n, kBlockThreads);
  switch (layer_elem_size(dtype)) {
    case 8: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned long long *)val, index, n, (unsigned long long *)out); break;
    case 4: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned int *)val, index, n, (unsigned int *)out); break;
    default: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned short *)val, index, n, (unsigned short *)out);
  }
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

}  // namespace comet
