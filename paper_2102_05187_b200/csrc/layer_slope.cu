// Gradients of the pre-activations and of the biases of a layer, and the pass that picks a transposed matrix's values.
//
//   one source:   dz0 = dC * f'(z0)                          two (gated):  dz0 = dC * z1 * f'(z0),  dz1 = dC * f(z0)
//   bias along the rows: sum of dz over r;  along the columns: sum of dz over i
//
// One pass over dC and the kept pre-activations writes dz and the sums: bound by memory. As many lanes to a row as it needs, up to
// 32, with the widest pieces that all operands' rows are aligned to, join the row's sum by shuffles; a column's sum is taken over blocks of rows first and the blocks are added by a
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

__device__ __forceinline__ int64_t ceil_to(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

template <class T> __device__ __forceinline__ void slopes(const SlopeArgs<T> &a, typename Num<T>::acc g, typename Num<T>::acc z0, typename Num<T>::acc z1,
                                                          typename Num<T>::acc (&d)[2]) {
  if (a.sources == 1) {
    d[0] = a.act == COMET_ACT_NONE ? g : g * activate_slope<sizeof(T) == 2>(a.act, z0);
  } else {
    d[0] = a.act == COMET_ACT_NONE ? g * z1 : g * z1 * activate_slope<sizeof(T) == 2>(a.act, z0);
    d[1] = g * activate<sizeof(T) == 2>(a.act, z0);
  }
}

// `lanes` (a power of two) to a row, V values a lane and round.
template <class T, int V> __global__ void __launch_bounds__(kSlopeThreads) layer_slope_kernel(const SlopeArgs<T> a, int lanes) {
  using acc_t = typename Num<T>::acc;
  const int l = threadIdx.x & (lanes - 1), each = kSlopeThreads / lanes;
  const int64_t step = (int64_t)gridDim.x * each, last = ceil_to(a.rows, each);
  for (int64_t i = (int64_t)blockIdx.x * each + threadIdx.x / lanes; i < last; i += step) {           // whole warps go on together
    double sum[2] = {0.0, 0.0};
    for (int64_t col = (int64_t)l * V; col < a.R && i < a.rows; col += (int64_t)lanes * V) {
      Values<T, V> g, z[2], out[2];
      const bool full = V == 1 || col + V <= a.R;
      if (full) {
        g.read(a.dC + i * a.lddc + col);
        if (a.z[0]) z[0].read(a.z[0] + i * a.ldz + col);
        if (a.sources == 2) z[1].read(a.z[1] + i * a.ldz + col);
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
        if (full) out[q].write(to);
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
      for (int off = lanes / 2; off >= 1; off >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], off);
      if (l == 0 && i < a.rows) a.row_bias[q][i] = narrow<T, acc_t>((acc_t)sum[q]);
    }
  }
}

// Z: the products' type.
template <class T> struct FinishArgs {
  using Z = typename Num<T>::acc;
  const Z *z[2];
  const T *bias[2], *res;
  T *pre[2], *C;
  int64_t rows, R, ldzin, ldz, ldr, ldc;
  int act, bias_along, sources;
  bool sum;
};

template <class T, int V> __global__ void __launch_bounds__(kSlopeThreads) layer_finish_kernel(const FinishArgs<T> a, int lanes) {
  using acc_t = typename Num<T>::acc;
  const int l = threadIdx.x & (lanes - 1), each = kSlopeThreads / lanes;
  const int64_t step = (int64_t)gridDim.x * each;
  for (int64_t i = (int64_t)blockIdx.x * each + threadIdx.x / lanes; i < a.rows; i += step) {
    for (int64_t col = (int64_t)l * V; col < a.R; col += (int64_t)lanes * V) {
      Values<T, V> r, keep[2], out;
      acc_t x[2][V];
      const bool full = V == 1 || col + V <= a.R;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (q >= a.sources) continue;
        constexpr int kAtOnce = V * (int)sizeof(acc_t) <= 16 ? V : 16 / (int)sizeof(acc_t);
        if (full) {
#pragma unroll
          for (int v = 0; v < V; v += kAtOnce) {
            Values<acc_t, kAtOnce> y;
            y.read(a.z[q] + i * a.ldzin + col + v);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) x[q][v + k] = y.at[k];
          }
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) x[q][v] = col + v < a.R ? a.z[q][i * a.ldzin + col + v] : (acc_t)0;
        }
      }
      if (full) {
        if (a.res) r.read(a.res + i * a.ldr + col);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (col + v >= a.R) continue;
          if (a.res) r.at[v] = a.res[i * a.ldr + col + v];
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!full && col + v >= a.R) continue;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          if (q >= a.sources) continue;
          if (a.bias[q]) x[q][v] += widen(a.bias[q][a.bias_along == COMET_BIAS_ROWS ? i : col + v]);
          keep[q].at[v] = narrow<T, acc_t>(x[q][v]);
        }
        acc_t y = a.sum ? x[0][v] + x[1][v] : activate<sizeof(T) == 2>(a.act, x[0][v]);
        if (a.sources == 2 && !a.sum) y *= x[1][v];
        if (a.res) y += widen(r.at[v]);
        out.at[v] = narrow<T, acc_t>(y);
      }
      if (full) {
        out.write(a.C + i * a.ldc + col);
#pragma unroll
        for (int q = 0; q < 2; ++q)
          if (a.pre[q]) keep[q].write(a.pre[q] + i * a.ldz + col);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (col + v >= a.R) continue;
          a.C[i * a.ldc + col + v] = out.at[v];
#pragma unroll
          for (int q = 0; q < 2; ++q)
            if (a.pre[q]) a.pre[q][i * a.ldz + col + v] = keep[q].at[v];
        }
      }
    }
  }
}

// Values that can be moved at once from every row of an operand: as many as its alignment and that of its rows allow, 16 bytes at most.
template <class T> int widest(const void *p, int64_t ld) {
  int bytes = 16;
  if (p)
    while (bytes > (int)sizeof(T) && (((uintptr_t)p | (uintptr_t)(ld * (int64_t)sizeof(T))) & (uintptr_t)(bytes - 1))) bytes /= 2;
  return bytes / (int)sizeof(T);
}
inline int lanes_for(int64_t R, int V) {
  int lanes = 1;
  while (lanes < 32 && (int64_t)lanes * V < R) lanes *= 2;
  return lanes;
}
template <class T> unsigned row_grid(int64_t rows, int lanes) {
  const int64_t blocks = ceil_div(rows, kSlopeThreads / lanes);
  return (unsigned)(blocks < 16 * kSmCount ? blocks : 16 * kSmCount);
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
#pragma unroll 8
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

constexpr int kJoinThreads = 1024;
template <class T> __global__ void __launch_bounds__(kJoinThreads) column_join_kernel(const double *__restrict__ part, int64_t blocks, int64_t R, T *__restrict__ out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ double joined[kJoinThreads / 32][33];
  const int64_t col = (int64_t)blockIdx.x * 32 + lane;
  double sum = 0.0;
  if (col < R) {
#pragma unroll 8
    for (int64_t b = warp; b < blocks; b += kJoinThreads / 32) sum += part[b * R + col];
  }
  joined[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && col < R) {
    for (int w = 1; w < kJoinThreads / 32; ++w) sum += joined[w][lane];
    out[col] = narrow<T, typename Num<T>::acc>((typename Num<T>::acc)sum);
  }
}

template <class T> comet_status_t slope_typed(Context *ctx, const SlopeCall &c, cudaStream_t s) {
  SlopeArgs<T> a{};
  a.dC = (const T *)c.dC;
  a.rows = c.rows; a.R = c.R; a.lddc = c.lddc; a.ldz = c.ldz; a.lddz = c.lddz;
  a.act = c.act; a.sources = c.sources;
  int V = widest<T>(c.dC, c.lddc);
  bool rows_pass = false;
  for (int q = 0; q < c.sources; ++q) {
    a.z[q] = (const T *)c.z[q];
    a.dz[q] = (T *)c.dz[q];
    if (c.bias_along == COMET_BIAS_ROWS) a.row_bias[q] = (T *)c.bias[q];
    const int vz = widest<T>(c.z[q], c.ldz), vd = widest<T>(c.dz[q], c.lddz);
    V = vz < V ? vz : V;
    V = vd < V ? vd : V;
    rows_pass = rows_pass || a.dz[q] || a.row_bias[q];
  }
  if (rows_pass) {
    const int lanes = lanes_for(c.R, V);
    const unsigned grid = row_grid<T>(c.rows, lanes);
    if (V * sizeof(T) == 16) layer_slope_kernel<T, 16 / sizeof(T)><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
    else if (V == 4) layer_slope_kernel<T, sizeof(T) == 2 ? 4 : 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
    else if (V == 2) layer_slope_kernel<T, sizeof(T) <= 4 ? 2 : 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
    else layer_slope_kernel<T, 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
    COMET_LAUNCH_CHECK(ctx);
  }
  if (c.bias_along == COMET_BIAS_COLS && c.bias[0]) {
    int64_t blocks = ceil_div(c.rows, 64);
    const int64_t most = 4 * kSmCount;
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
      column_join_kernel<T><<<(unsigned)ceil_div(b.R, 32), kJoinThreads, 0, s>>>(part, blocks, b.R, (T *)c.bias[0] + first);
      ctx->launches += 2;
      e = cudaGetLastError();
    }
    ctx_free(ctx, part, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
  }
  return COMET_OK;
}

template <class T> comet_status_t finish_typed(Context *ctx, const FinishCall &c, cudaStream_t s) {
  FinishArgs<T> a{};
  a.rows = c.rows; a.R = c.R; a.ldzin = c.ldzin; a.ldz = c.ldz; a.ldr = c.ldr; a.ldc = c.ldc;
  a.act = c.act; a.bias_along = c.bias_along; a.sources = c.sources; a.sum = c.sum;
  a.res = (const T *)c.residual;
  a.C = (T *)c.C;
  int V = widest<T>(c.C, c.ldc);
  const auto also = [&](const void *p, int64_t ld) { const int v = widest<T>(p, ld); V = v < V ? v : V; };
  also(c.residual, c.ldr);
  for (int q = 0; q < c.sources; ++q) {
    a.z[q] = (const typename FinishArgs<T>::Z *)c.z[q];
    a.bias[q] = (const T *)c.bias[q];
    a.pre[q] = (T *)c.pre[q];
    if (sizeof(T) >= 4) also(c.z[q], c.ldzin);             // (16-bit outputs: the products are this library's own, padded)
    also(c.pre[q], c.ldz);
  }
  const int lanes = lanes_for(c.R, V);
  const unsigned grid = row_grid<T>(c.rows, lanes);
  if (V * sizeof(T) == 16) layer_finish_kernel<T, 16 / sizeof(T)><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
  else if (V == 4) layer_finish_kernel<T, sizeof(T) == 2 ? 4 : 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
  else if (V == 2) layer_finish_kernel<T, sizeof(T) <= 4 ? 2 : 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
  else layer_finish_kernel<T, 1><<<grid, kSlopeThreads, 0, s>>>(a, lanes);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

template <class V> __global__ void __launch_bounds__(kBlockThreads) layer_pick_kernel(const V *__restrict__ val, const int32_t *__restrict__ index, int64_t n,
                                                                                      V *__restrict__ out) {
  const int64_t first = (int64_t)blockIdx.x * (4 * kBlockThreads) + threadIdx.x;
  int32_t at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) at[j] = first + j * kBlockThreads < n ? ld_stream(index + first + j * kBlockThreads) : 0;
  V x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = __ldg(val + at[j]);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (first + j * kBlockThreads < n) out[first + j * kBlockThreads] = x[j];
}

template <class T> __global__ void __launch_bounds__(kBlockThreads) layer_widen_values_kernel(const T *__restrict__ val, const int32_t *__restrict__ index, int64_t n,
                                                                                              float *__restrict__ out) {
  const int64_t first = (int64_t)blockIdx.x * (4 * kBlockThreads) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t p = first + j * kBlockThreads;
    if (p < n) out[p] = widen(val[index ? (int64_t)__ldg(index + p) : p]);
  }
}

// `lanes` to a row, four values each.
template <class T> __global__ void __launch_bounds__(kSlopeThreads) layer_widen_kernel(const T *__restrict__ in, int64_t rows, int64_t R, int64_t ld, int64_t ldo,
                                                                                       int lanes, float *__restrict__ out) {
  const int l = threadIdx.x & (lanes - 1), each = kSlopeThreads / lanes;
  for (int64_t i = (int64_t)blockIdx.x * each + threadIdx.x / lanes; i < rows; i += (int64_t)gridDim.x * each)
    for (int64_t col = 4 * l; col < R; col += 4 * lanes) {
      float4 x;
      const T *p = in + i * ld + col;
      x.x = widen(p[0]);
      x.y = col + 1 < R ? widen(p[1]) : 0.0f;
      x.z = col + 2 < R ? widen(p[2]) : 0.0f;
      x.w = col + 3 < R ? widen(p[3]) : 0.0f;
      *reinterpret_cast<float4 *>(out + i * ldo + col) = x;
    }
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

comet_status_t layer_finish(Context *ctx, int dtype, const FinishCall &c, cudaStream_t s) {
  switch (dtype) {
    case COMET_F64: return finish_typed<double>(ctx, c, s);
    case COMET_F32: return finish_typed<float>(ctx, c, s);
    case COMET_BF16: return finish_typed<__nv_bfloat16>(ctx, c, s);
    default: return finish_typed<__half>(ctx, c, s);
  }
}

comet_status_t layer_widen(Context *ctx, int dtype, const void *in, int64_t rows, int64_t R, int64_t ld, float *out, cudaStream_t s) {
  if (rows == 0) return COMET_OK;
  const int64_t ldo = layer_padded(COMET_F32, R);
  const int lanes = lanes_for(R, 4);
  const unsigned grid = row_grid<float>(rows, lanes);
  if (dtype == COMET_BF16) layer_widen_kernel<<<grid, kSlopeThreads, 0, s>>>((const __nv_bfloat16 *)in, rows, R, ld, ldo, lanes, out);
  else layer_widen_kernel<<<grid, kSlopeThreads, 0, s>>>((const __half *)in, rows, R, ld, ldo, lanes, out);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

comet_status_t layer_widen_values(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, float *out, cudaStream_t s) {
  if (n == 0) return COMET_OK;
  const unsigned blocks = (unsigned)ceil_div(n, 4 * kBlockThreads);
  if (dtype == COMET_BF16) layer_widen_values_kernel<<<blocks, kBlockThreads, 0, s>>>((const __nv_bfloat16 *)val, index, n, out);
  else layer_widen_values_kernel<<<blocks, kBlockThreads, 0, s>>>((const __half *)val, index, n, out);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

comet_status_t layer_pick(Context *ctx, int dtype, const void *val, const int32_t *index, int64_t n, void *out, cudaStream_t s) {
  if (n == 0) return COMET_OK;
  const unsigned blocks = (unsigned)ceil_div(n, 4 * kBlockThreads);
  switch (layer_elem_size(dtype)) {
    case 8: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned long long *)val, index, n, (unsigned long long *)out); break;
    case 4: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned int *)val, index, n, (unsigned int *)out); break;
    default: layer_pick_kernel<<<blocks, kBlockThreads, 0, s>>>((const unsigned short *)val, index, n, (unsigned short *)out);
  }
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

}  // namespace comet
