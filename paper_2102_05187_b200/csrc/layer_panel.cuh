// The sparse x dense product with its epilogue for a few columns (single tokens): rows of B of up to 16 bytes, matrices that are dense enough.
// Template of the types' units.
//
// What bounds such a call should be the matrix's entries, each read once. Gathering B's short rows from L1 is not free, though: a warp's 32 entries
// touch up to 32 lines, a line a cycle (35 us for one token through a gated pair of 13 M entries, whose bytes take 12). So B, padded to V values a
// row, is laid down in shared memory, as many rows at a time as fit (a panel), where 32 arbitrary rows cost the bank conflicts alone. One CTA
// of 32 warps per SM owns a stretch of rows; `parts` warps share a row, each with a contiguous part of its entries, 8 entries a lane and
// round, the next round's in flight meanwhile. A part stops where its columns leave the panel and goes on from there with the
// next one. The parts' sums meet in shared memory and are added in their order.
#pragma once

#include "layer.cuh"

namespace comet {
namespace {

constexpr int kPanelThreads = 1024, kPanelWarps = kPanelThreads / 32;
constexpr int kPanelUnits = 256;               // row parts (of one source) that a CTA works on at a time
constexpr int kPanelSmem = 200 * 1024;

template <class T> struct PanelArgs {
  struct Source { const int32_t *pos, *crd; const T *val; const T *B; int64_t ldb; const T *bias; T *pre; bool aligned; } src[2];
  int64_t ldc, ldr, ldz;
  T *C;
  const T *res;
  int32_t rows, cols, panel_rows, panels, parts;
  int R, act, bias_along, nsrc;
};

template <class T> struct Round {
  int32_t c[8];                                // -1: none
  T v[8];
  // entries base + 4 * (32 * e + lane) .. + 3, e = 0, 1, as far as they lie in [from, end)
  __device__ __forceinline__ void read(const int32_t *__restrict__ crd, const T *__restrict__ val, int64_t base, int32_t from, int32_t end, bool aligned) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t i = base + 4 * (32 * e + lane);
      if (aligned && i >= from && i + 4 <= end) {
        const int4 x = __ldcs(reinterpret_cast<const int4 *>(crd + i));
        c[4 * e] = x.x; c[4 * e + 1] = x.y; c[4 * e + 2] = x.z; c[4 * e + 3] = x.w;
        if (sizeof(T) == 2) {
          const uint2 y = __ldcs(reinterpret_cast<const uint2 *>(val + i));
          *reinterpret_cast<uint2 *>(v + 4 * e) = y;
        } else {
#pragma unroll
          for (int k = 0; k < (int)sizeof(T) / 4; ++k)
            reinterpret_cast<uint4 *>(v + 4 * e)[k] = __ldcs(reinterpret_cast<const uint4 *>(val + i) + k);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool have = i + k >= from && i + k < end;
          c[4 * e + k] = have ? __ldg(crd + i + k) : -1;
          v[4 * e + k] = have ? val[i + k] : (T)0.0f;
        }
      }
    }
  }
};

template <class T, int V> struct alignas(sizeof(T) * V) Few { T at[V]; };

template <class T, int V, int NACC>
__global__ void __launch_bounds__(kPanelThreads, 1) layer_panel_kernel(const PanelArgs<T> a) {
  using acc_t = typename Num<T>::acc;
  using sum_t = typename Num<T>::sum;
  extern __shared__ __align__(16) char smem[];
  __shared__ sum_t sums[NACC][kPanelUnits][V];
  __shared__ int32_t reached[NACC == 2 ? 2 : 1][kPanelUnits];            // where a part goes on (one source at a time, or the pair's two)
  Few<T, V> *panel = reinterpret_cast<Few<T, V> *>(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int32_t row_begin = (int32_t)((int64_t)a.rows * blockIdx.x / gridDim.x), row_end = (int32_t)((int64_t)a.rows * (blockIdx.x + 1) / gridDim.x);
  const int32_t rows_at_once = kPanelUnits / a.parts;
  const int passes = NACC == 2 ? 1 : a.nsrc;                             // the sum of two products goes over the sources one after the other
  int held = -1;                                                         // the panel in shared memory
  for (int32_t row0 = row_begin; row0 < row_end; row0 += rows_at_once) {
    const int32_t rows = min(rows_at_once, row_end - row0), units = rows * a.parts;
    for (int k = threadIdx.x; k < NACC * units * V; k += kPanelThreads) (&sums[0][0][0])[(k / (units * V)) * (kPanelUnits * V) + k % (units * V)] = (sum_t)0;
    for (int pass = 0; pass < passes; ++pass) {
      for (int32_t p = 0; p < a.panels; ++p) {
        const int32_t c0 = p * a.panel_rows, c1 = min(a.cols, c0 + a.panel_rows);
        __syncthreads();
        if (held != pass * a.panels + p) {
          held = pass * a.panels + p;
          const T *B = a.src[pass].B;
          const int64_t ldb = a.src[pass].ldb;
          if (ldb == V && a.R == V && (reinterpret_cast<uintptr_t>(B) & 15) == 0) {          // rows side by side: 16 bytes at a time
            const int64_t first = (int64_t)c0 * V * sizeof(T), bytes = (int64_t)(c1 - c0) * V * sizeof(T), whole = first % 16 ? 0 : bytes / 16;
            const char *from = reinterpret_cast<const char *>(B) + first;
            for (int64_t k = threadIdx.x; k < whole; k += kPanelThreads) reinterpret_cast<uint4 *>(smem)[k] = __ldg(reinterpret_cast<const uint4 *>(from) + k);
            for (int64_t k = whole * 16 / (int64_t)sizeof(T) + threadIdx.x; k < bytes / (int64_t)sizeof(T); k += kPanelThreads)
              reinterpret_cast<T *>(smem)[k] = reinterpret_cast<const T *>(from)[k];
          } else {
            for (int32_t k = threadIdx.x; k < (c1 - c0) * V; k += kPanelThreads) {
              const int32_t j = k / V, r = k % V;
              reinterpret_cast<T *>(smem)[k] = r < a.R ? B[(int64_t)(c0 + j) * ldb + r] : (T)0.0f;
            }
          }
          __syncthreads();
        }
        for (int u = warp; u < units * NACC; u += kPanelWarps) {
          const int q = NACC == 2 ? u % 2 : 0, unit = NACC == 2 ? u / 2 : u;
          const typename PanelArgs<T>::Source &s = a.src[NACC == 2 ? q : pass];
          const int32_t row = row0 + unit / a.parts, part = unit % a.parts;
          const int32_t b = __ldg(s.pos + row), n = __ldg(s.pos + row + 1) - b;
          // parts begin on multiples of 4 entries
          const int32_t share = (n / a.parts + 4) & ~3;
          const int32_t mine = (int32_t)min((int64_t)n, (int64_t)part * share), end = b + (int32_t)min((int64_t)n, (int64_t)(part + 1) * share);
          int32_t from = b + mine;
          if (p > 0) from = reached[q][unit];
          acc_t acc[V];
          sum_t sum[V];
#pragma unroll
          for (int v = 0; v < V; ++v) sum[v] = (sum_t)0;
          int64_t base = from & ~3;
          Round<T> now, next;
          int32_t stop = end;
          now.read(s.crd, s.val, base, from, end, s.aligned);
          while (base < stop) {
            next.read(s.crd, s.val, base + 256, from, end, s.aligned);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = (acc_t)0;
            int32_t left = -1;                                            // this lane's first entry beyond the panel
#pragma unroll
            for (int e = 7; e >= 0; --e) {
              const uint32_t j = (uint32_t)(now.c[e] - c0);
              if (j < (uint32_t)(c1 - c0)) {
                const Few<T, V> x = panel[j];
                const acc_t w = widen(now.v[e]);
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += w * widen(x.at[v]);
              } else if (now.c[e] >= c1) {
                left = (int32_t)(base + 4 * (32 * (e >> 2) + lane) + (e & 3));
              }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += acc[v];
            if (a.panels > 1) {
              const uint32_t nearest = __reduce_min_sync(0xffffffffu, (uint32_t)left);
              if (nearest != 0xffffffffu) { stop = (int32_t)nearest; break; }
            }
            now = next;
            base += 256;
          }
          for (int off = 16; off >= 1; off >>= 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += __shfl_xor_sync(0xffffffffu, sum[v], off);
          }
          if (lane == 0) {
            if (a.panels > 1) reached[q][unit] = stop;
#pragma unroll
            for (int v = 0; v < V; ++v) sums[q][unit][v] += sum[v];
          }
        }
      }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < rows * a.R; k += kPanelThreads) {
      const int32_t r = k / a.R, col = k % a.R;
      const int64_t i = row0 + r;
      acc_t z[NACC];
#pragma unroll
      for (int q = 0; q < NACC; ++q) {
        sum_t t = (sum_t)0;
        for (int part = 0; part < a.parts; ++part) t += sums[q][r * a.parts + part][col];
        if (a.src[q].bias) t += widen(a.src[q].bias[a.bias_along == COMET_BIAS_ROWS ? i : col]);
        z[q] = (acc_t)t;
        if (a.src[q].pre) a.src[q].pre[i * a.ldz + col] = narrow<T, acc_t>(z[q]);
      }
      acc_t y = activate<sizeof(T) == 2>(a.act, z[0]);
      if (NACC == 2) y *= z[NACC - 1];
      if (a.res) y += widen(a.res[i * a.ldr + col]);
      a.C[i * a.ldc + col] = narrow<T, acc_t>(y);
    }
    __syncthreads();
  }
}

template <class T, int V, int NACC> comet_status_t panel_launch(Context *ctx, PanelArgs<T> &a, int64_t nnz, cudaStream_t s) {
  const int most = kPanelSmem / (int)(V * sizeof(T));
  a.panels = (int32_t)ceil_div(a.cols, most);
  a.panel_rows = (int32_t)align_up((size_t)ceil_div(a.cols, a.panels), 16);
  const unsigned grid = (unsigned)(a.rows < kSmCount ? a.rows : kSmCount);
  // Parts of a row: so many that every warp of a CTA has one, but of 128 entries at least.
  const int64_t rows_each = ceil_div(a.rows, grid) * NACC, mean = nnz / ((int64_t)a.rows * a.nsrc);
  a.parts = 1;
  while (a.parts < kPanelWarps && rows_each * a.parts < kPanelWarps && mean / (a.parts * 2) >= 128) a.parts *= 2;
  const size_t bytes = (size_t)(a.panel_rows < a.cols ? a.panel_rows : a.cols) * V * sizeof(T);
  auto *kernel = layer_panel_kernel<T, V, NACC>;
  COMET_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPanelSmem));
  kernel<<<grid, kPanelThreads, bytes, s>>>(a);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

template <class T, int V> comet_status_t panel_mode(Context *ctx, PanelArgs<T> &a, bool gated, int64_t nnz, cudaStream_t s) {
  return gated ? panel_launch<T, V, 2>(ctx, a, nnz, s) : panel_launch<T, V, 1>(ctx, a, nnz, s);
}

}  // namespace

template <class T> comet_status_t layer_panel_typed(Context *ctx, const GatherCall &c, cudaStream_t s) {
  PanelArgs<T> a{};
  a.nsrc = c.mode == kLayer ? 1 : 2;
  int64_t nnz = 0;
  for (int q = 0; q < a.nsrc; ++q) {
    const GatherSource &g = c.src[q];
    a.src[q] = {g.A.pos, g.A.crd, (const T *)g.A.val, (const T *)g.B, g.ldb, (const T *)g.bias, (T *)g.pre,
                ((uintptr_t)g.A.crd & 15) == 0 && ((uintptr_t)g.A.val & 15) == 0};
    nnz += g.A.nnz;
  }
  a.ldc = c.ldc; a.ldr = c.ldr; a.ldz = c.ldz;
  a.C = (T *)c.C;
  a.res = (const T *)c.residual;
  a.rows = (int32_t)c.src[0].A.rows; a.cols = (int32_t)c.src[0].A.cols;
  a.R = (int)c.R;
  a.act = c.act; a.bias_along = c.bias_along;
  const bool gated = c.mode == kGated;
  if constexpr (sizeof(T) <= 2) {
    if (c.R > 4) return panel_mode<T, 8>(ctx, a, gated, nnz, s);
  }
  if constexpr (sizeof(T) <= 4) {
    if (c.R > 2) return panel_mode<T, 4>(ctx, a, gated, nnz, s);
  }
  return c.R > 1 ? panel_mode<T, 2>(ctx, a, gated, nnz, s) : panel_mode<T, 1>(ctx, a, gated, nnz, s);
}

}  // namespace comet
