// The sparse x dense product with its epilogue for a few columns (single tokens): rows of B of up to 16 bytes, matrices that are dense enough.
// Template of the types' units.
//
// What bounds such a call should be the matrix's entries, each read once. Gathering B's short rows from L1 is not free, though: a warp's 32 entries
// touch up to 32 lines, a line a cycle (35 us for one token through a gated pair of 13 M entries, whose bytes take 12). So B, padded to V values a
// row, is laid down in shared memory, as many rows at a time as fit (a panel), where 32 arbitrary rows cost the bank conflicts alone. One CTA
// of 32 warps per SM owns a stretch of rows; `parts` warps share a row, each with a contiguous part of its entries, 8 entries a lane and
// round (4 of fp64), the next round's in flight meanwhile. A part stops where its columns leave the panel and goes on from there with the
// next one, which takes ordered rows; one panel does not. The parts' sums meet in shared memory and are added in their order.
#pragma once

#include "layer.cuh"

namespace comet {
namespace {

constexpr int kPanelThreads = 1024, kPanelWarps = kPanelThreads / 32;
constexpr int kPanelUnits = 256;               // row parts (of one source) that a CTA works on at a time

template <class T> struct PanelArgs {
  struct Source { const int32_t *pos, *crd; const T *val; const T *B; int64_t ldb; const T *bias; T *pre; bool aligned; } src[2];
  int64_t ldc, ldr, ldz;
  T *C;
  const T *res;
  int32_t rows, cols, panel_rows, panels, parts, log_parts;
  int R, act, bias_along, nsrc;
};

constexpr int32_t kNoColumn = 2147483647;

// Entries of one lane in a round: kE fours, 128 entries apart.
template <class T> struct Round {
  static constexpr int kE = sizeof(T) == 8 ? 1 : 2, kEntries = 128 * kE;
  int32_t c[4 * kE];
  T v[4 * kE];
  __device__ __forceinline__ void read4(const int32_t *__restrict__ crd, const T *__restrict__ val, int32_t i, int e, bool aligned) {
    if (aligned) {
      const int4 x = __ldcs(reinterpret_cast<const int4 *>(crd + i));
      c[4 * e] = x.x; c[4 * e + 1] = x.y; c[4 * e + 2] = x.z; c[4 * e + 3] = x.w;
      if (sizeof(T) == 2) {
        *reinterpret_cast<uint2 *>(v + 4 * e) = __ldcs(reinterpret_cast<const uint2 *>(val + i));
      } else {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 4; ++k) reinterpret_cast<uint4 *>(v + 4 * e)[k] = __ldcs(reinterpret_cast<const uint4 *>(val + i) + k);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        c[4 * e + k] = __ldg(crd + i + k);
        v[4 * e + k] = val[i + k];
      }
    }
  }
  // i: the lane's first entry; fours that do not begin before `end` (a multiple of 4) get the column `none` and zeros
  __device__ __forceinline__ void read(const typename PanelArgs<T>::Source &s, int32_t i, int32_t end, int32_t none) {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      if (i + 128 * e < end) {
        read4(s.crd, s.val, i + 128 * e, e, s.aligned);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) { c[4 * e + k] = none; v[4 * e + k] = (T)0.0f; }
      }
    }
  }
};

template <class T, int V> struct alignas(sizeof(T) * V) Few { T at[V]; };

// A row part: which one, and its entries.
struct Part {
  int q, unit;
  int32_t from, end;
  // This lane's first entry among the fours (they start on multiples of 4), and how many entries of fours there are.
  __device__ __forceinline__ void split(int32_t &i, int32_t &left) const {
    const int32_t first = min(end, (from + 3) & ~3), last = max(first, end & ~3);
    i = first + 4 * (threadIdx.x & 31);
    left = last - first;
  }
};
// The up to three entries in front of a part's first four and behind its last one: a lane each.
template <class T> struct Single {
  int32_t c, at;
  T v;
  __device__ __forceinline__ void read(const typename PanelArgs<T>::Source &s, const Part &w, int32_t none) {
    const int lane = threadIdx.x & 31;
    const int32_t first = min(w.end, (w.from + 3) & ~3), last = max(first, w.end & ~3);
    at = lane < 4 ? w.from + lane : last + lane - 4;
    const bool have = lane < 4 ? at < first : lane < 8 && at < w.end;
    c = have ? __ldg(s.crd + at) : none;
    v = have ? s.val[at] : (T)0.0f;
  }
};

// One part's sums over its entries, as far as their columns lie in the panel [c0, c1). Returns the first entry beyond the panel, or the part's end.
// `several`: there are more panels than this one. Behind the panel's rows lies one of zeros: entries that are none of the panel's are
// multiplied by it, with a weight of zero, so that the sums need no branches.
template <class T, int V, bool several>
__device__ __forceinline__ int32_t part_sum(const typename PanelArgs<T>::Source &s, const Part &part, int32_t c0, int32_t c1, const Few<T, V> *panel,
                                            typename Num<T>::sum (&sum)[V]) {
  using acc_t = typename Num<T>::acc;
  constexpr int kStep = Round<T>::kEntries;
  const int32_t none = several ? kNoColumn : c1;
  const Few<T, V> *at = panel - c0;
  uint32_t beyond = 0xffffffffu;                                 // this lane's first entry beyond the panel
  bool going = true;
  const auto use = [&](const Round<T> &r, int32_t i) {
    acc_t acc[V];
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] = (acc_t)0;
#pragma unroll
    for (int e = 0; e < 4 * Round<T>::kE; ++e) {
      const Few<T, V> x = at[several ? min(r.c[e], c1) : r.c[e]];
      const acc_t w = !several || r.c[e] < c1 ? widen(r.v[e]) : (acc_t)0;
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] += w * widen(x.at[k]);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] += acc[k];
    if (several && __shfl_sync(0xffffffffu, r.c[4 * Round<T>::kE - 1], 31) >= c1) {
#pragma unroll
      for (int e = 4 * Round<T>::kE - 1; e >= 0; --e)
        if (r.c[e] >= c1 && r.c[e] != kNoColumn) beyond = (uint32_t)(i + 128 * (e >> 2) + (e & 3));
      going = !__any_sync(0xffffffffu, beyond != 0xffffffffu);
    }
  };
  Single<T> one;
  one.read(s, part, none);
  int32_t i, left;
  part.split(i, left);
  const int32_t last = i + left - 4 * (int32_t)(threadIdx.x & 31);
  Round<T> x, y;
  x.read(s, i, last, none);
  while (left > 0) {
    if (left > kStep) y.read(s, i + kStep, last, none);
    use(x, i);
    i += kStep;
    left -= kStep;
    if (left <= 0 || !going) break;
    if (left > kStep) x.read(s, i + kStep, last, none);
    use(y, i);
    i += kStep;
    left -= kStep;
    if (!going) break;
  }
  if (one.c < c1) {
    const Few<T, V> b = at[one.c];
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] += widen(one.v) * widen(b.at[k]);
  } else if (several && one.c != kNoColumn) {
    beyond = min(beyond, (uint32_t)one.at);
  }
  return several ? (int32_t)min((uint32_t)part.end, __reduce_min_sync(0xffffffffu, beyond)) : part.end;
}

template <class T, int V, int NACC, bool several>
__global__ void __launch_bounds__(kPanelThreads, 1) layer_panel_kernel(const PanelArgs<T> a) {
  using acc_t = typename Num<T>::acc;
  using sum_t = typename Num<T>::sum;
  extern __shared__ __align__(16) char smem[];
  __shared__ sum_t sums[NACC][kPanelUnits][V];
  __shared__ int32_t reached[NACC][kPanelUnits];                         // where a part goes on (one source at a time, or the pair's two)
  __shared__ int32_t bounds[2][kPanelUnits + 1];                         // of the rows at hand
  Few<T, V> *panel = reinterpret_cast<Few<T, V> *>(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int32_t row_begin = (int32_t)((int64_t)a.rows * blockIdx.x / gridDim.x), row_end = (int32_t)((int64_t)a.rows * (blockIdx.x + 1) / gridDim.x);
  const int32_t rows_at_once = kPanelUnits / a.parts;
  const int passes = NACC == 2 ? 1 : a.nsrc;                             // the sum of two products goes over the sources one after the other
  int held = -1;                                                         // the panel in shared memory
  for (int32_t row0 = row_begin; row0 < row_end; row0 += rows_at_once) {
    const int32_t rows = min(rows_at_once, row_end - row0), units = rows * a.parts;
    for (int k = threadIdx.x; k < NACC * units * V; k += kPanelThreads) (&sums[0][0][0])[(k / (units * V)) * (kPanelUnits * V) + k % (units * V)] = (sum_t)0;
    for (int q = 0; q < a.nsrc; ++q)
      for (int k = threadIdx.x; k <= rows; k += kPanelThreads) bounds[q][k] = __ldg(a.src[q].pos + row0 + k);
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
          if (threadIdx.x < V) reinterpret_cast<T *>(smem)[(c1 - c0) * V + threadIdx.x] = (T)0.0f;
          __syncthreads();
        }
        const int total = units * NACC;
        const auto part_of = [&](int u) {
          Part w;
          w.q = NACC == 2 ? u & 1 : 0;
          w.unit = NACC == 2 ? u >> 1 : u;
          const int32_t *at = bounds[NACC == 2 ? w.q : pass] + (w.unit >> a.log_parts);
          const int32_t n = at[1] - at[0], share = ((n >> a.log_parts) + 4) & ~3, first = (w.unit & (a.parts - 1)) * (int64_t)share > n ? n : (w.unit & (a.parts - 1)) * share;
          w.from = at[0] + first;
          w.end = at[0] + (int32_t)min((int64_t)n, (int64_t)first + share);
          return w;
        };
        const auto join = [&](const Part &w, sum_t (&sum)[V]) {
          for (int off = 16; off >= 1; off >>= 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += __shfl_xor_sync(0xffffffffu, sum[v], off);
          }
          if (lane == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) sums[w.q][w.unit][v] += sum[v];
          }
#pragma unroll
          for (int v = 0; v < V; ++v) sum[v] = (sum_t)0;
        };
        sum_t sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = (sum_t)0;
        for (int u = warp; u < total; u += kPanelWarps) {
          Part w = part_of(u);
          if (several && p > 0) w.from = reached[w.q][w.unit];
          const int32_t stop = part_sum<T, V, several>(a.src[NACC == 2 ? w.q : pass], w, c0, c1, panel, sum);
          if (several && lane == 0) reached[w.q][w.unit] = stop;
          join(w, sum);
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
  // Panels of one size, in steps of 16 rows (they start on 16 bytes); no more than fit beside the row of zeros, and none that is empty.
  const int most = panel_capacity(V * (int)sizeof(T));
  a.panel_rows = (int32_t)align_up((size_t)ceil_div(a.cols, ceil_div(a.cols, most)), 16);
  a.panels = (int32_t)ceil_div(a.cols, a.panel_rows);
  const unsigned grid = (unsigned)(a.rows < kSmCount ? a.rows : kSmCount);
  // Parts of a row: so many that every warp of a CTA has one, but of 128 entries at least.
  const int64_t rows_each = ceil_div(a.rows, grid) * NACC, mean = nnz / ((int64_t)a.rows * a.nsrc);
  a.parts = 1;
  while (a.parts < kPanelWarps && rows_each * a.parts < kPanelWarps && mean / (a.parts * 2) >= 128) { a.parts *= 2; ++a.log_parts; }
  const size_t bytes = (size_t)((a.panel_rows < a.cols ? a.panel_rows : a.cols) + 1) * V * sizeof(T);
  auto *kernel = a.panels > 1 ? layer_panel_kernel<T, V, NACC, true> : layer_panel_kernel<T, V, NACC, false>;
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
