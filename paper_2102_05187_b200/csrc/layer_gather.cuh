// The sparse x dense product with its epilogue, by gathers (any type, any width): template of the four types' units.
//
//   Z[i, r] = sum over the entries p of row i of val[p] * B[crd[p], r], then the epilogue of the call on Z, one store.
//
// A worker of WS lanes owns a row and a block of columns: W of its lanes own the columns (16 bytes of a row each, or 4 or 1 single
// values where rows are not 16-byte aligned), and its WS / W groups of W lanes take the row's entries in turn; the groups' sums are
// joined by shuffles and the first group applies the epilogue, so that Z never goes through memory. Entries are loaded WS at a time, a lane each,
// and handed round by shuffles; 4 (few columns) or 8 rows of B are in flight per group. What bounds it is the gathers: nnz * R values through
// L2 and L1, where the workers of a CTA, which own neighbouring rows and walk them in step, find part of them.
// Rows of more than `long_len` entries are put off until the CTA's other rows are done and then shared out to all of its workers (a power law's
// heaviest rows otherwise end the kernel alone); rows of more than kHugeRow, where the matrix can have any, are cut into items for
// a launch of their own. Sums are joined in a fixed order everywhere: results do not change from run to run.
#pragma once

#include "layer.cuh"

namespace comet {
namespace {

constexpr int kGatherThreads = 256;
constexpr int32_t kHugeRow = 16384;      // entries from which a row is cut into items of kHugeItem
constexpr int32_t kHugeItem = 4096;

template <class T> struct GatherArgs {
  struct Source { const int32_t *pos, *crd; const T *val; const T *B; int64_t ldb; const T *bias; T *pre; } src[2];
  int64_t R, col_block0, ldc, ldr, ldz;
  T *C;
  const T *res;
  int32_t rows, long_len, huge_len;
  int log_w, log_ws, act, bias_along, nsrc;
  bool gated, vec_out;
};

struct HugeItem { int32_t row, src, beg, len; };
struct HugeRow { int32_t row, first, count0, count1; };     // items of source 0, then of source 1

// Columns of one lane: V of them, contiguous (VEC) or W apart.
template <class T, int V, bool VEC> struct Lane {
  int64_t col;             // first column
  int apart, cols;         // distance, how many exist (0: the lane idles)
  __device__ __forceinline__ Lane(int64_t block, int W, int l, int64_t R) {
    const int64_t base = block * W * V;
    apart = VEC ? 1 : W;
    col = base + (VEC ? (int64_t)l * V : l);
    int64_t left = R - col;
    if (!VEC) left = left <= 0 ? 0 : (left + W - 1) / W;
    cols = left <= 0 ? 0 : left >= V ? V : (int)left;
  }
  __device__ __forceinline__ void load(const T *p, T (&x)[V]) const {      // p: the row's address at this lane's first column
    if (VEC && cols == V) {
      Piece<T> q;
      q.raw = __ldg(reinterpret_cast<const uint4 *>(p));
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = q.at[v];
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = v < cols ? p[v * apart] : (T)0.0f;
    }
  }
};

template <class T, int V, bool VEC, bool FEW>
__device__ __forceinline__ void walk(const int32_t *__restrict__ crd, const T *__restrict__ val, int n, int nmax, const T *__restrict__ Bc,
                                     int64_t ldb, const Lane<T, V, VEC> &lane, int log_w, int log_ws, typename Num<T>::sum (&sum)[V]) {
  using acc_t = typename Num<T>::acc;
  const int W = 1 << log_w, WS = 1 << log_ws, G = WS >> log_w;
  const int at = threadIdx.x & 31, in_worker = at & (WS - 1), first = at & ~(WS - 1), group = in_worker >> log_w;
  const bool live = lane.cols > 0;
  for (int base = 0; base < nmax; base += 4 * WS) {
    int c[4];
    acc_t a[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = base + e * WS + in_worker;
      c[e] = i < n ? __ldg(crd + i) : -1;
      a[e] = i < n ? widen(val[i]) : (acc_t)0;
    }
    acc_t acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = (acc_t)0;
    if (FEW) {
      for (int k = 0; k < W; ++k) {
        T x[4][V];
        const int from = first + k * G + group;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = __shfl_sync(0xffffffffu, c[e], from);
          if (live && j >= 0) lane.load(Bc + (int64_t)j * ldb, x[e]);
          else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[e][v] = (T)0.0f;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const acc_t y = __shfl_sync(0xffffffffu, a[e], from);
#pragma unroll
          for (int v = 0; v < V; ++v) acc[v] += y * widen(x[e][v]);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        for (int k = 0; k < W && base + e * WS + k * G < nmax; k += 8) {
          T x[8][V];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int j = __shfl_sync(0xffffffffu, c[e], first + (k + u) * G + group);
            if (live && j >= 0) lane.load(Bc + (int64_t)j * ldb, x[u]);
            else {
#pragma unroll
              for (int v = 0; v < V; ++v) x[u][v] = (T)0.0f;
            }
          }
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const acc_t y = __shfl_sync(0xffffffffu, a[e], first + (k + u) * G + group);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] += y * widen(x[u][v]);
          }
        }
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] += acc[v];
  }
  for (int off = W; off < WS; off <<= 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] += __shfl_xor_sync(0xffffffffu, sum[v], off);
  }
}

// The call's epilogue on one lane's columns of row i.
template <class T, int V, bool VEC, int NACC>
__device__ __forceinline__ void finish_row(const GatherArgs<T> &a, int64_t i, const Lane<T, V, VEC> &lane,
                                           const typename Num<T>::sum (&sum)[NACC][V]) {
  using acc_t = typename Num<T>::acc;
  if (lane.cols == 0) return;
  const bool vec = VEC && a.vec_out && lane.cols == V;
  acc_t out[V];
  Piece<T> keep[NACC], res;
  if (vec && a.res) res.raw = __ldg(reinterpret_cast<const uint4 *>(a.res + i * a.ldr + lane.col));
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (v >= lane.cols) continue;
    const int64_t col = lane.col + v * lane.apart;
    acc_t z[NACC];
#pragma unroll
    for (int q = 0; q < NACC; ++q) {
      typename Num<T>::sum t = sum[q][v];
      if (a.src[q].bias) t += widen(a.src[q].bias[a.bias_along == COMET_BIAS_ROWS ? i : col]);
      z[q] = (acc_t)t;
      if (a.src[q].pre) {
        if (vec) keep[q].at[VEC ? v : 0] = narrow<T, acc_t>(z[q]);
        else a.src[q].pre[i * a.ldz + col] = narrow<T, acc_t>(z[q]);
      }
    }
    acc_t y = activate<sizeof(T) == 2>(a.act, z[0]);
    if (NACC == 2) y *= z[NACC - 1];
    if (a.res) y += widen(vec ? res.at[VEC ? v : 0] : a.res[i * a.ldr + col]);
    out[v] = y;
  }
  if (vec) {
    Piece<T> o;
#pragma unroll
    for (int v = 0; v < V; ++v) o.at[VEC ? v : 0] = narrow<T, acc_t>(out[v]);
    *reinterpret_cast<uint4 *>(a.C + i * a.ldc + lane.col) = o.raw;
#pragma unroll
    for (int q = 0; q < NACC; ++q)
      if (a.src[q].pre) *reinterpret_cast<uint4 *>(a.src[q].pre + i * a.ldz + lane.col) = keep[q].raw;
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v < lane.cols) a.C[i * a.ldc + lane.col + v * lane.apart] = narrow<T, acc_t>(out[v]);
  }
}

template <class T, int V, bool VEC, bool FEW, int NACC>
__global__ void __launch_bounds__(kGatherThreads) layer_gather_kernel(const GatherArgs<T> a) {
  using sum_t = typename Num<T>::sum;
  constexpr int kWorkers = kGatherThreads;                 // at most: a worker of one lane
  __shared__ sum_t part[NACC][kGatherThreads * V];
  __shared__ int32_t long_row[kWorkers];
  __shared__ int long_rows;
  const int W = 1 << a.log_w, WS = 1 << a.log_ws, workers = kGatherThreads >> a.log_ws;
  const int worker = threadIdx.x >> a.log_ws, l = threadIdx.x & (W - 1);
  const bool leads = (threadIdx.x & (WS - 1)) < W;         // the worker's first group
  const Lane<T, V, VEC> lane(a.col_block0 + blockIdx.y, W, l, a.R);
  if (threadIdx.x == 0) long_rows = 0;
  __syncthreads();
  const int64_t row = (int64_t)blockIdx.x * workers + worker;
  bool mine = row < a.rows;
  int32_t beg[2] = {0, 0}, len[2] = {0, 0};
  if (mine) {
    int32_t most = 0;
    for (int q = 0; q < a.nsrc; ++q) {
      beg[q] = __ldg(a.src[q].pos + row);
      len[q] = __ldg(a.src[q].pos + row + 1) - beg[q];
      most = max(most, len[q]);
    }
    if (most > a.long_len) {
      mine = false;
      if (most <= a.huge_len && (threadIdx.x & (WS - 1)) == 0) long_row[atomicAdd(&long_rows, 1)] = (int32_t)row;
    }
  }
  sum_t sum[NACC][V];
#pragma unroll
  for (int q = 0; q < NACC; ++q)
#pragma unroll
    for (int v = 0; v < V; ++v) sum[q][v] = (sum_t)0;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (q >= a.nsrc) break;
    const int n = mine ? len[q] : 0, nmax = __reduce_max_sync(0xffffffffu, n);
    sum_t part_sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) part_sum[v] = (sum_t)0;
    walk<T, V, VEC, FEW>(a.src[q].crd + beg[q], a.src[q].val + beg[q], n, nmax, a.src[q].B + lane.col, a.src[q].ldb, lane, a.log_w, a.log_ws, part_sum);
#pragma unroll
    for (int v = 0; v < V; ++v) sum[NACC == 2 ? q : 0][v] += part_sum[v];
  }
  if (mine && leads) finish_row<T, V, VEC, NACC>(a, row, lane, sum);

  __syncthreads();
  for (int k = 0; k < long_rows; ++k) {
    const int64_t i = long_row[k];
#pragma unroll
    for (int q = 0; q < NACC; ++q)
#pragma unroll
      for (int v = 0; v < V; ++v) sum[q][v] = (sum_t)0;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (q >= a.nsrc) break;
      const int32_t b = __ldg(a.src[q].pos + i), n = __ldg(a.src[q].pos + i + 1) - b;
      const int32_t share = (n + workers - 1) / workers;                      // n <= 2^31 - 1, workers <= 256: worker * share < 2^31 + 2^16
      const int64_t from = (int64_t)worker * share;
      const int mine_n = from >= n ? 0 : (int)min((int64_t)share, n - from);
      const int64_t at = b + (mine_n ? from : 0);
      sum_t part_sum[V];
#pragma unroll
      for (int v = 0; v < V; ++v) part_sum[v] = (sum_t)0;
      walk<T, V, VEC, FEW>(a.src[q].crd + at, a.src[q].val + at, mine_n, __reduce_max_sync(0xffffffffu, mine_n), a.src[q].B + lane.col, a.src[q].ldb,
                           lane, a.log_w, a.log_ws, part_sum);
#pragma unroll
      for (int v = 0; v < V; ++v) sum[NACC == 2 ? q : 0][v] += part_sum[v];
    }
    if (leads) {
#pragma unroll
      for (int q = 0; q < NACC; ++q)
#pragma unroll
        for (int v = 0; v < V; ++v) part[q][(worker * V + v) * W + l] = sum[q][v];
    }
    __syncthreads();
    if (threadIdx.x < W) {
#pragma unroll
      for (int q = 0; q < NACC; ++q)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          sum_t t = (sum_t)0;
          for (int w = 0; w < workers; ++w) t += part[q][(w * V + v) * W + l];
          sum[q][v] = t;
        }
      finish_row<T, V, VEC, NACC>(a, i, lane, sum);
    }
    __syncthreads();
  }
}

// ---- rows of more than kHugeRow entries
// counts[0]: items, counts[1]: rows. A row's items are consecutive, whatever order the rows come in.
template <class T>
__global__ void __launch_bounds__(kBlockThreads) huge_rows_kernel(const GatherArgs<T> a, int32_t *__restrict__ counts, HugeItem *__restrict__ items,
                                                                  HugeRow *__restrict__ rows) {
  const int64_t i = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x;
  if (i >= a.rows) return;
  int32_t beg[2] = {0, 0}, len[2] = {0, 0};
  for (int q = 0; q < a.nsrc; ++q) {
    beg[q] = __ldg(a.src[q].pos + i);
    len[q] = __ldg(a.src[q].pos + i + 1) - beg[q];
  }
  if (max(len[0], len[1]) <= a.huge_len) return;
  const int32_t n0 = (int32_t)(((int64_t)len[0] + kHugeItem - 1) / kHugeItem), n1 = (int32_t)(((int64_t)len[1] + kHugeItem - 1) / kHugeItem);
  const int32_t at = atomicAdd(counts, n0 + n1);
  rows[atomicAdd(counts + 1, 1)] = HugeRow{(int32_t)i, at, n0, n1};
  for (int q = 0; q < 2; ++q)
    for (int32_t k = 0; k < (q ? n1 : n0); ++k)
      items[at + (q ? n0 : 0) + k] = HugeItem{(int32_t)i, q, beg[q] + k * kHugeItem, min(kHugeItem, len[q] - k * kHugeItem)};
}

// part[item, 0..R) = the item's sum; a CTA per item and block of columns
template <class T, int V, bool VEC, bool FEW>
__global__ void __launch_bounds__(kGatherThreads) huge_items_kernel(const GatherArgs<T> a, const int32_t *__restrict__ counts,
                                                                    const HugeItem *__restrict__ items, typename Num<T>::sum *__restrict__ part) {
  using sum_t = typename Num<T>::sum;
  __shared__ sum_t joined[kGatherThreads * V];
  const int W = 1 << a.log_w, WS = 1 << a.log_ws, workers = kGatherThreads >> a.log_ws;
  const int worker = threadIdx.x >> a.log_ws, l = threadIdx.x & (W - 1);
  const Lane<T, V, VEC> lane(a.col_block0 + blockIdx.y, W, l, a.R);
  const int32_t count = __ldg(counts);
  for (int32_t k = blockIdx.x; k < count; k += gridDim.x) {
    const HugeItem it = items[k];
    const typename GatherArgs<T>::Source &src = a.src[it.src];
    const int share = (it.len + workers - 1) / workers, from = worker * share;
    const int n = max(0, min(share, it.len - from));
    const int64_t at = (int64_t)it.beg + (n ? from : 0);
    sum_t sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = (sum_t)0;
    walk<T, V, VEC, FEW>(src.crd + at, src.val + at, n, __reduce_max_sync(0xffffffffu, n), src.B + lane.col, src.ldb, lane, a.log_w, a.log_ws, sum);
    if ((threadIdx.x & (WS - 1)) < W) {
#pragma unroll
      for (int v = 0; v < V; ++v) joined[(worker * V + v) * W + l] = sum[v];
    }
    __syncthreads();
    if (threadIdx.x < W) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (v >= lane.cols) continue;
        sum_t t = (sum_t)0;
        for (int w = 0; w < workers; ++w) t += joined[(w * V + v) * W + l];
        part[(int64_t)k * a.R + lane.col + v * lane.apart] = t;
      }
    }
    __syncthreads();
  }
}

// The epilogue of the huge rows: a warp per row and block of columns
template <class T, int V, bool VEC, int NACC>
__global__ void __launch_bounds__(kGatherThreads) huge_finish_kernel(const GatherArgs<T> a, const int32_t *__restrict__ counts,
                                                                     const HugeRow *__restrict__ rows, const typename Num<T>::sum *__restrict__ part) {
  using sum_t = typename Num<T>::sum;
  const int W = 1 << a.log_w, l = threadIdx.x & 31;
  const int32_t count = __ldg(counts + 1);
  const Lane<T, V, VEC> lane(a.col_block0 + blockIdx.y, W, l & (W - 1), a.R);
  for (int32_t k = blockIdx.x * (kGatherThreads / 32) + (threadIdx.x >> 5); k < count; k += gridDim.x * (kGatherThreads / 32)) {
    if (l >= W) continue;
    const HugeRow r = rows[k];
    sum_t sum[NACC][V];
#pragma unroll
    for (int q = 0; q < NACC; ++q)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        sum_t t = (sum_t)0;
        const int32_t from = r.first + (NACC == 2 && q ? r.count0 : 0);
        const int32_t n = NACC == 2 ? (q ? r.count1 : r.count0) : r.count0 + r.count1;
        if (v < lane.cols)
          for (int32_t j = 0; j < n; ++j) t += part[(int64_t)(from + j) * a.R + lane.col + v * lane.apart];
        sum[q][v] = t;
      }
    finish_row<T, V, VEC, NACC>(a, r.row, lane, sum);
  }
}

inline int log2_ceil(int64_t x) {
  int k = 0;
  while ((1ll << k) < x) ++k;
  return k;
}

template <class T, int V, bool VEC, bool FEW, int NACC>
comet_status_t gather_launch(Context *ctx, GatherArgs<T> &a, int64_t nnz, bool huge, cudaStream_t s) {
  const int64_t per_block = (int64_t)V << a.log_w, blocks = ceil_div(a.R, per_block);
  const unsigned groups = (unsigned)ceil_div(a.rows, kGatherThreads >> a.log_ws);
  int32_t *counts = nullptr;
  HugeItem *items = nullptr;
  HugeRow *rows = nullptr;
  typename Num<T>::sum *part = nullptr;
  char *mem = nullptr;
  cudaError_t e = cudaSuccess;
  // at most nnz / kHugeRow rows, with an item for each kHugeItem entries and at most one more per source
  const int64_t max_rows = nnz / kHugeRow, max_items = nnz / kHugeItem + 2 * max_rows;
  const size_t b_items = align_up((size_t)max_items * sizeof(HugeItem), 256), b_rows = align_up((size_t)max_rows * sizeof(HugeRow), 256);
  if (huge) mem = (char *)ctx_alloc(ctx, 256 + b_items + b_rows + (size_t)max_items * (size_t)a.R * sizeof(*part), s);
  if (!mem) {                            // none, or no room for them: they are rows like the other long ones
    huge = false;
    a.huge_len = 2147483647;
  }
  if (huge) {
    counts = (int32_t *)mem;
    items = (HugeItem *)(mem + 256);
    rows = (HugeRow *)(mem + 256 + b_items);
    part = (typename Num<T>::sum *)(mem + 256 + b_items + b_rows);
    e = cudaMemsetAsync(counts, 0, 256, s);
    if (e == cudaSuccess) {
      huge_rows_kernel<T><<<(unsigned)ceil_div(a.rows, kBlockThreads), kBlockThreads, 0, s>>>(a, counts, items, rows);
      ctx->launches += 1;
      e = cudaGetLastError();
    }
  }
  for (int64_t b = 0; b < blocks && e == cudaSuccess; b += 65535) {
    a.col_block0 = b;
    const unsigned ys = (unsigned)(blocks - b < 65535 ? blocks - b : 65535);
    layer_gather_kernel<T, V, VEC, FEW, NACC><<<dim3(groups, ys), kGatherThreads, 0, s>>>(a);
    ctx->launches += 1;
    e = cudaGetLastError();
    if (huge && e == cudaSuccess) {
      huge_items_kernel<T, V, VEC, FEW><<<dim3(4 * kSmCount, ys), kGatherThreads, 0, s>>>(a, counts, items, part);
      huge_finish_kernel<T, V, VEC, NACC><<<dim3(kSmCount, ys), kGatherThreads, 0, s>>>(a, counts, rows, part);
      ctx->launches += 2;
      e = cudaGetLastError();
    }
  }
  if (mem) ctx_free(ctx, mem, s);
  return e == cudaSuccess ? COMET_OK : cuda_fail(ctx, e);
}

template <class T, int V, bool VEC>
comet_status_t gather_width(Context *ctx, GatherArgs<T> &a, int64_t nnz, bool huge, cudaStream_t s) {
  a.log_w = log2_ceil(ceil_div(a.R, V));
  if (a.log_w > 5) a.log_w = 5;
  // Groups per worker: a quarter of a row's mean entries each, so that short rows share a warp and long ones have all of it.
  const int64_t mean = a.rows ? nnz / ((int64_t)a.rows * a.nsrc) : 0;
  a.log_ws = a.log_w + log2_ceil(mean / 4 > 0 ? mean / 4 : 1);
  if (a.log_ws > 5) a.log_ws = 5;
  const bool few = a.log_w < 3;
  if (a.gated)
    return few ? gather_launch<T, V, VEC, true, 2>(ctx, a, nnz, huge, s) : gather_launch<T, V, VEC, false, 2>(ctx, a, nnz, huge, s);
  return few ? gather_launch<T, V, VEC, true, 1>(ctx, a, nnz, huge, s) : gather_launch<T, V, VEC, false, 1>(ctx, a, nnz, huge, s);
}

inline bool aligned16(const void *p, int64_t ld, size_t es) { return !p || (((uintptr_t)p & 15) == 0 && (ld * (int64_t)es) % 16 == 0); }

}  // namespace

template <class T> comet_status_t layer_gather_typed(Context *ctx, const GatherCall &c, cudaStream_t s) {
  const int64_t rows = c.src[0].A.rows;
  if (rows == 0 || c.R == 0) return COMET_OK;
  GatherArgs<T> a{};
  a.nsrc = c.mode == kLayer ? 1 : 2;
  a.gated = c.mode == kGated;
  int64_t nnz = 0, cols = 0, most = 0;
  bool vec = true, vec_out = aligned16(c.C, c.ldc, sizeof(T)) && aligned16(c.residual, c.ldr, sizeof(T));
  for (int q = 0; q < a.nsrc; ++q) {
    const GatherSource &g = c.src[q];
    a.src[q] = {g.A.pos, g.A.crd, (const T *)g.A.val, (const T *)g.B, g.ldb, (const T *)g.bias, (T *)g.pre};
    nnz += g.A.nnz;
    cols = g.A.cols > cols ? g.A.cols : cols;
    most = g.A.nnz > most ? g.A.nnz : most;
    vec = vec && aligned16(g.B, g.ldb, sizeof(T));
    vec_out = vec_out && aligned16(g.pre, c.ldz, sizeof(T));
  }
  a.R = c.R; a.ldc = c.ldc; a.ldr = c.ldr; a.ldz = c.ldz;
  a.C = (T *)c.C;
  a.res = (const T *)c.residual;
  a.rows = (int32_t)rows;
  a.act = c.act; a.bias_along = c.bias_along;
  a.vec_out = vec_out;
  // (Weights of 1,600 entries a row go a worker to a row all the same.)
  const int64_t mean = nnz / (rows * a.nsrc);
  a.long_len = mean > 128 ? (int32_t)(4 * mean < kHugeRow ? 4 * mean : kHugeRow) : 512;
  most = most < cols ? most : cols;                          // a row's columns are distinct
  const bool huge = most > kHugeRow;
  a.huge_len = huge ? kHugeRow : 2147483647;
  constexpr int V = 16 / sizeof(T);
  if (vec && c.R >= V) return gather_width<T, V, true>(ctx, a, nnz, huge, s);
  return c.R >= 8 ? gather_width<T, 4, false>(ctx, a, nnz, huge, s) : gather_width<T, 1, false>(ctx, a, nnz, huge, s);
}

}  // namespace comet
