// The product of two dense matrices sampled at a sparse matrix's cells: out[p] = sum over r of P[row of p, r] * Q[crd[p], r]. It is the
// gradient of the stored values of a sparse x dense product (P = the result's gradient, Q = the dense operand).
//
// A warp owns a run of stored entries, wherever rows begin and end in it, so that heavy rows need no care. W lanes take an entry's dot product
// (16 bytes of both rows a lane), 32 / W entries side by side, `kDeep` deep; the lanes' sums are joined by shuffles. The row of an entry is found
// from the 32 row ends that follow the run's current row. What bounds it is the gathers of Q's rows; P's row is the same for the entries of a
// row and comes from L1. Every output value has one writer and a fixed order of its sum.
#include "kernels.cuh"
#include "layer.cuh"

namespace comet {
namespace {

constexpr int kSampleThreads = 256;
// Entries of a group at a time, and CTAs that an SM is to hold beside each other: as many registers as eight (fp64: four) rows of Q take.
template <class T> constexpr int kMany = sizeof(T) == 8 ? 4 : 8;
template <class T> constexpr int kResident = sizeof(T) == 8 ? 3 : 4;

template <class T> struct SampleArgs {
  const int32_t *pos, *crd;
  const T *P, *Q;
  int64_t ldp, ldq, R, nnz;
  T *out;
  int32_t rows, run;       // entries per warp, a multiple of 32
  int log_w;
};

// Row of entry x: the last row whose first entry is at or before x, among [lo, rows).
__device__ __forceinline__ int32_t row_of(const int32_t *__restrict__ pos, int32_t lo, int32_t rows, int32_t x) {
  int32_t hi = rows;                                         // pos[lo] <= x < pos[hi]
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (__ldg(pos + mid) <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The same by a whole warp: 32 probes a round.
__device__ __forceinline__ int32_t row_of_warp(const int32_t *__restrict__ pos, int32_t rows, int32_t x) {
  int32_t lo = 0, hi = rows;                                 // pos[lo] <= x < pos[hi]
  const int lane = threadIdx.x & 31;
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 31) / 32;
    const int64_t at = (int64_t)lo + (int64_t)lane * step;
    const bool before = at < hi && __ldg(pos + at) <= x;     // holds for lane 0
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, before));
    lo += last * step;
    hi = (int32_t)min((int64_t)hi, (int64_t)lo + step);
  }
  return lo;
}

template <class T, int V, bool VEC>
__device__ __forceinline__ void load_piece(const T *p, int64_t col, int64_t R, int apart, T (&x)[V]) {
  if (VEC && col + V <= R) {
    Piece<T> q;
    q.raw = __ldg(reinterpret_cast<const uint4 *>(p + col));
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = q.at[VEC ? v : 0];
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = col + (int64_t)v * apart < R ? p[col + (int64_t)v * apart] : (T)0.0f;
  }
}

template <class T, int V, bool VEC, int kDeep>
__global__ void __launch_bounds__(kSampleThreads, kResident<T>) layer_sample_kernel(const SampleArgs<T> a) {
  using acc_t = typename Num<T>::acc;
  using sum_t = typename Num<T>::sum;
  const int W = 1 << a.log_w, G = 32 >> a.log_w;
  const int at = threadIdx.x & 31, group = at >> a.log_w, l = at & (W - 1);
  const int64_t warp = (int64_t)blockIdx.x * (kSampleThreads / 32) + (threadIdx.x >> 5);
  const int64_t begin = warp * a.run, end = min(a.nnz, begin + a.run);
  if (begin >= end) return;
  const int apart = VEC ? 1 : W;
  const int64_t stride = (int64_t)W * V, col0 = VEC ? (int64_t)l * V : l;
  int32_t row0 = row_of_warp(a.pos, a.rows, (int32_t)begin);
  for (int64_t base = begin; base < end; base += 32) {
    // this lane's entry: its column and its row
    const int64_t mine = base + at;
    const bool have = mine < end;
    const int32_t c = have ? __ldg(a.crd + mine) : 0;
    const int64_t e = (int64_t)row0 + 1 + at;
    const int32_t row_end = e <= a.rows ? __ldg(a.pos + e) : 2147483647;     // where row row0 + at ends
    const int32_t last = (int32_t)min(base + 31, end - 1);
    int32_t row;
    if (__shfl_sync(0xffffffffu, row_end, 31) > last) {                      // the chunk's rows all end among the 32
      int before = 0;                                                        // how many of the 32 rows end at or before this entry
#pragma unroll
      for (int half = 16; half >= 1; half >>= 1) {
        const int32_t v = __shfl_sync(0xffffffffu, row_end, before + half - 1);
        if (v <= (int32_t)min(mine, end - 1)) before += half;
      }
      row = row0 + before;
    } else {
      row = row_of(a.pos, row0, a.rows, (int32_t)min(mine, end - 1));
    }
    row0 = __shfl_sync(0xffffffffu, row, 31);
    if constexpr (kDeep > 1) {
      // kDeep entries of a group at a time (W >= kDeep); their sums change hands while they are joined, so that the lanes end up with an entry for each
      // W / kDeep of them (with 8: 7 + log2(W / 8) exchanges for eight sums instead of 8 log2(W)).
      for (int k = 0; k < W; k += kDeep) {
        if (base + (int64_t)k * G >= end) break;
        acc_t dot[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) dot[u] = (acc_t)0;
        const int from = k * G + group;
        sum_t wide[kDeep];
        int rounds = 0;
        for (int64_t col = col0; col - col0 < a.R; col += stride, ++rounds) {  // the same number of rounds for every lane
          T y[kDeep][V];
#pragma unroll
          for (int u = 0; u < kDeep; ++u) load_piece<T, V, VEC>(a.Q + (int64_t)__shfl_sync(0xffffffffu, c, from + u * G) * a.ldq, col, a.R, apart, y[u]);
#pragma unroll
          for (int u = 0; u < kDeep; ++u) {
            T x[V];
            load_piece<T, V, VEC>(a.P + (int64_t)__shfl_sync(0xffffffffu, row, from + u * G) * a.ldp, col, a.R, apart, x);
#pragma unroll
            for (int v = 0; v < V; ++v) dot[u] += widen(x[v]) * widen(y[u][v]);
          }
          if ((rounds & 15) == 15) {                                           // at most 16 V terms in the narrower type
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
              wide[u] = rounds == 15 ? (sum_t)dot[u] : wide[u] + (sum_t)dot[u];
              dot[u] = (acc_t)0;
            }
          }
        }
        if (rounds >= 16) {
#pragma unroll
          for (int u = 0; u < kDeep; ++u) dot[u] = (acc_t)(wide[u] + (sum_t)dot[u]);
        }
#pragma unroll
        for (int half = kDeep / 2; half >= 1; half >>= 1) {
          const int off = W * half / kDeep;                                    // W / 2, W / 4, ..
          const bool upper = (l & off) != 0;
#pragma unroll
          for (int u = 0; u < half; ++u) {
            const acc_t give = upper ? dot[u] : dot[u + half], keep = upper ? dot[u + half] : dot[u];
            dot[u] = keep + __shfl_xor_sync(0xffffffffu, give, off);
          }
        }
        for (int off = W / (2 * kDeep); off >= 1; off >>= 1) dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], off);
        const int64_t at_entry = base + (k + l / (W / kDeep)) * G + group;         // the lane's bits from the top chose the halves
        if (l % (W / kDeep) == 0 && at_entry < end) a.out[at_entry] = narrow<T, acc_t>(dot[0]);
      }
      continue;
    }
    // One to four lanes to an entry.
    sum_t result = (sum_t)0;                                                 // of this lane's entry
    for (int k = 0; k < W; ++k) {
      const int from = k * G + group;
      const T *p = a.P + (int64_t)__shfl_sync(0xffffffffu, row, from) * a.ldp, *q = a.Q + (int64_t)__shfl_sync(0xffffffffu, c, from) * a.ldq;
      sum_t dot = (sum_t)0;
      for (int64_t col = col0; col - col0 < a.R; col += stride) {
        T x[V], y[V];
        load_piece<T, V, VEC>(q, col, a.R, apart, y);
        load_piece<T, V, VEC>(p, col, a.R, apart, x);
        acc_t t = (acc_t)0;
#pragma unroll
        for (int v = 0; v < V; ++v) t += widen(x[v]) * widen(y[v]);
        dot += (sum_t)t;
      }
      for (int off = 1; off < W; off <<= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
      // entry k * G + g belongs to the lane of that number; its sum sits in every lane of group g
      const int j = at - k * G;
      const sum_t got = __shfl_sync(0xffffffffu, dot, (j >= 0 && j < G ? j : 0) << a.log_w);
      if (j >= 0 && j < G) result = got;
    }
    if (have) a.out[mine] = narrow<T, acc_t>((acc_t)result);
  }
}

template <class T, int V, bool VEC> comet_status_t sample_launch(Context *ctx, SampleArgs<T> &a, cudaStream_t s) {
  a.log_w = 0;
  while (a.log_w < 5 && ((int64_t)V << a.log_w) < a.R) ++a.log_w;
  // runs of up to 256 entries, shorter where there would not be 32 warps for every SM
  int64_t run = align_up((size_t)ceil_div(a.nnz, (int64_t)kSmCount * 32), 32);
  a.run = (int32_t)(run > 256 ? 256 : run);
  const int64_t blocks = ceil_div(ceil_div(a.nnz, a.run), kSampleThreads / 32);
  if (a.log_w >= 3) layer_sample_kernel<T, V, VEC, kMany<T>><<<(unsigned)blocks, kSampleThreads, 0, s>>>(a);
  else if (a.log_w == 2) layer_sample_kernel<T, V, VEC, 4><<<(unsigned)blocks, kSampleThreads, 0, s>>>(a);
  else layer_sample_kernel<T, V, VEC, 1><<<(unsigned)blocks, kSampleThreads, 0, s>>>(a);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

template <class T> comet_status_t sample_typed(Context *ctx, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R,
                                               void *out, cudaStream_t s) {
  SampleArgs<T> a{};
  a.pos = A.pos; a.crd = A.crd;
  a.P = (const T *)P; a.Q = (const T *)Q;
  a.ldp = ldp; a.ldq = ldq; a.R = R; a.nnz = A.nnz;
  a.out = (T *)out;
  a.rows = (int32_t)A.rows;
  constexpr int V = 16 / sizeof(T);
  const auto ok = [](const void *p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * (int64_t)sizeof(T)) % 16 == 0; };
  if (R >= V && ok(P, ldp) && ok(Q, ldq)) return sample_launch<T, V, true>(ctx, a, s);
  return R >= 8 ? sample_launch<T, 4, false>(ctx, a, s) : sample_launch<T, 1, false>(ctx, a, s);
}

}  // namespace

comet_status_t layer_sample(Context *ctx, int dtype, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R,
                            void *out, cudaStream_t s) {
  if (A.nnz == 0) return COMET_OK;
  switch (dtype) {
    case COMET_F64: return sample_typed<double>(ctx, A, P, ldp, Q, ldq, R, out, s);
    case COMET_F32: return sample_typed<float>(ctx, A, P, ldp, Q, ldq, R, out, s);
    case COMET_BF16: return sample_typed<__nv_bfloat16>(ctx, A, P, ldp, Q, ldq, R, out, s);
    default: return sample_typed<__half>(ctx, A, P, ldp, Q, ldq, R, out, s);
  }
}

}  // namespace comet
