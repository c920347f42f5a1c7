// What the tensor-core products spread (layer_tile_product.cu): a matrix's entries by 128 x 64 tiles instead of by rows. An entry becomes one 32-bit word, its
// 16-bit value below and its place in the tile's shared-memory image (swizzled, in bytes) above, and a tile's words lie together, in any
// order. Spreading is then a load, a shift and a store per entry at full width. Three passes:
//
//   starts  starts[i][b] = the first entry of row i at or beyond block b of k: a warp walks a row, and its lanes write where blocks change
//   shifts  the words of tile (t, b) begin behind those of the strip's rows in earlier blocks: bases[t][b] = pos[first row] + sum over the
//           strip's 128 rows of starts[i][b] - pos[i], no scan over tiles; within it row by row. What has to be added to an entry's
//           number to get its word's goes beside the starts, in the second half of the row's words
//   words   a warp walks a row again, 32 entries at a time, and every lane puts its word where it belongs
//
// (Spreading rows' pieces in the product kernel, 8 lanes to a row, took 1,230 cycles for a block of 820 entries, 2,900 instructions, where the block's
// products take 512, and writing words piece by piece 67 us for 6.5 M entries; a row's pieces are too short for either.)
#include "layer_tile.cuh"

namespace comet {
namespace {

constexpr int kListThreads = 256, kListWarps = kListThreads / 32, kAhead = 4;

struct ListArgs {
  struct Source {
    const int32_t *pos, *crd, *pick;
    const uint16_t *val;
    int32_t *starts, *bases;                               // starts: pitch words a row
    uint32_t *words;
  } src[2];
  int32_t rows, k_blocks;
  int64_t pitch;
};

__global__ void __launch_bounds__(kListThreads) tile_starts_kernel(const ListArgs a) {
  const ListArgs::Source &s = a.src[blockIdx.y];
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kListWarps + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const int32_t beg = __ldg(s.pos + row), end = __ldg(s.pos + row + 1);
  int32_t *starts = s.starts + row * a.pitch;
  int32_t last = -1;                                       // block of the entry before
  int32_t next[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) next[j] = (int64_t)beg + 32 * j + lane < end ? __ldg(s.crd + beg + 32 * j + lane) : 0;
  for (int64_t i = beg; i < end; i += 32 * kAhead) {
    int32_t now[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      now[j] = next[j];
      const int64_t q = i + 32 * (kAhead + j) + lane;
      next[j] = q < end ? __ldg(s.crd + q) : 0;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t first = i + 32 * j;
      if (first >= end) break;
      const int32_t b = min(now[j] >> 6, a.k_blocks - 1);
      int32_t before = __shfl_up_sync(0xffffffffu, b, 1);
      if (lane == 0) before = last;
      if (first + lane < end)
        for (int32_t k = before + 1; k <= b; ++k) starts[k] = (int32_t)first + lane;
      last = __shfl_sync(0xffffffffu, b, (int)min((int64_t)31, end - first - 1));
    }
  }
  for (int32_t k = last + 1 + lane; k <= a.k_blocks; k += 32) starts[k] = end;
}

// A CTA per strip and 32 blocks of k: a lane per block, a warp for 16 of the strip's rows.
__global__ void __launch_bounds__(kListThreads) tile_shifts_kernel(const ListArgs a) {
  const ListArgs::Source &s = a.src[blockIdx.z];
  __shared__ int32_t front[kListWarps][32], words[kListWarps][32];
  constexpr int kRows = 128 / kListWarps;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t b = (int32_t)blockIdx.y * 32 + lane;
  const int64_t row0 = (int64_t)blockIdx.x * 128, first = row0 + warp * kRows;
  const bool have = b <= a.k_blocks;
  int32_t start[kRows], n[kRows], sum = 0, before = 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const bool row = have && first + r < a.rows;
    const int32_t *p = s.starts + (first + r) * a.pitch + b;
    start[r] = row ? p[0] : 0;
    const int32_t end = row && b < a.k_blocks ? p[1] : start[r];
    before += row ? start[r] - __ldg(s.pos + first + r) : 0;
    n[r] = end - start[r];
    sum += n[r];
  }
  front[warp][lane] = before;
  words[warp][lane] = sum;
  __syncthreads();
  int32_t base = __ldg(s.pos + row0);
  for (int w = 0; w < kListWarps; ++w) base += front[w][lane];
  if (warp == 0 && have) s.bases[(int64_t)blockIdx.x * (a.k_blocks + 1) + b] = base;
  for (int w = 0; w < warp; ++w) base += words[w][lane];
  if (!have) return;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (first + r < a.rows) s.starts[(first + r) * a.pitch + a.pitch / 2 + b] = base - start[r];
    base += n[r];
  }
}

__global__ void __launch_bounds__(kListThreads) tile_words_kernel(const ListArgs a) {
  const ListArgs::Source &s = a.src[blockIdx.y];
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kListWarps + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const int32_t beg = __ldg(s.pos + row), end = __ldg(s.pos + row + 1);
  const int32_t *shift = s.starts + row * a.pitch + a.pitch / 2;
  const uint32_t r = (uint32_t)row & 127u, line = r * 128, twist = (r & 7u) << 4;
  for (int64_t i = beg; i < end; i += 32 * kAhead) {
    int32_t c[kAhead], to[kAhead], at[kAhead];
    uint32_t v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t p = i + 32 * j + lane;
      c[j] = p < end ? __ldg(s.crd + p) : 0;
      at[j] = p < end ? (s.pick ? __ldg(s.pick + p) : (int32_t)p) : 0;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      v[j] = __ldg(s.val + at[j]);
      to[j] = __ldg(shift + min(c[j] >> 6, a.k_blocks - 1));
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t p = i + 32 * j + lane;
      if (p < end) s.words[p + to[j]] = (line + ((((uint32_t)c[j] & 63u) << 1) ^ twist)) << 16 | v[j];
    }
  }
}

struct ListSizes {
  size_t words, starts, bases;
  int64_t pitch;
  explicit ListSizes(const RowView &A) {
    const int64_t blocks = ceil_div(A.cols, 64) + 1;
    pitch = 2 * (int64_t)align_up((size_t)blocks, 8);      // a row's starts, then its shifts
    words = align_up((size_t)A.nnz * 4, 256);
    starts = align_up((size_t)A.rows * (size_t)pitch * 4, 256);
    bases = align_up((size_t)ceil_div(A.rows, 128) * (size_t)blocks * 4, 256);
  }
};

}  // namespace

bool tile_lists_fit(const RowView &A) { return A.cols <= (65535ll * 32 - 1) * 64; }      // 32 starts of blocks of 64 columns for each blockIdx.y

size_t tile_list_bytes(const RowView &A) {
  const ListSizes z(A);
  return z.words + z.starts + z.bases;
}

comet_status_t tile_lists(Context *ctx, const RowView *A, const int32_t *const *pick, int sources, char *const *mem, TileList *lists, cudaStream_t s) {
  ListArgs a{};
  a.rows = (int32_t)A[0].rows;
  a.k_blocks = (int32_t)ceil_div(A[0].cols, 64);
  for (int q = 0; q < sources; ++q) {
    const ListSizes z(A[q]);
    a.pitch = z.pitch;
    a.src[q] = {A[q].pos, A[q].crd, pick[q], (const uint16_t *)A[q].val, (int32_t *)(mem[q] + z.words), (int32_t *)(mem[q] + z.words + z.starts),
                (uint32_t *)mem[q]};
    lists[q] = TileList{a.src[q].words, a.src[q].bases};
  }
  const dim3 rows((unsigned)ceil_div(a.rows, kListWarps), (unsigned)sources);
  tile_starts_kernel<<<rows, kListThreads, 0, s>>>(a);
  COMET_LAUNCH_CHECK(ctx);                                 // each pass trusts what the one before it wrote
  tile_shifts_kernel<<<dim3((unsigned)ceil_div(a.rows, 128), (unsigned)ceil_div(a.k_blocks + 1, 32), (unsigned)sources), kListThreads, 0, s>>>(a);
  COMET_LAUNCH_CHECK(ctx);
  tile_words_kernel<<<rows, kListThreads, 0, s>>>(a);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

}  // namespace comet
