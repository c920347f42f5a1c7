// The sparse x dense product with its epilogue on the tensor cores: 16-bit values, matrices that are dense enough (pruned weights), 8 or more
// columns. The stored cells of a 128 x 64 block of A are written into a zeroed tile of shared memory and multiplied as a dense tile, so
// that every entry is read once per block of up to 256 columns and a row of B serves 128 rows of A from shared memory, where the gathers
// fetch it once per entry. Ordered rows only: a cell has one place in the tile.
//
//   D[128 x N] += A_tile[128 x 64] B_tile[64 x N]        kind::f16, fp32 accumulators in tensor memory; two of them for the gated pair
//
// A CTA is eighteen warps: one thread copies B's tiles by tensor map, one issues the products, sixteen warps spread A's entries, listed by
// tiles beforehand (layer_tile_list.cu), and afterwards apply the epilogue, a lane per row. Stages of (A tiles, B tile) go round a ring. Where there are few tiles the blocks of k are split
// over the CTAs of a cluster, which add their accumulators through distributed shared memory in the order of the ranks.
// An unstored cell is a zero here, and 0 * inf is NaN: an element whose sum is not finite is computed again over its stored cells alone.
#include <cooperative_groups.h>

#include "layer_tile.cuh"

#include <stdlib.h>

namespace cg = cooperative_groups;

namespace comet {
namespace {

constexpr int kTileRows = 128, kTileK = 64, kPitch = kTileRows + 1;
constexpr int kTileWarps = 18;                                 // copies, products, and 16 spreading warps
constexpr int kATile = kTileRows * kTileK * 2;                 // bytes
constexpr int kTileSmem = 226 * 1024;                          // most dynamic shared memory asked for

template <class T> struct TileArgs {
  struct Source { const int32_t *pos, *crd, *pick; const T *val; const T *B; int64_t ldb; const T *bias; T *pre; TileList list; } src[2];
  int64_t R, ldc, ldr, ldz;
  T *C;
  const T *res;
  int32_t rows, k_blocks, steps;        // k_blocks: blocks of 64 along one matrix's columns; steps: of all products of a tile
  int nsrc, n, stages, act, bias_along;
  bool vec_out;
  int32_t *status;
  int64_t patience;
};

// sum over row i's stored cells, column r, of one source
template <class T> __device__ __noinline__ float stored_dot(const typename TileArgs<T>::Source &s, int64_t i, int64_t r) {
  float sum = 0.0f;
  for (int32_t p = s.pos[i]; p < s.pos[i + 1]; ++p) sum += widen(s.val[s.pick ? s.pick[p] : p]) * widen(s.B[(int64_t)s.crd[p] * s.ldb + r]);
  return sum;
}

template <class T> __device__ __forceinline__ void residual4(const TileArgs<T> &a, int64_t i, int64_t col, int64_t limit, T (&res)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) res[j] = a.res && i < a.rows && col + 32 * j < limit ? a.res[i * a.ldr + col + 32 * j] : (T)0.0f;
}
// Any alignment: a lane's four columns col, col + 32, .. of a row, as far as they lie before `limit`; a warp's lanes have neighbouring ones.
template <class T, int NACC> __device__ __forceinline__ void finish4(const TileArgs<T> &a, int64_t i, int64_t col, int64_t limit, float (&z)[NACC][4], const T (&res)[4]) {
#pragma unroll
  for (int q = 0; q < NACC; ++q) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = col + 32 * j;
      if (at >= limit) continue;
      if (!isfinite(z[q][j])) {
        z[q][j] = stored_dot<T>(a.src[q], i, at);
        if (NACC == 1 && a.nsrc == 2) z[q][j] += stored_dot<T>(a.src[1], i, at);
      }
      if (a.src[q].bias) z[q][j] += widen(a.src[q].bias[a.bias_along == COMET_BIAS_ROWS ? i : at]);
      if (a.src[q].pre) a.src[q].pre[i * a.ldz + at] = narrow<T, float>(z[q][j]);
    }
  }
  activate_all<true>(a.act, z[0]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (col + 32 * j >= limit) continue;
    float y = z[0][j];
    if (NACC == 2) y *= z[NACC - 1][j];
    if (a.res) y += widen(res[j]);
    a.C[i * a.ldc + col + 32 * j] = narrow<T, float>(y);
  }
}

// The rows of a tile by the sixteen warps, eight each: `cols` columns from `col` on, whose sums lie at sums[(q * apart + c) * kPitch + row].
template <class T, int NACC>
__device__ __forceinline__ void finish_rows(const TileArgs<T> &a, int64_t row0, int64_t col, int cols, const float *sums, int apart) {
  constexpr int kEach = kTileRows / (kTileWarps - 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t limit = min(a.R, col + cols);
  for (int c = lane; col + c - lane < limit; c += 128) {
    T res[kEach][4];
#pragma unroll
    for (int k = 0; k < kEach; ++k) residual4<T>(a, row0 + (warp - 2) * kEach + k, col + c, limit, res[k]);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int r = (warp - 2) * kEach + k;
      if (row0 + r >= a.rows) break;
      float z[NACC][4];
#pragma unroll
      for (int q = 0; q < NACC; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[q][j] = c + 32 * j < cols ? sums[(q * apart + c + 32 * j) * kPitch + r] : 0.0f;
      finish4<T, NACC>(a, row0 + r, col + c, limit, z, res[k]);
    }
  }
}

template <class T> __device__ __forceinline__ void write16(T *to, const float (&x)[16], int live) {
  uint32_t w[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) w[v] = narrow2(x[2 * v], x[2 * v + 1], T());
  if (live == 16) {
    reinterpret_cast<uint4 *>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4 *>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (v < live) reinterpret_cast<uint16_t *>(to)[v] = (uint16_t)(v & 1 ? w[v / 2] >> 16 : w[v / 2]);
  }
}

// Sixteen columns of one row; everything that is read or written starts on 16 bytes.
template <class T, int NACC> __device__ __forceinline__ void finish16(const TileArgs<T> &a, int64_t i, int64_t col, float (&z)[NACC][16]) {
  const int live = (int)min((int64_t)16, a.R - col);
  if (i >= a.rows || live <= 0) return;
  Piece<T> res[2];
  const bool whole = live == 16;
  if (a.res && whole) {
    res[0].raw = __ldg(reinterpret_cast<const uint4 *>(a.res + i * a.ldr + col));
    res[1].raw = __ldg(reinterpret_cast<const uint4 *>(a.res + i * a.ldr + col + 8));
  }
#pragma unroll
  for (int q = 0; q < NACC; ++q) {
    float odd = 0.0f;                                      // stays zero unless a value is not finite
#pragma unroll
    for (int v = 0; v < 16; ++v) odd = fmaf(z[q][v], 0.0f, odd);
    if (odd != 0.0f) {
#pragma unroll 1
      for (int v = 0; v < live; ++v) {
        float x = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) x = k == v ? z[q][k] : x;
        if (isfinite(x)) continue;
        x = stored_dot<T>(a.src[q], i, col + v);
        if (NACC == 1 && a.nsrc == 2) x += stored_dot<T>(a.src[1], i, col + v);
#pragma unroll
        for (int k = 0; k < 16; ++k) z[q][k] = k == v ? x : z[q][k];
      }
    }
    if (a.src[q].bias) {
      if (a.bias_along == COMET_BIAS_ROWS) {
        const float b = widen(a.src[q].bias[i]);
#pragma unroll
        for (int v = 0; v < 16; ++v) z[q][v] += b;
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) z[q][v] += v < live ? widen(a.src[q].bias[col + v]) : 0.0f;
      }
    }
    if (a.src[q].pre) write16<T>(a.src[q].pre + i * a.ldz + col, z[q], live);
  }
  activate_all<true>(a.act, z[0]);
  if (NACC == 2) {
#pragma unroll
    for (int v = 0; v < 16; ++v) z[0][v] *= z[NACC - 1][v];
  }
  if (a.res) {
#pragma unroll
    for (int v = 0; v < 16; ++v) z[0][v] += whole ? widen(res[v / 8].at[v % 8]) : v < live ? widen(a.res[i * a.ldr + col + v]) : 0.0f;
  }
  write16<T>(a.C + i * a.ldc + col, z[0], live);
}

// Spreads the words of one matrix's tiles over zeroed A tiles: four warps, every kTurns-th block of k, with the words of their next block in registers.
template <int kWords> struct Spreader {
  const uint32_t *words;
  const int32_t *bases;                                    // of this strip
  uint32_t w[kWords];
  int32_t at, end;                                         // of the tile whose words are held; w[j] is word at + 128 j + thread
  __device__ __forceinline__ void read(int32_t block, int thread) {
    at = __ldg(bases + block) + thread;
    end = __ldg(bases + block + 1);
#pragma unroll
    for (int j = 0; j < kWords; ++j)
      if (at + 128 * j < end) w[j] = __ldg(words + at + 128 * j);
  }
  __device__ __forceinline__ void put(uint32_t tile, uint32_t word) const {
    // (Inside the tile whatever the word: a descriptor that was not validated may leave words unwritten.)
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(tile + (word >> 16 & (uint32_t)(kATile - 2))), "h"((uint16_t)word) : "memory");
  }
  __device__ __forceinline__ void spread(uint32_t tile) const {
#pragma unroll
    for (int j = 0; j < kWords; ++j)
      if (at + 128 * j < end) put(tile, w[j]);
    for (int32_t i = at + 128 * kWords; i < end; i += 128) put(tile, __ldg(words + i));
  }
};

// A place in the ring of stages: its number and the parity of the round.
struct Place {
  int stage = 0;
  uint32_t round = 0;
  __device__ __forceinline__ void next(int stages, int by = 1) {
    stage += by;
    if (stage >= stages) {         // by <= stages
      stage -= stages;
      ++round;
    }
  }
};

template <class T, int NACC, int kWords>
__global__ void __launch_bounds__(kTileWarps * 32, 1) tile_product_kernel(const __grid_constant__ CUtensorMap map0, const __grid_constant__ CUtensorMap map1,
                                                                          const __grid_constant__ TileArgs<T> a) {
  extern __shared__ char raw_smem[];
  __shared__ uint64_t bars[3 * 8 + 1];
  __shared__ uint32_t tmem_at;
  __shared__ int failed;
  char *smem = reinterpret_cast<char *>(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = a.n, stages = a.stages, stage_bytes = NACC * kATile + kTileK * 2 * n;
  // Of a stage: A's tiles spread, B's tile landed, products done with both.
  const uint32_t full = smem_u32(bars), landed = full + 8 * stages, empty = full + 16 * stages, done = full + 24 * stages;
  int32_t issued = 0;                                          // copies, in the thread that issues them
  const int split = gridDim.z, rank = blockIdx.z;
  const int32_t from = (int32_t)((int64_t)a.steps * rank / split), to = (int32_t)((int64_t)a.steps * (rank + 1) / split);
  const int64_t row0 = (int64_t)blockIdx.x * kTileRows, col0 = (int64_t)blockIdx.y * n;
  uint32_t columns = 32;
  while (columns < (uint32_t)(NACC * n)) columns <<= 1;

  if (threadIdx.x == 0) {
    failed = a.patience <= 0;
    for (int s = 0; s < stages; ++s) {
      bar_init(full + 8 * s, 4 * NACC);
      bar_init(landed + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    bar_init(done, 1);
    fence_bar_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_at), columns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t d = tmem_at;

  if (warp == 0) {
    if (lane == 0) {
      Place at;
      for (int32_t t = from; t < to; ++t, ++issued, at.next(stages)) {
        if (at.round > 0 && !bar_wait(empty + 8 * at.stage, (at.round - 1) & 1, &failed, a.patience)) break;
        const bool second = t >= a.k_blocks;
        const int32_t block = second ? t - a.k_blocks : t;
        const uint32_t bar = landed + 8 * at.stage, b = smem_u32(smem + at.stage * stage_bytes + NACC * kATile);
        bar_expect(bar, (uint32_t)(kTileK * 2 * n));
        for (int j = 0; j < n / 64; ++j) copy_box(b + j * (64 * kTileK * 2), second ? &map1 : &map0, (int)col0 + j * 64, block * kTileK, bar);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t kind = product_kind(Num<T>::is_bf16, true, kTileRows, n);
      Place at;
      for (int32_t t = from; t < to; ++t, at.next(stages)) {
        if (!bar_wait(landed + 8 * at.stage, at.round & 1, &failed, a.patience) || !bar_wait(full + 8 * at.stage, at.round & 1, &failed, a.patience)) break;
        tc_fence_after();
        const uint32_t tile = smem_u32(smem + at.stage * stage_bytes);
        const uint64_t b = operand_at(tile + NACC * kATile, 64 * kTileK * 2, 1024);
#pragma unroll
        for (int q = 0; q < NACC; ++q) {
          const uint64_t x = operand_at(tile + q * kATile, 16, 1024);
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k)
            tc_product(d + q * n, x + k * 2, b + k * 128, kind, t > from || k > 0);       // 32 bytes along A's rows, 16 rows of B
        }
        tc_commit(empty + 8 * at.stage);
      }
      tc_commit(done);
    }
  } else {
    // groups of four warps; those of one matrix take turns at its blocks
    constexpr int kTurns = 4 / NACC;
    const int group = (warp - 2) >> 2, q = NACC == 2 ? group >> 1 : 0, turn = NACC == 2 ? group & 1 : group, thread = (warp - 2 & 3) * 32 + lane;
    Spreader<kWords> e;
    int source = -1;
    Place at;
    for (int k = 0; k < turn; ++k) at.next(stages);
    for (int32_t t = from + turn; t < to; t += kTurns) {
      const bool second = NACC == 1 && t >= a.k_blocks;
      const int now = NACC == 2 ? q : second;
      const int32_t block = second ? t - a.k_blocks : t;
      if (now != source) {
        source = now;
        e.words = a.src[now].list.words;
        e.bases = a.src[now].list.bases + (int64_t)blockIdx.x * (a.k_blocks + 1);
        e.read(block, thread);
      }
      // (A wait that has run out does not leave the loop: the group's other warps may be at its barrier. From then on no wait takes time.)
      const bool go = at.round == 0 || bar_wait_warp(empty + 8 * at.stage, (at.round - 1) & 1, &failed, a.patience);
      const uint32_t tile = smem_u32(smem + at.stage * stage_bytes + q * kATile);
#pragma unroll
      for (int k = 0; k < 8 && go; ++k)
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (k * 128 + thread) * 16), "r"(0) : "memory");
      asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
      if (go) e.spread(tile);
      if (t + kTurns < to && block + kTurns < a.k_blocks) e.read(block + kTurns, thread);
      else source = -1;                                      // the next one, if any, is of another matrix
      fence_async_smem();
      __syncwarp();
      if (lane == 0 && go) bar_arrive(full + 8 * at.stage);
      for (int k = 0; k < kTurns; ++k) at.next(stages);
    }
  }

  // A spreading warp reads the accumulators of 32 rows (a lane each), each kParts-th group of 16 columns.
  __syncwarp();
  const bool over = bar_wait_warp(done, 0, &failed, a.patience), ok = over && !__any_sync(0xffffffffu, failed);
  if (warp == 1 && !over) bar_wait_end(done, 0);               // the products in flight, before tensor memory and stages go
  tc_fence_after();
  constexpr int kParts = (kTileWarps - 2) / 4;
  const int quarter = warp & 3, part = (warp - 2) >> 2;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const int64_t i = row0 + quarter * 32 + lane;
  float *sums = reinterpret_cast<float *>(smem);       // [NACC][columns][kPitch rows]: the stages are free
  if (split == 1 && a.vec_out) {
    if (warp >= 2 && ok) {
      for (int c = part * 16; c < n; c += 16 * kParts) {
        float z[NACC][16];
#pragma unroll
        for (int q = 0; q < NACC; ++q) tmem_load16(d + lanes + q * n + c, z[q]);
        finish16<T, NACC>(a, i, col0 + c, z);
      }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
      tc_fence_after();
      tmem_free(d, columns);
    }
  } else if (split == 1) {
    // Rows that do not start on 16 bytes: through shared memory, so that a warp writes a row's neighbouring elements together.
    const int chunk = min(n, 256 / NACC);
    for (int first = 0; first < n; first += chunk) {
      if (warp >= 2 && ok) {
        for (int c = part * 16; c < min(chunk, n - first); c += 16 * kParts) {
#pragma unroll
          for (int q = 0; q < NACC; ++q) {
            float x[16];
            tmem_load16(d + lanes + q * n + first + c, x);
#pragma unroll
            for (int v = 0; v < 16; ++v) sums[(q * chunk + c + v) * kPitch + quarter * 32 + lane] = x[v];
          }
        }
      }
      __syncthreads();
      if (warp >= 2 && ok) finish_rows<T, NACC>(a, row0, col0 + first, min(chunk, n - first), sums, chunk);
      tc_fence_before();
      __syncthreads();
      tc_fence_after();
    }
    if (warp == 1) tmem_free(d, columns);
  } else {
    // The cluster's CTAs put their accumulators into shared memory and each finishes a share of the columns. Tensor memory is given back first: no
    // CTA waits for another while it holds any, since that other one may wait for it.
    if (warp >= 2 && ok) {
      for (int c = part * 16; c < n; c += 16 * kParts) {
#pragma unroll
        for (int q = 0; q < NACC; ++q) {
          float x[16];
          tmem_load16(d + lanes + q * n + c, x);
#pragma unroll
          for (int v = 0; v < 16; ++v) sums[(q * n + c + v) * kPitch + quarter * 32 + lane] = x[v];
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
      tc_fence_after();
      tmem_free(d, columns);
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int share = n / split;
    if (warp >= 2 && ok) {
      for (int c = part * 16; c < share; c += 16 * kParts) {
        float z[NACC][16];
#pragma unroll
        for (int q = 0; q < NACC; ++q)
#pragma unroll
          for (int v = 0; v < 16; ++v) z[q][v] = 0.0f;
        for (int k = 0; k < split; ++k) {
          const float *there = cluster.map_shared_rank(sums, k);
#pragma unroll
          for (int q = 0; q < NACC; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] += there[(q * n + rank * share + c + v) * kPitch + quarter * 32 + lane];
        }
        if (a.vec_out) {
          finish16<T, NACC>(a, i, col0 + rank * share + c, z);
        } else {                                        // back into this CTA's own columns, which nobody else reads
#pragma unroll
          for (int q = 0; q < NACC; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) sums[(q * n + rank * share + c + v) * kPitch + quarter * 32 + lane] = z[q][v];
        }
      }
    }
    if (!a.vec_out) {
      __syncthreads();
      if (warp >= 2 && ok) finish_rows<T, NACC>(a, row0, col0 + rank * share, share, sums + rank * share * kPitch, n);
    }
    cluster.sync();                                     // nobody's shared memory goes while another reads it
  }
  if (threadIdx.x == 0 && failed) give_up(landed, stages, issued, a.status);
}

template <class T, int NACC, int kWords>
comet_status_t launch(Context *ctx, const CUtensorMap &m0, const CUtensorMap &m1, TileArgs<T> &a, int64_t row_tiles, int64_t col_tiles, int split, cudaStream_t s) {
  const int stage_bytes = NACC * kATile + kTileK * 2 * a.n;
  const int64_t steps_each = a.steps / split;
  a.stages = (kTileSmem - 1024) / stage_bytes;
  if (a.stages > 8) a.stages = 8;
  if (a.stages > steps_each + 1) a.stages = (int)steps_each + 1;
  if (a.stages < 2) a.stages = 2;
  size_t bytes = (size_t)a.stages * stage_bytes;
  const size_t join = split > 1 || !a.vec_out ? (size_t)(NACC * a.n < 256 ? NACC * a.n : 256) * kPitch * sizeof(float) : 0;
  if (join > bytes) bytes = join;
  bytes += 1024;
  auto *kernel = tile_product_kernel<T, NACC, kWords>;
  COMET_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileSmem));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)row_tiles, (unsigned)col_tiles, (unsigned)split);
  cfg.blockDim = dim3(kTileWarps * 32);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1; at.val.clusterDim.y = 1; at.val.clusterDim.z = (unsigned)split;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  COMET_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, kernel, m0, m1, a));
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

template <class T> comet_status_t product_typed(Context *ctx, const GatherCall &c, const TileList *lists, cudaStream_t s) {
  TileArgs<T> a{};
  a.nsrc = c.mode == kLayer ? 1 : 2;
  const auto ok16 = [](const void *p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && ld % 8 == 0); };
  a.vec_out = ok16(c.C, c.ldc) && ok16(c.residual, c.ldr);
  for (int q = 0; q < a.nsrc; ++q) {
    const GatherSource &g = c.src[q];
    a.src[q] = {g.A.pos, g.A.crd, g.pick, (const T *)g.A.val, (const T *)g.B, g.ldb, (const T *)g.bias, (T *)g.pre, lists[q]};
    a.vec_out = a.vec_out && ok16(g.pre, c.ldz);
  }
  a.R = c.R; a.ldc = c.ldc; a.ldr = c.ldr; a.ldz = c.ldz;
  a.C = (T *)c.C;
  a.res = (const T *)c.residual;
  a.rows = (int32_t)c.src[0].A.rows;
  a.act = c.act; a.bias_along = c.bias_along;
  a.status = ctx->h_pinned + kLayerStatusWord;
  a.patience = wait_patience();
  a.k_blocks = (int32_t)ceil_div(c.src[0].A.cols, kTileK);
  const bool gated = c.mode == kGated;
  a.steps = c.mode == kSumOfTwo ? 2 * a.k_blocks : a.k_blocks;
  // As few column tiles as 256 columns each allow, then of one width, in steps of 64.
  // (Two accumulators that a cluster joins have to fit shared memory: 128 columns each.)
  const int64_t groups = ceil_div(c.R, 64), row_tiles = ceil_div(a.rows, kTileRows);
  const int widest = gated && row_tiles * ceil_div(groups, 4) * 2 <= kSmCount ? 2 : 4;
  const int64_t col_tiles = ceil_div(groups, widest);
  a.n = (int)(ceil_div(groups, col_tiles) * 64);
  int split = 1;
  while (split < 8 && row_tiles * col_tiles * split * 2 <= kSmCount + kSmCount / 4 && a.steps / (split * 2) >= 8 && a.n % (split * 32) == 0 &&
         (gated ? 2 : 1) * a.n <= 256)
    split *= 2;
  CUtensorMap m0, m1;
  if (!tile_map(&m0, Num<T>::is_bf16, c.src[0].B, c.src[0].A.cols, c.R, c.src[0].ldb, kTileK)) return COMET_ERR_CUDA;
  m1 = m0;
  if (c.mode == kSumOfTwo && !tile_map(&m1, Num<T>::is_bf16, c.src[1].B, c.src[1].A.cols, c.R, c.src[1].ldb, kTileK)) return COMET_ERR_CUDA;
  // Words that a thread holds: 8 where a tile's mean number is up to 900, else 16.
  double nnz = 0;
  for (int q = 0; q < a.nsrc; ++q) nnz += (double)c.src[q].A.nnz;
  const bool few = nnz / ((double)a.nsrc * a.rows * a.k_blocks) * kTileRows <= 900;
  if (gated) return few ? launch<T, 2, 8>(ctx, m0, m1, a, row_tiles, col_tiles, split, s) : launch<T, 2, 16>(ctx, m0, m1, a, row_tiles, col_tiles, split, s);
  return few ? launch<T, 1, 8>(ctx, m0, m1, a, row_tiles, col_tiles, split, s) : launch<T, 1, 16>(ctx, m0, m1, a, row_tiles, col_tiles, split, s);
}

}  // namespace

// Tiles do the work of all cells, entries or not, in steps of 64 columns, behind some 25 us of listing; a worker per row does the entries' alone, at about 1.1 us
// a million of entries x columns. So tiles pay from 40 million of those on, where there is at least one for every cell, and 20 columns. Measured, tiles and
// rows, bf16, us: 10 % of 1728^2, 64 columns (19 M) 36 and 21, of 2496^2 (39 M) 39 and 45, of 3520^2 (77 M) 44 and 61; 40 %, 256 columns 36 and 34 at
// 15 M, 44 and 69 at 69 M; 2 % of 8192^2, 32 columns (0.6 a cell) 67 and 44, 48 columns (1.0) 68 and 75; 10 % of 8192^2, 16 columns 97
// and 82, 24 columns 99 and 143; 30 % of 4096^2, 16 columns 68 and 53, 24 columns 67 and 92; 1/64 of 4096^2, 512 columns 52 and 112.
// Below 1/64 of the cells the lists outgrow the entries.
static bool enough_work(double nnz, double cells, int64_t R) {
  const double work = nnz * (double)R;
  if (const char *e = getenv("COMET_LAYER_TILE_WORK")) return work >= atof(e);
  return work >= 40e6 && work >= cells && R >= 20;
}

bool tile_product_fits(int dtype, const GatherCall &c) {
  if (dtype != COMET_BF16 && dtype != COMET_F16) return false;
  if (c.R < 8 || c.R > 65535ll * 64) return false;         // column tiles are counted by blockIdx.y
  const int n = c.mode == kLayer ? 1 : 2;
  double nnz = 0, cells = 0;
  for (int q = 0; q < n; ++q) {
    const GatherSource &g = c.src[q];
    if (!g.A.ordered || !tile_lists_fit(g.A)) return false;
    nnz += (double)g.A.nnz;
    cells += (double)g.A.rows * (double)g.A.cols;
  }
  return cells > 0 && nnz < 2147480000.0 && nnz * 64 >= cells && enough_work(nnz, cells, c.R);
}

comet_status_t tile_product(Context *ctx, int dtype, const GatherCall &c, const TileList *lists, cudaStream_t s) {
  return dtype == COMET_BF16 ? product_typed<__nv_bfloat16>(ctx, c, lists, s) : product_typed<__half>(ctx, c, lists, s);
}

}  // namespace comet
