// The sparse x dense product with its epilogue on the tensor cores: 16-bit values, matrices that are dense enough (pruned weights), 8 or more
// columns. The stored cells of a 128 x 64 block of A are written into a zeroed tile of shared memory and multiplied as a dense tile, so
// that every entry is read once per block of up to 256 columns and a row of B serves 128 rows of A from shared memory, where the gathers
// fetch it once per entry.
//
//   D[128 x N] += A_tile[128 x 64] B_tile[64 x N]        kind::f16, fp32 accumulators in tensor memory; two of them for the gated pair
//
// A CTA is ten warps: one thread copies B's tiles by tensor map, one issues the products, eight warps spread A's entries, 8 lanes to a row, and
// afterwards apply the epilogue, a lane per row. Stages of (A tiles, B tile) go round a ring. Where there are few tiles the blocks of k are split
// over the CTAs of a cluster, which add their accumulators through distributed shared memory in the order of the ranks.
// An unstored cell is a zero here, and 0 * inf is NaN: an element whose sum is not finite is computed again over its stored cells alone.
#include <cooperative_groups.h>

#include "layer_tile.cuh"

namespace cg = cooperative_groups;

namespace comet {
namespace {

constexpr int kTileRows = 128, kTileK = 64, kPitch = kTileRows + 1;
constexpr int kTileWarps = 18;                                 // copies, products, and up to 16 spreading warps: groups of four for each matrix
constexpr int kATile = kTileRows * kTileK * 2;                 // bytes
constexpr int kTileSmem = 226 * 1024;                          // most dynamic shared memory asked for

template <class T> struct TileArgs {
  struct Source { const int32_t *pos, *crd; const T *val; const T *B; int64_t ldb; const T *bias; T *pre; int32_t nnz; bool aligned; } src[2];
  int64_t R, ldc, ldr, ldz;
  T *C;
  const T *res;
  int32_t rows, k_blocks, steps;        // k_blocks: blocks of 64 along one matrix's columns; steps: of all products of a tile
  int nsrc, n, stages, slots, groups, act, bias_along;
  bool vec_out;
  int32_t *status;
};

// sum over row i's stored cells, column r, of one source
template <class T> __device__ __noinline__ float stored_dot(const typename TileArgs<T>::Source &s, int64_t i, int64_t r) {
  float sum = 0.0f;
  for (int32_t p = s.pos[i]; p < s.pos[i + 1]; ++p) sum += widen(s.val[p]) * widen(s.B[(int64_t)s.crd[p] * s.ldb + r]);
  return sum;
}

// Any alignment: one element.
template <class T, int NACC> __device__ __forceinline__ void finish1(const TileArgs<T> &a, int64_t i, int64_t col, float (&z)[NACC]) {
#pragma unroll
  for (int q = 0; q < NACC; ++q) {
    if (!isfinite(z[q])) {
      z[q] = stored_dot<T>(a.src[q], i, col);
      if (NACC == 1 && a.nsrc == 2) z[q] += stored_dot<T>(a.src[1], i, col);
    }
    if (a.src[q].bias) z[q] += widen(a.src[q].bias[a.bias_along == COMET_BIAS_ROWS ? i : col]);
    if (a.src[q].pre) a.src[q].pre[i * a.ldz + col] = narrow<T, float>(z[q]);
  }
  float y = activate<true>(a.act, z[0]);
  if (NACC == 2) y *= z[NACC - 1];
  if (a.res) y += widen(a.res[i * a.ldr + col]);
  a.C[i * a.ldc + col] = narrow<T, float>(y);
}

template <class T, int NACC> __device__ __forceinline__ void finish16(const TileArgs<T> &a, int64_t i, int64_t col, float (&z)[NACC][16]) {
  const int live = (int)min((int64_t)16, a.R - col);
  if (i >= a.rows || live <= 0) return;
#pragma unroll
  for (int q = 0; q < NACC; ++q) {
    bool finite = true;
#pragma unroll
    for (int v = 0; v < 16; ++v) finite = finite && isfinite(z[q][v]);
    if (finite) continue;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if (v >= live || isfinite(z[q][v])) continue;
      z[q][v] = stored_dot<T>(a.src[q], i, col + v);
      if (NACC == 1 && a.nsrc == 2) z[q][v] += stored_dot<T>(a.src[1], i, col + v);
    }
  }
  const float row_bias[2] = {a.src[0].bias && a.bias_along == COMET_BIAS_ROWS ? widen(a.src[0].bias[i]) : 0.0f,
                             NACC == 2 && a.src[1].bias ? widen(a.src[1].bias[i]) : 0.0f};
  const bool col_bias = a.src[0].bias && a.bias_along == COMET_BIAS_COLS;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int64_t c = col + half * 8;
    const int n = live - half * 8;
    if (n <= 0) break;
    const bool vec = a.vec_out && n >= 8;
    Piece<T> out, keep[NACC], res;
    if (a.res) {
      if (vec) res.raw = __ldg(reinterpret_cast<const uint4 *>(a.res + i * a.ldr + c));
      else {
#pragma unroll
        for (int v = 0; v < 8; ++v) res.at[v] = v < n ? a.res[i * a.ldr + c + v] : (T)0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      float z0 = z[0][half * 8 + v] + row_bias[0];
      if (col_bias && v < n) z0 += widen(a.src[0].bias[c + v]);
      if (a.src[0].pre) keep[0].at[v] = narrow<T, float>(z0);
      float y = activate<sizeof(T) == 2>(a.act, z0);
      if (NACC == 2) {
        const float z1 = z[NACC - 1][half * 8 + v] + row_bias[1];
        if (a.src[1].pre) keep[NACC - 1].at[v] = narrow<T, float>(z1);
        y *= z1;
      }
      if (a.res) y += widen(res.at[v]);
      out.at[v] = narrow<T, float>(y);
    }
    if (vec) {
      *reinterpret_cast<uint4 *>(a.C + i * a.ldc + c) = out.raw;
#pragma unroll
      for (int q = 0; q < NACC; ++q)
        if (a.src[q].pre) *reinterpret_cast<uint4 *>(a.src[q].pre + i * a.ldz + c) = keep[q].raw;
    } else {
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        if (v >= n) continue;
        a.C[i * a.ldc + c + v] = out.at[v];
#pragma unroll
        for (int q = 0; q < NACC; ++q)
          if (a.src[q].pre) a.src[q].pre[i * a.ldz + c + v] = keep[q].at[v];
      }
    }
  }
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from, uint32_t bytes) {      // what lies beyond `bytes` becomes zero
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// Spreads the entries of one row, a lane each, over the row's line of the A tiles. Entries come in eights (a sector of columns, 16 bytes of
// values) through a ring of `slots` eights per lane in shared memory, filled by asynchronous copies: their addresses do not depend
// on where a block of k ends, so the ring runs ahead of the blocks, and a block waits for memory only where it takes more of it than has landed
// (eights asked for in the last block may be on their way). Held in registers instead, in-flight entries had to be waited for when
// the next block looked at them or moved them: 2,700 to 5,000 cycles a block against the 300 that the work takes.
template <class T> struct Spreader {
  static constexpr int kBytes = 48;            // of a lane's slot: 8 columns, 8 values
  static constexpr int32_t kNear = 48;         // entries
  const int32_t *crd;
  const T *val;
  int32_t base, lo, end, nnz;                  // base: lo rounded down to an eight
  int32_t head, asked, ready, before;
  uint32_t ring;                               // address of this warp's ring
  int mask;
  bool aligned;

  __device__ __forceinline__ uint32_t slot(int32_t j) const { return ring + (uint32_t)(j & mask) * (32 * kBytes) + (threadIdx.x & 31) * 16; }
  __device__ __forceinline__ void ask() {
    const int64_t i = (int64_t)base + 8 * (int64_t)asked;
    if (i < end) {
      const uint32_t to = slot(asked);
      if (aligned && i + 8 <= nnz) {
        copy16(to, crd + i);
        copy16(to + 512, crd + i + 4);
        copy16(to + 1024, val + i);
      } else if (aligned) {
        const int32_t left = (int32_t)min((int64_t)8, nnz - i);
        copy16(to, crd + i, (uint32_t)min(left, 4) * 4);
        if (left > 4) copy16(to + 512, crd + i + 4, (uint32_t)(left - 4) * 4);
        copy16(to + 1024, val + i, (uint32_t)left * 2);
      } else {
        for (int e = 0; e < 8; ++e) {
          if (i + e >= end) break;
          const int32_t x = __ldg(crd + i + e);
          asm volatile("st.shared.s32 [%0], %1;" ::"r"(to + (e >> 2) * 512 + (e & 3) * 4), "r"(x) : "memory");
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + 1024 + e * 2), "h"(reinterpret_cast<const uint16_t *>(val)[i + e]) : "memory");
        }
      }
    }
    ++asked;
  }
  __device__ __forceinline__ void close_group() {
    asm volatile("cp.async.commit_group;" ::: "memory");
    ready = before;
    before = asked;
  }
  // Sets out for block `first` of k: at an entry before the row's first one in it, but not many before (what lies before the block is passed over).
  // A pruned row's columns are spread about evenly: the first guess by proportion is nearly always good, and each probe is a line from DRAM.
  __device__ __forceinline__ void begin(const typename TileArgs<T>::Source &s, int32_t rows, int64_t row, int32_t first, int32_t blocks) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    crd = s.crd;
    val = s.val;
    aligned = s.aligned;
    nnz = s.nnz;
    lo = 0;
    end = 0;
    if (row < rows) {
      lo = __ldg(s.pos + row);
      end = __ldg(s.pos + row + 1);
    }
    if (first > 0) {
      const int32_t key = first * kTileK;
      int32_t hi = end, c_lo = 0, c_hi = blocks * kTileK;            // the first entry at or beyond `key` lies in [lo, hi]
      for (int round = 0; hi - lo > kNear; ++round) {
        const float share = (float)(key - c_lo) / (float)max(c_hi - c_lo, 1) * (float)(hi - lo);
        if (round > 0 && share < (float)kNear) break;                // lo is near enough
        int32_t probe = round < 4 ? lo + (int32_t)share - kNear / 2 : lo + (hi - lo) / 2;
        probe = min(max(probe, lo + 1), hi - 1);
        const int32_t c = __ldg(s.crd + probe);
        if (c < key) { lo = probe; c_lo = c; } else { hi = probe; c_hi = c; }
      }
    }
    base = lo & ~7;
    head = asked = 0;
    for (int j = 0; j <= mask; ++j) ask();
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_all;" ::: "memory");
    ready = before = asked;
  }
  // line: the row's 128 bytes of the (zeroed) tile; r: its number in the tile
  __device__ __forceinline__ void spread(uint32_t line, int r, int32_t block) {
    const int32_t k0 = block * kTileK;
    line ^= (uint32_t)(r & 7) << 4;            // the swizzle: 16-byte chunk k / 8 of row r sits at chunk (k / 8) ^ (r % 8); lines start on 128 bytes
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    bool used;
    do {
      const int32_t i = base + 8 * head;
      const bool live = i < end;
      if (__any_sync(0xffffffffu, live && head >= ready)) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        ready = asked;
      }
      used = false;
      if (live) {
        int32_t c[8];
        uint32_t v[4];
        const uint32_t at = slot(head);
        asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3]) : "r"(at) : "memory");
        asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(c[4]), "=r"(c[5]), "=r"(c[6]), "=r"(c[7]) : "r"(at + 512) : "memory");
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at + 1024) : "memory");
        const int32_t from = lo - i, left = end - i;       // entries from .. left - 1 of the eight are this row's
        if (from > 0 || left < 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < from || e >= left) c[e] = -1;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t k = (uint32_t)(c[e] - k0);
          if (k < (uint32_t)kTileK)
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(line ^ (k << 1)), "h"((uint16_t)(e & 1 ? v[e >> 1] >> 16 : v[e >> 1])) : "memory");
        }
        // the eight is done with when its last entry lies in this block (or before it)
        used = left > 8 ? c[7] - k0 < kTileK : false;
        if (used) {
          ++head;
          ask();
        }
      }
    } while (__any_sync(0xffffffffu, used));
    close_group();
  }
};

// The order in which a CTA takes its blocks of k: the groups of spreading warps take turns, each with a stretch of blocks of its own, so that a
// group has as many steps' time to spread a block as there are groups. (Counters, no divisions: seven of those a step kept the one
// thread that issues the copies busy for 700 cycles.)
struct Order {
  int32_t from, each, extra;       // group g: each + (g < extra) blocks from from + g * each + min(g, extra) on
  __device__ __forceinline__ Order(int32_t first, int32_t last, int32_t groups) : from(first), each((last - first) / groups), extra((last - first) % groups) {}
  __device__ __forceinline__ int32_t block(int32_t group, int32_t turn) const { return from + group * each + min(group, extra) + turn; }
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

template <class T, int NACC>
__global__ void __launch_bounds__(kTileWarps * 32, 1) tile_product_kernel(const __grid_constant__ CUtensorMap map0, const __grid_constant__ CUtensorMap map1,
                                                                          const TileArgs<T> a) {
  extern __shared__ char raw_smem[];
  __shared__ uint64_t bars[2 * 8 + 1];
  __shared__ uint32_t tmem_at;
  __shared__ int failed;
  char *smem = reinterpret_cast<char *>(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = a.n, stages = a.stages, stage_bytes = NACC * kATile + kTileK * 2 * n;
  const uint32_t full = smem_u32(bars), empty = full + 8 * stages, done = full + 16 * stages;
  const int split = gridDim.z, rank = blockIdx.z;
  const int32_t from = (int32_t)((int64_t)a.steps * rank / split), to = (int32_t)((int64_t)a.steps * (rank + 1) / split);
  const int64_t row0 = (int64_t)blockIdx.x * kTileRows, col0 = (int64_t)blockIdx.y * n;
  uint32_t columns = 32;
  while (columns < (uint32_t)(NACC * n)) columns <<= 1;

  if (threadIdx.x == 0) {
    failed = 0;
    for (int s = 0; s < stages; ++s) {
      bar_init(full + 8 * s, 4 * NACC + 1);
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

  const Order order(from, to, a.groups);
  if (warp == 0) {
    if (lane == 0) {
      Place at;
      int32_t group = 0, turn = 0;
      for (int32_t t = from; t < to; ++t, at.next(stages)) {
        if (at.round > 0 && !bar_wait(empty + 8 * at.stage, (at.round - 1) & 1, &failed)) break;
        int32_t block = order.block(group, turn);
        if (++group == a.groups) { group = 0; ++turn; }
        const bool second = block >= a.k_blocks;
        if (second) block -= a.k_blocks;
        const uint32_t bar = full + 8 * at.stage, b = smem_u32(smem + at.stage * stage_bytes + NACC * kATile);
        bar_expect(bar, (uint32_t)(kTileK * 2 * n));
        for (int j = 0; j < n / 64; ++j) copy_box(b + j * (64 * kTileK * 2), second ? &map1 : &map0, (int)col0 + j * 64, block * kTileK, bar);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t kind = product_kind(Num<T>::is_bf16, true, kTileRows, n);
      Place at;
      for (int32_t t = from; t < to; ++t, at.next(stages)) {
        if (!bar_wait(full + 8 * at.stage, at.round & 1, &failed)) break;
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
    // four warps, a lane per row, for each matrix and group
    const int w = warp - 2, q = NACC == 2 ? (w >> 2) & 1 : 0, group = w / (4 * NACC), r = (w & 3) * 32 + lane;
    Spreader<T> e;
    e.ring = smem_u32(smem + stages * stage_bytes) + (uint32_t)(w * a.slots * 32 * Spreader<T>::kBytes);
    e.mask = a.slots - 1;
    const int32_t turns = group < a.groups ? order.each + (group < order.extra) : 0;
    int source = -1;
    Place at;
    at.stage = group;                                      // groups <= stages
    for (int32_t turn = 0; turn < turns; ++turn, at.next(stages, a.groups)) {
      int32_t block = order.block(group, turn);
      const int now = NACC == 2 ? q : block >= a.k_blocks;
      if (NACC == 1 && now) block -= a.k_blocks;
      if (now != source) {
        source = now;
        e.begin(a.src[now], a.rows, row0 + r, block, a.k_blocks);
      }
      if (at.round > 0 && !bar_wait_warp(empty + 8 * at.stage, (at.round - 1) & 1, &failed)) break;
      char *tile = smem + at.stage * stage_bytes + q * kATile, *mine = tile + (w & 3) * 32 * 128;
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(mine + i * 512 + lane * 16) = make_uint4(0, 0, 0, 0);
      __syncwarp();
      e.spread(smem_u32(tile + r * 128), r, block);
      if (turn + 1 == turns) asm volatile("cp.async.wait_all;" ::: "memory");     // the rings' memory may be used again when all products are done
      fence_async_smem();
      __syncwarp();
      if (lane == 0) bar_arrive(full + 8 * at.stage);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }

  // A spreading warp reads the accumulators of 32 rows (a lane each), each kParts-th group of 16 columns.
  __syncwarp();
  const bool ok = bar_wait_warp(done, 0, &failed) && !__any_sync(0xffffffffu, failed);
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
      if (warp >= 2 && ok) {
        for (int r = warp - 2; r < kTileRows && row0 + r < a.rows; r += kTileWarps - 2) {
          for (int c = lane; c < min(chunk, n - first) && col0 + first + c < a.R; c += 32) {
            float z[NACC];
#pragma unroll
            for (int q = 0; q < NACC; ++q) z[q] = sums[(q * chunk + c) * kPitch + r];
            finish1<T, NACC>(a, row0 + r, col0 + first + c, z);
          }
        }
      }
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
    if (warp >= 2 && ok && a.vec_out) {
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
        finish16<T, NACC>(a, i, col0 + rank * share + c, z);
      }
    } else if (warp >= 2 && ok) {
      for (int r = warp - 2; r < kTileRows && row0 + r < a.rows; r += kTileWarps - 2) {
        for (int c = rank * share + lane; c < (rank + 1) * share && col0 + c < a.R; c += 32) {
          float z[NACC];
#pragma unroll
          for (int q = 0; q < NACC; ++q) z[q] = 0.0f;
          for (int k = 0; k < split; ++k) {
            const float *there = cluster.map_shared_rank(sums, k);
#pragma unroll
            for (int q = 0; q < NACC; ++q) z[q] += there[(q * n + c) * kPitch + r];
          }
          finish1<T, NACC>(a, row0 + r, col0 + c, z);
        }
      }
    }
    cluster.sync();                                     // nobody's shared memory goes while another reads it
  }
  if (threadIdx.x == 0 && failed) give_up(full, stages, a.status);
}

template <class T, int NACC>
comet_status_t launch(Context *ctx, const CUtensorMap &m0, const CUtensorMap &m1, TileArgs<T> &a, int64_t row_tiles, int64_t col_tiles, int split, cudaStream_t s) {
  const int stage_bytes = NACC * kATile + kTileK * 2 * a.n;
  const int64_t steps_each = a.steps / split;
  // As many groups of spreading warps as can have a stage and their rings (4 or 8 eights a lane, by the mean number of a row's entries in a block) in
  // shared memory; stages in what is left of it.
  double nnz = 0, cells = 0;
  for (int q = 0; q < a.nsrc; ++q) { nnz += a.src[q].nnz; cells += (double)a.rows * a.k_blocks; }
  a.slots = nnz > 14 * cells ? 8 : 4;
  const int group_rings = 4 * NACC * a.slots * 32 * Spreader<T>::kBytes;
  a.groups = 4 / NACC;
  while (a.groups > 1 && (a.groups > steps_each || a.groups * (stage_bytes + group_rings) + 1024 > kTileSmem)) --a.groups;
  const int rings = a.groups * group_rings;
  a.stages = (kTileSmem - 1024 - rings) / stage_bytes;
  if (a.stages > 8) a.stages = 8;
  if (a.stages > steps_each + 1) a.stages = (int)steps_each + 1;
  if (a.stages < 2) a.stages = 2;
  size_t bytes = (size_t)a.stages * stage_bytes + rings;
  const size_t join = split > 1 || !a.vec_out ? (size_t)(NACC * a.n < 256 ? NACC * a.n : 256) * kPitch * sizeof(float) : 0;
  if (join > bytes) bytes = join;
  bytes += 1024;
  auto *kernel = tile_product_kernel<T, NACC>;
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

template <class T> comet_status_t product_typed(Context *ctx, const GatherCall &c, cudaStream_t s) {
  TileArgs<T> a{};
  a.nsrc = c.mode == kLayer ? 1 : 2;
  const auto ok16 = [](const void *p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && ld % 8 == 0); };
  a.vec_out = ok16(c.C, c.ldc) && ok16(c.residual, c.ldr);
  for (int q = 0; q < a.nsrc; ++q) {
    const GatherSource &g = c.src[q];
    a.src[q] = {g.A.pos, g.A.crd, (const T *)g.A.val, (const T *)g.B, g.ldb, (const T *)g.bias, (T *)g.pre, (int32_t)g.A.nnz,
                ((uintptr_t)g.A.crd & 15) == 0 && ((uintptr_t)g.A.val & 15) == 0};
    a.vec_out = a.vec_out && ok16(g.pre, c.ldz);
  }
  a.R = c.R; a.ldc = c.ldc; a.ldr = c.ldr; a.ldz = c.ldz;
  a.C = (T *)c.C;
  a.res = (const T *)c.residual;
  a.rows = (int32_t)c.src[0].A.rows;
  a.act = c.act; a.bias_along = c.bias_along;
  a.status = ctx->h_pinned + kTileStatusWord;
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
  return gated ? launch<T, 2>(ctx, m0, m1, a, row_tiles, col_tiles, split, s) : launch<T, 1>(ctx, m0, m1, a, row_tiles, col_tiles, split, s);
}

}  // namespace

bool tile_product_fits(int dtype, const GatherCall &c) {
  if (dtype != COMET_BF16 && dtype != COMET_F16) return false;
  if (c.R < 8 || c.R >= (1ll << 24)) return false;
  const int n = c.mode == kLayer ? 1 : 2;
  double nnz = 0, cells = 0;
  for (int q = 0; q < n; ++q) {
    const GatherSource &g = c.src[q];
    nnz += (double)g.A.nnz;
    cells += (double)g.A.rows * (double)g.A.cols;
  }
  return cells > 0 && nnz < 2147480000.0 && nnz * 64 >= cells;      // (entry numbers run past a row by up to 96)
}

comet_status_t tile_product(Context *ctx, int dtype, const GatherCall &c, cudaStream_t s) {
  const comet_status_t st = tile_status(ctx);
  if (st != COMET_OK) return st;
  return dtype == COMET_BF16 ? product_typed<__nv_bfloat16>(ctx, c, s) : product_typed<__half>(ctx, c, s);
}

}  // namespace comet
