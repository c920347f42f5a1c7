// The sampled product on the tensor cores: 16-bit values and matrices whose cells are stored densely enough that computing the whole block
// P[128 rows] Q[N rows]^T and keeping the stored cells of it costs less than a dot product per cell.
//
// A CTA of eighteen warps: one thread copies tiles of P and Q (64 values of k, by tensor map, zeros outside), one issues the products, and
// eight warps meanwhile look up where each of the 128 rows' entries enter and leave the block's columns; then sixteen move the block from tensor memory to
// shared memory and write the stored cells of it, a warp per row, entries in order, four rows at a time.
#include "layer_tile.cuh"

namespace comet {
namespace {

constexpr int kRows = 128, kK = 64, kWarps = 18;
constexpr int kStages = 4;
constexpr int kSampleSmem = kStages * (kRows + 256) * kK * 2 + 1024;   // most dynamic shared memory: blocks of 256 columns
static_assert(256 * (kRows + 1) * (int)sizeof(float) + 1024 <= kSampleSmem, "the block of results takes the stages' place");

template <class T> struct SampleTileArgs {
  const int32_t *pos, *crd;
  T *out;
  int32_t rows, cols, k_blocks, n;
  int32_t *status;
  int64_t patience;
};

template <class T>
__global__ void __launch_bounds__(kWarps * 32, 1) tile_sample_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q,
                                                                     const SampleTileArgs<T> a) {
  extern __shared__ char raw_smem[];
  __shared__ uint64_t bars[2 * kStages + 1];
  __shared__ uint32_t tmem_at;
  __shared__ int failed;
  __shared__ int32_t first[kRows], last[kRows];
  char *smem = reinterpret_cast<char *>(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = a.n;
  const int stage_bytes = (kRows + n) * kK * 2;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, done = full + 16 * kStages;
  const int32_t row0 = (int32_t)blockIdx.x * kRows, col0 = (int32_t)blockIdx.y * n;
  int32_t issued = 0;                                  // copies, in the thread that issues them
  uint32_t columns = 32;
  while (columns < (uint32_t)n) columns <<= 1;
  if (threadIdx.x == 0) {
    failed = a.patience <= 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
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
      for (int32_t t = 0; t < a.k_blocks; ++t, ++issued) {
        const int s = t % kStages, round = t / kStages;
        if (round > 0 && !bar_wait(empty + 8 * s, (round - 1) & 1, &failed, a.patience)) break;
        const uint32_t p = smem_u32(smem + s * stage_bytes);
        bar_expect(full + 8 * s, (uint32_t)stage_bytes);
        copy_box(p, &map_p, t * kK, row0, full + 8 * s);
        copy_box(p + kRows * kK * 2, &map_q, t * kK, col0, full + 8 * s);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t kind = product_kind(Num<T>::is_bf16, false, kRows, n);
      for (int32_t t = 0; t < a.k_blocks; ++t) {
        const int s = t % kStages, round = t / kStages;
        if (!bar_wait(full + 8 * s, round & 1, &failed, a.patience)) break;
        tc_fence_after();
        const uint32_t p = smem_u32(smem + s * stage_bytes);
        const uint64_t x = operand_at(p, 16, 1024), y = operand_at(p + kRows * kK * 2, 16, 1024);
#pragma unroll
        for (int k = 0; k < kK / 16; ++k) tc_product(d, x + k * 2, y + k * 2, kind, t > 0 || k > 0);
        tc_commit(empty + 8 * s);
      }
      tc_commit(done);
    }
  } else if (warp < 10) {
    // where each row's entries enter the block's columns (threads 64..191) and leave them (192..319)
    const int k = (int)threadIdx.x - 64, r = k & (kRows - 1);
    const int32_t i = row0 + r;
    int32_t lo = 0, hi = 0;
    if (i < a.rows) { lo = __ldg(a.pos + i); hi = __ldg(a.pos + i + 1); }
    const int32_t limit = k < kRows ? col0 : (int32_t)min((int64_t)a.cols, (int64_t)col0 + n);
    while (lo < hi) {
      const int32_t mid = lo + (hi - lo) / 2;
      if (__ldg(a.crd + mid) < limit) lo = mid + 1; else hi = mid;
    }
    (k < kRows ? first : last)[r] = lo;
  }

  __syncwarp();
  const bool over = bar_wait_warp(done, 0, &failed, a.patience), ok = over && !__any_sync(0xffffffffu, failed);
  if (warp == 1 && !over) bar_wait_end(done, 0);       // the products in flight, before tensor memory and stages go
  tc_fence_after();
  float *block = reinterpret_cast<float *>(smem);      // [n][kRows + 1]: the stages are free
  if (warp >= 2 && ok) {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    for (int c = part * 16; c < n; c += 16 * ((kWarps - 2) / 4)) {
      float x[16];
      tmem_load16(d + ((uint32_t)(quarter * 32) << 16) + c, x);
#pragma unroll
      for (int v = 0; v < 16; ++v) block[(c + v) * (kRows + 1) + quarter * 32 + lane] = x[v];
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp >= 2 && ok) {
    // Four rows at a time: their first 64 entries are asked for together, what a row has beyond waits for memory.
    constexpr int kEach = kRows / (kWarps - 2);
#pragma unroll
    for (int k0 = 0; k0 < kEach; k0 += 4) {
      int32_t from[4], to[4], c[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = (warp - 2) * kEach + k0 + k;
        from[k] = first[r] + lane;
        to[k] = last[r];
#pragma unroll
        for (int w = 0; w < 2; ++w) c[k][w] = from[k] + 32 * w < to[k] ? __ldg(a.crd + from[k] + 32 * w) : col0;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float *line = block + (warp - 2) * kEach + k0 + k;
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (from[k] + 32 * w < to[k]) a.out[from[k] + 32 * w] = narrow<T, float>(line[min((uint32_t)(c[k][w] - col0), (uint32_t)n - 1u) * (kRows + 1)]);
        for (int32_t p = from[k] + 64; p < to[k]; p += 32)
          a.out[p] = narrow<T, float>(line[min((uint32_t)(__ldg(a.crd + p) - col0), (uint32_t)n - 1u) * (kRows + 1)]);
      }
    }
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_free(d, columns);
  }
  if (threadIdx.x == 0 && failed) give_up(full, kStages, issued, a.status);
}

template <class T>
comet_status_t sample_tiles(Context *ctx, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R, void *out, cudaStream_t s) {
  SampleTileArgs<T> a{};
  a.pos = A.pos; a.crd = A.crd;
  a.out = (T *)out;
  a.rows = (int32_t)A.rows; a.cols = (int32_t)A.cols;
  a.k_blocks = (int32_t)ceil_div(R, kK);
  const int64_t groups = ceil_div(A.cols, 64), tiles = ceil_div(groups, 4);
  a.n = (int)(ceil_div(groups, tiles) * 64);
  a.status = ctx->h_pinned + kLayerStatusWord;
  a.patience = wait_patience();
  const size_t ring = (size_t)kStages * (kRows + a.n) * kK * 2, block = (size_t)a.n * (kRows + 1) * sizeof(float);
  const size_t bytes = (ring > block ? ring : block) + 1024;
  auto *kernel = tile_sample_kernel<T>;
  // (In front of the maps: their encoder wants a context, which a thread has from its first call of the runtime on.)
  COMET_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleSmem));      // the device's, not this call's
  CUtensorMap mp, mq;
  if (!tile_map(&mp, Num<T>::is_bf16, P, A.rows, R, ldp, kRows) || !tile_map(&mq, Num<T>::is_bf16, Q, A.cols, R, ldq, a.n)) return COMET_ERR_CUDA;
  kernel<<<dim3((unsigned)ceil_div(A.rows, kRows), (unsigned)tiles), kWarps * 32, bytes, s>>>(mp, mq, a);
  COMET_LAUNCH_CHECK(ctx);
  return COMET_OK;
}

}  // namespace

bool tile_sample_fits(int dtype, const RowView &A, int64_t R) {
  if (dtype != COMET_BF16 && dtype != COMET_F16) return false;
  if (R < 8 || R >= (1ll << 24) || !A.ordered) return false;          // a row's entries of a block of columns lie together
  // A block costs about the same whatever it keeps of its cells, gathers cost what the entries x columns do. Measured on 4096^2, bf16, tiles and gathers, us: 16
  // columns at 1/6 of the cells 30 and 44, at 1/12 26 and 30, at 1/24 24 and 15; 32 columns at 1/24 24 and 25, at 1/48 24 and 15; 128 columns at 1/64 23 and
  // 44, at 1/128 23 and 26, at 1/256 22 and 20; 512 columns at 1/128 30 and 75.
  const double nnz = (double)A.nnz, cells = (double)A.rows * (double)A.cols;
  return nnz * (double)R >= cells && nnz * 128 >= cells && A.cols < 65535ll * 64;
}

comet_status_t tile_sample(Context *ctx, int dtype, const RowView &A, const void *P, int64_t ldp, const void *Q, int64_t ldq, int64_t R, void *out,
                           cudaStream_t s) {
  return dtype == COMET_BF16 ? sample_tiles<__nv_bfloat16>(ctx, A, P, ldp, Q, ldq, R, out, s) : sample_tiles<__half>(ctx, A, P, ldp, Q, ldq, R, out, s);
}

// ---- tensor maps
// The driver's encoder, found through the runtime (nothing links against libcuda).
bool tile_map(CUtensorMap *map, bool bf16, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(base), dims, strides, box, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace comet
