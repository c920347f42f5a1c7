// extern "C" entry points of the layer operators: the sparse x dense product with bias, activation and residual in its epilogue, the
// gated pair of products, their backward passes, the sampled product and the structure of the transpose.
#include "kernels.cuh"
#include "layer.cuh"

#include <stdlib.h>
#include <string.h>

namespace comet {

int64_t wait_patience() {
  const char *e = getenv("COMET_LAYER_WAIT_CYCLES");
  return e ? atoll(e) : 8000000000ll;                      // about four seconds
}

template <class T> comet_status_t layer_gather_typed(Context *ctx, const GatherCall &c, cudaStream_t s);   // layer_gather.cuh, a unit per type

template <class T> comet_status_t layer_panel_typed(Context *ctx, const GatherCall &c, cudaStream_t s);    // layer_panel.cuh, likewise

// A few columns of matrices whose entries are worth laying B down in every SM's shared memory: rows of B of up to 16 bytes, no more of
// them (148 times) than the matrix has bytes, 1/64 of the cells (no row is more than 64 times as long as the mean then), and rows of 48 entries on average, since a row
// has a warp of its own; ordered rows where it takes several panels. Measured, panels and the other forms, us: 100,000 rows of 250 entries, one column of bf16 49
// and 79, of 62 entries 36 and 32, of 31 34 and 20; eight columns 121 and 324, 94 and 239, 90 and 62; one column of fp32 53 and 74, 39 and 32, 36
// and 20; four 87 and 142, 62 and 121, 59 and 68; 300,000 rows of 16 entries, one column of bf16 86 and 28, eight 247 and 83. With 4096 columns of A 1/64 of the
// cells are rows of 64 entries: 13 us either way.
bool panel_fits(int dtype, const GatherCall &c) {
  const double es = (double)layer_elem_size(dtype);
  if ((double)c.R * es > 16.0) return false;
  const int n = c.mode == kLayer ? 1 : 2;
  int row_bytes = (int)layer_elem_size(dtype);
  while (row_bytes < c.R * (int)layer_elem_size(dtype)) row_bytes *= 2;
  double nnz = 0, cells = 0;
  for (int q = 0; q < n; ++q) {
    if (!c.src[q].A.ordered && c.src[q].A.cols > panel_capacity(row_bytes)) return false;
    nnz += (double)c.src[q].A.nnz;
    cells += (double)c.src[q].A.rows * (double)c.src[q].A.cols;
  }
  return cells > 0 && nnz < 2147480000.0 && nnz * 64 >= cells && nnz >= 48.0 * n * (double)c.src[0].A.rows && nnz * (4 + es) >= kSmCount * (double)c.src[0].A.cols * (double)c.R * es;
}
comet_status_t layer_panel(Context *ctx, int dtype, const GatherCall &c, cudaStream_t s) {
  switch (dtype) {
    case COMET_F64: return layer_panel_typed<double>(ctx, c, s);
    case COMET_F32: return layer_panel_typed<float>(ctx, c, s);
    case COMET_BF16: return layer_panel_typed<__nv_bfloat16>(ctx, c, s);
    default: return layer_panel_typed<__half>(ctx, c, s);
  }
}

comet_status_t layer_gather(Context *ctx, int dtype, const GatherCall &c, cudaStream_t s) {
  switch (dtype) {
    case COMET_F64: return layer_gather_typed<double>(ctx, c, s);
    case COMET_F32: return layer_gather_typed<float>(ctx, c, s);
    case COMET_BF16: return layer_gather_typed<__nv_bfloat16>(ctx, c, s);
    default: return layer_gather_typed<__half>(ctx, c, s);
  }
}

namespace {

constexpr int64_t kLdLimit = 1ll << 28;

// Temporary blocks of one call, given back (in stream order) when it returns.
struct Temps {
  Context *ctx;
  cudaStream_t s;
  static constexpr int kMost = 32;
  void *block[kMost];
  int count = 0;
  Temps(Context *c, cudaStream_t stream) : ctx(c), s(stream) {}
  ~Temps() { for (int i = 0; i < count; ++i) ctx_free(ctx, block[i], s); }
  void *get(size_t bytes) {
    if (count == kMost) return nullptr;
    void *p = ctx_alloc(ctx, bytes, s);
    if (p) block[count++] = p;
    return p;
  }
};

// A copy of a dense operand into rows that start on 16 bytes, which the tensor-core forms cannot do without.
comet_status_t pad_operand(Context *ctx, int dtype, const void *&B, int64_t &ldb, int64_t rows, int64_t R, Temps &temps) {
  const int64_t ld = layer_padded(dtype, R);
  void *copy = temps.get((size_t)rows * (size_t)ld * layer_elem_size(dtype));
  if (!copy) return COMET_ERR_ALLOC;
  const comet_status_t st = layer_pad(ctx, dtype, B, rows, R, ldb, copy, temps.s);
  B = copy;
  ldb = ld;
  return st;
}
// The sampled product by gathers reads both operands' rows once per entry, in pieces of 16 bytes or value by value: a copy pays from a few entries per row and some
// pieces on (fp32, 1.7 M entries, 50 columns 153 us against 192; 6.7 M, 129 columns 1,144 against 2,201; 0.3 M, 50 columns the same). The products by a
// worker per row hide single values behind their many entries in flight, and a copy only costs them (1.7 M entries in 4,096 rows, fp32, 50 columns 59 us, with
// one 78; bf16, 17 columns 40 and 55; 6.7 M, fp32, 129 columns 709 and 694).
bool gathers_pay_padding(int dtype, int64_t nnz, int64_t rows, int64_t R) {
  return nnz >= 100000 && nnz >= 4 * rows && R * (int64_t)layer_elem_size(dtype) >= 32;
}

// Matrices of short rows (of fp64: all) that are no case for the forms above: the gather kernels of comet_spmm, whose tiles cut long rows and join short ones, and
// the epilogue in a pass of its own where there is one; 16-bit operands as fp32 copies. (Graph of 3.2 M entries, 50 columns of fp32: 470 us by a worker per
// row, 173 like this; of 3.7 M entries, 64 columns of bf16: 1,590 and 210.) Rows need not be ordered for them (long ones are cut by searches
// over one range each, whose results ascend whatever they find). They keep carries in a handle's scratch; each product gets a context with
// scratch of its own here, so that calls may overlap.
bool apart_fits(int dtype, const GatherCall &c) {
  const bool plain = c.mode == kLayer && c.act == COMET_ACT_NONE && !c.src[0].bias && !c.src[0].pre && !c.residual;
  // Rows of some length keep a worker of their own busy, and its epilogue costs nothing: 1.7 M entries in 4,096 rows, 32 columns of fp32 33 us against
  // 44, 16 of bf16 29 against 49; but 0.8 M entries, 100 columns of fp64 197 against 79.
  // Short rows: what decides is how even they are, which the host does not know. The numbers of entries lie between the two. Apart and by rows, fp32, us: power-law
  // rows, 0.17 M entries, 8 columns 27 and 28 (a layer 31 and 28, a pair 57 and 40), 50 columns 24 and 71 (30 and 72, 53 and 102); 0.42 M, 8 columns 31 and 46 (36 and 47, 68
  // and 78), 50 columns 37 and 126; even rows of 20, 0.16 M, 8 columns 20 and 12, 50 columns 18 and 24 (24 and 26, 41 and 36); 0.32 M, 8 columns 22 and 12 (25 and 13, 47 and 14),
  // 50 columns 28 and 37 (36 and 38, 63 and 59).
  if (dtype != COMET_F64 && c.src[0].A.nnz >= 64 * c.src[0].A.rows) return false;
  return c.R >= 4 && c.src[0].A.nnz >= (plain ? 100000 : c.mode == kLayer ? 250000 : 500000);
}

comet_status_t plain_product(Context *ctx, int dtype, const GatherSource &g, int64_t R, void *C, int64_t ldc, cudaStream_t s) {
  const int64_t es = (int64_t)layer_elem_size(dtype), most = 512 / es;       // columns of one launch of those kernels
  for (int64_t first = 0; first < R; first += most) {
    Context own = *ctx;
    own.scratch = nullptr;
    own.scratch_bytes = 0;
    own.has_last_stream = false;
    own.counters_dirty = false;
    own.launches = 0;
    const comet_status_t st = seg_gather(&own, dtype, g.A.pos + 1, g.A.crd, g.A.val, g.A.rows, g.A.nnz, (const char *)g.B + first * es, g.ldb,
                                         R - first < most ? R - first : most, (char *)C + first * es, ldc, nullptr, g.A.rows, g.A.cols, true, false, s);
    if (own.scratch) ctx_free(ctx, own.scratch, s);
    ctx->launches += own.launches;
    if (st != COMET_OK) {
      ctx->last_cuda_error = own.last_cuda_error;
      return st;
    }
  }
  return COMET_OK;
}

bool overlap(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, int64_t R, int64_t es) {
  const char *x = (const char *)a, *y = (const char *)b;
  return a && b && x < y + ((rows - 1) * ldb + R) * es && y < x + ((rows - 1) * lda + R) * es;
}

comet_status_t product_apart(Context *ctx, int dtype, const GatherCall &c, Temps &temps) {
  const bool half = dtype == COMET_BF16 || dtype == COMET_F16;
  const int wide = half ? (int)COMET_F32 : dtype;
  const int64_t rows = c.src[0].A.rows, es = (int64_t)layer_elem_size(wide);
  const int n = c.mode == kLayer ? 1 : 2;
  const bool plain = c.mode == kLayer && c.act == COMET_ACT_NONE && !c.src[0].bias && !c.src[0].pre && !c.residual;
  if (plain && !half) return plain_product(ctx, dtype, c.src[0], c.R, c.C, c.ldc, temps.s);
  FinishCall f{};
  f.rows = rows; f.R = c.R;
  f.act = c.act; f.bias_along = c.bias_along; f.sources = n; f.sum = c.mode == kSumOfTwo;
  f.ldz = c.ldz;
  f.residual = c.residual; f.ldr = c.ldr;
  f.C = c.C; f.ldc = c.ldc;
  // Each product goes where its pre-activation is kept, or the first to C, or to temporary memory.
  const bool kept = !half && c.src[0].pre;
  const bool in_place = !half && !kept && n == 1 && !overlap(c.residual, c.ldr, c.C, c.ldc, rows, c.R, es);
  f.ldzin = kept ? c.ldz : in_place ? c.ldc : layer_padded(wide, c.R);
  float *B = nullptr;
  for (int q = 0; q < n; ++q) {
    GatherSource g = c.src[q];
    if (half) {
      float *val = (float *)temps.get((size_t)g.A.nnz * sizeof(float));
      if (!val) return COMET_ERR_ALLOC;
      comet_status_t st = layer_widen_values(ctx, dtype, g.A.val, g.pick, g.A.nnz, val, temps.s);
      g.A.val = val;
      g.pick = nullptr;
      const int64_t ld = layer_padded(COMET_F32, c.R);
      if (!B || c.mode != kGated) {                           // the gated pair has one operand
        B = (float *)temps.get((size_t)g.A.cols * (size_t)ld * sizeof(float));
        if (!B) return COMET_ERR_ALLOC;
        if (st == COMET_OK) st = layer_widen(ctx, dtype, g.B, g.A.cols, c.R, g.ldb, B, temps.s);
      }
      if (st != COMET_OK) return st;
      g.B = B;
      g.ldb = ld;
    }
    void *z = kept ? c.src[q].pre : in_place ? c.C : temps.get((size_t)rows * (size_t)f.ldzin * (size_t)es);
    if (!z) return COMET_ERR_ALLOC;
    const comet_status_t st = plain_product(ctx, wide, g, c.R, z, f.ldzin, temps.s);
    if (st != COMET_OK) return st;
    f.z[q] = z;
    f.bias[q] = c.src[q].bias;
    f.pre[q] = c.src[q].pre;
  }
  return layer_finish(ctx, dtype, f, temps.s);
}

// The values of a transposed matrix in its own order.
comet_status_t pick_values(Context *ctx, int dtype, GatherSource &g, Temps &temps) {
  void *val = temps.get((size_t)g.A.nnz * layer_elem_size(dtype));
  if (!val) return COMET_ERR_ALLOC;
  const comet_status_t st = layer_pick(ctx, dtype, g.A.val, g.pick, g.A.nnz, val, temps.s);
  g.A.val = val;
  g.pick = nullptr;
  return st;
}

comet_status_t pick_values(Context *ctx, int dtype, GatherCall &c, Temps &temps) {
  for (int q = 0; q < (c.mode == kLayer ? 1 : 2); ++q) {
    if (!c.src[q].pick) continue;
    const comet_status_t st = pick_values(ctx, dtype, c.src[q], temps);
    if (st != COMET_OK) return st;
  }
  return COMET_OK;
}

comet_status_t product_tiles(Context *ctx, int dtype, GatherCall &c, Temps &temps) {
  comet_status_t st = COMET_OK;
  for (int q = 0; q < (c.mode == kLayer ? 1 : 2); ++q) {
    GatherSource &g = c.src[q];
    if (layer_aligned(dtype, g.B, g.ldb)) continue;
    if (q == 1 && c.mode == kGated) {                       // one operand for both matrices
      g.B = c.src[0].B;
      g.ldb = c.src[0].ldb;
      continue;
    }
    if ((st = pad_operand(ctx, dtype, g.B, g.ldb, g.A.cols, c.R, temps)) != COMET_OK) return st;
  }
  const int n = c.mode == kLayer ? 1 : 2;
  RowView A[2];
  const int32_t *pick[2];
  char *mem[2];
  TileList lists[2];
  for (int q = 0; q < n; ++q) {
    A[q] = c.src[q].A;
    pick[q] = c.src[q].pick;
    mem[q] = (char *)temps.get(tile_list_bytes(A[q]));
    if (!mem[q]) return COMET_ERR_ALLOC;
  }
  st = tile_lists(ctx, A, pick, n, mem, lists, temps.s);
  return st != COMET_OK ? st : tile_product(ctx, dtype, c, lists, temps.s);
}

// A form that finds no room for its lists or copies leaves the product to the workers per row, which need none (but for the values of a transposed matrix, which
// all but the tiles want in its own order). What it has written by then is written again.
comet_status_t product(Context *ctx, int dtype, GatherCall &c, Temps &temps) {
  if (c.src[0].A.rows == 0) return COMET_OK;
  const bool panel = panel_fits(dtype, c);
  comet_status_t st = COMET_ERR_ALLOC;
  if (!panel && tile_product_fits(dtype, c)) {
    if ((st = product_tiles(ctx, dtype, c, temps)) != COMET_ERR_ALLOC) return st;
  } else if (!panel && apart_fits(dtype, c)) {
    if (layer_elem_size(dtype) != 2 && (st = pick_values(ctx, dtype, c, temps)) != COMET_OK) return st;       // 16 bits: widened by number
    if ((st = product_apart(ctx, dtype, c, temps)) != COMET_ERR_ALLOC) return st;
  }
  if ((st = pick_values(ctx, dtype, c, temps)) != COMET_OK) return st;
  return panel ? layer_panel(ctx, dtype, c, temps.s) : layer_gather(ctx, dtype, c, temps.s);
}

// (P and Q are left padded where they were copied, for a second call on them.)
comet_status_t sampled(Context *ctx, int dtype, const RowView &A, const void *&P, int64_t &ldp, const void *&Q, int64_t &ldq, int64_t R, void *out, Temps &temps) {
  const bool tiles = tile_sample_fits(dtype, A, R);
  comet_status_t st = COMET_OK;
  if (tiles || gathers_pay_padding(dtype, A.nnz, A.rows + A.cols, R)) {
    if (!layer_aligned(dtype, P, ldp)) st = pad_operand(ctx, dtype, P, ldp, A.rows, R, temps);
    if (st == COMET_OK && !layer_aligned(dtype, Q, ldq)) st = pad_operand(ctx, dtype, Q, ldq, A.cols, R, temps);
    if (st != COMET_OK && st != COMET_ERR_ALLOC) return st;
  }
  // no room for a copy: the gathers take operands as they are
  return tiles && st == COMET_OK ? tile_sample(ctx, dtype, A, P, ldp, Q, ldq, R, out, temps.s) : layer_sample(ctx, dtype, A, P, ldp, Q, ldq, R, out, temps.s);
}

// What a kernel of an earlier call has left behind that gave up: COMET_ERR_CUDA once, COMET_OK otherwise.
comet_status_t earlier_calls(Context *ctx) {
  volatile int32_t *word = ctx->h_pinned + kLayerStatusWord;
  if (!*word) return COMET_OK;
  *word = 0;
  ctx->last_cuda_error = (int)cudaErrorLaunchTimeout;
  return COMET_ERR_CUDA;
}

bool off_type(const void *p, size_t es) { return ((uintptr_t)p & (es - 1)) != 0; }

comet_status_t check_matrix(const comet_sptensor_t *A) {
  if (!A) return COMET_ERR_INVALID_ARG;
  if (A->order == 2 && !layer_dtype(A->dtype)) return COMET_ERR_UNSUPPORTED_FORMAT;
  const comet_status_t st = check_levels(A, 2);
  if (st != COMET_OK) return st;
  const int a0 = A->attr[0], a1 = A->attr[1];
  if (!((a0 == COMET_D && a1 == COMET_CU) || (a0 == COMET_CU && a1 == COMET_CU) || (a0 == COMET_CN && a1 == COMET_S))) return COMET_ERR_UNSUPPORTED_FORMAT;
  return COMET_OK;
}

int64_t row_count(const comet_sptensor_t *A) { return A->dims[A->mode_order[0]]; }
int64_t col_count(const comet_sptensor_t *A) { return A->dims[A->mode_order[1]]; }

// A by rows; [CU,CU] and [CN,S] matrices get the row boundaries that [D,CU] stores from a search per row into temporary memory.
comet_status_t view_rows(Context *ctx, const comet_sptensor_t *A, Temps &temps, RowView *v) {
  *v = RowView{A->pos[1], A->crd[1], A->val, row_count(A), col_count(A), A->nnz, A->attr[1] == COMET_CU};
  if (A->attr[0] == COMET_D) return COMET_OK;
  int32_t *pos = (int32_t *)temps.get((size_t)(v->rows + 1) * sizeof(int32_t));
  if (!pos) return COMET_ERR_ALLOC;
  v->pos = pos;
  return row_starts(ctx, A, v->rows, pos, temps.s);
}

// At as comet_transpose_symbolic makes it of A.
comet_status_t check_transpose(const comet_sptensor_t *A, const comet_sptensor_t *At) {
  if (!At) return COMET_ERR_INVALID_ARG;
  const comet_status_t st = check_levels(At, 2);
  if (st != COMET_OK) return st;
  if (At->dtype != COMET_I32 || At->attr[0] != COMET_D || At->attr[1] != COMET_CU || At->nnz != A->nnz || At->dims[0] != A->dims[0] ||
      At->dims[1] != A->dims[1] || At->mode_order[0] != A->mode_order[1])
    return COMET_ERR_INVALID_ARG;
  return COMET_OK;
}

bool good_act(int act) { return act >= COMET_ACT_NONE && act <= COMET_ACT_SILU; }

// The transpose as a source of a product: its entries' values are A's, by number.
void view_transpose(const comet_sptensor_t *A, const comet_sptensor_t *At, GatherSource *g) {
  g->A = RowView{At->pos[1], At->crd[1], A->val, row_count(At), col_count(At), At->nnz, true};
  g->pick = (const int32_t *)At->val;
}

__global__ void entry_rows_kernel(const int32_t *__restrict__ pos, int32_t rows, int64_t n, int32_t *__restrict__ row, int32_t *__restrict__ number) {
  const int64_t p = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (p >= n) return;
  int32_t lo = 0, hi = rows;
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if ((int64_t)__ldg(pos + mid) <= p) lo = mid; else hi = mid;
  }
  row[p] = lo;
  number[p] = (int32_t)p;
}

}  // namespace
}  // namespace comet

using namespace comet;

extern "C" comet_status_t comet_spmm_epilogue(comet_handle_t handle, const comet_sptensor_t *A, const void *B, int64_t R, int64_t ldb,
                                              const comet_epilogue_t *h_epilogue, void *C, int64_t ldc, void *stream) {
  if (!handle || !B || !C || !h_epilogue || R < 1 || ldb < R || ldc < R) return COMET_ERR_INVALID_ARG;
  const comet_epilogue_t &e = *h_epilogue;
  if (!good_act(e.act) || (e.bias_along != COMET_BIAS_ROWS && e.bias_along != COMET_BIAS_COLS)) return COMET_ERR_INVALID_ARG;
  if ((e.residual && e.ldr < R) || (e.preact && e.ldz < R)) return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(A);
  if (st != COMET_OK) return st;
  const size_t es = layer_elem_size(A->dtype);
  if (off_type(B, es) || off_type(C, es) || off_type(e.bias, es) || off_type(e.residual, es) || off_type(e.preact, es)) return COMET_ERR_MISALIGNED;
  if (ldb >= kLdLimit) return COMET_ERR_INDEX_OVERFLOW;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  GatherCall c{};
  c.mode = kLayer;
  st = view_rows(ctx, A, temps, &c.src[0].A);
  if (st != COMET_OK) return st;
  c.src[0].B = B; c.src[0].ldb = ldb;
  c.src[0].bias = e.bias;
  c.src[0].pre = e.preact;
  c.R = R;
  c.act = e.act; c.bias_along = e.bias_along;
  c.residual = e.residual; c.ldr = e.ldr; c.ldz = e.ldz;
  c.C = C; c.ldc = ldc;
  return product(ctx, A->dtype, c, temps);
}

extern "C" comet_status_t comet_spmm_gated(comet_handle_t handle, const comet_sptensor_t *G, const comet_sptensor_t *U, const void *B, int64_t R,
                                           int64_t ldb, int32_t act, const void *bias_g, const void *bias_u, void *preact_g, void *preact_u,
                                           int64_t ldz, void *C, int64_t ldc, void *stream) {
  if (!handle || !B || !C || R < 1 || ldb < R || ldc < R || !good_act(act)) return COMET_ERR_INVALID_ARG;
  if (!preact_g != !preact_u || (preact_g && ldz < R)) return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(G);
  if (st == COMET_OK) st = check_matrix(U);
  if (st != COMET_OK) return st;
  if (G->dtype != U->dtype || row_count(G) != row_count(U) || col_count(G) != col_count(U)) return COMET_ERR_INVALID_ARG;
  const size_t es = layer_elem_size(G->dtype);
  if (off_type(B, es) || off_type(C, es) || off_type(bias_g, es) || off_type(bias_u, es) || off_type(preact_g, es) || off_type(preact_u, es))
    return COMET_ERR_MISALIGNED;
  if (ldb >= kLdLimit) return COMET_ERR_INDEX_OVERFLOW;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  GatherCall c{};
  c.mode = kGated;
  st = view_rows(ctx, G, temps, &c.src[0].A);
  if (st == COMET_OK) st = view_rows(ctx, U, temps, &c.src[1].A);
  if (st != COMET_OK) return st;
  for (int q = 0; q < 2; ++q) {
    c.src[q].B = B; c.src[q].ldb = ldb;
    c.src[q].bias = q ? bias_u : bias_g;
    c.src[q].pre = q ? preact_u : preact_g;
  }
  c.R = R;
  c.act = act; c.bias_along = COMET_BIAS_ROWS;
  c.ldz = ldz;
  c.C = C; c.ldc = ldc;
  return product(ctx, G->dtype, c, temps);
}

extern "C" comet_status_t comet_sddmm(comet_handle_t handle, const comet_sptensor_t *A, const void *P, int64_t ldp, const void *Q, int64_t ldq,
                                      int64_t R, void *out_val, void *stream) {
  if (!handle || R < 1 || ldp < R || ldq < R) return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(A);
  if (st != COMET_OK) return st;
  if (A->nnz > 0 && (!P || !Q || !out_val)) return COMET_ERR_INVALID_ARG;
  const size_t es = layer_elem_size(A->dtype);
  if (off_type(P, es) || off_type(Q, es) || off_type(out_val, es)) return COMET_ERR_MISALIGNED;
  if (ldp >= kLdLimit || ldq >= kLdLimit) return COMET_ERR_INDEX_OVERFLOW;
  if (A->nnz == 0) return COMET_OK;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  RowView v;
  st = view_rows(ctx, A, temps, &v);
  if (st != COMET_OK) return st;
  return sampled(ctx, A->dtype, v, P, ldp, Q, ldq, R, out_val, temps);
}

extern "C" comet_status_t comet_transpose_symbolic(comet_handle_t handle, const comet_sptensor_t *A, void *stream, comet_sptensor_t *At) {
  if (!handle || !At) return COMET_ERR_INVALID_ARG;
  if (A != At) memset(At, 0, sizeof(*At));
  else return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(A);
  if (st != COMET_OK) return st;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  int32_t *row = (int32_t *)temps.get((size_t)A->nnz * sizeof(int32_t)), *number = (int32_t *)temps.get((size_t)A->nnz * sizeof(int32_t));
  if (!row || !number) return COMET_ERR_ALLOC;
  RowView v;
  st = view_rows(ctx, A, temps, &v);
  if (st != COMET_OK) return st;
  if (A->nnz > 0) {
    entry_rows_kernel<<<(unsigned)ceil_div(A->nnz, kBlockThreads), kBlockThreads, 0, s>>>(v.pos, (int32_t)v.rows, A->nnz, row, number);
    COMET_LAUNCH_CHECK(ctx);
  }
  // The entry numbers ride through the packing as 32-bit values: it copies values bitwise.
  const int32_t *coords[2];
  coords[A->mode_order[0]] = row;
  coords[A->mode_order[1]] = A->crd[1];
  const int32_t order[2] = {A->mode_order[1], A->mode_order[0]}, attr[2] = {COMET_D, COMET_CU};
  st = comet_pack(handle, 2, A->dims, A->nnz, coords, number, COMET_F32, order, attr, stream, At);
  if (st == COMET_OK) At->dtype = COMET_I32;
  return st;
}

// dZ is held in the operands' type, so that both of its products run as the forward one does, in 16 bits on the tensor cores. A 16-bit gradient is thereby rounded
// twice, as dZ and when it is stored: in bf16 it is 2.3e-3 of its norm off the result in 64 bits, where one rounding leaves 1.7e-3 (fp16: an eighth of both, and a dZ
// beyond 65,504 is infinite). The bias gradients are sums from before that rounding. Two 16-bit terms for dZ would take twice the products: sampled, 8192 x
// 2048 at 20 % and 512 columns 46 us instead of 36, the sum of two products about 310 instead of 158; a graph of 3.2 M entries, 64 columns 472 instead of 247.
extern "C" comet_status_t comet_spmm_epilogue_backward(comet_handle_t handle, const comet_sptensor_t *A, const comet_sptensor_t *At, const void *B,
                                                       int64_t R, int64_t ldb, int32_t act, const void *preact, int64_t ldz, const void *dC,
                                                       int64_t lddc, int32_t bias_along, void *dbias, void *dval, void *dB, int64_t lddb, void *stream) {
  if (!handle || R < 1 || !dC || lddc < R || !good_act(act)) return COMET_ERR_INVALID_ARG;
  if (act != COMET_ACT_NONE && (!preact || ldz < R)) return COMET_ERR_INVALID_ARG;
  if (dbias && bias_along != COMET_BIAS_ROWS && bias_along != COMET_BIAS_COLS) return COMET_ERR_INVALID_ARG;
  if ((dval && (!B || ldb < R)) || (dB && lddb < R)) return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(A);
  if (st != COMET_OK) return st;
  if (dB && (st = check_transpose(A, At)) != COMET_OK) return st;
  const size_t es = layer_elem_size(A->dtype);
  if ((dval && off_type(B, es)) || off_type(dC, es) || off_type(dbias, es) || off_type(dval, es) || off_type(dB, es) ||
      (act != COMET_ACT_NONE && off_type(preact, es)))
    return COMET_ERR_MISALIGNED;
  if ((dval && ldb >= kLdLimit) || lddc >= kLdLimit || R >= kLdLimit) return COMET_ERR_INDEX_OVERFLOW;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  const void *dz = dC;
  int64_t lddz = lddc;
  SlopeCall g{};
  g.rows = row_count(A); g.R = R;
  g.act = act; g.sources = 1;
  g.dC = dC; g.lddc = lddc;
  g.bias_along = bias_along;
  g.bias[0] = dbias;
  if (act != COMET_ACT_NONE) {
    g.z[0] = preact; g.ldz = ldz;
    if (dval || dB) {
      g.lddz = layer_padded(A->dtype, R);
      g.dz[0] = temps.get((size_t)g.rows * (size_t)g.lddz * es);
      if (!g.dz[0]) return COMET_ERR_ALLOC;
      dz = g.dz[0];
      lddz = g.lddz;
    }
  }
  if (g.dz[0] || dbias) {
    st = layer_slope(ctx, A->dtype, g, s);
    if (st != COMET_OK) return st;
  }
  if (dval && A->nnz > 0) {
    RowView v;
    st = view_rows(ctx, A, temps, &v);
    if (st == COMET_OK) st = sampled(ctx, A->dtype, v, dz, lddz, B, ldb, R, dval, temps);
    if (st != COMET_OK) return st;
  }
  if (!dB) return COMET_OK;
  GatherCall c{};
  c.mode = kLayer;
  view_transpose(A, At, &c.src[0]);
  c.src[0].B = dz; c.src[0].ldb = lddz;
  c.R = R;
  c.C = dB; c.ldc = lddb;
  return product(ctx, A->dtype, c, temps);
}

extern "C" comet_status_t comet_spmm_gated_backward(comet_handle_t handle, const comet_sptensor_t *G, const comet_sptensor_t *Gt,
                                                    const comet_sptensor_t *U, const comet_sptensor_t *Ut, const void *B, int64_t R, int64_t ldb,
                                                    int32_t act, const void *preact_g, const void *preact_u, int64_t ldz, const void *dC,
                                                    int64_t lddc, void *dbias_g, void *dbias_u, void *dval_g, void *dval_u, void *dB, int64_t lddb,
                                                    void *stream) {
  if (!handle || R < 1 || !dC || lddc < R || !preact_g || !preact_u || ldz < R || !good_act(act)) return COMET_ERR_INVALID_ARG;
  const bool dvals = dval_g || dval_u;
  if ((dvals && (!B || ldb < R)) || (dB && lddb < R)) return COMET_ERR_INVALID_ARG;
  comet_status_t st = check_matrix(G);
  if (st == COMET_OK) st = check_matrix(U);
  if (st != COMET_OK) return st;
  if (G->dtype != U->dtype || row_count(G) != row_count(U) || col_count(G) != col_count(U)) return COMET_ERR_INVALID_ARG;
  if (dB) {
    st = check_transpose(G, Gt);
    if (st == COMET_OK) st = check_transpose(U, Ut);
    if (st != COMET_OK) return st;
  }
  const size_t es = layer_elem_size(G->dtype);
  if ((dvals && off_type(B, es)) || off_type(dC, es) || off_type(preact_g, es) || off_type(preact_u, es) || off_type(dbias_g, es) ||
      off_type(dbias_u, es) || off_type(dval_g, es) || off_type(dval_u, es) || off_type(dB, es))
    return COMET_ERR_MISALIGNED;
  if ((dvals && ldb >= kLdLimit) || R >= kLdLimit) return COMET_ERR_INDEX_OVERFLOW;
  Context *ctx = reinterpret_cast<Context *>(handle);
  if ((st = earlier_calls(ctx)) != COMET_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  Temps temps(ctx, s);
  SlopeCall g{};
  g.rows = row_count(G); g.R = R;
  g.act = act; g.sources = 2;
  g.dC = dC; g.lddc = lddc;
  g.z[0] = preact_g; g.z[1] = preact_u; g.ldz = ldz;
  g.bias_along = COMET_BIAS_ROWS;
  g.bias[0] = dbias_g; g.bias[1] = dbias_u;
  g.lddz = layer_padded(G->dtype, R);
  const bool need[2] = {dB || dval_g, dB || dval_u};
  for (int q = 0; q < 2; ++q) {
    if (!need[q]) continue;
    g.dz[q] = temps.get((size_t)g.rows * (size_t)g.lddz * es);
    if (!g.dz[q]) return COMET_ERR_ALLOC;
  }
  st = layer_slope(ctx, G->dtype, g, s);
  if (st != COMET_OK) return st;
  for (int q = 0; q < 2; ++q) {
    const comet_sptensor_t *A = q ? U : G;
    void *dval = q ? dval_u : dval_g;
    if (!dval || A->nnz == 0) continue;
    RowView v;
    st = view_rows(ctx, A, temps, &v);
    const void *dz = g.dz[q];
    int64_t lddz = g.lddz;
    if (st == COMET_OK) st = sampled(ctx, G->dtype, v, dz, lddz, B, ldb, R, dval, temps);
    if (st != COMET_OK) return st;
  }
  if (!dB) return COMET_OK;
  GatherCall c{};
  c.mode = kSumOfTwo;
  for (int q = 0; q < 2; ++q) {
    view_transpose(q ? U : G, q ? Ut : Gt, &c.src[q]);
    c.src[q].B = g.dz[q]; c.src[q].ldb = g.lddz;
  }
  c.R = R;
  c.C = dB; c.ldc = lddb;
  return product(ctx, G->dtype, c, temps);
}
