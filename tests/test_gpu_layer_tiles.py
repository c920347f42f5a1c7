"""The tensor-core product of the layer operators against its definition, in each of its variants: sizes around the edges of its tiles, one and several column
tiles, the blocks of k split over 2, 4 and 8 CTAs, epilogues of aligned and unaligned rows, the gated pair, the transposed product and the sum
of two, infinities beside the stored cells. Each test counts the launches of its calls, so that another form cannot stand in for the tiles."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import ACTS, TYPES, Matrix, act64, act_bound, assert_within, place, random_mask, slope64, stored, u_of, values, z_bound  # noqa: E402
from test_gpu_layers import TILES, check_backward, check_epilogue, check_gated, untouched  # noqa: E402

LISTS, PRODUCT, COPY = 3, 1, 1                             # launches: the entries' lists, the product, the copy of an unaligned operand


class Launches:
    """Counts the launches of a block and asks for a number of them."""

    def __init__(self, want):
        self.want, self.handle = want, comet.default_handle()

    def __enter__(self):
        self.before = self.handle.kernel_launches()

    def __exit__(self, kind, *_):
        if kind is None:
            assert self.handle.kernel_launches() - self.before == self.want, "another form was taken"


@pytest.fixture
def any_work(monkeypatch):
    monkeypatch.setenv("COMET_LAYER_TILE_WORK", "0")


def check_sum(g, u, dt, R, act, rng, pad=0, off=0, launches=None):
    """dB of the gated pair: the sum of two transposed products."""
    rows, cols = g.mask.shape
    (dC, dC64), (zg, zg64), (zu, zu64) = (values((rows, R), dt, rng) for _ in range(3))
    Gt, Ut = comet.transpose_symbolic(g.t), comet.transpose_symbolic(u.t)
    args = (g.t, Gt, u.t, Ut, None, place(dC, pad, off), (place(zg, pad, off), place(zu, pad, off)))
    with Launches(launches if launches is not None else 1 + LISTS + PRODUCT):               # the slopes in front of it
        dB = comet.spmm_gated_backward(*args, act=ACTS[act], need_val=False)[2]
    dg, du = dC64 * zu64 * slope64(act, zg64), dC64 * act64(act, zg64)
    sg = stored(dt, dg, 28 * u_of(dt) * (dC64 * zu64).abs() * (1 + zg64.abs()))
    su = stored(dt, du, 20 * u_of(dt) * dC64.abs() * zg64.abs())
    want = g.dense.t() @ dg + u.dense.t() @ du
    N = g.dense.abs().t() @ (dg.abs() + sg) + u.dense.abs().t() @ (du.abs() + su)
    assert_within(dB, want, stored(dt, want, g.dense.abs().t() @ sg + u.dense.abs().t() @ su + z_bound(dt, g.tallest + u.tallest, N, want)), "dB")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [t for t in TILES], ids=lambda s: "x".join(map(str, s)))
def test_edges_of_tiles(cuda_device, any_work, dtype, size):
    rows, cols, density, R = size
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows + cols)
    empty = (0, rows // 2, rows - 1) if rows > 2 else ()
    scale = (cols * density) ** -0.5
    m = Matrix(random_mask(rows, cols, density, rng, empty), dt, rng, scale=scale)
    u = Matrix(random_mask(rows, cols, 0.7 * density, rng, empty[:1]), dt, rng, scale=scale)
    # up to 16 bytes of columns belong to the panels where the matrix has enough entries for them
    tiles = R > 8 or m.t.nnz * 6 < 148 * cols * R * 2
    if tiles:
        with Launches(LISTS + PRODUCT):
            check_epilogue(m, dt, R, "none", "none", False, False, rng)
        with Launches(LISTS + PRODUCT):
            check_epilogue(m, dt, R, "gelu", "rows", True, True, rng, pad=8)
        with Launches(COPY + LISTS + PRODUCT):             # rows that start on single elements, in front and behind
            for out in check_epilogue(m, dt, R, "silu", "cols", True, True, rng, pad=3, off=1)[:2]:
                untouched(out, 3)
    check_gated(m, u, dt, R, "silu", True, rng, pad=8)
    check_gated(u, m, dt, R, "gelu", True, rng, pad=1, off=5)
    check_gated(u, m, dt, R, "none", False, rng)
    if R > 8:
        check_backward(m, dt, R, "gelu_tanh", "rows", rng, pad=8)
        check_sum(m, u, dt, R, "silu", rng, pad=8)
        check_sum(u, m, dt, R, "gelu", rng, pad=1, off=1)


SPLITS = [  # rows, cols, density, R: 2 to 8 CTAs share the blocks of k (at least 8 blocks and 16 columns each)
    (130, 8300, 0.1, 256), (128, 8192, 0.3, 250), (120, 4200, 0.3, 128), (250, 4100, 0.05, 121), (130, 2100, 0.2, 64), (100, 1024, 0.2, 57), (129, 20_000, 0.03, 33),
    (384, 8200, 0.05, 505), (64, 8192, 0.1, 130),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,cols,density,R", SPLITS)
def test_blocks_of_k_split(cuda_device, any_work, dtype, rows, cols, density, R):
    """Few tiles and many blocks of k: the CTAs of a cluster take parts of them and add their sums, each for a share of the columns."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(cols + R)
    scale = (cols * density) ** -0.5
    m = Matrix(random_mask(rows, cols, density, rng, (0, rows - 1)), dt, rng, scale=scale)
    u = Matrix(random_mask(rows, cols, density / 2, rng, (1,)), dt, rng, scale=scale)
    copy = COPY if R % 8 else 0
    with Launches(copy + LISTS + PRODUCT):
        check_epilogue(m, dt, R, "none", "none", False, False, rng)
    with Launches(copy + LISTS + PRODUCT):
        pad = -R % 8
        for out in check_epilogue(m, dt, R, "silu", "rows", True, True, rng, pad=0 if copy else 8)[:2]:
            untouched(out, 0 if copy else 8)
    with Launches((0 if pad else COPY) + LISTS + PRODUCT):  # rows a whole number of 16 bytes apart, or not
        for out in check_epilogue(m, dt, R, "gelu", "cols", True, True, rng, pad=pad or 1)[:2]:
            untouched(out, pad or 1)
    for p in (0, pad or 8, 1):
        with Launches((COPY if (R + p) % 8 else 0) + LISTS + PRODUCT):
            check_gated(m, u, dt, R, "silu", True, rng, pad=p)
    # the transposed product of a matrix that is as long the other way round, alone and as a sum of two
    mt, ut = (Matrix(k.mask.T.copy(), dt, rng, scale=scale) for k in (m, u))
    check_sum(mt, ut, dt, R, "gelu_tanh", rng)
    check_sum(ut, mt, dt, R, "none", rng, pad=1)
    check_backward(mt, dt, R, "silu", "rows", rng, pad=pad)
    check_backward(mt, dt, R, "none", "none", rng, pad=1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_enough_calls_take_tiles(cuda_device, dtype):
    """Without the variable: 80 million products in every direction."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(3)
    m, u = (Matrix(random_mask(1025, 2050, 0.3, rng, (0, 1024)), dt, rng, scale=0.05) for _ in range(2))
    for R, copy in ((128, 0), (131, COPY)):
        with Launches(copy + LISTS + PRODUCT):
            check_epilogue(m, dt, R, "gelu", "rows", True, True, rng)
        with Launches(copy + LISTS + PRODUCT):
            check_gated(m, u, dt, R, "silu", True, rng)
        check_sum(m, u, dt, R, "silu", rng)
        check_backward(m, dt, R, "silu", "cols", rng)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cols", [300, 2100])              # one CTA for the blocks of k, and several
@pytest.mark.parametrize("R,pad", [(64, 0), (64, 8), (61, 0), (272, 1), (272, 0)])
def test_only_stored_cells_count_in_tiles(cuda_device, any_work, dtype, cols, R, pad):
    """Infinities and NaN in rows of the dense operand that a row does not store leave its result alone; those that it stores reach it. The elements beside
    them are added again over the stored cells, in fp32: within z_bound as ever."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(cols + R)

    def matrix():
        mask = random_mask(200, cols, 0.3, rng)
        mask[:, 5:8] = False
        mask[150:, 5] = True
        mask[10, 6] = True
        return Matrix(mask, dt, rng, scale=0.1)

    m, u = matrix(), matrix()
    B, _ = values((cols, R), dt, rng)
    B[5], B[6, 0], B[7, R - 1], B[7, 3] = float("nan"), float("inf"), -float("inf"), float("nan")
    B64 = torch.nan_to_num(B.double(), nan=0.0, posinf=0.0, neginf=0.0)
    z, dz = [], []
    for k in (m, u):
        z.append(k.dense @ B64)
        dz.append(z_bound(dt, k.longest, k.dense.abs() @ B64.abs(), z[-1]))

    def others(got, want, bound, what):
        assert bool(torch.isnan(got[150:]).all()) and not bool(torch.isfinite(got[10, 0])), what
        got = got.cpu().double()[:150]
        got[10, 0] = want[10, 0]
        assert_within(got, want[:150], bound[:150], what)

    b = place(B, pad)
    copy = COPY if (R + pad) % 8 else 0
    with Launches(copy + LISTS + PRODUCT):
        out = comet.spmm_epilogue(m.t, b, out=place(torch.zeros(200, R, dtype=dt), pad))
    others(out, z[0], stored(dt, z[0], dz[0]), "product")
    with Launches(copy + LISTS + PRODUCT):
        out = comet.spmm_gated(m.t, u.t, b, act=ACTS["silu"], out=place(torch.zeros(200, R, dtype=dt), pad))
    f, df = act64("silu", z[0]), act_bound(dt, dz[0], z[0])
    want = f * z[1]
    others(out, want, stored(dt, want, df * z[1].abs() + (f.abs() + df) * dz[1] + 2 * u_of(dt) * want.abs()), "gated pair")
    # the same through the sum of two transposed products: dZg = dC * zu, dZu = dC * zg with zu = zg = 1
    mt, ut = (Matrix(k.mask.T.copy(), dt, rng, scale=0.1) for k in (m, u))
    ones = torch.ones(cols, R, dtype=dt, device="cuda")
    dB = comet.spmm_gated_backward(mt.t, comet.transpose_symbolic(mt.t), ut.t, comet.transpose_symbolic(ut.t), None, b, (ones, ones), act=ACTS["none"], need_val=False)[2]
    want = (mt.dense + ut.dense).t() @ B64
    N = (mt.dense.abs() + ut.dense.abs()).t() @ B64.abs()
    others(dB, want, stored(dt, want, z_bound(dt, mt.tallest + ut.tallest, N, want)), "sum of two")


def test_one_copy_of_a_gradient_for_both_of_its_products(cuda_device, any_work):
    """Without an activation dZ is dC itself: where its rows do not start on 16 bytes it is copied once, for dval and dB."""
    dt = torch.bfloat16
    rng = np.random.default_rng(4)
    m = Matrix(random_mask(300, 400, 0.3, rng), dt, rng, scale=0.1)
    (B, B64), (dC, dC64) = values((400, 61), dt, rng), values((300, 61), dt, rng)
    At, B, dC = comet.transpose_symbolic(m.t), B.cuda(), dC.cuda()
    with Launches(COPY + COPY + 1 + LISTS + PRODUCT):      # dC, B, the sampled product, dB
        dval, dB, _ = comet.spmm_epilogue_backward(m.t, At, B, dC)
    r, c = m.rc
    want, N = (dC64[r] * B64[c]).sum(1), (dC64[r].abs() * B64[c].abs()).sum(1)
    assert_within(dval, want, stored(dt, want, 71 * u_of(dt) * N), "dval")
    want, N = m.dense.t() @ dC64, m.dense.abs().t() @ dC64.abs()
    assert_within(dB, want, stored(dt, want, z_bound(dt, m.tallest, N, want)), "dB")


@pytest.mark.parametrize("rows,cols,density,R,launches", [
    (2500, 8000, 0.2, 19, 1), (2500, 8000, 0.2, 20, COPY + LISTS + PRODUCT), (2700, 16_000, 0.02, 48, 1), (2700, 16_000, 0.02, 56, LISTS + PRODUCT),
    (2500, 20_000, 0.02, 48, 4),                           # by rows as well: three launches for rows of more than 16,384 entries, which it could have
])
def test_where_tiles_begin(cuda_device, rows, cols, density, R, launches):
    """With enough work: from 20 columns on, and as many products as cells."""
    rng = np.random.default_rng(R)
    dt = torch.bfloat16
    m = Matrix(random_mask(rows, cols, density, rng), dt, rng, scale=(cols * density) ** -0.5)
    with Launches(launches):
        check_epilogue(m, dt, R, "gelu", "rows", True, True, rng)


IN_PLACE = {  # rows, cols, density, type, columns, columns between rows: each form that adds a residual
    "tile": (200, 1000, 0.3, "bf16", 64, 0), "tile, unaligned": (200, 1000, 0.3, "f16", 61, 2), "split": (130, 8300, 0.1, "bf16", 256, 0),
    "split, unaligned": (130, 4200, 0.3, "bf16", 121, 1), "panel": (3000, 900, 0.3, "f32", 3, 1), "panels": (450, 12_801, 0.5, "f64", 2, 0),
    "rows": (300, 700, 0.4, "f32", 50, 0), "huge row": (40, 40_000, 0.02, "f16", 12, 4), "short rows, 16 bits": (24_000, 1800, 0.0145, "bf16", 20, 0),
    "short rows, kept": (24_000, 1800, 0.0145, "f64", 6, 1),
}


@pytest.mark.parametrize("kind", list(IN_PLACE))
def test_residual_in_place_in_every_form(cuda_device, any_work, kind):
    """C += .. where the residual is C itself, its padding left alone, with and without the pre-activation kept; the same bits as with a residual of its own, and again on
    another stream."""
    rows, cols, density, dtype, R, pad = IN_PLACE[kind]
    dt = TYPES[dtype]
    rng = np.random.default_rng(R)
    mask = random_mask(rows, cols, density, rng)
    if kind == "huge row":
        mask[3, :30_000] = True
    m = Matrix(mask, dt, rng, scale=(cols * density) ** -0.5)
    (B, _), (r, _) = values((cols, R), dt, rng), values((rows, R), dt, rng)
    B = B.cuda()
    for keep in (False, True):
        pre = torch.empty(rows, R, dtype=dt, device="cuda") if keep else None
        want = comet.spmm_epilogue(m.t, B, act=ACTS["gelu_tanh"], residual=place(r, pad), preact=pre)
        kept = pre.clone() if keep else None
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        for s in (torch.cuda.current_stream(), stream):
            with torch.cuda.stream(s):
                out = place(r, pad, fill=7.0)
                comet.spmm_epilogue(m.t, B, act=ACTS["gelu_tanh"], residual=out, preact=pre, out=out)
                torch.cuda.synchronize()
                assert torch.equal(out, want)
                untouched(out, pad)
                assert not keep or torch.equal(pre, kept)
