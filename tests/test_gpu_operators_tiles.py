"""GPU tests of the dense projection's kernels: every tile of the forward product with every activation, with and without slices of the
summation, the gradients' tiles that other shapes leave out, and numbers that are not finite next to the edges of the largest
tiles.  Each test first says which tiles it is about, so that a change of the plan cannot move it elsewhere unseen
(test_operators_host.py checks that the shapes leave none out).  Whole numbers, as in test_gpu_operators.py: sums are exact."""
import pytest
import torch

import paper_2402_12399_amd as rr
from tests import gpu_util as gu
from tests import operators_ref as ref
from tests.test_gpu_operators import ACT, BF16, DT, F32, U, V, Guarded, gen, linear_case, nearest, run_backward, run_linear, whole, within

pytestmark = pytest.mark.gpu

# (dtype, activation, M, K, N, tile rows x staged rows of W (0 x 0: few rows, no tiles), more than one slice, fp32 operands as bf16 parts)
FORWARD = [
    ("f32", "gelu", 4, 1000, 264, (0, 0), False, False), ("f32", "gelu", 31, 512, 264, (0, 0), False, False),
    ("f32", "swiglu", 21, 1872, 3784, (0, 0), False, False),
    ("f32", "gelu", 15113, 8, 72, (64, 128), False, False),
    ("f32", "none", 2187, 1336, 72, (64, 128), True, False), ("f32", "gelu", 2187, 1336, 72, (64, 128), True, False),
    ("f32", "none", 21525, 168, 72, (64, 128), False, True), ("f32", "gelu", 21525, 168, 72, (64, 128), False, True),
    ("f32", "none", 3214, 664, 5952, (128, 128), False, True), ("f32", "gelu", 59077, 136, 72, (128, 128), False, True),
    ("f32", "swiglu", 13001, 144, 200, (128, 128), False, True),
    ("bf16", "gelu", 3, 120, 12592, (32, 64), False, False),
    ("bf16", "none", 4269, 80, 72, (32, 128), False, False), ("bf16", "gelu", 5083, 72, 72, (32, 128), False, False),
    ("bf16", "gelu", 1361, 3128, 80, (32, 128), True, False), ("bf16", "swiglu", 133, 4000, 552, (32, 128), True, False),
    ("bf16", "none", 3, 3920, 8432, (32, 128), True, False), ("bf16", "gelu", 3, 4392, 8728, (32, 128), True, False),
    ("bf16", "gelu", 35, 8, 10608, (64, 128), False, False),
    ("bf16", "none", 2067, 3032, 72, (64, 128), True, False), ("bf16", "gelu", 4471, 1440, 80, (64, 128), True, False),
    ("bf16", "gelu", 33, 3016, 4424, (64, 128), True, False),
    ("bf16", "none", 8401, 920, 8, (128, 128), True, False), ("bf16", "gelu", 9107, 920, 8, (128, 128), True, False),
    ("bf16", "gelu", 67, 2272, 5528, (128, 128), True, False), ("bf16", "swiglu", 77, 2576, 3064, (128, 128), True, False),
    ("bf16", "gelu", 33227, 8, 8, (256, 128), False, False), ("bf16", "gelu", 20011, 520, 1032, (256, 128), False, False),
    ("bf16", "gelu", 8803, 1576, 8, (256, 128), True, False), ("bf16", "swiglu", 11175, 1784, 8, (256, 128), True, False),
    ("bf16", "gelu", 137, 3816, 6904, (256, 128), True, False), ("bf16", "swiglu", 177, 3896, 3080, (256, 128), True, False),
    # 256 x 256: whole chunks and ragged rows, a last round that is cut by rows, ragged columns
    ("bf16", "gelu", 4099, 1000, 4104, (256, 256), False, False), ("bf16", "gelu", 2051, 4160, 4104, (256, 256), False, False),
    ("bf16", "gelu", 35045, 464, 136, (256, 256), False, False),
    ("bf16", "swiglu", 4099, 1000, 4104, (256, 256), False, False), ("bf16", "swiglu", 20011, 520, 1032, (256, 256), False, False),
    ("bf16", "swiglu", 8195, 2048, 5632, (256, 256), False, False), ("bf16", "swiglu", 34299, 416, 88, (256, 256), False, False),
    ("bf16", "none", 941, 8000, 3040, (256, 256), True, False), ("bf16", "gelu", 941, 8000, 3040, (256, 256), True, False),
    ("bf16", "swiglu", 138, 6400, 6000, (256, 256), True, False),
]
# (dtype, M, K, N, which gradient, tile, more than one slice, parts)
GRADIENTS = [
    ("f32", 24875, 152, 136, "dx", (128, 128), False, True),
    ("f32", 65, 8, 24, "dw", (0, 0), False, False), ("f32", 655, 8, 12416, "dw", (128, 128), True, True),
    ("bf16", 21673, 144, 3648, "dx", (256, 256), True, False),
]
ROLE = {"dx": 1, "dw": 2}


def config(dtype, act, M, K, N):
    return rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, ACT[act])


def assert_plan(cfg, role, tile, several, parts):
    bm, brows, slices, cut = gu.linear_plans(cfg)[role]
    assert ((bm, brows), slices > 1, bool(cut)) == (tile, several, parts), "another kernel than this case is about"


@pytest.mark.parametrize("dtype,act,M,K,N,tile,several,parts", FORWARD)
def test_forward_tiles(dtype, act, M, K, N, tile, several, parts):
    assert_plan(config(dtype, act, M, K, N), 0, tile, several, parts)
    for bias, residual in ((True, True), (False, False)):
        x, w, b, r, _ = linear_case(M, K, N, dtype, act, whole, M + N, bias, residual)
        y, z = run_linear(x, w, b, r, act, dtype, N)
        want, want_z = ref.linear(x, w, b, r, act)
        assert torch.equal(z, nearest(want_z, dtype))
        if act == "none":
            assert torch.equal(y, nearest(want, dtype))
            continue
        # of an exact z.  GELU: Phi to 16 u absolutely (its function, argument and sum: a dozen roundings), then a product.  SwiGLU: exponential, sum,
        # division and two products, 10 u; below -88.7 its exponential is infinite and silu, at most 2.7e-37, is taken for 0.  Then the residual's sum
        if act == "gelu":
            e = 16 * U * (want_z.abs() + ref.act(want_z, act).abs()) + 2 * U * want.abs()
        else:
            g, u = want_z.chunk(2, dim=1)
            e = 10 * U * ref.act(want_z, act).abs() + 2 * U * want.abs() + 2.7e-37 * u.abs()
        within(y, want, e + (V if dtype == "bf16" else U) * (want.abs() + e) + 1e-38, "y")


@pytest.mark.parametrize("dtype,act,M,K,N,tile,several,parts", [f for f in FORWARD if f[5] >= (128, 128)])
def test_forward_tiles_in_place(dtype, act, M, K, N, tile, several, parts):
    """y may be the residual: lanes trade columns of it before they store."""
    x, w, b, r, _ = linear_case(M, K, N, dtype, act, whole, M + N)
    y, _ = run_linear(x, w, b, r, act, dtype, N)
    cfg = config(dtype, act, M, K, N)
    rr.rr_linear(cfg, x, w, b, r, r, None, rr.alloc_linear_workspace(cfg))
    assert torch.equal(y, r)


@pytest.mark.parametrize("act,M,K,N,cut", [("swiglu", 2057, 456, 4488, 3), ("swiglu", 2314, 456, 3720, 5), ("swiglu", 2057, 456, 4104, 6), ("swiglu", 2314, 456, 3592, 7),
                                           ("none", 5655, 456, 3336, 3), ("none", 7454, 456, 2312, 5), ("gelu", 8225, 456, 2056, 6), ("none", 7197, 456, 2312, 7)])
def test_cut_tiles_add_the_residual_once(act, M, K, N, cut):
    """Tiles of the last round, cut by rows into parts whose equal shares do not add up to the tile: no row is computed twice, which y in the residual's
    place would show."""
    assert_plan(config("bf16", act, M, K, N), 0, (256, 256), False, False)
    columns = 128 if act == "swiglu" else 256
    left = -(-M // 256) * -(-N // columns) % torch.cuda.get_device_properties(0).multi_processor_count
    assert torch.cuda.get_device_properties(0).multi_processor_count // left == cut
    x, w, b, r, _ = linear_case(M, K, N, "bf16", act, whole, M + N)
    y, _ = run_linear(x, w, b, r, act, "bf16", N, pre=False)
    cfg = config("bf16", act, M, K, N)
    ws = rr.alloc_linear_workspace(cfg)
    for i in range(20):
        at = r.clone()
        rr.rr_linear(cfg, x, w, b, at, at, None, ws)
        assert torch.equal(y, at), i


@pytest.mark.parametrize("dtype,M,K,N,name,tile,several,parts", GRADIENTS)
def test_gradient_tiles(dtype, M, K, N, name, tile, several, parts):
    assert_plan(config(dtype, "none", M, K, N), ROLE[name], tile, several, parts)
    x, w, _, _, _ = linear_case(M, K, N, dtype, "none", whole, M, False, False)
    dy = whole(gen(1), M, N, dtype=DT[dtype])
    want = ref.linear_backward(x, w, None, dy, "none")
    got = run_backward(x, w, None, dy, "none", dtype, N)
    for n in got:
        assert torch.equal(got[n], nearest(want[n], dtype) if n != "dbias" else want[n].to(F32)), n


def between_nan(t):
    """A copy that lies between NaN: what a kernel reads before or behind an operand shows in its sums."""
    g = Guarded(tuple(t.shape), t.dtype)
    g.t.copy_(t)
    return g.t


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("M,K,N", [(4099, 1000, 4104), (2051, 4160, 4104)])
def test_not_finite_in_large_forward_tiles(M, K, N, act):
    """x[m, k] reaches row m of y, w[n, k] column n - also from the first elements of a row, which follow the last ones of the row before in memory."""
    assert_plan(config("bf16", act, M, K, N), 0, (256, 256), False, False)
    x, w, _, _, _ = linear_case(M, K, N, "bf16", "none", whole, 17, False, False)
    x, w = between_nan(x), between_nan(w)
    _, clean = run_linear(x, w, None, None, act, "bf16", N)
    assert bool(torch.isfinite(clean).all())
    nan, inf = float("nan"), float("inf")
    x[5, 3], x[8, 0], x[300, K - 1], x[M - 1, 1] = nan, inf, -inf, nan
    w[11, 2], w[260, 0], w[N - 1, K - 1] = inf, nan, nan
    cfg, y, z = config("bf16", act, M, K, N), torch.empty_like(clean), torch.empty_like(clean)
    rr.rr_linear(cfg, x, w, None, None, y, z, rr.alloc_linear_workspace(cfg))
    rows, cols = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    rows[[5, 8, 300, M - 1]] = False
    cols[[11, 260, N - 1]] = False
    assert torch.equal(z[rows][:, cols], clean[rows][:, cols]) and bool(torch.isfinite(y[rows][:, cols]).all())
    assert not bool(torch.isfinite(z[~rows]).any()) and not bool(torch.isfinite(z[:, ~cols]).any())


@pytest.mark.parametrize("M,K,N", [(8195, 2048, 1416), (2051, 4160, 4104)])
def test_not_finite_in_large_turned_tiles(M, K, N):
    """x[m, k] reaches column k of dw, dy[m, n] row m of dx and row n of dw, w[n, k] column k of dx.  Both summations end inside a
    chunk, whose other rows and pieces read as zero, and the staged rows of ragged tiles go on into the next row of the memory."""
    plans = gu.linear_plans(config("bf16", "none", M, K, N))
    assert plans[1][:2] == (256, 256) and plans[2][:2] == (256, 256) and N % 64 and M % 64
    x, w, _, _, _ = linear_case(M, K, N, "bf16", "none", whole, 18, False, False)
    x, w, dy = between_nan(x), between_nan(w), between_nan(whole(gen(19), M, N, dtype=BF16))
    clean = run_backward(x, w, None, dy, "none", "bf16", N, ("dx", "dw"))
    want = ref.linear_backward(x, w, None, dy, "none")
    assert all(torch.equal(clean[n], nearest(want[n], "bf16")) for n in clean)
    nan, inf = float("nan"), float("inf")
    x[5, 3], x[M - 1, 0], x[100, K - 1] = nan, inf, nan
    dy[7, 2], dy[9, 0], dy[M - 1, 1], dy[50, N - 1] = inf, nan, nan, -inf
    w[11, 0], w[N - 1, 5] = inf, nan
    cfg, dx, dw = config("bf16", "none", M, K, N), torch.empty_like(x), torch.empty_like(w)
    rr.rr_linear_backward(cfg, x, w, None, dy, dx, dw, None, rr.alloc_linear_workspace(cfg, True))
    keep = lambda n, gone: torch.tensor([i not in gone for i in range(n)], device="cuda")
    for got, ok, rows, cols in ((dx, clean["dx"], keep(M, (7, 9, M - 1, 50)), keep(K, (0, 5))),
                                (dw, clean["dw"], keep(N, (0, 1, 2, N - 1)), keep(K, (0, 3, K - 1)))):
        assert torch.equal(got[rows][:, cols], ok[rows][:, cols])
        assert not bool(torch.isfinite(got[~rows]).any()) and not bool(torch.isfinite(got[:, ~cols]).any())
