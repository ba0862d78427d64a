"""GPU tests of the operators around the MoE layer against plain 64-bit implementations (tests/operators_ref.py).

Outputs start as NaN (or a sentinel) and lie between guard words, so that an element left unwritten or a write past the end
shows.  Tolerances, u = 2^-24 (half a step of fp32), v = 2^-8 (of bf16):
  dropout   one product by a rounded scale and one sum in fp32: u (2 |x s| + |out|), then bf16: v |out|
  balance   see balance_bounds
  linear    on small whole numbers every product and sum is exact in fp32: equal bits.  On normal numbers: see linear_bound
"""
import math

import numpy as np
import pytest
import torch

import paper_2402_12399_amd as rr
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

U, V = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
DT = {"f32": F32, "bf16": BF16}
ACT = {"none": rr.RR_ACT_NONE, "gelu": rr.RR_ACT_GELU, "swiglu": rr.RR_ACT_SWIGLU}
GUARD = 64  # elements before and after every output


class Guarded:
    """A tensor inside a larger buffer of a sentinel value."""

    def __init__(self, shape, dtype):
        n = math.prod(shape)
        self.fill = -12345 if dtype == torch.int32 else float("nan")
        self.buf = torch.full((n + 2 * GUARD,), self.fill, dtype=dtype, device="cuda")
        self.t = self.buf[GUARD:GUARD + n].view(shape)

    def check(self):
        edge = torch.cat([self.buf[:GUARD], self.buf[-GUARD:]])
        assert bool((edge == self.fill).all() if self.buf.dtype == torch.int32 else edge.isnan().all()), "written outside the output"
        if self.buf.dtype != torch.int32:
            assert bool((~self.t.isnan()).all()), "an element is not written"
        return self.t


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def whole(g, *shape, dtype=F32, top=2):
    return torch.randint(-top, top + 1, shape, generator=g, device="cuda").to(dtype)


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound.clamp_min(1e-300)).max()):.3g} of the bound"


# ------------------------------------------------------------------ dropout

def dropout_bound(x, out, scale, dtype):
    b = U * (2 * x.double().abs() * scale + out.abs()) * 1.001 + 1e-45
    return b + (V * (out.abs() + b) + 2.0 ** -134 if dtype == BF16 else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 63, 64, 2047, 2048, 2049, 16384, 100003, (1 << 21) + 13])
def test_dropout(n, residual, dtype):
    g = gen(n)
    x = normal(g, n, dtype=DT[dtype])
    r = normal(g, n, dtype=DT[dtype]) if residual else None
    for p, seed, offset in ((0.1, 1, 0), (0.5, 2 ** 64 - 3, 2 ** 64 - 2), (0.0, 5, 6), (1.0, 7, 8), (1e-6, 9, 10)):
        out = Guarded((n,), DT[dtype])
        rr.rr_dropout(x, p, seed, offset, out.t, residual=r)
        want, keep, scale = ref.dropout(x, r, p, seed, offset)
        got = out.check()
        within(got, want, dropout_bound(x, want, scale, DT[dtype]), f"p {p}")
        base = torch.zeros_like(x) if r is None else r
        assert bool((got[~keep] == base[~keep]).all())
        dx = Guarded((n,), DT[dtype])
        rr.rr_dropout_backward(x, p, seed, offset, dx.t)
        want, _, _ = ref.dropout(x, None, p, seed, offset)
        within(dx.check(), want, dropout_bound(x, want, scale, DT[dtype]), f"backward p {p}")


def test_dropout_drops_nan_and_infinities():
    n = 4096
    x = torch.full((n,), float("nan"), device="cuda")
    x[::2] = float("inf")
    r = normal(gen(1), n)
    _, keep, _ = ref.dropout(x, None, 0.5, 11, 12)
    out = torch.empty_like(x)
    rr.rr_dropout(x, 0.5, 11, 12, out, residual=r)
    assert torch.equal(out[~keep], r[~keep]) and not bool(torch.isfinite(out[keep]).any())
    rr.rr_dropout(x, 1.0, 11, 12, out, residual=r)
    assert torch.equal(out, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_in_place_parts_and_gradient(dtype):
    g, n = gen(2), 40000
    x, r = normal(g, n, dtype=DT[dtype]), normal(g, n, dtype=DT[dtype])
    whole_ = torch.empty_like(x)
    rr.rr_dropout(x, 0.3, 21, 100, whole_, residual=r)
    for alias in ("x", "residual"):  # out may be either input
        a, b = x.clone(), r.clone()
        rr.rr_dropout(a, 0.3, 21, 100, a if alias == "x" else b, residual=b)
        assert torch.equal(a if alias == "x" else b, whole_)
    parts = torch.empty_like(x)  # a part that starts at group 17 makes the same mask from offset + 17
    cut = 17 * 8
    rr.rr_dropout(x[:cut], 0.3, 21, 100, parts[:cut], residual=r[:cut])
    rr.rr_dropout(x[cut:], 0.3, 21, 117, parts[cut:], residual=r[cut:])
    assert torch.equal(parts, whole_)
    # the operator is linear in x: its gradient is the difference quotient, exactly where nothing rounds
    e, d, dx = whole(g, n, dtype=DT[dtype]), whole(g, n, dtype=DT[dtype]), torch.empty_like(x)
    rr.rr_dropout_backward(d, 0.5, 21, 100, dx)
    y = torch.empty_like(x)
    rr.rr_dropout(e, 0.5, 21, 100, y)
    assert float((y.double() * d.double()).sum()) == float((e.double() * dx.double()).sum())


# ------------------------------------------------------------------ balance loss

def balance_bounds(want, logits, coef, dloss):
    """With s the widest span of a row's scores: a probability's exponent is off by at most u s (the difference's rounding), the
    exponential, the sum over up to 64 experts (8 levels), the reciprocal and the product by 16 u more, and so is the sum it is
    divided by: c = (2 s + 20) u relative.  The gradient p (f - mean) takes f from two more roundings and the mean from sums
    of f p of 8 levels.  An exponential below t = 2^-126, the smallest normal number, is taken for 0: p, at most the
    exponential because the sum is at least 1, is then off by t, P_e too, the loss by coef E t, the gradient by 2 scale t."""
    finite = logits[torch.isfinite(logits)]
    s = float((finite.max() - finite.min())) if finite.numel() else 0.0
    c = (2 * s + 20) * U
    E = want["f"].numel()
    pf = (want["p"] * want["f"]).sum(dim=1, keepdim=True)
    n = max(int(want["counts"][-1]), 1)
    scale = abs(dloss * coef) * E / n
    grad = scale * want["p"] * ((c + 8 * U) * (want["f"] + pf) + c * (want["f"] - pf).abs() + (c + 12 * U) * pf)
    t = 2.0 ** -126
    return (c * want["mean_prob"] + t + 1e-40, (c + 4 * U) * float(want["loss"].abs()) + abs(coef) * E * t + 1e-40,
            grad + 2 * scale * t + 1e-40)


def run_balance(a, ranks, k, coef, mask=None, dloss=None, accumulate=None):
    T, E = a.shape
    cfg = rr.RRConfig(T, 8, 0, E, k, 1, 1.0, rr.RR_F32, rr.RR_ACT_SWIGLU, 0)
    loss, counts, mean, grad = Guarded((1,), F32), Guarded((E + 1,), torch.int32), Guarded((E,), F32), Guarded((T, E), F32)
    if accumulate is not None:
        grad.t.copy_(accumulate)
    ws = rr.alloc_balance_workspace(cfg).fill_(255)
    rr.rr_balance_loss(cfg, a, ranks, coef, loss.t, counts.t, ws, mean_prob=mean.t, token_mask=mask)
    d = None if dloss is None else torch.tensor([dloss], device="cuda")
    rr.rr_balance_loss_backward(cfg, a, counts.t, coef, grad.t, dloss=d, token_mask=mask, accumulate=accumulate is not None)
    return loss.check(), counts.check(), mean.check(), grad.check()


def check_balance(a, ranks, k, coef, mask=None, dloss=None):
    loss, counts, mean, grad = run_balance(a, ranks, k, coef, mask, dloss)
    want = ref.balance(a, ranks, k, coef, mask, 1.0 if dloss is None else dloss)
    assert torch.equal(counts.long(), want["counts"])
    bm, bl, bg = balance_bounds(want, a if mask is None else a[mask.bool()], coef, 1.0 if dloss is None else dloss)
    within(mean, want["mean_prob"], bm, "mean_prob")
    assert abs(float(loss) - float(want["loss"])) <= bl, (float(loss), float(want["loss"]))
    within(grad, want["dlogits"], bg, "dlogits")
    return want


def ranks_of(a, k):
    T, E = a.shape
    r = torch.full((T, k + 1), -1, dtype=torch.int32, device=a.device)
    o = torch.sort(torch.nan_to_num(a, nan=0.0), dim=1, descending=True, stable=True).indices[:, :k + 1]
    r[:, :o.shape[1]] = o.int()
    return r


@pytest.mark.parametrize("E", [1, 2, 3, 4, 5, 8, 11, 16, 17, 32, 33, 48, 58, 63, 64])
@pytest.mark.parametrize("T", [1, 2, 63, 257, 5000])
def test_balance(T, E):
    g = gen(T * 100 + E)
    a = normal(g, T, E, scale=2.0)
    k = min(E, 1 + (T + E) % 4)
    check_balance(a, ranks_of(a, k), k, 0.01)
    mask = torch.rand(T, generator=g, device="cuda") < 0.6
    poisoned = a.clone()
    poisoned[~mask] = float("nan")  # what a masked row holds does not matter
    ranks = ranks_of(a, k)
    ranks[~mask] = 1 << 30
    check_balance(poisoned, ranks, k, -0.7, mask, 1.75)
    check_balance(poisoned, ranks, k, -0.7, mask.to(torch.uint8) * 3, 1.75)


@pytest.mark.parametrize("T,E,k", [(200001, 64, 2), (65536, 8, 4), (1 << 20, 6, 1)])
def test_balance_many_tokens(T, E, k):
    g = gen(T)
    a = normal(g, T, E) + normal(g, E, scale=2.0)
    ranks = ranks_of(a, k)
    check_balance(a, ranks, k, 0.01, None, 0.5)
    one, two = run_balance(a, ranks, k, 0.01), run_balance(a, ranks, k, 0.01)
    assert all(torch.equal(p, q) for p, q in zip(one, two))  # the same from run to run


def test_balance_edges():
    g = gen(5)
    a = normal(g, 40, 8)
    ranks = ranks_of(a, 2)
    # nobody counts
    loss, counts, mean, grad = run_balance(a, ranks, 2, 0.5, torch.zeros(40, dtype=torch.uint8, device="cuda"))
    assert float(loss) == 0 and not bool(counts.any()) and not bool(mean.any()) and not bool(grad.any())
    # experts switched off by -infinity, a row of nothing else, the lowest number
    b = a.clone()
    b[:, 3] = float("-inf")
    b[7] = float("-inf")
    b[9, 1] = torch.finfo(F32).min
    want = ref.balance(b, ranks, 2, 0.5)
    loss, counts, mean, grad = run_balance(b, ranks, 2, 0.5)
    bm, bl, bg = balance_bounds(want, a, 0.5, 1.0)
    within(mean, want["mean_prob"], bm, "mean_prob")
    within(grad, want["dlogits"], bg, "dlogits")
    assert torch.equal(counts.long(), want["counts"]) and not bool(grad[7].any()) and not bool(grad[:, 3].any())
    # huge scores, and choices that are no expert
    check_balance(a * 50 + 3e4, ranks, 2, 0.5)
    bad = ranks.clone()
    bad[::3, 0], bad[1::3, 1] = -1, 8
    check_balance(a, bad, 2, 0.5)
    # all on one expert
    check_balance(a, torch.full_like(ranks, 5), 2, 0.5)
    # every expert chosen as often as any other: the gradient is zero, and so is what is written
    for E in (3, 4, 8):
        a = normal(g, 40, E)
        rolled = (torch.arange(40, device="cuda")[:, None] + torch.arange(3, device="cuda")) % E
        _, _, _, grad = run_balance(a[:E * 3], rolled[:E * 3].int(), 2, 0.5)
        assert not bool(grad.any())


@pytest.mark.parametrize("coef,dloss", [(1e37, 1.0), (-1e37, 1.5), (1e30, 1e8), (1e-37, 1e30), (1e-30, 1e-12)])
def test_balance_of_any_finite_coefficient(coef, dloss):
    """coef times the experts and dloss times coef may lie outside fp32's range; their quotient by the tokens does not."""
    g, T, E = gen(15), 300, 64
    a = normal(g, T, E)
    check_balance(a, ranks_of(a, 2), 2, coef, None, dloss)


@pytest.mark.parametrize("E", [6, 7, 8, 64])
def test_balance_accumulates_and_takes_any_alignment(E):
    g, T = gen(6), 333
    a = normal(g, T, E)
    ranks = ranks_of(a, 1)
    mask = torch.rand(T, generator=g, device="cuda") < 0.5
    _, _, _, grad = run_balance(a, ranks, 1, 3.0, mask)
    base = normal(g, T, E)
    _, _, _, both = run_balance(a, ranks, 1, 3.0, mask, accumulate=base)
    assert torch.equal(both, torch.where(mask[:, None], base + grad, base))
    # rows that start 4 bytes behind a 16-byte boundary
    cfg = rr.RRConfig(T, 8, 0, E, 1, 1, 1.0, rr.RR_F32, rr.RR_ACT_SWIGLU, 0)
    buf = torch.empty(T * E + 1, device="cuda")
    buf[1:] = a.reshape(-1)
    out = Guarded((T * E + 1,), F32)
    loss, counts = torch.empty(1, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    rr.rr_balance_loss(cfg, buf[1:].view(T, E), ranks, 3.0, loss, counts, rr.alloc_balance_workspace(cfg), token_mask=mask)
    out.t[0] = 0.0
    rr.rr_balance_loss_backward(cfg, buf[1:].view(T, E), counts, 3.0, out.t[1:].view(T, E), token_mask=mask)
    want = ref.balance(a, ranks, 1, 3.0, mask)
    _, _, bg = balance_bounds(want, a, 3.0, 1.0)
    within(out.check()[1:].view(T, E), want["dlogits"], bg, "dlogits")


# ------------------------------------------------------------------ dense projection

# tiles' edges, single rows, row lengths that are no multiple of 64, K beyond and below a chunk, few rows with long rows
SHAPES = [(1, 8, 8), (2, 24, 16), (1, 4096, 512), (3, 8200, 72), (16, 1000, 264), (17, 64, 128), (33, 72, 136), (64, 256, 264), (65, 2048, 64),
          (129, 192, 320), (255, 200, 520), (256, 256, 256), (257, 1000, 1368), (513, 320, 2056), (1030, 2048, 1544), (3001, 1000, 360),
          (4099, 512, 512), (130, 4160, 1032), (2048, 64, 64), (9000, 72, 40)]


# the tiles and slices that the shapes above leave out (test_operators_host.py checks that none is left)
MORE = [(34, 2712, 4512), (4102, 80, 912), (9095, 8, 1984), (8445, 1688, 8), (1032, 4152, 48), (2471, 5832, 8), (4199, 8, 2864), (5, 5640, 1848),
        (3650, 8, 2480), (7, 2520, 3008), (1228, 1440, 8), (26, 480, 4256), (27, 128, 10600), (12, 2800, 5504), (33, 8, 8672), (42, 1592, 8328),
        (72, 8, 8744), (82, 2952, 5952), (129, 8, 8624), (198, 3224, 10104), (145, 4408, 1224), (38, 2624, 1384), (3, 512, 520), (4, 1000, 264),
        (31, 512, 264), (3, 5144, 4184), (18, 7920, 9840)]


def linear_case(M, K, N, dtype, act, make, seed, bias=True, residual=True):
    g, dt = gen(seed), DT[dtype]
    R = 2 * N if act == "swiglu" else N
    x, w = make(g, M, K, dtype=dt), make(g, R, K, dtype=dt)
    return x, w, make(g, R) if bias else None, make(g, M, N, dtype=dt) if residual else None, R


def run_linear(x, w, bias, residual, act, dtype, N, pre=True):
    M, K = x.shape
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, ACT[act])
    y, z = Guarded((M, N), x.dtype), Guarded((M, w.shape[0]), x.dtype)
    rr.rr_linear(cfg, x, w, bias, residual, y.t, z.t if pre else None, rr.alloc_linear_workspace(cfg).fill_(255))
    return y.check(), z.check() if pre else None


def run_backward(x, w, pre, dy, act, dtype, N, want=("dx", "dw", "dbias")):
    M, K = x.shape
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, ACT[act])
    out = {"dx": Guarded((M, K), x.dtype), "dw": Guarded(tuple(w.shape), x.dtype), "dbias": Guarded((w.shape[0],), F32)}
    args = [out[n].t if n in want else None for n in ("dx", "dw", "dbias")]
    rr.rr_linear_backward(cfg, x, w, pre, dy, *args, rr.alloc_linear_workspace(cfg, True).fill_(255))
    return {n: out[n].check() for n in want}


def nearest(want, dtype):
    return want.to(F32).to(DT[dtype])  # fp32 holds it exactly, so this rounds once


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES + MORE)
def test_linear_exact_sums(M, K, N, dtype):
    """Whole numbers up to 2: sums stay below 2^24, so the output is the rounded exact one, bit for bit."""
    for bias, residual in ((True, True), (False, False)):
        x, w, b, r, _ = linear_case(M, K, N, dtype, "none", whole, M + K + N, bias, residual)
        y, z = run_linear(x, w, b, r, "none", dtype, N)
        want, want_z = ref.linear(x, w, b, r, "none")
        assert torch.equal(z, nearest(want_z, dtype)) and torch.equal(y, nearest(want, dtype))
    y2, _ = run_linear(x, w, None, None, "none", dtype, N, pre=False)
    assert torch.equal(y, y2)
    dy = whole(gen(1), M, N, dtype=DT[dtype])
    want = ref.linear_backward(x, w, None, dy, "none")
    got = run_backward(x, w, None, dy, "none", dtype, N)
    for n in got:
        assert torch.equal(got[n], nearest(want[n], dtype) if n != "dbias" else want[n].to(F32)), n


# 256 x 256 tiles in the forward product, in dx (W read as it lies) and in dw (dz and x read as they lie); rows and row lengths that end
# inside a tile and inside a chunk, a last round of tiles that is cut by rows, and slices of dw
LARGE = [(4099, 1000, 4104, "none"), (8195, 2048, 1416, "swiglu"), (2051, 4160, 4104, "gelu"), (33001, 1032, 520, "none"), (20011, 520, 1032, "swiglu")]


@pytest.mark.parametrize("M,K,N,act", LARGE)
def test_linear_large_tiles(M, K, N, act):
    from tests import gpu_util as gu
    plans = gu.linear_plans(rr.RRLinearConfig(M, K, N, rr.RR_BF16, ACT[act]))
    print(plans)
    x, w, b, r, R = linear_case(M, K, N, "bf16", "none", whole, M)
    cfg = rr.RRLinearConfig(M, K, R, rr.RR_BF16, rr.RR_ACT_NONE)
    if act == "none":
        y, z = run_linear(x, w, b, r, "none", "bf16", N)
        want, want_z = ref.linear(x, w, b, r, "none")
        assert torch.equal(z, nearest(want_z, "bf16")) and torch.equal(y, nearest(want, "bf16"))
    # the products of the gradients on whole numbers: without an activation dz is dy
    dy = whole(gen(1), M, N, dtype=BF16)
    want = ref.linear_backward(x, w, None, dy, "none")
    got = run_backward(x, w, None, dy, "none", "bf16", N)
    for n in got:
        assert torch.equal(got[n], nearest(want[n], "bf16") if n != "dbias" else want[n].to(F32)), n
    x[5] = float("nan")  # a row that is not finite reaches its own row and column of the gradients only
    dy[7] = float("inf")
    bad = run_backward(torch.nan_to_num(x), w, None, torch.nan_to_num(dy, posinf=1.0), "none", "bf16", N, ("dx",))
    assert bool(torch.isfinite(bad["dx"]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", MORE)
def test_linear_gated_tiles(M, K, N, dtype):
    """The gated forward product of the shapes above: the pre-activations are exact sums, and y is made of them."""
    x, w, b, r, _ = linear_case(M, K, N, dtype, "swiglu", whole, M)
    y, z = run_linear(x, w, b, r, "swiglu", dtype, N)
    want, want_z = ref.linear(x, w, b, r, "swiglu")
    assert torch.equal(z, nearest(want_z, dtype))
    g, u = want_z.chunk(2, dim=1)
    # silu of an exact number: exponential, sum, division and product, 8 u of it; the product with u, the residual's sum and the rounding.
    # Below g = -88.7 exp(-g) is infinite in fp32 and silu(g), at most 88.7 exp(-88.7) = 2.7e-37 there, is taken for 0
    e = 10 * U * (torch.nn.functional.silu(g) * u).abs() + 2 * U * want.abs() + 2.7e-37 * u.abs()
    within(y, want, e + (V if dtype == "bf16" else U) * (want.abs() + e) + 1e-38, "y")


def linear_bound(abs_sum, terms, value, dtype, slope=1.0, extra=0.0):
    """abs_sum = sum of |products|, terms of them added in fp32 in any order: every partial sum is at most abs_sum and is
    rounded once (twice in a matrix instruction): 2 u abs_sum per addition in the worst case, and at most 8 sqrt(terms) of
    those behind one another in the same direction with probability 1 - 1e-14 (independent roundings); never more than terms."""
    b = 2 * U * abs_sum * min(terms, 8 * math.sqrt(terms) + 8) * slope + extra
    return b + (V if dtype == "bf16" else 2 * U) * (value.abs() + b) + 1e-38


ACT_SLOPE = {"none": 1.0, "gelu": 1.13, "swiglu": 1.1}


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_linear_values_and_gradients(M, K, N, dtype, act):
    make = lambda g, *s, dtype=F32: normal(g, *s, dtype=dtype, scale=1.0 if s[-1] != K or s[0] == M else K ** -0.5)
    x, w, b, r, R = linear_case(M, K, N, dtype, act, make, M * 3 + K + N)
    y, pre = run_linear(x, w, b, r, act, dtype, N)
    want, z = ref.linear(x, w, b, r, act)
    a = torch.mm(x.double().abs(), w.double().abs().t()) + b.double().abs()
    within(pre, z, linear_bound(a, K + 1, z, dtype), "pre")
    # the activation's own arithmetic: a dozen roundings of its value; an error of z passes by its slope (swiglu: times the other factor)
    if act == "swiglu":
        g_, u_ = z.chunk(2, dim=1)
        ag, au = a.chunk(2, dim=1)
        own = ref.act(z, act)
        e = linear_bound(ag, K + 1, g_, "f32") * (u_.abs() * 1.1 + linear_bound(au, K + 1, u_, "f32")) + linear_bound(au, K + 1, u_, "f32") * torch.nn.functional.silu(g_).abs()
    else:
        own = ref.act(z, act)
        e = linear_bound(a, K + 1, z, "f32") * ACT_SLOPE[act]
    e = e + 16 * U * (own.abs() + (z[:, :N].abs() if act != "none" else 0.0)) + 2 * U * r.double().abs()
    within(y, want, e + (V if dtype == "bf16" else U) * (want.abs() + e) + 1e-38, "y")
    if dtype == "f32":  # and as a whole: roundings of sums that grow like sqrt(k) add up to u sqrt(K / 6) of the result, 4 times that is never reached
        err = float((pre.double() - z).norm() / z.norm())
        assert err <= 4 * U * math.sqrt(K / 6) + 2 * U, err

    dy = normal(gen(9), M, N, dtype=DT[dtype])
    zs = None if act == "none" else pre
    want = ref.linear_backward(x, w, zs, dy, act)
    got = run_backward(x, w, zs, dy, act, dtype, N)
    dz = want["dz"]
    # dz: 24 roundings of products of factors up to |dy| (1 + |z|) (the gated one: its partner), in bf16 one to bf16 more
    if act == "none":
        edz = torch.zeros_like(dz)
    else:
        zz = zs.double()
        f = torch.cat([zz[:, N:].abs() + 1e-3, zz[:, :N].abs() + 1e-3], dim=1) if act == "swiglu" else torch.ones_like(zz)
        edz = 24 * U * torch.cat([dy.double().abs()] * (R // N), dim=1) * f * (1 + zz.abs().repeat(1, 1)) if act == "gelu" else \
            24 * U * torch.cat([dy.double().abs()] * 2, dim=1) * f * (1 + torch.cat([zz[:, :N].abs()] * 2, dim=1))
    within(got["dbias"], want["dbias"], edz.sum(dim=0) + 2 * U * dz.abs().sum(dim=0) + U * want["dbias"].abs() + 1e-38, "dbias")
    rdz = edz + (V * (dz.abs() + edz) if dtype == "bf16" and act != "none" else 0.0)
    for name, left, right, dleft, terms in (("dx", dz.abs(), w.double().abs(), rdz, R), ("dw", dz.t().abs(), x.double().abs(), rdz.t(), M)):
        s = torch.mm(left.contiguous(), right)
        # independent roundings of dz: eight standard deviations of their sum, never more than all of them
        spread = torch.minimum(torch.mm(dleft.contiguous(), right), 8 * torch.sqrt(torch.mm(dleft.contiguous() ** 2, right ** 2)))
        within(got[name], want[name], linear_bound(s, terms, want[name], dtype, extra=spread), name)


def test_linear_outputs_on_request():
    x, w, b, r, R = linear_case(130, 72, 136, "bf16", "swiglu", whole, 1)
    _, pre = run_linear(x, w, b, None, "swiglu", "bf16", 136)
    dy = whole(gen(2), 130, 136, dtype=BF16)
    full = run_backward(x, w, pre, dy, "swiglu", "bf16", 136)
    for want in (("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ("dw", "dbias"), ("dx", "dw")):
        got = run_backward(x, w, pre, dy, "swiglu", "bf16", 136, want)
        assert all(torch.equal(got[n], full[n]) for n in want), want
    # x serves dw only, w serves dx only
    cfg = rr.RRLinearConfig(130, 72, 136, rr.RR_BF16, rr.RR_ACT_SWIGLU)
    ws = rr.alloc_linear_workspace(cfg, True)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    rr.rr_linear_backward(cfg, None, w, pre, dy, dx, None, None, ws)
    rr.rr_linear_backward(cfg, x, None, pre, dy, None, dw, None, ws)
    assert torch.equal(dx, full["dx"]) and torch.equal(dw, full["dw"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 512, 64), (40, 1024, 136), (300, 256, 520), (1100, 1024, 1032)])
def test_linear_residual_is_the_output(M, K, N, dtype):
    x, w, b, r, _ = linear_case(M, K, N, dtype, "gelu", normal, 5)
    y, _ = run_linear(x, w, b, r, "gelu", dtype, N)
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, rr.RR_ACT_GELU)
    rr.rr_linear(cfg, x, w, b, r, r, None, rr.alloc_linear_workspace(cfg))
    assert torch.equal(r, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(5, 512, 72), (600, 264, 520)])
def test_linear_infinities_and_nan_stay_in_their_rows(M, K, N, dtype):
    x, w, b, _, _ = linear_case(M, K, N, dtype, "none", normal, 6)
    clean, _ = run_linear(x, w, b, None, "none", dtype, N, pre=False)
    x[2, 7], x[4, K - 1] = float("nan"), float("inf")
    w[9, 5] = float("-inf")
    y = torch.empty_like(clean)
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, rr.RR_ACT_NONE)
    rr.rr_linear(cfg, x, w, b, None, y, None, rr.alloc_linear_workspace(cfg))
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[2] = rows[4] = False
    cols = torch.ones(N, dtype=torch.bool, device="cuda")
    cols[9] = False
    # fp32 rows next to a number that is not finite may be summed another way: both results are within the bound of the exact one
    x[2], x[4], w[9] = 0.0, 0.0, 0.0
    a = torch.mm(x.double().abs(), w.double().abs().t()) + b.double().abs()
    both = 2 * linear_bound(a, K + 1, clean.double(), dtype) if dtype == "f32" else torch.zeros_like(a)
    within(y[rows][:, cols], clean[rows][:, cols].double(), both[rows][:, cols], "rows and columns without them")
    assert bool(y[2].isnan().all()) and not bool(torch.isfinite(y[4]).any()) and not bool(torch.isfinite(y[:, 9]).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(70, 72, 136), (700, 1000, 264), (1030, 2048, 1544)])
def test_gradients_keep_nan_and_infinities_apart(M, K, N, dtype):
    """x[m, k] reaches column k of dw, dy[m, n] row m of dx and row n of dw; all other sums are of whole numbers, exact either way."""
    x, w, _, _, _ = linear_case(M, K, N, dtype, "none", whole, 7, False, False)
    dy = whole(gen(8), M, N, dtype=DT[dtype])
    clean = run_backward(x, w, None, dy, "none", dtype, N, ("dx", "dw"))
    x[5, 3], dy[7, 2] = float("nan"), float("inf")
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, rr.RR_ACT_NONE)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    rr.rr_linear_backward(cfg, x, w, None, dy, dx, dw, None, rr.alloc_linear_workspace(cfg, True))
    rows = torch.arange(M, device="cuda") != 7
    outs, cols = torch.arange(N, device="cuda") != 2, torch.arange(K, device="cuda") != 3
    assert torch.equal(dx[rows], clean["dx"][rows]) and torch.equal(dw[outs][:, cols], clean["dw"][outs][:, cols])
    assert not bool(torch.isfinite(dx[7][w[2] != 0]).any()) and bool(dw[:, 3].isnan().all())


@pytest.mark.parametrize("M,K,N", [(3, 264, 72), (20, 264, 72), (300, 264, 520), (600, 2048, 264)])
@pytest.mark.parametrize("ex,ew", [(60, 40), (-100, -20), (-140, 20), (20, -60)])
def test_linear_f32_keeps_the_whole_range(M, K, N, ex, ew):
    """Whole numbers times powers of two, subnormal ones among them: sums are exact however the operands are cut."""
    x, w, _, _, _ = linear_case(M, K, N, "f32", "none", whole, 9, False, False)
    big, want = x * 2.0 ** ex, torch.mm(x.double(), w.double().t()) * 2.0 ** (ex + ew)
    y, _ = run_linear(big, w * 2.0 ** ew, None, None, "none", "f32", N, pre=False)
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("M,K,N", [(37, 520, 264), (130, 264, 1032), (1030, 2048, 1544), (700, 1000, 200)])
@pytest.mark.parametrize("ed,eo", [(60, 40), (-100, -20), (-140, 20), (20, -60)])
def test_gradients_f32_keep_the_whole_range(M, K, N, ed, eo):
    """As above, of operands that lie the other way round."""
    x, w, _, _, _ = linear_case(M, K, N, "f32", "none", whole, 21, False, False)
    dy = whole(gen(22), M, N, dtype=F32)
    got = run_backward(x * 2.0 ** eo, w * 2.0 ** eo, None, dy * 2.0 ** ed, "none", "f32", N, ("dx", "dw"))
    for name, want in (("dx", torch.mm(dy.double(), w.double())), ("dw", torch.mm(dy.double().t().contiguous(), x.double()))):
        assert torch.equal(got[name].double(), want * 2.0 ** (ed + eo)), name


def test_linear_bias_needs_four_byte_alignment_only():
    for M, act in ((2, "none"), (40, "gelu"), (300, "swiglu")):
        x, w, b, r, R = linear_case(M, 264, 136, "bf16", act, normal, 10)
        y, _ = run_linear(x, w, b, r, act, "bf16", 136)
        shifted = torch.empty(R + 1, device="cuda")
        shifted[1:] = b
        again, _ = run_linear(x, w, shifted[1:], r, act, "bf16", 136)
        assert torch.equal(y, again)


# ------------------------------------------------------------------ offsets beyond 32 bits, the longest rows and the most of them

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1 << 21, 1032, 64), (40, 1 << 18, 16), (3, 1 << 18, 16), (40, 16, 1 << 18), (300, 1 << 17, 72)])
def test_linear_at_the_limits(M, K, N, dtype):
    """Whole numbers, sums below 2^24: exact.  Of the many rows some are compared, and every sum over them (dw, dbias)."""
    g, dt = gen(12), DT[dtype]
    x, w, dy = whole(g, M, K, dtype=dt, top=1), whole(g, N, K, dtype=dt, top=1), whole(g, M, N, dtype=dt, top=1)
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dtype == "f32" else rr.RR_BF16, rr.RR_ACT_NONE)
    y, dx, dw, db = torch.full((M, N), float("nan"), dtype=dt, device="cuda"), torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.empty(N, device="cuda")
    rr.rr_linear(cfg, x, w, None, None, y, None, rr.alloc_linear_workspace(cfg))
    rr.rr_linear_backward(cfg, x, w, None, dy, dx, dw, db, rr.alloc_linear_workspace(cfg, True))
    some = torch.unique(torch.cat([torch.arange(min(M, 300), device="cuda"), torch.arange(max(0, M - 300), M, device="cuda"),
                                   torch.randint(0, M, (300,), generator=g, device="cuda")]))
    assert torch.equal(y[some], nearest(torch.mm(x[some].double(), w.double().t()), dtype))
    assert torch.equal(dx[some], nearest(torch.mm(dy[some].double(), w.double()), dtype))
    want = torch.zeros(N, K, dtype=torch.float64, device="cuda")
    for a in range(0, M, 1 << 17):
        want += torch.mm(dy[a:a + (1 << 17)].double().t().contiguous(), x[a:a + (1 << 17)].double())
    assert torch.equal(dw, nearest(want, dtype)) and torch.equal(db.double(), dy.double().sum(dim=0))


def test_dropout_beyond_32_bits():
    n = (1 << 31) + 13
    x = torch.ones(n, dtype=BF16, device="cuda")
    out = torch.zeros_like(x)
    rr.rr_dropout(x, 0.25, 3, 2 ** 63, out, residual=x)
    for a in (0, (1 << 30) - 8, (1 << 31) - 4096):
        b = min(n, a + 8192)
        want, _, _ = ref.dropout(x[a:b], x[a:b], 0.25, 3, 2 ** 63 + a // 8)
        assert torch.equal(out[a:b], nearest(want, "bf16"))


def test_balance_of_the_most_tokens():
    T, E, k = 1 << 24, 64, 2
    g = gen(14)
    a = torch.randn((T, E), generator=g, device="cuda")
    ranks = torch.randint(0, E, (T, k + 1), generator=g, device="cuda", dtype=torch.int32)
    cfg = rr.RRConfig(T, 8, 0, E, k, 1, 1.0, rr.RR_F32, rr.RR_ACT_SWIGLU, 0)
    loss, counts, mean, grad = (torch.empty(s, device="cuda") for s in (1, E + 1, E, a.shape))
    counts = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    rr.rr_balance_loss(cfg, a, ranks, 1.0, loss, counts, rr.alloc_balance_workspace(cfg), mean_prob=mean)
    rr.rr_balance_loss_backward(cfg, a, counts, 1.0, grad)
    total, want_counts = torch.zeros(E, dtype=torch.float64, device="cuda"), torch.zeros(E, dtype=torch.int64, device="cuda")
    for t in range(0, T, 1 << 21):
        total += torch.softmax(a[t:t + (1 << 21)].double(), dim=1).sum(dim=0)
        want_counts += torch.bincount(ranks[t:t + (1 << 21), :k].reshape(-1).long(), minlength=E)
    assert torch.equal(counts[:E].long(), want_counts) and int(counts[E]) == T
    s = float(a.max() - a.min())
    c = (2 * s + 20) * U
    within(mean, total / T, c * total / T, "mean_prob")
    f = want_counts.double() / (k * T)
    assert abs(float(loss) - float(E * (f * total / T).sum())) <= (c + 4 * U) * float(E * (f * total / T).sum())
    for t in (0, T // 2 - 1000, T - 4096):
        p = torch.softmax(a[t:t + 4096].double(), dim=1)
        pf = (p * f).sum(dim=1, keepdim=True)
        scale = E / T
        bound = scale * p * ((c + 8 * U) * (f + pf) + c * (f - pf).abs() + (c + 12 * U) * pf) + 1e-40
        within(grad[t:t + 4096], scale * p * (f - pf), bound, "dlogits")


def test_neighbours_in_one_buffer():
    """Operands and results that lie next to one another, without a byte between them, are all there is to tell apart."""
    M, K, N, at = 48, 64, 32, 0
    store = torch.empty(1 << 16, dtype=BF16, device="cuda")

    def take(*shape):
        nonlocal at
        n = math.prod(shape)
        at += n
        return store[at - n:at].view(shape)
    x, y, w, pre, dy, dx, dw = take(M, K), take(M, N), take(2 * N, K), take(M, 2 * N), take(M, N), take(M, K), take(2 * N, K)
    for t in (x, w, dy):
        t.copy_(normal(gen(31), *t.shape, dtype=BF16))
    cfg = rr.RRLinearConfig(M, K, N, rr.RR_BF16, rr.RR_ACT_SWIGLU)
    rr.rr_linear(cfg, x, w, None, None, y, pre, rr.alloc_linear_workspace(cfg))
    rr.rr_linear_backward(cfg, x, w, pre, dy, dx, dw, None, rr.alloc_linear_workspace(cfg, True))
    x, w, dy = x.clone(), w.clone(), dy.clone()
    apart_y, apart_pre = run_linear(x, w, None, None, "swiglu", "bf16", N)
    assert torch.equal(apart_y, y) and torch.equal(apart_pre, pre)
    apart = run_backward(x, w, apart_pre, dy, "swiglu", "bf16", N, ("dx", "dw"))
    assert torch.equal(apart["dx"], dx) and torch.equal(apart["dw"], dw)
    a, b = store[:1000], store[1000:2000]
    rr.rr_dropout(a, 0.5, 1, 2, b)
    assert torch.equal(b, (lambda o: (rr.rr_dropout(a, 0.5, 1, 2, o), o)[1])(torch.empty_like(a)))


# ------------------------------------------------------------------ streams, graphs, both calls at once

def _calls():
    """(name, call on given buffers -> outputs) of each operator at a size of several workgroups"""
    g = gen(7)
    x, w, b, r, R = linear_case(300, 520, 264, "bf16", "swiglu", normal, 7)
    lc = rr.RRLinearConfig(300, 520, 264, rr.RR_BF16, rr.RR_ACT_SWIGLU)
    ws, wsb = rr.alloc_linear_workspace(lc), rr.alloc_linear_workspace(lc, True)
    y, pre, dy = torch.empty(300, 264, dtype=BF16, device="cuda"), torch.empty(300, R, dtype=BF16, device="cuda"), normal(g, 300, 264, dtype=BF16)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(R, device="cuda")
    a = normal(g, 20000, 24)
    ranks, mask = ranks_of(a, 2), (torch.rand(20000, generator=g, device="cuda") < 0.9)
    bc = rr.RRConfig(20000, 8, 0, 24, 2, 1, 1.0, rr.RR_F32, rr.RR_ACT_SWIGLU, 0)
    bws = rr.alloc_balance_workspace(bc)
    loss, counts, mean, da = torch.empty(1, device="cuda"), torch.empty(25, dtype=torch.int32, device="cuda"), torch.empty(24, device="cuda"), torch.empty_like(a)
    d, res, out, ddx = normal(g, 99991), normal(g, 99991), torch.empty(99991, device="cuda"), torch.empty(99991, device="cuda")

    def linear():
        rr.rr_linear(lc, x, w, b, r, y, pre, ws)
        rr.rr_linear_backward(lc, x, w, pre, dy, dx, dw, db, wsb)
        return [y, pre, dx, dw, db]

    def balance():
        rr.rr_balance_loss(bc, a, ranks, 0.01, loss, counts, bws, mean_prob=mean, token_mask=mask)
        rr.rr_balance_loss_backward(bc, a, counts, 0.01, da, dloss=loss, token_mask=mask)
        return [loss, counts, mean, da]

    def dropout():
        rr.rr_dropout(d, 0.2, 3, 4, out, residual=res)
        rr.rr_dropout_backward(out, 0.2, 3, 4, ddx)
        return [out, ddx]
    return [("linear", linear), ("balance", balance), ("dropout", dropout)]


def test_captured_and_replayed():
    rr.rr_init()
    for name, call in _calls():
        eager = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = call()
        for _ in range(3):
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for got, want in zip(outs, eager):
                assert torch.equal(got, want), name


def test_captured_dropout_draws_another_mask_each_replay():
    rr.rr_init()
    x, out = torch.ones(8 * 1000, device="cuda"), torch.empty(8 * 1000, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rr.rr_dropout(x, 0.5, 77, 5, out, device_offset=step)
        step += 1000
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want, _, _ = ref.dropout(x, None, 0.5, 77, 5 + 1000 * i)
        assert torch.equal(out.double(), want), i


def test_streams_of_the_caller():
    """A call runs on the caller's current stream, behind what that stream still has to do; calls on two streams do not meet."""
    calls = _calls()
    alone = {name: [t.clone() for t in call()] for name, call in calls}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    outs = {}
    for (name, call), s in zip(calls, streams):
        with torch.cuda.stream(s):
            outs[name] = call()
    torch.cuda.synchronize()
    for name in outs:
        assert all(torch.equal(p, q) for p, q in zip(outs[name], alone[name])), name
    x, late = torch.ones(1 << 22, device="cuda"), torch.empty(1 << 22, device="cuda")
    with torch.cuda.stream(streams[0]):
        for _ in range(20):
            x = x * 1.0
        x = x + 1.0
        rr.rr_dropout(x, 0.5, 1, 0, late)
    torch.cuda.synchronize()
    want, _, _ = ref.dropout(torch.full_like(late, 2.0), None, 0.5, 1, 0)
    assert torch.equal(late.double(), want)


# ------------------------------------------------------------------ all of them together

def test_training_step_of_two_layers():
    """A routed layer, its dropout and residual, a dense SwiGLU layer with its residual and the balance loss: forward, then every gradient
    that the library makes, against 64 bits; then the same captured in a graph and replayed."""
    from oracle import rectify_router as orc
    from paper_2402_12399_amd import workloads as wl
    from tests import gpu_util as gu
    w = wl.C1
    inputs = wl.make_inputs(w)
    cfg = gu.config_of(w)
    T, d, F, E = w.T, w.d_model, 192, w.E
    dev = {n: None if inputs[n] is None else torch.from_numpy(inputs[n]).cuda() for n in ("x", "w_router", "bias", "w1", "w2")}
    g = gen(11)
    up_w, down_w, up_b = normal(g, 2 * F, d, scale=d ** -0.5), normal(g, d, F, scale=F ** -0.5), normal(g, 2 * F, scale=0.1)
    dy = normal(g, T, d)
    p, seed, offset, coef = 0.1, 5, 1000, 0.01
    f32 = lambda *s: torch.full(s, float("nan"), device="cuda")
    out, logits, tables, ws = f32(T, d), f32(T, E), rr.alloc_tables(cfg), rr.alloc_workspace(cfg)
    up_cfg, down_cfg = rr.RRLinearConfig(T, d, F, rr.RR_F32, rr.RR_ACT_SWIGLU), rr.RRLinearConfig(T, F, d, rr.RR_F32, rr.RR_ACT_NONE)
    lws = torch.empty(max(rr.rr_linear_workspace_bytes(c, b) for c in (up_cfg, down_cfg) for b in (False, True)), dtype=torch.uint8, device="cuda")
    bws = rr.alloc_balance_workspace(cfg)
    r1, h, pre, y = f32(T, d), f32(T, F), f32(T, 2 * F), f32(T, d)
    loss, counts, dloss = f32(1), torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.full((1,), 2.0, device="cuda")
    dh, d_down, dr1, d_up, d_upb, dout, dlogits = f32(T, F), f32(d, F), f32(T, d), f32(2 * F, d), f32(2 * F), f32(T, d), f32(T, E)

    def step():
        rr.rr_moe_forward(cfg, dev["x"], dev["w_router"], dev["bias"], dev["w1"], None, dev["w2"], out, tables, logits, ws)
        rr.rr_dropout(out, p, seed, offset, r1, residual=dev["x"])
        rr.rr_linear(up_cfg, r1, up_w, up_b, None, h, pre, lws)
        rr.rr_linear(down_cfg, h, down_w, None, r1, y, None, lws)
        rr.rr_balance_loss(cfg, logits, tables.rank_expert, coef, loss, counts, bws)
        rr.rr_linear_backward(down_cfg, h, down_w, None, dy, dh, d_down, None, lws)
        rr.rr_linear_backward(up_cfg, r1, up_w, pre, dh, dr1, d_up, d_upb, lws)
        dr1.add_(dy)  # the residual of the dense layer
        rr.rr_dropout_backward(dr1, p, seed, offset, dout)
        rr.rr_router_backward(cfg, dout, logits, tables, ws, dlogits)
        rr.rr_balance_loss_backward(cfg, logits, counts, coef, dlogits, dloss=dloss, accumulate=True)
    step()
    torch.cuda.synchronize()
    results = dict(y=y, loss=loss, counts=counts, dh=dh, d_down=d_down, d_up=d_up, d_upb=d_upb, dout=dout, dlogits=dlogits)
    eager = {n: t.clone() for n, t in results.items()}

    a, want_t, moe = orc.moe_forward(inputs["x"], inputs["w_router"], inputs["bias"], inputs["w1"], None, inputs["w2"], w.k, w.G,
                                     w.capacity_factor, w.act, True, True)
    moe = torch.from_numpy(np.asarray(moe)).double().cuda().requires_grad_()
    up, dn, ub = (t.double().requires_grad_() for t in (up_w, down_w, up_b))
    _, keep, scale = ref.dropout(out, None, p, seed, offset)
    r = dev["x"].double() + torch.where(keep, moe * scale, torch.zeros_like(moe))
    z = torch.mm(r, up.t()) + ub
    hid = torch.nn.functional.silu(z[:, :F]) * z[:, F:]
    hid.retain_grad()
    yy = r + torch.mm(hid, dn.t())
    (yy * dy.double()).sum().backward()
    la = torch.from_numpy(np.asarray(a)).cuda()
    bal = ref.balance(la, tables.rank_expert, w.k, coef, dloss=2.0)
    _, da = orc.router_score_gradient(inputs["x"], a, want_t, w.k, inputs["w1"], None, inputs["w2"], w.act, moe.grad.cpu().numpy())
    want = dict(y=yy, loss=bal["loss"].reshape(1), dh=hid.grad, d_down=dn.grad, d_up=up.grad, d_upb=ub.grad, dout=moe.grad,
                dlogits=torch.from_numpy(np.asarray(da)).cuda() + bal["dlogits"])
    # fp32 throughout, sums of up to 384 terms, three products behind one another: the bar of the layer's fp32 tests
    for n, v in want.items():
        err = float((eager[n].double() - v.detach()).norm() / v.detach().norm())
        assert err <= 1e-5, (n, err)
    assert torch.equal(eager["counts"].long(), bal["counts"])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in results.values():
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, eager[n]) for n, t in results.items())


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_linear_gradients_against_differences(act):
    """Central differences of the kernel's own forward pass along random directions.  With step s the difference is off by s^2 / 6 of a
    third derivative (below 3 per unit of z here) and by the roundings of two losses, each a sum of 200 x 48 terms of about 1."""
    M, K, N = 200, 64, 48
    g = gen(13)
    R = 2 * N if act == "swiglu" else N
    x, w, b, dy = normal(g, M, K), normal(g, R, K, scale=K ** -0.5), normal(g, R, scale=0.3), normal(g, M, N)
    _, pre = run_linear(x, w, b, None, act, "f32", N)
    got = run_backward(x, w, pre, dy, act, "f32", N)
    loss = lambda x, w, b: float((run_linear(x, w, b, None, act, "f32", N, pre=False)[0].double() * dy.double()).sum())
    s = 2.0 ** -7
    for which, grad in ((0, got["dx"]), (1, got["dw"]), (2, got["dbias"])):
        args = [x, w, b]
        dirn = normal(g, *args[which].shape)
        up, dn = list(args), list(args)
        up[which], dn[which] = args[which] + s * dirn, args[which] - s * dirn
        num = (loss(*up) - loss(*dn)) / (2 * s)
        want = float((grad.double() * dirn.double()).sum())
        # z moves by at most 6 per unit of s; 9600 terms: s^2 / 6 * 3 * 6^3 * |dy| of each, signs at random (8 sigma);
        # roundings 2 u K^1/2 of a term, the same way
        slack = 8 * math.sqrt(M * N) * (s * s / 6 * 3 * 6 ** 3 + 8 * U * math.sqrt(K) / s)
        assert abs(num - want) <= slack and abs(want) > 0, (which, num, want, slack)
