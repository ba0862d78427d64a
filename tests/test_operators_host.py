"""CPU checks of the operators around the layer: what the plain implementations of the tests rest on, and every refusal - nothing
here reaches a kernel launch."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

import paper_2402_12399_amd as rr
from paper_2402_12399_amd import binding
from tests import operators_ref as ref

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE, ODD16, ODD4 = C.c_void_p(0x1000), C.c_void_p(0x1008), C.c_void_p(0x1002)
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rr.library_path()):
        from paper_2402_12399_amd import build
        build.build(verbose=False)
    return rr.load_library()


# ------------------------------------------------------------------ the plain implementations

@pytest.mark.parametrize("low,high,key,want", [
    # the published known answers of Philox4x32-10
    (0, 0, 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    (0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822, (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(low, high, key, want):
    assert tuple(int(v) for v in ref.philox4x32([low], key, high)[0]) == want


def test_generator_is_uniform_and_counters_wrap():
    u = ref.random_halves(12345, 7, 1 << 20)
    # a mean of 2^20 uniform numbers: sigma 65536 / sqrt(12 * 2^20) = 18.5
    assert abs(u.astype(np.float64).mean() - 32767.5) < 6 * 18.5
    assert np.array_equal(u[8:24], ref.random_halves(12345, 8, 16))
    assert np.array_equal(ref.random_halves(5, 2 ** 64 - 1, 16)[8:], ref.random_halves(5, 0, 8))


@pytest.mark.parametrize("name", ["none", "gelu", "swiglu"])
def test_plain_linear_gradients_against_differences(name):
    g = torch.Generator().manual_seed(3)
    R = 12 if name == "swiglu" else 6
    x, w = torch.randn(5, 4, generator=g).double(), torch.randn(R, 4, generator=g).double()
    b, dy = torch.randn(R, generator=g).double(), torch.randn(5, 6, generator=g).double()
    loss = lambda x, w, b: float((ref.linear(x, w, b, None, name)[0] * dy).sum())
    got = ref.linear_backward(x, w, ref.linear(x, w, b, None, name)[1], dy, name)
    h = 1e-6
    for which, t, grad in ((0, x, got["dx"]), (1, w, got["dw"]), (2, b, got["dbias"])):
        for i in range(t.numel()):
            args = [x.clone(), w.clone(), b.clone()]
            args[which].view(-1)[i] += h
            up = loss(*args)
            args[which].view(-1)[i] -= 2 * h
            assert abs((up - loss(*args)) / (2 * h) - float(grad.reshape(-1)[i])) < 1e-7 * (1 + abs(float(grad.reshape(-1)[i]))) + 1e-8


def test_plain_balance_gradient_against_differences():
    g = torch.Generator().manual_seed(4)
    a = torch.randn(7, 5, generator=g).double()
    ranks = torch.argsort(-a, dim=1)[:, :3].int()
    mask = torch.tensor([1, 1, 0, 1, 1, 1, 0])
    got = ref.balance(a, ranks, 2, 0.3, mask)
    h = 1e-6
    for t in range(7):
        for e in range(5):
            up, dn = a.clone(), a.clone()
            up[t, e] += h
            dn[t, e] -= h
            d = (ref.balance(up, ranks, 2, 0.3, mask)["loss"] - ref.balance(dn, ranks, 2, 0.3, mask)["loss"]) / (2 * h)
            assert abs(float(d - got["dlogits"][t, e])) < 1e-8
    # uniform routing: the loss is the coefficient
    u = ref.balance(torch.zeros(4, 4), torch.tensor([[0, 1, 2], [1, 2, 3], [2, 3, 0], [3, 0, 1]]), 2, 0.3)
    assert math.isclose(float(u["loss"]), 0.3, rel_tol=1e-12)


def test_plain_dropout_expectation():
    x = torch.ones(1 << 18)
    out, keep, scale = ref.dropout(x, None, 0.1, 99, 0)
    # sigma of the mean: sqrt(p / (1 - p) / n)
    assert abs(float(out.mean()) - 1.0) < 6 * math.sqrt(0.1 / 0.9 / x.numel())
    assert set(out[keep].tolist()) == {scale} and not out[~keep].any()


# ------------------------------------------------------------------ refusals at the C entries

def _linear(**kw):
    c = dict(M=16, K=64, N=64, dtype=rr.RR_BF16, act=rr.RR_ACT_GELU)
    c.update(kw)
    return rr.RRLinearConfig(**c).c()


@pytest.mark.parametrize("kw,want", [
    (dict(), 0), (dict(M=1, K=8, N=8), 0), (dict(M=0), INVALID), (dict(K=0), INVALID), (dict(N=-8), INVALID),
    (dict(K=60), UNSUPPORTED), (dict(N=4), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(act=3), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(M=1 << 21), 0), (dict(M=(1 << 21) + 1), UNSUPPORTED), (dict(K=1 << 18), 0), (dict(K=(1 << 18) + 8), UNSUPPORTED),
    (dict(N=1 << 18), 0), (dict(N=(1 << 18) + 8), UNSUPPORTED), (dict(N=1 << 18, act=rr.RR_ACT_SWIGLU), UNSUPPORTED),
    (dict(N=1 << 17, act=rr.RR_ACT_SWIGLU), 0),
])
def test_linear_configurations(lib, kw, want):
    n, c = C.c_size_t(0), _linear(**kw)
    for backward in (0, 1):
        assert lib.rr_linear_workspace_bytes(C.byref(c), backward, C.byref(n)) == want
        if want == 0:
            assert n.value % 256 == 0
    if want:
        assert lib.rr_linear(C.byref(c), FAKE, FAKE, None, None, FAKE, None, FAKE, BIG, None) == want
        assert lib.rr_linear_backward(C.byref(c), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG, None) == want


def test_linear_refusals(lib):
    c = _linear()
    n = C.c_size_t(0)
    assert lib.rr_linear_workspace_bytes(None, 0, C.byref(n)) == INVALID
    assert lib.rr_linear_workspace_bytes(C.byref(c), 0, None) == INVALID
    assert lib.rr_linear_workspace_bytes(C.byref(c), 2, C.byref(n)) == INVALID
    good = dict(x=FAKE, w=FAKE, bias=FAKE, residual=FAKE, y=FAKE, pre=FAKE, ws=FAKE, size=BIG)

    def forward(**kw):
        a = dict(good, **kw)
        return lib.rr_linear(C.byref(c), a["x"], a["w"], a["bias"], a["residual"], a["y"], a["pre"], a["ws"], a["size"], None)
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(x=ODD16), dict(w=ODD16), dict(bias=ODD4), dict(residual=ODD16), dict(y=ODD16),
               dict(pre=ODD16)):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=C.c_void_p(0x1010)), dict(size=0)):
        assert forward(**kw) == WORKSPACE, kw
    assert lib.rr_linear(None, FAKE, FAKE, None, None, FAKE, None, FAKE, BIG, None) == INVALID
    good = dict(x=FAKE, w=FAKE, pre=FAKE, dy=FAKE, dx=FAKE, dw=FAKE, dbias=FAKE, ws=FAKE, size=BIG)

    def backward(cfg=c, **kw):
        a = dict(good, **kw)
        return lib.rr_linear_backward(C.byref(cfg), a["x"], a["w"], a["pre"], a["dy"], a["dx"], a["dw"], a["dbias"], a["ws"], a["size"], None)
    for kw in (dict(dy=None), dict(pre=None), dict(dx=None, dw=None, dbias=None), dict(x=None), dict(w=None), dict(x=ODD16), dict(w=ODD16),
               dict(pre=ODD16), dict(dy=ODD16), dict(dx=ODD16), dict(dw=ODD16), dict(dbias=ODD4)):
        assert backward(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=C.c_void_p(0x1010)), dict(size=0)):
        assert backward(**kw) == WORKSPACE, kw


def at(byte):
    return C.c_void_p(0x100000 + byte)


def test_linear_outputs_do_not_overlap(lib):
    """Each pair that may not meet, by as little as 16 bytes (bias: 4); y may be residual, but not a part of it."""
    M, K, N = 16, 64, 32
    c = _linear(M=M, K=K, N=N, act=rr.RR_ACT_SWIGLU)
    x, w, y, z, b = M * K * 2, 2 * N * K * 2, M * N * 2, M * 2 * N * 2, 2 * N * 4
    gap = 1 << 15
    size = dict(x=x, w=w, bias=b, residual=y, y=y, pre=z)
    good = {name: gap * i for i, name in enumerate(size)}

    def forward(**kw):
        a = {name: at(v) for name, v in dict(good, **kw).items()}
        return lib.rr_linear(C.byref(c), a["x"], a["w"], a["bias"], a["residual"], a["y"], a["pre"], at(8 * gap), BIG, None)
    for out in ("y", "pre"):
        for other in size:
            if other == out:
                continue
            last = 4 if other == "bias" else 16
            for place in (good[other] - size[out] + 16, good[other] + (size[other] - last) // 16 * 16):
                assert forward(**{out: place}) == INVALID, (out, other, place)
            if (out, other) != ("y", "residual"):
                assert forward(**{out: good[other]}) == INVALID, (out, other)
    size = dict(x=x, w=w, pre=z, dy=y, dx=x, dw=w, dbias=b)
    good = {name: gap * i for i, name in enumerate(size)}

    def backward(**kw):
        a = {name: at(v) for name, v in dict(good, **kw).items()}
        return lib.rr_linear_backward(C.byref(c), a["x"], a["w"], a["pre"], a["dy"], a["dx"], a["dw"], a["dbias"], at(8 * gap), BIG, None)
    for out in ("dx", "dw", "dbias"):
        for other in size:
            if other != out:
                for place in (good[other] - size[out] + 16, good[other], good[other] + size[other] - 16):
                    assert backward(**{out: place}) == INVALID, (out, other, place)


def test_dropout_and_balance_outputs_do_not_overlap(lib):
    gap = 1 << 15
    for dtype, es in ((rr.RR_F32, 4), (rr.RR_BF16, 2)):
        n = 1000
        for place in (-n * es + 16, -16, 16, n * es - 16):
            assert lib.rr_dropout(n, dtype, at(gap), None, 0.1, 1, 2, None, at(gap + place), None) == INVALID
            assert lib.rr_dropout(n, dtype, at(gap), at(5 * gap), 0.1, 1, 2, None, at(5 * gap + place), None) == INVALID
            assert lib.rr_dropout_backward(n, dtype, at(gap), 0.1, 1, 2, None, at(gap + place), None) == INVALID
    c = rr.RRConfig(T=64, d_model=64, d_ff=0, E=8, k=2, G=2, capacity_factor=1.0).c()
    for place in (-64 * 8 * 4 + 4, 0, 64 * 8 * 4 - 4):
        assert lib.rr_balance_loss_backward(C.byref(c), at(gap), at(5 * gap), None, 0.1, None, 0, at(gap + place), None) == INVALID
        assert lib.rr_balance_loss_backward(C.byref(c), at(gap), at(5 * gap), None, 0.1, None, 2, at(gap + place), None) == INVALID


def test_balance_outputs_do_not_overlap(lib):
    """Each pair that may not meet, by as little as four bytes (the mask: one); counts are read while dlogits is written."""
    T, E, k = 64, 8, 2
    c = rr.RRConfig(T=T, d_model=64, d_ff=0, E=E, k=k, G=2, capacity_factor=1.0).c()
    gap = 1 << 15
    size = dict(logits=4 * T * E, rank=4 * T * (k + 1), mask=T, loss=4, counts=4 * (E + 1), mean=4 * E)
    good = {name: gap * i for i, name in enumerate(size)}

    def forward(**kw):
        a = {name: at(v) for name, v in dict(good, **kw).items()}
        return lib.rr_balance_loss(C.byref(c), a["logits"], a["rank"], a["mask"], 0.1, a["loss"], a["counts"], a["mean"], at(8 * gap), BIG, None)
    for out in ("loss", "counts", "mean"):
        for other in size:
            if other != out:
                for place in (good[other] - size[out] + 4, good[other], good[other] + size[other] - 4):
                    assert forward(**{out: place}) == INVALID, (out, other, place)
    size = dict(logits=4 * T * E, counts=4 * (E + 1), mask=T, dloss=4, dlogits=4 * T * E)
    good = {name: gap * i for i, name in enumerate(size)}

    def backward(flags, **kw):
        a = {name: at(v) for name, v in dict(good, **kw).items()}
        return lib.rr_balance_loss_backward(C.byref(c), a["logits"], a["counts"], a["mask"], 0.1, a["dloss"], flags, a["dlogits"], None)
    for other in ("logits", "counts", "mask", "dloss"):
        for place in (good[other] - size["dlogits"] + 4, good[other], good[other] + size[other] - 4):
            for flags in (0, 2):
                assert backward(flags, dlogits=place) == INVALID, (other, place)


def test_workspaces_lie_apart(lib):
    """What a call needs of its workspace shares no byte with an operand; what lies behind that may."""
    ends = lambda start, size, need: (start - need + 256, start, start + (size - 1) // 256 * 256)
    M, K, N, gap = 16, 64, 32, 1 << 22
    c = _linear(M=M, K=K, N=N, act=rr.RR_ACT_SWIGLU)
    x, w, y, z, b = M * K * 2, 2 * N * K * 2, M * N * 2, M * 2 * N * 2, 2 * N * 4
    need = C.c_size_t(0)
    size = dict(x=x, w=w, bias=b, residual=y, y=y, pre=z)
    good = {name: gap * (i + 1) for i, name in enumerate(size)}
    a = {name: at(v) for name, v in good.items()}
    assert lib.rr_linear_workspace_bytes(C.byref(c), 0, C.byref(need)) == 0 and need.value < gap
    for name in size:
        for place in ends(good[name], size[name], need.value):
            assert lib.rr_linear(C.byref(c), a["x"], a["w"], a["bias"], a["residual"], a["y"], a["pre"], at(place), BIG, None) == INVALID, (name, place)
    size = dict(x=x, w=w, pre=z, dy=y, dx=x, dw=w, dbias=b)
    good = {name: gap * (i + 1) for i, name in enumerate(size)}
    a = {name: at(v) for name, v in good.items()}
    assert lib.rr_linear_workspace_bytes(C.byref(c), 1, C.byref(need)) == 0 and need.value < gap
    for name in size:
        for place in ends(good[name], size[name], need.value):
            assert lib.rr_linear_backward(C.byref(c), a["x"], a["w"], a["pre"], a["dy"], a["dx"], a["dw"], a["dbias"], at(place), BIG, None) == INVALID, (name, place)
    T, E, k = 64, 8, 2
    c = rr.RRConfig(T=T, d_model=64, d_ff=0, E=E, k=k, G=2, capacity_factor=1.0).c()
    size = dict(logits=4 * T * E, rank=4 * T * (k + 1), mask=T, loss=4, counts=4 * (E + 1), mean=4 * E)
    good = {name: gap * (i + 1) for i, name in enumerate(size)}
    a = {name: at(v) for name, v in good.items()}
    assert lib.rr_balance_workspace_bytes(C.byref(c), C.byref(need)) == 0 and need.value < gap
    for name in size:
        for place in ends(good[name], size[name], need.value):
            assert lib.rr_balance_loss(C.byref(c), a["logits"], a["rank"], a["mask"], 0.1, a["loss"], a["counts"], a["mean"], at(place), BIG, None) == INVALID, (name, place)


def test_dropout_counter_outside_the_result(lib):
    """device_offset is read by every workgroup, some after others have written."""
    gap, n = 1 << 15, 1000
    for place in (0, 8, 2 * n - 8):
        assert lib.rr_dropout(n, rr.RR_BF16, at(0), None, 0.1, 1, 2, at(gap + place), at(gap), None) == INVALID
        assert lib.rr_dropout(n, rr.RR_BF16, at(0), at(gap), 0.1, 1, 2, at(gap + place), at(gap), None) == INVALID
        assert lib.rr_dropout_backward(n, rr.RR_BF16, at(gap), 0.1, 1, 2, at(gap + place), at(gap), None) == INVALID


def test_dropout_refusals(lib):
    def call(n=64, dtype=rr.RR_BF16, x=FAKE, residual=None, p=0.1, dev=None, out=FAKE):
        a = lib.rr_dropout(n, dtype, x, residual, p, 1, 2, dev, out, None)
        if residual is None:
            assert lib.rr_dropout_backward(n, dtype, x, p, 1, 2, dev, out, None) == a
        return a
    for kw in (dict(n=0), dict(n=-1), dict(x=None), dict(out=None), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(x=ODD16), dict(out=ODD16),
               dict(residual=ODD16), dict(dev=C.c_void_p(0x1004))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(dtype=2), dict(n=(1 << 40) + 1)):
        assert call(**kw) == UNSUPPORTED, kw


def test_balance_refusals(lib):
    cfg = lambda **kw: rr.RRConfig(**dict(dict(T=64, d_model=64, d_ff=0, E=8, k=2, G=2, capacity_factor=1.0), **kw)).c()
    c, n = cfg(), C.c_size_t(0)
    assert lib.rr_balance_workspace_bytes(C.byref(c), C.byref(n)) == 0 and n.value % 256 == 0
    assert lib.rr_balance_workspace_bytes(C.byref(c), None) == INVALID and lib.rr_balance_workspace_bytes(None, C.byref(n)) == INVALID
    good = dict(c=c, logits=FAKE, rank=FAKE, mask=None, coef=0.1, loss=FAKE, counts=FAKE, mean=FAKE, ws=FAKE, size=BIG)

    def forward(**kw):
        a = dict(good, **kw)
        return lib.rr_balance_loss(C.byref(a["c"]), a["logits"], a["rank"], a["mask"], a["coef"], a["loss"], a["counts"], a["mean"], a["ws"],
                                   a["size"], None)
    for kw in (dict(logits=None), dict(rank=None), dict(loss=None), dict(counts=None), dict(coef=float("nan")), dict(coef=float("inf")),
               dict(logits=ODD4), dict(rank=ODD4), dict(loss=ODD4), dict(counts=ODD4), dict(mean=ODD4), dict(c=cfg(T=0)), dict(c=cfg(k=9))):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=C.c_void_p(0x1010)), dict(size=0)):
        assert forward(**kw) == WORKSPACE, kw
    assert forward(c=cfg(E=128)) == UNSUPPORTED
    other = C.c_void_p(0x2000)

    def backward(c=c, logits=FAKE, counts=FAKE, coef=0.1, dloss=None, flags=0, dlogits=other):
        return lib.rr_balance_loss_backward(C.byref(c), logits, counts, None, coef, dloss, flags, dlogits, None)
    for kw in (dict(logits=None), dict(counts=None), dict(dlogits=None), dict(dlogits=FAKE), dict(coef=float("nan")), dict(flags=1), dict(flags=4),
               dict(logits=ODD4), dict(counts=ODD4), dict(dloss=ODD4), dict(dlogits=ODD4), dict(c=cfg(T=0))):
        assert backward(**kw) == INVALID, kw


# ------------------------------------------------------------------ refusals of the binding

def test_binding_refuses_tensors_off_the_gpu():
    f = lambda *s: torch.zeros(s)
    cfg = rr.RRLinearConfig(4, 8, 8, rr.RR_F32)
    with pytest.raises(rr.RRError, match="not on the current GPU"):
        rr.rr_linear(cfg, f(4, 8), f(8, 8), None, None, f(4, 8), None, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(rr.RRError, match="not on the current GPU"):
        rr.rr_linear_backward(cfg, f(4, 8), f(8, 8), None, f(4, 8), f(4, 8), None, None, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(rr.RRError, match="not on the current GPU"):
        rr.rr_dropout(f(8), 0.1, 1, 2, f(8))
    with pytest.raises(rr.RRError, match="unsupported type"):
        rr.rr_dropout_backward(f(8).half(), 0.1, 1, 2, f(8).half())
    cfg = rr.RRConfig(4, 8, 0, 4, 2, 1, 1.0)
    with pytest.raises(rr.RRError, match="not on the current GPU"):
        rr.rr_balance_loss(cfg, f(4, 4), torch.zeros((4, 3), dtype=torch.int32), 0.1, f(1), torch.zeros(5, dtype=torch.int32),
                           torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(rr.RRError, match="not on the current GPU"):
        rr.rr_balance_loss_backward(cfg, f(4, 4), torch.zeros(5, dtype=torch.int32), 0.1, f(4, 4))
    with pytest.raises(rr.RRError, match="unsupported dtype"):
        rr.rr_linear(rr.RRLinearConfig(4, 8, 8, 7), f(4, 8), f(8, 8), None, None, f(4, 8), None, None)


@pytest.mark.parametrize("kw", [dict(M=(1 << 32) + 16), dict(K=(1 << 32) + 64), dict(N=(1 << 32) + 64), dict(act=(1 << 32) + rr.RR_ACT_SWIGLU),
                                dict(M=16 - (1 << 32)), dict(dtype=1 << 32)])
def test_linear_configuration_does_not_wrap(kw):
    """Sizes and types that 32 bits do not hold are no others."""
    cfg = rr.RRLinearConfig(**dict(dict(M=16, K=64, N=64), **kw))
    with pytest.raises(rr.RRError, match="32 bits"):
        rr.rr_linear_workspace_bytes(cfg)


@pytest.mark.parametrize("kw", [dict(T=(1 << 32) + 4), dict(k=(1 << 32) + 2), dict(E=(1 << 32) + 8), dict(T=4 - (1 << 32))])
def test_balance_configuration_does_not_wrap(kw):
    cfg = rr.RRConfig(**dict(dict(T=4, d_model=8, d_ff=0, E=4, k=2, G=1, capacity_factor=1.0), **kw))
    with pytest.raises(rr.RRError, match="32 bits"):
        rr.rr_balance_workspace_bytes(cfg)


@pytest.mark.parametrize("seed", [2 ** 64, 2 ** 64 + 5, -2 ** 63 - 1])
def test_dropout_seed_does_not_wrap(seed):
    """A seed that 64 bits do not hold is no other, whose mask it would share."""
    x = torch.zeros(8)
    with pytest.raises(rr.RRError, match="64 bits"):
        rr.rr_dropout(x, 0.1, seed, 0, x)
    with pytest.raises(rr.RRError, match="64 bits"):
        rr.rr_dropout_backward(x, 0.1, seed, 0, x)
    for fits in (2 ** 64 - 1, -2 ** 63):  # (then it is the tensor's place that is refused)
        with pytest.raises(rr.RRError, match="not on the current GPU"):
            rr.rr_dropout(x, 0.1, fits, 0, x)
    with pytest.raises(rr.RRError, match="not on the current GPU"):  # counters run on through 2^64, and so may the offset that a program advances
        rr.rr_dropout(x, 0.1, 0, 2 ** 64 + 8, x)


def test_struct_layout_matches_header():
    assert C.sizeof(binding._LinearConfig) == 20
    assert rr.RRLinearConfig(1, 8, 16, act=rr.RR_ACT_SWIGLU).rows == 32 and rr.RRLinearConfig(1, 8, 16).rows == 16


# ------------------------------------------------------------------ plans and workspaces

def test_linear_workspace_fits_every_smaller_batch(lib):
    rng = np.random.default_rng(5)
    for _ in range(200):
        K, N = 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        dtype, act = int(rng.integers(0, 2)), int(rng.integers(0, 3))
        sizes = sorted(int(2 ** v) for v in rng.uniform(0, 17, 12))
        for backward in (False, True):
            need = [rr.rr_linear_workspace_bytes(rr.RRLinearConfig(M, K, N, dtype, act), backward) for M in sizes]
            assert need == sorted(need), (K, N, dtype, act, list(zip(sizes, need)))


def _plan_keys(M, K, N):
    from tests import gpu_util as gu
    for dtype in (rr.RR_F32, rr.RR_BF16):
        for act in (rr.RR_ACT_NONE, rr.RR_ACT_SWIGLU):
            for role, (bm, brows, slices, parts) in enumerate(gu.linear_plans(rr.RRLinearConfig(M, K, N, dtype, act))):
                if role == 0 or act == rr.RR_ACT_NONE:
                    yield dtype, role, bm, brows, parts, slices > 1, role == 0 and 0 < bm and M <= bm  # (one tile of rows: weights read once)


def test_the_gpu_tests_reach_every_tile(lib):
    """Whatever tiles the plan gives products of up to 8e9 multiplications, the shapes of the GPU tests get too."""
    from tests import test_gpu_operators as t
    reached = {k for s in t.SHAPES + t.MORE + [l[:3] for l in t.LARGE] for k in _plan_keys(*s)}
    rng = np.random.default_rng(6)
    for _ in range(4000):
        M, K, N = int(2 ** rng.uniform(2.3, 14.6)), 8 * int(2 ** rng.uniform(0, 10.4)), 8 * int(2 ** rng.uniform(0, 10.4))
        if M * K * N <= 8e9 and M * max(K, N) <= 6e7:
            assert set(_plan_keys(M, K, N)) <= reached, (M, K, N, set(_plan_keys(M, K, N)) - reached)


def _kernel_keys(M, K, N, dtype, act, roles=(0, 1, 2)):
    """One key per kernel that the products of a call are made by: the activation is a part of the forward one's."""
    from tests import gpu_util as gu
    cfg = rr.RRLinearConfig(M, K, N, dtype, act)
    for role, (bm, brows, slices, parts) in enumerate(gu.linear_plans(cfg)):
        if role not in roles:
            continue
        few = 0
        if bm == 0:  # one kernel per number of rows up to the dot products' most, then one up to 16 and one up to 32
            rows = cfg.rows if role == 2 else M
            few = rows if rows <= (2 if dtype == rr.RR_BF16 else 4) else 16 if rows <= 16 else 32
        once = role == 0 and dtype == rr.RR_BF16 and 0 < M <= bm and (bm, brows) != (256, 256)  # (weights read once)
        yield dtype, act if role == 0 else None, role, bm, brows, parts, slices > 1, once, few


def test_the_gpu_tests_run_every_kernel(lib):
    """Whatever kernels the plan gives products of up to 6e10 multiplications, one of the GPU tests runs them and compares: counted from what each
    of those tests calls, with its types and activations."""
    from tests import test_gpu_operators as t, test_gpu_operators_tiles as tiles
    none, gelu, swiglu = rr.RR_ACT_NONE, rr.RR_ACT_GELU, rr.RR_ACT_SWIGLU
    both = (rr.RR_F32, rr.RR_BF16)
    runs = [(s, d, none, (0, 1, 2)) for s in t.SHAPES + t.MORE for d in both]  # test_linear_exact_sums
    runs += [(s, d, swiglu, (0,)) for s in t.MORE for d in both]  # test_linear_gated_tiles
    runs += [(s, d, a, (0, 1, 2)) for s in t.SHAPES for d in both for a in (gelu, swiglu)]  # test_linear_values_and_gradients
    runs += [(l[:3], rr.RR_BF16, none, (0, 1, 2) if l[3] == "none" else (1, 2)) for l in t.LARGE]  # test_linear_large_tiles
    runs += [(f[2:5], rr.RR_F32 if f[0] == "f32" else rr.RR_BF16, t.ACT[f[1]], (0,)) for f in tiles.FORWARD]
    runs += [(g[1:4], rr.RR_F32 if g[0] == "f32" else rr.RR_BF16, none, (tiles.ROLE[g[4]],)) for g in tiles.GRADIENTS]
    reached = {k for s, d, a, roles in runs for k in _kernel_keys(*s, d, a, roles)}
    rng = np.random.default_rng(8)
    for _ in range(6000):
        M, K, N = int(2 ** rng.uniform(0, 16)), 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        if M * K * N <= 6e10 and M * max(K, N) <= 1e8:
            for d in both:
                for a in (none, gelu, swiglu):
                    keys = set(_kernel_keys(M, K, N, d, a))
                    assert keys <= reached, (M, K, N, keys - reached)


def test_the_gpu_tests_tiles_are_the_plan_s(lib):
    """Each case of test_gpu_operators_tiles.py is about the kernel that it names."""
    from tests import test_gpu_operators_tiles as tiles
    for dtype, act, M, K, N, *plan in tiles.FORWARD:
        tiles.assert_plan(tiles.config(dtype, act, M, K, N), 0, *plan)
    for dtype, M, K, N, name, *plan in tiles.GRADIENTS:
        tiles.assert_plan(tiles.config(dtype, "none", M, K, N), tiles.ROLE[name], *plan)


@pytest.mark.parametrize("cut", range(1, 9))
def test_parts_of_a_cut_tile_share_no_row(lib, cut):
    """The last round of 256 x 256 tiles is cut by rows into up to eight parts: together they are the tile, no row twice (y may lie in the
    residual's place) and none of the next tile's."""
    for m0 in (0, 256, 3840):
        for rows in range(1, 257):
            got = []
            for part in range(cut):
                r = (C.c_int32 * 2)()
                assert lib.rr_linear_cut(m0, rows, cut, part, r) == 0
                got += range(r[0], r[1])
            assert got == list(range(m0, m0 + rows)), (m0, rows, cut)


def test_linear_slices_fit_the_workspace(lib):
    """The slices' sums, rows x columns x slices floats, fit what the workspace keeps for them, and no slice is empty."""
    from tests import gpu_util as gu
    rng = np.random.default_rng(7)
    for _ in range(3000):
        M, K, N = int(2 ** rng.uniform(0, 17)), 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        dtype, act = int(rng.integers(0, 2)), int(rng.choice([rr.RR_ACT_NONE, rr.RR_ACT_SWIGLU]))
        cfg = rr.RRLinearConfig(M, K, N, dtype, act)
        R, chunk = cfg.rows, 64 if dtype == rr.RR_BF16 else 32
        forward, backward = rr.rr_linear_workspace_bytes(cfg), rr.rr_linear_workspace_bytes(cfg, True)
        sums = [(M * R, K), (M * K, R), (R * K, M)]
        for role, (_, _, slices, parts) in enumerate(gu.linear_plans(cfg)):
            outputs, length = sums[role]
            if role == 2 and dtype == rr.RR_F32 and not parts:
                length = (M + 63) // 64 * 64  # of the transposes' rows
            if slices > 1:
                assert outputs * 4 * slices <= (backward if role else forward), (cfg, role, slices)
                each = (length // slices + chunk - 1) // chunk * chunk
                assert each * slices >= length > each * (slices - 1), (cfg, role, slices)
