"""The operators around the MoE layer, as calls with their sizes: what a training or serving program runs beside `rr_moe_forward`.

Kinds of cases:

  linear           y = residual + act(x W^T + bias), one call; with "pre" the pre-activations too, for the backward pass
  linear_backward  gradients of x, W and bias from dy and the stored pre-activations
  dropout          out = residual + dropout(x), the mask a function of (seed, offset, element)
  dropout_backward dx from dout, the mask made again
  balance          loss, per-expert counts and mean probabilities, then the gradient of the router scores

`run` computes them in elementary torch operations, or with `own` set through the entry points of the package.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_ACT_COLUMNS = {"none": 1, "gelu": 1, "swiglu": 2}  # rows of W per output column


def _linear(kind, M, K, N, dtype, act, bias, residual=False, pre=False, name=None):
    c = dict(kind=kind, M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual, pre=pre)
    return c if name is None else dict(c, name=name)


def _dropout(kind, n, dtype, p, residual=False, name=None):
    c = dict(kind=kind, n=n, dtype=dtype, p=p, residual=residual)
    return c if name is None else dict(c, name=name)


def _balance(T, E, k, masked, name=None):
    c = dict(kind="balance", T=T, E=E, k=k, masked=masked)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one token through a square projection with its residual: serving, the weights are read for a single row
        _linear("linear", 1, 4096, 4096, "bf16", "none", False, residual=True, name="linear 1 token"),
        # one decoding step of 16 sequences through the up projection of a dense FFN
        _linear("linear", 16, 4096, 11008, "bf16", "swiglu", False, name="linear decode 16"),
        # a short odd prompt through a GELU layer with bias whose row lengths are no multiple of 64
        _linear("linear", 301, 1000, 2728, "bf16", "gelu", True, name="linear ragged gelu"),
        # the up projection of a training micro-batch: pre-activations kept for the backward pass
        _linear("linear", 8192, 2048, 5632, "bf16", "swiglu", False, pre=True, name="linear up 8k"),
        # the down projection of a large micro-batch, joined to the residual stream
        _linear("linear", 16384, 11008, 4096, "bf16", "none", False, residual=True, name="linear down 16k"),
        # gradients of the up projection
        _linear("linear_backward", 8192, 2048, 5632, "bf16", "swiglu", False, name="linear backward 8k"),
        # gradients of a layer kept in fp32 throughout, odd number of rows
        _linear("linear_backward", 2001, 1024, 2816, "f32", "gelu", True, name="linear backward f32"),
        # a tiny fp32 batch: a call that is all launch
        _dropout("dropout", 256 * 64, "f32", 0.1, residual=True, name="dropout tiny"),
        # the residual connection of a training micro-batch
        _dropout("dropout", 16384 * 4096, "bf16", 0.1, residual=True, name="dropout add 16k"),
        # its gradient at the heaviest batch of the benchmark
        _dropout("dropout_backward", 32768 * 4096, "bf16", 0.1, name="dropout backward 32k"),
        # a small batch whose last sequences are padded
        _balance(1001, 16, 2, 0.25, name="balance 1k padded"),
        # routing at a million tokens
        _balance(1 << 20, 64, 2, 0.0, name="balance 1m"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _wide(rng, lo, hi):  # a row length: a multiple of 8, of 64 most often
    step = rng.choice((8, 64, 64, 64))
    return max(1, round(_log(rng, lo, hi) / step)) * step


def draw(rng):
    while True:
        kind = rng.choice(("linear",) * 4 + ("linear_backward",) * 3 + ("dropout", "dropout_backward", "balance", "balance"))
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        if kind == "balance":
            E = rng.randint(2, 64)
            c = _balance(_log(rng, 1, 1 << 20), E, rng.randint(1, min(4, E)), rng.choice((0.0, 0.0, 0.1, 0.5)))
        elif kind.startswith("dropout"):
            c = _dropout(kind, _log(rng, 1, 32768 * 4096), dtype, rng.choice((0.05, 0.1, 0.1, 0.2, 0.5)),
                         kind == "dropout" and rng.random() < 0.7)
        else:
            act = rng.choice(("none", "gelu", "swiglu"))
            backward = kind == "linear_backward"
            c = _linear(kind, _log(rng, 1, 32768), _wide(rng, 64, 11008), _wide(rng, 64, 11008), dtype, act, rng.random() < 0.5,
                        not backward and rng.random() < 0.5, not backward and act != "none" and rng.random() < 0.5)
        w = work(c)
        if w["bytes"] <= 0.6e9 and w["flops"] <= (1.4e12 if dtype == "bf16" else 6e10):
            return c


def _tdt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    s = {"case": case}
    if case["kind"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = normal(T, E) + normal(E, scale=0.5)
        s["rank_expert"] = torch.full((T, k + 1), -1, dtype=torch.int32, device="cuda")
        order = torch.sort(s["logits"], dim=1, descending=True, stable=True).indices[:, :k + 1]
        s["rank_expert"][:, :order.shape[1]] = order.to(torch.int32)
        s["token_mask"] = None
        if case["masked"]:  # the last tokens of the batch are padding
            s["token_mask"] = (torch.arange(T, device="cuda") < T - int(case["masked"] * T)).to(torch.uint8)
        s["dloss"] = torch.full((1,), 0.5 + 0.25 * (seed % 5), device="cuda")
    elif case["kind"].startswith("dropout"):
        s["x"] = normal(case["n"], dtype=_tdt(case))
        s["residual"] = normal(case["n"], dtype=_tdt(case)) if case["residual"] else None
        s["seed"], s["offset"] = (seed * 0x9E3779B1 + 12345) & ((1 << 63) - 1), (seed * 1000003) & ((1 << 40) - 1)
    else:
        M, K, N, dt = case["M"], case["K"], case["N"], _tdt(case)
        rows = N * _ACT_COLUMNS[case["act"]]
        s["x"] = normal(M, K, dtype=dt)
        s["w"] = normal(rows, K, scale=0.02, dtype=dt)
        if case["kind"] == "linear":
            s["bias"] = normal(rows, scale=0.1) if case["bias"] else None
            s["residual"] = normal(M, N, dtype=dt) if case["residual"] else None
        else:
            s["pre"] = normal(M, rows, dtype=dt) if case["act"] != "none" else None
            s["dy"] = normal(M, N, dtype=dt)
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    """Output buffers and workspaces, which a program keeps from call to call."""
    import paper_2402_12399_amd as rr
    if case["kind"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        s["cfg"] = rr.RRConfig(T, 64, 0, E, k, 1, 1.0, rr.RR_F32, rr.RR_ACT_SWIGLU, rr.RR_INTRA_GPU)
        s["workspace"] = rr.alloc_balance_workspace(s["cfg"])
        s["loss"] = torch.empty(1, device="cuda")
        s["counts"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
        s["mean_prob"] = torch.empty(E, device="cuda")
        s["dlogits"] = torch.empty_like(s["logits"])
    elif case["kind"].startswith("dropout"):
        s["out"] = torch.empty_like(s["x"])
    else:
        M, K, N, dt = case["M"], case["K"], case["N"], _tdt(case)
        rows = N * _ACT_COLUMNS[case["act"]]
        act = {"none": rr.RR_ACT_NONE, "gelu": rr.RR_ACT_GELU, "swiglu": rr.RR_ACT_SWIGLU}[case["act"]]
        s["cfg"] = rr.RRLinearConfig(M, K, N, rr.RR_F32 if dt == torch.float32 else rr.RR_BF16, act)
        backward = case["kind"] == "linear_backward"
        s["workspace"] = rr.alloc_linear_workspace(s["cfg"], backward)
        if backward:
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["dbias"] = torch.empty(rows, device="cuda") if case["bias"] else None
        else:
            s["y"] = torch.empty((M, N), dtype=dt, device="cuda")
            s["pre"] = torch.empty((M, rows), dtype=dt, device="cuda") if case["pre"] else None


def _run_own(s):
    import paper_2402_12399_amd as rr
    kind = s["case"]["kind"]
    if kind == "balance":
        rr.rr_balance_loss(s["cfg"], s["logits"], s["rank_expert"], 0.01, s["loss"], s["counts"], s["workspace"],
                           mean_prob=s["mean_prob"], token_mask=s["token_mask"])
        rr.rr_balance_loss_backward(s["cfg"], s["logits"], s["counts"], 0.01, s["dlogits"], dloss=s["dloss"],
                                    token_mask=s["token_mask"])
        return {n: s[n] for n in ("loss", "counts", "mean_prob", "dlogits")}
    if kind == "dropout":
        rr.rr_dropout(s["x"], s["case"]["p"], s["seed"], s["offset"], s["out"], residual=s["residual"])
        return s["out"]
    if kind == "dropout_backward":
        rr.rr_dropout_backward(s["x"], s["case"]["p"], s["seed"], s["offset"], s["out"])
        return s["out"]
    if kind == "linear":
        rr.rr_linear(s["cfg"], s["x"], s["w"], s["bias"], s["residual"], s["y"], s["pre"], s["workspace"])
        return {n: s[n] for n in ("y", "pre") if s[n] is not None}
    rr.rr_linear_backward(s["cfg"], s["x"], s["w"], s["pre"], s["dy"], s["dx"], s["dw"], s["dbias"], s["workspace"])
    return {n: s[n] for n in ("dx", "dw", "dbias") if s[n] is not None}


def _philox(counter, seed):
    """Philox4x32 with ten rounds (Salmon et al., SC 2011) on int64 tensors: counter words (counter, 0), key = seed."""
    low = 0xFFFFFFFF
    c0, c1 = counter & low, (counter >> 32) & low
    c2, c3 = torch.zeros_like(c0), torch.zeros_like(c0)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _keep(n, p, seed, offset):
    groups = torch.arange((n + 7) // 8, device="cuda") + offset
    halves = [h for word in _philox(groups, seed) for h in (word & 0xFFFF, word >> 16)]
    threshold = int(math.floor(p * 65536 + 0.5))
    return torch.stack(halves, dim=1).reshape(-1)[:n] >= threshold, 65536.0 / (65536 - threshold)


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "swiglu":
        g, u = z.chunk(2, dim=1)
        return g / (1.0 + torch.exp(-g)) * u
    return z


def _act_gradient(dy, z, act):
    if act == "gelu":
        return dy * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi))
    if act == "swiglu":
        g, u = z.chunk(2, dim=1)
        s = 1.0 / (1.0 + torch.exp(-g))
        return torch.cat([dy * u * s * (1.0 + g * (1.0 - s)), dy * g * s], dim=1)
    return dy


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "balance":
        return _plain_balance(s)
    dt = _tdt(case)
    if case["kind"].startswith("dropout"):
        keep, scale = _keep(case["n"], case["p"], s["seed"], s["offset"])
        out = torch.where(keep, s["x"].float() * scale, 0.0)
        return (out if s["residual"] is None else out + s["residual"].float()).to(dt)
    x, w = s["x"].float(), s["w"].float()
    if case["kind"] == "linear":
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt), "pre": z.to(dt)} if case["pre"] else {"y": y.to(dt)}
    dz = _act_gradient(s["dy"].float(), None if s["pre"] is None else s["pre"].float(), case["act"])
    out = {"dx": (dz @ w).to(dt), "dw": (dz.t() @ x).to(dt)}
    if case["bias"]:
        out["dbias"] = dz.sum(dim=0)
    return out


def _plain_balance(s):
    a, E, k = s["logits"], s["case"]["E"], s["case"]["k"]
    live = torch.ones(a.shape[0], dtype=torch.bool, device="cuda") if s["token_mask"] is None else s["token_mask"] != 0
    z = torch.exp(a - a.max(dim=1, keepdim=True).values)
    p = torch.where(live[:, None], z / z.sum(dim=1, keepdim=True), 0.0)
    n = live.sum()
    chosen = torch.where(live[:, None], s["rank_expert"][:, :k], -1)
    counts = torch.stack([(chosen == e).sum() for e in range(E)])
    f = counts.float() / (k * n)
    mean_prob = (p.double().sum(dim=0) / n).float()  # a million addends: 32 bits would lose what the loss is compared by
    loss = 0.01 * E * (f * mean_prob).sum().reshape(1)
    dlogits = s["dloss"] * (0.01 * E / n) * p * (f - (p * f).sum(dim=1, keepdim=True))
    return {"loss": loss, "counts": torch.cat([counts, n.reshape(1)]).to(torch.int32), "mean_prob": mean_prob, "dlogits": dlogits}


def work(case):
    if case["kind"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        mask = T if case["masked"] else 0
        return {"bytes": float(2 * 4 * T * E + 4 * T * (k + 1) + mask + 12 * E), "flops": 16.0 * T * E}
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("dropout"):
        return {"bytes": float(case["n"] * es * (3 if case["residual"] else 2)), "flops": 2.0 * case["n"]}
    M, K, N = case["M"], case["K"], case["N"]
    rows = N * _ACT_COLUMNS[case["act"]]
    if case["kind"] == "linear":
        nb = es * (M * K + rows * K + M * N * (2 if case["residual"] else 1) + (M * rows if case["pre"] else 0))
        return {"bytes": float(nb + (4 * rows if case["bias"] else 0)), "flops": 2.0 * M * K * rows}
    nb = es * (2 * M * K + 2 * rows * K + M * N + (M * rows if case["act"] != "none" else 0))
    return {"bytes": float(nb + (4 * rows if case["bias"] else 0)), "flops": 4.0 * M * K * rows}


def _random_words(first, count, key):
    """The generator's 16-bit numbers of counters first .. first + count - 1, numpy, 64-bit products."""
    m0, m1, mask, shift = np.uint64(0xD2511F53), np.uint64(0xCD9E8D57), np.uint64(0xFFFFFFFF), np.uint64(32)
    index = np.uint64(first) + np.arange(count, dtype=np.uint64)
    x = [index & mask, index >> shift, np.zeros(count, dtype=np.uint64), np.zeros(count, dtype=np.uint64)]
    keys = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        p0, p1 = x[0] * m0, x[2] * m1
        x = [(p1 >> shift) ^ x[1] ^ np.uint64(keys[0]), p1 & mask, (p0 >> shift) ^ x[3] ^ np.uint64(keys[1]), p0 & mask]
        keys = [(keys[0] + 0x9E3779B9) % (1 << 32), (keys[1] + 0xBB67AE85) % (1 << 32)]
    return np.stack(x, axis=1).astype("<u4").view("<u2").reshape(-1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "balance":
        a = s["logits"].double()
        live = torch.ones(case["T"], dtype=torch.float64, device="cuda") if s["token_mask"] is None else s["token_mask"].double()
        n = float(live.sum())
        p = torch.softmax(a, dim=1) * live[:, None]
        hot = torch.zeros_like(a).scatter_(1, s["rank_expert"][:, :case["k"]].long(), 1.0) * live[:, None]
        counts = hot.sum(dim=0)
        f, mean = counts / (n * case["k"]), p.sum(dim=0) / n
        weights = s["dloss"].double() * 0.01 * case["E"] / n * f
        grad = p * weights - p * (p @ weights)[:, None]
        whole = torch.cat([counts, live.sum().reshape(1)]).round().to(torch.int32)
        return {"loss": (0.01 * case["E"] * (f @ mean)).reshape(1), "counts": whole, "mean_prob": mean, "dlogits": grad}
    if case["kind"].startswith("dropout"):
        n, cut = case["n"], int(math.floor(case["p"] * 65536 + 0.5))
        words = _random_words(s["offset"], (n + 7) // 8, s["seed"])[:n]
        kept = torch.from_numpy(words.astype(np.int32) >= cut).cuda()
        out = s["x"].double() * kept * (65536 / (65536 - cut))
        return out if s["residual"] is None else out + s["residual"].double()
    x, w, act = s["x"].double(), s["w"].double(), case["act"]
    N = case["N"]
    if case["kind"] == "linear":
        z = torch.mm(x, w.t())
        if s["bias"] is not None:
            z += s["bias"].double()
        if act == "gelu":
            y = z * torch.special.ndtr(z)
        elif act == "swiglu":
            y = z[:, :N] * torch.sigmoid(z[:, :N]) * z[:, N:]
        else:
            y = z.clone()
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"y": y, "pre": z} if case["pre"] else {"y": y}
    dy = s["dy"].double()
    if act == "none":
        dz = dy
    elif act == "gelu":
        z = s["pre"].double()
        dz = dy * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    else:
        g, u = s["pre"][:, :N].double(), s["pre"][:, N:].double()
        t = torch.sigmoid(g)
        dz = torch.cat([dy * u * (t + g * t * (1 - t)), dy * g * t], dim=1)
    out = {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t().contiguous(), x)}
    if case["bias"]:
        out["dbias"] = dz.sum(dim=0)
    return out
