"""Plain 64-bit implementations of the operators around the MoE layer, written from their formulas, for the tests.

numpy for the random numbers, torch in float64 for the rest (on whatever device the inputs are)."""
import math

import numpy as np
import torch


def random_halves(seed: int, offset: int, n: int) -> np.ndarray:
    """The first n 16-bit numbers of Philox4x32-10 at counters offset, offset + 1, ...: uint16 [n]."""
    words = philox4x32(np.uint64(offset % 2 ** 64) + np.arange((n + 7) // 8, dtype=np.uint64), seed)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=2)  # [groups, 4, 2]
    return halves.reshape(-1)[:n].astype(np.uint16)


def philox4x32(counter, seed: int, high=0) -> np.ndarray:
    """Philox4x32 with ten rounds (Salmon et al., SC 2011): 64-bit counters (low words), one high half -> [n, 4] words."""
    c = np.asarray(counter, dtype=np.uint64)
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = [c & low, c >> sh, np.full_like(c, high & 0xFFFFFFFF), np.full_like(c, high >> 32)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> sh) ^ x[1] ^ np.uint64(k[0]), b & low, (a >> sh) ^ x[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(x, axis=1)


def dropout(x, residual, p, seed, offset):
    """float64 out, the mask, the scale"""
    m = math.floor(65536.0 * float(np.float32(p)) + 0.5)
    keep = torch.from_numpy(random_halves(seed, offset, x.numel()).astype(np.int64) >= m).to(x.device).reshape(x.shape)
    scale = 65536.0 / (65536 - m) if m < 65536 else 0.0
    out = torch.where(keep, x.double() * scale, torch.zeros((), dtype=torch.float64, device=x.device))
    return (out if residual is None else out + residual.double()), keep, scale


def balance(logits, rank_expert, k, coef, mask=None, dloss=1.0):
    a = logits.double()
    T, E = a.shape
    live = torch.ones(T, dtype=torch.bool, device=a.device) if mask is None else mask.bool()
    n = int(live.sum())
    top = a.max(dim=1, keepdim=True).values
    z = torch.exp(a - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = z.sum(dim=1, keepdim=True)
    p = torch.where(live[:, None] & (total != 0), z / total, torch.zeros_like(z))
    chosen = rank_expert[:, :k][live].reshape(-1).long()
    chosen = chosen[(chosen >= 0) & (chosen < E)]
    counts = torch.bincount(chosen, minlength=E)
    f = counts.double() / (k * n) if n else torch.zeros(E, dtype=torch.float64, device=a.device)
    mean = p.sum(dim=0) / n if n else torch.zeros_like(f)
    grad = dloss * coef * E / max(n, 1) * p * (f - (p * f).sum(dim=1, keepdim=True))
    return {"loss": coef * E * (f * mean).sum(), "counts": torch.cat([counts, counts.new_tensor([n])]), "mean_prob": mean,
            "dlogits": grad, "p": p, "f": f}


def act(z, name):
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        return g * torch.sigmoid(g) * u
    return z


def act_gradient(dy, z, name):
    if name == "gelu":
        return dy * (0.5 * (1.0 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-z * z / 2) / math.sqrt(2.0 * math.pi))
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        s = torch.sigmoid(g)
        return torch.cat([dy * u * (s + g * s * (1 - s)), dy * g * s], dim=1)
    return dy


def linear(x, w, bias, residual, name):
    """float64 y and z"""
    z = torch.mm(x.double(), w.double().t())
    if bias is not None:
        z = z + bias.double()
    y = act(z, name)
    return (y if residual is None else y + residual.double()), z


def linear_backward(x, w, pre, dy, name):
    dz = act_gradient(dy.double(), None if pre is None else pre.double(), name)
    return {"dz": dz, "dx": torch.mm(dz, w.double()), "dw": torch.mm(dz.t().contiguous(), x.double()), "dbias": dz.sum(dim=0)}
