"""The layer operators in 64 bits on the host, and how far a kernel may be from them.

Error bounds. u is half a step of the operator's type (bf16 2^-8, fp16 2^-11, fp32
2^-24) and e = 2^-24 that of the fp32 the kernels compute in:
- a sum of n products: each of its n roundings is at most e times a partial sum, which
  is at most S = sum |a b|; as a random walk, 4 e sqrt(n + 32) S holds with a margin of
  more than four standard deviations for every element (fp32 products formed from bf16
  parts add 2 e |a b| each: inside the 32).
- the activations and their derivatives: a few fp32 roundings, and functions good to a
  few e of their value; cancellation in 1 + erf and in s + z s (1 - s) is at most of
  terms of size 1 + |z|: 16 e (1 + |z|) covers both, times what they are multiplied with.
  Their slopes are at most 1.13, so an error of z passes on at most 1.13 times.
- the result is rounded once: u |y|, or half the smallest subnormal (fp16 2^-25).
- g is rounded to the type before its two products: each product of the sum is off by
  at most u |g w|, independent: 4 u sqrt(sum (g w)^2).
"""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
E = 2.0 ** -24
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def philox(counter, key):
    """Philox4x32-10: counter [..., 4] and key [2] of uint32 values -> [..., 4] uint32."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    lo, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k[0]), b & lo, (a >> sh) ^ c[3] ^ np.uint64(k[1]), a & lo]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1).astype(np.uint32)


def threshold(p):
    return int(math.floor(float(np.float32(p)) * 65536 + 0.5))


def keep_mask(seed, offset, rows, cols, p):
    """[rows, cols] bool, element by element from the definition."""
    m = (1 << 64) - 1
    seed, offset = int(seed) & m, int(offset) & m
    nb = -(-cols // 8)
    with np.errstate(over="ignore"):
        at = np.uint64(offset) + np.arange(rows * nb, dtype=np.uint64)
    ctr = np.zeros((rows * nb, 4), np.uint32)
    ctr[:, 0] = at & np.uint64(0xFFFFFFFF)
    ctr[:, 1] = at >> np.uint64(32)
    w = philox(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(rows, nb * 8)[:, :cols]
    return u >= threshold(p)


def drop_scale(p):
    t = threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def factor(rng, rows, cols, p):
    """keep / q, float64 [rows, cols]; rng: (seed, offset)"""
    if threshold(p) == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    return torch.from_numpy(keep_mask(rng[0], rng[1], rows, cols, p)).double() * drop_scale(p)


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _d(t):
    return None if t is None else t.detach().cpu().double()


def forward(X, W, b, r, name, p, rng, dtype):
    """(y, z, bound of y, bound of z) of a forward call on tensors of the type."""
    X, W, b, r = _d(X), _d(W), _d(b), _d(r)
    z, S = X @ W, X.abs() @ W.abs()
    if b is not None:
        z, S = z + b, S + b.abs()
    a = act(z, name)
    f = factor(rng, z.shape[0], z.shape[1], p)
    y = f * a
    ez = 4 * E * math.sqrt(W.shape[0] + 32) * S
    ea = 1.13 * ez + (0 if name in ("none", "relu") else 16 * E * (1 + z.abs()) * z.abs().clamp(min=1))
    by = f * ea + 4 * E * y.abs()
    if r is not None:
        y = y + r
        by = by + 2 * E * (y.abs() + r.abs())
    return y, z, by + U[dtype] * (y.abs() + by) + TINY[dtype], ez + U[dtype] * (z.abs() + ez) + TINY[dtype]


def backward(X, W, Z, dY, name, p, rng, dtype):
    """{"dx", "dw", "db", "g"} and their bounds, for tensors of the type; Z may be None."""
    X, W, Z, dY = _d(X), _d(W), _d(Z), _d(dY)
    f = factor(rng, dY.shape[0], dY.shape[1], p)
    v = dY * f
    g, eg = v, 4 * E * v.abs()
    if name != "none":
        g = v * act_grad(Z, name)
        eg = v.abs() * 16 * E * (1 + Z.abs()) * Z.abs().clamp(min=1)
    u, tiny = U[dtype], TINY[dtype]
    ref, bound = {"g": g}, {}

    def prod(a, b, ea, n, ga):   # ga: whether the rounded g is a (else b)
        y, S = a @ b, a.abs() @ b.abs()
        e = 4 * E * math.sqrt(n + 32) * S + 4 * u * torch.sqrt((a * a) @ (b * b))
        e = e + (ea @ b.abs() + tiny * b.abs().sum(0) if ga else a.abs() @ ea + tiny * a.abs().sum(1, keepdim=True))
        return y, e + u * (y.abs() + e) + tiny

    ref["dx"], bound["dx"] = prod(g, W.t(), eg, W.shape[1], True)
    ref["dw"], bound["dw"] = prod(X.t(), g, eg, X.shape[0], False)
    ref["db"] = g.sum(0)
    e = 4 * E * math.sqrt(g.shape[0] + 32) * g.abs().sum(0) + eg.sum(0)
    bound["db"] = e + u * (ref["db"].abs() + e) + tiny
    return ref, bound


def check(what, got, ref, bound):
    """Every element within its bound; prints the worst one's share of its bound."""
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if got.numel() == 0:
        return
    off = (got - ref).abs()
    share = float((off / bound).max())
    norm = float(ref.norm())
    print("%-8s worst share of its bound %.3f, normwise %.2e" % (what, share, float(off.norm()) / norm if norm else 0.0),
          flush=True)
    assert bool((off <= bound).all()), (what, share)
