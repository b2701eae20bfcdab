"""A plain 64-bit implementation of the 8-bit cache and of decode over it, and drawn caches."""
import math

import numpy as np
import torch

DEV = "cuda"
TOP = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100
NEG_INF = float("-inf")


def dtype_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def quantise(x, code):
    """Codes (as float64 numbers) and scales (float32) of blocks [..., T, d] of stored values: scale, inverse and
    product rounded to fp32 as the definition says, the rounding to a code in float64."""
    x = np.asarray(x, np.float32)
    a = np.where(np.isfinite(x), np.abs(x), np.float32(0)).max((-2, -1))
    top = np.float32(TOP[code])
    fine = a >= np.float32(TINY)
    safe = np.where(fine, a, np.float32(1))
    scale = np.where(fine, safe / top, np.float32(0)).astype(np.float32)
    inv = np.where(fine, top / safe, np.float32(0)).astype(np.float32)
    with np.errstate(all="ignore"):
        y = (x * inv[..., None, None]).astype(np.float32).astype(np.float64)
    y = np.clip(np.where(np.isnan(y), 0.0, y), -TOP[code], TOP[code])
    if code == "int8":
        return np.rint(y), scale
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -9))), -6)
    ulp = 2.0 ** (e - 3)
    return np.rint(y / ulp) * ulp, scale


def host(t):
    return t.detach().float().cpu().numpy()


class Model:
    """What a cache of one problem holds, by sequence: the rows themselves, on the host."""

    def __init__(self, B, H, d, block, code):
        self.B, self.H, self.d, self.T, self.code = B, H, d, block, code
        self.k = [np.zeros((H, 0, d), np.float32) for _ in range(B)]
        self.v = [np.zeros((H, 0, d), np.float32) for _ in range(B)]

    def append(self, b, k, v):
        self.k[b] = np.concatenate((self.k[b], host(k)), 1)
        self.v[b] = np.concatenate((self.v[b], host(v)), 1)

    def blocks(self, b):
        n = self.k[b].shape[1] // self.T
        cut = lambda x: x[:, :n * self.T].reshape(self.H, n, self.T, self.d)
        return n, quantise(cut(self.k[b]), self.code), quantise(cut(self.v[b]), self.code)

    def values(self, b):
        """The rows that a decode attends over, float64."""
        n, (k, ks), (v, vs) = self.blocks(b)
        flat = lambda q, s: (q * s.astype(np.float64)[..., None, None]).reshape(self.H, n * self.T, self.d)
        return (np.concatenate((flat(k, ks), self.k[b][:, n * self.T:]), 1),
                np.concatenate((flat(v, vs), self.v[b][:, n * self.T:]), 1))


def held(cache, b, n):
    """(K codes, V codes as rows, scales, tails) of the first n entries, on the host."""
    T = cache.block
    whole = n // T * T
    K = host(cache.K[b, :, :whole])
    V = host(cache.V[b, :, :whole // 16].float().permute(0, 1, 3, 2)).reshape(K.shape)
    return K, V, host(cache.k_scale[b, :, :whole // T]), host(cache.v_scale[b, :, :whole // T]), \
        host(cache.k_tail[b, :, :n - whole]), host(cache.v_tail[b, :, :n - whole])


def assert_holds(cache, m, note=""):
    """The cache holds bit for bit what the definition gives for the model's rows."""
    for b in range(m.B):
        n, (k, ks), (v, vs) = m.blocks(b)
        L = m.k[b].shape[1]
        flat = lambda q: q.reshape(m.H, n * m.T, m.d).astype(np.float32)
        want = (flat(k), flat(v), ks, vs, m.k[b][:, n * m.T:], m.v[b][:, n * m.T:])
        for name, x, y in zip(("K", "V", "k_scale", "v_scale", "k_tail", "v_tail"), held(cache, b, L), want):
            assert np.array_equal(x, y, equal_nan=True), (note, b, name, L)


def fill(cache, seed):
    """Every buffer of a cache set to arbitrary bytes (floats to NaN): what it must not depend on."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    for t in (cache.K, cache.V):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, device=DEV, dtype=torch.uint8))
    for t in (cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail):
        t.fill_(float("nan"))


def rows(g, *shape, dtype):
    """Rows with a few large channels, as keys have them."""
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., :: 13] *= 4.0
    return x.to(dtype_of(dtype))


def attention(q, k, v, bias, G, scale):
    """out [H G, d] in float64 for the rows k, v [H, n, d] of one sequence; bias [H, n] or None; and max |x|."""
    H, n, d = k.shape
    out = np.zeros((H * G, d))
    big = 0.0
    for h in range(H):
        if n == 0:
            continue
        keep = np.ones(n, bool) if bias is None else bias[h] > -np.inf
        if not keep.any():
            continue
        x = q[h * G:(h + 1) * G].astype(np.float64) @ k[h, keep].T * scale
        big = max(big, np.abs(x).max())
        if bias is not None:
            x = x + bias[h, keep].astype(np.float64)
        w = np.exp(x - x.max(-1, keepdims=True))
        out[h * G:(h + 1) * G] = w @ v[h, keep] / w.sum(-1, keepdims=True)
    return out, big


def assert_near(got, want, big, note=""):
    """Relative 2-norm per query head.  Queries, codes and softmax weights enter the products whole and sums are fp32:
    a logit x carries the roundings of a sum of d products, of its scale and of its own 32 bits, a dozen steps of 2^-24
    at x = 1 and growing with |x|, and as a weight's exponent makes them the weight's; the sums over entries, their
    merging and the division add another dozen.  An empty row is exactly 0."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    empty = (want == 0).all(-1)
    assert (got[empty] == 0).all(), note
    if empty.all():
        return
    err = np.linalg.norm(got - want, axis=-1)[~empty] / np.linalg.norm(want, axis=-1)[~empty]
    tol = 2.0 ** -24 * (24 + 2 * big)
    assert err.max() < tol, (note, err.max(), tol)


def scale_of(d):
    return 1.0 / math.sqrt(d)
