"""Plain 64-bit implementations of the paged cache's calls, and drawn caches and trees."""
import numpy as np
import torch

DEV = "cuda"
NEG_INF = float("-inf")


def dtype_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def half_step(name):
    """What one rounding to the type moves a value by at most, relative to it."""
    return torch.finfo(dtype_of(name)).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def rows(g, *shape, dtype):
    """Rows with a few large channels, as keys have them."""
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., ::13] *= 4.0
    return x.to(dtype_of(dtype))


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def make_cache(S, p, lens, n, page, g, dtype, bias=True, spare=2, columns=None, poison=True):
    """A cache whose sequences hold `lens` entries and have room for n more, on pages in no order.  Rows that hold
    nothing are NaN."""
    B, H, d = p.batch, p.n_heads_kv, p.head_dim
    need = [-(-(max(x, 0) + n) // page) for x in lens]
    total = sum(need) + spare
    place = torch.randperm(total, generator=torch.Generator().manual_seed(1 + total)).tolist()
    columns = columns or max(need) + 1
    table = torch.full((B, columns), -1, dtype=torch.int32)
    for b in range(B):
        for j in range(min(need[b], columns)):
            table[b, j] = place.pop()
    nan = float("nan")
    c = S.PagedCache.over(p, torch.full((total, H, page, d), nan, device=DEV).to(dtype_of(dtype)),
                          torch.full((total, H, page, d), nan, device=DEV).to(dtype_of(dtype)), table.to(DEV),
                          torch.full((total, H, page), nan, device=DEV) if bias else None)
    for b in range(B):
        if lens[b] > 0:
            put(c, b, 0, rows(g, lens[b], H, d, dtype=dtype), rows(g, lens[b], H, d, dtype=dtype),
                None if not bias else torch.where(torch.rand((lens[b], H), generator=g, device=DEV) < 0.2,
                                                  torch.rand((lens[b], H), generator=g, device=DEV), 0.0))
    return c


def places(c, b, first, count):
    e = torch.arange(first, first + count, device=DEV)
    return c.table[b].long()[e // c.page], e % c.page


def put(c, b, first, k, v, bias=None):
    """Rows [m, H, d] (and biases [m, H]) as entries first .. of sequence b, by indexing."""
    pg, row = places(c, b, first, k.shape[0])
    c.K[pg, :, row], c.V[pg, :, row] = k, v
    if c.bias is not None:
        c.bias[pg, :, row] = 0.0 if bias is None else bias


def entries(c, b, first, count):
    """(K [count, H, d], V, bias [count, H]) on the host, float64."""
    pg, row = places(c, b, first, count)
    return host(c.K[pg, :, row]), host(c.V[pg, :, row]), \
        np.zeros((count, c.K.shape[1])) if c.bias is None else host(c.bias[pg, :, row])


def tree(kind, n, seed):
    """parent [n] of a chain, of a drawn tree, of a star, or of one with parents that are none."""
    r = np.random.default_rng(seed)
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "tree":
        return [-1] + [int(i * r.random() ** 0.5) for i in range(1, n)]
    return [[-1, -5, i, i + 1, 1 << 30, -(1 << 31), max(0, i - 2)][r.integers(7)] for i in range(n)]


def above(parent):
    """[n, n]: whether node j is node i or above it; a parent that is no earlier node is none."""
    n = len(parent)
    m = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while True:
            m[i, j] = True
            if not 0 <= parent[j] < j:
                break
            j = parent[j]
    return m


def attention(q, k, v, bias, see, G, scale):
    """Rows [n, H G, d] in float64 of nodes q that see [n, entries] of the rows k, v [entries, H, d]; and, per output,
    the same sum over |v|, and the largest |logit|."""
    n, heads, d = q.shape
    out, size, big = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for h in range(heads):
        b = bias[:, h // G]
        for i in range(n):
            on = see[i] & (b > NEG_INF)
            if not on.any():
                continue
            x = k[on, h // G] @ q[i, h] * scale
            big = max(big, np.abs(x).max())
            x = x + b[on]
            w = np.exp(x - x.max())
            w /= w.sum()
            out[i, h], size[i, h] = w @ v[on, h // G], w @ np.abs(v[on, h // G])
    return out, size, big


def assert_near(got, want, size, big, entries, dtype, note=""):
    """Per row, in the 2-norm.  Of a weight a logit's roundings move a dozen steps of 2^-24 at |x| = 1, growing with |x|
    (a sum of d products, its scale, its bias, the exponential); an accumulator of a wave adds a quarter of the
    entries one after the other at most, the merges another dozen.  bf16 weights enter as two numbers, which leaves
    2^-16 of each at most (2^-8 of what 2^-8 left).  Then one rounding to the output's type."""
    got = np.asarray(got, np.float64)
    empty = (size == 0).all(-1)
    assert (got[empty] == 0).all(), note
    if empty.all():
        return
    norm = lambda x: np.linalg.norm(x, axis=-1)[~empty]
    tol = (2.0 ** -24 * (24 + 2 * big + entries / 4) + (2.0 ** -16 if dtype == "bf16" else 0)) * norm(size) \
        + half_step(dtype) * norm(want)
    err = norm(got - want)
    assert (err <= tol).all(), (note, (err / tol).max())
    # and by channel, so that no single one hides
    tol = (2.0 ** -24 * (24 + 4 * big + entries / 4) + (2.0 ** -16 if dtype == "bf16" else 0)) * (size + norm_of(size)) \
        + half_step(dtype) * np.abs(want) * 1.01
    assert (np.abs(got - want) <= tol).all(), (note, (np.abs(got - want) / tol).max())


def norm_of(size):
    return size.mean(-1, keepdims=True)


def turn(x, pos, freq, layout, scale):
    """Rows [m, h, d] turned by positions [m] in float64, and a bound of what two products of them add up to."""
    r = 2 * len(freq)
    a = pos.astype(np.float64)[:, None] * freq[None]
    cos, sin = np.cos(a)[:, None] * scale, np.sin(a)[:, None] * scale
    y, size = x.copy(), np.zeros_like(x)
    lo, hi = (np.arange(r // 2), np.arange(r // 2) + r // 2) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    size[..., lo] = size[..., hi] = (np.abs(x[..., lo]) + np.abs(x[..., hi])) * abs(scale)
    return y, size
