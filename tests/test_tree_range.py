"""selkv_tree_attn over the range of fp32: finite biases and values however large, and infinite values with hardly a weight."""
import numpy as np
import pytest
import torch

from tests import paged_util as U
from tests.test_tree_gpu import S, Call  # noqa: F401  (S is a fixture)

pytestmark = pytest.mark.gpu
DEV = U.DEV

# nodes, G, entries, counts: one row tile, two, the kernels that share tiles, sequences whose rows half of the waves hold;
# every one in a single workgroup and in splits
SHAPES = [(1, 2, 90, None), (1, 2, 700, None), (9, 2, 700, None), (11, 4, 40, None), (11, 4, 700, None), (12, 8, 700, None),
          (26, 8, 40, None), (26, 8, 700, None), (26, 8, 700, [26, 12])]
LOWEST = torch.finfo(torch.float32).min


def call(S, dtype, n, G, L, counts, seed, d=128, **kw):
    B = 2 if counts else 1
    return Call(S, B, 2, G, d, dtype, 16, [L] * B, n, counts=counts, seed=seed, **kw)


def bias_of(c, b, first, count, value):
    pg, row = U.places(c.c, b, first, count)
    c.c.bias[pg, :, row] = value


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
def test_a_finite_mask_on_a_prefix_is_a_mask(S, dtype, n, G, L, counts):
    """Left padding: tiles, waves and splits that hold nothing else.  The weights are 0 in any precision, so the outputs
    are those of a mask of -inf, bit for bit."""
    for first, count in ((0, L * 3 // 4), (0, L), (L // 3, L // 3)):
        c = call(S, dtype, n, G, L, counts, 41)
        for b in range(len(c.lens)):
            bias_of(c, b, first, count, U.NEG_INF)
        want = c.run()
        c.check(want)
        for value in (-1e4, -1e9, -3e9, -1e10, -1e11, -1e20, -1e30, -1e38, -2.4e38, LOWEST):
            for b in range(len(c.lens)):
                bias_of(c, b, first, count, value)
            assert torch.equal(c.run().nan_to_num(7.0), want.nan_to_num(7.0)), (value, first, count)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
def test_one_large_bias_on_every_entry(S, dtype, n, G, L, counts):
    """Where the logits drown in it every seen entry counts alike; where they do not, their roundings are those of the
    bias."""
    c = call(S, dtype, n, G, L, counts, 42)
    for value in (-3000.0, 1e4, -1e4, -1e9, 1e9, -1e10, 1e10, -1e11, 1e11, -1e30, 1e30, -1e38, 1e38, 2.4e38, 3.4e38, LOWEST):
        for b in range(len(c.lens)):
            bias_of(c, b, 0, L + n, value)
        out = c.run()
        for b in range(len(c.lens)):
            want, size, big, entries = c.want(b)
            if abs(value) >= 1e9:          # the logits, less than 20, are below half of its last place
                m = c.nodes(b)
                _, v, _ = U.entries(c.c, b, 0, L + m)
                see = np.ones((m, L + m), bool)
                see[:, L:] = U.above(c.parents[b])[:m, :m]
                want = np.stack([[v[see[i], h // G].mean(0) for h in range(2 * G)] for i in range(m)])
                size = np.stack([[np.abs(v[see[i], h // G]).mean(0) for h in range(2 * G)] for i in range(m)])
                assert big < 20
                big = 0.0
            else:
                big += abs(value)          # a logit's sum with it is rounded to 2^-24 of both
            U.assert_near(U.host(out[b, :c.nodes(b)]), want, size, big, entries, dtype, (value, b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
def test_biases_of_many_sizes(S, dtype, n, G, L, counts):
    """The largest takes all: what is far below it has no weight, in whatever order they come."""
    values = [-1e38, -1e30, -1e11, -1e10, -3e9, -1e5, 1e5, 3e9, 1e10, 1e11, 1e30, 1e38]
    for order in (values, values[::-1], values[1::2] + values[::2]):
        c = call(S, dtype, n, G, L, counts, 43)
        step = L // len(values)
        for b in range(len(c.lens)):
            for i, value in enumerate(order):
                bias_of(c, b, i * step, step, value)
        out = c.run()
        at = order.index(1e38) * step
        for b in range(len(c.lens)):
            m = c.nodes(b)
            _, v, _ = U.entries(c.c, b, at, step)
            mean, size = (np.broadcast_to(np.repeat(x.mean(0), G, 0), (m, 2 * G, 128)) for x in (v, np.abs(v)))
            U.assert_near(U.host(out[b, :m]), mean, size, 0.0, step, dtype, b)


def assert_means(c, b, out, note):
    """Every output against 64 bits.  One entry may be all that counts in a channel, so the error of a single weight does:
    a logit is a sum of d products, and each of d + 2 roundings is at most 2^-24 of A, the sum of the products'
    magnitudes and the bias; a weight's error is that of its logit and of the sum of weights, each rounded in an
    exponential of 2^-22 and, for bf16, in two numbers, 2^-16.  The accumulators' roundings are those of assert_near."""
    want, size, _, entries = c.want(b)
    m = c.nodes(b)
    k, _, bias = U.entries(c.c, b, 0, entries)
    q, d = np.abs(U.host(c.q[b, :m])), c.q.shape[-1]
    A = max((q[:, h] @ np.abs(k[:, h // c.G]).T * c.scale).max() for h in range(q.shape[1])) + np.abs(bias).max()
    rel = 2 * (d + 2) * 2.0 ** -24 * A + 2.0 ** -21 + 2.0 ** -24 * (24 + entries / 4) + (2.0 ** -15 if c.dtype == "bf16" else 0)
    got = U.host(out[b, :m])
    assert np.isfinite(got).all(), note
    tol = rel * size + U.half_step(c.dtype) * np.abs(want) * 1.01
    assert (np.abs(got - want) <= tol).all(), (note, (np.abs(got - want) / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
@pytest.mark.parametrize("where", ["all", "a few", "one split", "nodes"])
def test_finite_values_give_finite_means(S, dtype, n, G, L, counts, where):
    """Values up to 3e38: their weighted mean is finite, so is the output."""
    for signs, spread in ((False, 1.0), (True, 1.0), (True, 6.0)):
        c = call(S, dtype, n, G, L, counts, 44, spread=spread)
        g = U.gen(45)
        for b in range(len(c.lens)):
            m = c.nodes(b)
            first, count = {"all": (0, L + m), "a few": (L // 2, 3), "one split": (0, min(L, 128)), "nodes": (L, m)}[where]
            pg, row = U.places(c.c, b, first, count)
            x = 10.0 ** (36.0 + 2.47 * torch.rand((count, 2, 128), generator=g, device=DEV).double())
            if signs:
                x *= torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.5, -1.0, 1.0)
            c.c.V[pg, :, row] = x.to(c.c.V.dtype)
        assert bool(torch.isfinite(c.c.V[c.c.table[0, 0].long()]).all())
        out = c.run()
        for b in range(len(c.lens)):
            assert_means(c, b, out, (where, signs, spread, b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
def test_finite_values_under_large_biases(S, dtype, n, G, L, counts):
    """Means of 3e38 and of 1e38 and 3e38: between them, to the roundings of weights, sums and output."""
    for value in (-1.6e7, -1e6, -1500.0, 1500.0, 1e6, 1.6e7):
        c = call(S, dtype, n, G, L, counts, 47)
        for b in range(len(c.lens)):
            bias_of(c, b, 0, L + n, value)
            pg, row = U.places(c.c, b, 0, L + n)
            c.c.V[pg, :, row] = 3e38
            c.c.V[pg[::3], :, row[::3], 64:] = 1e38
        out = c.run()
        for b in range(len(c.lens)):
            got = out[b, :c.nodes(b)].double() / 1e38
            rel = 2.0 ** -7 + (L + n) * 2.0 ** -22
            assert bool(((got[..., :64] - 3.0).abs() <= 3 * rel).all()), value
            assert bool((got[..., 64:] <= 3 * (1 + rel)).all()) and bool((got[..., 64:] >= 1 - rel).all()), value


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G,L,counts", SHAPES)
def test_infinite_values_with_hardly_a_weight(S, dtype, n, G, L, counts):
    """e^-200 of infinity is infinite, wherever the entry lies: in a row's first tile or its last, in tiles, waves and
    splits of such entries alone or beside others."""
    inf = float("inf")
    for first, count in ((0, L * 3 // 4), (L // 4, L * 3 // 4), (0, 0)):
        c = call(S, dtype, n, G, L, counts, 46)
        for b in range(len(c.lens)):
            bias_of(c, b, first, count, -200.0)
        good = c.run()
        for b in range(len(c.lens)):
            for j, e in enumerate((0, 5, L // 3, L // 2, L - 1)):
                pg, row = U.places(c.c, b, e, 1)
                c.c.V[pg, :, row, 10 + j] = -inf if j % 2 else inf
                c.c.bias[pg, :, row] = -200.0
        for b in range(len(c.lens)):
            bias_of(c, b, 0, 5, -300.0)        # behind which more comes in any case
        out = c.run()
        for b in range(len(c.lens)):
            m = c.nodes(b)
            for j in range(5):
                assert bool((out[b, :m, :, 10 + j] == (-inf if j % 2 else inf)).all()), (first, b, j)
            rest = [j for j in range(128) if not 10 <= j < 15]
            assert bool(torch.isfinite(out[b, :m][..., rest]).all()) and bool(torch.isfinite(good[b, :m]).all())
