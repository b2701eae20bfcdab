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
