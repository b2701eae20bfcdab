"""selkv_tree_attn where a workgroup's waves share entries (more than 32 rows a KV head), and over caches of many pages a
workgroup: masks, entries without a page, values that are NaN or infinite."""
import numpy as np
import pytest
import torch

from tests import paged_util as U
from tests.test_tree_gpu import S, Call, i32  # noqa: F401  (S is a fixture)

pytestmark = pytest.mark.gpu
DEV = U.DEV
ROWS = [(11, 4), (12, 8), (26, 8), (64, 5)]      # 44, 96, 208 and 320 rows


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,G", ROWS)
def test_lengths_and_masks(S, dtype, d, n, G):
    for i, L in enumerate((0, 31, 64, 127, 129, 700)):
        c = Call(S, 2, 1, G, d, dtype, [16, 64][i % 2], [L, L], n, seed=100 + i)
        if L > 64:
            pg, row = U.places(c.c, 0, 3, 60)
            c.c.bias[pg, :, row] = U.NEG_INF
            pg, row = U.places(c.c, 1, 0, L + n)
            c.c.bias[pg, :, row] = U.NEG_INF
        out = c.run()
        c.check(out, L)
        assert L <= 64 or bool((out[1] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G", ROWS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_what_is_masked_may_hold_anything(S, dtype, n, G, bad):
    c = Call(S, 2, 2, G, 128, dtype, 16, [400, 300], n, counts=[n, n - 1], seed=12)
    good = c.run()
    pg, row = U.places(c.c, 0, 140, 70)
    c.c.bias[pg, :, row] = U.NEG_INF
    masked = c.run()
    c.c.K[pg, :, row], c.c.V[pg, :, row] = bad, bad
    assert torch.equal(c.run().nan_to_num(7.0), masked.nan_to_num(7.0))
    see = U.above(c.parents[1])
    pg, row = U.places(c.c, 1, 300 + 5, 1)
    c.c.K[pg, :, row], c.c.V[pg, :, row] = bad, bad
    out = c.run()
    for i in range(n - 1):
        if not see[i, 5]:
            assert torch.equal(out[1, i], good[1, i]), i
        elif bad != 3e38:
            assert not bool(torch.isfinite(out[1, i]).any())
    assert torch.equal(out[0], masked[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G", ROWS)
def test_bad_rows_stay_alone(S, dtype, n, G):
    c = Call(S, 1, 1, G, 64, dtype, 64, [500], n, seed=14)
    good = c.run()
    c.q[0, 2, 1, 5], c.q[0, n - 1, 0, 7] = float("nan"), float("inf")
    out = c.run()
    keep = torch.ones(out.shape[:3], dtype=torch.bool, device=DEV)
    keep[0, 2, 1] = keep[0, n - 1, 0] = False
    assert torch.equal(out[keep], good[keep]) and bool(torch.isnan(out[~keep]).all())
    pg, row = U.places(c.c, 0, 0, 500)
    c.c.V[pg[77], 0, row[77], 3], c.c.V[pg[300], 0, row[300], 4] = float("inf"), float("nan")
    out = c.run()[keep].float()
    assert bool((out[:, 3] == float("inf")).all()) and bool(torch.isnan(out[:, 4]).all())
    rest = [j for j in range(64) if j not in (3, 4)]
    assert torch.equal(out[:, rest], good[keep][:, rest].float())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G", [(1, 2), (9, 2), (11, 4), (26, 8)])
def test_entries_without_a_page(S, dtype, n, G):
    for first, count in ((0, 1), (7, 3), (60, 2)):
        c = Call(S, 1, 2, G, 64, dtype, 16, [1000], n, seed=16)
        pg, row = U.places(c.c, 0, 16 * first, 16 * count)
        held = c.c.bias[pg, :, row].clone()
        c.c.bias[pg, :, row] = U.NEG_INF
        want = c.run()
        c.c.bias[pg, :, row] = held
        c.c.table[0, first:first + count] = c.c.n_pages
        assert torch.equal(c.run(), want), first


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G", [(1, 2), (7, 4), (5, 8), (9, 12)])
def test_many_pages_a_workgroup(S, dtype, n, G):
    """264 KV heads: a workgroup takes all of a sequence, 150 pages and more; one page missing far behind."""
    lens = [2400] * 33
    c = Call(S, 33, 8, G, 64, dtype, 16, lens, n, seed=18)
    c.c.table[5, 140] = -1
    pg, row = U.places(c.c, 6, 2240, 16)
    c.c.bias[pg, :, row] = U.NEG_INF
    out = c.run()
    c.lens = lens
    for b in (0, 6, 32):
        want, size, big, entries = c.want(b)
        U.assert_near(U.host(out[b]), want, size, big, entries, dtype, b)
    # the sequence with a hole, its entries gathered without it
    k, v, bias = U.entries(c.c, 5, 0, 2400 + n)
    bias[2240:2256] = -np.inf
    see = np.ones((n, 2400 + n), bool)
    see[:, 2400:] = U.above(c.parents[5])
    want, size, big = U.attention(U.host(c.q[5]), k, v, bias, see, G, c.scale)
    U.assert_near(U.host(out[5]), want, size, big, 2400 + n, dtype)


def test_zero_biases_are_none_in_every_kernel(S):
    for dtype in ("bf16", "fp32"):
        for n, G in [(1, 1), (9, 3)] + ROWS:
            c = Call(S, 1, 2, G, 128, dtype, 64, [333], n, bias=False, seed=18)
            plain = c.run()
            c.c = S.PagedCache.over(c.p, c.c.K, c.c.V, c.c.table, torch.zeros(c.c.K.shape[:3], device=DEV))
            assert torch.equal(c.run(), plain)


def test_a_node_does_not_depend_on_those_that_come_along(S):
    """Alone, in a chain and in a large tree, a node attends to the same entries; to the rounding of other divisions."""
    c = Call(S, 1, 2, 4, 64, "fp32", 16, [777], 64, kind="star", seed=20)
    full = c.run()
    for n in (2, 9, 20, 40):
        ws = S.tree_workspace(c.p, c.c, 64)
        q, out = c.q[:, :n].contiguous(), torch.empty_like(c.q[:, :n])
        S.tree_attn(c.p, c.c, q, i32(c.parents)[:, :n].contiguous(), 777, out, ws)
        assert float((out - full[:, :n]).norm() / full[:, :n].norm()) < 2.0 ** -24 * 64
