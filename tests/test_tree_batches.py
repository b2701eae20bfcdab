"""selkv_tree_attn over batches of many lengths: sequences in any order, more than 64 of them, and some that hold so few of
the nodes that half of a workgroup's waves hold all of their rows."""
import pytest
import torch

from tests import paged_util as U
from tests.test_tree_gpu import S, Call, i32  # noqa: F401  (S is a fixture)

pytestmark = pytest.mark.gpu
DEV = U.DEV


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,G,d,n", [(8, 8, 128, 26), (2, 8, 64, 20), (3, 4, 128, 33), (1, 5, 64, 64)])
def test_few_and_many_of_the_nodes(S, dtype, H, G, d, n):
    """Over and up to half of the rows of a workgroup, one row, none; lengths that end in either tile of a turn."""
    half = (128 if dtype == "bf16" or d == 64 else 64) // G
    counts = [n, min(n, half), min(n, half + 1), 1, 0, 3, min(n, half - 1), 2]
    lens = [700, 65, 1000, 1301, 900, 0, 31, 96]
    c = Call(S, 8, H, G, d, dtype, 32, lens, n, counts=counts, seed=30)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,G", [(1, 2), (6, 4), (9, 8)])
@pytest.mark.parametrize("B", [63, 64, 65, 131])
def test_many_sequences(S, dtype, n, G, B):
    lens = [(37 * b * b + 11 * b) % 190 for b in range(B)]
    counts = [(5 * b) % (n + 1) for b in range(B)]
    lens[B // 2] = lens[B - 1] = lens[0]           # as long as another
    c = Call(S, B, 2, G, 64, dtype, 16, lens, n, counts=counts, seed=31)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_what_is_masked_where_half_of_the_waves_share_the_rows(S, dtype, bad):
    c = Call(S, 3, 2, 8, 128, dtype, 16, [640, 500, 333], 26, counts=[26, 12, 5], seed=32)
    for b, first in ((1, 70), (2, 300)):
        pg, row = U.places(c.c, b, first, 33)
        c.c.bias[pg, :, row] = U.NEG_INF
    good = c.run()
    for b, first in ((1, 70), (2, 300)):
        pg, row = U.places(c.c, b, first, 33)
        c.c.K[pg, :, row], c.c.V[pg, :, row] = bad, bad
    out = c.run()
    for b, count in enumerate((26, 12, 5)):
        assert torch.equal(out[b, :count], good[b, :count]), b


@pytest.mark.parametrize("n,G", [(5, 4), (26, 8)])
def test_the_order_changes_no_bit(S, n, G):
    """A sequence's outputs do not depend on its place in the batch."""
    lens, counts = [0, 900, 41, 900, 333], [n, n // 2, 1, n, n - 1]
    c = Call(S, 5, 8, G, 128, "bf16", 16, lens, n, counts=counts, seed=33)
    out = c.run()
    order = torch.tensor([3, 0, 4, 2, 1], device=DEV)
    cache = S.PagedCache.over(c.p, c.c.K, c.c.V, c.c.table[order].contiguous(), c.c.bias)
    to = torch.empty_like(out)
    S.tree_attn(c.p, cache, c.q[order].contiguous(), i32(c.parents)[order].contiguous(), 900, to,
                S.tree_workspace(c.p, cache, n), lens=i32(lens)[order].contiguous(), counts=i32(counts)[order].contiguous())
    for at, b in enumerate(order.tolist()):
        assert torch.equal(to[at, :counts[b]], out[b, :counts[b]]), b
