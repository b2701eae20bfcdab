"""selkv_tree_verify where the walk's sums are spread over launches: as many as there are launches, more and fewer, and walks
that are over before the last one."""
import numpy as np
import pytest
import torch

from tests import paged_util as U
from tests.test_verify_gpu import S, check, drawn, run, walk  # noqa: F401  (S is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,kind", [(33, "star"), (40, "tree"), (64, "star"), (64, "tree"), (64, "broken")])
def test_trees_of_many_nodes_over_a_large_vocabulary(S, dtype, n, kind):
    """More than 32 nodes and 65536 tokens: four launches.  Drafts far from the target are refused many times at a node."""
    vocab = 70001
    for noise in (0.2, 3.0):
        tokens, parent, target, draft, u = drawn(4, n, vocab, kind, dtype, n, noise, 1.2)
        counts = [n, n, max(1, n // 2), 2]
        check(S, tokens, parent, target, draft, u, counts, (n, kind, noise))
        if kind == "star":
            u[:, 1:] = 1.0 - 2.0 ** -24          # all but tokens that the target likes better are refused
            check(S, tokens, parent, target, draft, u, counts, (n, kind, noise, "refused"))


@pytest.mark.parametrize("vocab,n,launches", [(20001, 9, 1), (40001, 9, 2), (70001, 9, 3), (70001, 40, 4)])
def test_refusals_counted(S, vocab, n, launches):
    """Walks with 0 .. launches + 2 sums, all in one call: children that are refused one after the other, each of which
    wants a sum, and at the end the token's own where the last child was accepted.  The draw reads the sums of the launch
    that made the last of them."""
    B = 2 * (launches + 3)
    g = U.gen(vocab + n)
    x = torch.rand((B, n, vocab), generator=g, device=U.DEV) + 0.5
    target = x / x.sum(-1, keepdim=True)
    draft = torch.rand((B, n, vocab), generator=g, device=U.DEV) + 0.5
    # tokens 0 .. n - 1 are the children's: the target never says them, the draft does; token n it likes
    target[..., :n] = 0.0
    target[..., n] = 0.5
    draft[..., n] = 1e-3
    target, draft = (t / t.sum(-1, keepdim=True) for t in (target, draft))
    parent = [U.tree("star", n, 0)] * B
    tokens, counts = np.zeros((B, n), np.int64), []
    for b in range(B):
        refused = min(b // 2, n - 2)
        tokens[b, 1:] = np.arange(1, n)
        if b % 2:
            tokens[b, 1 + refused] = n            # accepted after so many refusals
            counts.append(2 + refused)
        else:
            counts.append(1 + refused)
    u = np.random.default_rng(7).random((B, n)).astype(np.float32)
    lengths = check(S, tokens, parent, target, draft, u, counts, (vocab, n))
    assert lengths == [1 + b % 2 for b in range(B)]
