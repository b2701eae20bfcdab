"""selkv_tree_verify: which rows of the draft a walk may look at."""
import numpy as np
import pytest
import torch

from tests import paged_util as U
from tests.test_verify_gpu import S, drawn, run, walk  # noqa: F401  (S is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 257, 2049, 32000, 70001])
@pytest.mark.parametrize("n,kind", [(1, "chain"), (5, "chain"), (9, "tree"), (7, "star")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_no_child_was_drawn_from_are_not_looked_at(S, dtype, vocab, n, kind, bad):
    """A draft is not run on the last tokens that it drafted: the rows of leaves, and of nodes that are not there, hold
    whatever their memory held."""
    tokens, parent, target, draft, u = drawn(6, n, vocab, kind, dtype, vocab + n, noise=0.1)
    counts = [n, n, n, max(1, n // 2), 1, n]
    t, q = U.host(target), U.host(draft)
    inner = [{parent[b][i] for i in range(1, counts[b])} for b in range(6)]
    for b in range(6):
        for i in range(n):
            if i not in inner[b]:
                draft[b, i] = bad
    path, n_path, nxt = (x.cpu().numpy() for x in run(S, tokens, parent, target, draft, u, counts))
    ends = 0
    for b in range(6):
        want, token = walk(tokens[b], parent[b], t[b], q[b], u[b].astype(np.float64), counts[b])
        assert list(path[b]) == want + [-1] * (n - len(want)) and n_path[b] == len(want) and nxt[b] == token, (b, want, token, nxt[b])
        ends += want[-1] not in inner[b]
    assert ends > 0          # walks that end at such a row


@pytest.mark.parametrize("vocab", [300, 70001])
def test_a_row_whose_token_is_drawn_from_the_target_itself(S, vocab):
    """Nothing is left of the target after a refusal: the draft's other probabilities do not matter either."""
    t = torch.zeros((1, 2, vocab), device=U.DEV)
    q = torch.zeros((1, 2, vocab), device=U.DEV)
    t[..., 7], t[..., 200] = 0.25, 0.75
    q[0, 0, 7], q[0, 0, 200], q[0, 0, 9] = float("inf"), float("inf"), 1.0
    for u0, token in ((0.0, 7), (0.2, 7), (0.3, 200), (0.99, 200)):
        path, n_path, nxt = run(S, [[0, 9]], [[-1, 0]], t, q, [[u0, 0.5]])
        assert path.tolist() == [[0, -1]] and n_path.tolist() == [1] and nxt.tolist() == [token]
