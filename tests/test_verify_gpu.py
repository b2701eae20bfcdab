"""selkv_tree_verify against the walk on the distributions themselves, in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import paged_util as U

pytestmark = pytest.mark.gpu
DEV = U.DEV


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_16213_amd import selkv
    return selkv


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def walk(tokens, parent, target, draft, u, count):
    """(path, next) of one sequence: the residual itself, normalised after every refusal."""
    n, vocab = target.shape
    if not 1 <= count <= n:
        return [], -1
    at, path = 0, [0]
    r, mass, gone = target[0].copy(), 1.0, set()
    while True:
        found = None
        for i in range(at + 1, count):
            if not (0 <= parent[i] < i and parent[i] == at):
                continue
            x = int(tokens[i])
            ok = 0 <= x < vocab
            if draft is not None:
                if ok and u[i] * draft[at, x] < r[x]:
                    found = i
                    break
                left = np.maximum(r - draft[at], 0.0)
                r = left / left.sum() if left.sum() > 0 else np.zeros_like(left)
            elif ok:
                if x not in gone and u[i] * mass < r[x]:
                    found = i
                    break
                mass = max(mass - (0.0 if x in gone else r[x]), 0.0)
                gone.add(x)
        if found is None:
            break
        at = found
        path.append(at)
        r, mass, gone = target[at].copy(), 1.0, set()
    r[list(gone)] = 0.0
    if not r.sum() > 0:
        r = target[at]
    cum = np.cumsum(r)
    past = np.nonzero((cum > u[0] * cum[-1]) & (r > 0))[0]
    if len(past):
        return path, int(past[0])
    some = np.nonzero(r > 0)[0]
    return path, int(some[-1]) if len(some) else -1


def run(S, tokens, parent, target, draft, u, counts=None, ws=None):
    B, n, vocab = target.shape
    path = torch.full((B, n), 77, dtype=torch.int32, device=DEV)
    n_path, nxt = (torch.full((B,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    ws = S.tree_verify_workspace(B, n, vocab, DEV).fill_(255) if ws is None else ws
    S.tree_verify(i32(tokens), i32(parent), target, draft, torch.tensor(u, dtype=torch.float32, device=DEV), path, n_path,
                  nxt, ws, i32(counts))
    return path, n_path, nxt


def check(S, tokens, parent, target, draft, u, counts=None, note=""):
    B, n, vocab = target.shape
    u = np.asarray(u, np.float32)
    path, n_path, nxt = (t.cpu().numpy() for t in run(S, tokens, parent, target, draft, u, counts))
    t, q = U.host(target), None if draft is None else U.host(draft)
    lengths = []
    for b in range(B):
        par = [i - 1 for i in range(n)] if parent is None else parent[b]
        want, token = walk(tokens[b], par, t[b], None if q is None else q[b], u[b].astype(np.float64),
                           n if counts is None else counts[b])
        assert list(path[b]) == want + [-1] * (n - len(want)), (note, b, path[b], want)
        assert n_path[b] == len(want) and nxt[b] == token, (note, b, n_path[b], nxt[b], token)
        lengths.append(len(want))
    return lengths


def drawn(B, n, vocab, kind, dtype, seed, noise=0.7, peak=1.0):
    """Trees whose nodes' tokens are drawn from their parents' drafts."""
    r = np.random.default_rng(seed)
    g = U.gen(seed)
    x = torch.log(torch.rand((B, n, vocab), generator=g, device=DEV) * vocab + 1.0) * -peak
    target = torch.softmax(x, -1).to(U.dtype_of(dtype))
    draft = torch.softmax(x + noise * torch.randn(x.shape, generator=g, device=DEV), -1).to(U.dtype_of(dtype))
    parent = [U.tree(kind, n, seed + b) for b in range(B)]
    tokens = np.zeros((B, n), np.int64)
    q = U.host(draft)
    for b in range(B):
        for i in range(1, n):
            c = np.cumsum(q[b, parent[b][i] if 0 <= parent[b][i] < i else 0])
            tokens[b, i] = min(np.searchsorted(c, r.random() * c[-1], "right"), vocab - 1)
    return tokens, parent, target, draft, r.random((B, n)).astype(np.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 63, 257, 2047, 2048, 2049, 4099, 32000, 50001])
def test_vocabularies(S, dtype, vocab):
    """Rows that start anywhere in a 16-byte block; chunks that end anywhere."""
    total = 0
    for n, kind in ((1, "chain"), (4, "chain"), (9, "tree"), (7, "star")):
        tokens, parent, target, draft, u = drawn(3, n, vocab, kind, dtype, vocab + n)
        total += sum(check(S, tokens, parent, target, draft, u, note=(n, kind)))
        check(S, tokens, parent, target, None, u, note=(n, kind, "no draft"))
    assert total > 12


@pytest.mark.parametrize("kind", ["chain", "tree", "star", "broken"])
@pytest.mark.parametrize("draft", [True, False])
def test_trees(S, kind, draft):
    """Many sequences with up to 64 nodes, counts of their own, none and all of them among them."""
    for n, noise in ((64, 0.3), (64, 1.5), (26, 0.7), (2, 0.7)):
        tokens, parent, target, q, u = drawn(24, n, 701, kind, "fp32", n, noise, 1.3)
        counts = [n, 1, 0, -1, n + 1, max(1, n // 2)] + [n - b % n for b in range(18)]
        lengths = check(S, tokens, parent, target, q if draft else None, u, counts, (n, noise))
        assert lengths[1] == 1 and lengths[2:5] == [0, 0, 0]
    if kind == "chain":
        check(S, tokens, None, target, q if draft else None, u)


def test_all_accepted_and_all_refused(S):
    tokens, parent, target, draft, u = drawn(4, 33, 3001, "chain", "fp32", 5)
    assert check(S, tokens, parent, target, target, u) == [33] * 4              # the draft is the target
    other = torch.zeros_like(target)
    other[..., 7] = 1.0
    t = target.clone()
    t[..., 7] = 0.0
    tokens[:] = 7
    for par in (parent, [U.tree("star", 33, 0)] * 4):
        assert check(S, tokens, par, t, other, u) == [1] * 4                    # a token that the target never says
        assert check(S, tokens, par, t, None, u) == [1] * 4


def test_tokens_out_of_range_and_repeated(S):
    tokens, parent, target, draft, u = drawn(6, 12, 40, "star", "fp32", 6, peak=0.2)
    tokens[0, 1:] = 40
    tokens[1, 1:6] = -1
    tokens[2, 1:] = tokens[2, 1]
    tokens[3, 1::2] = 1 << 30
    for q in (draft, None):
        assert check(S, tokens, parent, target, q, u)[0] == 1
    u[2] = 0.999
    for q in (draft, None):
        check(S, tokens, parent, target, q, u)


def test_borders(S):
    """Probabilities and numbers that are exact in binary: u * total on a border takes the token behind it, a test that
    holds with equality refuses."""
    V = 4096
    target = torch.full((1, 2, V), 1.0 / V, device=DEV)
    draft = torch.zeros((1, 2, V), device=DEV)
    draft[0, 0, :V // 2] = 2.0 / V
    parent = [[-1, 0]]
    for x, u1, taken in ((5, 0.5, False), (5, 0.49999997, True), (0, 0.0, True), (V // 2, 0.0, True), (V - 1, 0.999, True)):
        # p / q = 1/2 in the draft's half; where it gives nothing, whatever the target has is taken
        for u0 in (0.0, 0.25, 0.5, 1.0 - 2.0 ** -24):
            u = [[u0, u1]]
            lengths = check(S, [[0, x]], parent, target, draft, u, note=(x, u1, u0))
            assert lengths == [2 if taken else 1]
            path, n_path, nxt = run(S, [[0, x]], parent, target, draft, u)
            want = int(u0 * V) if taken else V // 2 + int(u0 * (V // 2))
            assert int(nxt[0]) == min(want, V - 1)


def test_nothing_left_of_the_target(S):
    """A residual that is empty, a row without probabilities, negative ones and NaN, infinite ones."""
    V = 100
    t = torch.zeros((5, 3, V), device=DEV)
    q = torch.zeros((5, 3, V), device=DEV)
    t[0, :, 3], q[0, :, 3], q[0, :, 4] = 0.5, 0.5, 0.5          # refused at 4; nothing is left: drawn from the target
    q[1, :, 9] = 1.0                                            # a target without any probability
    t[2, :, 10], t[2, :, 20], t[2, :, 30] = -1.0, float("nan"), 0.25
    q[2, :, 50] = 1.0
    t[3, :, 7], q[3, :, 8] = float("inf"), 1.0
    t[4, :, 7], q[4, :, 7] = 0.5, float("nan")
    tokens = [[0, 4, 4], [0, 9, 9], [0, 50, 20], [0, 8, 8], [0, 7, 7]]
    path, n_path, nxt = run(S, tokens, [[-1, 0, 0]] * 5, t, q, [[0.3, 0.9, 0.9]] * 5)
    assert n_path.tolist() == [1] * 5 and nxt.tolist()[:3] == [3, -1, 30]
    assert nxt.tolist()[3] in (7, -1) and nxt.tolist()[4] in (7, -1)
    assert path.tolist() == [[0, -1, -1]] * 5


def test_the_tokens_have_the_targets_distribution(S):
    """The first token after the root over many sequences of one target and draft: whatever the draft, however many
    children.  Each count is binomial; over 3 x 2 x 12 of them five standard deviations are passed once in 25000 runs."""
    B, V = 40000, 12
    r = np.random.default_rng(9)
    p = r.dirichlet(np.ones(V)).astype(np.float32)
    q = r.dirichlet(np.ones(V) * 0.7).astype(np.float32)
    for n in (2, 4, 7):
        cum = np.cumsum(q.astype(np.float64))
        tokens = np.minimum(np.searchsorted(cum, r.random((B, n)) * cum[-1], "right"), V - 1)
        target = torch.tensor(p, device=DEV).expand(B, n, V).contiguous()
        u = r.random((B, n)).astype(np.float32)
        for draft in (torch.tensor(q, device=DEV).expand(B, n, V).contiguous(), None):
            path, n_path, nxt = (t.cpu().numpy() for t in run(S, tokens, [U.tree("star", n, 0)] * B, target, draft, u))
            first = np.where(n_path > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
            seen = np.bincount(first, minlength=V)
            pn = p.astype(np.float64) / p.astype(np.float64).sum()
            assert (np.abs(seen - B * pn) <= 5 * np.sqrt(B * pn * (1 - pn)) + 1).all(), (n, draft is None)


def test_many_sequences_and_a_large_vocabulary(S):
    tokens, parent, target, draft, u = drawn(2, 5, 151937, "tree", "fp32", 21, peak=0.9)
    for u0 in (0.0, 0.37, 0.999999):
        u[:, 0] = u0
        check(S, tokens, parent, target, draft, u)
    tokens, parent, target, draft, u = drawn(300, 3, 33, "tree", "bf16", 22)
    check(S, tokens, parent, target, draft, u)


def test_streams_graphs_and_refusals(S):
    tokens, parent, target, draft, u = drawn(3, 9, 5000, "tree", "fp32", 31)
    eager = run(S, tokens, parent, target, draft, u)
    ws = S.tree_verify_workspace(3, 9, 5000, DEV)
    tk, pa, uu = i32(tokens), i32(parent), torch.tensor(u, device=DEV)
    path, n_path, nxt = (torch.empty_like(t) for t in eager)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    S.tree_verify(tk, pa, target, draft, uu, path, n_path, nxt, ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((path, n_path, nxt), eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.tree_verify(tk, pa, target, draft, uu, path, n_path, nxt, ws)
    for k in range(3):
        t2, p2, tt, dd, u2 = drawn(3, 9, 5000, ["star", "chain", "tree"][k], "fp32", 40 + k)
        tk.copy_(i32(t2)); pa.copy_(i32(p2)); target.copy_(tt); draft.copy_(dd); uu.copy_(torch.tensor(u2))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((path, n_path, nxt), run(S, t2, p2, tt, dd, u2))), k
    ok = dict(tokens=tk, parent=pa, target=target, draft=draft, u=uu, path=path, n_path=n_path, next_token=nxt, ws=ws)
    for bad in (dict(tokens=tk.long()), dict(tokens=tk[:, :8]), dict(parent=pa.float()), dict(draft=draft.bfloat16()),
                dict(draft=draft[..., :4999]), dict(u=uu.double()), dict(path=path[:2]), dict(n_path=n_path.long()),
                dict(next_token=nxt[:2]), dict(target=target.double()), dict(counts=i32([1, 2])), dict(tokens=tk.cpu())):
        with pytest.raises(ValueError):
            S.tree_verify(**{**ok, **bad})
    t65 = torch.zeros((1, 65, 4), device=DEV)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    with pytest.raises(S.SelkvError, match="EUNSUPPORTED"):
        S.tree_verify(z(1, 65), None, t65, None, torch.zeros((1, 65), device=DEV), z(1, 65), z(1), z(1), None)
    assert math.isfinite(float(uu.sum()))
