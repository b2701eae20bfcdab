"""selkv_tree_attn against plain 64-bit code."""
import itertools

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
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


class Call:
    """A cache whose sequences hold lens[b] entries and the rows of counts[b] nodes behind them, and the nodes' queries."""

    def __init__(self, S, B, H, G, d, dtype, page, lens, n, counts=None, kind="tree", bias=True, seed=0, top=None,
                 spread=1.0, scale=0.0):
        self.S, self.n, self.dtype, self.lens, self.counts, self.G = S, n, dtype, lens, counts, G
        g = U.gen(seed)
        self.p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype, scale=scale)
        self.scale = scale or d ** -0.5
        self.c = U.make_cache(S, self.p, [max(x, 0) + n for x in lens], 0, page, g, dtype, bias)
        self.parents = [U.tree(kind, n, 100 * seed + b) for b in range(B)]
        self.q = (torch.randn((B, n, H * G, d), generator=g, device=DEV) * spread).to(U.dtype_of(dtype))
        self.top = max(lens) if top is None else top
        self.uniform = counts is None and len(set(lens)) == 1 and self.top == lens[0]
        self.kind = kind

    def nodes(self, b):
        m = self.n if self.counts is None else self.counts[b]
        return m if 0 <= self.lens[b] <= self.top and 0 <= m <= self.n else 0

    def run(self, ws=None, out=None, stream=None, parent="given"):
        out = torch.full_like(self.q, float("nan")) if out is None else out
        parent = (None if self.kind == "chain" else i32(self.parents)) if parent == "given" else parent
        ws = self.S.tree_workspace(self.p, self.c, self.n) if ws is None else ws
        self.S.tree_attn(self.p, self.c, self.q, parent, self.top, out, ws, None if self.uniform else i32(self.lens),
                         i32(self.counts), stream)
        return out

    def want(self, b):
        m, L = self.nodes(b), self.lens[b]
        k, v, bias = U.entries(self.c, b, 0, L + m)
        see = np.ones((m, L + m), bool)
        see[:, L:] = U.above(self.parents[b])[:m, :m]
        return (*U.attention(U.host(self.q[b, :m]), k, v, bias, see, self.G, self.scale), L + m)

    def check(self, out, note=""):
        torch.cuda.synchronize()
        for b in range(len(self.lens)):
            m = self.nodes(b)
            assert bool(torch.isnan(out[b, m:]).all()), (note, b)      # rows that are not there stay
            if m:
                want, size, big, entries = self.want(b)
                U.assert_near(U.host(out[b, :m]), want, size, big, entries, self.dtype, (note, b))


LENGTHS = [0, 1, 15, 31, 32, 33, 127, 128, 130, 1000, 2333]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 5, 13, 64])
def test_lengths(S, dtype, d, n):
    for i, L in enumerate(LENGTHS):
        c = Call(S, 1, 2, 3, d, dtype, [16, 64, 256][i % 3], [L], n, kind=["tree", "chain", "star"][i % 3], seed=i)
        c.check(c.run(), L)


@pytest.mark.parametrize("G", [1, 2, 4, 5, 7, 8, 16, 33, 64])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_heads_of_a_group(S, G, dtype):
    """Rows from one tile to all that a call may have."""
    for n in (1, 3, 8, 33) if G < 33 else (1, 17, 64):
        c = Call(S, 2, 2 if G < 16 else 1, G, 64, dtype, 32, [210, 210], n, seed=G)
        c.check(c.run(), n)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("kind", ["tree", "chain", "star", "broken"])
def test_pages_and_trees(S, page, kind):
    for L in (3, page - 1, page, 4 * page + 7):
        c = Call(S, 2, 2, 2, 128, "bf16", page, [L, L], 21, kind=kind, seed=page + L)
        c.check(c.run(), L)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bias", [True, False])
def test_ragged(S, dtype, bias):
    """Sequences of their own lengths and counts, from nothing on; some that take no part."""
    c = Call(S, 9, 2, 4, 128, dtype, 32, [0, 700, 33, 5, 64, 1, 300, 301, -1], 26,
             counts=[26, 3, 0, 1, 25, 26, 27, 5, 4], bias=bias, seed=7, top=700)
    c.check(c.run())
    c = Call(S, 4, 2, 4, 64, dtype, 64, [120, 121, 5000, 90], 9, counts=[9, 9, 9, -1], bias=bias, seed=8, top=120)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_and_many(S, dtype):
    """Splits of one head, of several, and none where the heads fill the chip."""
    for (B, H, G, n, L) in [(1, 1, 4, 5, 9001), (1, 8, 4, 12, 3001), (40, 8, 2, 3, 300), (130, 8, 1, 1, 70)]:
        c = Call(S, B, H, G, 128 if B == 1 else 64, dtype, 64, [L] * B, n, seed=B + H)
        c.check(c.run(), (B, L))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_peaked_rows(S, dtype):
    """Logits of some tens, a scale of its own."""
    c = Call(S, 1, 2, 4, 128, dtype, 64, [1500], 10, spread=12.0, seed=3)
    c.check(c.run())
    c = Call(S, 1, 2, 4, 128, dtype, 64, [1500], 10, scale=0.5, seed=4)
    c.check(c.run())


def test_a_single_node_is_a_decode_step(S):
    """The contiguous cache's decode over the same entries, to what the output's rounding allows."""
    for L in (1, 64, 1027):
        c = Call(S, 3, 4, 4, 128, "fp32", 64, [L - 1] * 3, 1, seed=L)
        rows = [U.places(c.c, b, 0, L) for b in range(3)]
        K, V = (torch.stack([x[pg, :, row].transpose(0, 1) for pg, row in rows]).contiguous() for x in (c.c.K, c.c.V))
        bias = torch.stack([c.c.bias[pg, :, row].t() for pg, row in rows]).contiguous()
        ref = S.Decoder(c.p, L, DEV).run(c.q[:, 0].contiguous(), K, V, bias)
        out = c.run()[:, 0]
        assert float((out - ref).norm() / ref.norm()) < 2.0 ** -24 * 48


def test_masked_entries(S):
    """Masks of every kind: single entries, whole tiles, nodes, everything, fp32's lowest value, plus infinity."""
    for dtype in ("bf16", "fp32"):
        c = Call(S, 5, 2, 2, 64, dtype, 16, [200] * 5, 9, seed=11)
        for b, first, count in ((0, 0, 64), (0, 77, 1), (1, 0, 209), (2, 0, 200), (3, 200, 9)):
            pg, row = U.places(c.c, b, first, count)
            c.c.bias[pg, :, row] = U.NEG_INF
        out = c.run()
        assert bool((out[1] == 0).all())
        c.check(out, dtype)
        # all of them at the lowest finite value: the logits drown, and every seen entry counts alike
        pg, row = U.places(c.c, 4, 0, 209)
        c.c.bias[pg, :, row] = torch.finfo(torch.float32).min
        out = U.host(c.run()[4])
        k, v, _ = U.entries(c.c, 4, 0, 209)
        see = np.concatenate((np.ones((9, 200), bool), U.above(c.parents[4])), 1)
        want = np.stack([[v[see[i], h // 2].mean(0) for h in range(4)] for i in range(9)])
        size = np.stack([[np.abs(v[see[i], h // 2]).mean(0) for h in range(4)] for i in range(9)])
        U.assert_near(out, want, size, 0.0, 209, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_what_is_masked_may_hold_anything(S, dtype, bad):
    c = Call(S, 2, 2, 2, 128, dtype, 16, [150, 150], 12, seed=12)
    good = c.run()
    # masked by their bias
    pg, row = U.places(c.c, 0, 40, 7)
    c.c.bias[pg, :, row] = U.NEG_INF
    masked = c.run()
    c.c.K[pg, :, row], c.c.V[pg, :, row] = bad, bad
    assert torch.equal(c.run(), masked)
    # a node that others do not attend to: its row reaches those that do and no one else
    see = U.above(c.parents[1])
    pg, row = U.places(c.c, 1, 150 + 5, 1)
    for t in (c.c.K, c.c.V):
        t[pg, :, row] = bad
    out = c.run()
    for i in range(12):
        if not see[i, 5]:
            assert torch.equal(out[1, i], good[1, i]), i
    # rows behind the nodes, and pages of no one
    c.c.V[:, :, :] = torch.where(torch.isnan(c.c.V), bad, c.c.V)
    assert torch.equal(c.run()[0], masked[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_and_nan_values_reach_their_rows(S, dtype):
    inf, nan = float("inf"), float("nan")
    c = Call(S, 1, 1, 2, 64, dtype, 16, [100], 8, kind="chain", seed=13)
    good = c.run()
    pg, row = U.places(c.c, 0, 0, 108)
    c.c.V[pg[20], 0, row[20], 3] = inf
    c.c.V[pg[21], 0, row[21], 4] = -inf
    c.c.V[pg[22], 0, row[22], 5] = nan
    c.c.V[pg[23], 0, row[23], 6], c.c.V[pg[97], 0, row[97], 6] = inf, -inf
    c.c.V[pg[104], 0, row[104], 9] = -inf     # node 4
    out = c.run()[0].float()
    assert bool((out[..., 3] == inf).all()) and bool((out[..., 4] == -inf).all())
    assert bool(torch.isnan(out[..., 5]).all()) and bool(torch.isnan(out[..., 6]).all())
    assert bool((out[4:, :, 9] == -inf).all()) and torch.equal(out[:4, :, 9], good[0, :4, :, 9].float())
    rest = [j for j in range(64) if j not in (3, 4, 5, 6, 9)]
    assert torch.equal(out[..., rest], good[0][..., rest].float())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bad_queries_and_logits_stay_in_their_rows(S, dtype):
    c = Call(S, 2, 2, 2, 64, dtype, 64, [90, 90], 6, seed=14)
    good = c.run()
    c.q[0, 2, 1, 5] = float("nan")
    c.q[0, 4, 0, 5] = float("inf")
    out = c.run()
    assert bool(torch.isnan(out[0, 2, 1]).all()) and bool(torch.isnan(out[0, 4, 0]).all())
    keep = torch.ones(out.shape[:3], dtype=torch.bool, device=DEV)
    keep[0, 2, 1] = keep[0, 4, 0] = False
    assert torch.equal(out[keep], good[keep])
    # all masked: 0 whatever the query
    c.c.bias.fill_(U.NEG_INF)
    assert bool((c.run() == 0).all())
    # a NaN bias reaches every row of its head that sees the entry
    c = Call(S, 1, 2, 2, 64, dtype, 64, [90], 6, seed=15)
    good = c.run()
    pg, row = U.places(c.c, 0, 31, 1)
    c.c.bias[pg, 0, row] = float("nan")
    out = c.run()
    assert bool(torch.isnan(out[:, :, :2]).all()) and torch.equal(out[:, :, 2:], good[:, :, 2:])


def test_entries_without_a_page(S):
    """Left out: the same as masked by their biases."""
    for dtype, bad in itertools.product(("bf16", "fp32"), (-1, 1 << 30, -(1 << 31))):
        c = Call(S, 1, 2, 2, 64, dtype, 16, [200], 7, seed=16)
        pg, row = U.places(c.c, 0, 48, 32)
        held = c.c.bias[pg, :, row].clone()
        c.c.bias[pg, :, row] = U.NEG_INF
        want = c.run()
        c.c.bias[pg, :, row] = held
        c.c.table[0, 3:5] = bad
        assert torch.equal(c.run(), want)
        c.c.table[0, :] = bad
        assert bool((c.run() == 0).all())


def test_shared_pages_and_a_table_that_ends_early(S):
    """Two sequences with one prefix; entries past the last column are left out."""
    c = Call(S, 2, 2, 2, 64, "fp32", 16, [96, 96], 4, seed=17)
    c.c.table[1, :6] = c.c.table[0, :6]
    c.check(c.run())
    cut = S.PagedCache.over(c.p, c.c.K, c.c.V, c.c.table[:, :6].contiguous(), c.c.bias)     # 96 entries, no nodes
    out, ref = torch.empty_like(c.q), torch.empty_like(c.q)
    lens = i32([96, 96])
    S.tree_attn(c.p, cut, c.q, i32(c.parents), 96, out, S.tree_workspace(c.p, cut, 4), lens)
    pg, row = U.places(c.c, 0, 96, 4)
    c.c.bias[pg, :, row] = U.NEG_INF
    pg, row = U.places(c.c, 1, 96, 4)
    c.c.bias[pg, :, row] = U.NEG_INF
    S.tree_attn(c.p, c.c, c.q, i32(c.parents), 96, ref, S.tree_workspace(c.p, c.c, 4), lens)
    assert float((out - ref).norm() / ref.norm()) < 2.0 ** -24 * 48


def test_zero_biases_are_none(S):
    for dtype in ("bf16", "fp32"):
        c = Call(S, 2, 2, 3, 128, dtype, 64, [333, 333], 9, bias=False, seed=18)
        plain = c.run()
        c.c = S.PagedCache.over(c.p, c.c.K, c.c.V, c.c.table, torch.zeros(c.c.K.shape[:3], device=DEV))
        assert torch.equal(c.run(), plain)


def test_deterministic_and_free_of_what_was_there(S):
    c = Call(S, 3, 8, 4, 128, "bf16", 64, [2000, 0, 1500], 20, counts=[20, 20, 11], seed=19)
    first = c.run()
    ws = torch.full((S.tree_workspace_bytes(c.p, c.c, 20),), 255, dtype=torch.uint8, device=DEV)   # NaNs
    for _ in range(3):
        assert torch.equal(c.run(ws).view(torch.int16), first.view(torch.int16))
    # a node's outputs do not depend on how many nodes come along, nor on the others' rows
    c.check(first)


def test_past_4_gib(S):
    p = S.params(batch=1, n_heads_kv=8, group=2, head_dim=128, kv_dtype="bf16")
    c = S.PagedCache(p, 34000, 6, DEV, page=64)
    c.table.copy_(torch.tensor([[33999, 1, 33500, 33001, 2, 33700]], dtype=torch.int32))
    call = Call(S, 1, 8, 2, 128, "bf16", 64, [370], 5, seed=20)
    g = U.gen(21)
    U.put(c, 0, 0, U.rows(g, 375, 8, 128, dtype="bf16"), U.rows(g, 375, 8, 128, dtype="bf16"))
    call.c = c
    call.check(call.run())


def test_streams_and_a_replayed_graph(S):
    """A captured call follows lens, counts, parents and the table from replay to replay."""
    c = Call(S, 3, 4, 4, 64, "bf16", 32, [601, 601, 601], 12, counts=[12, 5, 1], seed=22, top=600)   # all hold 613 rows
    c.lens = [600, 300, 10]
    side = torch.cuda.Stream()
    ws = S.tree_workspace(c.p, c.c, 12)
    eager = c.run(ws)
    side.wait_stream(torch.cuda.current_stream())
    out = torch.full_like(c.q, float("nan"))
    lens, counts, parent = i32(c.lens), i32(c.counts), i32(c.parents)
    torch.cuda.synchronize()
    S.tree_attn(c.p, c.c, c.q, parent, 600, out, ws, lens, counts, stream=side)
    side.synchronize()
    assert torch.equal(out.nan_to_num(7.0), eager.nan_to_num(7.0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.tree_attn(c.p, c.c, c.q, parent, 600, out, ws, lens, counts)
    for k in range(4):
        c.lens = [[600, 300, 10], [0, 600, 31], [599, -1, 32], [64, 63, 601]][k]
        c.counts = [[12, 5, 1], [1, 12, 0], [11, 2, 13], [12, 12, 12]][k]
        c.parents = [U.tree(["tree", "star", "chain", "broken"][k], 12, 30 + 3 * k + b) for b in range(3)]
        c.kind = "tree"
        lens.copy_(i32(c.lens)); counts.copy_(i32(c.counts)); parent.copy_(i32(c.parents))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        c.top = 600
        assert torch.equal(out.nan_to_num(7.0), c.run(ws).nan_to_num(7.0)), k
        c.check(out, k)


def test_refusals(S):
    c = Call(S, 2, 2, 2, 64, "bf16", 16, [20, 20], 4, seed=23)
    ws, out, par = S.tree_workspace(c.p, c.c, 4), torch.empty_like(c.q), i32(c.parents)
    run = lambda **k: S.tree_attn(**{**dict(p=c.p, cache=c.c, q=c.q, parent=par, cache_len=20, out=out, ws=ws), **k})
    run()
    for bad in (dict(q=c.q.float()), dict(q=c.q[:, :3]), dict(out=out.float()), dict(parent=par.long()),
                dict(parent=par[:, :3]), dict(lens=i32([1])), dict(counts=i32([1, 2, 3])), dict(ws=ws.cpu()),
                dict(q=c.q.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            run(**bad)
    with pytest.raises(S.SelkvError, match="EINVAL"):
        run(cache_len=c.c.capacity - 3)
    with pytest.raises(S.SelkvError, match="EUNSUPPORTED"):
        q = torch.zeros((2, 65, 4, 64), dtype=torch.bfloat16, device=DEV)
        run(q=q, out=torch.zeros_like(q), parent=None)
    big = Call(S, 1, 2, 2, 64, "bf16", 16, [5000], 4, seed=24)
    with pytest.raises(S.SelkvError, match="EWORKSPACE"):
        S.tree_attn(big.p, big.c, big.q, None, 5000, torch.empty_like(big.q), None)
