"""The calls of speculative generation together, as a program uses them: a cache is compressed, stored in pages, and
generates with drafted trees; the same with plain 64-bit code beside it."""
import numpy as np
import pytest
import torch

from tests import paged_util as U
from tests.test_verify_gpu import walk

pytestmark = pytest.mark.gpu
DEV = U.DEV


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_16213_amd import selkv
    return selkv


class Rows:
    """What the sequences hold, on the host, as stored."""

    def __init__(self, B):
        self.k, self.v, self.b = [None] * B, [None] * B, [None] * B

    def put(self, s, k, v, b):
        cat = lambda a, x: x if a is None else np.concatenate((a, x))
        self.k[s], self.v[s], self.b[s] = cat(self.k[s], k), cat(self.v[s], v), cat(self.b[s], b)


def held(c, b, n):
    k, v, bias = U.entries(c, b, 0, n)
    return k, v, bias


@pytest.mark.parametrize("dtype,layout", [("bf16", "half"), ("fp32", "interleaved")])
@pytest.mark.parametrize("captured", [False, True])
def test_compress_store_generate(S, dtype, layout, captured):
    B, H, G, d, n, vocab, steps, seq = 2, 2, 3, 64, 9, 3000, 6, 700
    g, r = U.gen(51), np.random.default_rng(51)
    dt = U.dtype_of(dtype)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, seq_len=seq, window=16, kv_dtype=dtype)
    K, V, Q = U.rows(g, B, H, seq, d, dtype=dtype), U.rows(g, B, H, seq, d, dtype=dtype), U.rows(g, B, H * G, 16, d, dtype=dtype)
    comp = S.Compressor(p, DEV).run(K, V, Q)
    m = comp.m
    cache = S.PagedCache(p, 40, 9, DEV, page=32)
    order = torch.randperm(40, generator=torch.Generator().manual_seed(3))[:18].view(B, 9)
    cache.table.copy_(order.to(torch.int32))
    comp.store_paged(cache)
    model = Rows(B)
    for b in range(B):
        model.put(b, U.host(comp.K_out[b].transpose(0, 1)), U.host(comp.V_out[b].transpose(0, 1)), U.host(comp.bias[b].t()))
    freq, scale = S.rope_frequencies(d, 10000.0, DEV)
    rope = S.Rope(freq, layout, scale)
    dec = S.TreeDecoder(p, cache, n, vocab)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    lens, counts, pos, parent, tokens = torch.full((B,), m, dtype=torch.int32, device=DEV), i32(B), i32(B, n), i32(B, n), i32(B, n)
    q, k, v = (torch.zeros((B, n, h, d), dtype=dt, device=DEV) for h in (H * G, H, H))
    target, draft = (torch.zeros((B, n, vocab), device=DEV) for _ in range(2))
    u = torch.zeros((B, n), device=DEV)
    out = path = n_path = nxt = None

    def step():
        o = dec.attend(q, k, v, m + steps * n, parent, lens, counts, rope, pos)
        pa, np_, nx = dec.verify(tokens, target, draft, u, parent, counts)
        dec.keep(pa, np_, m + steps * n, lens)
        lens.add_(np_)
        return o, pa, np_, nx

    graph = None
    total = 0
    for t in range(steps):
        parents = [U.tree("tree", n, 10 * t + b) for b in range(B)]
        number = [int(r.integers(1, n + 1)) for _ in range(B)]
        at = [len(model.k[b]) for b in range(B)]
        # positions go on from the text's length, not the compressed cache's
        depth = [[int(U.above(parents[b])[i].sum()) - 1 for i in range(n)] for b in range(B)]
        where = np.array([[seq + at[b] - m + depth[b][i] for i in range(n)] for b in range(B)])
        counts.copy_(torch.tensor(number)); pos.copy_(torch.tensor(where)); parent.copy_(torch.tensor(parents))
        for x in (q, k, v):
            x.copy_(U.rows(g, *x.shape, dtype=dtype))
        x = torch.log(torch.rand((B, n, vocab), generator=g, device=DEV) * vocab + 1.0) * -1.2
        target.copy_(torch.softmax(x, -1))
        draft.copy_(torch.softmax(x + 0.3 * torch.randn(x.shape, generator=g, device=DEV), -1))
        tok = np.zeros((B, n), np.int64)
        dq = U.host(draft)
        for b in range(B):
            for i in range(1, n):
                c = np.cumsum(dq[b, parents[b][i]])
                tok[b, i] = min(np.searchsorted(c, r.random() * c[-1], "right"), vocab - 1)
        tokens.copy_(torch.tensor(tok))
        u.copy_(torch.tensor(r.random((B, n)).astype(np.float32)))
        torch.cuda.synchronize()
        if captured and t == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out, path, n_path, nxt = step()
        if graph is not None:
            graph.replay()
        else:
            out, path, n_path, nxt = step()
        torch.cuda.synchronize()
        uh, th = U.host(u), U.host(target)
        for b in range(B):
            c, L = number[b], at[b]
            ks, ksize = U.turn(U.host(k[b, :c]), where[b, :c], U.host(freq), layout, scale)
            qs, qsize = U.turn(U.host(q[b, :c]), where[b, :c], U.host(freq), layout, scale)
            # the stored rows are the turned ones to their own rounding; attention is checked on the rows as stored
            want, token = walk(tok[b], parents[b], th[b], dq[b], uh[b], c)
            assert path[b].tolist() == want + [-1] * (n - len(want)) and int(nxt[b]) == token, (t, b)
            kept = torch.tensor(want, device=DEV)
            got_k, got_v, got_b = held(cache, b, L + len(want))
            tol = 8 * 2.0 ** -24 * ksize + U.half_step(dtype) * np.abs(ks) * 1.01 + 2.0 ** -40
            assert (np.abs(got_k[L:] - ks[want]) <= tol[want]).all()
            assert np.array_equal(got_v[L:], U.host(v[b, kept])) and (got_b[L:] == 0).all()
            assert np.array_equal(got_k[:L], model.k[b]) and np.array_equal(got_v[:L], model.v[b])
            assert np.array_equal(got_b[:L], model.b[b])
            # attention of the kept nodes: all of their ancestors are kept before them
            see = np.tril(np.ones((len(want),) * 2, bool))
            see = np.concatenate((np.ones((len(want), L), bool), see), 1)
            turned = U.host(dec.q[b, :c])[want] if n == dec.n else None
            ref, size, big = U.attention(turned, got_k, got_v, got_b, see, G, d ** -0.5)
            U.assert_near(U.host(out[b])[want], ref, size, big, L + len(want), dtype, (t, b))
            assert (np.abs(turned - qs[want]) <= (8 * 2.0 ** -24 * qsize + U.half_step(dtype) * np.abs(qs) * 1.01 + 2.0 ** -40)[want]).all()
            model.put(b, got_k[L:], got_v[L:], got_b[L:])
            total += len(want)
        assert lens.tolist() == [len(model.k[b]) for b in range(B)]
    assert total > 2 * steps          # trees are worth something


def test_one_cache_on_two_streams(S):
    """Two sequences of one pool, generated by two decoders on streams of their own at the same time."""
    p = S.params(batch=1, n_heads_kv=4, group=2, head_dim=64, kv_dtype="bf16")
    pool = S.PagedCache(p, 64, 20, DEV, page=32)
    g = U.gen(61)
    caches, decs, streams, lens = [], [], [], []
    for i in range(2):
        table = torch.arange(32 * i, 32 * i + 20, dtype=torch.int32, device=DEV).view(1, 20)
        c = S.PagedCache.over(p, pool.K, pool.V, table, pool.bias)
        rows = U.rows(g, 1, 500, 4, 64, dtype="bf16")
        S.paged_append(p, c, rows, rows, 0)
        caches.append(c); decs.append(S.TreeDecoder(p, c, 5)); streams.append(torch.cuda.Stream()); lens.append(500)
    new = [[(U.rows(g, 1, 5, 8, 64, dtype="bf16"), U.rows(g, 1, 5, 4, 64, dtype="bf16")) for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for t in range(10):
        for i in range(2):
            q, k = new[i][t]
            with torch.cuda.stream(streams[i]):
                outs[i].append(decs[i].attend(q, k, k, 500 + 5 * t).clone())
    torch.cuda.synchronize()
    for i in range(2):
        for t in range(10):
            kk, vv, bb = U.entries(caches[i], 0, 0, 500 + 5 * t + 5)
            see = np.ones((5, 505 + 5 * t), bool)
            see[:, 500 + 5 * t:] = np.tril(np.ones((5, 5), bool))
            ref, size, big = U.attention(U.host(new[i][t][0][0]), kk, vv, bb, see, 2, 0.125)
            U.assert_near(U.host(outs[i][t][0]), ref, size, big, 505 + 5 * t, "bf16", (i, t))


def test_the_decoder_refuses_what_it_was_not_made_for(S):
    p = S.params(batch=1, n_heads_kv=2, group=2, head_dim=64, kv_dtype="bf16")
    c = S.PagedCache(p, 4, 4, DEV, page=16)
    dec = S.TreeDecoder(p, c, 3)
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="made for 3"):
        dec.attend(z(1, 4, 4, 64), z(1, 4, 2, 64), z(1, 4, 2, 64), 0)
    with pytest.raises(ValueError):
        dec.verify(torch.zeros((1, 4), dtype=torch.int32, device=DEV), z(1, 4, 9).float(), None, z(1, 4).float())
