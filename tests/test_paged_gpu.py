"""selkv_paged_append and selkv_paged_keep against plain 64-bit code."""
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


def snapshot(c):
    return [None if t is None else t.clone() for t in (c.K, c.V, c.bias)]


def same(a, b):
    return a is b is None or torch.equal(a.view(torch.int32), b.view(torch.int32))


def check_append(S, B, H, G, d, dtype, page, lens, n, counts=None, layout=None, rot=None, positions=None, bias=True,
                 new_bias=True, queries=True, head_major=False, seed=0, cache_len=None, columns=None, scale=1.25):
    """One call against the definition: the rows that it stores, and nothing else changed."""
    g = U.gen(seed)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
    c = U.make_cache(S, p, lens, n, page, g, dtype, bias, columns=columns)
    if head_major:
        k, v, q = (U.rows(g, B, h, n, d, dtype=dtype).transpose(1, 2) for h in (H, H, H * G))
    else:
        wide = U.rows(g, B, n, H * (G + 2), d, dtype=dtype)
        q, k, v = wide[:, :, :H * G], wide[:, :, H * G:H * (G + 1)], wide[:, :, H * (G + 1):]
    bn = torch.randn((B, H, n), generator=g, device=DEV) if bias and new_bias else None
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    rope = q_out = None
    if layout:
        freq, _ = S.rope_frequencies(rot, 10000.0, DEV)
        rope = S.Rope(freq, layout, scale)
        if queries:
            q_out = torch.full((B, n, H * G, d), float("nan"), device=DEV).to(U.dtype_of(dtype))
    before = snapshot(c)
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
    uniform = len(set(lens)) == 1 and cache_len is None and counts is None
    S.paged_append(p, c, k, v, lens[0] if uniform else max(lens) if cache_len is None else cache_len,
                   lens=None if uniform else i32(lens), counts=i32(counts), bias_new=bn, rope=rope, positions=pos,
                   q=q if q_out is not None else None, q_out=q_out)
    torch.cuda.synchronize()
    top = max(lens) if cache_len is None else cache_len
    want = before
    for b in range(B):
        m = n if counts is None else counts[b]
        if not (0 <= lens[b] <= top and 0 <= m <= n):
            m = 0
        stored = [i for i in range(m) if (lens[b] + i) // page < c.columns and 0 <= int(c.table[b, (lens[b] + i) // page]) < c.n_pages]
        if m and layout:
            at = np.array(positions[b][:m]) if positions is not None else lens[b] + np.arange(m)
            for x, y in ((k, None), (q, q_out)):
                if x is q and q_out is None:
                    continue
                ref, size = U.turn(U.host(x[b, :m]), at, U.host(freq), layout, float(np.float32(scale)))
                # products and a sum in fp32 with sine and cosine a few steps off, the angle's two roundings of 2^-53,
                # and the rounding to the type
                tol = (8 * 2.0 ** -24 + 2.0 ** -52 * np.abs(at).max()) * size + U.half_step(dtype) * np.abs(ref) * 1.01
                if y is None:
                    got = np.zeros_like(ref)
                    if stored:
                        pg, row = U.places(c, b, lens[b], max(stored) + 1)
                        got[:max(stored) + 1] = U.host(c.K[pg.clamp(min=0), :, row])
                    rows_ = np.array(stored, int)
                else:
                    got, rows_ = U.host(y[b, :m]), np.arange(m)
                err = np.abs(got - ref)[rows_]
                assert (err <= tol[rows_]).all(), (b, (err / np.maximum(tol[rows_], 1e-300)).max())
                rest = ref.shape[-1] - rot
                if rest:
                    assert np.array_equal(got[rows_][..., rot:], U.host(x[b, :m])[rows_][..., rot:])
        if q_out is not None:
            assert bool(torch.isnan(q_out[b, m:]).all())
        for i in stored:
            pg, row = int(c.table[b, (lens[b] + i) // page]), (lens[b] + i) % page
            want[0][pg, :, row] = c.K[pg, :, row] if layout else k[b, i]
            want[1][pg, :, row] = v[b, i]
            if bias:
                want[2][pg, :, row] = bn[b, :, i] if bn is not None else 0.0
    for x, y in zip((c.K, c.V, c.bias), want):
        assert same(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", [None, "half", "interleaved"])
def test_append_prompt_and_token(S, dtype, d, layout):
    for n, lens in ((1, [0]), (1, [63]), (1, [64]), (77, [0]), (130, [50])):
        check_append(S, 1, 2, 3, d, dtype, 64, lens, n, layout=layout, rot=d)


@pytest.mark.parametrize("layout,rot", [("half", 16), ("half", 48), ("interleaved", 16), ("interleaved", 80), ("half", 112)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_turns_part_of_the_head(S, dtype, layout, rot):
    check_append(S, 2, 3, 2, 128, dtype, 16, [33, 33], 19, layout=layout, rot=rot)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("bias,new_bias", [(True, True), (True, False), (False, False)])
def test_append_pages_and_biases(S, page, bias, new_bias):
    check_append(S, 3, 2, 1, 64, "bf16", page, [0, 5, 300], 70, counts=[70, 69, 1], bias=bias, new_bias=new_bias, queries=False)


def test_append_ragged(S):
    """Sequences of their own lengths and counts; some that take no part; rows that do not fit."""
    check_append(S, 6, 2, 2, 64, "fp32", 16, [0, 40, 17, 9, 16, 40], 21, counts=[21, 0, 1, 20, -1, 22], layout="half", rot=64)
    check_append(S, 4, 2, 2, 64, "bf16", 16, [30, -1, 41, 3], 21, counts=[21, 4, 4, 4], layout="interleaved", rot=32, cache_len=40)
    check_append(S, 3, 2, 2, 64, "bf16", 16, [30, 40, 47], 21, layout="half", rot=32, columns=3, cache_len=48)


def test_append_without_a_page(S):
    """Rows for a column that is no page are not stored; their queries are turned all the same."""
    g = U.gen(3)
    p = S.params(batch=1, n_heads_kv=2, group=2, head_dim=64, kv_dtype="bf16")
    for bad in (-1, 5, 1 << 30, -(1 << 31)):
        c = S.PagedCache(p, 5, 4, DEV, page=16)
        c.table.copy_(torch.tensor([[2, bad, 0, 4]], dtype=torch.int32))
        k = U.rows(g, 1, 64, 2, 64, dtype="bf16")
        S.paged_append(p, c, k, k, 0)
        for j, pg in ((0, 2), (2, 0), (3, 4)):
            assert torch.equal(c.K[pg].transpose(0, 1), k[0, 16 * j:16 * j + 16])
        assert bool((c.K[[1, 3]] == 0).all()) and bool((c.V[[1, 3]] == 0).all())


def test_append_positions(S):
    """Given positions, far ones and negative ones too."""
    for at in ([7, 7, 0, 100000, 2 ** 20, 12345678], [2 ** 31 - 1, -3, -100000, 1, 2, 3]):
        check_append(S, 1, 2, 2, 128, "fp32", 64, [10], 6, layout="half", rot=128, positions=[at])
        check_append(S, 1, 2, 2, 64, "bf16", 64, [10], 6, layout="interleaved", rot=64, positions=[at])


def test_append_many_heads_and_head_major_rows(S):
    check_append(S, 2, 8, 8, 128, "bf16", 64, [100, 100], 37, layout="half", rot=128)
    check_append(S, 2, 32, 1, 64, "bf16", 64, [100, 100], 9, layout="half", rot=64, head_major=True)
    check_append(S, 2, 1, 64, 64, "fp32", 64, [0, 0], 9, layout="interleaved", rot=64, head_major=True)
    check_append(S, 1, 8, 4, 128, "bf16", 64, [0], 1111, queries=False, head_major=True)


def test_append_broadcast_rows_and_queries_in_place(S):
    g = U.gen(4)
    p = S.params(batch=3, n_heads_kv=2, group=2, head_dim=64, kv_dtype="fp32")
    c = U.make_cache(S, p, [9, 9, 9], 5, 16, g, "fp32")
    one = U.rows(g, 1, 1, 2, 64, dtype="fp32").expand(3, 5, 2, 64)
    q = U.rows(g, 3, 5, 4, 64, dtype="fp32")
    freq, scale = S.rope_frequencies(64, 500000.0, DEV, "yarn", 8.0, original_len=8192)
    rope, apart = S.Rope(freq, "half", scale), torch.empty_like(q)
    S.paged_append(p, c, one, one, 9, rope=rope, q=q, q_out=apart)
    S.paged_append(p, c, one, one, 9, rope=rope, q=q, q_out=q)
    assert torch.equal(q, apart)
    pg, row = U.places(c, 1, 9, 5)
    assert torch.equal(c.V[pg, :, row], one[1])


def test_append_past_4_gib(S):
    """Pages whose offsets need more than 32 bits."""
    p = S.params(batch=1, n_heads_kv=8, group=1, head_dim=128, kv_dtype="bf16")
    c = S.PagedCache(p, 34000, 3, DEV, page=64)     # 4.4 GB each of K and V
    c.table.copy_(torch.tensor([[33999, 0, 33000]], dtype=torch.int32))
    g = U.gen(5)
    k, v = U.rows(g, 1, 150, 8, 128, dtype="bf16"), U.rows(g, 1, 150, 8, 128, dtype="bf16")
    S.paged_append(p, c, k, v, 0)
    pg, row = U.places(c, 0, 0, 150)
    assert torch.equal(c.K[pg, :, row], k[0]) and torch.equal(c.V[pg, :, row], v[0])
    path = torch.tensor([[0, 2, 60]], dtype=torch.int32, device=DEV)
    S.paged_keep(p, c, path, torch.tensor([3], dtype=torch.int32, device=DEV), 60)
    pg, row = U.places(c, 0, 0, 150)
    want = v[0].clone()
    want[60:63] = v[0, [60, 62, 120]]
    # node 60 is outside a tree of three nodes: its row stays
    want[62] = v[0, 62]
    assert torch.equal(c.V[pg, :, row], want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("bias", [True, False])
def test_keep(S, dtype, d, page, bias):
    """Paths of every kind: nothing to move, chains with gaps, full trees, ones that are no path, repeated nodes."""
    n = 64
    paths = [[0], [0, 1, 2], [0, 5], [0, 2, 3, 63], list(range(64)), [1] + [0] + list(range(63, 1, -1)), [0, 9, 9, 9], [],
             [3, -1, 64, 2, 1 << 30], [0, 7, 8]]
    number = [len(x) for x in paths]
    number[-1], lens = 65, [0, 15, 16, 40, 7, 100, 31, 3, 12, 5]
    B = len(paths)
    p = S.params(batch=B, n_heads_kv=3, group=1, head_dim=d, kv_dtype=dtype)
    c = U.make_cache(S, p, [x + n for x in lens], 0, page, U.gen(6), dtype, bias)
    want = snapshot(c)
    for b in range(B):
        if number[b] > n:
            continue
        src = [(j, x) for j, x in enumerate(paths[b]) if 0 <= x < n]
        old = [U.places(c, b, lens[b], n)]
        pg, row = old[0]
        for x, w in zip((c.K, c.V, c.bias), want):
            if x is not None and src:
                j, i = (torch.tensor(t, device=DEV) for t in zip(*src))
                w[pg[j], :, row[j]] = x[pg[i], :, row[i]]
    path = torch.full((B, n), 1, dtype=torch.int32)
    for b in range(B):
        path[b, :len(paths[b])] = torch.tensor(paths[b], dtype=torch.int32)
    S.paged_keep(p, c, path.to(DEV), torch.tensor(number, dtype=torch.int32, device=DEV), max(lens),
                 torch.tensor(lens, dtype=torch.int32, device=DEV))
    for x, w in zip((c.K, c.V, c.bias), want):
        assert same(x, w)


def test_keep_without_pages_and_out_of_range(S):
    p = S.params(batch=3, n_heads_kv=2, group=1, head_dim=64, kv_dtype="fp32")
    c = S.PagedCache(p, 6, 2, DEV, page=16)
    c.K.normal_(); c.V.normal_(); c.bias.normal_()
    c.table.copy_(torch.tensor([[0, -1], [6, 2], [3, 4]], dtype=torch.int32))
    before = snapshot(c)
    path = torch.tensor([[0, 10, 11]] * 3, dtype=torch.int32, device=DEV)
    # the first's source is on no page, the second's target is on none, the third is longer than the bound
    S.paged_keep(p, c, path, torch.tensor([3, 3, 3], dtype=torch.int32, device=DEV), 13,
                 torch.tensor([13, 13, 14], dtype=torch.int32, device=DEV))
    for x, w in zip((c.K, c.V, c.bias), before):
        assert same(x, w)


def test_refusals_on_a_gpu(S):
    p = S.params(batch=2, n_heads_kv=2, group=2, head_dim=64, kv_dtype="bf16")
    c = S.PagedCache(p, 8, 4, DEV, page=16, bias=False)
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device=DEV)
    k = z(2, 5, 2, 64)
    rope = S.Rope(S.rope_frequencies(64, 1e4, DEV)[0])
    with pytest.raises(ValueError, match="channels"):
        S.paged_append(p, c, z(2, 5, 64, 2).transpose(2, 3), k, 0)
    with pytest.raises(ValueError, match="16 bytes"):
        S.paged_append(p, c, z(2, 5, 2, 68)[..., :64], k, 0)
    with pytest.raises(S.SelkvError, match="EALIGN"):
        S.paged_append(p, c, z(2 * 5 * 2 * 64 + 4)[4:].view(2, 5, 2, 64), k, 0)
    with pytest.raises(ValueError, match="shape"):
        S.paged_append(p, c, k, z(2, 4, 2, 64), 0)
    with pytest.raises(ValueError, match="dtype"):
        S.paged_append(p, c, k.float(), k, 0)
    with pytest.raises(ValueError, match="rope and q_out"):
        S.paged_append(p, c, k, k, 0, q=z(2, 5, 4, 64))
    with pytest.raises(S.SelkvError, match="EINVAL"):          # no biases in the cache
        S.paged_append(p, c, k, k, 0, bias_new=z(2, 2, 5, t=torch.float32))
    with pytest.raises(S.SelkvError, match="EINVAL"):          # no room
        S.paged_append(p, c, k, k, 60)
    with pytest.raises(ValueError, match="positions"):
        S.paged_append(p, c, k, k, 0, rope=rope, positions=z(2, 5, t=torch.int64))
    with pytest.raises(ValueError, match="was made for"):
        S.paged_append(S.params(batch=2, n_heads_kv=2, group=2, head_dim=64, kv_dtype="fp32"), c, k.float(), k.float(), 0)
    with pytest.raises(KeyError):
        S.Rope(S.rope_frequencies(64, 1e4, DEV)[0], "spiral")
    with pytest.raises(ValueError, match="float64"):
        S.Rope(torch.ones(32, device=DEV))
    S.paged_append(p, c, k[:, :0], k[:, :0], 64)               # nothing to do
    with pytest.raises(ValueError, match="n_path"):
        S.paged_keep(p, c, z(2, 3, t=torch.int32), z(3, t=torch.int32), 0)
