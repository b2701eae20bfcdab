"""GPU: the 8-bit cache against plain 64-bit code: what is written, what is read back, and decode over it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import cache8_util as U

pytestmark = pytest.mark.gpu
DEV, NEG_INF = "cuda", float("-inf")
CODES = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def S():
    from paper_2607_16213_amd import selkv
    return selkv


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def make(S, B, H, G, d, dtype, code, block, cap, seed=1):
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
    c = S.Cache8(p, cap, DEV, code=code, block=block)
    U.fill(c, seed)
    return p, c, U.Model(B, H, d, block, code)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---- write ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,H,d,block", [(1, 2, 64, 16), (2, 3, 128, 16), (1, 5, 64, 32), (2, 1, 128, 32),
                                         (1, 3, 64, 64), (2, 2, 128, 64), (1, 2, 64, 128), (1, 3, 128, 128)])
def test_write_in_pieces(S, B, H, d, block, dtype, code):
    """Pieces of every size hold what one write of all rows holds: the definition, bit for bit."""
    g = gen(d + block)
    pieces = [1, block - 1, 1, block, 2 * block + 5, 3, block - 8, 7 * block, block - 1, 2]
    cap = sum(pieces) + block
    p, c, m = make(S, B, H, 1, d, dtype, code, block, cap)
    n = 0
    for k in pieces:
        K, V = U.rows(g, B, H, k, d, dtype=dtype), U.rows(g, B, H, k, d, dtype=dtype)
        S.cache8_write(p, c, K, V, n)
        n += k
        for b in range(B):
            m.append(b, K[b], V[b])
        U.assert_holds(c, m, f"after {n}")
    p2, c2, _ = make(S, B, H, 1, d, dtype, code, block, cap, seed=2)
    back = lambda x: torch.stack([torch.from_numpy(r) for r in x]).to(DEV, U.dtype_of(dtype)).contiguous()
    S.cache8_write(p2, c2, back(m.k), back(m.v), 0)
    U.assert_holds(c2, m, "one write")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("block", [16, 64, 128])
def test_write_ragged(S, block, code):
    """Lengths and counts of their own, sequences that take no part or get nothing, counts beyond what fits; what lies
    behind the new entries keeps its bytes."""
    B, H, d, n_new = 7, 2, 128, 2 * block + 3
    g = gen(block)
    p, c, m = make(S, B, H, 1, d, "bf16", code, block, 6 * block)
    start = [0, 5, block, block - 1, 2 * block + 7, 6 * block - 4, 3]
    for b in range(B):
        K = U.rows(g, B, H, max(start[b], 1), d, dtype="bf16")
        V = U.rows(g, B, H, max(start[b], 1), d, dtype="bf16")
        only = [0] * B
        only[b] = start[b]
        S.cache8_write(p, c, K, V, c.capacity, i32(*([0] * B)), i32(*only))
        m.append(b, K[b, :, :start[b]], V[b, :, :start[b]])
    U.assert_holds(c, m, "start")
    before = [t.clone() for t in (c.K, c.V, c.k_scale, c.v_scale, c.k_tail, c.v_tail)]
    K, V = U.rows(g, B, H, n_new, d, dtype="bf16"), U.rows(g, B, H, n_new, d, dtype="bf16")
    counts = [n_new, 0, block, 1, n_new + 100, n_new, -3]
    lens = list(start)
    lens[2] = -1                                     # takes no part
    S.cache8_write(p, c, K, V, c.capacity, i32(*lens), i32(*counts))
    got = [max(0, min(k, n_new, c.capacity - n)) for k, n in zip(counts, start)]
    got[2] = 0
    for b in range(B):
        m.append(b, K[b, :, :got[b]], V[b, :, :got[b]])
    U.assert_holds(c, m, "after")
    for b in range(B):
        n0, n1 = start[b], start[b] + got[b]
        lo, hi = n0 // block * block, n1 // block * block     # the codes that the call may change
        for t, x, unit in zip((c.K, c.V, c.k_scale, c.v_scale), before[:4], (1, 16, block, block)):
            bits = torch.uint8 if t.element_size() == 1 else torch.int32      # scales hold NaN where nothing is
            t, x = t.view(bits)[b], x.view(bits)[b]
            assert torch.equal(t[:, :lo // unit], x[:, :lo // unit]), b
            assert torch.equal(t[:, hi // unit:], x[:, hi // unit:]), b
        if lo == hi:                                          # rows of the tail behind the new ones
            for t, x in ((c.k_tail, before[4]), (c.v_tail, before[5])):
                assert torch.equal(t[b, :, n1 % block:].view(torch.int16), x[b, :, n1 % block:].view(torch.int16)), b


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_write_extreme_values(S, dtype, code):
    """Infinities, NaN, zeros, denormals, the type's largest and lowest values: each block by itself."""
    B, H, d, block = 1, 2, 64, 16
    dt = U.dtype_of(dtype)
    p, c, m = make(S, B, H, 1, d, dtype, code, block, 12 * block)
    K = U.rows(gen(3), B, H, 12 * block, d, dtype=dtype)
    V = U.rows(gen(4), B, H, 12 * block, d, dtype=dtype)
    blk = lambda i: (slice(None), slice(None), slice(i * block, (i + 1) * block))
    for X in (K, V):
        X[blk(1)] = 0
        X[0, :, 2 * block + 3, 5] = float("inf")
        X[0, :, 2 * block + 4, 6] = NEG_INF
        X[0, :, 3 * block + 1, 7] = float("nan")
        X[blk(4)] = float("nan")
        X[blk(5)] = float("inf")
        X[blk(6)] *= 2.0 ** -120                      # below the smallest block that is kept
        X[blk(7)] *= 2.0 ** -90
        X[0, :, 8 * block, 0] = torch.finfo(dt).max
        X[0, :, 9 * block, 0] = torch.finfo(dt).min
        X[blk(10)] = torch.finfo(dt).tiny
        X[blk(11)] = 2.0 ** -100
    S.cache8_write(p, c, K, V, 0)
    m.append(0, K[0], V[0])
    U.assert_holds(c, m)
    assert np.isfinite(U.host(c.K)).all() and np.isfinite(U.host(c.V)).all()
    assert torch.isfinite(c.k_scale).all() and torch.isfinite(c.v_scale).all()
    Ko, Vo = torch.empty_like(K), torch.empty_like(V)
    S.cache8_read(p, c, Ko, Vo, 12 * block)
    assert torch.isfinite(Ko).all() and torch.isfinite(Vo).all()
    largest = torch.finfo(dt).max * (1 - 2.0 ** -7)          # within a step of bf16 of where they were
    assert Ko[0, 0, 8 * block, 0] >= largest and Vo[0, 0, 9 * block, 0] <= -largest


@pytest.mark.parametrize("code", CODES)
def test_a_full_sequence_keeps_its_entries(S, code):
    """Steps and writes in a graph-like loop whose bound is capacity - 1: a sequence that has become full is left alone."""
    B, H, G, d, block, cap = 3, 2, 2, 64, 16, 32
    g = gen(2)
    p, c, m = make(S, B, H, G, d, "bf16", code, block, cap)
    K, V = U.rows(g, B, H, cap, d, dtype="bf16"), U.rows(g, B, H, cap, d, dtype="bf16")
    have = [cap, cap - 1, 20]
    S.cache8_write(p, c, K, V, cap, i32(0, 0, 0), i32(*have))
    for b in range(B):
        m.append(b, K[b, :, :have[b]], V[b, :, :have[b]])
    lens, bias, dec = i32(*have), torch.ones((B, H, cap), device=DEV), S.Decoder8(p, c)
    for _ in range(3):
        now = lens.tolist()
        k, v = U.rows(g, B, H, d, dtype="bf16"), U.rows(g, B, H, d, dtype="bf16")
        q = torch.randn((B, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
        out = dec.step(q, k, v, cap - 1, bias, lens)
        for b in range(B):
            if now[b] >= cap:
                assert (out[b] == 0).all()
            else:
                assert (out[b] != 0).any()
                m.append(b, k[b][:, None], v[b][:, None])
        U.assert_holds(c, m, str(now))
        lens += 1
    assert (bias[0] == 1).all()
    before = [t.clone() for t in (c.K, c.V, c.k_tail, c.v_tail)]
    S.cache8_write(p, c, K, V, cap, i32(cap, cap + 1, -1))
    for t, x in zip((c.K, c.V, c.k_tail, c.v_tail), before):
        assert torch.equal(t.view(torch.uint8), x.view(torch.uint8))


# ---- read ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,block", [(64, 16), (128, 32), (128, 64), (64, 128)])
def test_read(S, d, block, dtype, code):
    """Every range: code * scale, rounded to fp32 and then to the storage type, the tail's rows as they are; rows that
    a sequence does not hold stay."""
    B, H, dt = 4, 3, U.dtype_of(dtype)
    g = gen(block)
    cap = 5 * block
    p, c, m = make(S, B, H, 1, d, dtype, code, block, cap)
    lens = [3 * block + 5, 0, block, 5 * block]
    K, V = U.rows(g, B, H, cap, d, dtype=dtype), U.rows(g, B, H, cap, d, dtype=dtype)
    S.cache8_write(p, c, K, V, 0, i32(0, 0, 0, 0), i32(*lens))
    for b in range(B):
        m.append(b, K[b, :, :lens[b]], V[b, :, :lens[b]])
    want = []
    for b in range(B):
        n, k, v = m.blocks(b)
        w = [(torch.from_numpy((q * s.astype(np.float64)[..., None, None]).reshape(H, n * block, d)).float(),
              torch.from_numpy(r[:, n * block:])) for (q, s), r in ((k, m.k[b]), (v, m.v[b]))]
        want.append([torch.cat(x, 1).to(dt) for x in w])
    for first, count in [(0, cap), (3, 1), (block - 1, 2), (17, 2 * block), (cap - 1, 1), (3 * block, block), (1, cap - 1)]:
        Ko = torch.full((B, H, count, d), 7.5, dtype=dt, device=DEV)
        Vo = torch.full_like(Ko, 7.5)
        S.cache8_read(p, c, Ko, Vo, cap, first, i32(lens[0], -1, lens[2], lens[3]))
        for b in range(B):
            for out, w in zip((Ko, Vo), want[b]):
                there = max(0, min(first + count, lens[b]) - first)
                assert torch.equal(out[b, :, :there].cpu(), w[:, first:first + there]), (first, count, b)
                assert (out[b, :, there:] == 7.5).all(), (first, count, b)


# ---- attention -----------------------------------------------------------------------------------------------------

def run_attn(S, p, c, q, bias, n, lens=None, ws=None):
    out = torch.full((p.batch, p.n_heads_kv * p.group, p.head_dim), float("nan"), device=DEV)
    if ws is None:
        ws = torch.randint(0, 256, (max(S.decode8_workspace_bytes(p, c), 1),), dtype=torch.uint8, device=DEV)
    S.decode8_attn(p, c, q, bias, n, out, ws, lens)
    return out


def check_attn(m, out, q, bias, G, d, note, scale=None):
    for b in range(m.B):
        k, v = m.values(b)
        n = k.shape[1]
        bb = None if bias is None else U.host(bias[b, :, :n])
        want, big = U.attention(U.host(q[b]), k, v, bb, G, scale or U.scale_of(d))
        U.assert_near(U.host(out[b]), want, big, f"{note} sequence {b}")


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 130, 191, 200, 255, 256, 300, 512, 777, 1000, 2113]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,G,d,block", [(2, 1, 128, 64), (3, 8, 128, 32), (5, 3, 64, 128), (8, 4, 64, 16), (2, 7, 128, 16),
                                         (1, 5, 64, 64)])
def test_attn_lengths(S, H, G, d, block, dtype, code):
    g = gen(H + d)
    for n in LENGTHS:
        p, c, m = make(S, 1, H, G, d, dtype, code, block, n + 1)
        if n:
            K, V = U.rows(g, 1, H, n, d, dtype=dtype), U.rows(g, 1, H, n, d, dtype=dtype)
            S.cache8_write(p, c, K, V, 0)
            m.append(0, K[0], V[0])
        q = torch.randn((1, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
        bias = torch.rand((1, H, c.capacity), generator=g, device=DEV)
        bias[:, :, n:] = float("nan")                 # behind the cache: not read
        check_attn(m, run_attn(S, p, c, q, bias, n), q, bias, G, d, f"n={n}")
        plain = run_attn(S, p, c, q, None, n)
        check_attn(m, plain, q, None, G, d, f"n={n} no bias")
        zero = run_attn(S, p, c, q, torch.zeros_like(bias), n)
        assert torch.equal(plain, zero), n
        assert torch.equal(plain, run_attn(S, p, c, q, None, n)), n       # deterministic


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("B,H,G,d,block,cap,dtype", [(9, 8, 8, 128, 32, 4096, "bf16"), (5, 32, 1, 64, 64, 1024, "bf16"),
                                                     (40, 8, 4, 128, 128, 640, "bf16"), (3, 2, 6, 128, 16, 3200, "fp32"),
                                                     (64, 16, 2, 64, 16, 160, "fp32")])
def test_attn_ragged_and_masked(S, B, H, G, d, block, cap, dtype, code):
    """Lengths on the device, from none up to the capacity; entries masked by -inf, some rows wholly."""
    g = gen(B)
    p, c, m = make(S, B, H, G, d, dtype, code, block, cap)
    lens = [(i * 7919 + 13) % (cap + 1) for i in range(B)]
    lens[0], lens[1], lens[2] = cap, 0, 1
    K, V = U.rows(g, B, H, cap, d, dtype=dtype), U.rows(g, B, H, cap, d, dtype=dtype)
    S.cache8_write(p, c, K, V, cap, i32(*([0] * B)), i32(*lens))
    for b in range(B):
        m.append(b, K[b, :, :lens[b]], V[b, :, :lens[b]])
    U.assert_holds(c, m)
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
    check_attn(m, run_attn(S, p, c, q, None, cap, i32(*lens)), q, None, G, d, "plain")
    bias = torch.randn((B, H, cap), generator=g, device=DEV)
    bias[torch.rand((B, H, cap), generator=g, device=DEV) < 0.3] = NEG_INF
    bias[0, 0] = NEG_INF
    bias[B // 2] = NEG_INF
    bias[B - 1, :, : lens[B - 1] // 2] = NEG_INF
    check_attn(m, run_attn(S, p, c, q, bias, cap, i32(*lens)), q, bias, G, d, "masked")
    # lengths outside [0, bound]: the sequence takes no part
    lens2 = list(lens)
    lens2[0], lens2[B - 1] = cap + 5, -1
    out = run_attn(S, p, c, q, None, cap, i32(*lens2))
    for b in (0, B - 1):
        assert (out[b] == 0).all()
        m.k[b], m.v[b] = m.k[b][:, :0], m.v[b][:, :0]
    check_attn(m, out, q, None, G, d, "no part")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attn_lowest_bias_and_masked_garbage(S, dtype, code):
    """A bias of the type's lowest value is a number: a row of them averages its values.  Masked entries hold NaN and
    infinities, in whole blocks and in the tail, and change nothing."""
    B, H, G, d, block, n = 2, 2, 3, 128, 32, 32 * 9 + 11
    g = gen(8)
    p, c, m = make(S, B, H, G, d, dtype, code, block, n)
    K, V = U.rows(g, B, H, n, d, dtype=dtype), U.rows(g, B, H, n, d, dtype=dtype)
    S.cache8_write(p, c, K, V, 0)
    for b in range(B):
        m.append(b, K[b], V[b])
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
    low = torch.full((B, H, c.capacity), torch.finfo(torch.float32).min, device=DEV)
    check_attn(m, run_attn(S, p, c, q, low, n), q, low, G, d, "lowest")
    part = torch.randn((B, H, c.capacity), generator=g, device=DEV)
    part[:, :, ::2] = torch.finfo(torch.float32).min
    check_attn(m, run_attn(S, p, c, q, part, n), q, part, G, d, "half lowest")
    bad = torch.zeros(n, dtype=torch.bool)
    bad[[3, 40, 41, 100, n - 1, n - 5]] = True
    bad[64:96] = True
    K2, V2 = K.clone(), V.clone()
    K2[:, :, bad], V2[:, :, bad] = float("nan"), float("inf")
    V2[:, :, 40] = float("nan")
    p2, c2, m2 = make(S, B, H, G, d, dtype, code, block, n)
    S.cache8_write(p2, c2, K2, V2, 0)
    for b in range(B):
        m2.append(b, K2[b], V2[b])
    U.assert_holds(c2, m2)
    bias = torch.zeros((B, H, c.capacity), device=DEV)
    bias[:, :, :n][:, :, bad] = NEG_INF
    check_attn(m2, run_attn(S, p2, c2, q, bias, n), q, bias, G, d, "garbage")


@pytest.mark.parametrize("B,H,G,d,n", [
    (1, 8, 4, 128, 768), (1, 8, 4, 128, 769), (1, 4, 2, 64, 1024), (1, 4, 2, 64, 1025),   # one workgroup a head, and splits
    (1, 1, 2, 64, 20000),                              # more partials than one trip of the combining kernel
    (1, 2, 8, 128, 9000), (4, 6, 1, 64, 2700),
    (32, 8, 1, 64, 3000),                              # a round of workgroups that comes out even
    (33, 8, 2, 64, 300), (96, 8, 3, 64, 1100),         # more heads than CUs: four waves a head, without and with the tail
])
def test_attn_work_division(S, B, H, G, d, n):
    """Both sides of the rules that divide the work, with a step on top."""
    g = gen(n)
    p, c, m = make(S, B, H, G, d, "bf16", "int8", 64, n + 1)
    K, V = U.rows(g, B, H, n, d, dtype="bf16"), U.rows(g, B, H, n, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0)
    some = sorted({0, B // 2, B - 1})                  # sequences that are compared
    keep = U.Model(len(some), H, d, 64, "int8")
    for i, b in enumerate(some):
        keep.append(i, K[b], V[b])
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    bias = torch.rand((B, H, c.capacity), generator=g, device=DEV)
    out = run_attn(S, p, c, q, bias, n)
    check_attn(keep, out[some], q[some], bias[some], G, d, f"n={n}")
    assert torch.equal(out, run_attn(S, p, c, q, bias, n))
    k, v = U.rows(g, B, H, d, dtype="bf16"), U.rows(g, B, H, d, dtype="bf16")
    dec = S.Decoder8(p, c)
    out = dec.step(q, k, v, n, bias)
    for i, b in enumerate(some):
        kk, vv = keep.values(i)
        kk, vv = np.concatenate((kk, U.host(k[b])[:, None]), 1), np.concatenate((vv, U.host(v[b])[:, None]), 1)
        want, big = U.attention(U.host(q[b]), kk, vv, U.host(bias[b, :, :n + 1]), G, U.scale_of(d))
        U.assert_near(U.host(out[b]), want, big, f"step, sequence {b}")


def test_odd_alignment_counts_alone_and_short_reads(S):
    """Biases and scales aligned to an element only, counts without lengths, and a read past what is there."""
    B, H, G, d, block, cap, dtype = 2, 3, 5, 128, 16, 80 * 16, "bf16"
    g = gen(41)
    p, c0, m = make(S, B, H, G, d, dtype, "int8", block, cap)
    off = lambda shape: torch.full((int(np.prod(shape)) + 1,), float("nan"), device=DEV)[1:].view(shape)
    c = S.Cache8.over(p, c0.K, c0.V, off(c0.k_scale.shape), off(c0.v_scale.shape), c0.k_tail, c0.v_tail)
    assert c.k_scale.data_ptr() % 16 == 4
    first = U.rows(g, B, H, 7, d, dtype=dtype), U.rows(g, B, H, 7, d, dtype=dtype)
    S.cache8_write(p, c, *first, 0)
    n = 1000
    K, V = U.rows(g, B, H, n, d, dtype=dtype), U.rows(g, B, H, n, d, dtype=dtype)
    counts = [n, 333]
    S.cache8_write(p, c, K, V, 7, counts=i32(*counts))
    for b in range(B):
        m.append(b, first[0][b], first[1][b])
        m.append(b, K[b, :, :counts[b]], V[b, :, :counts[b]])
    U.assert_holds(c, m)
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    bias = off((B, H, cap)).copy_(torch.randn((B, H, cap), generator=g, device=DEV))
    check_attn(m, run_attn(S, p, c, q, bias, cap, i32(7 + counts[0], 7 + counts[1])), q, bias, G, d, "odd")
    few = run_attn(S, p, c, q, bias, 7 + counts[1])          # the entries that both sequences hold
    m1 = U.Model(1, H, d, block, "int8")
    m1.append(0, first[0][1], first[1][1])
    m1.append(0, K[1, :, :counts[1]], V[1, :, :counts[1]])
    check_attn(m1, few[1:], q[1:], bias[1:], G, d, "few")
    Ko = torch.full((B, H, 50, d), 2.5, dtype=torch.bfloat16, device=DEV)
    Vo = torch.full_like(Ko, 2.5)
    S.cache8_read(p, c, Ko, Vo, 21, 3)
    for got, want in zip((Ko, Vo), m.values(0)):
        assert torch.equal(got[0, :, :13].cpu(), torch.from_numpy(want[:, 3:16]).float().to(torch.bfloat16))
        assert (got[:, :, 18:] == 2.5).all() and (got[:, :, :18] != 2.5).any()


def test_most_heads(S):
    """65535 KV heads, the most of one call: write, read, decode and a step that completes every block."""
    B, H, G, d, block, n = 21845, 3, 2, 64, 16, 31
    g = gen(6)
    p, c, _ = make(S, B, H, G, d, "bf16", "int8", block, 32)
    K, V = U.rows(g, B, H, n, d, dtype="bf16"), U.rows(g, B, H, n, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0)
    some = [0, 10000, B - 1]
    m = U.Model(len(some), H, d, block, "int8")
    for i, b in enumerate(some):
        m.append(i, K[b], V[b])
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    check_attn(m, run_attn(S, p, c, q, None, n)[some], q[some], None, G, d, "most heads")
    k, v = U.rows(g, B, H, d, dtype="bf16"), U.rows(g, B, H, d, dtype="bf16")
    S.Decoder8(p, c).step(q, k, v, n)
    Ko, Vo = (torch.empty((B, H, 32, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    S.cache8_read(p, c, Ko, Vo, 32)
    for i, b in enumerate(some):
        m.append(i, k[b][:, None], v[b][:, None])
        for got, want in zip((Ko[b], Vo[b]), m.values(i)):
            assert torch.equal(got.cpu(), torch.from_numpy(want).float().to(torch.bfloat16)), b


def test_write_and_read_in_a_replayed_graph(S):
    """A chunk appended and read back in a captured graph, lengths and counts on the device and changed between replays."""
    B, H, d, block, cap, n = 3, 2, 128, 32, 320, 40
    g = gen(14)
    p, c, m = make(S, B, H, 1, d, "fp32", "e4m3", block, cap)
    K, V = (torch.zeros((B, H, n, d), device=DEV) for _ in range(2))
    Ko, Vo = (torch.zeros((B, H, cap, d), device=DEV) for _ in range(2))
    lens, counts = i32(0, 0, 0), i32(0, 0, 0)

    def chunk():
        S.cache8_write(p, c, K, V, cap, lens, counts)
        lens.add_(counts)
        S.cache8_read(p, c, Ko, Vo, cap, 0, lens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chunk()                                    # nothing: the counts are 0
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chunk()
    for i in range(7):
        K.copy_(U.rows(g, B, H, n, d, dtype="fp32"))
        V.copy_(U.rows(g, B, H, n, d, dtype="fp32"))
        take = [n, (i * 17) % (n + 1), i % 2]
        counts.copy_(i32(*take))
        chunk() if i == 3 else graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            m.append(b, K[b, :, :take[b]], V[b, :, :take[b]])
        U.assert_holds(c, m, f"replay {i}")
        for b in range(B):
            for got, want in zip((Ko, Vo), m.values(b)):
                assert torch.equal(got[b, :, :want.shape[1]].cpu(), torch.from_numpy(want).float()), (i, b)


def test_attn_lengths_far_below_the_bound(S):
    """A bound of the whole capacity and short sequences: their slots are cut from their own lengths."""
    B, H, G, d, cap = 5, 2, 4, 128, 64 * 400
    g = gen(55)
    p, c, m = make(S, B, H, G, d, "bf16", "e4m3", 64, cap)
    lens = [5, 300, 2000, 0, 9000]
    K, V = U.rows(g, B, H, 9000, d, dtype="bf16"), U.rows(g, B, H, 9000, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0, i32(*([0] * B)), i32(*lens))
    for b in range(B):
        m.append(b, K[b, :, :lens[b]], V[b, :, :lens[b]])
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    check_attn(m, run_attn(S, p, c, q, None, cap, i32(*lens)), q, None, G, d, "short")
    uniform = run_attn(S, p, c, q, None, 5)            # the same number for all: only what every sequence holds
    tail = c.k_tail[0, :, :5]
    out0, big = U.attention(U.host(q[0]), U.host(tail).astype(np.float64), U.host(c.v_tail[0, :, :5]).astype(np.float64),
                            None, G, U.scale_of(d))
    U.assert_near(U.host(uniform[0]), out0, big, "uniform")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [20, 300, 3000])
def test_attn_nan_reaches_the_outputs(S, n, dtype):
    """A NaN that counts is not lost: of a query its head's outputs, of a tail key all outputs, of a tail value its
    channel.  (Where nothing counts the outputs are 0.)"""
    H, G, d, block = 2, 3, 128, 64
    g = gen(n)
    p, c, m = make(S, 1, H, G, d, dtype, "int8", block, n)
    K, V = U.rows(g, 1, H, n, d, dtype=dtype), U.rows(g, 1, H, n, d, dtype=dtype)
    S.cache8_write(p, c, K, V, 0)
    q = torch.randn((1, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
    good = run_attn(S, p, c, q, None, n)
    q[0, 1, 5] = float("nan")
    out = run_attn(S, p, c, q, None, n)
    assert torch.isnan(out[0, 1]).all()
    keep = [0, 2, 3, 4, 5]
    assert torch.equal(out[0, keep], good[0, keep])
    q[0, 1, 5] = 1.0
    good = run_attn(S, p, c, q, None, n)
    c.v_tail[0, 0, n % block - 1, 7] = float("nan")
    out = run_attn(S, p, c, q, None, n)
    assert torch.isnan(out[0, :G, 7]).all() and torch.isnan(out).sum() == G
    assert torch.equal(out[0, G:], good[0, G:])
    c.k_tail[0, 1, n % block - 1, 0] = float("nan")
    out = run_attn(S, p, c, q, None, n)
    assert torch.isnan(out[0, G:]).all() and not torch.isnan(out[0, :G, 8:]).any()
    bias = torch.full((1, H, c.capacity), NEG_INF, device=DEV)
    assert (run_attn(S, p, c, q, bias, n) == 0).all()
    bias[0, 1, 3] = float("nan")
    out = run_attn(S, p, c, q, bias, n)
    assert (out[0, :G] == 0).all() and torch.isnan(out[0, G:]).all()


def test_two_streams_on_one_cache(S):
    """Two decodes over the same cache at once, each with a workspace of its own, give what one alone gives."""
    H, G, d, n = 8, 4, 128, 6000
    g = gen(12)
    p, c, m = make(S, 1, H, G, d, "bf16", "int8", 64, n)
    K, V = U.rows(g, 1, H, n, d, dtype="bf16"), U.rows(g, 1, H, n, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0)
    qs = [torch.randn((1, H * G, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    alone = [run_attn(S, p, c, q, None, n) for q in qs]
    streams, wss = [torch.cuda.Stream() for _ in range(2)], [S.decode8_workspace(p, c) for _ in range(2)]
    outs = [torch.zeros_like(alone[0]) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, st, ws, out in zip(qs, streams, wss, outs):
            S.decode8_attn(p, c, q, None, n, out, ws, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)


def test_attn_scale_and_long_logits(S):
    """A scale of its own, and logits far apart (one entry takes all the weight)."""
    H, G, d, block, n = 4, 4, 128, 64, 5000
    g = gen(21)
    p, c, m = make(S, 1, H, G, d, "bf16", "int8", block, n)
    K, V = U.rows(g, 1, H, n, d, dtype="bf16"), U.rows(g, 1, H, n, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0)
    m.append(0, K[0], V[0])
    q = torch.randn((1, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    for scale in (0.013, 1.0):
        p.scale = scale
        check_attn(m, run_attn(S, p, c, q, None, n), q, None, G, d, f"scale {scale}", scale=np.float32(scale).item())


def test_attn_offsets_beyond_32_bits(S):
    """Two heads of 2^26 entries: codes, biases and scales at byte offsets past 4 GiB."""
    H, G, d, block, cap, n = 2, 2, 64, 128, 1 << 26, 300
    g = gen(5)
    p = S.params(batch=1, n_heads_kv=H, group=G, head_dim=d, kv_dtype="bf16")
    c = S.Cache8(p, cap, DEV, block=block)
    K, V = U.rows(g, 1, H, n, d, dtype="bf16"), U.rows(g, 1, H, n, d, dtype="bf16")
    at = cap - 384                                        # 2 blocks and a part of a third
    S.cache8_write(p, c, K, V, at)
    m = U.Model(1, H, d, block, "int8")
    m.append(0, K[0], V[0])
    q = torch.randn((1, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    bias = torch.full((1, H, cap), NEG_INF, device=DEV)
    bias[:, :, at:] = torch.randn((1, H, cap - at), generator=g, device=DEV)
    out = run_attn(S, p, c, q, bias, at + n)
    check_attn(m, out, q, bias[:, :, at:], G, d, "past 4 GiB")
    Ko, Vo = torch.empty_like(K), torch.empty_like(V)
    S.cache8_read(p, c, Ko, Vo, at + n, at)
    for got, want in zip((Ko, Vo), m.values(0)):
        assert torch.equal(got[0].cpu(), torch.from_numpy(want).float().to(torch.bfloat16))


# ---- generation steps ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("H,G,d,block,dtype,start", [(2, 4, 128, 16, "bf16", 0), (3, 1, 64, 32, "fp32", 61),
                                                     (8, 4, 128, 64, "bf16", 1020), (2, 8, 64, 128, "bf16", 120),
                                                     (1, 2, 128, 16, "fp32", 2040)])
def test_steps(S, H, G, d, block, dtype, start, code):
    """Steps through the ends of two blocks: each attends over what is there with the new row, and leaves the cache as
    a write leaves it."""
    g = gen(start + d)
    steps = block + 20
    p, c, m = make(S, 1, H, G, d, dtype, code, block, start + steps)
    bias = torch.rand((1, H, c.capacity), generator=g, device=DEV)
    if start:
        K, V = U.rows(g, 1, H, start, d, dtype=dtype), U.rows(g, 1, H, start, d, dtype=dtype)
        S.cache8_write(p, c, K, V, 0)
        m.append(0, K[0], V[0])
    dec = S.Decoder8(p, c)
    for i in range(steps):
        n = start + i
        k, v = U.rows(g, 1, H, d, dtype=dtype), U.rows(g, 1, H, d, dtype=dtype)
        q = torch.randn((1, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
        want_bias = bias.clone()
        want_bias[:, :, n] = 0
        out = dec.step(q, k, v, n, bias)
        assert torch.equal(bias, want_bias), n
        # the rows of the open block, the new one among them, are attended to as given
        kk, vv = m.values(0)
        kk, vv = np.concatenate((kk, U.host(k[0])[:, None]), 1), np.concatenate((vv, U.host(v[0])[:, None]), 1)
        want, big = U.attention(U.host(q[0]), kk, vv, U.host(bias[0, :, :n + 1]), G, U.scale_of(d))
        U.assert_near(U.host(out[0]), want, big, f"step at {n}")
        m.append(0, k[0][:, None], v[0][:, None])
        if i % 8 == 0 or (n + 1) % block < 2:
            U.assert_holds(c, m, f"step at {n}")
    U.assert_holds(c, m, "end")


def test_ragged_steps_in_a_replayed_graph(S):
    """A captured step with the lengths on the device, which the graph advances: replays, eager steps between them, and
    a sequence that takes no part."""
    B, H, G, d, block, cap = 4, 2, 4, 128, 16, 256
    g = gen(77)
    p, c, m = make(S, B, H, G, d, "bf16", "int8", block, cap)
    start = [30, 0, 100, 15]
    K, V = U.rows(g, B, H, 100, d, dtype="bf16"), U.rows(g, B, H, 100, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0, i32(0, 0, 0, 0), i32(*start))
    for b in range(B):
        m.append(b, K[b, :, :start[b]], V[b, :, :start[b]])
    idle = 2
    bias = torch.rand((B, H, cap), generator=g, device=DEV)
    lens = i32(*start)
    lens[idle] = -1000
    q = torch.zeros((B, H * G, d), dtype=torch.bfloat16, device=DEV)
    k, v = (torch.zeros((B, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dec = S.Decoder8(p, c)
    one = i32(1, 1, 1, 1)

    def step():
        dec.step(q, k, v, cap - 1, bias, lens)
        lens.add_(one)

    def check(note):
        nonlocal_lens = lens.clone()
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        k.copy_(U.rows(g, B, H, d, dtype="bf16"))
        v.copy_(U.rows(g, B, H, d, dtype="bf16"))
        bias_before = bias.clone()
        yield
        torch.cuda.synchronize()
        for b in range(B):
            if b == idle:
                assert (dec.out[b] == 0).all() and torch.equal(bias[b], bias_before[b]), note
                continue
            n = int(nonlocal_lens[b])
            assert n == m.k[b].shape[1]
            kk, vv = m.values(b)
            kk = np.concatenate((kk, U.host(k[b])[:, None]), 1)
            vv = np.concatenate((vv, U.host(v[b])[:, None]), 1)
            want, big = U.attention(U.host(q[b]), kk, vv, U.host(bias[b, :, :n + 1]), G, U.scale_of(d))
            U.assert_near(U.host(dec.out[b]), want, big, f"{note} sequence {b}")
            m.append(b, k[b][:, None], v[b][:, None])
        U.assert_holds(c, m, note)
        yield

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t = check("warm up")
        next(t)
        step()
        next(t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(24):
        t = check(f"step {i}")
        next(t)
        if i % 5 == 3:
            step()
        else:
            graph.replay()
        next(t)


def test_given_stream(S):
    """A call on a stream of its own, behind work of that stream."""
    H, G, d, n = 4, 2, 64, 1500
    g = gen(31)
    p, c, m = make(S, 1, H, G, d, "bf16", "e4m3", 64, n + 1)
    K, V = U.rows(g, 1, H, n, d, dtype="bf16"), U.rows(g, 1, H, n, d, dtype="bf16")
    m.append(0, K[0], V[0])
    q = torch.randn((1, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
    K0, V0 = torch.zeros_like(K), torch.zeros_like(V)
    out, Ko, Vo = torch.zeros((1, H * G, d), device=DEV), torch.zeros_like(K), torch.zeros_like(V)
    ws = S.decode8_workspace(p, c)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        K0.copy_(K)
        V0.copy_(V)
    S.cache8_write(p, c, K0, V0, 0, stream=st)
    S.decode8_attn(p, c, q, None, n, out, ws, stream=st)
    S.cache8_read(p, c, Ko, Vo, n, stream=st)
    st.synchronize()
    check_attn(m, out, q, None, G, d, "stream")
    for got, want in zip((Ko, Vo), m.values(0)):
        assert torch.equal(got[0].cpu(), torch.from_numpy(want).float().to(torch.bfloat16))


# ---- together ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("code", CODES)
def test_compress_store_generate_and_compress_again(S, code):
    """The path of a serving loop: compress a prompt, keep it in 8 bits, generate over it, read it back and compress it
    once more.  The decode is compared with the same decode over the unquantised compressed cache, too: with codes a
    half step of 1/127 or 2^-4 from their rows, the attention output is off by a few hundredths at most."""
    from paper_2607_16213_amd import synth
    w = synth.WORKLOADS["llama_layer"].replace(seq_len=2048)
    t = synth.make_layer(w, 0, DEV)
    H, G, d = w.n_heads_kv, w.group, w.head_dim
    p = S.params(batch=1, n_heads_kv=H, group=G, head_dim=d, seq_len=w.seq_len, window=w.window, kv_dtype="bf16")
    comp = S.Compressor(p, DEV).run(t["K"], t["V"], t["Qwin"])
    steps, mlen = 70, comp.m
    cache = S.Cache8(p, mlen + steps, DEV, code=code)
    bias = torch.zeros((1, H, cache.capacity), device=DEV)
    comp.store8(cache, bias)
    m = U.Model(1, H, d, cache.block, code)
    m.append(0, comp.K_out[0], comp.V_out[0])
    U.assert_holds(cache, m, "stored")
    assert torch.equal(bias[:, :, :mlen], comp.bias)
    dec = S.Decoder8(p, cache)
    full = S.Decoder(p, mlen, DEV)
    g = gen(9)
    q = synth.make_decode_queries(w, 0, 1, DEV)[0]
    near = dec.run(q, mlen, bias)
    check_attn(m, near, q, bias, G, d, "decode")
    plain = full.run(q, comp.K_out, comp.V_out, comp.bias)
    assert ((near - plain).norm() / plain.norm()).item() < (0.05 if code == "int8" else 0.3)
    for i in range(steps):
        k, v = U.rows(g, 1, H, d, dtype="bf16"), U.rows(g, 1, H, d, dtype="bf16")
        q = torch.randn((1, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
        dec.step(q, k, v, mlen + i, bias)
        m.append(0, k[0][:, None], v[0][:, None])
    U.assert_holds(cache, m, "generated")
    n = mlen + steps
    check_attn(m, dec.run(q, n, bias), q, bias, G, d, "after")
    K2, V2 = (torch.empty((1, H, n, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    S.cache8_read(p, cache, K2, V2, n)
    p2 = S.params(batch=1, n_heads_kv=H, group=G, head_dim=d, seq_len=n, window=w.window, kv_dtype="bf16")
    again = S.Compressor(p2, DEV).run(K2, V2, t["Qwin"])
    kept = again.kept.long()
    rows = K2.gather(2, kept[..., None].expand(-1, -1, -1, d))
    assert torch.equal(again.K_out, rows)


def test_refusals_with_device_tensors(S):
    p, c, _ = make(S, 2, 2, 2, 64, "bf16", "int8", 16, 64)
    bf = dict(dtype=torch.bfloat16, device=DEV)
    new, q = torch.zeros((2, 2, 5, 64), **bf), torch.zeros((2, 4, 64), **bf)
    out, ws = torch.zeros((2, 4, 64), device=DEV), S.decode8_workspace(p, c)
    with pytest.raises(ValueError, match="shape"):
        S.cache8_write(p, c, new, new[:, :, :4].contiguous(), 0)
    with pytest.raises(ValueError, match="contiguous"):
        S.cache8_write(p, c, new, new.transpose(0, 1), 0)
    with pytest.raises(ValueError, match="dtype"):
        S.cache8_write(p, c, new.float(), new.float(), 0)
    with pytest.raises(ValueError, match="device"):
        S.cache8_write(p, c, new.cpu(), new, 0)
    with pytest.raises(ValueError, match="lens"):
        S.cache8_write(p, c, new, new, 0, lens=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError, match="counts"):
        S.cache8_write(p, c, new, new, 0, counts=torch.zeros(3, dtype=torch.int32, device=DEV))
    with pytest.raises(S.SelkvError, match="EINVAL"):
        S.cache8_write(p, c, new, new, 60)
    with pytest.raises(ValueError, match="bias"):
        S.decode8_attn(p, c, q, torch.zeros((2, 2, 60), device=DEV), 10, out, ws)
    with pytest.raises(ValueError, match="workspace"):
        S.decode8_attn(p, c, q, None, 10, out, ws.cpu())
    with pytest.raises(ValueError, match="out has"):
        S.decode8_attn(p, c, q, None, 10, out.half(), ws)
    with pytest.raises(ValueError, match="was made for"):
        S.decode8_attn(S.params(batch=1, n_heads_kv=2, group=2, head_dim=64), c, q, None, 10, out, ws)
    with pytest.raises(S.SelkvError, match="EINVAL"):
        S.decode8_append(p, c, q, new[:, :, 0].contiguous(), new[:, :, 0].contiguous(), None, 64, out, ws)
    S.cache8_write(p, c, new[:, :, :0].contiguous(), new[:, :, :0].contiguous(), 0)      # nothing to write
