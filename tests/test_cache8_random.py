"""GPU: randomly drawn 8-bit caches through a random run of calls, every call checked against plain 64-bit code."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import cache8_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("seed", range(24))
def test_random_calls(seed):
    from paper_2607_16213_amd import selkv as S
    r = random.Random(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, H, G = r.randint(1, 6), r.randint(1, 4), r.randint(1, 8)
    d, block, dtype, code = r.choice([64, 128]), r.choice([16, 32, 64, 128]), r.choice(["bf16", "fp32"]), \
        r.choice(["int8", "e4m3"])
    cap = block * r.randint(1, max(2, r.choice([300, 2500]) // block))
    dt = U.dtype_of(dtype)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
    c, m = S.Cache8(p, cap, DEV, code=code, block=block), U.Model(B, H, d, block, code)
    U.fill(c, seed)
    bias = torch.randn((B, H, cap), generator=g, device=DEV)
    bias[torch.rand((B, H, cap), generator=g, device=DEV) < 0.2] = float("-inf")
    dec = S.Decoder8(p, c)
    dec.ws.random_(0, 256)
    dec.out.fill_(float("nan"))
    where = f"seed {seed}: B {B} H {H} G {G} d {d} block {block} {dtype} {code} cap {cap}"
    lens = [0] * B
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)

    def attended(b, out, k=None, v=None, with_bias=True):
        kk, vv = m.values(b)
        if k is not None:
            kk, vv = np.concatenate((kk, U.host(k)[:, None]), 1), np.concatenate((vv, U.host(v)[:, None]), 1)
        want, big = U.attention(U.host(q[b]), kk, vv, U.host(bias[b, :, :kk.shape[1]]) if with_bias else None, G,
                                U.scale_of(d))
        U.assert_near(U.host(out[b]), want, big, where)

    for i in range(10):
        call = r.choice(["write", "write", "attn", "step", "step", "read"]) if i else "write"
        q = torch.randn((B, H * G, d), generator=g, device=DEV).to(dt)
        bound = r.choice([max(lens), cap])
        if call == "write":
            n = r.randint(1, max(1, cap // 2))
            counts = [r.choice([0, n, r.randint(0, n)]) for _ in range(B)]
            K, V = U.rows(g, B, H, n, d, dtype=dtype), U.rows(g, B, H, n, d, dtype=dtype)
            S.cache8_write(p, c, K, V, bound, dev(lens), dev(counts))
            for b in range(B):
                got = min(counts[b], cap - lens[b])
                m.append(b, K[b, :, :got], V[b, :, :got])
                lens[b] += got
            U.assert_holds(c, m, where)
        elif call == "attn":
            with_bias = r.random() < 0.7
            out = dec.run(q, bound, bias if with_bias else None, dev(lens))
            for b in range(B):
                attended(b, out, with_bias=with_bias)
        elif call == "step":
            if max(lens) >= cap:
                continue
            k, v = U.rows(g, B, H, d, dtype=dtype), U.rows(g, B, H, d, dtype=dtype)
            idle = r.randrange(B)
            given = [-1 if b == idle and B > 1 else n for b, n in enumerate(lens)]
            out = dec.step(q, k, v, min(bound, cap - 1), bias, dev(given))
            for b in range(B):
                if given[b] < 0:
                    assert (out[b] == 0).all(), where
                    continue
                assert (bias[b, :, lens[b]] == 0).all(), where
                attended(b, out, k[b], v[b])
                m.append(b, k[b][:, None], v[b][:, None])
                lens[b] += 1
            U.assert_holds(c, m, where)
        else:
            first = r.randrange(cap)
            count = r.randint(1, cap - first)
            K = torch.full((B, H, count, d), 3.0, dtype=dt, device=DEV)
            V = torch.full_like(K, 3.0)
            S.cache8_read(p, c, K, V, cap, first, dev(lens))
            for b in range(B):
                there = max(0, min(first + count, lens[b]) - first)
                for got, want in zip((K, V), m.values(b)):
                    want = torch.from_numpy(want[:, first:first + there]).float().to(dt)
                    assert torch.equal(got[b, :, :there].cpu(), want), where
                    assert (got[b, :, there:] == 3).all(), where
