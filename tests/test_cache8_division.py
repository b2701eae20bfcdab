"""GPU: both sides of the rules that divide the 8-bit decode's work, for every storage and code type, with equal lengths
and with lengths of their own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import cache8_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype,code", [("bf16", "e4m3"), ("fp32", "int8"), ("fp32", "e4m3")])
@pytest.mark.parametrize("B,H,G,d,n", [
    (4, 5, 8, 128, 700),            # eight waves a head
    (33, 8, 8, 128, 300),           # four waves a head, more than four query heads
    (16, 8, 7, 128, 770),           # barely split
    (32, 8, 2, 128, 3000),          # one round of workgroups that comes out even
    (5, 3, 6, 64, 6000),            # as many splits as a head may have
    (96, 8, 3, 64, 1100),           # 768 heads, past the length of one workgroup a head
    (100, 8, 8, 128, 1500),         # a round and a little more
])
def test_division(B, H, G, d, n, dtype, code, ragged):
    from paper_2607_16213_amd import selkv as S
    block, dt = 32, U.dtype_of(dtype)
    g = torch.Generator(device=DEV).manual_seed(n + B)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
    c = S.Cache8(p, n + 1, DEV, code=code, block=block)
    U.fill(c, n)
    some = [0, 1, B // 2, B - 1]                                      # the sequences that are compared
    sizes = [n * (b * 7 % 11) // 10 % (n + 1) for b in range(B)] if ragged else [n] * B
    if ragged:
        sizes[0], sizes[1], sizes[B // 2] = n, 0, block - 1
    lens = torch.tensor(sizes, dtype=torch.int32, device=DEV) if ragged else None
    K, V = U.rows(g, B, H, n, d, dtype=dtype), U.rows(g, B, H, n, d, dtype=dtype)
    S.cache8_write(p, c, K, V, 0, torch.zeros_like(lens) if ragged else None, lens)
    m = U.Model(len(some), H, d, block, code)
    for i, b in enumerate(some):
        m.append(i, K[b, :, :sizes[b]], V[b, :, :sizes[b]])
    del K, V
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(dt)
    bias = torch.randn((B, H, c.capacity), generator=g, device=DEV)
    bias[torch.rand(bias.shape, generator=g, device=DEV) < 0.1] = float("-inf")
    dec = S.Decoder8(p, c)
    dec.ws.random_(0, 256)
    out = dec.run(q, n, bias, lens, out=torch.full_like(dec.out, float("nan")))
    assert torch.isfinite(out).all()
    k, v = U.rows(g, B, H, d, dtype=dtype), U.rows(g, B, H, d, dtype=dtype)
    held = bias.clone()
    stepped = dec.step(q, k, v, n, bias, lens, out=torch.full_like(dec.out, float("nan")))
    assert torch.isfinite(stepped).all()
    for i, b in enumerate(some):
        kk, vv = m.values(i)
        size = sizes[b]
        want, big = U.attention(U.host(q[b]), kk, vv, U.host(held[b, :, :size]), G, U.scale_of(d))
        U.assert_near(U.host(out[b]), want, big, f"sequence {b}")
        kk, vv = np.concatenate((kk, U.host(k[b])[:, None]), 1), np.concatenate((vv, U.host(v[b])[:, None]), 1)
        want, big = U.attention(U.host(q[b]), kk, vv, U.host(bias[b, :, :size + 1]), G, U.scale_of(d))
        U.assert_near(U.host(stepped[b]), want, big, f"step, sequence {b}")
        m.append(i, k[b][:, None], v[b][:, None])
    for t in ("K", "V", "k_scale", "v_scale", "k_tail", "v_tail"):     # of the compared sequences
        setattr(c, t, getattr(c, t)[some])
    U.assert_holds(c, m, "after the step")
