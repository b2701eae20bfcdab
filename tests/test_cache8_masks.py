"""GPU: masks of the 8-bit decode against queries and entries whose products leave fp32's range."""
import pytest

torch = pytest.importorskip("torch")

from tests import cache8_util as U

pytestmark = pytest.mark.gpu
DEV, NEG_INF = "cuda", float("-inf")


def made(B, H, G, d, dtype, code, block, n, seed):
    """A cache of n entries, and the rows it holds."""
    from paper_2607_16213_amd import selkv as S
    g = torch.Generator(device=DEV).manual_seed(seed)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype=dtype)
    c, m = S.Cache8(p, n + 1, DEV, code=code, block=block), U.Model(B, H, d, block, code)
    K, V = U.rows(g, B, H, n, d, dtype=dtype), U.rows(g, B, H, n, d, dtype=dtype)
    q = torch.randn((B, H * G, d), generator=g, device=DEV).to(U.dtype_of(dtype))
    return S, p, c, m, K, V, q


# the tail alone, one workgroup a head, and splits
@pytest.mark.parametrize("n", [20, 300, 3000])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), NEG_INF])
def test_a_full_mask_is_zero_for_every_query(n, code, dtype, bad):
    H, G, d = 2, 3, 128
    S, p, c, _, K, V, q = made(1, H, G, d, dtype, code, 64, n, n)
    S.cache8_write(p, c, K, V, 0)
    dec = S.Decoder8(p, c)
    bias = torch.zeros((1, H, c.capacity), device=DEV)
    bias[0, 0] = NEG_INF
    good = dec.run(q, n, bias).clone()
    q[0, 1, 5] = bad              # of the head that the mask leaves nothing of
    q[0, G] = bad                 # of the other
    out = dec.run(q, n, bias)
    assert (out[0, :G] == 0).all()
    assert torch.isnan(out[0, G]).all()               # an unmasked row carries it on
    assert torch.equal(out[0, G + 1:], good[0, G + 1:])
    bias[0, 0, n // 2] = 0                            # one entry left, in a partial mask
    out = dec.run(q, n, bias)
    assert torch.isfinite(out[0, [0, 2]]).all()
    if bad != bad:                                    # (an infinity's logit may be -inf, a weight of 0)
        assert torch.isnan(out[0, 1]).all()


@pytest.mark.parametrize("n", [50, 300, 3000])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_masked_entries_whose_logits_overflow(n, code, dtype):
    """Finite keys whose products with the query are past fp32's largest number: masked, they change nothing."""
    H, G, d, block = 2, 4, 64, 32
    S, p, c, m, K, V, q = made(1, H, G, d, dtype, code, block, n, n + 1)
    q[..., 0] = 100.0
    where = [1, n // 2, n - 1]
    K[:, :, where] = 0.0
    K[:, :, where, 0] = 3.0e38                       # 100 * 3e38 / 8
    K[:, 1, where[1], 0] = -3.0e38
    S.cache8_write(p, c, K, V, 0)
    m.append(0, K[0], V[0])
    bias = torch.randn((1, H, c.capacity), generator=torch.Generator(device=DEV).manual_seed(n), device=DEV)
    bias[:, :, where] = NEG_INF
    out = S.Decoder8(p, c).run(q, n, bias)
    want, big = U.attention(U.host(q[0]), *m.values(0), U.host(bias[0, :, :n]), G, U.scale_of(d))
    U.assert_near(U.host(out[0]), want, big)
