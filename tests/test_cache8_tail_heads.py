"""GPU: more than four query heads to a KV head, which the waves of the tail share, in every division of the work."""
import pytest

torch = pytest.importorskip("torch")

from tests import cache8_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("G", [1, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("B,H,n", [(1, 3, 9), (1, 3, 200), (130, 2, 200), (1, 2, 1600)])
# the tail alone, eight waves a head, four waves a head, splits
def test_heads_shared_by_the_waves_of_the_tail(B, H, n, G):
    """Every query head's maximum and sum are those of the wave that took it, also where its rows are far below the
    other heads': the first head of a wave is large, the last small."""
    from paper_2607_16213_amd import selkv as S
    d, block = 128, 128
    g = torch.Generator(device=DEV).manual_seed(G + n)
    p = S.params(batch=B, n_heads_kv=H, group=G, head_dim=d, kv_dtype="bf16")
    c, m = S.Cache8(p, n + 1, DEV, block=block), U.Model(1, H, d, block, "int8")
    K, V = U.rows(g, B, H, n, d, dtype="bf16"), U.rows(g, B, H, n, d, dtype="bf16")
    S.cache8_write(p, c, K, V, 0)
    q = torch.randn((B, H, G, d), generator=g, device=DEV)
    q = (q * torch.tensor([4.0, 0.25, 1.0, 0.0625], device=DEV).repeat(2)[:G, None]).view(B, H * G, d).to(torch.bfloat16)
    out = S.Decoder8(p, c).run(q, n)
    assert torch.isfinite(out).all()
    m.append(0, K[B - 1], V[B - 1])
    want, big = U.attention(U.host(q[B - 1]), *m.values(0), None, G, U.scale_of(d))
    U.assert_near(U.host(out[B - 1]), want, big)
