"""TreeDecoder.attend: rotary positions of a tree's nodes."""
import pytest
import torch

from tests import paged_util as U

pytestmark = pytest.mark.gpu


def test_a_tree_is_not_turned_as_a_chain():
    """Siblings are at one position.  With a rope a tree without positions is refused before anything is stored; with
    them, and for a chain without, keys are turned by where they are."""
    from paper_2607_16213_amd import selkv as S
    p = S.params(batch=2, n_heads_kv=2, group=2, head_dim=64, kv_dtype="fp32")
    c = S.PagedCache(p, 8, 4, U.DEV, page=16)
    c.table.copy_(torch.arange(8, dtype=torch.int32).view(2, 4))
    dec, g = S.TreeDecoder(p, c, 4), U.gen(1)
    q, k = U.rows(g, 2, 4, 4, 64, dtype="fp32"), U.rows(g, 2, 4, 2, 64, dtype="fp32")
    freq, _ = S.rope_frequencies(64, 10000.0, U.DEV)
    rope = S.Rope(freq)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=U.DEV)
    star, lens = i32([[-1, 0, 0, 0]] * 2), i32([20, 3])
    for given in (dict(lens=lens), dict()):
        with pytest.raises(ValueError, match="positions"):
            dec.attend(q, k, k, 20, star, rope=rope, **given)
    assert bool((c.K == 0).all()) and bool((c.V == 0).all())

    def check(positions):
        for b, L in enumerate((20, 3)):
            want, size = U.turn(U.host(k[b]), U.host(i32(positions[b])), U.host(freq), "half", 1.0)
            pg, row = U.places(c, b, L, 4)
            # products and a sum in fp32 with sine and cosine a few steps off, and the rounding to the type
            assert (abs(U.host(c.K[pg, :, row]) - want) <= 9 * 2.0 ** -24 * size + 2.0 ** -40).all()

    at = [[20, 21, 21, 21], [3, 4, 4, 4]]
    dec.attend(q, k, k, 20, star, lens=lens, rope=rope, positions=i32(at))
    check(at)
    dec.attend(q, k, k, 20, None, lens=lens, rope=rope)
    check([[20, 21, 22, 23], [3, 4, 5, 6]])
    dec.attend(q, k, k, 20, star, lens=lens)          # nothing is turned: no positions are needed
