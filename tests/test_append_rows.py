"""selkv_paged_append of more rows than the workgroups of one launch may hold."""
import pytest
import torch

from tests import paged_util as U

pytestmark = pytest.mark.gpu


def test_append_of_more_than_2_to_the_27_rows():
    """One row repeated (a stride of 0): only the pages at the borders exist, rows for the others are not stored."""
    from paper_2607_16213_amd import selkv as S
    n, page = (1 << 27) + 300, 256
    p = S.params(batch=1, n_heads_kv=1, group=1, head_dim=64, kv_dtype="bf16")
    columns = -(-(n + 10) // page)
    c = S.PagedCache(p, 8, columns, U.DEV, page=page)
    there = [0, (1 << 18) - 1, 1 << 18, (1 << 19) - 1, 1 << 19, columns - 1]     # around rows 2^26 and 2^27, and the last
    for i, column in enumerate(there):
        c.table[0, column] = i
    one = U.rows(U.gen(1), 1, 1, 1, 64, dtype="bf16")
    rows = one.expand(1, n, 1, 64)
    S.paged_append(p, c, rows, rows, 10)
    torch.cuda.synchronize()
    for x in (c.K, c.V):
        for i, column in enumerate(there):
            first, last = max(10 - column * page, 0), min(n + 10 - column * page, page)
            assert bool((x[i, 0, first:last] == one[0, 0, 0]).all()), column
            assert bool((x[i, 0, :first] == 0).all()) and bool((x[i, 0, last:] == 0).all()), column
        assert bool((x[6:] == 0).all())
