"""Attention of rows that see places past their table's width, down to a width of none,
by one kernel and in shares: no result for them, all of theirs for the others."""
import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from kv_reference import BF16, F16, Case, near

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

SHARES, WHOLE = 1000, 10  # tokens of the prefix: where a row has many to read, its work is cut


def check(c, prefix):
    """Rows that see no further than the table goes as the definition has them, the others NaN."""
    need = ops.prefix_attention_workspace_bytes(c.tokens, c.heads, c.cache, c.batch)
    assert (need > 0) == (prefix == SHARES)
    got, want = c.attend(), c.expected()
    place = torch.cat([torch.arange(m - n, m, device="cuda") for n, m in zip(c.new, c.own)])
    past = place >= c.table.shape[1] * c.page
    assert past.any() and not past.all()
    for name in ("out", "lse"):
        x = getattr(got, name)[:sum(c.new)]
        assert x[past].isnan().all(), f"{name}: a result for a row that sees past the table"
        near(x[~past], want[name][0][~past], want[name][1][~past], name)
        assert (getattr(got, name)[sum(c.new):] == 77.0).all()


@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("prefix", [SHARES, WHOLE])
def test_a_table_without_columns(prefix, dtype, dim):
    """Rows in front of their sequence's first place see the prefix alone; the others have
    tokens of their own, and no page for them."""
    check(Case([1, 2, 1, 3], [1, 1, 0, 300], prefix=prefix, width=0, dim=dim, dtype=dtype, seed=1, spare=2), prefix)


@pytest.mark.parametrize("prefix", [SHARES, WHOLE])
@pytest.mark.parametrize("sequences", [64, 65, 130])
def test_many_sequences_without_columns(sequences, prefix):
    own = [i % 3 for i in range(sequences)]
    check(Case([1] * sequences, own, prefix=prefix, width=0, heads=4, kv_heads=1, dim=64, page=16, seed=sequences),
          prefix)


@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("prefix", [SHARES, WHOLE])
@pytest.mark.parametrize("width", [1, 4, 8])
def test_tables_narrower_than_the_lengths(width, prefix, dtype, dim):
    end = 16 * width
    check(Case([4, 1, 40, 1], [end + 2, 10, end + 17, end + 400], prefix=prefix, page=16, width=width, dim=dim,
               dtype=dtype, seed=width), prefix)
