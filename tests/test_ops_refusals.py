"""Calls of the adapters that are refused before anything is enqueued (CPU only:
addresses are numbers that nothing reads)."""
import pytest

from paper_2504_11651_amd import ops

from test_ops_host import A, INVALID, UNSUPPORTED, lora, lora_backward


@pytest.mark.parametrize("tokens, rows", [(1 << 24, 1 << 23), (1 << 23, 1 << 23), (1 << 24, 1 << 15)])
def test_more_products_than_a_grid_holds(tokens, rows):
    """Tokens x columns of a result that one launch cannot cover: refused with the
    shapes, not after the first kernels are under way."""
    big = dict(tokens=tokens, rows=rows, ws_bytes=1 << 62)
    assert lora(**big, base_stride=rows, out_stride=rows) == UNSUPPORTED
    assert lora_backward(**big, dy_stride=rows) == UNSUPPORTED
    assert lora_backward(tokens=tokens, cols=rows, ws_bytes=1 << 62, x_stride=rows, dx_stride=rows,
                         dx_base_stride=rows) == UNSUPPORTED
    for sizes in ((tokens, 128, rows, 8, 2), (tokens, rows, 64, 8, 2)):
        with pytest.raises(ops.codec.DF11Error):
            ops.lora_backward_workspace_bytes(*sizes)
    assert ops.lora_workspace_bytes(tokens, 128, 64, 8, 2) > 0


@pytest.mark.parametrize("change", [dict(x=3 * A), dict(dy=3 * A), dict(x=3 * A, dx_base=3 * A)])
def test_dx_in_place_of_what_the_adapters_gradients_still_read(change):
    """da and db are made of x and dy after dx is written."""
    assert lora_backward(dx=3 * A, **change) == INVALID
