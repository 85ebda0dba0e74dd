"""CPU tests of refusals of the row layers that depend on how arguments fit together, before anything is launched."""
import pytest
import torch

from paper_2402_07710_amd import binding as sc
from tests.test_row_layers_arguments import half, heads, rope_bwd, rope_fwd

EINVAL = sc.SC_EINVAL


@pytest.fixture(scope="module")
def lib():
    return sc.load()


def test_rope_outputs_that_overlap(lib):
    """Rows 0, heads 0 apart; heads within each other; rows that start inside the heads of others.  (Inputs may: they are only read.)"""
    for row, head, n in ((0, 64, 2), (128, 0, 2), (128, 63, 2), (127, 64, 2), (63, 1 << 20, 2), (64, 128, 3), (100, 350, 2), (150, 160, 2)):
        out = heads(row=row, head=head, n=n)
        assert rope_fwd(lib, rows=5, q=heads(n=n), qo=out) == EINVAL, (row, head, n)
        assert rope_fwd(lib, rows=5, k=heads(n=n), ko=out) == EINVAL, (row, head, n)
        assert rope_bwd(lib, rows=5, dqo=heads(n=n), dq=out) == EINVAL, (row, head, n)
        assert rope_bwd(lib, rows=5, dko=heads(n=n), dk=out) == EINVAL, (row, head, n)


def test_fewer_rows_than_entries():
    """Without a list entry p reads row p, so there has to be one."""
    starts, w = torch.zeros(4, dtype=torch.int32), half(3, 32, 64)
    with pytest.raises(ValueError, match="x has fewer rows than there are entries"):
        sc.sc_grouped_fwd(half(9, 32), w, starts, half(10, 64), stream=0)
    with pytest.raises(ValueError, match="x has fewer rows than there are entries"):
        sc.sc_grouped_bwd(half(10, 64), half(9, 32), None, starts, grad_weight=w, stream=0)
    rows = torch.zeros(10, dtype=torch.int32)
    for x, kw in ((half(11, 32), {}), (half(9, 32), dict(rows=rows))):
        with pytest.raises(ValueError, match="device tensor expected"):
            sc.sc_grouped_fwd(x, w, starts, half(10, 64), stream=0, **kw)
        with pytest.raises(ValueError, match="device tensor expected"):
            sc.sc_grouped_bwd(half(10, 64), x, None, starts, grad_weight=w, stream=0, **kw)


def test_channels_that_no_int_holds():
    """2^32 + 32 channels are not 32."""
    wide, many = (torch.empty(shape, dtype=torch.float16, device="meta") for shape in ((1, (1 << 32) + 32), ((1 << 32) + 32, 64)))
    with pytest.raises(ValueError, match="x has too many channels"):
        sc.sc_linear_fwd(wide, many, half(1, 64), stream=0)


def test_weights_of_rows_that_are_not_given():
    """x may be None where no weight gradient is asked for; shapes are then the weights'."""
    grad = half(10, 64)
    with pytest.raises(ValueError, match="device tensor expected"):
        sc.sc_linear_bwd(grad, None, half(32, 64), grad_x=half(10, 32), stream=0)
    with pytest.raises(ValueError, match="grad_x has the wrong shape"):
        sc.sc_linear_bwd(grad, None, half(32, 64), grad_x=half(10, 31), stream=0)
    with pytest.raises(ValueError, match="weight has the wrong shape"):
        sc.sc_linear_bwd(grad, None, half(32, 63), grad_x=half(10, 32), stream=0)
    starts = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor expected"):
        sc.sc_grouped_bwd(grad, None, half(3, 32, 64), starts, grad_x=half(10, 32), stream=0)
    with pytest.raises(ValueError, match="grad_x has the wrong shape"):
        sc.sc_grouped_bwd(grad, None, half(3, 32, 64), starts, grad_x=half(10, 31), stream=0)
    with pytest.raises(ValueError, match="weight has the wrong shape"):
        sc.sc_grouped_bwd(grad, None, half(2, 32, 64), starts, grad_x=half(10, 32), stream=0)


def test_positions_without_the_axes_of_the_table():
    """The table says by how many axes it turns; one that does not is taken as it is."""
    q, table = half(5, 2, 64), torch.zeros(512, dtype=torch.uint8)
    two, three = (torch.zeros(5, n, dtype=torch.int32) for n in (2, 3))
    with pytest.raises(ValueError, match="device tensor expected"):
        sc.sc_qk_rope_fwd(q, None, two, table, q, None, stream=0)
    table.rope_axes = 3
    with pytest.raises(ValueError, match="table turns by more axes than pos has"):
        sc.sc_qk_rope_fwd(q, None, two, table, q, None, stream=0)
    with pytest.raises(ValueError, match="table turns by more axes than pos has"):
        sc.sc_qk_rope_bwd(q, None, None, None, two, table, q, None, stream=0)
    with pytest.raises(ValueError, match="device tensor expected"):
        sc.sc_qk_rope_fwd(q, None, three, table, q, None, stream=0)
    table.rope_axes = "three"
    with pytest.raises(TypeError):
        sc.sc_qk_rope_fwd(q, None, three, table, q, None, stream=0)
