"""How rows are dealt to workgroups in the norms' backward pass, seen from the workspace that it asks for."""
import pytest


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 8192), (2, 64), (255, 8192), (257, 8192), (300, 8192), (520, 8192), (700, 5000), (1025, 4096),
                                       (2313, 1155), (5000, 6144)])
def test_every_slab_has_rows(harp, rows, cols):
    """Four vectors of partial sums a slab (and 256 bytes over, in multiples of 256).  Slabs of ceil(rows / slabs) rows: the last
    of them begins before the rows end."""
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    slabs = (ops.norm_workspace(ctx, rows, cols).numel() - 256) // (16 * cols)
    assert 1 <= slabs <= rows and (slabs - 1) * -(-rows // slabs) < rows, slabs
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("per,groups,cols", [(257, 9, 1155), (300, 1, 8192), (130, 2, 8192), (999, 3, 4096)])
def test_every_slab_of_a_gate_has_rows(harp, per, groups, cols):
    """The same of the slabs of each gate's rows, with a fifth vector a slab for the gate's gradient."""
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    slabs = (ops.norm_workspace(ctx, per * groups, cols, per).numel() - 256) // (20 * cols)
    assert slabs % groups == 0
    slabs //= groups
    assert (slabs - 1) * -(-per // slabs) < per, slabs
    ctx.close()
