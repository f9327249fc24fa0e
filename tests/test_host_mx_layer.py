"""The layer's objects on microscaled rows: whose memory they hold and what they leave behind, without a GPU."""
import pytest
import torch

from paper_2204_04903_amd import binding as pk
from paper_2204_04903_amd import layer as L


@pytest.mark.parametrize("cols", [224, 832])
@pytest.mark.parametrize("align", [4, 128])
def test_a_dense_layers_weights_are_its_own(cols, align):
    """whether the given rows already lie as the product wants them makes no difference"""
    rows = L.MxRows(6, cols, pk.PK_MXFP4, device="cpu", align=align)
    rows.data.random_(0, 128)
    need = pk.pk_mx_row_bytes(pk.PK_MXFP4, cols)
    before = rows.data[:, :need].clone()
    dense = L.QuantizedLinear(rows)
    assert torch.equal(dense.weight.data[:, :need], before)
    rows.data.zero_()
    assert torch.equal(dense.weight.data[:, :need], before)
    assert dense.weight.stride % 128 == 0
