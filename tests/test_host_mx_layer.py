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


@pytest.fixture
def plans(monkeypatch):
    """the plans that are alive"""
    alive, create, destroy = set(), pk.pk_plan_create, pk.pk_plan_destroy

    def created(*a, **kw):
        plan = create(*a, **kw)
        alive.add(plan)
        return plan

    def destroyed(plan):
        alive.remove(plan)
        destroy(plan)
    monkeypatch.setattr(pk, "pk_plan_create", created)
    monkeypatch.setattr(pk, "pk_plan_destroy", destroyed)
    return alive


TABLES, FIELDS = [(50, 8, 0), (30, 40, 1)], [(0, 0), (1, 1)]


def rows(total, nbytes, **kw):
    return torch.zeros((total, nbytes), dtype=torch.uint8, **kw)


@pytest.mark.parametrize("packs", [
    [],
    [rows(50, 8)],
    [rows(50, 8), rows(30, 24), rows(30, 24)],
    [rows(49, 8), rows(30, 24)],                             # a row too few
    [rows(50, 8), rows(30, 20)],                             # rows too short
    [rows(50, 12), rows(30, 24)],                            # rows that do not stand close together
    [rows(50, 8), rows(30, 48)[:, ::2]],
    [torch.zeros(50, 8), rows(30, 24)],
    [rows(50, 8, device="meta"), rows(30, 24)],
])
def test_refused_tables_leave_no_plan(plans, packs):
    with pytest.raises(ValueError):
        L.QuantizedEmbedding(TABLES, FIELDS, device="cpu", rows=packs)
    assert not plans
    good = L.QuantizedEmbedding(TABLES, FIELDS, device="cpu", rows=[rows(50, 8), rows(30, 24)])
    assert len(plans) == 1
    good.close()
    assert not plans


def test_a_layer_that_cannot_be_taken_over_leaves_no_plan(plans):
    source = L.PackedEmbedding(TABLES, FIELDS, device="cpu")
    with pytest.raises(ValueError):                          # (its tables are not on a GPU: nothing can round them)
        L.QuantizedEmbedding.from_layer(source)
    assert len(plans) == 1
    with pytest.raises(ValueError):
        L.QuantizedEmbedding.from_layer(source, max_shards=2)
    assert len(plans) == 1
    source.close()
    assert not plans
