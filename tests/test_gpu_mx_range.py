"""Numbers at the end of fp32's range in microscaled rows: whatever is finite is read back as a finite number.

A block whose largest magnitude is above 1.5 * 2^127 (4 bits) or 1.75 * 2^127 (8 bits) has the scale 2^126 or 2^120, and the nearest
code of what lies above 1.75 * 2^127 or 1.9375 * 2^127 stands for 2^128.  The code below it stands for 1.5 * 2^127 or 1.875 * 2^127,
which is off by less than 2^-2 or 2^-4 of any number up to 2^128: the formats' half step, relative."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOP = {"f32": torch.finfo(torch.float32).max, "bf16": torch.finfo(torch.bfloat16).max}
HALF_STEP = (2.0 ** -2, 2.0 ** -4)


def top_values(dtype, C):
    """a row for each place of the last binade, both signs, smaller numbers of every size beside them"""
    m = np.concatenate([np.linspace(1.0, 1.9921875, 64), [1.4999999, 1.5000001, 1.7499999, 1.75, 1.7500001, 1.8749999, 1.8750001, 1.9374999, 1.9375, 1.9375001, 1.9999999]])
    x = np.outer(np.append(m, -m) * 2.0 ** 127, np.exp2(-np.arange(C) % 11 * 0.37))
    return torch.from_numpy(np.clip(x, -TOP[dtype], TOP[dtype]).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 5, 32, 70])
def test_finite_numbers_are_read_back_finite(C, dtype, fmt):
    from paper_2204_04903_amd.layer import MxRows
    x = top_values(dtype, C)
    m = MxRows(x.shape[0], C, fmt).quantize(x.cuda())
    want = mx.encode(x.float().numpy(), fmt)
    assert np.array_equal(m.data.cpu().numpy()[:, :want.shape[1]], want)
    v = x.double().numpy()
    for dt in DT.values():
        y = m.dequantize(dtype=dt).cpu().double().numpy()
        assert np.isfinite(y).all()
        # half a step of the format at the element's size, or of its smallest step at the block's scale: 2^126 / 4, 2^120 / 2^10
        assert (np.abs(y - v) <= np.maximum(HALF_STEP[fmt] * np.abs(v), 2.0 ** 124 if fmt == 0 else 2.0 ** 110)).all()


@pytest.mark.parametrize("M", [1, 40])
def test_dense_product_of_the_largest_numbers(M):
    """x and the weights at the end of the range, each against a partner small enough for a finite product (few rows, and tiles)"""
    from paper_2204_04903_amd.layer import QuantizedLinear
    big, small = torch.full((M, 300), TOP["f32"]), torch.full((20, 300), 2.0 ** -100)
    for x, w in ((big, small), (torch.full((M, 300), 2.0 ** -100), torch.full((20, 300), TOP["f32"]))):
        y = QuantizedLinear(w.cuda()).forward(x.cuda()).cpu()
        assert (y == 300 * 1.5 * 2.0 ** 27).all()             # (450 * 2^27: exact)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_weight_gradient_of_the_largest_numbers(dt):
    from paper_2204_04903_amd.layer import ActivationCheckpoint
    dy = torch.full((90, 12), 2.0 ** -100, dtype=DT[dt]).cuda()
    dw = ActivationCheckpoint(90, 40).quantize(torch.full((90, 40), -TOP["f32"]).cuda()).weight_grad(dy)
    assert (dw.cpu() == -90 * 1.875 * 2.0 ** 27).all()


def test_lookup_of_the_largest_numbers():
    from paper_2204_04903_amd.layer import QuantizedEmbedding
    layer = QuantizedEmbedding([(4, 40, 0)], [(0, 0)])
    try:
        layer.load_table(0, torch.full((4, 40), TOP["f32"]) * torch.tensor([[1.0], [-1.0], [0.0], [0.5]]))
        out = layer.forward(torch.arange(4, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda"), 4).cpu()
        assert torch.equal(out, torch.tensor([[1.5], [-1.5], [0.0], [1.0]]).mul(2.0 ** 127).expand(4, 40))
    finally:
        layer.close()
