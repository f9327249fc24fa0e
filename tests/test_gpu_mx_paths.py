"""Parts of the microscaled operators' kernels that only larger or mixed sizes reach.

Products and gradients get numbers that their format holds exactly, and so few bits that every sum of them is a whole multiple of
a unit, below 2^24 of it: they are compared bit for bit (the bound is beside each).  Lookups as in test_gpu_mx_lookup.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from helpers import small_problem
from test_gpu_mx_lookup import close, layer_of, pooled, run

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def fp4_matrix(R, C, seed):
    """elements of E2M1 with scales 1 and 2, every block's largest element among them: multiples of 0.5, up to 12"""
    g = torch.Generator().manual_seed(seed)
    v = E2M1[torch.randint(0, 8, (R, C), generator=g)] * (torch.randint(0, 2, (R, C), generator=g) * 2 - 1)
    v[:, ::32] = 6.0
    return v * (1.0 + torch.randint(0, 2, (R, (C + 31) // 32), generator=g)).repeat_interleave(32, 1)[:, :C]


def linear_exactly(M, N, K, xdt, ydt, bias, seed):
    # units of 0.25 (the bias too): K products of at most 144 and a bias of at most 64 stay below 2^24 units for K <= 29000
    from paper_2204_04903_amd.layer import QuantizedLinear
    assert 4 * (144 * K + 64) < 2 ** 24
    x, w = fp4_matrix(M, K, seed), fp4_matrix(N, K, seed + 1)
    b = torch.randint(-256, 257, (N,), generator=torch.Generator().manual_seed(seed + 2)) / 4.0 if bias else None
    y = QuantizedLinear(w.cuda(), b.cuda() if bias else None).forward(x.to(DT[xdt]).cuda(), dtype=DT[ydt])
    ref = x.double().cuda() @ w.double().cuda().t()
    if bias:
        ref = ref + b.double().cuda()
    assert torch.equal(y, ref.float().to(DT[ydt]))


@pytest.mark.parametrize("ydt", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(2050, 2051, 4609), (2050, 2051, 8230), (2100, 4100, 4096)])
def test_linear_with_scales_of_more_steps_than_are_held(M, N, K, ydt):
    """(more than 256 tiles: K is not cut, and a tile's stretch has 19, 33 and 16 steps)"""
    linear_exactly(M, N, K, "f32", ydt, True, K)


@pytest.mark.parametrize("xdt", ["f32", "bf16"])
@pytest.mark.parametrize("ydt", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K", [(40, 70, 6007), (130, 71, 6144), (40, 257, 12000)])
def test_linear_in_several_stretches(M, N, K, xdt, ydt, bias):
    linear_exactly(M, N, K, xdt, ydt, bias, M + N)


@pytest.mark.parametrize("xdt", ["f32", "bf16"])
@pytest.mark.parametrize("ydt", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1024, 832), (5, 33, 1000), (16, 40, 4096), (16, 17, 256), (3, 100, 21000), (1, 16, 128)])
def test_linear_of_few_rows_in_whole_steps(M, N, K, xdt, ydt):
    linear_exactly(M, N, K, xdt, ydt, True, K)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,K", [(33, 70), (40, 71), (130, 129), (17, 32)])
@pytest.mark.parametrize("B", [700, 1500])
def test_gradient_added_up_from_stretches(B, N, K, dt):
    """two micro-batches of several stretches each, on top of what is there: 2 B |dY| |X| and what is there stay below 2^24"""
    from paper_2204_04903_amd.layer import ActivationCheckpoint
    g = torch.Generator().manual_seed(B + K)
    assert 2 * B * 255 * 15 + 4096 < 2 ** 24
    dw = torch.randint(-4096, 4097, (N, K + 3), generator=g).float().cuda()
    ref, between = dw.double(), dw[:, K:].clone()
    for _ in range(2):
        x, dy = torch.randint(-15, 16, (B, K), generator=g).float().cuda(), torch.randint(-255, 256, (B, N), generator=g).float().cuda()
        ActivationCheckpoint(B, K).quantize(x).weight_grad(dy.to(DT[dt]), out=dw[:, :K], accumulate=True)
        ref[:, :K] += dy.double().t() @ x.double()
    assert torch.equal(dw[:, :K].double(), ref[:, :K]) and torch.equal(dw[:, K:], between)


def with_lengths(pr, ranges, seed):
    """the problem with bags of other lengths: ranges[f] = (least, most), a field's own, the others 0 to 2"""
    rng = np.random.default_rng(seed)
    B, F = pr["B"], len(pr["fields"])
    lens = np.array([rng.integers(ranges.get(f, (0, 2))[0], ranges.get(f, (0, 2))[1] + 1, B) for f in range(F)])
    pr["offsets"] = np.concatenate([[0], np.cumsum(lens.reshape(-1))]).astype(np.int32)
    pr["ids"] = rng.integers(0, 10 ** 6, pr["offsets"][-1])
    return pr


@pytest.mark.parametrize("dims", [(16, 64, 8, 32), (200, 5, 100, 256), (3, 48)])
def test_more_sequences_than_wavefronts(dims):
    """(more than 4096 bags, of which those of three fields have 64 IDs and more on average: about 5 bags a wavefront)"""
    tables = [(300 + 40 * t, dims[t % len(dims)], 0) for t in range(12)]
    pr = small_problem(1, B=1024, tables=tables, fields=[(t, t % 2) for t in range(12)], max_len=1)
    run(with_lengths(pr, {1: (64, 150), 2: (30, 120), 7: (0, 200)}, 2))


@pytest.mark.parametrize("B", [300, 3001])
@pytest.mark.parametrize("F", [33, 40, 61])
def test_fields_dealt_to_xcds_in_many_tiles(F, B):
    dims = (8, 13, 32, 64, 100, 200)
    tables = [(50 + 7 * t, dims[t % 6], 0) for t in range(F)]
    pr = small_problem(F, B=B, tables=tables, fields=[(t, t % 2) for t in range(F)], max_len=1)
    run(with_lengths(pr, {f: (0, 9) for f in range(0, F, 3)}, B), pad=2)


@pytest.mark.parametrize("B", [5, 20])
def test_sequences_among_many_fields(B):
    """(fields are looked at 256 at a time; 1500 bags have a wavefront each, 6000 do not)"""
    tables = [(20 + t, (8, 16, 40)[t % 3], 0) for t in range(300)]
    pr = small_problem(3, B=B, tables=tables, fields=[(t, t % 2) for t in range(300)], max_len=1)
    run(with_lengths(pr, {f: (64, 400) for f in (0, 255, 256, 299)}, 4))


@pytest.mark.parametrize("place", [0, 1500, 2048, 4096])
def test_rejected_offsets_of_dealt_sequences(place):
    """(every read is bounded by nnz)"""
    tables = [(300, 24, 0), (200, 64, 0), (100, 8, 0), (90, 16, 0), (80, 16, 0)]
    pr = with_lengths(small_problem(8, B=1024, tables=tables, fields=[(t, 0) for t in range(5)], max_len=1), {0: (64, 150), 1: (70, 130)}, 9)
    layer, dec = layer_of(pr)
    try:
        pr["offsets"][place] = 2 ** 31 - 1 if place else 5
        got = layer.forward(torch.from_numpy(pr["ids"]).cuda(), torch.from_numpy(pr["offsets"]).cuda(), 1024).cpu().numpy()
        assert layer.error_word() == 1
        ref, mag = pooled(pr, dec)
        assert close(got, ref, mag)
    finally:
        layer.close()
