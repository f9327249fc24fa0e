"""A dense product of one row with 2^30 columns of weights: more than one launch of the kernel for few rows holds."""
import pytest

torch = pytest.importorskip("torch")

from paper_2204_04903_amd import binding as pk

pytestmark = pytest.mark.gpu


def test_one_row_and_two_to_the_thirty_columns():
    N, K = 2 ** 30, 8
    x = torch.tensor([[6.0, -0.5, 1.0, 3.0, -4.0, 2.0, 0.0, 1.5]], device="cuda")          # held exactly
    w = torch.randint(0, 256, (N, 8), dtype=torch.uint8, device="cuda")                     # 4 bytes of codes, a scale, 3 of zeros
    w[:, 4] = 127
    w[:, 5:] = 0
    y = torch.full((1, N), float("nan"), device="cuda")
    nbytes = pk.pk_mx_linear_workspace_bytes(1, N, K)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    pk.pk_mx_linear(x, pk.PK_F32, K, 1, w, 8, N, K, None, y, pk.PK_F32, N, ws, nbytes, torch.cuda.current_stream().cuda_stream)
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    value = torch.cat([value, -value])
    for n in range(0, N, 2 ** 26):                           # sums of eight multiples of 0.25: exact
        c = w[n:n + 2 ** 26, :4]
        ref = torch.zeros(c.shape[0], device="cuda")
        for k in range(K):
            ref += value[((c[:, k // 2] >> 4) if k % 2 else (c[:, k // 2] & 15)).int()] * x[0, k]
        assert torch.equal(y[0, n:n + 2 ** 26], ref)
