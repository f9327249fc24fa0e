"""Dense products whose launch would not fit: fewer than 2^32 threads is what a launch may have."""
import pytest

from paper_2204_04903_amd import binding as pk

FAKE = 0x10000      # never dereferenced: every call below fails validation first


@pytest.mark.parametrize("K,N", [(8, 2 ** 30), (256, 2 ** 30), (257, 2 ** 29), (4096, 2 ** 26), (65536, 2 ** 26)])
def test_few_rows_with_many_columns_go_by_tiles(K, N):
    """16 columns of y a block of 64 threads for each 256 columns of K, 16 times that at most: 2^32 threads from N on"""
    one_launch = pk.pk_mx_linear_workspace_bytes(1, 16, K)
    assert pk.pk_mx_linear_workspace_bytes(1, N - 16, K) == one_launch
    assert pk.pk_mx_linear_workspace_bytes(1, N, K) > one_launch             # x is rounded into the workspace there


@pytest.mark.parametrize("M,N", [(2 ** 30, 129), (2 ** 30 - 511, 129), (129, 2 ** 30), (2 ** 20, 2 ** 18)])
def test_products_of_too_many_tiles_are_refused(M, N):
    """blocks of 256 threads, one a tile, in eights: up to 2^24 - 8 of them"""
    with pytest.raises(pk.PkError) as e:
        pk.pk_mx_linear(FAKE, 0, 64, M, FAKE, 48, N, 64, None, FAKE, 0, N, FAKE, 2 ** 62)
    assert e.value.status == pk.PK_EOVERFLOW


def test_weight_gradients_of_too_many_tiles_are_refused():
    with pytest.raises(pk.PkError) as e:
        pk.pk_mx_weight_grad(FAKE, 0, 2 ** 24, FAKE, pk.pk_mx_row_bytes(1, 2 ** 14), 4, 2 ** 24, 2 ** 14, FAKE, 2 ** 14, False, FAKE, 2 ** 62)
    assert e.value.status == pk.PK_EOVERFLOW
