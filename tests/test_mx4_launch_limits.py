"""Matrices and products that no launch can hold (HIP takes fewer than 2^32 threads along x) are refused by the host's checks, without a GPU:
the addresses here reach no kernel."""
import pytest

from paper_2601_17768_amd import binding as B


# a workgroup of 256 threads makes four records of 16 x 256
@pytest.mark.parametrize("rows,cols", [(2 ** 30, 1), (2 ** 30, 256), (2 ** 30 - 32, 32), (2 ** 29, 257), (16, 2 ** 26), (2 ** 12 + 1, 2 ** 26)])
def test_matrices_of_more_records_than_a_launch_takes(rows, cols):
    lib = B.load_library()
    records = -(-rows // 16) * -(-cols // 256)
    too_large = -(-records // 4) * 256 >= 2 ** 32
    code = B.LLM42_EINVAL if too_large else B.LLM42_EWORKSPACE          # (the buffer is too small for the ones that are not)
    assert lib.llm42_mx4_quantize(4096, B.LLM42_BF16, cols, rows, cols, 4096, 2 ** 62 if too_large else 2175, None) == code
    assert lib.llm42_mx4_dequantize(4096, 2 ** 62 if too_large else 2175, rows, cols, 4096, B.LLM42_F32, cols, None) == code
    if too_large:
        assert lib.llm42_mx4_matmul(4096, 2 ** 62, rows, cols, 4096, cols, 1, 4096, B.LLM42_BF16, rows, None, 0, None) == code


# up to 16 rows a workgroup of 512 threads has 8 of the 2^26 - 4 blocks of 16 features; 17 to 256 rows fit (14 blocks by 256 rows to a
# workgroup of 512: 4.8 M of them), 256 times as many do not
@pytest.mark.parametrize("rows,n,k", [(1, 2 ** 30 - 64, 32), (8, 2 ** 30 - 64, 32), (16, 2 ** 30 - 64, 64), (B.LLM42_MAX_ROWS, 2 ** 30 - 64, 32)])
def test_products_of_more_features_than_a_launch_takes(rows, n, k):
    lib = B.load_library()
    assert lib.llm42_mx4_matmul(4096, 2 ** 62, n, k, 4096, k, rows, 4096, B.LLM42_BF16, n, None, 0, None) == B.LLM42_EINVAL
    assert b"features" in lib.llm42_last_error()


def test_rows_that_no_launch_brings_in_order():
    """65536 rows of 2^20 + 1 columns that are not 4-byte aligned: 2^33 pieces of 16 bytes."""
    lib = B.load_library()
    args = (2 ** 62, 16, 2 ** 20 + 1, 4098, 2 ** 20 + 1, B.LLM42_MAX_ROWS, 4096, B.LLM42_BF16, 16, 4096, 2 ** 62, None)
    assert lib.llm42_mx4_matmul(4096, *args) == B.LLM42_EINVAL
    assert b"rows" in lib.llm42_last_error()
