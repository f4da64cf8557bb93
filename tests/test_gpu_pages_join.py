"""Splits of contexts joined apart, by one and by several threads each: clients with many splits, few and none in one pass, rows that fill
no workgroup, and long masked parts that leave splits without a seen token."""
import pytest

from tests.test_gpu_pages import attend_case, random_tree

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("before", [[6000], [20011], [70000]])
@pytest.mark.parametrize("rows", [5, 16, 33, 64, 128])
def test_one_client_in_many_splits(before, rows, dim):
    attend_case(16, 2, dim, "bf16", before, [rows], [random_tree(rows, rows)], seed=rows)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_clients_with_and_without_splits(dim, dtype):
    before, rows = [0, 30000, 17, 4000, 200, 9000, 1], [3, 9, 40, 17, 1, 33, 64]
    attend_case(16, 2, dim, dtype, before, rows, [random_tree(r, r, roots=b > 0) for b, r in zip(before, rows)], seed=3)
    attend_case(32, 1, dim, dtype, before[::-1], rows, None, seed=4)


@gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_a_long_chain_whose_first_rows_see_no_token_of_the_last_splits(dim):
    attend_case(8, 1, dim, "bf16", [100], [2048], None, seed=5)
    attend_case(8, 1, dim, "f32", [100], [700], None, seed=6)
