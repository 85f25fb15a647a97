"""Every kernel that the selection of pages and the attention over shared prefixes choose from, against the definitions in 64 bits (oracle/cache.py): by a table's
width and a call's rows, by a head's elements, by the query heads of a key head, by the columns of a prefix.  Tolerances: test_gpu_selection_and_prefix.py."""
import numpy as np
import pytest

from test_gpu_selection_and_prefix import check_prefix, check_select, prefix_case, select_case

pytestmark = pytest.mark.gpu

# query heads of the key head, elements: reads that are filled and that are not, one and two fours of query heads at a time
HEADS = [(4, 128), (8, 128), (8, 72), (3, 40), (13, 256), (1, 96)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hq,dim", HEADS)
@pytest.mark.parametrize("pages", [900, 1500, 2048, 3000, 9000])
def test_selection_of_rows_in_pieces_by_every_kernel(dtype, hq, dim, pages):
    # keys a lane holds: 4 and 8 of 256 threads, 8 of 1024 threads, none
    check_select(select_case([2 * pages - 1, pages, 0, 37, pages // 2], hq, 1, dim, 2, 60, dtype, seed=pages + hq, width=pages), 2)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hq,dim", HEADS)
@pytest.mark.parametrize("width", [500, 1500, 3000, 9000])
def test_selection_of_whole_rows_by_every_kernel(dtype, hq, dim, width):
    # more rows than are split; keys a lane holds: 4, 8 and 32 of 256 threads, none
    rng = np.random.default_rng(width)
    lengths = rng.integers(0, 25, 1030)
    lengths[[3, 1029]] = 2 * width, width
    check_select(select_case(lengths, hq, 1, dim, 2, 9, dtype, seed=width + hq, width=width), 2)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("members", [1, 3, 7, 14, 30, 65])
def test_prefix_by_every_number_of_columns(dtype, dim, members):
    # 4, 12, 28, 56, 120 and 260 query heads of a key head; a page that ends inside every unit of keys
    check_prefix(prefix_case([(members, 333)], np.arange(members) * 7 % 60, 8, 2, dim, 24, dtype, seed=dim + members), dtype)
    check_prefix(prefix_case([(members, 500), (members, 40)], np.arange(2 * members) * 7 % 60, 8, 2, dim, 16, dtype, seed=dim + members, heads_first=True), dtype)
