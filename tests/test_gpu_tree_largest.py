"""The largest calls of the tree operators: 64 nodes, 16 heads to a key-value head, accepted paths of 16 tokens with up to 256 query
rows."""
import pytest

from test_gpu_tree import check as check_attend
from test_gpu_tree_commit import check as check_commit
from tree_cases import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("B,live,nodes", [(300, [300, 1], [64, 63]), (1500, [1499, 0], [64, 9])])
def test_a_thousand_query_rows(dtype, d, B, live, nodes):
    check_attend(make(B + d, S=2, G=2, B=B, d=d, T=64, group=16, dtype=dtype, live=live, nodes=nodes))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("group", [3, 5, 8, 13, 16])
@pytest.mark.parametrize("T,B,live", [(16, 140, [140, 130]), (64, 1030, [1030, 1020])])
def test_paths_of_sixteen_tokens(dtype, d, group, T, B, live):
    c = make(B + group, S=2, G=2, B=B, d=d, T=T, group=group, dtype=dtype, live=live, shape="chain")
    check_commit(c, [list(range(16)), list(range(11))], 16, 30)


@pytest.mark.parametrize("group", [1, 4, 16])
def test_paths_of_sixteen_tokens_of_many_units(group):
    c = make(7 + group, S=1, G=300, B=150, d=128, T=16, group=group, dtype="bf16", live=[148], shape="chain")
    check_commit(c, [list(range(16))], 16, 30)
