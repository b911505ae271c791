"""Depths of drafted rows (paged_tree.depths), with parents of rows that do not count."""
import torch

from paper_2606_31160_gb300 import paged_tree


def test_parents_of_rows_that_do_not_count_may_be_anything():
    """They are neither followed nor looked up; the rows before them keep their depths."""
    good = [-1, 0, 0, 1, 3]
    for rest in ([1 << 20, -7, 1 << 30], [5, 6, 7], [7, 5, 6], [-(1 << 31), (1 << 31) - 1, 8]):
        parents = torch.tensor([good + rest, [-1, 0, 1, 2, 3, 4, 5, 6]], dtype=torch.int32)
        got = paged_tree.depths(parents)
        assert got.dtype is torch.int32 and got[0, :5].tolist() == [0, 1, 1, 2, 3] and got[1].tolist() == list(range(8))


def test_forests_and_single_rows():
    assert paged_tree.depths(torch.tensor([[-1, -1, 1, 0]], dtype=torch.int32)).tolist() == [[0, 0, 1, 1]]
    assert paged_tree.depths(torch.tensor([[-1], [9]], dtype=torch.int32)).tolist() == [[0], [0]]
