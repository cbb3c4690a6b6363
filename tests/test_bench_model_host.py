"""The drafted trees of bench_model.py, without a GPU."""
import torch

import bench_model


def test_a_path_draws_with_a_number_for_each_node():
    parents = [-1, 0, 0, 1, 1, 2, 4, 4]
    depths = [0, 1, 1, 2, 2, 2, 3, 3]
    u = torch.arange(12.0).view(3, 4) / 16
    chance = bench_model.draft_chances(u, parents).view(3, 8)
    for b in range(3):
        assert chance[b].tolist() == [float(u[b, d]) for d in depths]
        for leaf in (3, 5, 6, 7):
            path, at = [], leaf
            while at >= 0:
                path.append(float(chance[b, at]))
                at = parents[at]
            assert len(set(path)) == len(path)
    assert len(set(chance[:, 0].tolist())) == 3


def test_one_level():
    u = torch.tensor([[0.25, 0.5]])
    assert bench_model.draft_chances(u, [-1, 0, 0]).tolist() == [0.25, 0.5, 0.5]
