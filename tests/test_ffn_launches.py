"""What the host launches for calls of include/topoep_ffn.h, seen without a GPU
(tests/launches.py)."""
import pytest

import launches
from launches import BF16


def few_grids(answers):
    return [grid[0] * (4 if name.endswith("1>") else 1) for _, got in answers for name, grid, _ in got
            if name.startswith("few_")]


@pytest.mark.parametrize("T,H,I,E,L,k", [(512, 4096, 4096, 256, 1, 8), (512, 7168, 2048, 256, 8, 8),
                                         (448, 2048, 768, 256, 32, 8), (256, 512, 256, 256, 4, 8)])
def test_few_rows_of_a_share_have_a_grid_of_the_rows_expected(T, H, I, E, L, k, tmp_path):
    """Tiles of 16 rows of weights (8 units of both halves) for spans of 4 rows at least: of twice the expected
    rows and one more a group, or 4096."""
    answers, _ = launches.record([launches.forward(T, H, I, BF16, L, k, E)], tmp_path)
    spans = 2 * -(-T * k * L // E) / 4 + min(L, T * k) + 1
    up, down = few_grids(answers)
    assert up <= max(4100, spans * I / 8) and down <= max(4100, spans * H / 16 + 4)


def test_few_rows_of_experts_that_are_all_here_have_a_tile_each(tmp_path):
    T, H, I, E, k = 64, 2048, 768, 128, 8
    answers, _ = launches.record([launches.forward(T, H, I, BF16, E, k, E)], tmp_path)
    up, down = few_grids(answers)
    # eight columns a tile at most: 512 rows and a remainder of every expert
    assert up >= (512 // 8 + 128) * I // 8 and down >= (512 // 8 + 128) * H // 16
