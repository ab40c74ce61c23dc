"""The helpers that make the rotary call's positions (no GPU needed)."""
import itertools

import pytest
import torch

import paper_2505_18875_amd as svg2


@pytest.mark.parametrize("grid,first", [((5,), None), ((3, 2), (1, -4)), ((2, 3, 4), None), ((2, 3, 4), (7, 0, 1)), ((2, 1, 3, 2), None),
                                        ((2, 3, 2, 2), (1, 2, 3, 4))])
def test_grid_positions_have_every_axis(grid, first):
    """Raster order over as many axes as the grid has, one to the four that the rotary call takes."""
    more = {} if first is None else {"first": first}
    pos = svg2.svg2_grid_positions(grid, extra=3, device="cpu", **more)
    start = first or (0,) * len(grid)
    want = [tuple(f + i for f, i in zip(start, at)) for at in itertools.product(*(range(n) for n in grid))]
    assert pos.dtype == torch.int32 and pos.is_contiguous()
    assert [tuple(p) for p in pos.tolist()] == want + [(0,) * len(grid)] * 3


def test_grid_positions_refuse_a_start_of_fewer_axes():
    with pytest.raises(ValueError):
        svg2.svg2_grid_positions((2, 3, 2, 2), first=(0, 0, 0), device="cpu")
