"""Positions of text and image nodes on three axes (host), against the rule written out token by token."""
import numpy as np
import pytest

import paper_2511_00413_amd as T


def by_rule(parent, seg, grid, offsets):
    """Children in ascending id, depth first; what follows a node starts behind its largest position."""
    out, roots = [], [i for i, p in enumerate(parent) if p < 0]

    def visit(i, start):
        t, h, w = grid[i] if grid is not None else (0, 0, 0)
        if t:
            pos = [(start + a, start + b, start + c) for a in range(t) for b in range(h) for c in range(w)]
        else:
            pos = [(start + a,) * 3 for a in range(seg[i])]
        out.extend(pos)
        nxt = max((max(p) for p in pos), default=start - 1) + 1
        for j, p in enumerate(parent):
            if p == i:
                visit(j, nxt)
    for r, i in enumerate(roots):
        visit(i, offsets[r] if offsets is not None else 0)
    return np.array(out, np.int32).reshape(-1, 3).T


@pytest.mark.parametrize("parent,seg,grid,offsets", [
    ([-1], [5], None, None),
    ([-1, 0, 1, 0], [4, 12, 3, 2], [[0, 0, 0], [1, 3, 4], [0, 0, 0], [0, 0, 0]], None),
    ([-1, 0, 1, 1, -1], [3, 24, 0, 7, 6], [[0] * 3, [2, 3, 4], [0] * 3, [7, 1, 1], [1, 1, 6]], [10, -4]),
    ([2, -1, 1], [1, 2, 0], None, [7]),
    ([], [], None, None),
])
def test_positions(parent, seg, grid, offsets):
    got = T.tree_axis_positions(parent, seg, None if grid is None else np.array(grid).reshape(-1, 3), offsets)
    assert np.array_equal(got, by_rule(parent, seg, grid, offsets)) and got.dtype == np.int32


def test_text_only_is_the_depth_of_the_token():
    rng = np.random.default_rng(0)
    parent = [-1] + [int(rng.integers(-1, i)) for i in range(1, 30)]
    seg = rng.integers(0, 9, 30).tolist()
    meta = T.tree_build_meta(parent, seg)
    assert np.array_equal(T.tree_axis_positions(parent, seg), np.stack([meta.tok_pos] * 3))


@pytest.mark.parametrize("parent,seg,grid,offsets,code", [
    ([-1], [5], [[1, 2, 2]], None, -2), ([-1], [4], [[1, 2, 0]], None, -2), ([-1], [4], [[-1, -2, 2]], None, -2),
    ([-1], [0], [[65536, 65536, 65536]], None, -2), ([-1], [4], [[0, 0, 0]], [2 ** 31 - 3], -2), ([0], [4], None, None, -3),
    ([-1], [16], [[2 ** 30, 2 ** 30, 16]], None, -2)])
def test_refusals(parent, seg, grid, offsets, code):
    with pytest.raises(T.TreeTrainError) as e:
        T.tree_axis_positions(parent, seg, grid, offsets)
    assert e.value.status == code


def test_wrong_shapes():
    with pytest.raises(ValueError):
        T.tree_axis_positions([-1, 0], [1])
    with pytest.raises(ValueError):
        T.tree_axis_positions([-1], [1], grid=[1, 1, 1])
    with pytest.raises(ValueError):
        T.tree_axis_positions([-1], [1], root_pos_offset=[1, 2])
