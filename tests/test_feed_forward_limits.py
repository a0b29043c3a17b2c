"""The largest matrices that the feed-forward functions take: host logic, no GPU call."""
import pytest

import paper_1410_0759_amd as ig

F, B = ig.IGC_DATA_FLOAT, ig.IGC_DATA_BFLOAT16
MOST_ROWS, MOST_COLUMNS = 1 << 30, 1 << 26


def rows(dt, M, C):
    return ig.TensorDescriptor().set(dt, M, C, 1, 1, (C, 1, 1, 1))


def norm(M, C):
    d = rows(F, M, C)
    try:
        ig.get_layer_norm_backward_workspace_size(ig.Handle(), d, d, d)
    except ig.IgcError as e:
        return e.status
    return ig.IGC_STATUS_SUCCESS


def product(M, C, K, query=ig.get_linear_forward_workspace_size, dt=B):
    w = ig.FilterDescriptor().set(dt, K, C, 1, 1)
    try:
        query(ig.Handle(), rows(dt, M, C), w, rows(dt, M, K))
    except ig.IgcError as e:
        return e.status
    return ig.IGC_STATUS_SUCCESS


def test_rows_and_columns():
    ok, no = ig.IGC_STATUS_SUCCESS, ig.IGC_STATUS_NOT_SUPPORTED
    assert norm(MOST_ROWS, 1) == ok and norm(MOST_ROWS + 1, 1) == no
    assert norm(2, MOST_COLUMNS) == ok and norm(2, MOST_COLUMNS + 1) == no
    for dt in (F, B):
        assert product(MOST_ROWS, 1, 2, dt=dt) == ok and product(MOST_ROWS + 1, 1, 2, dt=dt) == no
        assert product(2, MOST_COLUMNS, 1, dt=dt) == ok and product(2, MOST_COLUMNS + 1, 1, dt=dt) == no
        assert product(2, 1, MOST_COLUMNS, dt=dt) == ok and product(2, 1, MOST_COLUMNS + 1, dt=dt) == no


def test_rows_counted_over_all_positions():
    # 2^16 x 2^15 positions and 2^11 x 2^10 x 2^10
    for n, h, w in ((1 << 16, 1 << 15, 1), (1 << 11, 1 << 10, 1 << 10)):
        d = ig.TensorDescriptor().set(B, n, 8, h, w, (h * w * 8, 1, w * 8, 8))
        with pytest.raises(ig.IgcError) as e:
            ig.get_layer_norm_backward_workspace_size(ig.Handle(), d, d, d)
        assert e.value.status == ig.IGC_STATUS_NOT_SUPPORTED
