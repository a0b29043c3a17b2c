"""Float products of few tokens read the filter as it lies, whatever the reduction's length: their workspaces hold no copy of it.  Host logic, no GPU call."""
import pytest

import paper_1410_0759_amd as ig

F = ig.IGC_DATA_FLOAT


def rows(M, C, pad=0):
    return ig.TensorDescriptor().set(F, M, C, 1, 1, (C + pad, 1, 1, 1))


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("tokens", [1, 8, 60])
@pytest.mark.parametrize("reduced", [4000, 4001, 4002, 4003])
def test_no_copy_of_the_filter(reduced, tokens, pad):
    h, features = ig.Handle(), 8192
    filt = 4 * reduced * features
    w = ig.FilterDescriptor().set(F, features, reduced, 1, 1)
    assert ig.get_linear_forward_workspace_size(h, rows(tokens, reduced, pad), w, rows(tokens, features, pad)) < filt / 2
    w = ig.FilterDescriptor().set(F, reduced, features, 1, 1)
    assert ig.get_linear_backward_data_workspace_size(h, w, rows(tokens, reduced, pad), rows(tokens, features, pad)) < filt / 2
