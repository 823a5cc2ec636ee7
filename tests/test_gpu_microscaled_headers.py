"""Headers that do not fit a call's arguments, where there is nothing else to read: products of no columns."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, enec

pytestmark = pytest.mark.gpu


def empty_stream(rows):
    return torch.from_numpy(ref.stream(np.zeros((1, rows, 0)))).cuda()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 17, 300])
def test_products_of_no_columns_look_at_the_headers(dt, tokens):
    E = enec()
    rows = 70
    x, w = empty_stream(tokens), empty_stream(rows)
    y = torch.empty(tokens, rows + 3, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()

    def call(both, x, w):
        y.fill_(5)
        status.zero_()
        if both:
            assert E.enec_matmul_microscaled_both(x, x.numel(), tokens, w, w.numel(), rows, 0, dt, y, rows + 3, status) == 0
        else:
            assert E.enec_matmul_microscaled(None, dt, tokens, 0, w, w.numel(), rows, 0, y, rows + 3, status) == 0
        return int(status.item())
    for both in (False, True):
        assert call(both, x, w) == 0
        assert (y[:, :rows] == 0).all() and (y[:, rows:] == 5).all()
        for at in (0, 4, 8, 12, 16, 20, 24):
            bad = w.clone()
            bad[at] ^= 1
            assert call(both, x, bad) == -4 and (y == 5).all()
            if both:
                bad = x.clone()
                bad[at] ^= 1
                assert call(both, bad, w) == -4 and (y == 5).all()
