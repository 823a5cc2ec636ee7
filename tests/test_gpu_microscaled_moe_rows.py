"""Expert layers with rows of which one token's digits leave room for two or three records of weights in flight."""
import numpy as np
import pytest
import torch

from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, enec
from test_gpu_microscaled_moe import bound_of, call, check, inputs, undecided

pytestmark = pytest.mark.gpu


# 13312 values are 52 records of columns, the last with four stages; 13568 has three, 14337 and 15000 two
@pytest.mark.parametrize("tokens", [1, 33])
@pytest.mark.parametrize("hidden, inter", [(200, 14336), (14336, 72), (13312, 40), (40, 13568), (14337, 33), (100, 15000)])
def test_rows_beyond_four_stages(tokens, hidden, inter):
    check(tokens, hidden, inter, 3, 2, tokens % 2, seed=hidden + tokens)


def test_rows_beside_large_tables():
    check(64, 15000, 16, 16, 16, 0, seed=2)
    check(64, 16, 15000, 40, 16, 0, seed=3)


@pytest.mark.parametrize("tokens", [1, 4])
def test_a_layer_of_4096_by_14336(tokens):
    E = enec()
    hidden, inter, experts, top = 4096, 14336, 2, 1 + tokens // 4
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, router, _ = inputs(tokens, hidden, 1, experts, 0, 7)
    streams, values = [], []
    for r, c in ((inter, hidden), (inter, hidden), (hidden, inter)):
        w = torch.randn(experts, r, c, generator=g, device="cuda") * c ** -0.5
        streams.append(E.quantize_tensor(w))
        values.append(E.dequantize_tensor(streams[-1], torch.float32, w.shape).cpu().double().numpy())
    y = torch.full((tokens, hidden), 5.0, dtype=DTYPES[0], device="cuda")
    status = status_tensor()
    assert call(E, x.cuda(), router.cuda(), streams, inter, top, True, 0, y, hidden, status=status) == 0
    assert int(status.item()) == 0
    x, router = x.double().numpy(), router.double().numpy()
    assert not undecided(x, router, top)[0].any()
    want, bound = bound_of(x, router, *values, top, True, 0)
    off = np.abs(y.cpu().double().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()
