"""Products whose sums are exact in fp32 whatever their order: every result is the exact one, rounded once, bit for bit. So each digit of an
activation, each code and each column counts, which bounds that grow with the number of terms do not show."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, enec, strided
from test_gpu_microscaled_moe import call as call_layer

pytestmark = pytest.mark.gpu


def product(x, w, dt, gap_x=0):
    E = enec()
    (tokens, cols), rows = x.shape, w.shape[0]
    stream = torch.from_numpy(ref.stream(w[None])).cuda()
    y = torch.empty(tokens, rows, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert E.enec_matmul_microscaled(strided(x, gap_x, float("nan")), dt, tokens, cols + gap_x, stream, stream.numel(), rows, cols, y, rows, status) == 0
    assert int(status.item()) == 0
    return y.cpu()


def rounded(exact, dt):
    """float64 values that fp32 holds, rounded once."""
    assert (exact.astype(np.float32) == exact).all()
    return torch.from_numpy(exact).to(DTYPES[dt])


def values_of_all_digits(tokens, cols, dt, g):
    """Values whose last bit is at least 2^-21 of their block's largest one's power of two, the first of each 32 (1 to 2 times it): 8 bits
    and 14 powers of two below in bf16, 11 bits and 11 powers in fp16."""
    bits, below = (8, 14) if dt == 0 else (11, 11)
    m = torch.randint(1 << (bits - 1), 1 << bits, (tokens, cols), generator=g).double() / (1 << (bits - 1))
    e = torch.randint(0, below + 1, (tokens, cols), generator=g)
    e[:, ::32] = 0
    e = e + torch.randint(0, 3, (tokens, 1), generator=g)
    sign = torch.randint(0, 2, (tokens, cols), generator=g) * 2.0 - 1
    return (m * sign * torch.exp2(-e.double())).to(DTYPES[dt])


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 5, 16, 17, 100, 300])
@pytest.mark.parametrize("cols", [32, 257, 1500])
@pytest.mark.parametrize("gap", [0, 1])
def test_every_value_of_x_alone(dt, tokens, cols, gap):
    """One weight in each row: the result is a value of x times a power of two."""
    g = torch.Generator().manual_seed(tokens + cols)
    x = values_of_all_digits(tokens, cols, dt, g)
    power = torch.exp2(torch.randint(-2, 3, (cols,), generator=g).double())
    order = torch.randperm(cols, generator=g)
    w = np.zeros((cols, cols))
    w[np.arange(cols), order] = power.numpy()
    got = product(x, w, dt, gap)
    assert torch.equal(got, rounded(x.double().numpy()[:, order] * power.numpy(), dt))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 16])
def test_values_up_to_16_tokens_count_to_2_to_the_minus_22(dt, tokens):
    """Values of any size beside a largest one whose weight is zero: off by 2^-22 of that one at most, half a unit of the last digit
    (the largest's power of two times 2^-21), and by the result's own rounding."""
    g = torch.Generator().manual_seed(tokens)
    cols = 320
    x = torch.randn(tokens, cols, generator=g) * torch.exp2(-torch.randint(0, 13 if dt else 30, (tokens, cols), generator=g).float())
    x[:, ::32] = 1 + torch.rand(tokens, cols // 32, generator=g) / 2
    x = x.clamp(-1.75, 1.75).to(DTYPES[dt])
    w = np.eye(cols)
    w[::32] = 0
    got = product(x, w, dt).double().numpy()
    want = x.double().numpy()
    want[:, ::32] = 0
    half_step = torch.finfo(DTYPES[dt]).eps / 2
    assert (np.abs(got - want) <= 2.0 ** -22 + half_step * (np.abs(want) + 2.0 ** -22)).all()


def whole_numbers(shape, g, most=8):
    return torch.randint(-most, most + 1, shape, generator=g).float()


def grid_weights(rows, cols, g):
    """All codes, with a block's first value at 6: one scale, so that the weights are what the grid says."""
    w = ref.GRID[torch.randint(0, 8, (rows, cols), generator=g).numpy()] * (torch.randint(0, 2, (rows, cols), generator=g).numpy() * 2.0 - 1)
    w[:, ::32] = 6
    return w


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols, gap", [(1, 1, 1, 0), (1, 300, 4096, 0), (3, 20, 60000, 0), (8, 48, 14336, 0), (16, 515, 2055, 1), (16, 1500, 1100, 0), (17, 515, 2055, 1),
                                                     (17, 2048, 4096, 0), (33, 640, 2300, 0), (64, 700, 5000, 8), (77, 1411, 2055, 5), (144, 150, 832, 0), (256, 300, 4100, 0),
                                                     (300, 129, 700, 3), (600, 5000, 290, 0), (520, 5100, 257, 1)])
def test_whole_numbers_times_the_grid(dt, tokens, rows, cols, gap):
    """Terms are multiples of a half up to 48, so sums of 60000 of them are below 2^24 halves."""
    g = torch.Generator().manual_seed(tokens + cols)
    x, w = whole_numbers((tokens, cols), g), grid_weights(rows, cols, g)
    x = (x / 32 if dt else x).to(DTYPES[dt])       # 60000 x 48 / 32 is within fp16's range for sums of random signs
    exact = x.double().numpy() @ w.T
    assert np.abs(exact).max() < 60000 or dt == 0
    assert torch.equal(product(x, w, dt, gap), rounded(exact, dt))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols", [(16, 48, 14336), (3, 20, 60000), (16, 700, 4100), (17, 100, 4100), (65, 20, 20000), (70, 300, 3400), (256, 5100, 1500), (300, 200, 2055)])
def test_every_record_of_long_rows_alone(dt, tokens, rows, cols):
    """Each token has values in one block of 32 columns, another one for every token and call: the first, the last, and between them. Sums have
    at most 32 terms, below 2^9."""
    g = torch.Generator().manual_seed(tokens + cols)
    w = grid_weights(rows, cols, g)
    blocks = -(-cols // 32)
    for turn in range(max(1, min(8, blocks // tokens))):
        block = torch.linspace(0, blocks - 1, tokens).round().long() if turn == 0 else torch.randint(0, blocks, (tokens,), generator=g)
        if turn == 1:   # ends and beginnings of records
            block = (8 * torch.randint(0, -(-blocks // 8), (tokens,), generator=g) - torch.randint(0, 2, (tokens,), generator=g)).clamp(0, blocks - 1)
        x = torch.zeros(tokens, blocks * 32)
        for t in range(tokens):
            x[t, 32 * block[t]:32 * block[t] + 32] = whole_numbers((32,), g)
        x = x[:, :cols].to(DTYPES[dt])
        assert torch.equal(product(x, w, dt), rounded(x.double().numpy() @ w.T, dt))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols", [(1, 1, 1), (200, 515, 2055), (129, 1411, 300), (2000, 4096, 512), (64, 100, 20000)])
def test_two_streams_of_the_grid(dt, tokens, rows, cols):
    """Terms are multiples of a quarter up to 36."""
    E = enec()
    g = torch.Generator().manual_seed(tokens + cols)
    x, w = grid_weights(tokens, cols, g), grid_weights(rows, cols, g)
    x[:, ::32] = np.where(np.arange(x[:, ::32].shape[1]) % 2, 6.0, -6.0)
    x = x / 64 if dt else x
    xs, ws = (torch.from_numpy(ref.stream(v[None])).cuda() for v in (x, w))
    y = torch.empty(tokens, rows, dtype=DTYPES[dt], device="cuda")
    assert E.enec_matmul_microscaled_both(xs, xs.numel(), tokens, ws, ws.numel(), rows, cols, dt, y, rows) == 0
    assert torch.equal(y.cpu(), rounded(x @ w.T, dt))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, width, experts", [(1, 64, 1), (4, 700, 8), (16, 300, 3), (40, 520, 5)])
def test_a_layer_that_hands_its_values_through(dt, tokens, width, experts):
    """One expert a token, so its weight is p / p = 1. gate gives 32 to every hidden value, where silu(a) = a / (1 + e^-a) is a in fp32; up and
    down have one power of two in each row. So a token's results are its values times powers of two, by the digits of x and of the
    hidden values. The router sends the tokens to the experts in turn."""
    E = enec()
    g = torch.Generator().manual_seed(tokens + width)
    x = values_of_all_digits(tokens, width, dt, g)
    x[:, 0] = 1.0
    x[:, 1:32] /= 8                                  # below 1 in the first block, and not below its last digit: all of it is exact
    x[:, 1:32] = torch.where(x[:, 1:32].abs() < 2.0 ** -9, torch.zeros(()).to(x.dtype), x[:, 1:32])
    router = torch.zeros(experts, width).to(DTYPES[dt])
    tag = width - 1 - torch.arange(experts)          # the columns that choose an expert
    x[:, tag] = 0
    chosen = torch.arange(tokens) % experts
    x[torch.arange(tokens), tag[chosen]] = 1.0
    router[torch.arange(experts), tag] = 4.0
    gate, up, down = (torch.zeros(experts, width, width).double() for _ in range(3))
    gate[:, :, 0] = 32.0
    orders = []
    for e in range(experts):
        first, second = torch.randperm(width, generator=g), torch.randperm(width, generator=g)
        p, q = (torch.exp2(torch.randint(-2, 1, (width,), generator=g).double()) for _ in range(2))
        up[e, torch.arange(width), first] = p
        down[e, torch.arange(width), second] = q
        orders.append((first, second, p, q))
    streams = [torch.from_numpy(ref.stream(w.numpy())).cuda() for w in (gate, up, down)]
    y = torch.empty(tokens, width, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert call_layer(E, x.cuda(), router.cuda(), streams, width, 1, True, dt, y, width, status=status) == 0
    assert int(status.item()) == 0
    got = y.cpu().double()

    def tops(v):
        return torch.from_numpy(np.abs(ref.blocks_of(v.numpy())).max(-1)).repeat_interleave(32)[:width]

    def on_grid(v):   # multiples of 2^-21 of their block's largest one's power of two, half of which (2^-22) is what digits round
        return v / torch.exp2(torch.floor(torch.log2(tops(v))) - 21) % 1 == 0
    half_step = torch.finfo(DTYPES[dt]).eps / 2
    for t in range(tokens):
        first, second, p, q = orders[chosen[t]]
        v = x[t].double()
        hidden, want = 32 * v[first] * p, (32 * v[first] * p)[second] * q
        # both x (a block's largest may be the 1 that chooses the expert) and the hidden values, whose neighbours `first` has exchanged, count
        # to 2^-22 of their block's largest: where both are on their grids, the result is exact
        off = ((32 * 2.0 ** -22 * tops(v)[first] * p) + 2.0 ** -22 * (1 + 2.0 ** -22) * tops(hidden))[second] * q
        assert ((got[t] - want).abs() <= off + half_step * (want.abs() + off)).all()
        exact = (on_grid(hidden) & on_grid(v)[first])[second]
        assert exact.double().mean() > 0.5 and torch.equal(got[t][exact], want[exact])
