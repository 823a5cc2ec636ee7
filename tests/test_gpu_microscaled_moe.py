"""The expert layer over microscaled streams against plain numpy in 64 bits, with a bound for every value derived below."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, HALF_STEP, block_tops, enec, strided

pytestmark = pytest.mark.gpu


def silu(a):
    return a / (1 + np.exp(-a))


def undecided(x, router, top):
    """The tokens whose last chosen logit and the next one are nearer than fp32 sums may be off, and the choice that has the next one
    instead. Either choice of such a token is right."""
    logits = x @ router.T
    order = np.argsort(-logits, axis=-1, kind="stable")
    if top == router.shape[0]:
        return np.zeros(x.shape[0], dtype=bool), order
    off = (x.shape[1] + 16) * 2.0 ** -24 * (np.abs(x) @ np.abs(router).T).max(-1)
    last, following = (np.take_along_axis(logits, order[:, i:i + 1], 1)[:, 0] for i in (top - 1, top))
    return last - following <= 2 * off, np.concatenate([order[:, :top - 1], order[:, top:top + 1]], 1)


def bound_of(x, router, gate, up, down, top, renormalize, dt, chosen=None):
    """The layer in 64 bits and how far each value may be off. Products as in test_gpu_microscaled.product_bound: operands to 2^-22 of the
    largest of their block, sums of n terms in fp32 to 3 n 2^-24 of the magnitudes' sum; sums of parts of the columns add up to 8 more
    roundings. |silu'| <= 1.1; expf, the division and the products of fp32 add 2^-21 of a value at most."""
    e24 = 2.0 ** -24
    want, chosen = ref.layer(x, router, gate, up, down, top, renormalize, chosen)
    tokens, hidden = x.shape
    inter = gate.shape[1]
    logits = x @ router.T
    logit_off = (hidden + 16) * e24 * (np.abs(x) @ np.abs(router).T).max(-1)
    p = np.exp(logits - logits.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    off = np.zeros_like(want)
    x_off = 2.0 ** -22 * block_tops(x)
    for t in range(tokens):
        w = p[t, chosen[t]]
        w = w / w.sum() if renormalize else w
        for e, share in zip(chosen[t], w):
            a, u = gate[e] @ x[t], up[e] @ x[t]
            a_off, u_off = (np.abs(m[e]) @ (x_off[t] + 3 * (hidden + 24) * e24 * (np.abs(x[t]) + x_off[t])) for m in (gate, up))
            h = silu(a) * u
            h_off = 1.1 * a_off * (np.abs(u) + u_off) + (np.abs(silu(a)) + 1.1 * a_off) * u_off + 2.0 ** -21 * np.abs(h)
            rounding = 2.0 ** -22 * block_tops(np.abs(h) + h_off)
            part = down[e] @ h
            part_off = np.abs(down[e]) @ (h_off + rounding + 3 * (inter + 24) * e24 * (np.abs(h) + h_off + rounding))
            off[t] += share * (part_off + (4 * logit_off[t] + 2.0 ** -20) * (np.abs(part) + part_off))
    tiny = torch.finfo(DTYPES[dt]).smallest_normal * HALF_STEP[dt]
    return want, off + HALF_STEP[dt] * (np.abs(want) + off) + tiny


def inputs(tokens, hidden, inter, experts, dt, seed, skew=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, hidden, generator=g).to(DTYPES[dt])
    router = torch.randn(experts, hidden, generator=g) * hidden ** -0.5
    if skew:   # every token is drawn to the first experts
        router[:2] += skew * x.float().mean(0) / x.float().mean(0).norm()
    router = router.to(DTYPES[dt])
    weights = [torch.randn(experts, r, c, generator=g) * c ** -0.5 for r, c in ((inter, hidden), (inter, hidden), (hidden, inter))]
    return x, router, weights


def call(E, x, router, streams, inter, top, renormalize, dt, y, ld_y, gap=0, workspace=None, status=None):
    tokens, hidden = x.shape
    experts = router.shape[0]
    need = E.enec_moe_microscaled_workspace(tokens, hidden, inter, experts, top)
    if workspace is None:
        workspace = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    args = [a for s in streams for a in (s, s.numel())]
    return E.enec_moe_microscaled(strided(x.cpu(), gap, float("nan")) if gap else x, dt, tokens, hidden, hidden + gap, router, experts, top, renormalize,
                                  *args, inter, y, ld_y, workspace, need, status)


def check(tokens, hidden, inter, experts, top, dt, renormalize=True, gap=0, seed=1, skew=0.0):
    E = enec()
    x, router, weights = inputs(tokens, hidden, inter, experts, dt, seed, skew)
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    values = [ref.values(w.double().numpy()) for w in weights]
    y = torch.full((tokens, hidden + gap), 5.0, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert call(E, x.cuda(), router.cuda(), streams, inter, top, renormalize, dt, y, hidden + gap, gap, None, status) == 0
    got = y.cpu().double().numpy()
    assert int(status.item()) == 0
    x, router = x.double().numpy(), router.double().numpy()
    want, bound = bound_of(x, router, *values, top, renormalize, dt)
    off = np.abs(got[:, :hidden] - want)
    near = (off <= bound).all(-1)
    either, other = undecided(x, router, top)
    if (either & ~near).any():
        want, bound = bound_of(x, router, *values, top, renormalize, dt, other)
        near |= either & (np.abs(got[:, :hidden] - want) <= bound).all(-1)
    assert near.all(), (off / bound).max(-1)
    assert (got[:, hidden:] == 5).all()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 2, 8, 9, 16, 33, 64])
@pytest.mark.parametrize("experts, top", [(4, 2), (8, 1), (40, 6)])
def test_layer(dt, tokens, experts, top):
    check(tokens, 320, 192, experts, top, dt)


@pytest.mark.parametrize("hidden, inter", [(1, 1), (31, 33), (130, 515), (1000, 77), (2048, 1408)])
@pytest.mark.parametrize("tokens", [3, 20])
def test_odd_sizes(hidden, inter, tokens):
    check(tokens, hidden, inter, 3, 2 if hidden > 1 else 3, 0, seed=hidden)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("gap", [0, 3, 8])
def test_weights_and_rows_apart(dt, renormalize, gap):
    check(6, 200, 100, 16, 3, dt, renormalize, gap)


@pytest.mark.parametrize("tokens", [12, 64])
def test_an_expert_of_all_tokens(tokens):
    """More pairs of one expert than a group holds; other experts without any."""
    check(tokens, 256, 160, 16, 2, 0, skew=8.0)


def test_all_experts_of_one_and_many_experts():
    check(5, 128, 64, 1, 1, 0)
    check(5, 128, 64, 16, 16, 1)
    check(20, 96, 40, 512, 8, 0, seed=4)


@pytest.mark.parametrize("tokens, experts, top", [(64, 384, 16), (48, 512, 16), (1, 512, 16), (64, 1, 1)])
def test_the_limits_of_tokens_and_experts(tokens, experts, top):
    check(tokens, 72, 40, experts, top, 0, seed=tokens)


def test_rows_that_do_not_fit_are_refused():
    E = enec()
    for hidden, inter in ((20000, 64), (64, 20000)):
        x, router = torch.zeros(1, hidden, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, hidden, dtype=torch.bfloat16, device="cuda")
        streams = [torch.zeros(E.enec_microscaled_size(1, r, c), dtype=torch.uint8, device="cuda") for r, c in ((inter, hidden),) * 2 + ((hidden, inter),)]
        y = torch.full((1, hidden), 5.0, dtype=torch.bfloat16, device="cuda")
        assert call(E, x, router, streams, inter, 1, True, 0, y, hidden) == -8
        torch.cuda.synchronize()
        assert (y == 5).all()


def test_long_rows():
    """Rows of which eight do not fit beside one another: smaller groups, both in front of and behind the activation."""
    check(16, 9000, 64, 2, 1, 0)
    check(16, 64, 9001, 2, 1, 1)


def test_ties_go_to_the_lower_expert():
    E = enec()
    x, router, weights = inputs(5, 256, 64, 12, 0, 9)
    router[3] = router[7]
    router[11] = router[7]
    router[[3, 7, 11]] += 4 * x.float().mean(0) / x.float().mean(0).norm() * x.float().mean(0).norm()
    router = router.to(torch.bfloat16)
    router[3] = router[7]
    router[11] = router[7]
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    y = [torch.empty(5, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert call(E, x.cuda(), router.cuda(), streams, 64, 2, True, 0, y[0], 256) == 0
    # with the weights of every expert above the second of the equals made NaN, a token that chose by the rule is not touched
    logits = x.double() @ router.double().t()
    order = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :2]
    unused = [e for e in range(12) if e not in order]
    for s, w in zip(streams, weights):
        w[unused] = float("nan")
    dirty = [E.quantize_tensor(w.cuda()) for w in weights]
    assert call(E, x.cuda(), router.cuda(), dirty, 64, 2, True, 0, y[1], 256) == 0
    assert 11 in unused and torch.equal(y[0], y[1])


def test_nan_stays_in_its_token():
    E = enec()
    x, router, weights = inputs(6, 256, 64, 8, 0, 3)
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    y = [torch.empty(6, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert call(E, x.cuda(), router.cuda(), streams, 64, 2, True, 0, y[0], 256) == 0
    x[2, 100] = float("nan")
    assert call(E, x.cuda(), router.cuda(), streams, 64, 2, True, 0, y[1], 256) == 0
    assert torch.isnan(y[1][2]).all()
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(y[0][keep], y[1][keep])


@pytest.mark.parametrize("which", [0, 1, 2])
def test_wrong_headers_leave_the_output(which):
    E = enec()
    x, router, weights = inputs(6, 256, 64, 8, 0, 3)
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    streams[which][16] += 1
    y = torch.full((6, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    status = status_tensor()
    assert call(E, x.cuda(), router.cuda(), streams, 64, 2, True, 0, y, 256, status=status) == 0
    assert int(status.item()) == -4 and (y == 5).all()


@pytest.mark.parametrize("tokens", [2, 30])
def test_repeated_captured_and_concurrent_calls_agree_bit_for_bit(tokens):
    E = enec()
    x, router, weights = inputs(tokens, 512, 256, 8, 0, 3)
    x, router = x.cuda(), router.cuda()
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    need = E.enec_moe_microscaled_workspace(tokens, 512, 256, 8, 2)
    ys = [torch.zeros(tokens, 512, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    spaces = [torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(4)]

    def run(i):
        assert call(E, x, router, streams, 256, 2, True, 0, ys[i], 512, workspace=spaces[i]) == 0
    run(0)
    run(0)
    torch.cuda.synchronize()
    for i in (1, 2):
        s = torch.cuda.Stream(priority=-1)
        with torch.cuda.stream(s):
            run(i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(3)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(ys[0], y) for y in ys[1:])
