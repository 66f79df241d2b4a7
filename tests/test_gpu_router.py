"""The router and its gradient on the GPU against plain implementations in 64
bits: every width of a row, types, scores, groups, biases, strides, masked
and unusual logits, from one token to many.

Ids have one right value.  Weights: the kernel forms exp(d) as 2^(d log2 e),
so rounding the product costs |d| 2^-24 relative, at most 4e-6 for the |d|
< 64 drawn here; sums, the quotient and the exponential add a few 2^-24: 1e-5
relative, and 1e-30 where a score is next to nothing.  Gradients are
differences of such terms, each at most c max|dw|: 1e-5 of that absolute,
and half a unit in the last place of the logits' type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe, topoep  # noqa: E402

DEV = torch.device("cuda:0")
NEG = float("-inf")
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def clean(x):
    return torch.nan_to_num(x.double().cpu(), nan=NEG, posinf=torch.finfo(torch.float32).max, neginf=NEG)


def ref_ids(logits, k, bias, groups, top_groups):
    """numpy's sort on (closed group, key descending, id ascending)."""
    x = clean(logits).float()
    key = x + bias.cpu() if bias is not None else x
    key = torch.where(torch.isnan(key), NEG, key).numpy()
    T, E = key.shape
    col = np.broadcast_to(np.arange(E), (T, E))
    best = key.reshape(T, groups, E // groups).max(2)
    order = np.lexsort((np.broadcast_to(np.arange(groups), best.shape), -best))[:, :top_groups]
    open_ = np.zeros((T, groups), dtype=bool)
    np.put_along_axis(open_, order, True, 1)
    closed = ~np.repeat(open_, E // groups, axis=1)
    return torch.from_numpy(np.lexsort((col, -key, closed))[:, :k].copy())


def ref_scores(x, ids, scoring, renorm):
    at = x.gather(1, ids)
    if scoring == "sigmoid":
        s = torch.sigmoid(at)
        return torch.nan_to_num(s / s.sum(1, keepdim=True), nan=0.0) if renorm else s
    if renorm:
        return torch.nan_to_num(torch.softmax(at, 1), nan=0.0)
    return torch.nan_to_num(torch.softmax(x, 1), nan=0.0).gather(1, ids)


def check(logits, k, scoring="softmax", renorm=True, scale=1.0, bias=None, groups=1, top_groups=1):
    kw = dict(scoring=scoring, renorm=renorm, scale=scale)
    print("router", tuple(logits.shape), logits.dtype, k, kw, groups, top_groups, bias is not None, flush=True)
    ids, weights = moe.route(logits, k, bias=bias, groups=groups, top_groups=top_groups, **kw)
    torch.cuda.synchronize()
    want = ref_ids(logits, k, bias, groups, top_groups)
    assert torch.equal(ids.cpu().long(), want)
    ref = scale * ref_scores(clean(logits), want, scoring, renorm)
    err = (weights.cpu().double() - ref).abs()
    assert bool((err <= 1e-5 * ref.abs() + 1e-30).all()), float(err.max())
    g = torch.randn(weights.shape, generator=torch.Generator().manual_seed(5))
    grad = moe.route_backward(logits, ids, g.to(DEV), **kw)
    torch.cuda.synchronize()
    x = clean(logits).requires_grad_()
    s = ref_scores(x, want, scoring, renorm)
    (scale * s * g.double()).sum().backward()
    ref = torch.nan_to_num(x.grad, nan=0.0)   # rows with every logit masked: no gradient
    err = (grad.cpu().double() - ref).abs()
    most = abs(scale) * float(g.abs().max()) if g.numel() else 0.0
    assert grad.dtype == logits.dtype and grad.shape == logits.shape
    assert bool((err <= 1e-5 * most + HALF_UNIT[logits.dtype] * ref.abs() + 6e-8 * (logits.dtype == torch.float16))
                .all()), float(err.max())
    return ids, weights


def draw(T, E, dtype=torch.float32, seed=0, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 977 * T + E)
    return torch.randn((T, E + extra), generator=g, device=DEV).mul_(2.0).to(dtype)[:, :E]


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (8, 2), (15, 4), (16, 8), (17, 3), (33, 16), (60, 6), (64, 8), (65, 8),
                                 (100, 17), (128, 8), (160, 8), (255, 8), (256, 64), (320, 6), (511, 8), (512, 8),
                                 (640, 8), (1023, 32), (1024, 64)])
@pytest.mark.parametrize("T", [1, 7, 300])
def test_every_width(E, k, T):
    check(draw(T, E), k)
    check(draw(T, E, seed=1), k, renorm=False)


@pytest.mark.parametrize("E,k,T", [(8, 2, 70001), (16, 16, 33000), (37, 5, 20011), (100, 8, 20011), (128, 8, 20011),
                                   (200, 6, 20011), (256, 8, 20011), (300, 8, 20011)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens(E, k, T, dtype):
    x = draw(T, E, dtype)
    x[-1000:] = NEG
    x[::37, ::3] = NEG
    check(x, k, renorm=False)
    check(x, k, scoring="sigmoid", scale=2.5)
    if E % 4 == 0:
        check(x, min(k, E // 2), bias=torch.randn(E, generator=torch.Generator().manual_seed(1)).to(DEV), groups=4,
              top_groups=2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("extra", [0, 3])
def test_types_scores_and_strides(dtype, scoring, renorm, extra):
    for T, E, k in ((5, 128, 8), (129, 96, 4), (9000, 64, 6)):
        check(draw(T, E, dtype, extra=extra), k, scoring=scoring, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("E,groups,top_groups,k", [(16, 4, 1, 4), (16, 16, 3, 2), (60, 5, 2, 8), (64, 64, 9, 9),
                                                   (256, 4, 2, 8), (256, 32, 4, 8), (320, 32, 4, 8), (512, 32, 4, 8),
                                                   (640, 64, 64, 8), (1024, 8, 3, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_groups_with_a_bias(E, groups, top_groups, k, dtype):
    x = draw(203, E, dtype)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).to(DEV)
    check(x, k, bias=bias, groups=groups, top_groups=top_groups)
    check(x, k, scoring="sigmoid", groups=groups, top_groups=top_groups)
    x[:, : E // groups * (groups - 1)] = NEG   # one group left with anything in it
    x[100:] = NEG
    check(x, k, renorm=False, bias=bias, groups=groups, top_groups=top_groups)


@pytest.mark.parametrize("E", [16, 130, 512])
@pytest.mark.parametrize("scoring,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True)])
def test_ties_masks_and_unusual_logits(E, scoring, renorm):
    low, inf, nan = torch.finfo(torch.float32).min, float("inf"), float("nan")
    x = draw(16, E)
    x[0] = 0.0                      # all equal
    x[1] = NEG                      # nothing left
    x[2] = low                      # the type's lowest value is a logit like others
    x[3] = nan
    x[4, :] = NEG
    x[4, E - 1] = 1.0               # one expert left
    x[5, ::2] = nan
    x[6, 3] = inf
    x[7] = inf
    x[8, ::2] = 0.0
    x[8, 1::2] = -0.0               # one key
    x[9] = x[9].round()             # many ties
    x[10] = low
    x[10, 5] = NEG
    x[11] = torch.where(x[11] > 0, x[11], NEG)
    check(x, 8, scoring=scoring, renorm=renorm)
    bias = torch.zeros(E, device=DEV)
    bias[2], bias[7] = nan, 100.0
    check(x, 8, scoring=scoring, renorm=renorm, bias=bias)


def test_gradient_against_differences():
    """A step of 2^-6 in single logits of 64-bit inputs' nearest 32-bit ones:
    central differences of the weights the kernel gives (error of the
    difference: step^2 / 6 times a third derivative below 1, and the weights'
    2e-6 over the step: 2e-4)."""
    T, E, k = 4, 24, 5
    x = draw(T, E)
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(3)).to(DEV)
    for kw in (dict(), dict(renorm=False), dict(scoring="sigmoid"), dict(scoring="sigmoid", renorm=False)):
        ids, _ = moe.route(x, k, **kw)
        got = moe.route_backward(x, ids, g, **kw)
        top, step = x.gather(1, ids.long()), 2.0 ** -6
        gap = (top[:, k - 1] - x.masked_fill(torch.zeros_like(x, dtype=torch.bool).scatter(1, ids.long(), True), NEG)
               .amax(1)).min()
        order = (top[:, :-1] - top[:, 1:]).min()
        step = min(step, float(gap) / 4, float(order) / 4)   # the choice stays
        for e in range(E):
            hi, lo = x.clone(), x.clone()
            hi[:, e] += step
            lo[:, e] -= step
            ih, wh = moe.route(hi, k, **kw)
            il, wl = moe.route(lo, k, **kw)
            assert torch.equal(ih, ids) and torch.equal(il, ids)
            want = ((wh - wl).double() * g.double()).sum(1) / (hi[:, e] - lo[:, e]).double()
            bound = k * float(g.abs().max()) * (step ** 2 / 6 + 4e-6 / step)
            assert bool(((got[:, e] - want).abs() <= bound).all()), (kw, e)


def test_autograd_and_the_planner_take_the_ids():
    """The weights' gradient reaches the logits, and a planner takes the ids as
    they come."""
    T, E, k, R = 512, 16, 2, 8
    x = draw(T, E).requires_grad_()
    ids, w = moe.route(x, k)
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(3)).to(DEV)
    (w * g).sum().backward()
    assert torch.equal(x.grad, moe.route_backward(x.detach(), ids, g))
    topo = topoep.topology(R, 4, E, 0, 1, 4, 4096, 1 << 20)
    omega = torch.zeros((R, E), dtype=torch.int32, device=DEV)
    omega[0] = torch.bincount(ids.view(-1), minlength=E).to(torch.int32)
    _, dest, send, status = topoep.plan(topo, omega, ids, 1)
    torch.cuda.synchronize()
    assert int(status[0]) == 0 and int(send.sum()) == T * k and int(dest.min()) >= 0


def test_no_tokens_and_refusals():
    ids, w = moe.route(torch.empty((0, 16), device=DEV), 4)
    assert ids.shape == (0, 4) and w.shape == (0, 4)
    x = draw(4, 16)
    with pytest.raises(TypeError):
        moe.route(x.double(), 4)
    with pytest.raises(TypeError):
        moe.route(x.cpu(), 4)
    with pytest.raises(ValueError):
        moe.route(x.t(), 4)
    with pytest.raises(ValueError):
        moe.route(x, 4, scoring="tanh")
    with pytest.raises(ValueError):
        moe.route(x, 4, bias=torch.zeros(15, device=DEV))
    with pytest.raises(topoep.TopoepError):
        moe.route(x, 17)
    with pytest.raises(topoep.TopoepError):
        moe.route(x, 5, groups=4)   # one open group of four experts
    ids, _ = moe.route(x, 4)
    with pytest.raises(TypeError):
        moe.route_backward(x, ids.long(), torch.zeros(4, 4, device=DEV))
    with pytest.raises(ValueError):
        moe.route_backward(x, ids, torch.zeros(4, 3, device=DEV))


def test_equal_calls_equal_bits_on_another_stream_and_in_a_graph():
    x = draw(9001, 96, torch.bfloat16)
    first = moe.route(x, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = moe.route(x, 8, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = moe.route(x, 8)
        back = moe.route_backward(x, third[0], third[1])
    for seed in range(3):
        x.copy_(draw(9001, 96, torch.bfloat16, seed=seed + 50))
        graph.replay()
        torch.cuda.synchronize()
        want = moe.route(x, 8)
        assert all(torch.equal(a, b) for a, b in zip(third, want))
        assert torch.equal(back, moe.route_backward(x, *want))
