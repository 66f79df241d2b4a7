"""The experts' products as they are used together: behind the router in a
training step, as a chain of 8-bit products, from streams and captured graphs."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ffnmodel  # noqa: E402
from paper_2609_35481_amd import ffn, moe, train_decode  # noqa: E402
from test_gpu_ffn import case, gradients, run_experts  # noqa: E402
from test_gpu_int8 import product, weights as int8_weights  # noqa: E402

DEV = torch.device("cuda:0")
BF16 = torch.bfloat16


def test_router_experts_and_clip():
    """Gradients through the experts and the router: the logits' against the router's formula in 64 bits on
    the weights' gradient that the experts give (within its bound, times the slope at most 1)."""
    x, _, _, up, down, _, dout = case(200, 64, 48, 8, 8, 2, BF16, seed=5)
    gate = (torch.randn(8, 64, generator=torch.Generator().manual_seed(1)) * 0.2).to(DEV).requires_grad_()
    up, down = up.to(DEV).requires_grad_(), down.to(DEV).requires_grad_()
    logits = x.to(DEV).float() @ gate.t()
    logits.retain_grad()
    ids, weights = moe.route(logits, 2)
    weights.retain_grad()
    out = ffn.experts(x.to(DEV), ids, weights, up, down)
    out.backward(dout.to(DEV))
    want = ffnmodel.layer(x, ids, weights, up, down, None, dout)
    for name, got in (("out", out), ("weights", weights.grad), ("up", up.grad), ("down", down.grad)):
        ffnmodel.within(got, *want[name], name)
    w, dw = weights.detach().cpu().double(), weights.grad.cpu().double()
    d = w * (dw - (dw * w).sum(1, keepdim=True))
    full = torch.zeros(200, 8, dtype=torch.float64).scatter(1, ids.cpu().long(), d)
    # the weights to 32 bits (2^-22 of them with their sum), their products and differences
    bound = 16 * ffnmodel.E32 * (dw.abs().amax(1, keepdim=True) + 1e-30).expand_as(full)
    ffnmodel.within(logits.grad, full, bound, "logits")
    grads = [gate.grad, up.grad, down.grad]
    before = [g.clone() for g in grads]
    norm = moe.clip_grads(grads, 0.5)
    exact = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    assert abs(float(norm) - exact) <= 1e-6 * exact and exact > 0.5
    for g, b in zip(grads, before):
        assert bool((g.float().abs() <= b.float().abs()).all()) and bool(g.any())


def test_gradients_accumulate_and_saved_tensors_are_watched():
    x, ids, weights, up, down, slot, dout = (v.to(DEV) for v in case(60, 64, 32, 8, 8, 2, BF16, seed=7))
    for t in (x, weights, up, down):
        t.requires_grad_()
    ffn.experts(x, ids, weights, up, down, slot).backward(dout)
    once = {n: t.grad.clone() for n, t in (("x", x), ("up", up), ("weights", weights))}
    ffn.experts(x, ids, weights, up, down, slot).backward(dout)
    assert torch.equal(x.grad, once["x"] * 2) and torch.equal(up.grad, once["up"] * 2)
    assert torch.equal(weights.grad, once["weights"] * 2)
    out = ffn.experts(x, ids, weights, up, down, slot)
    with torch.no_grad():
        up.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward(dout)
    with torch.inference_mode():
        assert torch.isfinite(ffn.experts(x, ids, weights, up, down, slot)).all()


def test_serving_chain_in_8_bits():
    """Router's choices -> rows by expert -> quantised gate and up -> quantised down -> sum, each product against 64
    bits on what the one before gave."""
    T, H, I, E, k = 50, 64, 96, 12, 3
    x, ids, weights, *_ = case(T, H, I, E, E, k, BF16, seed=9)
    (wu, su), (wd, sd) = int8_weights(1, E, 2 * I, H), int8_weights(2, E, H, I)
    offsets, pairs, places = ffn.expert_rows(ids.to(DEV), E)
    rows = x.to(DEV)[pairs.long() // k]
    q, s = ffn.quantize(rows)
    h = ffn.matmul_int8((q, s), wu.to(DEV), su.to(DEV), offsets, gated=True)
    ffnmodel.within(h, *product(q.cpu(), s.cpu(), wu, su, offsets.cpu(), True, BF16), "hidden")
    assert torch.equal(h, ffn.matmul_int8(rows, wu.to(DEV), su.to(DEV), offsets, gated=True))
    q, s = ffn.quantize(h)
    y = ffn.matmul_int8((q, s), wd.to(DEV), sd.to(DEV), offsets, dtype=torch.float32)
    ffnmodel.within(y, *product(q.cpu(), s.cpu(), wd, sd, offsets.cpu(), False, torch.float32), "output")
    out = (y[places.long()] * weights.to(DEV)[:, :, None]).sum(1)
    # the same layer with the weights as they are held: rows and hidden values are off by up to half a step, 1 / 254
    # of their largest (2.4 and about 6 times their size here), 0.58 of that on average: 0.6 and 1.4 %
    full = ffnmodel.layer(x, ids, weights, (wu.float() * su[..., None]).to(BF16), (wd.float() * sd[..., None]).to(BF16))
    ref = full["out"][0]
    assert float((out.cpu().double() - ref).norm() / ref.norm()) < 0.03


@pytest.mark.parametrize("T,H,I,E,L,k", [(1, 64, 32, 8, 8, 2), (40, 128, 64, 8, 5, 2), (700, 64, 128, 16, 16, 4)])
def test_streams_give_the_same(T, H, I, E, L, k):
    c = case(T, H, I, E, L, k, BF16, seed=11)
    want = run_experts(*c)
    x, ids, weights, up, down, slot, dout = (v.to(DEV) for v in c)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:                                    # two calls at once
        t = {"x": x.clone().requires_grad_(), "weights": weights.clone().requires_grad_(),
             "up": up.clone().requires_grad_(), "down": down.clone().requires_grad_()}
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            out = ffn.experts(t["x"], ids, t["weights"], t["up"], t["down"], slot)
            got.append({"out": out, **gradients(out, dout, **t)})
    named = torch.cuda.Stream()
    named.wait_stream(torch.cuda.current_stream())
    alone = ffn.experts(x, ids, weights, up, down, slot, stream=named)
    rows = ffn.expert_rows(ids, L, slot, stream=named)
    named.synchronize()
    for s in streams:
        s.synchronize()
    assert torch.equal(alone, want["out"])
    assert all(torch.equal(a, b) for a, b in zip(rows, ffn.expert_rows(ids, L, slot)))
    for g in got:
        for name in want:
            assert torch.equal(g[name], want[name]), name


def test_captured_calls_replay_alike():
    """A training step and an 8-bit chain in two graphs, replayed in turn with other inputs and eager work between."""
    x, ids, weights, up, down, slot, dout = (v.to(DEV) for v in case(150, 64, 96, 12, 8, 3, BF16, seed=13))
    (wu, su), (wd, sd) = int8_weights(1, 192, 64), int8_weights(2, 64, 96)
    wu, su, wd, sd = (v.to(DEV) for v in (wu, su, wd, sd))
    leaves = {"x": x.clone().requires_grad_(), "weights": weights.clone().requires_grad_(),
              "up": up.clone().requires_grad_(), "down": down.clone().requires_grad_()}

    def step():
        out = ffn.experts(leaves["x"], ids, leaves["weights"], leaves["up"], leaves["down"], slot)
        return {"out": out.detach(), **gradients(out, dout, **leaves)}

    def chain():
        with torch.no_grad():
            return ffn.matmul_int8(ffn.matmul_int8(leaves["x"], wu, su, gated=True), wd, sd)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(), chain()
    torch.cuda.current_stream().wait_stream(side)
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        held = step()
    with torch.cuda.graph(second):
        held_chain = chain()
    for i in range(4):
        with torch.no_grad():
            leaves["x"].copy_(torch.roll(x, i, 0))
            ids.copy_(torch.roll(ids, 1, 0))
            leaves["weights"].mul_(0.9)
        first.replay(), second.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in held.items()}
        got_chain = held_chain.clone()
        want = step()
        assert torch.equal(got_chain, chain()), i
        for name in want:
            assert torch.equal(got[name], want[name]), (i, name)


def test_example_trains_through_the_kernels():
    lines = []
    losses, norms, off, off8 = train_decode.run(steps=5, log=lines.append, half=True)
    print("\n".join(lines), flush=True)
    assert all(math.isfinite(v) for v in losses + norms) and min(norms) > 0
    # rows and hidden values to 8 bits of their largest: half a step each is 2^-8 of it, sums of 256 and 128 terms
    assert off < 2.0 ** -6 and off8 < 2.0 ** -4
