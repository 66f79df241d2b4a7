"""The layer for a few tokens on the GPU against a plain implementation in 64
bits, expert by expert.

Tolerance of an output, from how the kernel rounds: each hidden value is
rounded to the weights' type (half a unit in the last place, relative u), which
moves an output by at most u B, B = sum_j |w_j| sum_i |down_i| |h_i|; the sums
in 32 bits behind a hidden value err by at most about sqrt(H) 2^-23 of
sum |W| |x| each, far below u of it at these sizes, so another u B covers
them; rounding the output itself costs u |out|.  u = 2^-8 (bf16), 2^-10 (f16),
twice the half unit.  Router weights: 1e-4, from 32-bit logits of up
to sqrt(H) 2^-23 sum |gate| |x| error."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe, topoep  # noqa: E402

DEV = torch.device("cuda:0")
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def inputs(T, H, I, E, L, dtype=torch.bfloat16, seed=0, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed * 131 + T * 7 + H)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)

    x = normal(T, H + extra)[:, :H]
    return (x, normal(E, H, std=H ** -0.5), normal(L, 2 * I, H, std=H ** -0.5), normal(L, H, I, std=I ** -0.5))


def spread(E, L, seed=0):
    """Slots of L experts among E in no order, the others elsewhere (-1, or beyond L)."""
    g = torch.Generator().manual_seed(seed + 3)
    order = torch.randperm(E, generator=g)
    slot = torch.where(torch.arange(E) % 2 == 0, -1, L + 5).to(torch.int32)
    slot[order[:L]] = torch.randperm(L, generator=g).to(torch.int32)
    return slot.to(DEV)


def check(x, gate, up, down, k, slot=None, ws=None, got=None, **kw):
    T, H = x.shape
    E, (L, _, I) = gate.shape[0], down.shape
    print("layer", T, H, I, E, L, k, x.dtype, kw, flush=True)
    out, ids, w = got or moe.moe_few(x, gate, up, down, k, expert_slot=slot, workspace=ws, **kw)
    torch.cuda.synchronize()
    logits = x.double() @ gate.double().t()
    # the ids: a choice that the 64-bit logits confirm up to the logits' 32-bit error
    err = 2.0 ** -20 * float((x.double().abs() @ gate.double().abs().t()).max()) if T else 0.0
    key = logits + (kw["bias"].double() if kw.get("bias") is not None else 0.0)
    assert ids.dtype == torch.int32 and bool((ids >= 0).all()) and bool((ids < E).all())
    at = ids.long()
    chosen = key.gather(1, at)
    assert bool((chosen[:, 1:] <= chosen[:, :-1] + err).all())
    rest = key.scatter(1, at, float("-inf"))
    if kw.get("groups", 1) == 1 and T and k < E:
        assert bool((rest.amax(1) <= chosen[:, -1] + err).all())
    assert all(len(set(r)) == k for r in at.tolist())
    score = logits.gather(1, at)
    if kw.get("scoring", "softmax") == "sigmoid":
        s = torch.sigmoid(score)
        s = s / s.sum(1, keepdim=True) if kw.get("renorm", True) else s
    else:
        s = torch.softmax(score, 1) if kw.get("renorm", True) else torch.softmax(logits, 1).gather(1, at)
    want_w = kw.get("scale", 1.0) * s
    assert bool(((w - want_w).abs() <= 1e-4 * want_w).all())
    want, bound = torch.zeros_like(x, dtype=torch.float64), torch.zeros_like(x, dtype=torch.float64)
    place = slot.long()[at] if slot is not None else at
    place = torch.where((place >= 0) & (place < L), place, -1)
    for e in range(L):
        share = torch.where(place == e, want_w, 0.0).sum(1, keepdim=True)
        if bool((share != 0).any()):
            a = x.double() @ up[e].double().t()
            h = a[:, :I] * torch.sigmoid(a[:, :I]) * a[:, I:]
            want += share * (h @ down[e].double().t())
            bound += share.abs() * (h.abs() @ down[e].double().abs().t())
    assert out.dtype == x.dtype and out.shape == x.shape
    off = (out.double() - want).abs()
    u = UNIT[x.dtype]
    assert bool((off <= (2 * u + 2e-4) * bound + u * want.abs()).all()), float((off / (bound + 1e-9)).max())
    return out, ids, w


@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_token_counts(T, dtype):
    check(*inputs(T, 256, 128, 16, 16, dtype), 2)
    check(*inputs(T, 264, 72, 37, 5, dtype), 4, slot=spread(37, 5), scoring="sigmoid", scale=2.5)


@pytest.mark.parametrize("H,I", [(8, 8), (16, 24), (40, 8), (32, 136), (520, 40), (1000, 328), (2048, 768), (4096, 48),
                                 (72, 2056)])
def test_sizes(H, I):
    for T in (1, 5, 34):
        check(*inputs(T, H, I, 24, 24), 3)
        check(*inputs(T, H, I, 24, 7, torch.float16), 3, slot=spread(24, 7))


@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (3, 3), (8, 8), (64, 8), (65, 6), (130, 8), (256, 8), (300, 33),
                                 (512, 8), (640, 4), (1000, 64)])
def test_experts(E, k):
    for T in (1, 9, 70):
        check(*inputs(T, 64, 32, E, E), k, renorm=False)
        check(*inputs(T, 64, 32, E, 1), k, slot=spread(E, 1))


def test_every_token_on_one_expert():
    """All columns in one expert's tiles, the other experts empty."""
    for T in (1, 16, 48, 128):
        x, gate, up, down = inputs(T, 128, 64, 32, 32)
        bias = torch.zeros(32, device=DEV)
        bias[11] = 100.0
        _, ids, _ = check(x, gate, up, down, 1, bias=bias)
        assert bool((ids == 11).all())
        check(x, gate, up, down, 2, bias=bias, scoring="sigmoid", renorm=False)


def test_groups():
    E = 64
    bias = torch.randn(E, generator=torch.Generator().manual_seed(4)).to(DEV)
    for T in (1, 21):
        _, ids, _ = check(*inputs(T, 96, 64, E, 20), 6, slot=spread(E, 20), groups=8, top_groups=2, bias=bias)
        assert all(len(set(r)) <= 2 for r in (ids // 8).tolist())


def test_no_expert_here_gives_zeros():
    x, gate, up, down = inputs(7, 64, 32, 12, 3)
    out, ids, w = moe.moe_few(x, gate, up, down, 2, expert_slot=torch.full((12,), -1, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert not bool(out.any()) and bool((w > 0).all())


def test_two_experts_at_one_place():
    """An expert map may name one place twice: both experts' pairs are served."""
    x, gate, up, down = inputs(19, 64, 32, 4, 1)
    check(x, gate, up, down, 4, slot=torch.zeros(4, dtype=torch.int32, device=DEV))


def test_row_stride_and_no_tokens():
    check(*inputs(6, 128, 64, 16, 16, extra=8), 2)
    x, gate, up, down = inputs(0, 128, 64, 16, 16)
    out, ids, w = moe.moe_few(x, gate, up, down, 2)
    assert out.shape == (0, 128) and ids.shape == (0, 2) and w.shape == (0, 2)


def test_masked_places_do_not_leak():
    """Infinities and NaN in experts that no token picks, in tokens' neighbours
    and behind the rows' ends reach no output."""
    x, gate, up, down = inputs(5, 72, 40, 8, 8, extra=8)
    bias = torch.zeros(8, device=DEV)
    bias[5] = -1e30
    up[5], down[5] = float("nan"), float("inf")
    base = x.as_strided((5, 80), (80, 1))
    base[:, 72:] = float("nan")
    _, ids, _ = check(x, gate, up[:], down, 3, bias=bias)
    x2 = x.clone()
    x2[2] = float("inf")    # one token's own outputs, not the others'
    out, ids2, _ = moe.moe_few(x2, gate, up, down, 3, bias=bias)
    rows = [0, 1, 3, 4]
    same = moe.moe_few(x, gate, up, down, 3, bias=bias)[0]
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out[rows]).all()) and torch.equal(out[rows], same[rows])


def test_hidden_values_beyond_f16_saturate():
    x, gate, up, down = inputs(3, 64, 32, 4, 4, torch.float16)
    out, _, _ = moe.moe_few(x * 100, gate, up * 50, down * 1e-3, 2)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all())


def test_one_workspace_for_many_sizes_equal_bits():
    """Calls of other sizes leave a shared workspace ready; equal calls give equal bits."""
    need = max(moe.moe_workspace_bytes(H, I, E, E, k, 128) for H, I, E, k in ((512, 256, 64, 8), (128, 64, 300, 4)))
    ws = torch.zeros(need + 256, dtype=torch.uint8, device=DEV)
    a, b = inputs(128, 512, 256, 64, 64), inputs(3, 128, 64, 300, 300)
    first = [t.clone() for t in check(*a, 8, ws=ws)]
    check(*b, 4, ws=ws)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, moe.moe_few(*a, 8, workspace=ws)))
        moe.moe_few(*b, 4, workspace=ws)
    with pytest.raises(topoep.TopoepError):
        moe.moe_few(*a, 8, workspace=ws[:4096])


def test_graph_replays_and_another_stream():
    x, gate, up, down = inputs(9, 256, 128, 32, 32)
    ws = torch.zeros(moe.moe_workspace_bytes(256, 128, 32, 32, 4, 9) + 256, dtype=torch.uint8, device=DEV)
    ws2 = torch.zeros_like(ws)
    moe.moe_few(x, gate, up, down, 4, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = moe.moe_few(x, gate, up, down, 4, workspace=ws)
    for seed in range(4):
        x.copy_(inputs(9, 256, 128, 32, 32, seed=seed + 9)[0])
        graph.replay()
        torch.cuda.synchronize()
        want = moe.moe_few(x, gate, up, down, 4, workspace=ws2)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), seed
    check(x, gate, up, down, 4, got=got)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = moe.moe_few(x, gate, up, down, 4, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(other, got))


def test_refusals():
    x, gate, up, down = inputs(4, 64, 32, 8, 8)
    with pytest.raises(TypeError):
        moe.moe_few(x.float(), gate.float(), up.float(), down.float(), 2)
    with pytest.raises(TypeError):
        moe.moe_few(x, gate.half(), up, down, 2)
    with pytest.raises(ValueError):
        moe.moe_few(x, gate, up[:, :-8], down, 2)
    with pytest.raises(ValueError):
        moe.moe_few(x, gate, up.transpose(1, 2).contiguous().transpose(1, 2), down, 2)
    with pytest.raises(TypeError):
        moe.moe_few(x, gate, up, down, 2, expert_slot=torch.zeros(8, dtype=torch.int64, device=DEV))
    with pytest.raises(topoep.TopoepError):
        moe.moe_few(x, gate, up, down, 9)
    with pytest.raises(topoep.TopoepError):
        moe.moe_few(torch.cat([x] * 33), gate, up, down, 2)
    with pytest.raises(topoep.TopoepError):   # rows of 63 elements
        moe.moe_few(*inputs(4, 60, 32, 8, 8), 2)
