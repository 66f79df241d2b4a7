"""The global gradient norm and the clip on the GPU against 64-bit sums.

The kernel forms and sums squares in 64 bits, so the norm is the 64-bit one
rounded to 32 (2^-24 relative; 2^-23 allowed).  A clipped value is rounded
after the norm, the norm + 1e-6, the quotient, the factor and the product:
five times 2^-24 relative, and half a unit in the last place of the output's
type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe, topoep  # noqa: E402

DEV = torch.device("cuda:0")
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def tensors(sizes, dtype, seed=0, std=1.0, shift=0):
    """Views of one buffer, `shift` elements between them."""
    g = torch.Generator(device=DEV).manual_seed(seed + len(sizes))
    flat = torch.randn((sum(sizes) + shift * (len(sizes) + 1),), generator=g, device=DEV).mul_(std).to(dtype)
    out, at = [], shift
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + shift
    return out


def ref_norm(grads, ord=2):
    if not grads:
        return 0.0
    parts = [g.double().abs().max() if ord != 2 else g.double().square().sum() for g in grads if g.numel()]
    if not parts:
        return 0.0
    v = torch.stack(parts)
    return float(v.sum().sqrt() if ord == 2 else v.max())


def check_clip(grads, outs, before, max_norm, scale=1.0, ord=2, norm=None):
    got = moe.clip_grads(grads, max_norm, scale=scale, ord=ord, outs=outs, norm=norm)
    torch.cuda.synchronize()
    want = scale * ref_norm(before, ord) if norm is None else float(norm)
    assert abs(float(got) - want) <= 2.0 ** -23 * want
    f = scale * min(1.0, max_norm / (want + 1e-6))
    for o, b in zip(outs if outs is not None else grads, before):
        w = b.double() * f
        tol = 6 * 2.0 ** -24 * w.abs() + HALF_UNIT[o.dtype] * w.abs() + (6e-8 if o.dtype == torch.float16 else 1e-38)
        assert bool(((o.double() - w).abs() <= tol).all())
    return got


SETS = [[1], [0], [], [0, 1, 0], [7, 64, 1000], [16384], [16383, 16385, 1], [100003], [5] * 300,
        [3, 70000, 0, 129] * 60, [1 << 20, 4097, 333], [1 << 23]]


@pytest.mark.parametrize("sizes", SETS, ids=[str(len(s)) + "x" + str(sum(s)) for s in SETS])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 1])
def test_norms(sizes, dtype, shift):
    grads = tensors(sizes, dtype, shift=shift)
    print("norm", len(sizes), sum(sizes), dtype, shift, flush=True)
    for ord in (2, "inf"):
        for scale in (1.0, 0.125):
            got = moe.grad_norm(grads, scale=scale, ord=ord)
            torch.cuda.synchronize()
            want = scale * ref_norm(grads, ord)
            assert abs(float(got) - want) <= 2.0 ** -23 * want, (float(got), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("shift", [0, 3])
def test_clip_into_other_tensors(dtype, out, shift):
    for sizes in ([1], [7, 64, 1000], [16383, 16385, 1], [3, 70000, 0, 129] * 60):
        grads = tensors(sizes, dtype, shift=shift)
        outs = [torch.full_like(g, 9.0, dtype=out) for g in grads]
        before = [g.clone() for g in grads]
        print("clip", len(sizes), sum(sizes), dtype, out, flush=True)
        check_clip(grads, outs, before, 1.0, scale=0.5)
        check_clip(grads, outs, before, 1e9)
        check_clip(grads, outs, before, 0.25, ord="inf")
        assert all(torch.equal(g, b) for g, b in zip(grads, before))


@pytest.mark.parametrize("dtype", TYPES)
def test_clip_in_place(dtype):
    grads = tensors([3, 70000, 0, 129] * 60, dtype, shift=1)
    before = [g.clone() for g in grads]
    check_clip(grads, None, before, 1e9)          # factor 1: nothing changes
    assert all(torch.equal(g, b) for g, b in zip(grads, before))
    check_clip(grads, None, before, 1.0)
    before = [g.clone() for g in grads]
    check_clip(grads, None, before, float("inf"), scale=0.25)


def test_mixed_types_and_orders_of_axes():
    a = tensors([6000], torch.bfloat16)[0].view(60, 100)
    b = tensors([77], torch.float32)[0]
    c = tensors([2 * 3 * 500], torch.float16)[0].view(2, 3, 500).permute(2, 0, 1)
    grads = [a.t(), b, c]
    outs = [torch.empty_like(g, dtype=torch.float32) for g in grads]
    assert outs[0].stride() == grads[0].stride()
    check_clip(grads, outs, [g.clone() for g in grads], 1.0)


def test_gaps_and_neighbours_are_not_written():
    flat = torch.full((5000,), 7.0, device=DEV)
    grads = [flat[10:2011], flat[2013:4990]]
    check_clip(grads, None, [g.clone() for g in grads], 1.0)
    keep = torch.ones(5000, dtype=torch.bool, device=DEV)
    keep[10:2011] = False
    keep[2013:4990] = False
    assert bool((flat[keep] == 7.0).all())


@pytest.mark.parametrize("ord", [2, "inf"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_writes_nothing(ord, bad):
    for at in (0, 16384 * 3 + 5, 69999):
        grads = tensors([70000, 5], torch.float32)
        grads[0][at] = bad
        outs = [torch.full_like(g, 9.0) for g in grads]
        norm = moe.clip_grads(grads, 1.0, ord=ord, outs=outs)
        torch.cuda.synchronize()
        assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
        assert all(bool((o == 9.0).all()) for o in outs)
        assert math.isnan(bad) == math.isnan(float(moe.grad_norm(grads, ord=ord)))


def test_squares_beyond_32_bits():
    """Squares that overflow or vanish in 32 bits are summed in 64."""
    for v in (1e30, 1e-30):
        grads = [torch.full((1000,), v, device=DEV), torch.full((10,), v, device=DEV, dtype=torch.float32)]
        got = float(moe.grad_norm(grads))
        want = ref_norm(grads)
        assert abs(got - want) <= 2.0 ** -23 * want


def test_a_given_norm_of_a_whole_group():
    """Two ranks' sets: each clips by the norm of both."""
    mine, other = tensors([1000, 37], torch.bfloat16), tensors([999], torch.bfloat16, seed=1)
    both = (moe.grad_norm(mine).square() + moe.grad_norm(other).square()).sqrt()
    outs = [torch.empty_like(g, dtype=torch.float32) for g in mine]
    check_clip(mine, outs, [g.clone() for g in mine], 1.0, norm=both)


def test_equal_bits_graph_and_another_stream():
    grads = tensors([3, 70000, 0, 129] * 60, torch.bfloat16, shift=1)
    first = moe.grad_norm(grads)
    assert all(torch.equal(first, moe.grad_norm(grads)) for _ in range(5))
    outs = [torch.zeros_like(g, dtype=torch.float32) for g in grads]
    want = [torch.zeros_like(o) for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = moe.clip_grads(grads, 1.0, outs=outs)
    for i in range(3):
        for g in grads:
            g.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        n2 = moe.clip_grads(grads, 1.0, outs=want)
        assert torch.equal(norm, n2) and all(torch.equal(a, b) for a, b in zip(outs, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = moe.grad_norm(grads, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, n2)


def test_more_elements_than_32_bits_count():
    """One tensor of more than 2^32 elements."""
    n = (1 << 32) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g[-1], g[0], g[1 << 31], g[1 << 32] = 3.0, 4.0, 12.0, 84.0
    assert float(moe.grad_norm([g])) == 85.0 and float(moe.grad_norm([g], ord="inf")) == 84.0
    norm = moe.clip_grads([g], 17.0)
    torch.cuda.synchronize()
    assert float(norm) == 85.0
    for i, v in ((0, 0.8), (-1, 0.6), (1 << 31, 2.4), (1 << 32, 16.8)):
        assert abs(float(g[i]) - v) <= 2.0 ** -8 * v


def test_refusals():
    g = torch.zeros(100, device=DEV)
    with pytest.raises(TypeError):
        moe.grad_norm([g.double()])
    with pytest.raises(ValueError):
        moe.grad_norm([g.cpu()])
    with pytest.raises(ValueError):
        moe.grad_norm([g[::2]])
    with pytest.raises(ValueError):
        moe.grad_norm([g], ord=1)
    with pytest.raises(ValueError):
        moe.clip_grads([g], 1.0, outs=[])
    with pytest.raises(ValueError):
        moe.clip_grads([g], 1.0, outs=[torch.zeros(99, device=DEV)])
    with pytest.raises(topoep.TopoepError):
        moe.clip_grads([g], 0.0)
    with pytest.raises(topoep.TopoepError):
        moe.grad_norm([g], scale=float("nan"))
