"""The gated block's backward pass on what hooks on saved tensors give back: the
values in any layout, from the host or computed again.  Gradients have the bits of a pass
without hooks; what is not what was saved is an error."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from torch.autograd.graph import save_on_cpu, saved_tensors_hooks  # noqa: E402
from torch.utils.checkpoint import checkpoint  # noqa: E402

from paper_2609_35481_amd import ffn  # noqa: E402
from test_gpu_ffn import case, gradients  # noqa: E402

DEV = torch.device("cuda:0")
BF16 = torch.bfloat16


@pytest.fixture(params=["dense", "routed", "one token"])
def call(request):
    """(a function of the leaves, the leaves, the gradient of its result)"""
    T = 1 if request.param == "one token" else 70
    x, ids, weights, up, down, slot, dout = (v.to(DEV) for v in case(T, 72, 40, 8, 5, 2, BF16, seed=3))
    if request.param == "dense":
        t = {"x": x, "up": up[0].contiguous(), "down": down[0].contiguous()}
        f = lambda **v: ffn.feed_forward(v["x"], v["up"], v["down"])  # noqa: E731
    else:
        t = {"x": x, "weights": weights, "up": up, "down": down}
        f = lambda **v: ffn.experts(v["x"], ids, v["weights"], v["up"], v["down"], slot)  # noqa: E731
    return f, {n: v.requires_grad_() for n, v in t.items()}, dout


def equal(got, want):
    for name in want:
        assert torch.equal(got[name], want[name]), name


def turned(t):                  # columns along memory
    return t.transpose(-1, -2).contiguous().transpose(-1, -2) if t.dim() > 1 else t


def moved(t):                   # one element behind a multiple of 16 bytes
    to = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    return to.copy_(t)


def apart(t):                   # rows at no multiple of 16 bytes, the last of them whole
    if t.dim() != 2:
        return t
    return torch.full((t.shape[0], t.shape[1] + 3), 5, dtype=t.dtype, device=t.device)[:, :-3].copy_(t)


@pytest.mark.parametrize("layout", [turned, moved, apart])
def test_saved_tensors_in_another_layout(call, layout):
    f, t, dout = call
    want = gradients(f(**t), dout, **t)
    with saved_tensors_hooks(lambda v: v.detach(), layout):
        out = f(**t)
    equal(gradients(out, dout, **t), want)


def test_saved_tensors_on_the_host_and_computed_again(call):
    f, t, dout = call
    want = gradients(f(**t), dout, **t)
    with save_on_cpu():
        out = f(**t)
    equal(gradients(out, dout, **t), want)
    equal(gradients(checkpoint(lambda *v: f(**dict(zip(t, v))), *t.values(), use_reentrant=False), dout, **t), want)


def test_where_rows_are_is_out_of_reach(call):
    f, t, dout = call
    seen = []
    with saved_tensors_hooks(lambda v: seen.append(v.dtype) or v.detach(), lambda v: v):
        out = f(**t)
    assert seen and torch.int32 not in seen
    equal(gradients(out, dout, **t), gradients(f(**t), dout, **t))


@pytest.mark.parametrize("other", [lambda v: v.cpu(), lambda v: v.double(), lambda v: v[..., :-1], lambda v: v.reshape(-1)[None, None],
                                   lambda v: v.new_empty((0,)), lambda v: v.to_sparse()],
                         ids=["host", "type", "shape", "dimensions", "empty", "sparse"])
def test_other_tensors_than_were_saved(call, other):
    f, t, dout = call
    want = gradients(f(**t), dout, **t)
    count = []
    with saved_tensors_hooks(lambda v: count.append(0) or v.detach(), lambda v: v):
        f(**t)
    for which in range(len(count)):                      # each of them in turn
        number = iter(range(len(count)))
        with saved_tensors_hooks(lambda v: (next(number), v.detach()), lambda n: other(n[1]) if n[0] == which else n[1]):
            out = f(**t)
        with pytest.raises(RuntimeError, match="a hook on saved tensors"):
            gradients(out, dout, **t)
    equal(gradients(f(**t), dout, **t), want)
