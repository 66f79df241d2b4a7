"""The router over many rows and in all of its forms: what one row gets does not
depend on the rows beside it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe  # noqa: E402

DEV = torch.device("cuda:0")


def test_more_rows_than_a_grid_has_lanes_for():
    """2^30 rows at four lanes each are 2^32 lanes."""
    n = (1 << 30) + 5
    x = torch.zeros((n, 2), dtype=torch.bfloat16, device=DEV)
    x[::3, 1] = 1.0
    print("router", tuple(x.shape), flush=True)
    ids, weights = moe.route(x, 1, scale=0.5)
    torch.cuda.synchronize()
    for a, w, r in zip(ids.split(1 << 28), weights.split(1 << 28), x.split(1 << 28)):
        assert torch.equal(a[:, 0].bool(), r[:, 1] > r[:, 0]) and bool((w == 0.5).all())


@pytest.mark.parametrize("scoring,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("E,k", [(16, 6), (100, 8), (300, 20)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_weights_gradients_of_masked_choices_are_not_used(scoring, renorm, E, k, bad):
    """Rows with fewer logits than choices: what the weights' gradient holds at
    the others, which are masked (or name no expert), changes no bit.  What it
    holds at an unmasked one stays off the masked logits."""
    for T in (9, 9000):
        g = torch.Generator(device=DEV).manual_seed(T + E)
        x = torch.randn((T, E), generator=g, device=DEV)
        x[::2, 3:] = float("-inf")
        x[4] = float("-inf")
        ids, _ = moe.route(x, k, scoring=scoring, renorm=renorm)
        masked = torch.isinf(x.gather(1, ids.long()))
        grad = torch.randn((T, k), generator=g, device=DEV)
        print("masked", T, E, k, scoring, renorm, bad, flush=True)
        want = moe.route_backward(x, ids, torch.where(masked, 0.0, grad), scoring=scoring, renorm=renorm)
        got = moe.route_backward(x, ids, torch.where(masked, bad, grad), scoring=scoring, renorm=renorm)
        elsewhere = moe.route_backward(x, torch.where(masked, E + 5, ids), torch.where(masked, bad, grad), scoring=scoring,
                                       renorm=renorm)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(want).all()) and torch.equal(got, want) and torch.equal(elsewhere, want)
        assert not bool(want[torch.isinf(x)].any())
        grad[::2, 0] = bad
        grad[4, 0] = 0.0
        got = moe.route_backward(x, ids, grad, scoring=scoring, renorm=renorm)
        torch.cuda.synchronize()
        assert not bool(got[torch.isinf(x)].any()) and torch.equal(got[1::2], want[1::2])
