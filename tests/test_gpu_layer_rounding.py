"""How far the layer for a few tokens is from the layer in 64 bits, with a bound
that follows its roundings as independent errors, so that a lost tail of the
hidden axis or a hidden row of fewer bits shows, and the choice of its groups.

With r^2 = sum_j w_j^2 sum_i down_i^2 (h_i^2 + m^2), m^2 the mean of h^2 over an
expert's hidden axis, the terms of an output carry independent relative errors
of at most 2^-16 from h's two words and of about sqrt(H) 2^-24 from each sum
behind it; six deviations of both: 6 (2^-16 + sqrt(H) 2^-22) r.  A router weight
comes from 32-bit logits, of error 6 sqrt(H / 2) 2^-24 |x| |gate| (at most 2e-5
here), and moves by at most twice that, relative: 4e-5 sum |w_j y_j| and the
exponential's 1e-5 of it.  Rounding the output: half a unit, 2^-8 (bf16), 2^-11
(f16; at least 2^-25) of it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe  # noqa: E402

DEV = torch.device("cuda:0")
HALF_UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def inputs(T, H, I, E, L, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed * 131 + T * 7 + H + I)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)

    return normal(T, H), normal(E, H, std=H ** -0.5), normal(L, 2 * I, H, std=H ** -0.5), normal(L, H, I, std=I ** -0.5)


def ref_weights(x, gate, ids, scoring, renorm, scale):
    logits = x.double() @ gate.double().t()
    at = logits.gather(1, ids.long())
    if scoring == "sigmoid":
        s = torch.sigmoid(at)
        return scale * (s / s.sum(1, keepdim=True) if renorm else s)
    return scale * (torch.softmax(at, 1) if renorm else torch.softmax(logits, 1).gather(1, ids.long()))


def check(x, gate, up, down, k, slot=None, scoring="softmax", renorm=True, scale=1.0, bias=None):
    (T, H), (L, _, I) = x.shape, down.shape
    print("rounding", T, H, I, gate.shape[0], L, k, x.dtype, flush=True)
    out, ids, w = moe.moe_few(x, gate, up, down, k, expert_slot=slot, scoring=scoring, renorm=renorm, scale=scale, bias=bias)
    torch.cuda.synchronize()
    want_w = ref_weights(x, gate, ids, scoring, renorm, scale)
    place = ids.long() if slot is None else slot.long()[ids.long()]
    want, terms, spread = (torch.zeros((T, H), dtype=torch.float64, device=DEV) for _ in range(3))
    for e in range(L):
        share = torch.where(place == e, want_w, 0.0).sum(1, keepdim=True)
        rows = share[:, 0].nonzero()[:, 0]
        if not len(rows):
            continue
        a, d, s = x[rows].double() @ up[e].double().t(), down[e].double(), share[rows]
        h = a[:, :I] * torch.sigmoid(a[:, :I]) * a[:, I:]
        y = s * (h @ d.t())
        want[rows] += y
        terms[rows] += y.abs()
        spread[rows] += s.square() * ((h.square() + h.square().mean(1, keepdim=True)) @ d.square().t())
    off = (out.double() - want).abs()
    floor = 2.0 ** -25 if x.dtype == torch.float16 else 0.0
    bound = HALF_UNIT[x.dtype] * want.abs() + 6 * (2.0 ** -16 + H ** 0.5 * 2.0 ** -22) * spread.sqrt() + 5e-5 * terms + floor
    assert bool((off <= bound).all()), float((off / bound).max())
    return out, ids, w


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 2, 4, 5, 16, 33, 64, 128])
def test_hidden_values_keep_their_bits(T, dtype):
    check(*inputs(T, 256, 2056, 8, 8, dtype), 2)
    check(*inputs(T, 2048, 768, 32, 32, dtype), 8, scoring="sigmoid", scale=2.5)
    check(*inputs(T, 72, 40, 16, 16, dtype), 4, renorm=False)
    check(*inputs(T, 1032, 136, 5, 5, dtype), 5)


@pytest.mark.parametrize("H,I", [(1536, 1536), (512, 1536), (64, 3080)])
def test_widths_between_runs(H, I):
    for T in (1, 3, 20, 90):
        check(*inputs(T, H, I, 12, 12), 3)
        slot = torch.full((12,), -1, dtype=torch.int32, device=DEV)
        slot[2:7] = torch.arange(5, dtype=torch.int32, device=DEV).flip(0)
        check(*inputs(T, H, I, 12, 5, torch.float16), 3, slot=slot)


@pytest.mark.parametrize("T", [1, 3, 6, 40, 128])
def test_f16_hidden_values_beyond_the_types_largest(T):
    """Hidden values up to 2^27, of which the second product makes ordinary outputs."""
    x, gate, up, down = inputs(T, 64, 32, 4, 4, torch.float16)
    _, _, w = check(x * 8, gate / 8, up * 50, down * 2.0 ** -8, 2)
    a = (x * 8).double() @ (up * 50).double().flatten(0, 1).t()
    assert float(a.abs().max()) ** 2 > 4 * 65504.0


@pytest.mark.parametrize("T", [1, 5, 21, 100])
@pytest.mark.parametrize("renorm", [True, False])
def test_groups_open_by_their_largest_key(T, renorm):
    """The chosen groups hold the largest keys and the chosen experts are their
    best, up to the logits' 32-bit error."""
    for E, groups, top_groups, k in ((64, 8, 2, 6), (60, 5, 3, 8), (256, 4, 2, 8), (512, 32, 4, 8)):
        x, gate, up, down = inputs(T, 96, 64, E, 9)
        bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).to(DEV)
        slot = torch.full((E,), -1, dtype=torch.int32, device=DEV)
        slot[torch.randperm(E, generator=torch.Generator().manual_seed(1))[:9].to(DEV)] = \
            torch.arange(9, dtype=torch.int32, device=DEV)
        _, ids, _ = check_grouped(x, gate, up, down, k, slot, bias, groups, top_groups, renorm)


def check_grouped(x, gate, up, down, k, slot, bias, groups, top_groups, renorm):
    T, E = x.shape[0], gate.shape[0]
    m = E // groups
    print("groups", T, E, groups, top_groups, k, flush=True)
    out, ids, w = moe.moe_few(x, gate, up, down, k, expert_slot=slot, bias=bias, groups=groups, top_groups=top_groups,
                              renorm=renorm)
    torch.cuda.synchronize()
    key = x.double() @ gate.double().t() + bias.double()
    err = 2.0 ** -20 * float((x.double().abs() @ gate.double().abs().t()).max())
    best = key.view(T, groups, m).amax(2)
    at = ids.long()
    chosen = key.gather(1, at)
    assert bool((chosen[:, 1:] <= chosen[:, :-1] + err).all()) and all(len(set(r)) == k for r in at.tolist())
    # a group that may be open: at most top_groups - 1 others are surely better
    may = ((best[:, None, :] > best[:, :, None] + err).sum(2) < top_groups)
    # a group that must be: fewer than top_groups others are perhaps better
    must = ((best[:, None, :] > best[:, :, None] - err).sum(2) - 1 < top_groups)
    assert bool(may.gather(1, at // m).all())
    inside = must.repeat_interleave(m, 1).scatter(1, at, False)
    assert bool((torch.where(inside, key, float("-inf")).amax(1) <= chosen[:, -1] + err).all())
    want = ref_weights(x, gate, ids, "softmax", renorm, 1.0)
    assert bool(((w - want).abs() <= 1e-4 * want).all())
    return out, ids, w
