"""The layer for a few tokens under expert maps that name a place more than
once: a token then has more experts here than there are places, and every one
of them adds its share.  Against the layer in 64 bits with one set of weights an expert;
workspaces hold NaN before the call, so that a hidden row that nothing wrote
shows.  Tolerance as where each expert has its own place: u = 2^-8 (bf16),
2^-10 (f16) of sum |w| |down| |h| twice, and of the output once."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import moe  # noqa: E402

DEV = torch.device("cuda:0")
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def check(T, H, I, E, L, k, slot, dtype=torch.bfloat16, bias=None):
    print("map", T, H, I, E, L, k, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(T * 31 + E + k)

    def normal(*shape, std):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)

    x, gate = normal(T, H, std=1.0), normal(E, H, std=H ** -0.5)
    up, down = normal(L, 2 * I, H, std=H ** -0.5), normal(L, H, I, std=I ** -0.5)
    ws = torch.full((moe.moe_workspace_bytes(H, I, E, L, k, T, dtype) + 255,), 0xFF, dtype=torch.uint8, device=DEV)
    out, ids, w = moe.moe_few(x, gate, up, down, k, expert_slot=slot, workspace=ws, bias=bias)
    torch.cuda.synchronize()
    place = slot.long()[ids.long()]
    want, bound = torch.zeros((T, H), dtype=torch.float64, device=DEV), torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for e in range(L):
        share = torch.where(place == e, w.double(), 0.0).sum(1, keepdim=True)
        a = x.double() @ up[e].double().t()
        h = a[:, :I] * torch.sigmoid(a[:, :I]) * a[:, I:]
        want += share * (h @ down[e].double().t())
        bound += share * (h.abs() @ down[e].double().abs().t())
    u = UNIT[dtype]
    off = (out.double() - want).abs()
    assert bool((off <= (2 * u + 2e-4) * bound + u * want.abs()).all()), float((off / (bound + 1e-9)).max())


def shared(E, L):
    """Every place named by about E / L experts, in no order."""
    g = torch.Generator().manual_seed(E + L)
    return (torch.randperm(E, generator=g) % L).to(torch.int32).to(DEV)


@pytest.mark.parametrize("T", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_tokens_with_more_experts_here_than_places(T, dtype):
    for E, L, k in ((4, 1, 4), (8, 3, 8), (128, 5, 8), (200, 2, 16), (24, 1, 7)):
        check(T, 64, 32, E, L, k, shared(E, L), dtype)
        check(T, 520, 136, E, L, k, shared(E, L), dtype)
        # and some experts elsewhere
        slot = shared(E, L)
        slot[::3] = -1
        check(T, 64, 32, E, L, k, slot, dtype)


@pytest.mark.parametrize("H,I", [(64, 2048), (4096, 64)])   # a wave's own tiles of the first product, of the second
def test_waves_at_experts_of_other_counts(H, I):
    """More experts with tokens than places: a workgroup goes on to further
    experts, and its waves need not be at the same one, here of 1 to 30 tokens each."""
    for T, E, L, k in ((40, 40, 10, 8), (33, 64, 10, 6), (64, 80, 9, 4)):
        bias = torch.linspace(-1.5, 1.5, E, device=DEV)
        check(T, H, I, E, L, k, shared(E, L), bias=bias)
        check(T, H, I, E, L, k, shared(E, L), torch.float16, bias=bias)
