"""Shares of a routed layer that get other rows than the router's choices let expect."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ffnmodel  # noqa: E402
from test_gpu_ffn import case, check, run_experts  # noqa: E402


@pytest.mark.parametrize("T,H,I,E,L,k", [(600, 64, 40, 256, 1, 1),         # 3 rows expected, waves that share tiles
                                         (600, 1032, 136, 256, 8, 2),      # 38 expected
                                         (300, 136, 1032, 256, 8, 4),      # waves with tiles of their own, up
                                         (300, 2056, 40, 256, 8, 4)])      # and down
@pytest.mark.parametrize("share", ["all", "none but one", "one expert"])
def test_more_and_fewer_rows_than_expected(T, H, I, E, L, k, share):
    x, ids, weights, up, down, slot, dout = case(T, H, I, E, L, k, torch.bfloat16, seed=T + L)
    here, away = (slot >= 0).nonzero().flatten(), (slot < 0).nonzero().flatten()
    pick = torch.randint(0, L, ids.shape, generator=torch.Generator().manual_seed(1))
    if share == "all":
        ids = here[pick].int()
    else:
        ids = away[pick].int()
        if share == "one expert":
            ids[:, 0] = int(here[-1])
        else:
            ids[T // 2, 0] = int(here[-1])
    check(run_experts(x, ids, weights, up, down, slot, dout), ffnmodel.layer(x, ids, weights, up, down, slot, dout))
