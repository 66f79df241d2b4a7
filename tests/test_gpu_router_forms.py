"""Every form of the router that more than 1024 tokens take: lists of four and
eight over each number of lanes, groups inside a lane, over several lanes and of
any size, few and many of them open, with and without a bias, each against
the plain implementation in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_router import check, draw  # noqa: E402

DEV = torch.device("cuda:0")
NEG = float("-inf")


def rows(E, dtype):
    """Ordinary logits among rows with masks, ties and nothing left."""
    x = draw(1500, E, dtype, seed=7)
    x[::37, ::3] = NEG
    x[5] = 0.0
    x[6] = NEG
    x[7::100] = x[7::100].round()
    x[8, 1:] = NEG
    x[9, ::2] = float("nan")
    return x


@pytest.mark.parametrize("E", [13, 30, 64, 100, 128, 200, 256, 300, 512, 1000, 1024])
@pytest.mark.parametrize("k", [1, 2, 4, 5, 8])
def test_lists_over_every_width(E, k):
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        check(rows(E, dtype), k, renorm=False)
        bias = torch.randn(E, generator=torch.Generator().manual_seed(k)).to(DEV)
        check(rows(E, dtype), k, scoring="sigmoid", bias=bias)


GROUPS = [(128, 16), (128, 8), (128, 4), (128, 2), (256, 32), (256, 16), (256, 8), (256, 4), (256, 2), (512, 64), (512, 32),
          (512, 16), (512, 8), (512, 4), (512, 2),                          # 8 to 256 experts: parts of a lane, 1 to 8 lanes
          (24, 4), (64, 16), (96, 8), (100, 10), (160, 8), (320, 32), (640, 10), (1024, 64), (1020, 60)]   # of any size


@pytest.mark.parametrize("E,groups", GROUPS)
@pytest.mark.parametrize("share", [0.1, 0.5, 0.8, 1.0])
def test_groups_of_every_size_few_and_many_open(E, groups, share):
    top_groups = max(1, min(groups, round(groups * share)))
    k = min(8, top_groups * (E // groups))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        x = rows(E, dtype)
        bias = torch.randn(E, generator=torch.Generator().manual_seed(E + groups)).to(DEV)
        check(x, k, groups=groups, top_groups=top_groups)
        check(x, k, scoring="sigmoid", bias=bias, groups=groups, top_groups=top_groups)
        if k > 3:
            check(x, 3, renorm=False, bias=bias, groups=groups, top_groups=top_groups)
