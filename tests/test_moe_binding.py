"""The binding's own checks of sizes and rules (no GPU): what ctypes would cut
to 32 bits, and what one struct for many calls must not be made of."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def moe():
    from paper_2609_35481_amd import moe
    return moe


@pytest.mark.parametrize("kw", [dict(k=2 ** 32 + 2), dict(E=2 ** 32 + 16), dict(groups=2 ** 32 + 1), dict(top_groups=-2 ** 32 + 1),
                                dict(k=2 ** 31)])
def test_sizes_beyond_32_bits_are_not_cut(moe, kw):
    with pytest.raises(ValueError):
        moe.router(**{**dict(E=16, k=2), **kw})


def test_workspace_sizes_beyond_32_bits_are_not_cut(moe):
    good = dict(H=64, I=32, E=16, L=16, k=2, T=8)
    assert moe.moe_workspace_bytes(**good) > 0
    for name in good:
        with pytest.raises(ValueError):
            moe.moe_workspace_bytes(**{**good, name: good[name] + 2 ** 32})


@pytest.mark.parametrize("kw", [dict(scale=torch.tensor(2.0)), dict(renorm=torch.tensor(True)), dict(k=torch.tensor(2)),
                                dict(scale="2"), dict(k=2.5), dict(groups=torch.tensor(1)), dict(scale=None)])
def test_rules_are_plain_values(moe, kw):
    """A tensor among them would be remembered by its identity, and its first
    value used after it has changed."""
    args = {**dict(E=16, k=2), **kw}
    for _ in range(2):
        with pytest.raises(TypeError):
            moe.router(**args)


def test_numpy_values_are_plain_values(moe):
    r = moe.router(np.int64(20), np.int32(3), renorm=np.bool_(False), scale=np.float32(2.5), groups=np.int16(4), top_groups=2)
    assert (r.num_experts, r.topk, r.groups, r.top_groups, r.renorm, r.scale) == (20, 3, 4, 2, 0, 2.5)
