"""The example that takes the operators from a training step to decoding: the
loss falls over the steps, and the decoded tokens agree with the layer computed
in 32 bits (hidden values and outputs rounded to bfloat16: 2^-9 each, sums of
them, 2^-6 of the largest output allowed)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import train_decode  # noqa: E402


def test_training_steps_and_decoding():
    lines = []
    losses, norms, off = train_decode.run(steps=6, log=lines.append)
    print("\n".join(lines), flush=True)
    assert all(math.isfinite(v) for v in losses + norms) and min(norms) > 0
    assert losses[-1] < losses[0] and all(b < a * 1.05 for a, b in zip(losses, losses[1:]))
    assert all("plan status 0" in line for line in lines[:6])
    assert off < 2.0 ** -6
