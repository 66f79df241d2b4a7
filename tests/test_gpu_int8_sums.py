"""Sums of 8-bit products at both ends of their range.  Rows and channels of one value each, so that a
sum is K q w: exact in 64 bits, and with scales that are powers of two exact in the result.  Each shape is another
kernel: a few rows, workgroups that share the inner axis, tiles of 128 x 128 and of 256 x 256."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ffnmodel  # noqa: E402
from paper_2609_35481_amd import ffn  # noqa: E402

DEV = torch.device("cuda:0")
K = 1 << 17
VALUES = torch.tensor([-128, 127, -127, 1, 0, -128, 2])


def constant(n, shift=0):
    return torch.roll(VALUES, shift).repeat((n + 6) // 7)[:n]


def matrix(values):
    return values.to(torch.int8).to(DEV)[:, None].expand(-1, K).contiguous()


@pytest.mark.parametrize("M,N", [(3, 20), (12, 64), (100, 64), (3000, 2200), (3000, 3082)])
@pytest.mark.parametrize("groups", [0, 1])
def test_sums_at_both_ends(M, N, groups):
    qv, wv = constant(M), constant(N, 2)
    sums = K * qv[:, None] * wv[None]
    assert int(sums.max()) == 1 << 31 and int(sums.min()) == -127 * 128 * K
    q, w = matrix(qv), matrix(wv)
    scale, ws = torch.full((M,), 2.0 ** -20, device=DEV), torch.full((N,), 2.0 ** -11, device=DEV)
    args = ((q, scale), w[None], ws[None], torch.tensor([0, M], dtype=torch.int32, device=DEV)) if groups else ((q, scale), w, ws)
    got = ffn.matmul_int8(*args, dtype=torch.float32)
    assert torch.equal(got.cpu(), (sums.double() * 2.0 ** -31).float())
    # one product less than all of them
    q[0, K - 7] = 0
    got = ffn.matmul_int8(*args, dtype=torch.float32)[0].cpu()
    assert torch.equal(got, (((K - 1) * qv[0] * wv).double() * 2.0 ** -31).float())


@pytest.mark.parametrize("M,N", [(3, 20), (100, 64), (3000, 3082)])
def test_gated_sums_at_both_ends(M, N):
    qv, wv = constant(M), constant(N, 2)
    a = (K * qv[:, None] * wv[None]).double() * 2.0 ** -31
    got = ffn.matmul_int8((matrix(qv), torch.full((M,), 2.0 ** -20, device=DEV)), matrix(wv),
                          torch.full((N,), 2.0 ** -11, device=DEV), gated=True, dtype=torch.float32)
    z, u = a[:, :N // 2], a[:, N // 2:]
    # z and u are exact; the sigmoid and the two products are not
    value = z * torch.sigmoid(z) * u
    off = value.abs() * (2 * z.abs() + 8 + 3) * ffnmodel.E32
    ffnmodel.within(got, value, ffnmodel.rounded(value, off, torch.float32), "gated")
