"""Quantisation to 8 bits and the product in 8-bit integers, against 64 bits.

Integers and scales have to be equal.  The product's sum is exact; it is rounded
to 32 bits, times two scales (3 2^-24 in all), gated: the activation's sigmoid is
off by (2 |z| + 8) 2^-24 and by what z is off; then one rounding to the output's type."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ffnmodel  # noqa: E402
from paper_2609_35481_amd import ffn, moe  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def normal(seed, *shape, dtype=F32, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def quantized(x):
    x = x.double()
    scale = (x.abs().amax(1) / 127.0).float()
    q = torch.round(x / torch.where(scale > 0, scale, 1.0).double()[:, None]).clamp(-127, 127)
    return q.to(torch.int8), scale


def check_quantize(x):
    q, scale = ffn.quantize(x.to(DEV))
    wq, ws = quantized(x)
    assert q.dtype == torch.int8 and torch.equal(scale.cpu(), ws)
    assert torch.equal(q.cpu(), wq)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 16), (3, 7), (5, 2048), (4, 2049), (130, 255), (9, 7168), (2, 8192), (2, 8200),
                                 (2, 40000), (1000, 64)])
def test_quantize(M, K, dtype):
    check_quantize(normal(M + K, M, K, dtype=dtype) * normal(1, M, 1).exp().to(dtype))


def test_quantize_zeros_borders_and_small_values():
    x = torch.zeros(6, 64)
    x[1, 5] = -3.0
    x[2] = torch.arange(64) - 31.5               # borders: 127 / 63.5 a step
    x[2, 63] = 127.0                             # scale 1: halves tie to even
    x[3] = normal(3, 64) * 1e-38                 # denormal scale
    x[4] = normal(4, 64) * 3e-43
    x[5, 1] = 1e-45
    check_quantize(x)
    check_quantize(-x)
    # quotients whose rounding to 32 bits is a border that they do not lie on
    g = torch.Generator().manual_seed(8)
    top = torch.rand((4000, 1), generator=g) + 0.5
    scale = (top.double() / 127).float()
    n = torch.randint(0, 126, (4000, 64), generator=g)
    near = ((n + 0.5).double() * scale.double()).float()
    x = torch.cat([top, near, torch.nextafter(near, torch.zeros(())), torch.nextafter(near, torch.full((), 9.0))], 1)
    check_quantize(x)
    check_quantize(-x)


def test_quantize_strides_and_alignment():
    base = normal(5, 50, 131, dtype=BF16)
    for part in (base[:, 1:129], base[:, 2:130], base[::2, :128], base[3:4, 5:], base[:, :0 + 16]):
        wide = base.to(DEV)
        view = torch.as_strided(wide, part.shape, part.stride(), part.storage_offset())
        q, scale = ffn.quantize(view)
        wq, ws = quantized(part)
        assert torch.equal(q.cpu(), wq) and torch.equal(scale.cpu(), ws)


def test_quantize_more_rows_than_a_grid_has_threads_for():
    x = torch.randn(17000003, 16, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=BF16)
    q, scale = ffn.quantize(x)
    want = (x.double().abs().amax(1) / 127.0).float()
    assert torch.equal(scale, want)
    for part in (slice(0, 3000000), slice(16000000, None)):
        exact = torch.round(x[part].double() / want[part].double()[:, None]).clamp(-127, 127).to(torch.int8)
        assert torch.equal(q[part], exact)


@pytest.mark.parametrize("K", [64, 5000])
def test_quantize_infinities_and_nan(K):
    x = normal(6, 5, K)
    x[1, 3], x[2, 4], x[3, 5], x[3, 6] = float("inf"), float("nan"), float("-inf"), float("nan")
    q, scale = ffn.quantize(x.to(DEV))
    q, scale = q.cpu(), scale.cpu()
    assert scale[1] == float("inf") and torch.isnan(scale[2]) and torch.isnan(scale[3])
    assert not q[1:4].any()
    wq, ws = quantized(x[[0, 4]])
    assert torch.equal(q[[0, 4]], wq) and torch.equal(scale[[0, 4]], ws)


def product(q, scale, w, ws, offsets, gated, dtype):
    """(value, bound) in 64 bits."""
    M, E32 = q.shape[0], ffnmodel.E32
    ends = [0, M] if offsets is None else offsets.tolist()
    w, ws = (w[None], ws[None]) if offsets is None else (w, ws)
    a = torch.zeros(M, w.shape[1], dtype=torch.float64)
    for g in range(len(ends) - 1):
        r = slice(ends[g], ends[g + 1])
        a[r] = (q[r].double() @ w[g].double().t()) * scale[r].double()[:, None] * ws[g].double()
    off = 3 * E32 * a.abs()
    if gated:
        n = a.shape[1] // 2
        z, u = a[:, :n], a[:, n:]
        act = z * torch.sigmoid(z)
        off = (1.1 * 3 * E32 * z.abs() * u.abs() + (act * u).abs() * ((2 * z.abs() + 8) * E32 + 6 * E32)) + 1e-30
        a = act * u
    return a, ffnmodel.rounded(a, off, dtype)


def weights(seed, *shape):
    w = normal(seed, *shape, std=shape[-1] ** -0.5)
    q, s = quantized(w.reshape(-1, shape[-1]))
    return q.view(shape), s.view(shape[:-1])


SHAPES = [(1, 16, 16), (1, 1, 64), (1, 100, 4096), (2, 37, 208), (4, 128, 128), (5, 130, 144), (16, 64, 1024), (17, 66, 256),
          (33, 257, 80), (128, 128, 512), (129, 384, 272), (300, 129, 2064), (3000, 3082, 144),
          (100, 200, 4112), (70, 1040, 14336), (65, 1, 2048)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("gated,dtype,out", [(False, BF16, BF16), (True, F16, F32), (False, F32, F16), (True, BF16, BF16)])
def test_product(M, N, K, gated, dtype, out):
    N += N % 2 if gated else 0
    x, (w, ws) = normal(M, M, K, dtype=dtype), weights(N, N, K)
    q, scale = quantized(x)
    want = product(q, scale, w, ws, None, gated, out)
    got = ffn.matmul_int8(x.to(DEV), w.to(DEV), ws.to(DEV), gated=gated, dtype=out)
    assert got.dtype == out
    ffnmodel.within(got, *want, "from x")
    pair = ffn.matmul_int8((q.to(DEV), scale.to(DEV)), w.to(DEV), ws.to(DEV), gated=gated, dtype=out)
    assert torch.equal(pair, got)


GROUPS = [([0, 0, 1], 64, 64), ([0, 5, 5, 9, 9], 48, 128), ([0, 1, 2, 3, 40, 41], 130, 256), ([0, 128, 129, 300], 72, 144),
          ([0, 17, 300, 301], 256, 96), ([0] * 70 + [3] + [7] * 80 + [8], 34, 64),
          ([0, 1500, 1501, 4001], 2310, 80),
          ([0, 0, 65, 250], 96, 3088), ([0, 40, 41, 128], 136, 2064)]


@pytest.mark.parametrize("ends,N,K", GROUPS)
@pytest.mark.parametrize("gated,rest", [(False, 0), (True, 0), (False, 21), (True, 3)])
def test_product_by_groups(ends, N, K, gated, rest):
    G, M = len(ends) - 1, ends[-1] + rest
    offsets = torch.tensor(ends, dtype=torch.int32)
    x, (w, ws) = normal(M, M, K, dtype=BF16), weights(N, G, N, K)
    q, scale = quantized(x)
    want = product(q, scale, w, ws, offsets, gated, BF16)
    args = (x.to(DEV), w.to(DEV), ws.to(DEV), offsets.to(DEV), gated)
    got = ffn.matmul_int8(*args)
    ffnmodel.within(got, *want, "groups")
    assert not got[ends[-1]:].any()                       # rows of no group
    out = torch.full_like(got, 7.0)
    version = out._version
    assert ffn.matmul_int8(*args, out=out) is out and out._version > version
    assert torch.equal(out[:ends[-1]], got[:ends[-1]]) and bool((out[ends[-1]:] == 7.0).all())


def test_largest_sums_are_exact():
    K = 1 << 17
    q = torch.full((3, K), 127, dtype=torch.int8)
    q[1] = -127
    w = torch.full((20, K), 127, dtype=torch.int8)
    one = torch.ones(20)
    got = ffn.matmul_int8((q.to(DEV), torch.ones(3, device=DEV)), w.to(DEV), one.to(DEV), dtype=F32).cpu()
    top = 127.0 * 127.0 * K
    assert got[0].tolist() == [top] * 20 and got[1].tolist() == [-top] * 20


def test_rows_apart_no_rows_and_bad_scales():
    q, scale = quantized(normal(1, 40, 64))
    w, ws = weights(2, 50, 64)
    wide = torch.full((40, 96), 55, dtype=torch.int8)
    wide[:, 16:80] = q
    got = ffn.matmul_int8((wide.to(DEV)[:, 16:80], scale.to(DEV)), w.to(DEV), ws.to(DEV), dtype=F32)
    ffnmodel.within(got, *product(q, scale, w, ws, None, False, F32), "rows apart")
    assert ffn.matmul_int8(torch.zeros(0, 64, dtype=BF16, device=DEV), w.to(DEV), ws.to(DEV)).shape == (0, 50)
    x = normal(3, 9, 64)
    x[4, 4], x[5, 5] = float("nan"), float("inf")
    got = ffn.matmul_int8(x.to(DEV), w.to(DEV), ws.to(DEV)).cpu()
    assert torch.isnan(got[4:6]).all() and torch.isfinite(got[:4]).all() and torch.isfinite(got[6:]).all()


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes between the first and the last row and between the weights."""
    K, ld, M = 64, 1 << 26, 70
    flat = torch.zeros(M * ld, dtype=torch.int8, device=DEV)
    rows = flat.view(M, ld)[:, :K]
    q, scale = quantized(normal(1, M, K))
    rows.copy_(q)
    w, ws = weights(2, 30, K)
    got = ffn.matmul_int8((rows, scale.to(DEV)), w.to(DEV), ws.to(DEV), dtype=F32)
    ffnmodel.within(got, *product(q, scale, w, ws, None, False, F32), "rows far apart")


def test_forward_only_and_refusals():
    x, (w, ws) = normal(1, 8, 64).to(DEV), weights(2, 20, 64)
    w, ws = w.to(DEV), ws.to(DEV)
    asked = x.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="forward only"):
        ffn.matmul_int8(asked, w, ws).sum().backward()
    with pytest.raises(RuntimeError, match="forward only"):
        ffn.quantize(asked)[1].sum().backward()
    with pytest.raises(RuntimeError, match="forward only"):
        ffn.matmul_int8(x, w, ws.clone().requires_grad_()).sum().backward()
    for kw, kind in ((dict(w=w.float()), TypeError), (dict(w_scale=ws.half()), TypeError), (dict(w=w.t()), ValueError),
                     (dict(w_scale=ws[:-1]), ValueError), (dict(x=x[:, :48]), ValueError), (dict(x=x.double()), TypeError),
                     (dict(dtype=torch.float64), TypeError), (dict(x=(x, x)), (TypeError, ValueError)),
                     (dict(offsets=torch.zeros(2, dtype=torch.int32, device=DEV)), ValueError),
                     (dict(out=torch.zeros(8, 21, device=DEV)), ValueError),
                     (dict(out=torch.zeros(8, 20, device=DEV), dtype=BF16), TypeError),
                     (dict(w=w[:, :60].contiguous(), x=x[:, :60]), moe.TopoepError),
                     (dict(w=w[:19], w_scale=ws[:19], gated=True), moe.TopoepError), (dict(w=w.cpu()), TypeError), (dict(gated=torch.ones(())), TypeError), (dict(gated=torch.ones(())), TypeError)):
        with pytest.raises(kind):
            ffn.matmul_int8(**{**dict(x=x, w=w, w_scale=ws), **kw})
