"""The C ABI of the experts' products (include/topoep_ffn.h): every declared
function is exported and bound, the structs match, and what the host refuses is
refused before any device call (placeholder pointers are never launched on)."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "topoep_ffn.h")
EINVAL, EWORKSPACE, ELIMIT, OK = -1, -2, -4, 0


@pytest.fixture(scope="module")
def ffn():
    from paper_2609_35481_amd import ffn
    return ffn


def test_library_exports_every_declared_symbol(ffn):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^\s*int\s+(topoep_\w+)\s*\(", text, flags=re.M))
    assert names == set(ffn.EXPORTS)
    for name in names:
        assert hasattr(ffn._lib, name), name


def test_struct_layout_matches_header(ffn):
    assert ctypes.sizeof(ffn.Ffn) == 16
    assert ctypes.sizeof(ffn.Rows) == 40 and ffn.Rows.num_experts.offset == 36
    assert ctypes.sizeof(ffn.Int8) == 20


def test_rows_refusals(ffn):
    B, F = ffn._lib.topoep_expert_rows_workspace_bytes, ffn._lib.topoep_expert_rows
    out = ctypes.c_size_t(0)
    assert B(8, 2, 16, out) == OK and out.value % 256 == 0
    need = out.value
    assert B(0, 2, 16, out) == OK
    for bad in ((-1, 2, 16), (8, 0, 16), (8, 2, 0), (1 << 30, 2, 16)):
        assert B(*bad, out) == EINVAL, bad
    assert B(8, 2, 1025, out) == ELIMIT and B(8, 2, 16, None) == EINVAL
    good = dict(ids=256, T=8, k=2, slot=None, E=16, L=16, offsets=512, pairs=1024, places=2048, ws=4096, size=need)

    def call(**kw):
        return F(*{**good, **kw}.values(), None)

    for name in ("ids", "offsets", "pairs", "places", "ws"):
        assert call(**{name: None}) == EINVAL, name
    for kw in (dict(T=-1), dict(k=0), dict(T=1 << 30), dict(E=0), dict(L=0)):
        assert call(**kw) == EINVAL, kw
    assert call(L=1025) == ELIMIT
    assert call(size=need - 1) == EWORKSPACE and call(ws=4096 + 128) == EWORKSPACE


def test_block_refusals(ffn):
    N, F, B = ffn._lib.topoep_ffn_bytes, ffn._lib.topoep_ffn_forward, ffn._lib.topoep_ffn_backward
    f = ffn.Ffn(64, 32, 4, 1)
    rows = ffn.Rows(256, 512, 1024, 2048, 2, 8)
    need = [ctypes.c_size_t(0) for _ in range(3)]
    assert N(f, 8, rows, *need) == OK and all(n.value % 256 == 0 and n.value > 0 for n in need)
    assert N(f, 8, rows, None, None, None) == OK
    for bad in ((63, 32, 4, 1), (64, 31, 4, 1), (0, 32, 4, 1), (64, 0, 4, 1), (64, 32, 0, 1), (64, 32, 4, 0),
                (64, 32, 4, 3), ((1 << 17) + 8, 8, 1, 1), (1 << 17, 1 << 14, 1, 1)):
        assert N(ffn.Ffn(*bad), 8, rows, *need) == EINVAL, bad
    assert N(None, 8, rows, *need) == EINVAL and N(f, -1, rows, *need) == EINVAL
    assert N(f, 8, None, *need) == EINVAL                     # four blocks, no rows
    assert N(f, 8, ffn.Rows(256, 512, 1024, 2048, 0, 8), *need) == EINVAL
    assert N(f, 1 << 30, rows, *need) == EINVAL
    assert N(f, 8, ffn.Rows(256, 512, 1024, 2048, 2, 0), *need) == EINVAL
    assert N(f, 8, ffn.Rows(256, 512, 1024, 2048, 65, 128), *need) == ELIMIT
    assert N(ffn.Ffn(64, 32, 1025, 1), 8, rows, *need) == ELIMIT
    assert N(f, 8, rows, *need) == OK
    fw, saved, bw = (n.value for n in need)
    good = dict(f=f, x=256, ldx=64, T=8, rows=rows, up=512, down=1024, out=2048, saved=4096, ws=8192, size=fw)

    def forward(**kw):
        return F(*{**good, **kw}.values(), None)

    for name in ("x", "up", "down", "out", "ws", "f"):
        assert forward(**{name: None}) == EINVAL, name
    for name in ("x", "up", "down", "out", "saved"):
        assert forward(**{name: good[name] + 8}) == EINVAL, name
    for i in range(4):
        fields = [256, 512, 1024, 2048]
        fields[i] = None
        assert forward(rows=ffn.Rows(*fields, 2, 8)) == EINVAL, i
    assert forward(ldx=56) == EINVAL and forward(ldx=68) == EINVAL and forward(ldx=1 << 60) == EINVAL
    assert forward(size=fw - 1) == EWORKSPACE and forward(ws=8192 + 128) == EWORKSPACE
    assert forward(T=0, x=None, ws=None) == OK
    good = dict(f=f, x=256, ldx=64, T=8, rows=rows, up=512, down=1024, saved=2048, grad=4096, dx=8192, dw=16384,
                dup=32768, ddown=65536, ws=1 << 17, size=bw)

    def backward(**kw):
        return B(*{**good, **kw}.values(), None)

    for name in ("x", "up", "down", "saved", "grad", "ws", "f"):
        assert backward(**{name: None}) == EINVAL, name
    for name in ("x", "up", "down", "saved", "grad", "dx", "dup", "ddown"):
        assert backward(**{name: good[name] + 8}) == EINVAL, name
    assert backward(ldx=56) == EINVAL and backward(size=bw - 1) == EWORKSPACE and backward(ws=(1 << 17) + 16) == EWORKSPACE


def test_quantize_refusals(ffn):
    Q = ffn._lib.topoep_quantize
    good = dict(x=256, dtype=1, ldx=64, M=8, K=64, q=512, scale=1024)

    def call(**kw):
        return Q(*{**good, **kw}.values(), None)

    for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(dtype=3), dict(dtype=-1), dict(ldx=63), dict(M=-1),
               dict(K=0), dict(x=257), dict(scale=1026), dict(ldx=1 << 60)):
        assert call(**kw) == EINVAL, kw
    assert call(M=0, x=None) == OK


def test_int8_refusals(ffn):
    W, F = ffn._lib.topoep_matmul_int8_workspace_bytes, ffn._lib.topoep_matmul_int8
    p = ffn.Int8(48, 64, 3, 1, 1)
    need = ctypes.c_size_t(0)
    assert W(p, 8, need) == OK and need.value % 256 == 0
    for bad in ((0, 64, 3, 0, 1), (47, 64, 3, 1, 1), (48, 63, 3, 0, 1), (48, 0, 3, 0, 1), (48, 64, 0, 0, 1),
                (48, 64, 3, 0, 3), (48, 64, 3, 0, -1), (48, (1 << 17) + 16, 3, 0, 1), ((1 << 20) + 1, 64, 1, 0, 1)):
        assert W(ffn.Int8(*bad), 8, need) == EINVAL, bad
    assert W(ffn.Int8(48, 64, 1025, 0, 1), 8, need) == ELIMIT
    assert W(p, -1, need) == EINVAL and W(None, 8, need) == EINVAL and W(p, 8, None) == EINVAL
    assert W(p, 8, need) == OK
    good = dict(p=p, q=256, ldq=64, scale=512, M=8, offsets=1024, keep=0, w=2048, ws=4096, out=8192, work=16384,
                size=need.value)

    def call(**kw):
        return F(*{**good, **kw}.values(), None)

    for name in ("p", "q", "scale", "w", "ws", "out", "offsets"):
        assert call(**{name: None}) == EINVAL, name
    for name in ("q", "w", "out"):
        assert call(**{name: good[name] + 8}) == EINVAL, name
    assert call(ldq=48) == EINVAL and call(ldq=72) == EINVAL and call(ldq=1 << 60) == EINVAL
    assert call(work=16384 + 16) == EWORKSPACE
    p = good["p"] = ffn.Int8(64, 4096, 1, 0, 1)           # workgroups share the inner axis: their sums
    assert W(p, 100, need) == OK and need.value >= 2 * 100 * 64 * 4
    assert call(M=100, size=need.value - 1, ldq=4096) == EWORKSPACE and call(M=100, size=0, ldq=4096) == EWORKSPACE
    assert call(M=0, q=None) == OK


def test_rows_and_elements_that_32_bits_cannot_count_past(ffn):
    # a tile's last row, or a lane's next element, lies behind the last one there is
    out = ctypes.c_size_t(0)
    most, f, p = 1 << 30, ffn.Ffn(8, 8, 1, 1), ffn.Int8(16, 16, 1, 0, 1)
    two = ffn.Rows(256, 512, 1024, 2048, 2, 8)
    for rows, T in ((None, most), (two, most // 2)):
        assert ffn._lib.topoep_ffn_bytes(f, T, rows, out, out, out) == OK
        assert ffn._lib.topoep_ffn_bytes(f, T + 1, rows, out, out, out) == EINVAL
        assert ffn._lib.topoep_ffn_forward(f, 256, 8, T + 1, rows, 512, 1024, 2048, None, 4096, 1 << 40, None) == EINVAL
        assert ffn._lib.topoep_ffn_backward(f, 256, 8, T + 1, rows, 512, 1024, 2048, 256, 512, None, 1024, 2048, 4096,
                                            1 << 40, None) == EINVAL
    assert ffn._lib.topoep_matmul_int8_workspace_bytes(p, most, out) == OK
    assert ffn._lib.topoep_matmul_int8_workspace_bytes(p, most + 1, out) == EINVAL
    assert ffn._lib.topoep_matmul_int8(p, 256, 16, 512, most + 1, None, 0, 1024, 2048, 4096, 8192, 1 << 40, None) == EINVAL
    for K in (most + 1, (1 << 31) - 8):
        assert ffn._lib.topoep_quantize(256, 0, 1 << 31, 1, K, 512, 1024, None) == EINVAL


def test_binding_refuses_before_the_gpu(ffn):
    cpu = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call in (lambda: ffn.feed_forward(cpu, torch.zeros(64, 64), torch.zeros(64, 32)),
                 lambda: ffn.experts(cpu, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(2, 64, 64),
                                     torch.zeros(2, 64, 32)),
                 lambda: ffn.expert_rows(torch.zeros(4, 2, dtype=torch.int32), 8), lambda: ffn.quantize(cpu),
                 lambda: ffn.matmul_int8(cpu, torch.zeros(8, 64, dtype=torch.int8), torch.zeros(8))):
        with pytest.raises(TypeError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="dimensions"):
        ffn.quantize(torch.zeros(4))
    with pytest.raises(TypeError, match="not a tensor"):
        ffn.quantize([1.0])
    with pytest.raises(ValueError, match="beyond 32 bits"):
        ffn.expert_rows(torch.zeros(4, 2, dtype=torch.int32), 1 << 40)
    with pytest.raises(ValueError, match="scale"):
        ffn.matmul_int8((cpu,), torch.zeros(8, 64, dtype=torch.int8), torch.zeros(8))
