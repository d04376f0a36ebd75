"""Host-only checks of the entry points on grouped 4-bit weights: sizes, and refusals before a device is touched."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, ALIGN = 0, 1, 2, 3
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2207_08820_b200 import build
    build.build()
    from paper_2207_08820_b200 import _lib
    return _lib.lib()


@pytest.fixture(scope="module")
def at():
    buf = (ctypes.c_char * 8192)()
    yield (ctypes.addressof(buf) + 255) & ~255      # never dereferenced: validation fails first


def test_sizes(L):
    assert L.bs_w4_bytes(16, 128, 128, 0) == 1024 + 32
    assert L.bs_w4_bytes(17, 129, 32, 0) == 4 * (1024 + 4 * 32)
    assert L.bs_w4_bytes(17, 129, 64, 1) == 4 * (1024 + 2 * 64)
    assert L.bs_w4_bytes(1, 1, 1 << 20, 0) == 1024 + 32
    for bad in ((0, 128, 128), (16, 0, 128), (16, 128, 0), (16, 128, 48), (16, 128, 16), (16, 128, 192), (1 << 21, 128, 128), (16, 1 << 21, 128), (16, 128, 1 << 21), (16, 128, -128)):
        assert L.bs_w4_bytes(*bad, 0) == 0
    assert L.bs_w4_gemm_workspace_bytes(1, 64, 4611, 128, 4611) == 0
    assert L.bs_w4_gemm_workspace_bytes(5, 64, 4616, 128, 4616) == 0
    assert L.bs_w4_gemm_workspace_bytes(5, 64, 4611, 128, 4616) == 0
    assert L.bs_w4_gemm_workspace_bytes(5, 64, 4611, 128, 4611) == 5 * 4616 * 2
    assert L.bs_w4_gemm_workspace_bytes(0, 64, 4611, 128, 4611) == L.bs_w4_gemm_workspace_bytes(5, 64, 4611, 96, 4611) == 0
    assert L.bs_w4_gemm_workspace_bytes(300, 64, 4611, 128, 4611) == 300 * 4616 * 2
    assert L.bs_w4_gemm_workspace_bytes(4096, 64, 4611, 128, 4611) > 4096 * 4616 * 2       # parts of tiles as well
    assert L.bs_w4_moe_workspace_bytes(3, 2, 64, 50, 64) == 3 * 2 * 64 * 4 + 2 * 3 * 2 * 56 * 2
    assert L.bs_w4_moe_workspace_bytes(3, 2, 63, 50, 63) == 3 * 2 * 64 * 4 + 2 * 3 * 2 * 56 * 2 + 3 * 64 * 2
    assert L.bs_w4_moe_workspace_bytes(0, 2, 64, 50, 64) == 0


def test_quantise_and_prepare_refuse(L, at):
    def quantise(w=at, t=F32, O=16, K=128, ld=128, group=128, s=BF16, codes=at, scales=at, zeros=None):
        return L.bs_w4_quantise(w, t, O, K, ld, group, s, codes, scales, zeros, None)
    assert quantise(w=None) == quantise(codes=None) == quantise(scales=None) == INVALID
    assert quantise(t=3) == quantise(s=F32) == quantise(s=7) == quantise(O=0) == quantise(K=0) == quantise(ld=127) == quantise(group=0) == INVALID
    assert quantise(group=48) == quantise(O=(1 << 20) + 1) == UNSUPPORTED
    assert quantise(w=at + 8) == quantise(codes=at + 1) == quantise(scales=at + 2) == quantise(zeros=at + 1) == ALIGN

    def prepare(codes=at, scales=at, zeros=None, E=1, O=16, K=128, group=128, out=at):
        return L.bs_w4_prepare(codes, scales, zeros, E, O, K, group, out, None)
    assert prepare(codes=None) == prepare(scales=None) == prepare(out=None) == prepare(E=0) == prepare(O=-1) == prepare(K=0) == prepare(group=-32) == INVALID
    assert prepare(E=65536) == prepare(group=96) == UNSUPPORTED
    assert prepare(codes=at + 4) == prepare(scales=at + 2) == prepare(zeros=at + 1) == prepare(out=at + 8) == ALIGN


def test_gemm_refuses(L, at):
    def gemm(x=at, ldx=128, M=4, w=at, O=16, K=128, group=128, t=BF16, bias=None, y=at, ldy=16, ws=None, n=0):
        return L.bs_w4_gemm(x, ldx, M, w, O, K, group, 0, t, bias, y, ldy, ws, n, None)
    assert gemm(x=None) == gemm(w=None) == gemm(y=None) == gemm(M=-1) == gemm(O=0) == gemm(K=0) == gemm(ldx=127) == gemm(ldy=15) == gemm(t=F32) == gemm(t=9) == INVALID
    assert gemm(group=0) == INVALID and gemm(group=80) == gemm(M=(1 << 20) + 1) == UNSUPPORTED
    assert gemm(x=at + 2) == gemm(w=at + 4) == gemm(bias=at + 2) == gemm(y=at + 2) == gemm(ws=at + 8, n=99) == ALIGN
    assert gemm(ldx=129) == gemm(ldx=129, ws=at, n=4 * 128 * 2 - 1) == INVALID       # rows off 16-byte boundaries ask for a workspace
    assert gemm(M=0) == OK


def test_moe_refuses(L, at):
    def moe(x=at, ldx=64, T=3, router=at, E=4, H=64, I=48, gate=at, up=at, gu=32, down=at, gd=32, t=F16, k=2, y=at, experts=at, weights=at, ws=at, n=1 << 20):
        return L.bs_w4_moe(x, ldx, T, router, E, H, I, gate, up, gu, 0, down, gd, 0, t, k, 1, y, experts, weights, ws, n, None)
    for name in ("x", "router", "gate", "up", "down", "y", "experts", "weights"):
        assert moe(**{name: None}) == INVALID
        assert moe(**{name: at + 4}) == ALIGN
    assert moe(T=-1) == moe(E=0) == moe(H=0) == moe(I=0) == moe(ldx=63) == moe(k=0) == moe(k=5) == moe(t=F32) == moe(gu=0) == INVALID
    assert moe(E=513) == moe(E=64, k=33) == moe(gu=48) == moe(gd=192) == moe(T=16385) == UNSUPPORTED
    assert moe(ws=None) == moe(n=3 * 2 * 64 * 4 + 2 * 3 * 2 * 48 * 2 - 1) == INVALID and moe(ws=at + 8) == ALIGN
    assert moe(T=0) == OK


def test_binding_refuses_tensors_off_the_device():
    import torch
    from paper_2207_08820_b200 import api
    with pytest.raises(ValueError):
        api.quantise_w4(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        api.quantise_w4(torch.zeros(64))
    with pytest.raises(ValueError):
        api.quantise_w4(torch.zeros(4, 64), dtype=torch.float32)
    with pytest.raises(ValueError):
        api.prepare_w4(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.float16), group=32)
    w = api.W4Weights(torch.zeros(8, dtype=torch.uint8), 1, 16, 128, 128, False, torch.float16)
    with pytest.raises(ValueError):
        api.gemm_w4(torch.zeros(1, 128, dtype=torch.float16), w)
    with pytest.raises(ValueError):
        api.gemm_w4(torch.zeros(1, 128, dtype=torch.bfloat16), w)


def test_binding_refuses_what_requires_a_gradient():
    """Before the device is looked at: the messages tell the refusals apart."""
    import torch
    from paper_2207_08820_b200 import api
    t = torch.float16

    def weights(E, O, K):
        return api.W4Weights(torch.zeros(8, dtype=torch.uint8), E, O, K, 128, False, t)

    def tensors(*shapes, grad=None):
        return [torch.zeros(s, dtype=t, requires_grad=i == grad) for i, s in enumerate(shapes)]
    shapes = (2, 128), (16,), (2, 16)
    for grad in range(3):
        x, bias, out = tensors(*shapes, grad=grad)
        with pytest.raises(ValueError, match="gradient"):
            api.gemm_w4(x, weights(1, 16, 128), bias, out=out)
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
            api.gemm_w4(x, weights(1, 16, 128), bias, out=out)
    x, bias, out = tensors(*shapes)
    with pytest.raises(ValueError, match="CUDA"):
        api.gemm_w4(x, weights(1, 16, 128), bias, out=out)
    with pytest.raises(ValueError, match="gradient"):       # not a leaf
        api.gemm_w4(tensors((2, 128), grad=0)[0] * 2, weights(1, 16, 128))
    shapes = (2, 128), (4, 128), (2, 128)
    experts = weights(4, 16, 128), weights(4, 16, 128), weights(4, 128, 16)
    for grad in range(3):
        x, router, out = tensors(*shapes, grad=grad)
        with pytest.raises(ValueError, match="gradient"):
            api.moe_w4(x, router, *experts, 2, out=out)
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
            api.moe_w4(x, router, *experts, 2, out=out)
