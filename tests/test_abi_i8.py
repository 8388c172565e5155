"""CPU-only checks of the operators around an 8-bit linear layer: sizes and argument errors are found on the host, before
any launch, by the C ABI and by the binding."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def bl():
    import paper_2310_11453_amd as lib
    if not lib.LIB_PATH.exists():
        from paper_2310_11453_amd.build import build
        build(verbose=False)
    lib.load_library()
    return lib


@pytest.fixture(scope="module")
def lib(bl):
    return bl.load_library()


ONE = ctypes.c_void_p(256)  # never dereferenced: every call below fails, or has nothing to do, before a launch
ODD = ctypes.c_void_p(264)  # as little, and not 16-byte aligned
TWO = ctypes.c_void_p(512)  # as little
BIG = 1 << 40


def test_sizes(bl):
    # whole tiles of 16 x 64 codes
    assert bl.packed_bytes_i8(512, 256) == 512 * 256
    assert bl.packed_bytes_i8(17, 96) == 32 * 128 and bl.packed_bytes_i8(1, 32) == 16 * 64
    for bad in [(0, 32), (16, 48), (16, 0), (-1, 32), ((1 << 30) + 1, 32), (1 << 30, 2048)]:
        assert bl.packed_bytes_i8(*bad) == 0
    assert bl.workspace_bytes(bl.OP_QUANT_RMSNORM, 100, 1, 256) == 0
    assert bl.workspace_bytes(bl.OP_QUANT_RMSNORM, 100, 1, 256, True) >= 100 * 8
    assert bl.workspace_bytes(bl.OP_RMSNORM_BACKWARD, 100, 1, 256) >= 256 * 8
    assert bl.workspace_bytes(bl.OP_BACKWARD_I8, 100, 512, 256) >= 2 * (100 * 512 + 256 * 512 + 256 * 100)
    for op in (bl.OP_QUANT_RMSNORM, bl.OP_RMSNORM_BACKWARD, bl.OP_MATMUL_I8, bl.OP_BACKWARD_I8):
        assert bl.workspace_bytes(op, -1, 512, 256, True) == 0 and bl.workspace_bytes(op, 8, 512, 250, True) == 0
        assert bl.workspace_bytes(op, 0, 512, 256, True) <= bl.workspace_bytes(op, 1, 512, 256, True)
    for op in (bl.OP_MATMUL_I8, bl.OP_BACKWARD_I8):
        assert bl.workspace_bytes(op, 8, 0, 256) == 0 and bl.workspace_bytes(op, 8, 512, 65568) == 0


def rms(lib, X=ONE, x_type=0, R=ONE, h_type=1, M=8, K=64, gain=ONE, eps=1e-5, gran=0, H=TWO, codes=ONE, gamma=ONE,
        xhat=None, ws=ONE, ws_bytes=BIG):
    return lib.bitlinear_quant_rmsnorm(X, x_type, R, h_type, M, K, gain, eps, gran, H, codes, gamma, ONE, xhat, ws, ws_bytes,
                                       None)


def test_quant_rmsnorm_refusals(lib):
    assert rms(lib, M=-1) == -2 and rms(lib, K=48) == -2 and rms(lib, K=0) == -2 and rms(lib, M=1 << 30, K=2048) == -2
    assert rms(lib, x_type=2) == -3 and rms(lib, h_type=7) == -3 and rms(lib, gran=2) == -3
    for eps in (-1e-5, math.inf, math.nan):
        assert rms(lib, eps=eps) == -3
    assert rms(lib, X=None) == -1 and rms(lib, codes=None) == -1 and rms(lib, gamma=None) == -1
    assert rms(lib, R=None) == -3  # H without a residual
    assert rms(lib, H=ONE) == -3 and rms(lib, H=ONE, x_type=1, gran=1, ws=None) == -4  # over x of another type, of its own
    for odd in ("X", "R", "H", "gain", "codes", "xhat"):
        assert rms(lib, **{odd: ODD}) == -3
    assert rms(lib, gran=1, ws=None, ws_bytes=0) == -4 and rms(lib, gran=1, ws_bytes=32) == -4
    assert rms(lib, M=0, X=None, codes=None, gran=1, ws=None) == 0


def rms_backward(lib, G=ONE, g_type=0, H=ONE, h_type=0, dR=ONE, d_type=0, M=8, K=64, gain=ONE, eps=1e-5, dH=TWO, dgain=ONE,
                 ws=ONE, ws_bytes=BIG):
    return lib.bitlinear_rmsnorm_backward(G, g_type, H, h_type, dR, d_type, M, K, gain, eps, dH, dgain, ws, ws_bytes, None)


def test_rmsnorm_backward_refusals(lib):
    assert rms_backward(lib, M=-1) == -2 and rms_backward(lib, K=40) == -2
    assert rms_backward(lib, g_type=2) == -3 and rms_backward(lib, h_type=2) == -3 and rms_backward(lib, d_type=-1) == -3
    assert rms_backward(lib, eps=-1.0) == -3 and rms_backward(lib, eps=math.nan) == -3
    assert rms_backward(lib, G=None) == -1 and rms_backward(lib, H=None) == -1 and rms_backward(lib, dH=None) == -1
    for odd in ("G", "H", "dR", "gain", "dH"):
        assert rms_backward(lib, **{odd: ODD}) == -3
    for over in ("G", "H"):  # over an operand of another type
        assert rms_backward(lib, d_type=1, **{over: TWO}) == -3
        assert rms_backward(lib, **{over: TWO}, ws=None) == -4
    assert rms_backward(lib, ws=None, ws_bytes=0) == -4 and rms_backward(lib, ws_bytes=64) == -4
    assert rms_backward(lib, M=0, G=None, ws=None) == 0


def test_pack_refusals(lib):
    pack = lambda W=ONE, t=0, N=48, K=64, p=ONE, s=ONE: lib.bitlinear_pack_weights_i8(W, t, N, K, p, s, None)  # noqa: E731
    assert pack(N=0) == -2 and pack(K=16) == -2 and pack(t=3) == -3 and pack(t=-1) == -3
    assert pack(W=None) == -1 and pack(p=None) == -1 and pack(s=None) == -1 and pack(W=ODD) == -3 and pack(p=ODD) == -3
    unpack = lambda p=ONE, s=ONE, N=48, K=64, t=0, o=ONE: lib.bitlinear_unpack_weights_i8(p, s, N, K, t, o, None)  # noqa: E731
    assert unpack(N=0) == -2 and unpack(K=16) == -2 and unpack(t=3) == -3
    assert unpack(p=None) == -1 and unpack(s=None) == -1 and unpack(o=None) == -1 and unpack(o=ODD) == -3


def product(lib, codes=ONE, gamma=ONE, M=8, K=64, packed=ONE, N=48, scale=ONE, gran=0, flags=0, y_type=0, Y=ONE):
    return lib.bitlinear_matmul_i8(codes, gamma, M, K, packed, N, scale, gran, flags, y_type, Y, None, 0, None)


def test_product_refusals(lib):
    assert product(lib, M=-1) == -2 and product(lib, K=48) == -2 and product(lib, N=0) == -2
    assert product(lib, K=65568) == -3 and product(lib, gran=3) == -3 and product(lib, flags=1) == -3
    assert product(lib, y_type=2) == -3 and product(lib, flags=2, y_type=1) == -3
    for null in ("codes", "gamma", "packed", "scale", "Y"):
        assert product(lib, **{null: None}) == -1
    assert product(lib, flags=2, codes=None, gamma=None, scale=None) == -1
    assert product(lib, codes=ODD) == -3 and product(lib, packed=ODD) == -3
    assert product(lib, M=0, codes=None, Y=None) == 0


def backward(lib, dY=ONE, dy_type=1, M=8, N=48, K=64, codes=ONE, gamma=ONE, gran=1, packed=ONE, scale=ONE, dX=ONE, dx_type=1,
             dW=ONE, ws=ONE, ws_bytes=BIG):
    return lib.bitlinear_backward_ste_i8(dY, dy_type, M, N, K, codes, gamma, gran, packed, scale, dX, dx_type, dW, ws, ws_bytes,
                                         None)


def test_backward_refusals(lib):
    assert backward(lib, M=-1) == -2 and backward(lib, K=48) == -2 and backward(lib, N=0) == -2
    assert backward(lib, K=65568) == -3 and backward(lib, gran=3) == -3
    assert backward(lib, dy_type=2) == -3 and backward(lib, dx_type=2) == -3
    for null in ("dY", "codes", "gamma", "packed", "scale"):
        assert backward(lib, **{null: None}) == -1
    assert backward(lib, dY=ODD) == -3 and backward(lib, codes=ODD) == -3 and backward(lib, packed=ODD) == -3
    assert backward(lib, dX=ODD) == -3
    assert backward(lib, ws=None) == -4 and backward(lib, ws_bytes=1000) == -4
    # what a missing output needs is not looked at
    assert backward(lib, dX=None, packed=None, scale=None, ws=None) == -4
    assert backward(lib, dW=None, codes=None, gamma=None, ws=None) == -4
    assert backward(lib, dX=None, dW=None, ws=None) == 0 and backward(lib, M=0, dY=None, ws=None) == 0


def test_binding_refuses_what_is_not_on_the_gpu(bl):
    x, c = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8)
    for call in (lambda: bl.bitlinear_quant_rmsnorm(x), lambda: bl.bitlinear_rmsnorm_backward(x, x),
                 lambda: bl.bitlinear_pack_weights_i8(x), lambda: bl.bitlinear_unpack_weights_i8(c, None, 4, 64),
                 lambda: bl.bitlinear_matmul_i8(c, None, c, 4, None),
                 lambda: bl.bitlinear_backward_ste_i8(x, c, None, None, None)):
        with pytest.raises(bl.BitLinearError):
            call()


def test_more_tokens_than_a_size_can_hold(bl, lib):
    """M * K past 2^40, N * K within it."""
    assert product(lib, M=1 << 30, K=2048, N=16) == -2 and backward(lib, M=1 << 30, K=2048, N=16) == -2
    for op in (bl.OP_MATMUL_I8, bl.OP_BACKWARD_I8):
        assert bl.workspace_bytes(op, 1 << 30, 16, 2048) == 0
    # at the bound the next argument is looked at
    assert product(lib, M=1 << 29, K=2048, N=16, codes=None) == -1 and backward(lib, M=1 << 29, K=2048, N=16, dY=None) == -1
