"""CPU-only checks of the operators of a mixture of BitLinear layers: sizes and argument errors are found on the host,
before any launch, by the C ABI and by the binding."""
import ctypes

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
BIG = 1 << 40


def test_sizes(bl):
    # a sort within one workgroup needs nothing, a longer one a count for each of them and each expert, and a sum
    assert bl.workspace_bytes_experts(bl.OP_ROUTE, 2048, 2, 0, 0, 8) == 0
    assert bl.workspace_bytes_experts(bl.OP_ROUTE, 2049, 2, 0, 0, 8) >= 3 * 8 * 4
    assert bl.workspace_bytes_experts(bl.OP_ROUTE, 1 << 24, 1, 0, 0, 256) >= 4097 * 256 * 4
    assert bl.workspace_bytes_experts(bl.OP_QUANT_NONLINEAR, 100, 1, 0, 0, 0) == 0
    assert bl.workspace_bytes_experts(bl.OP_QUANT_NONLINEAR, 100, 1, 0, 0, 0, True) >= 100 * 16 + 4
    # no transposed copy of dY (200 slots and more of 512 bf16) with one gamma a tensor
    per_token = bl.workspace_bytes_experts(bl.OP_BACKWARD, 100, 2, 512, 256, 8)
    assert 0 < bl.workspace_bytes_experts(bl.OP_BACKWARD, 100, 2, 512, 256, 8, True) <= per_token - 200 * 512 * 2
    assert bl.workspace_bytes_experts(bl.OP_QUANT_NONLINEAR, 1 << 24, 1, 0, 0, 0, True) == 0
    for bad in [(bl.OP_ROUTE, -1, 2, 0, 0, 8), (bl.OP_ROUTE, (1 << 24) + 1, 1, 0, 0, 8), (bl.OP_ROUTE, 8, 2, 0, 0, 257),
                (bl.OP_BACKWARD, 8, 2, 512, 250, 8), (bl.OP_BACKWARD, 8, 0, 512, 256, 8), (bl.OP_BACKWARD, 8, 2, 0, 256, 8),
                (bl.OP_BACKWARD, 8, 2, 512, 65568, 8), (bl.OP_FORWARD, 8, 2, 512, 256, 8), (99, 8, 2, 512, 256, 8)]:
        assert bl.workspace_bytes_experts(*bad) == 0


def route(lib, M=8, top_k=2, E=4, ids=ONE, order=ONE, ws=ONE, ws_bytes=BIG):
    return lib.bitlinear_route(ids, M, top_k, E, order, ONE, ONE, ws, ws_bytes, None)


def test_route_refusals(lib):
    assert route(lib, M=-1) == -2 and route(lib, top_k=0) == -2 and route(lib, top_k=65) == -2
    assert route(lib, E=0) == -2 and route(lib, E=257) == -2 and route(lib, M=1 << 29, top_k=4) == -2
    assert route(lib, M=(1 << 24) + 1, top_k=1) == -3
    assert route(lib, ids=None) == -1 and route(lib, order=None) == -1
    assert route(lib, M=4097, ws=None, ws_bytes=0) == -4 and route(lib, M=4097, ws_bytes=8) == -4
    assert route(lib, M=0, ids=None, ws=None, ws_bytes=0) == 0


def product(lib, M=8, top_k=2, K=64, E=4, N=48, gran=0, flags=0, codes=ONE, offsets=ONE, Y=ONE):
    return lib.bitlinear_matmul_experts(codes, ONE, ONE, M, top_k, K, ONE, offsets, E, ONE, N, ONE, gran, flags, Y, None)


def test_product_refusals(lib):
    assert product(lib, M=-1) == -2 and product(lib, K=48) == -2 and product(lib, N=0) == -2 and product(lib, E=0) == -2
    assert product(lib, E=257) == -2 and product(lib, top_k=0) == -2 and product(lib, M=1 << 30, top_k=2) == -2
    assert product(lib, gran=2) == -3 and product(lib, flags=1) == -3 and product(lib, K=65568) == -3
    assert product(lib, codes=None) == -1 and product(lib, offsets=None) == -1 and product(lib, Y=None) == -1
    assert product(lib, codes=ODD) == -3
    assert product(lib, M=0, codes=None, offsets=None, Y=None) == 0


def backward(lib, M=8, top_k=2, N=48, K=64, gran=0, E=4, dY=ONE, codes=ONE, packed=ONE, dX=ONE, dW=ONE, ws=ONE,
             ws_bytes=BIG):
    return lib.bitlinear_backward_ste_experts(dY, M, top_k, N, K, codes, ONE, gran, ONE, ONE, E, packed, ONE, dX, dW, ws,
                                              ws_bytes, None)


def test_backward_refusals(lib, bl):
    assert backward(lib, K=40) == -2 and backward(lib, M=-1) == -2 and backward(lib, E=0) == -2
    assert backward(lib, gran=7) == -3 and backward(lib, K=65568) == -3
    assert backward(lib, dY=None) == -1 and backward(lib, packed=None) == -1 and backward(lib, codes=None) == -1
    assert backward(lib, codes=ODD) == -3 and backward(lib, packed=ODD) == -3
    # dY is read 16 bytes at a time where its rows are whole numbers of 32 columns; else not
    assert backward(lib, N=64, dY=ODD) == -3 and backward(lib, N=64, dY=ODD, dX=None) == -3
    assert backward(lib, N=48, dY=ODD, ws=None) == -4
    need = bl.workspace_bytes_experts(bl.OP_BACKWARD, 8, 2, 48, 64, 4)
    assert backward(lib, ws=None, ws_bytes=0) == -4 and backward(lib, ws_bytes=need // 2) == -4
    assert backward(lib, M=0, dY=None) == 0 and backward(lib, dX=None, dW=None, dY=None) == 0


def test_combine_refusals(lib):
    def fwd(M=8, top_k=2, N=32, slots=ONE, Y=ONE):
        return lib.bitlinear_combine(slots, ONE, None, M, top_k, N, Y, None)

    def bwd(M=8, top_k=2, N=32, slots=ONE, dweights=ONE, dY=ONE):
        return lib.bitlinear_combine_backward(dY, slots, ONE, None, M, top_k, N, ONE, dweights, None)

    for call in (fwd, bwd):
        assert call(M=-1) == -2 and call(top_k=0) == -2 and call(N=0) == -2 and call(M=1 << 30) == -2
        assert call(M=0, slots=None) == 0
    assert fwd(slots=None) == -1 and fwd(Y=None) == -1 and bwd(slots=None) == -1 and bwd(dY=None) == -1


def test_nonlinear_refusals(lib, bl):
    def fwd(M=8, K=64, fn=2, gran=0, U=ONE, check=ONE, scale=ONE, ws=ONE, ws_bytes=BIG):
        return lib.bitlinear_quant_nonlinear(U, M, K, fn, 1e-5, None, gran, ONE, ONE, ONE, check, scale, ws, ws_bytes, None)

    def bwd(M=8, K=64, fn=2, kind=1, dX=ONE, check=ONE, dU=ONE):
        return lib.bitlinear_nonlinear_backward(dX, check, ONE, M, K, fn, 1e-5, None, kind, dU, None)

    for call in (fwd, bwd):
        assert call(M=-1) == -2 and call(K=48) == -2 and call(K=0) == -2
        assert call(fn=4) == -3 and call(fn=-1) == -3 and call(K=32800) == -3
        assert call(M=0) == 0
        assert call(M=1 << 24) == -3 and call(M=(1 << 24) - 1, K=4128) == -3
    assert fwd(gran=2) == -3 and fwd(U=None) == -1 and fwd(scale=None) == -1 and bwd(check=None) == -1 and bwd(dU=None) == -1
    assert bwd(kind=2) == -3 and bwd(dX=ODD) == -3 and bwd(dU=ODD) == -3 and bwd(check=ODD) == -3
    assert fwd(U=ODD) == -3 and fwd(check=ODD) == -3 and fwd(gran=1, ws=ODD) == -3
    assert fwd(gran=1, ws=None, ws_bytes=0) == -4 and fwd(gran=1, ws_bytes=8 * 16) == -4


def test_binding_refuses_what_is_not_on_the_gpu(bl):
    ids, x = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 64)
    for call in (lambda: bl.bitlinear_route(ids, 4), lambda: bl.bitlinear_quant_nonlinear(x),
                 lambda: bl.bitlinear_combine(x, ids), lambda: bl.bitlinear_combine_backward(x, None, ids),
                 lambda: bl.bitlinear_nonlinear_backward(x, ids, x), lambda: bl.bitlinear_pack_weights_experts(x)):
        with pytest.raises(bl.BitLinearError):
            call()


def test_functions(lib, bl):
    """Which functions there are, and that any other number is refused before a pointer is looked at."""
    def fwd(fn):
        return lib.bitlinear_quant_nonlinear(None, 8, 64, fn, 1e-5, None, 0, ONE, ONE, ONE, ONE, ONE, ONE, BIG, None)

    def bwd(fn):
        return lib.bitlinear_nonlinear_backward(None, ONE, ONE, 8, 64, fn, 1e-5, None, 1, ONE, None)

    known = set(bl.FUNCTIONS.values())
    assert known == {0, 1, 2, 3, 8}
    for fn in range(-2, 20):
        assert fwd(fn) == bwd(fn) == (-1 if fn in known else -3)
