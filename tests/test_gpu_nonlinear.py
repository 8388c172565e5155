"""The non-linear function, LayerNorm and quantiser in one pass, its 8-bit checkpoint and the backward pass from it, on the
GPU, against 64-bit evaluations on the CPU.

Tolerances.  f and f' are fp32 functions of u, taken to be off by at most 2^-21 of |u| (f) and of 1 + |u| (f'): eight
roundings each.  The statistics of a row are sums in fp64, so x^ = (h - mean) / dev is off by what f makes of it (x_error:
the value's and the mean's error over dev, and x^ times the deviation's, mean(|x^| error of h) / dev) and one rounding to
fp32.  A code may differ from the rounded 64-bit value only where that lies
this close to a half.  The checkpoint is two fp32 operations: equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, FN = 2.0 ** -24, 2.0 ** -8, 2.0 ** -21
EPS = 1e-5
FUNCTIONS = ["relu", "relu2", "gelu", "silu"]


@pytest.fixture(scope="module")
def bl():
    import paper_2310_11453_amd as lib
    lib.load_library()
    assert torch.cuda.is_available()
    return lib


def f(u, fn):
    if fn == "relu":
        return u.clamp_min(0)
    if fn == "relu2":
        return u.clamp_min(0) ** 2
    if fn == "gelu":
        return u * torch.special.ndtr(u)
    return u * torch.sigmoid(u)


def f_error(u, fn):
    """What f may be off by in fp32."""
    return FN * (u.abs() if fn != "relu2" else u * u)


def normal(h):
    mean = h.mean(1, keepdim=True)
    return (h - mean) / ((h - mean).square().mean(1, keepdim=True) + EPS).sqrt()


def x_error(u, x, dev, fn):
    """(what x^ may be off by, what dev may be off by relative to it)."""
    h_off = f_error(u, fn)
    dev_off = (x.abs() * h_off).mean(1, keepdim=True) / dev
    return (h_off + h_off.mean(1, keepdim=True)) / dev + x.abs() * dev_off, dev_off


def make_u(M, K, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    u = torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))
    if kind == "outliers":
        u = torch.where(torch.rand(M, K, generator=g) < 0.01, 30 * u, u)
    if kind == "offset":
        u = u + 40.0
    return u


def check_forward(bl, u, fn, per_tensor, got):
    codes, gamma, rowsum = (t.cpu() for t in got[:3])
    h = f(u.double(), fn)
    x = normal(h)
    dev = (h.var(1, correction=0, keepdim=True) + EPS).sqrt()
    off = x_error(u.double(), x, dev, fn)[0] + 2 * F32 * x.abs()
    g = x.abs().amax().reshape(1, 1) if per_tensor else x.abs().amax(1, keepdim=True)
    g_off = off.amax() if per_tensor else off.amax(1, keepdim=True)
    g = g.clamp_min(1e-5)
    assert bool(((gamma.double().view(-1, 1) - g).abs() <= g_off).all())
    t = x * 128 / g
    t_off = 128 / g * (off + x.abs() / g * g_off) + 4 * F32 * t.abs()
    assert float(t_off.max()) < 0.25  # the comparison below says something
    c = codes.double()
    assert bool(((c - t.clamp(-128, 127)).abs() <= 0.5 + t_off).all())
    assert torch.equal(rowsum, codes.sum(1, dtype=torch.int32))


def plain_check(u):
    M, K = u.shape
    blocks = torch.nn.functional.pad(u, (0, -K % 128)).view(M, -1, 128)
    big = blocks.abs().amax(2, keepdim=True)
    # (a number divided by a tensor is a reciprocal and a product in torch: two roundings)
    up = torch.where(big > 0, torch.full_like(big, 127.0) / big, 0.0)
    return (blocks * up).round().view(M, -1)[:, :K].to(torch.int8), (big / 127.0).squeeze(2)


# a row of one float4 group, short last blocks, one to sixteen waves a row, ragged pieces, more rows than fit once
SHAPES = [(1, 32), (5, 96), (3, 256), (33, 544), (64, 1024), (9, 2080), (2500, 2048), (40, 4096), (7, 5472), (130, 8192),
          (3, 12320), (2, 28672), (1, 32768)]


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("fn", FUNCTIONS)
@pytest.mark.parametrize("per_tensor", [False, True])
def test_forward_and_checkpoint(bl, M, K, fn, per_tensor):
    print(f"nonlinear M={M} K={K} {fn} per_tensor={per_tensor}", flush=True)
    u = make_u(M, K, M + K, "outliers" if K % 64 else "normal")
    got = bl.bitlinear_quant_nonlinear(u.cuda(), fn, per_tensor=per_tensor, checkpoint=True)
    check_forward(bl, u, fn, per_tensor, got)
    check, scale = plain_check(u)
    assert torch.equal(got[3].cpu(), check) and torch.equal(got[4].cpu(), scale)
    # without a checkpoint: the same codes
    bare = bl.bitlinear_quant_nonlinear(u.cuda(), fn, per_tensor=per_tensor)
    assert bare[3] is None and torch.equal(bare[0], got[0]) and torch.equal(bare[1], got[1])


@pytest.mark.parametrize("fn", FUNCTIONS)
def test_rows_that_lose_everything(bl, fn):
    """Zeros, a constant, all below zero, one element, tiny values."""
    u = torch.zeros(6, 288)
    u[1] = 3.0
    u[2] = -torch.rand(288, generator=torch.Generator().manual_seed(1)) - 0.5
    u[3, 200] = 5.0
    u[4] = 1e-30
    u[5] = torch.linspace(-1, 1, 288) * 1e-20
    codes, gamma, rowsum, check, scale = (t.cpu() for t in bl.bitlinear_quant_nonlinear(u.cuda(), fn, checkpoint=True))
    want, want_scale = plain_check(u)
    assert torch.equal(check, want) and torch.equal(scale, want_scale)
    for r in (0, 1, 4, 5):
        assert int(codes[r].abs().max()) == 0 and float(gamma[r]) == pytest.approx(1e-5)
    if fn in ("relu", "relu2"):
        assert int(codes[2].abs().max()) == 0
    du = bl.bitlinear_nonlinear_backward(torch.ones(6, 288, device="cuda"), check.cuda(), scale.cuda(), fn)
    assert bool(torch.isfinite(du.float()).all())


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("fn", FUNCTIONS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward(bl, M, K, fn, dtype):
    print(f"nonlinear backward M={M} K={K} {fn} {dtype}", flush=True)
    u = make_u(M, K, M + 2 * K, "outliers" if K % 64 else "normal")
    check, scale = plain_check(u)
    d = torch.randn(M, K, generator=torch.Generator().manual_seed(3))
    v = (check.float() * scale.repeat_interleave(128, 1)[:, :K]).double().requires_grad_()
    x = normal(f(v, fn))
    x.backward(d.double())
    ref = v.grad.detach()
    with torch.no_grad():
        if fn in ("relu", "relu2"):
            ref = torch.where(v > 0, ref, 0.0)
        h = f(v, fn)
        rstd = 1 / (h.var(1, correction=0, keepdim=True) + EPS).sqrt()
        vv = v.detach().requires_grad_()
        with torch.enable_grad():
            slope, = torch.autograd.grad(f(vv, fn).sum(), vv)
        m1, m2 = d.double().mean(1, keepdim=True), (d.double() * x).mean(1, keepdim=True)
        most = d.double().abs() + m1.abs() + (x * m2).abs()
        n_off, dev_off = x_error(v, x, 1 / rstd, fn)
        m2_off = (d.double().abs() * n_off).mean(1, keepdim=True)
        allowed = rstd * (slope.abs() * (most * (8 * F32 + dev_off) + m2.abs() * n_off + x.abs() * m2_off)
                          + most * FN * (1 + v.abs()) * (2 if fn == "relu2" else 1))
        got = bl.bitlinear_nonlinear_backward(d.cuda(), check.cuda(), scale.cuda(), fn, dtype=dtype)
        assert got.dtype == dtype
        if dtype == torch.bfloat16:
            allowed = allowed * (1 + BF16) + BF16 * ref.abs()
        assert bool(((got.cpu().double() - ref).abs() <= allowed).all())


@pytest.mark.parametrize("fn", FUNCTIONS)
def test_gradient_against_differences(bl, fn):
    """The fp32 gradient against central differences of sum(d x^) at the checkpoint, in 64 bits."""
    u = make_u(2, 160, 5)
    check, scale = plain_check(u)
    d = torch.randn(2, 160, generator=torch.Generator().manual_seed(4))
    v = (check.float() * scale.repeat_interleave(128, 1)[:, :160]).double()
    got = bl.bitlinear_nonlinear_backward(d.cuda(), check.cuda(), scale.cuda(), fn, dtype=torch.float32).cpu().double()
    step = 1e-5
    for r in range(2):
        for k in range(0, 160, 7):
            if fn in ("relu", "relu2") and abs(float(v[r, k])) < 2 * step:
                continue  # a kink inside the interval
            up, down = v.clone(), v.clone()
            up[r, k] += step
            down[r, k] -= step
            diff = ((d.double() * (normal(f(up, fn)) - normal(f(down, fn)))).sum() / (2 * step)).item()
            # third derivatives of order ten: step^2; cancellation: 1e-16 * |sum| / step
            assert abs(got[r, k].item() - diff) <= 1e-5 * (1 + abs(diff))


@pytest.mark.parametrize("per_tensor", [False, True])
def test_rows_behind_the_last_are_left_alone(bl, per_tensor):
    """`rows` on the device: what lies behind is neither read (NaN there poisons nothing) nor written."""
    import ctypes
    M, K = 37, 1056
    lib = bl.load_library()
    for used in (0, 1, 20, 36, 37, 50):
        n = min(used, M)
        u = make_u(M, K, used).cuda()
        u[n:] = float("nan")
        rows = torch.tensor([used], dtype=torch.int32, device="cuda")
        codes = torch.full((M, K), 9, dtype=torch.int8, device="cuda")
        check = torch.full((M, K), 9, dtype=torch.int8, device="cuda")
        gamma = torch.full((1 if per_tensor else M,), 9.0, device="cuda")
        rowsum = torch.full((M,), 9, dtype=torch.int32, device="cuda")
        scale = torch.full((M, 9), 9.0, device="cuda")
        ws = torch.empty(max(256, bl.workspace_bytes_experts(bl.OP_QUANT_NONLINEAR, M, 1, 0, 0, 0, per_tensor)),
                         dtype=torch.uint8, device="cuda")
        p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
        assert lib.bitlinear_quant_nonlinear(p(u), M, K, 2, EPS, p(rows), int(per_tensor), p(codes), p(gamma), p(rowsum),
                                             p(check), p(scale), p(ws), ws.numel(),
                                             ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        if n:
            ref = bl.bitlinear_quant_nonlinear(u[:n].contiguous(), "gelu", per_tensor=per_tensor, checkpoint=True)
            for a, b in zip((codes, rowsum, check, scale), (ref[0], ref[2], ref[3], ref[4])):
                assert torch.equal(a[:n], b)
            assert torch.equal(gamma[: ref[1].numel()], ref[1])
        elif per_tensor:
            assert float(gamma) == torch.tensor(1e-5).item()  # its lower bound
        for t in (codes, rowsum, check, scale):
            assert bool((t[n:] == 9).all())
        if not per_tensor:
            assert bool((gamma[n:] == 9).all())
        d = torch.randn(M, K, device="cuda")
        d[n:] = float("nan")
        out = torch.full((M, K), 9.0, dtype=torch.bfloat16, device="cuda")
        bl.bitlinear_nonlinear_backward(d, check, scale, "gelu", rows=rows, out=out)
        assert bool((out[n:] == 9).all()) and bool(torch.isfinite(out[:n].float()).all())


# every pair of waves a row and float4 a lane: batches of rows that fill the chip, whole and ragged, and the numbers of waves
# that the library would not pick there
@pytest.mark.parametrize("M,K,waves", [(300, 4096, 0), (300, 3104, 0), (300, 8192, 0), (300, 5472, 0), (5, 512, 4), (5, 544, 8),
                                       (5, 2048, 1), (5, 2080, 8), (5, 4096, 4), (5, 8192, 4), (5, 12320, 8), (300, 2048, 8)])
@pytest.mark.parametrize("fn", FUNCTIONS)
def test_every_shape_of_a_row(bl, tuning, M, K, waves, fn):
    tuning(f"quant_wpr={waves}")
    for per_tensor in (False, True):
        test_forward_and_checkpoint(bl, M, K, fn, per_tensor)
    for dtype in (torch.float32, torch.bfloat16):
        test_backward(bl, M, K, fn, dtype)


# 127 / m would pass the largest float: the step of a block is 2^-127 or more
LEAST = 127 * 2.0 ** -127


def floored_check(u):
    """The checkpoint of rows whose blocks may be tiny: m is LEAST at the least, but in a block of zeros."""
    M, K = u.shape
    blocks = torch.nn.functional.pad(u, (0, -K % 128)).view(M, -1, 128)
    big = blocks.abs().amax(2, keepdim=True)
    big = torch.where(big > 0, big.clamp_min(LEAST), big)
    up = torch.where(big > 0, torch.full_like(big, 127.0) / big, 0.0)
    return (blocks * up).round().view(M, -1)[:, :K].to(torch.int8), (big / torch.full_like(big, 127.0)).squeeze(2)


@pytest.mark.parametrize("fn", FUNCTIONS)
def test_checkpoint_of_tiny_blocks(bl, fn):
    """Blocks whose largest magnitude is near the smallest floats, zeros among them, alone and beside ordinary blocks:
    zeros stay zeros, the rest is rounded to the block's step, and the gradient goes through what is positive."""
    g = torch.Generator().manual_seed(6)
    u = torch.randn(8, 288, generator=g)
    u[:, ::3] = 0.0
    for r, m in enumerate((1e-38, 3e-37, 3.8e-37, 7.4e-37, 7.5e-37, 2.0 ** -126, 1e-41, 5e-45)):
        u[r, :128] *= m / u[r, :128].abs().max()
    u[5, 128:] *= 1e-38
    check, scale = floored_check(u)
    _, _, _, got, got_scale = bl.bitlinear_quant_nonlinear(u.cuda(), fn, checkpoint=True)
    assert bool((got.cpu()[u == 0] == 0).all())
    assert torch.equal(got.cpu(), check) and torch.equal(got_scale.cpu(), scale)
    du = bl.bitlinear_nonlinear_backward(torch.randn(8, 288, generator=g).cuda(), got, got_scale, fn, dtype=torch.float32)
    assert bool(torch.isfinite(du).all())
    if fn == "relu":
        assert torch.equal(du.cpu() != 0, check > 0)


# ---- a rectifier whose checkpoint keeps what is positive -------------------------------------------------------
def marked_check(u):
    """plain_check's, but -128 for what is positive and rounds to 0."""
    check, scale = floored_check(u)
    return torch.where((u > 0) & (check == 0), torch.full_like(check, -128), check), scale


def make_sparse_u(M, K, seed, kind):
    u = make_u(M, K, seed, "outliers" if kind == "outliers" else "normal")
    return u - 2.0 * u.square().mean(1, keepdim=True).sqrt() if kind == "sparse" else u


@pytest.mark.parametrize("M,K", [(1, 32), (5, 96), (33, 544), (9, 2080), (300, 2048), (300, 5472), (130, 8192), (2, 28672)])
@pytest.mark.parametrize("kind", ["normal", "sparse", "outliers"])
@pytest.mark.parametrize("per_tensor", [False, True])
def test_marked_rectifier(bl, M, K, kind, per_tensor):
    """The forward is the rectifier's, bit for bit; the checkpoint and its gradient keep which elements are positive.

    The gradient against the derivative at the checkpoint with the slopes of u: eight fp32 roundings of what its terms'
    magnitudes add up to.  And against the derivative at u itself: a checkpoint moves an element of h by half a step s of its
    block at most, so the row's mean by mean(s / 2) and its deviation (a norm) by rms(s / 2); the differences of dU
    follow without any approximation."""
    print(f"marked rectifier M={M} K={K} {kind} per_tensor={per_tensor}", flush=True)
    u = make_sparse_u(M, K, M + K, kind)
    got = bl.bitlinear_quant_nonlinear(u.cuda(), "relu_marked", per_tensor=per_tensor, checkpoint=True)
    ref = bl.bitlinear_quant_nonlinear(u.cuda(), "relu", per_tensor=per_tensor)
    for a, b in zip(got[:3], ref[:3]):
        assert torch.equal(a, b)
    bare = bl.bitlinear_quant_nonlinear(u.cuda(), "relu_marked", per_tensor=per_tensor)
    assert bare[3] is None and torch.equal(bare[0], ref[0])
    check, scale = marked_check(u)
    assert torch.equal(got[3].cpu(), check) and torch.equal(got[4].cpu(), scale)
    d = torch.randn(M, K, generator=torch.Generator().manual_seed(3))
    du = bl.bitlinear_nonlinear_backward(d.cuda(), got[3], got[4], "relu_marked", dtype=torch.float32).cpu().double()
    off, d, h = scale.repeat_interleave(128, 1)[:, :K].double() * (0.5 + 64 * F32), d.double(), u.double().clamp_min(0)
    dev = (h.var(1, correction=0, keepdim=True) + EPS).sqrt()
    x, m1 = normal(h), d.mean(1, keepdim=True)
    m2 = (d * x).mean(1, keepdim=True)
    core = d - m1 - x * m2
    dev_off = off.square().mean(1, keepdim=True).sqrt()
    least = (dev - dev_off).clamp_min(EPS ** 0.5)
    x_off = (off + off.mean(1, keepdim=True) + x.abs() * dev_off) / least
    m2_off = (d.abs() * x_off).mean(1, keepdim=True)
    allowed = dev_off / (dev * least) * core.abs() + (x_off * (m2.abs() + m2_off) + x.abs() * m2_off) / least
    allowed = allowed + 8 * F32 / least * (d.abs() + m1.abs() + (x.abs() + x_off) * (m2.abs() + m2_off))
    slope = (u > 0).double()
    assert bool(((du - slope * core / dev).abs() <= slope * allowed).all())
    v = (check.float() * scale.repeat_interleave(128, 1)[:, :K]).double().clamp_min(0)
    x, dev = normal(v), (v.var(1, correction=0, keepdim=True) + EPS).sqrt()
    m2 = (d * x).mean(1, keepdim=True)
    most = d.abs() + m1.abs() + (x * m2).abs()
    assert bool(((du - slope * (d - m1 - x * m2) / dev).abs() <= slope * 8 * F32 * most / dev).all())
    half = bl.bitlinear_nonlinear_backward(d.float().cuda(), got[3], got[4], "relu_marked")
    assert torch.equal(half.cpu(), du.float().to(torch.bfloat16))


def test_marked_rectifier_of_tiny_and_no_values(bl):
    """What is positive keeps its slope however small, zeros and what is below have none."""
    u = torch.zeros(4, 160)
    u[0, ::2] = 1e-41
    u[1, ::2], u[1, 1::4] = 1e-30, -1e-30
    u[2, 3], u[2, 4] = 1.0, 1e-38
    u[2, 130:] = -1e-9
    check, scale = marked_check(u)
    _, _, _, got, got_scale = bl.bitlinear_quant_nonlinear(u.cuda(), "relu_marked", checkpoint=True)
    assert torch.equal(got.cpu(), check) and torch.equal(got_scale.cpu(), scale)
    d = torch.randn(4, 160, generator=torch.Generator().manual_seed(1)).cuda()
    du = bl.bitlinear_nonlinear_backward(d, got, got_scale, "relu_marked", dtype=torch.float32)
    assert torch.equal(du.cpu() != 0, u > 0)


def test_no_rows_leave_the_lower_bound_of_gamma(bl):
    """No rows at all, as with a `rows` of 0: a gamma per tensor is its lower bound, whatever memory it got."""
    for fn in FUNCTIONS:
        dirt = [torch.full((1,), 7.0, device="cuda") for _ in range(64)]
        del dirt  # one of these blocks is the next call's
        _, gamma, _, _, _ = bl.bitlinear_quant_nonlinear(torch.empty(0, 64, device="cuda"), fn, per_tensor=True)
        assert gamma.tolist() == [torch.tensor(1e-5).item()]
