"""The residual's addition, root-mean-square norm and 8-bit quantiser in one pass, and its backward pass, on the GPU,
against 64-bit evaluations on the CPU.

Tolerances (F32 = 2^-24 and BF16 = 2^-8, half a step).  h is one fp32 sum, rounded to its type: equal.  The mean square is a
sum in fp64, so x^ is off by its rounding to fp32 and by the product with the gain: 2 F32 |x^|.  gamma is the largest of
them.  A code may differ from the rounded 64-bit value only where that lies this close to a half, four roundings more:
128 / gamma, the product, and twice what gamma is off by.
Backward: t = g * gain (one rounding), n = h / rms (one), mean(t n) (its sum in fp64: what t and n are off by), their
product and difference (two), 1/rms and the product with it (two), the residual's gradient (one) and the type of the result:
with P = (|t| + |n mean(t n)|) / rms and Q = |n| mean|t n| / rms it is 6 F32 P + 3 F32 Q + F32 |dresidual| + 2 F32 |dh|.  The
gain's gradient: three roundings of every product, and its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5
F, B = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def bl():
    import paper_2310_11453_amd as lib
    lib.load_library()
    assert torch.cuda.is_available()
    return lib


def half_step(dtype):
    return F32 if dtype is F else BF16


def make(M, K, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g) * torch.exp(0.5 * torch.randn(M, 1, generator=g)) * size
    return torch.where(torch.rand(M, K, generator=g) < 0.01, 20 * x, x).to(dtype)


def forward64(x, r, gain, eps=EPS):
    h = x if r is None else (x.float() + r.float()).to(r.dtype)
    hd = h.double()
    rms = (hd.square().mean(1, keepdim=True) + eps).sqrt()
    n = torch.where(rms > 0, hd / rms, 0.0)
    return h, rms, n * (1.0 if gain is None else gain.double())


def check_forward(x, r, gain, per_tensor, got, eps=EPS):
    codes, gamma, rowsum, h, xhat = (None if t is None else t.cpu() for t in got)
    h_ref, _, x_ref = forward64(x, r, gain, eps)
    assert h.dtype == h_ref.dtype and torch.equal(h, h_ref)
    off = 2 * F32 * x_ref.abs() + 1e-44
    if xhat is not None:
        assert bool(((xhat.double() - x_ref).abs() <= off).all())
    a = x_ref.abs()
    g = (a.amax().reshape(1, 1) if per_tensor else a.amax(1, keepdim=True)).clamp_min(1e-5)
    assert gamma.shape == ((1,) if per_tensor else (x.shape[0],))
    assert bool(((gamma.double().view(-1, 1) - g).abs() <= 2 * F32 * g).all())
    t = x_ref * 128 / g
    t_off = 8 * F32 * t.abs() + 1e-30
    assert bool(((codes.double() - t.clamp(-128, 127)).abs() <= 0.5 + t_off).all())
    assert torch.equal(rowsum, codes.sum(1, dtype=torch.int32))


# one to sixteen waves a row, ragged pieces, rows past registers, more rows than fit at once
SHAPES = [(1, 32), (1, 2048), (5, 96), (3, 256), (33, 544), (64, 1024), (9, 2080), (2500, 2048), (40, 4096), (7, 5472),
          (130, 8192), (3, 12320), (2, 28672), (1, 32768), (3, 40000), (1100, 704), (1030, 1376), (300, 5472), (40, 10240),
          (300, 20480)]
TYPES = [(F, None), (B, None), (F, F), (F, B), (B, F), (B, B)]


def cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("x_type,h_type", TYPES)
@pytest.mark.parametrize("per_tensor", [False, True])
def test_forward(bl, M, K, x_type, h_type, per_tensor):
    print(f"quant_rmsnorm M={M} K={K} {x_type} {h_type} per_tensor={per_tensor}", flush=True)
    x = make(M, K, x_type, M + K)
    r = None if h_type is None else make(M, K, h_type, M + K + 1, 3.0)
    gain = None if (M + K) % 3 == 0 else 1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))
    got = bl.bitlinear_quant_rmsnorm(x.cuda(), cuda(r), gain=cuda(gain), per_tensor=per_tensor, want_xhat=True)
    check_forward(x, r, gain, per_tensor, got)
    bare = bl.bitlinear_quant_rmsnorm(x.cuda(), cuda(r), gain=cuda(gain), per_tensor=per_tensor)
    assert bare[4] is None and all(torch.equal(p, q) for p, q in zip(bare[:4], got[:4]))


@pytest.mark.parametrize("M,K", [(600, 8224), (513, 16384), (2100, 8224)])
@pytest.mark.parametrize("x_type,h_type", TYPES)
@pytest.mark.parametrize("per_tensor", [False, True])
def test_forward_of_many_wide_rows(bl, M, K, x_type, h_type, per_tensor):
    """Rows that need more than four waves, and more of them than a call per tensor has workgroups; multiples of one row, so
    that making them is quick."""
    gen = torch.Generator().manual_seed(M)
    size = torch.exp(torch.randn(M, 1, generator=gen))
    x, r = (None if t is None else (make(1, K, F, K + i) * size).to(t) for i, t in enumerate((x_type, h_type)))
    gain = 1 + 0.3 * torch.randn(K, generator=gen) if M % 2 else None
    check_forward(x, r, gain, per_tensor, bl.bitlinear_quant_rmsnorm(x.cuda(), cuda(r), gain=cuda(gain), per_tensor=per_tensor))


@pytest.mark.parametrize("K", [96, 4096, 9056, 20480, 40000])
def test_a_row_of_no_numbers_stays_in_it(bl, K):
    """Infinities and NaN in a row leave every other row's results (per token) as they are."""
    x, r, g = make(9, K, B, 1), make(9, K, B, 2), make(9, K, B, 3)
    bad, bad_g = x.clone(), g.clone()
    bad[2, 5], bad[6, K - 1], bad_g[4, 7] = float("inf"), float("nan"), float("nan")
    for rows, p, q in (([0, 1, 3, 4, 5, 7, 8], bad, g), ([0, 1, 2, 3, 5, 6, 7, 8], x, bad_g)):
        ref, got = (bl.bitlinear_quant_rmsnorm(t.cuda(), r.cuda()) for t in (x, p))
        assert all(torch.equal(s[rows], t[rows]) for s, t in zip(ref[:4], got[:4]))
        ref, got = (bl.bitlinear_rmsnorm_backward(t.cuda(), h) for t, h in ((g, ref[3]), (q, got[3])))
        assert torch.equal(ref[rows], got[rows])


@pytest.mark.parametrize("K", [64, 4096, 9056, 40000])
@pytest.mark.parametrize("per_tensor", [False, True])
def test_forward_in_place(bl, K, per_tensor):
    """h written over the residual, or over x."""
    for dtype in (F, B):
        M = 600 if K == 9056 else 37
        x, r = make(M, K, dtype, 1), make(M, K, dtype, 2)
        ref = bl.bitlinear_quant_rmsnorm(x.cuda(), r.cuda(), per_tensor=per_tensor)
        for over in (0, 1):
            pair = [x.cuda(), r.cuda()]
            got = bl.bitlinear_quant_rmsnorm(*pair, per_tensor=per_tensor, out=pair[over])
            assert got[3] is pair[over] and all(torch.equal(p, q) for p, q in zip(got[:4], ref[:4]))
            assert torch.equal(pair[1 - over].cpu(), (r, x)[over])  # the other one is as it was


@pytest.mark.parametrize("per_tensor", [False, True])
def test_forward_of_zeros_and_extremes(bl, per_tensor):
    x = make(6, 256, F, 3)
    x[1] = 0.0
    x[2] = 1e-30
    x[3] *= 1e30  # squares past the largest float
    x[4, 7:] = 0.0
    x[5] = -2.5
    for eps in (EPS, 0.0):
        got = bl.bitlinear_quant_rmsnorm(x.cuda(), eps=eps, per_tensor=per_tensor, want_xhat=True)
        check_forward(x, None, None, per_tensor, got, eps)
    assert bool((got[0][1].cpu() == 0).all())


def test_forward_without_a_place_for_h(bl):
    """Through the C ABI: H may be NULL, also per tensor, where the sum is then made twice."""
    lib = bl.load_library()
    x, r = make(20, 544, B, 1).cuda(), make(20, 544, F, 2).cuda()
    for per_tensor in (False, True):
        ref = bl.bitlinear_quant_rmsnorm(x, r, per_tensor=per_tensor)
        codes, gamma = torch.empty_like(ref[0]), torch.empty_like(ref[1])
        ws = torch.empty(bl.workspace_bytes(bl.OP_QUANT_RMSNORM, 20, 1, 544, True), dtype=torch.uint8, device="cuda")
        assert lib.bitlinear_quant_rmsnorm(x.data_ptr(), 1, r.data_ptr(), 0, 20, 544, None, EPS, int(per_tensor), None,
                                           codes.data_ptr(), gamma.data_ptr(), None, None, ws.data_ptr(), ws.numel(),
                                           torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(codes, ref[0]) and torch.equal(gamma, ref[1])


def test_forward_feeds_the_one_bit_product(bl):
    """The codes, gamma and row sums are what bitlinear_matmul reads."""
    g = torch.Generator().manual_seed(5)
    x, r = make(24, 1056, B, 6).cuda(), make(24, 1056, F, 7).cuda()
    W = 0.02 * torch.randn(300, 1056, generator=g)
    packed, alpha, beta = bl.bitlinear_pack_weights(W.cuda())
    codes, gamma, rowsum, _, _ = bl.bitlinear_quant_rmsnorm(x, r)
    y = bl.bitlinear_matmul(codes, gamma, rowsum, packed, 300, beta).cpu()
    sign = torch.where(W > alpha.cpu(), 1.0, -1.0).double()
    acc = codes.cpu().double() @ sign.T
    ref = acc * (beta.cpu().double() * gamma.cpu().double().view(-1, 1) / 128)
    assert bool(((y.double() - ref).abs() <= 4 * F32 * ref.abs()).all())


def backward64(g, h, gain, dr, eps=EPS):
    g, hd = g.double(), h.double()
    rms = (hd.square().mean(1, keepdim=True) + eps).sqrt()
    n = torch.where(rms > 0, hd / rms, 0.0)
    t = g if gain is None else g * gain.double()
    along = (t * n).mean(1, keepdim=True)
    inv = torch.where(rms > 0, 1 / rms, 0.0)
    d = (t - n * along) * inv
    P = (t.abs() + (n * along).abs()) * inv
    Q = n.abs() * (t * n).abs().mean(1, keepdim=True) * inv
    if dr is not None:
        d = d + dr.double()
    return d, P, Q, (g * n).sum(0), (g * n).abs().sum(0)


def check_backward(g, h, gain, dr, dtype, d_h, d_gain, eps=EPS):
    d, P, Q, dg, dg_abs = backward64(g, h, gain, dr, eps)
    tol = 6 * F32 * P + 3 * F32 * Q + 2 * F32 * d.abs() + (0 if dr is None else F32 * dr.double().abs()) + 1e-44
    if dtype is B:
        tol = tol + BF16 * (d.abs() + tol)
    assert d_h.dtype == dtype and bool(((d_h.cpu().double() - d).abs() <= tol).all())
    if d_gain is not None:
        assert bool(((d_gain.cpu().double() - dg).abs() <= 3 * F32 * dg_abs + F32 * dg.abs() + 1e-44).all())


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("g_type", [F, B])
@pytest.mark.parametrize("h_type", [F, B])
@pytest.mark.parametrize("d_type", [F, B])
def test_backward(bl, M, K, g_type, h_type, d_type):
    print(f"rmsnorm_backward M={M} K={K} {g_type} {h_type} {d_type}", flush=True)
    g, h = make(M, K, g_type, 2 * M + K, 1e-3), make(M, K, h_type, M + 2 * K)
    dr = make(M, K, d_type, M + K, 1e-3) if (M + K) % 4 else None
    gain = None if (M + K) % 3 == 0 else 1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))
    d_h, d_gain = bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), gain=cuda(gain), dresidual=cuda(dr), want_dgain=True,
                                                dtype=d_type)
    check_backward(g, h, gain, dr, d_type, d_h, d_gain)
    # without the gain's gradient, twice: the same bits
    again = [bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), gain=cuda(gain), dresidual=cuda(dr), dtype=d_type)
             for _ in range(2)]
    assert torch.equal(again[0], d_h) and torch.equal(again[1], d_h)


def test_backward_gain_over_many_rows(bl):
    """More rows than workgroups, and rows of zeros among them."""
    for M, K in [(257, 96), (3001, 160), (1024, 2048), (5000, 32), (600, 9056), (513, 16384)]:
        g, h = make(M, K, F, M), make(M, K, F, K)
        h[::7] = 0.0
        d_h, d_gain = bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), want_dgain=True, eps=0.0 if M % 2 else EPS)
        check_backward(g, h, None, None, F, d_h, d_gain, 0.0 if M % 2 else EPS)
        first = d_gain
        d_gain = bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), want_dgain=True, eps=0.0 if M % 2 else EPS)[1]
        assert torch.equal(first, d_gain)  # a fixed order


@pytest.mark.parametrize("M,K", [(300, 20480), (1100, 16416), (17000, 16416), (700, 32768)])
def test_backward_of_wide_rows(bl, M, K):
    """K > 16384: a column's products are summed in fp32 over a workgroup's rows: 64 at most, ceil(M / 256) where there are
    fewer, each sum one rounding more of the sum of magnitudes; h a multiple of one row, so that the check needs little memory."""
    gen = torch.Generator().manual_seed(K)
    base, size = make(1, K, F, M), torch.exp(torch.randn(M, 1, generator=gen)).cuda()
    g0 = make(1, K, F, K, 1e-3)
    h, g = base.cuda() * size, g0.cuda() * torch.randn(M, 1, generator=gen).cuda()
    d_h, d_gain = bl.bitlinear_rmsnorm_backward(g, h, want_dgain=True)
    some = [0, 1, M // 2, M - 1]
    check_backward(g[some].cpu(), h[some].cpu(), None, None, F, d_h[some], None)
    dg, mag = torch.zeros(K, dtype=torch.float64, device="cuda"), torch.zeros(K, dtype=torch.float64, device="cuda")
    for i in range(0, M, 500):
        hd, gd = h[i:i + 500].double(), g[i:i + 500].double()
        p = gd * hd / (hd.square().mean(1, keepdim=True) + EPS).sqrt()
        dg += p.sum(0)
        mag += p.abs().sum(0)
    rows = min(64, -(-M // 256))
    assert bool(((d_gain.double() - dg).abs() <= (3 + rows) * F32 * mag + F32 * dg.abs() + 1e-44).all())
    assert torch.equal(bl.bitlinear_rmsnorm_backward(g, h, want_dgain=True)[1], d_gain)


@pytest.mark.parametrize("K", [64, 4096, 20480, 40000])
def test_backward_in_place(bl, K):
    """dH over the gradient of the residual, of x^, or over h."""
    for dtype in (F, B):
        t = [make(37, K, dtype, i) for i in range(3)]
        ref = bl.bitlinear_rmsnorm_backward(t[0].cuda(), t[1].cuda(), dresidual=t[2].cuda(), want_dgain=True)
        for over in range(3):
            d = [v.cuda() for v in t]
            got = bl.bitlinear_rmsnorm_backward(d[0], d[1], dresidual=d[2], want_dgain=True, out=d[over])
            assert got[0] is d[over] and torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_backward_against_differences(bl):
    """Against central differences of the 64-bit forward: a sum of x^ with weights w has the gradient that dXhat = w gives."""
    x, gain = make(3, 64, F, 9).double(), 1 + 0.3 * torch.randn(64, generator=torch.Generator().manual_seed(1)).double()
    w = make(3, 64, F, 10)

    def loss(v, gn):
        rms = (v.square().mean(1, keepdim=True) + EPS).sqrt()
        return (w.double() * (v / rms * gn)).sum()

    d_h, d_gain = bl.bitlinear_rmsnorm_backward(w.cuda(), x.float().cuda(), gain=gain.float().cuda(), want_dgain=True)
    x, gain = x.float().double(), gain.float().double()
    step = 1e-5
    for i in range(3):
        for k in range(64):
            e = torch.zeros_like(x)
            e[i, k] = step
            diff = (loss(x + e, gain) - loss(x - e, gain)) / (2 * step)
            # third derivatives are of the size of w / rms^3: step^2 of them, and 64-bit noise over the step
            assert abs(float(d_h[i, k]) - float(diff)) <= 1e-6 * float(w.abs().max()) * 20
    for k in range(64):
        e = torch.zeros_like(gain)
        e[k] = step
        diff = (loss(x, gain + e) - loss(x, gain - e)) / (2 * step)
        assert abs(float(d_gain[k]) - float(diff)) <= 1e-6 * float(w.abs().max()) * 20


def test_nothing_to_do(bl):
    e = torch.empty(0, 64, device="cuda")
    codes, gamma, rowsum, h, _ = bl.bitlinear_quant_rmsnorm(e, e)
    assert codes.shape == (0, 64) and gamma.shape == (0,) and rowsum.shape == (0,) and h.shape == (0, 64)
    assert float(bl.bitlinear_quant_rmsnorm(e, per_tensor=True)[1]) == pytest.approx(1e-5)
    d, dg = bl.bitlinear_rmsnorm_backward(e, e, want_dgain=True)
    assert d.shape == (0, 64) and bool((dg == 0).all())


def test_more_than_2_to_32_elements(bl):
    M, K = (1 << 17) + 9, 32768
    x = torch.empty(M, K, dtype=B, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    row = torch.randn(K, device="cuda", generator=g).to(B)
    x[:] = row
    last = make(9, K, B, 5)
    x[-9:] = last.cuda()
    got = bl.bitlinear_quant_rmsnorm(x)
    check_forward(last, None, None, False, [got[0][-9:], got[1][-9:], got[2][-9:], last.cuda(), None])
    assert torch.equal(got[0][5], got[0][M - 10]) and bool((got[1][: M - 9] == got[1][0]).all())
    del got
    d = bl.bitlinear_rmsnorm_backward(x, x)
    check_backward(last, last, None, None, B, d[-9:], None)
    assert torch.equal(d[0], d[M - 10])


def test_binding_refuses(bl):
    x, r = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, device="cuda", dtype=B)
    for call in (lambda: bl.bitlinear_quant_rmsnorm(x.half()), lambda: bl.bitlinear_quant_rmsnorm(x, r[:3]),
                 lambda: bl.bitlinear_quant_rmsnorm(x.T.contiguous().T), lambda: bl.bitlinear_quant_rmsnorm(x, r, out=x),
                 lambda: bl.bitlinear_quant_rmsnorm(x, out=x), lambda: bl.bitlinear_quant_rmsnorm(x, gain=x[0, :32]),
                 lambda: bl.bitlinear_quant_rmsnorm(x, gain=r[0]), lambda: bl.bitlinear_quant_rmsnorm(x, r.cpu()),
                 lambda: bl.bitlinear_quant_rmsnorm(x[:, :48].contiguous()), lambda: bl.bitlinear_quant_rmsnorm(x, eps=-1.0),
                 lambda: bl.bitlinear_rmsnorm_backward(x, r[:3]), lambda: bl.bitlinear_rmsnorm_backward(x, r, dtype=torch.half),
                 lambda: bl.bitlinear_rmsnorm_backward(x, r, dresidual=r, dtype=F),
                 lambda: bl.bitlinear_rmsnorm_backward(x, r, out=r), lambda: bl.bitlinear_rmsnorm_backward(x, r, gain=x)):
        with pytest.raises(bl.BitLinearError):
            call()


# the kernels that no shape above takes: 2 and 4 float4 a lane of one wave, 4 and 8 of four, also with more rows than a call has
# workgroups, as at a training step; many rows are multiples of a few, so that making them is quick
@pytest.mark.parametrize("M,K", [(20, 480), (40, 960), (300, 4096), (300, 8192), (2100, 4096), (2100, 8192)])
@pytest.mark.parametrize("x_type,h_type", TYPES)
def test_rows_of_the_other_kernels(bl, M, K, x_type, h_type):
    gen = torch.Generator().manual_seed(M + K)
    size = torch.exp(torch.randn(M, 1, generator=gen))
    some = lambda t, seed, s=1.0: (make(20, K, F, seed, s).repeat(M // 20, 1) * size).to(t)  # noqa: E731
    x, r = some(x_type, 1), None if h_type is None else some(h_type, 2)
    gain = 1 + 0.3 * torch.randn(K, generator=gen) if h_type is not B else None
    for per_tensor in (False, True):
        print(f"quant_rmsnorm M={M} K={K} {x_type} {h_type} per_tensor={per_tensor}", flush=True)
        check_forward(x, r, gain, per_tensor, bl.bitlinear_quant_rmsnorm(x.cuda(), cuda(r), gain=cuda(gain), per_tensor=per_tensor))
    if r is not None:
        g = some(x_type, 3, 1e-3)
        got = bl.bitlinear_rmsnorm_backward(g.cuda(), r.cuda(), gain=cuda(gain), want_dgain=True, dtype=F)
        check_backward(g, r, gain, None, F, *got)


# every width of a row: one wave, four, eight, sixteen, rows past registers
BAD_SHAPES = [(9, 96), (1100, 2048), (300, 4096), (9, 4096), (600, 9056), (9, 20480), (9, 40000)]


@pytest.mark.parametrize("M,K", BAD_SHAPES)
@pytest.mark.parametrize("h_type", [None, F, B])
@pytest.mark.parametrize("with_gain", [False, True])
def test_a_row_of_no_numbers_is_seen(bl, M, K, h_type, with_gain):
    """A row with an infinity or a NaN has a gamma of NaN, so that products of its codes are NaN and nothing passes for a
    token; per tensor the one gamma is.  The other rows (per token) and h are as they were."""
    x = make(M, K, F, 1).cuda()
    r = None if h_type is None else make(M, K, h_type, 2).cuda()
    gain = (1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(3))).cuda() if with_gain else None
    ref = bl.bitlinear_quant_rmsnorm(x, r, gain=gain)
    bad = x.clone()
    bad[1, 5], bad[3, K - 1], bad[7, K // 2] = float("inf"), float("nan"), float("-inf")
    if M > 9:
        bad[M - 1] = float("nan")
    spoilt = ~bad.isfinite().all(1)
    got = bl.bitlinear_quant_rmsnorm(bad, r, gain=gain)
    assert bool(got[1][spoilt].isnan().all()) and bool(got[1][~spoilt].isfinite().all())
    assert all(torch.equal(p[~spoilt], q[~spoilt]) for p, q in zip(got[:4], ref[:4]))
    packed, scale = bl.bitlinear_pack_weights_i8(torch.ones(16, K, device="cuda"))
    y = bl.bitlinear_matmul_i8(got[0], got[1], packed, 16, scale)
    assert bool(y[spoilt].isnan().all()) and bool(y[~spoilt].isfinite().all())
    one = bl.bitlinear_quant_rmsnorm(bad, r, gain=gain, per_tensor=True)
    assert bool(one[1].isnan().all())
    for h in (got[3], one[3]):
        want = bad if r is None else (bad + r.float()).to(h_type)
        assert torch.equal(h.nan_to_num(1.5, 2.5, 3.5), want.nan_to_num(1.5, 2.5, 3.5))


@pytest.mark.parametrize("K", [96, 4096, 20480, 40000])
@pytest.mark.parametrize("per_tensor", [False, True])
def test_a_gain_of_no_numbers_is_seen(bl, K, per_tensor):
    """It is in every row."""
    x = make(9, K, B, 1).cuda()
    for bad in (float("nan"), float("inf")):
        gain = torch.ones(K, device="cuda")
        gain[K - 3] = bad
        assert not bool(bl.bitlinear_quant_rmsnorm(x, gain=gain, per_tensor=per_tensor)[1].isfinite().any())


@pytest.mark.parametrize("per_tensor", [False, True])
def test_a_sum_past_the_largest_number_is_seen(bl, per_tensor):
    """x and the residual are numbers, their sum in the residual's type is not."""
    x, r = make(4, 256, F, 1), make(4, 256, B, 2)
    x[2, 9], r[2, 9] = 3.3e38, torch.tensor(3.3e38).to(B)
    codes, gamma, _, h, _ = bl.bitlinear_quant_rmsnorm(x.cuda(), r.cuda(), per_tensor=per_tensor)
    assert bool(h[2, 9].isinf()) and bool(gamma[0 if per_tensor else 2].isnan())
    assert per_tensor or bool(gamma[[0, 1, 3]].isfinite().all())


@pytest.mark.parametrize("K", [96, 4096, 9056, 20480, 40000])
def test_backward_of_a_row_of_no_numbers(bl, K):
    """dh is NaN in all of such a row and in no other; the gain's gradient, a sum over rows, is."""
    g, h = make(20, K, F, 1).cuda(), make(20, K, F, 2).cuda()
    ref = bl.bitlinear_rmsnorm_backward(g, h)
    for value in (float("nan"), float("inf")):
        bad = h.clone()
        bad[6, 11] = value
        d_h, d_gain = bl.bitlinear_rmsnorm_backward(g, bad, want_dgain=True)
        rows = [i for i in range(20) if i != 6]
        assert torch.equal(d_h[rows], ref[rows]) and bool(d_h[6].isnan().all()) and bool(d_gain.isnan().all())


SIZES_K = [96, 480, 2048, 8192, 12320, 20480, 28672, 40000]


@pytest.mark.parametrize("K", SIZES_K)
@pytest.mark.parametrize("g_type,h_type", [(F, F), (B, B)])
def test_backward_gain_of_large_and_small_rows(bl, K, g_type, h_type):
    """Products g h that are no numbers, or have lost their digits, where g h / rms is an ordinary number."""
    for size, grad in ((1e30, 1e10), (1e-30, 1e-12)):
        g, h = make(37, K, g_type, K, grad), make(37, K, h_type, K + 1)
        h = (h.float() / h.float().abs().amax(1, keepdim=True) * size).to(h_type)
        gain = 1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))
        d_h, d_gain = bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), gain=gain.cuda(), eps=0.0, want_dgain=True, dtype=F)
        check_backward(g, h, gain, None, F, d_h, d_gain, 0.0)


@pytest.mark.parametrize("K", SIZES_K)
@pytest.mark.parametrize("g_type,h_type", [(F, F), (B, B)])
def test_backward_of_rows_at_the_ends_of_the_range(bl, K, g_type, h_type):
    """Rows so small that 1 / rms is past the largest float (eps = 0), or so large that it has lost digits, with gradients that
    are ordinary numbers."""
    for size, grad in ((1e-39, 1e-6), (1e35, 1e-3), (3e38, 1e4)):
        g, h = make(37, K, g_type, K, grad), make(37, K, F, K + 1)
        h = (h.sign() * size * (0.5 + 0.5 * h.abs() / h.abs().amax(1, keepdim=True))).to(h_type)
        gain = 1 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(K))
        d_h, d_gain = bl.bitlinear_rmsnorm_backward(g.cuda(), h.cuda(), gain=gain.cuda(), eps=0.0, want_dgain=True, dtype=F)
        check_backward(g, h, gain, None, F, d_h, d_gain, 0.0)
