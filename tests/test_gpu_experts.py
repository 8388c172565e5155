"""Mixtures of BitLinear layers on the GPU, through the binding: routing, the experts' products and their straight-through
backward, combination and its gradient, against plain evaluations on the CPU in integers and in 64 bits.

Tolerances.  A rounding to fp32 is off by at most 2^-24 of the value, one to bf16 by 2^-8.  A sum of n products in fp32 is
off by at most n roundings of what its terms' magnitudes add up to, in whatever order it is added; that is what the tests
of sums allow.  Integers, products of one rounding and copies are compared bit for bit."""
import numpy as np
import pytest
import torch

import workloads as wl

pytestmark = pytest.mark.gpu
F32, BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def bl():
    import paper_2310_11453_amd as lib
    lib.load_library()
    assert torch.cuda.is_available()
    return lib


def choices(M, top_k, E, seed, unrouted=0.0, skew=0.7, only=None):
    """Expert ids [M, top_k]; `only`: nobody chooses any other expert."""
    rng = np.random.default_rng(seed)
    if only is not None:
        ids = rng.choice(np.asarray(only), (M, top_k)).astype(np.int32)
    else:
        score = rng.standard_normal((M, E)) + skew * rng.standard_normal((1, E))
        ids = np.argsort(-score, axis=1)[:, :top_k].astype(np.int32)
    if unrouted:
        ids[rng.random((M, top_k)) < unrouted] = rng.choice([-1, E, 2 ** 31 - 1, -2 ** 31])
    return ids


def plain_route(ids, E):
    flat = ids.reshape(-1).astype(np.int64)
    order, position, offsets = [], np.full(flat.size, -1, np.int64), [0]
    for e in range(E):
        mine = np.flatnonzero(flat == e)
        position[mine] = len(order) + np.arange(mine.size)
        order.extend(mine)
        offsets.append(len(order))
    order = np.array(order + [-1] * (flat.size - len(order)), np.int64)
    return order, position.reshape(ids.shape), np.array(offsets)


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make(bl, M, top_k, E, K, N, gather, per_tensor, ids, seed=1):
    """Weights, codes and routing of a case: what the calls take, and what the plain evaluation takes."""
    order, position, offsets = plain_route(ids, E)
    T = M * top_k
    rows = M if gather else T
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(E, N, K, generator=g) * 0.02
    packed, _, beta = bl.bitlinear_pack_weights_experts(W.cuda())
    signs = torch.stack([torch.from_numpy(unpack(bl, packed[e], N, K)) for e in range(E)])
    codes = torch.randint(-128, 128, (rows, K), generator=g, dtype=torch.int8)
    gamma = torch.rand(1 if per_tensor else rows, generator=g) + 0.5
    rowsum = codes.sum(1, dtype=torch.int32)
    row = np.maximum(order, 0) // top_k if gather else np.arange(T)
    calls = dict(order=gpu(order.astype(np.int32)) if gather else None, top_k=top_k if gather else 1,
                 offsets=gpu(offsets.astype(np.int32)), per_tensor=per_tensor)
    return dict(packed=packed, beta=beta, signs=signs, codes=codes, gamma=gamma, rowsum=rowsum, row=torch.from_numpy(row),
                offsets=offsets, T=T, calls=calls, E=E)


def unpack(bl, blob, N, K):
    words = bl.bitlinear_packed_to_canonical(blob, N, K).cpu().numpy().view(np.uint32)
    bits = (words[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1
    return (2 * bits.reshape(N, K).astype(np.int8) - 1).astype(np.int8)


# ---- routing ---------------------------------------------------------------------------------------
# one choice; a row of 64 and its neighbours; a workgroup's 4096 and its neighbours; several workgroups; around 64 of
# them, above which their counts are scanned by a launch of its own; every expert number of bits; experts that nobody chooses
ROUTES = [(1, 1, 1), (1, 2, 8), (63, 1, 3), (64, 1, 4), (65, 1, 5), (16, 4, 64), (333, 3, 7), (4096, 1, 16), (4097, 1, 17),
          (2048, 2, 256), (5000, 8, 255), (8191, 8, 64), (70000, 2, 9), (131072, 2, 5), (131073, 2, 5), (400001, 1, 256)]


@pytest.mark.parametrize("M,top_k,E", ROUTES)
@pytest.mark.parametrize("unrouted", [0.0, 0.3, 1.0])
def test_route_sorts_stably(bl, M, top_k, E, unrouted):
    print(f"route M={M} top_k={top_k} E={E} unrouted={unrouted}", flush=True)
    ids = choices(M, top_k, E, M + E, unrouted) if top_k <= E else None
    order, position, offsets = (t.cpu().numpy() for t in bl.bitlinear_route(gpu(ids), E))
    ref = plain_route(ids, E)
    assert np.array_equal(offsets, ref[2]) and np.array_equal(position, ref[1]) and np.array_equal(order, ref[0])


def test_route_one_expert_takes_all_and_the_same_expert_twice(bl):
    for M, top_k, E, only in [(1000, 2, 8, [5]), (4100, 3, 256, [255]), (100, 2, 4, [0, 3])]:
        ids = choices(M, top_k, E, 3, only=only)
        got = [t.cpu().numpy() for t in bl.bitlinear_route(gpu(ids), E)]
        for a, b in zip(got, plain_route(ids, E)):
            assert np.array_equal(a, b)


def test_route_without_tokens(bl):
    order, position, offsets = bl.bitlinear_route(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 4)
    assert order.numel() == 0 and position.shape == (0, 2) and offsets.tolist() == [0] * 5


# ---- the experts' products -------------------------------------------------------------------------
# one token; fewer slots than experts; ragged K (one short chunk, several chunks and a part), N that ends inside a tile of 16;
# around the row counts where an expert's rows fill a tile; more experts than a wave has lanes
TILES = [0, 1, 2, 3, 4, 5]
PRODUCTS = [(1, 1, 1, 32, 1), (1, 2, 8, 256, 512), (3, 2, 4, 544, 40), (16, 2, 4, 512, 130), (40, 1, 3, 96, 300),
            (33, 4, 100, 160, 48), (130, 2, 4, 1056, 257), (300, 1, 2, 2048, 136), (700, 2, 5, 640, 520),
            (1500, 2, 3, 416, 264)]


# The library picks the tiles from the shape; the experts_tile switch forces each kind.
@pytest.mark.parametrize("M,top_k,E,K,N", PRODUCTS)
@pytest.mark.parametrize("gather,per_tensor", [(True, False), (True, True), (False, False)])
@pytest.mark.parametrize("tile", TILES)
def test_products_exact(bl, tuning, M, top_k, E, K, N, gather, per_tensor, tile):
    print(f"products M={M} top_k={top_k} E={E} K={K} N={N} gather={gather} per_tensor={per_tensor} tile={tile}", flush=True)
    tuning(f"experts_tile={tile}")
    check_products(bl, M, top_k, E, K, N, gather, per_tensor, choices(M, top_k, E, M + K, unrouted=0.1))


@pytest.mark.parametrize("only", [[0], [6], [2, 5]])
@pytest.mark.parametrize("M", [1, 20, 400, 1100])
@pytest.mark.parametrize("tile", TILES)
def test_products_when_few_experts_have_all_slots(bl, tuning, M, only, tile):
    print(f"products M={M} only {only} tile={tile}", flush=True)
    tuning(f"experts_tile={tile}")
    check_products(bl, M, 2, 7, 288, 272, True, False, choices(M, 2, 7, M, only=only))


@pytest.mark.parametrize("tile", TILES)
def test_products_when_no_choice_has_an_expert(bl, tuning, tile):
    tuning(f"experts_tile={tile}")
    check_products(bl, 50, 2, 4, 96, 64, True, False, np.full((50, 2), -1, np.int32))


# as many experts as there may be: the last of them, and each kind of tiles
@pytest.mark.parametrize("tile", TILES)
def test_products_of_256_experts(bl, tuning, tile):
    tuning(f"experts_tile={tile}")
    for M, only in ((900, None), (60, [0, 63, 64, 255])):
        print(f"products of 256 experts M={M} tile={tile}", flush=True)
        check_products(bl, M, 2, 256, 96, 144, True, False, choices(M, 2, 256, M, 0.1, only=only))


# A few rows at a time: one to eight weight tiles a workgroup, the last of them beyond N, and K of more chunks of 512 than a
# workgroup has waves.
@pytest.mark.parametrize("M,top_k,E,K,N", [(1, 2, 8, 2048, 520), (33, 4, 100, 160, 48), (48, 2, 6, 4640, 300), (130, 2, 4, 1056, 257),
                                           (20, 1, 3, 8224, 136)])
@pytest.mark.parametrize("gather,per_tensor", [(True, False), (False, True)])
@pytest.mark.parametrize("tiles", [1, 2, 4, 8])
def test_products_a_few_rows_at_a_time(bl, tuning, M, top_k, E, K, N, gather, per_tensor, tiles):
    print(f"products M={M} top_k={top_k} E={E} K={K} N={N} gather={gather} per_tensor={per_tensor} tiles={tiles}", flush=True)
    tuning(f"experts_tile=5,decode_tiles={tiles}")
    check_products(bl, M, top_k, E, K, N, gather, per_tensor, choices(M, top_k, E, M + K, unrouted=0.1))


def test_products_of_more_than_4_gib_of_codes(bl):
    """Offsets into the codes pass 32 bits.  Checked on slots from both ends and around the border."""
    T, K, N = 65540, 65536, 40
    codes = torch.randint(-128, 128, (T, K), dtype=torch.int8, device="cuda")
    rowsum = torch.cat([c.sum(1, dtype=torch.int32) for c in codes.split(4096)])
    W = torch.randn(2, N, K, device="cuda")
    packed, _, beta = bl.bitlinear_pack_weights_experts(W)
    signs = [torch.from_numpy(unpack(bl, packed[e], N, K)).double() for e in range(2)]
    offsets = torch.tensor([0, 40000, T], dtype=torch.int32, device="cuda")
    got = bl.bitlinear_matmul_experts(codes, torch.ones(1, device="cuda"), rowsum, packed, N, beta, offsets,
                                      per_tensor=True, flags=bl.FLAG_OUT_ACC_I32).cpu()
    for s in (0, 1, 32767, 32768, 39999, 40000, 65535, 65536, 65537, T - 1):
        assert torch.equal(got[s].double(), signs[int(s >= 40000)] @ codes[s].cpu().double())


@pytest.mark.parametrize("tile", TILES)
def test_products_of_more_than_2_to_32_outputs(bl, tuning, tile):
    """Offsets into Y pass 32 bits.  Checked on slots from both ends and around the border."""
    tuning(f"experts_tile={tile}")
    T, K, N = 262400, 64, 16384
    codes = torch.randint(-128, 128, (T, K), dtype=torch.int8, device="cuda")
    rowsum = codes.sum(1, dtype=torch.int32)
    packed, _, beta = bl.bitlinear_pack_weights_experts(torch.randn(2, N, K, device="cuda"))
    signs = [torch.from_numpy(unpack(bl, packed[e], N, K)).double() for e in range(2)]
    offsets = torch.tensor([0, 131000, T], dtype=torch.int32, device="cuda")
    got = bl.bitlinear_matmul_experts(codes, torch.ones(1, device="cuda"), rowsum, packed, N, beta, offsets,
                                      per_tensor=True, flags=bl.FLAG_OUT_ACC_I32)
    for s in (0, 130999, 131000, 131071, 131072, 262143, 262144, 262145, T - 1):
        assert torch.equal(got[s].cpu().double(), signs[int(s >= 131000)] @ codes[s].cpu().double())


def check_products(bl, M, top_k, E, K, N, gather, per_tensor, ids):
    c = make(bl, M, top_k, E, K, N, gather, per_tensor, ids)
    acc = torch.full((c["T"], N), 77, dtype=torch.int32)
    scale = torch.ones(c["T"])
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        # in float64: sums of at most 128 * 65536 are exact there
        acc[mine] = (c["codes"][c["row"][mine]].double() @ c["signs"][e].double().T).to(torch.int32)
        gamma = c["gamma"] if per_tensor else c["gamma"][c["row"][mine]]
        scale[mine] = (c["beta"][e].cpu() * gamma) / 128.0
    args = (c["codes"].cuda(), c["gamma"].cuda(), c["rowsum"].cuda(), c["packed"], N, c["beta"])
    used = int(c["offsets"][-1])
    # slots behind the last are left as they were
    out = torch.full((c["T"], N), 77, dtype=torch.int32, device="cuda")
    got = bl.bitlinear_matmul_experts(*args, **c["calls"], flags=bl.FLAG_OUT_ACC_I32, out=out).cpu()
    assert torch.equal(got, acc)
    out = torch.full((c["T"], N), -3.0, device="cuda")
    got = bl.bitlinear_matmul_experts(*args, **c["calls"], out=out).cpu()
    assert torch.equal(got[:used], acc[:used].float() * scale[:used, None])
    assert bool((got[used:] == -3.0).all())


def test_products_agree_with_the_plain_layer(bl):
    """One expert with every token: bitlinear_matmul, bit for bit."""
    for M, K, N in [(1, 512, 256), (24, 1056, 300), (200, 2048, 520)]:
        W = torch.from_numpy(wl.make_weight(N, K, 0.02, M)).cuda()
        packed, _, beta = bl.bitlinear_pack_weights(W)
        codes, gamma, rowsum, _ = bl.bitlinear_quant_act(torch.from_numpy(wl.make_activation(M, K, 5)).cuda())
        offsets = torch.tensor([0, M], dtype=torch.int32, device="cuda")
        y = bl.bitlinear_matmul_experts(codes, gamma, rowsum, packed.view(1, -1), N, beta, offsets)
        assert torch.equal(y, bl.bitlinear_matmul(codes, gamma, rowsum, packed, N, beta))


def test_packed_experts_are_the_grouped_layers_bytes(bl):
    W = torch.from_numpy(wl.make_weight(3 * 48, 544, 0.02, 9, mean=0.01)).cuda()
    packed, alpha, beta = bl.bitlinear_pack_weights_experts(W.view(3, 48, 544))
    p2, a2, b2 = bl.bitlinear_pack_weights_grouped(W, groups_n=3)
    assert torch.equal(packed.view(-1), p2) and torch.equal(alpha, a2.view(-1)) and torch.equal(beta, b2.view(-1))


# ---- straight-through backward -----------------------------------------------------------------------
BACKWARDS = [(1, 1, 1, 32, 1), (1, 2, 8, 96, 40), (5, 3, 4, 544, 33), (40, 2, 3, 256, 300), (130, 1, 2, 160, 130),
             (300, 2, 4, 288, 257), (700, 2, 5, 96, 64), (1100, 1, 2, 544, 520)]


@pytest.mark.parametrize("M,top_k,E,K,N", BACKWARDS)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("per_tensor", [True, False])
def test_backward(bl, M, top_k, E, K, N, gather, per_tensor):
    print(f"backward M={M} top_k={top_k} E={E} K={K} N={N} gather={gather} per_tensor={per_tensor}", flush=True)
    check_backward(bl, M, top_k, E, K, N, gather, per_tensor, choices(M, top_k, E, M + K, unrouted=0.1))


# Both tiles of either product, slices of the reductions (more of them than an expert has blocks of 32 slots), and fewer
# workgroups than tiles.
@pytest.mark.parametrize("spec", ["bwd_dx=1,bwd_ring=1", "bwd_dx=2,bwd_ring=2", "bwd_dx=1,bwd_ring=1,bwd_splits=3",
                                  "bwd_dx=2,bwd_ring=2,bwd_splits=5", "bwd_dx=1,bwd_ring=2,bwd_grid=8",
                                  "bwd_dx=2,bwd_ring=1,bwd_grid=4", "bwd_splits=16,bwd_grid=8"])
@pytest.mark.parametrize("M,top_k,E,K,N", [(5, 3, 4, 544, 33), (130, 1, 2, 160, 130), (700, 2, 5, 288, 520),
                                           (40, 2, 3, 544, 2080)])
def test_backward_variants(bl, tuning, M, top_k, E, K, N, spec):
    print(f"backward M={M} top_k={top_k} E={E} K={K} N={N} {spec}", flush=True)
    tuning(spec)
    check_backward(bl, M, top_k, E, K, N, True, True, choices(M, top_k, E, M + K, unrouted=0.1))
    check_backward(bl, M, top_k, E, K, N, True, True, choices(M, top_k, E, M, only=[1]))


# dW with one gamma a tensor and N a multiple of 32, where dY is read transposed: slots that end inside a block of 32 and
# experts without any, columns that end inside a tile, both tiles and slices.  On integers, so exact; one expert's NaN stay
# with it.
@pytest.mark.parametrize("M", [1, 16, 33, 200, 700])
@pytest.mark.parametrize("N,K", [(32, 32), (288, 160), (512, 416), (1312, 128)])
@pytest.mark.parametrize("spec", ["bwd_ring=1", "bwd_ring=2", "bwd_ring=2,bwd_splits=3", "bwd_ring=1,bwd_grid=2"])
def test_backward_dw_from_dy(bl, tuning, M, N, K, spec):
    print(f"backward dW from dY M={M} N={N} K={K} {spec}", flush=True)
    tuning(spec)
    E, top_k = 6, 2
    c = make(bl, M, top_k, E, K, N, True, True, choices(M, top_k, E, M + N, unrouted=0.1))
    dY = torch.randint(-4, 5, (c["T"], N), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    bad = int(np.argmax(np.diff(c["offsets"])))
    dY[c["offsets"][bad]:c["offsets"][bad + 1], ::7] = float("nan")
    dY[c["offsets"][-1]:] = float("nan")
    _, dw = bl.bitlinear_backward_ste_experts(dY.cuda(), c["codes"].cuda(), torch.full((1,), 128.0, device="cuda"), None,
                                              None, **c["calls"], want_dx=False)
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        ref = dY[mine].double().nan_to_num().T @ c["codes"].double()[c["row"][mine]]
        got = dw[e].cpu().double()
        if e == bad and mine.start < mine.stop:
            assert bool(got[::7].isnan().all())
            got[::7] = ref[::7]
        assert torch.equal(got, ref)


# 64 tiles of dW an expert and more, which the XCDs share: numbers of them that eight does not divide, in both tiles, from dY
# itself and from a scaled copy, whole rounds of workgroups and a few workgroups.  On integers, so exact.
@pytest.mark.parametrize("N,K", [(2336, 1184), (2304, 1056), (2056, 1184)])
@pytest.mark.parametrize("per_tensor", [True, False])
@pytest.mark.parametrize("spec", ["bwd_ring=1", "bwd_ring=2", "bwd_ring=1,bwd_grid=16", "bwd_ring=2,bwd_grid=24"])
def test_backward_dw_of_many_tiles(bl, tuning, N, K, per_tensor, spec):
    print(f"backward dW of many tiles N={N} K={K} per_tensor={per_tensor} {spec}", flush=True)
    tuning(spec)
    M, top_k, E = 300, 2, 6
    c = make(bl, M, top_k, E, K, N, True, per_tensor, choices(M, top_k, E, N, unrouted=0.1))
    dY = torch.randint(-4, 5, (c["T"], N), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    dY[c["offsets"][-1]:] = float("nan")
    _, dw = bl.bitlinear_backward_ste_experts(dY.cuda(), c["codes"].cuda(), torch.full_like(c["gamma"], 128.0).cuda(), None,
                                              None, **c["calls"], want_dx=False)
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        # in fp32: sums of a few hundred products of at most 512 are exact
        assert torch.equal(dw[e].cpu(), dY[mine].float().T @ c["codes"].float()[c["row"][mine]])


# dX in whole rounds of workgroups and a last one whose tiles are cut into slices: the number of slots moves the last round
# through nothing, a tile and more tiles than leave room for slices.  On integers, so exact.
@pytest.mark.parametrize("M", [1, 129, 500, 1000, 1040, 1100, 1500, 1900, 2048])
@pytest.mark.parametrize("spec", ["bwd_dx=2,bwd_grid=32", "bwd_dx=1,bwd_grid=64", "bwd_dx=2,bwd_grid=32,bwd_splits=4",
                                  "bwd_dx=2,bwd_grid=32,bwd_splits=1", ""])
def test_backward_dx_rounds(bl, tuning, M, spec):
    print(f"backward dX rounds M={M} {spec}", flush=True)
    tuning(spec)
    top_k, E, K, N = 2, 3, 800, 2080
    c = make(bl, M, top_k, E, K, N, True, True, choices(M, top_k, E, M, unrouted=0.05))
    dY = torch.randint(-4, 5, (c["T"], N), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    one = torch.ones(1, device="cuda")
    dx, _ = bl.bitlinear_backward_ste_experts(dY.cuda(), c["codes"].cuda(), one, c["packed"], one.expand(E).contiguous(),
                                              **c["calls"], want_dw=False)
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        assert torch.equal(dx[mine].cpu().double(), dY[mine].double() @ c["signs"][e].double())


@pytest.mark.parametrize("only", [[0], [4]])
@pytest.mark.parametrize("M", [1, 33, 300])
def test_backward_when_one_expert_has_all_slots(bl, M, only):
    print(f"backward M={M} only {only}", flush=True)
    check_backward(bl, M, 2, 5, 160, 136, True, True, choices(M, 2, 5, M, only=only))


@pytest.mark.parametrize("per_tensor", [True, False])
def test_backward_of_256_experts(bl, per_tensor):
    check_backward(bl, 700, 2, 256, 64, 40, True, per_tensor, choices(700, 2, 256, 3, unrouted=0.1))


@pytest.mark.parametrize("spec", ["", "bwd_splits=4", "bwd_ring=1", "bwd_ring=2"])
def test_backward_when_nothing_is_routed(bl, tuning, spec):
    """dW is zero whatever a gamma that no row has set holds; dX is left as it was."""
    tuning(spec)
    c = make(bl, 30, 2, 3, 96, 64, True, True, np.full((30, 2), -1, np.int32))
    dY = torch.full((60, 64), float("nan"), device="cuda").to(torch.bfloat16)
    _, dw = bl.bitlinear_backward_ste_experts(dY, c["codes"].cuda(), torch.full((1,), float("nan"), device="cuda"),
                                              c["packed"], c["beta"], **c["calls"])
    assert bool((dw == 0).all())


def test_nothing_to_do(bl):
    """No tokens: empty results, and a gradient of zeros for the weights."""
    E, K, N, top_k = 3, 64, 48, 2
    packed, _, beta = bl.bitlinear_pack_weights_experts(torch.randn(E, N, K, device="cuda"))
    order, position, offsets = bl.bitlinear_route(torch.empty(0, top_k, dtype=torch.int32, device="cuda"), E)
    codes, gamma, rowsum, check, scale = bl.bitlinear_quant_nonlinear(torch.empty(0, K, device="cuda"), checkpoint=True)
    assert check.shape == (0, K) and scale.shape == (0, 1)
    y = bl.bitlinear_matmul_experts(codes, gamma, rowsum, packed, N, beta, offsets, order, top_k)
    assert y.shape == (0, N) and bl.bitlinear_combine(y, position).shape == (0, N)
    dy, dw = bl.bitlinear_combine_backward(torch.empty(0, N, device="cuda"), y, position)
    assert dy.shape == (0, N) and dw.shape == (0, top_k)
    dX, dW = bl.bitlinear_backward_ste_experts(dy, codes, gamma, packed, beta, offsets, order, top_k)
    assert dX.shape == (0, K) and bool((dW == 0).all()) and dW.shape == (E, N, K)
    assert bl.bitlinear_nonlinear_backward(torch.empty(0, K, device="cuda"), check, scale).shape == (0, K)


def test_backward_of_more_than_2_to_32_outputs(bl):
    """Offsets into dX and into dW pass 32 bits.  On integers, so exact; checked at both ends and around the border."""
    one, g = torch.ones(1, device="cuda"), torch.Generator().manual_seed(3)
    T, K, N, E = 65664, 65536, 64, 2
    packed, _, _ = bl.bitlinear_pack_weights_experts(torch.randn(E, N, K, device="cuda"))
    signs = [torch.from_numpy(unpack(bl, packed[e], N, K)).double() for e in range(E)]
    offsets = torch.tensor([0, 30000, T], dtype=torch.int32, device="cuda")
    dY = torch.randint(-4, 5, (T, N), generator=g).to(torch.bfloat16)
    codes = torch.zeros(T, K, dtype=torch.int8, device="cuda")  # dX does not read them
    dX, _ = bl.bitlinear_backward_ste_experts(dY.cuda(), codes, one, packed, one.expand(E).contiguous(), offsets,
                                              per_tensor=True, want_dw=False)
    for s in (0, 29999, 30000, 32767, 32768, 65535, 65536, 65537, T - 1):
        assert torch.equal(dX[s].cpu().double(), dY[s].double() @ signs[int(s >= 30000)])
    del dX, codes
    T, K, N, E = 200, 8192, 8192, 65
    ids = np.random.default_rng(1).integers(0, E, (T, 1)).astype(np.int32)
    order, _, offsets = bl.bitlinear_route(gpu(ids), E)
    codes, dY = torch.randint(-128, 128, (T, K), generator=g, dtype=torch.int8), torch.randint(-4, 5, (T, N), generator=g)
    _, dW = bl.bitlinear_backward_ste_experts(dY.to(torch.bfloat16).cuda(), codes.cuda(), 128 * one, None, None, offsets,
                                              order, 1, True, want_dx=False)
    at = offsets.tolist()
    for e in (0, 31, 32, 63, 64):
        mine = slice(at[e], at[e + 1])
        ref = dY[mine].double().T @ codes[order[mine].cpu().long()].double()
        assert torch.equal(dW[e].cpu().double(), ref)


def check_backward(bl, M, top_k, E, K, N, gather, per_tensor, ids):
    c = make(bl, M, top_k, E, K, N, gather, per_tensor, ids)
    g = torch.Generator().manual_seed(7)
    dY = torch.randn(c["T"], N, generator=g).to(torch.bfloat16)
    used = int(c["offsets"][-1])
    dY[used:] = float("nan")  # slots behind the last are not read
    x = c["codes"].double()[c["row"]] * ((c["gamma"] if per_tensor else c["gamma"][c["row"]]).double() / 128).view(-1, 1)
    dx = torch.zeros(c["T"], K, dtype=torch.float64)
    dx_most, dw, dw_most = dx.clone(), torch.zeros(E, N, K, dtype=torch.float64), torch.zeros(E, N, K, dtype=torch.float64)
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        d, s, beta = dY[mine].double(), c["signs"][e].double(), float(c["beta"][e])
        dx[mine], dx_most[mine] = d @ s * beta, d.abs() @ s.abs() * beta
        dw[e], dw_most[e] = d.T @ x[mine], d.abs().T @ x[mine].abs()
    args = (dY.cuda(), c["codes"].cuda(), c["gamma"].cuda(), c["packed"], c["beta"])
    got_x, got_w = bl.bitlinear_backward_ste_experts(*args, **c["calls"])
    rows = int(np.diff(c["offsets"]).max())
    assert bool(((got_x.cpu().double() - dx).abs()[:used] <= (N + 2) * F32 * dx_most[:used]).all())
    # one gamma a token: its product with dY is rounded to fp32 and to bf16
    allowed = (rows + 2) * F32 + (0 if per_tensor else BF16 + 2 * F32)
    assert bool(((got_w.cpu().double() - dw).abs() <= allowed * dw_most).all())
    # either output alone: the same bits
    only_x, none = bl.bitlinear_backward_ste_experts(*args, **c["calls"], want_dw=False)
    assert none is None and torch.equal(only_x[:used], got_x[:used])
    none, only_w = bl.bitlinear_backward_ste_experts(args[0], args[1], args[2], None, None, **c["calls"], want_dx=False)
    assert none is None and torch.equal(only_w, got_w)


def test_backward_exact_on_integers(bl):
    """Small integers: every partial sum is exact, so the results are, whatever the layout of the work."""
    M, top_k, E, K, N = 500, 2, 4, 288, 264
    c = make(bl, M, top_k, E, K, N, True, True, choices(M, top_k, E, 1))
    dY = torch.randint(-4, 5, (c["T"], N), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    one = torch.ones(1, device="cuda")
    dx, dw = bl.bitlinear_backward_ste_experts(dY.cuda(), c["codes"].cuda(), 128 * one, c["packed"], one.expand(E).contiguous(),
                                               **c["calls"])
    for e in range(E):
        mine = slice(c["offsets"][e], c["offsets"][e + 1])
        d = dY[mine].double()
        assert torch.equal(dx[mine].cpu().double(), d @ c["signs"][e].double())
        assert torch.equal(dw[e].cpu().double(), d.T @ c["codes"].double()[c["row"][mine]])


# ---- slots back to tokens ------------------------------------------------------------------------------
COMBINES = [(1, 1, 1), (1, 2, 32), (7, 3, 33), (16, 2, 2048), (50, 8, 130), (333, 2, 1030), (1000, 1, 4096), (9, 2, 9000)]


@pytest.mark.parametrize("M,top_k,N", COMBINES)
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("unrouted", [0.0, 0.4])
def test_combine_and_its_gradient(bl, M, top_k, N, weighted, unrouted):
    print(f"combine M={M} top_k={top_k} N={N} weighted={weighted} unrouted={unrouted}", flush=True)
    E, T = 8, M * top_k
    _, position, offsets = plain_route(choices(M, top_k, E, M, unrouted), E)
    g = torch.Generator().manual_seed(2)
    slots, dY = torch.randn(T, N, generator=g), torch.randn(M, N, generator=g)
    slots[offsets[-1]:] = float("nan")  # nobody's slots are not read
    w = torch.rand(M, top_k, generator=g) if weighted else None
    has = torch.from_numpy(position >= 0)
    at = torch.from_numpy(np.maximum(position, 0))
    picked = torch.where(has[:, :, None], slots[at].double(), 0.0)
    factor = (w.double() if weighted else torch.ones(M, top_k, dtype=torch.float64)) * has
    y, most = (factor[:, :, None] * picked).sum(1), (factor[:, :, None] * picked).abs().sum(1)
    pos, wd = gpu(position.astype(np.int32)), None if w is None else w.cuda()
    got = bl.bitlinear_combine(slots.cuda(), pos, wd)
    assert bool(((got.cpu().double() - y).abs() <= (top_k + 1) * F32 * most).all())
    out = torch.full((T, N), 5.0, dtype=torch.bfloat16, device="cuda")
    dslots, dw = bl.bitlinear_combine_backward(dY.cuda(), slots.cuda(), pos, wd, out=out)
    ref = torch.full((T, N), 5.0, dtype=torch.bfloat16)  # slots that nobody has are left as they were
    products = dY[:, None, :] * (w if weighted else torch.ones(M, top_k))[:, :, None]
    ref[at[has]] = products[has].to(torch.bfloat16)
    assert torch.equal(dslots.cpu(), ref)
    dots = dY.double()[:, None, :] * picked
    assert bool(((dw.cpu().double() - dots.sum(2)).abs() <= (N + 1) * F32 * dots.abs().sum(2)).all())
    again, none = bl.bitlinear_combine_backward(dY.cuda(), None, pos, wd, out=torch.full_like(out, 5.0))
    assert none is None and torch.equal(again, dslots)


def test_combine_keeps_nan(bl):
    """A gradient that is not a number stays none in bf16, whatever its payload."""
    bits = torch.tensor([0x7fffffff, 0x7fc00000, -1, 0x7f800001], dtype=torch.int64).to(torch.int32).cuda()
    dY = bits.view(torch.float32).repeat(3, 2)  # rows of eight, and of one by one
    pos = torch.arange(3, dtype=torch.int32, device="cuda").view(3, 1)
    for g in (dY, dY[:, :7].contiguous()):
        assert bool(bl.bitlinear_combine_backward(g, None, pos)[0].isnan().all())


def test_combine_at_any_alignment(bl):
    """Rows of whole float4 behind an unaligned address: the same bits."""
    M, top_k, N = 20, 2, 64
    _, position, _ = plain_route(choices(M, top_k, 4, 1), 4)
    pos, w = gpu(position.astype(np.int32)), torch.rand(M, top_k, device="cuda")
    slots, dY = torch.randn(M * top_k, N, device="cuda"), torch.randn(M, N, device="cuda")

    def moved(t):
        return torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].copy_(t.reshape(-1)).view(t.shape)

    y, (ds, dw) = bl.bitlinear_combine(slots, pos, w), bl.bitlinear_combine_backward(dY, slots, pos, w)
    assert torch.equal(bl.bitlinear_combine(moved(slots), pos, w), y)
    assert torch.equal(bl.bitlinear_combine(slots, pos, w, out=moved(y)), y)
    for a, b, o in ((moved(dY), slots, ds), (dY, moved(slots), ds), (dY, slots, moved(ds))):
        ds2, dw2 = bl.bitlinear_combine_backward(a, b, pos, w, out=o)
        assert torch.equal(ds2, ds) and bool(((dw2 - dw).abs() <= 2 * N * F32 * (dY.abs().amax() * slots.abs().amax() * N)).all())


# ---- refusals of the binding: a wrong shape would lead a kernel out of a tensor -----------------------------
def test_binding_refuses_wrong_shapes(bl):
    M, top_k, E, K, N = 6, 2, 4, 64, 48
    c = make(bl, M, top_k, E, K, N, True, False, choices(M, top_k, E, 1))
    good = dict(codes=c["codes"].cuda(), gamma=c["gamma"].cuda(), rowsum=c["rowsum"].cuda(), packed=c["packed"], N=N,
                beta=c["beta"], **{k: v for k, v in c["calls"].items() if k != "per_tensor"})
    bl.bitlinear_matmul_experts(**good)
    for name, bad in [("gamma", good["gamma"][:-1]), ("rowsum", good["rowsum"][1:]), ("packed", good["packed"][1:]),
                      ("beta", good["beta"][1:]), ("offsets", good["offsets"][1:]), ("order", good["order"][1:]), ("top_k", 3),
                      ("N", 64), ("codes", good["codes"].float()), ("rowsum", good["rowsum"].cpu())]:
        with pytest.raises(bl.BitLinearError):
            bl.bitlinear_matmul_experts(**{**good, name: bad})
    dY = torch.zeros(M * top_k, N, dtype=torch.bfloat16, device="cuda")
    rest = (good["codes"], good["gamma"], good["packed"], good["beta"], good["offsets"])
    for bad in (dY[1:], dY.float()):
        with pytest.raises(bl.BitLinearError):
            bl.bitlinear_backward_ste_experts(bad, *rest, order=good["order"], top_k=top_k)
    pos = torch.zeros(M, top_k, dtype=torch.int32, device="cuda")
    slots = torch.zeros(M * top_k, N, device="cuda")
    for args in ((slots[1:], pos), (slots, pos[1:]), (slots, pos, torch.ones(M, 1, device="cuda")), (slots, pos.long())):
        with pytest.raises(bl.BitLinearError):
            bl.bitlinear_combine(*args)
    with pytest.raises(bl.BitLinearError):
        bl.bitlinear_quant_nonlinear(slots[:, :32].contiguous(), "tanh")


# ---- all of them together --------------------------------------------------------------------------------
def mixture_forward(bl, X, ids, weights, up, down, fn, per_tensor, train):
    (p1, b1, N1), (p2, b2, N2) = up, down
    E, top_k = b1.numel(), ids.shape[1]
    codes, gamma, rowsum, _ = bl.bitlinear_quant_act(X, per_tensor=per_tensor)
    order, position, offsets = bl.bitlinear_route(ids, E)
    u = bl.bitlinear_matmul_experts(codes, gamma, rowsum, p1, N1, b1, offsets, order, top_k, per_tensor)
    q2, g2, r2, check, scale = bl.bitlinear_quant_nonlinear(u, fn, per_tensor=per_tensor, checkpoint=train, rows=offsets[E:])
    y = bl.bitlinear_matmul_experts(q2, g2, r2, p2, N2, b2, offsets, per_tensor=per_tensor)
    return bl.bitlinear_combine(y, position, weights), dict(codes=codes, gamma=gamma, order=order, position=position,
                                                            offsets=offsets, u=u, q2=q2, g2=g2, check=check, scale=scale, y=y)


def mixture_backward(bl, dY, X, ids, weights, up, down, fn, per_tensor, s):
    (p1, b1, _), (p2, b2, _) = up, down
    E, top_k = b1.numel(), ids.shape[1]
    rows = s["offsets"][E:]
    dy, dw = bl.bitlinear_combine_backward(dY, s["y"], s["position"], weights)
    dx2, dW2 = bl.bitlinear_backward_ste_experts(dy, s["q2"], s["g2"], p2, b2, s["offsets"], per_tensor=per_tensor)
    du = bl.bitlinear_nonlinear_backward(dx2, s["check"], s["scale"], fn, rows=rows)
    dx1, dW1 = bl.bitlinear_backward_ste_experts(du, s["codes"], s["gamma"], p1, b1, s["offsets"], s["order"], top_k, per_tensor)
    dxhat = bl.bitlinear_combine(dx1, s["position"])
    return bl.bitlinear_layernorm_backward(dxhat, X), dW1, dW2, dw


def mixture(bl, M, top_k, E, d, width, unrouted=0.1):
    g = torch.Generator().manual_seed(M)
    W1, W2 = torch.randn(E, width, d, generator=g) * 0.02, torch.randn(E, d, width, generator=g) * 0.02
    p1, _, b1 = bl.bitlinear_pack_weights_experts(W1.cuda())
    p2, _, b2 = bl.bitlinear_pack_weights_experts(W2.cuda())
    X = torch.randn(M, d, generator=g).cuda()
    ids = gpu(choices(M, top_k, E, M, unrouted))
    weights = torch.rand(M, top_k, generator=g).cuda()
    return X, ids, weights, (p1, b1, width), (p2, b2, d)


@pytest.mark.parametrize("M,top_k,E,d,width", [(1, 2, 4, 256, 512), (40, 2, 6, 160, 544), (600, 2, 4, 256, 1024)])
@pytest.mark.parametrize("per_tensor", [False, True])
def test_mixture_forward_and_backward(bl, M, top_k, E, d, width, per_tensor):
    """A feed-forward network of experts against the same network out of the library's plain layers, an expert at a time
    (one rounding to bf16 at the same places), and its gradients against autograd in 64 bits."""
    print(f"mixture M={M} top_k={top_k} E={E} {d} {width} per_tensor={per_tensor}", flush=True)
    X, ids, weights, up, down = mixture(bl, M, top_k, E, d, width)
    Y, s = mixture_forward(bl, X, ids, weights, up, down, "gelu", per_tensor, True)
    at = s["offsets"].tolist()
    token = s["order"].long().clamp_min(0) // top_k
    codes, gamma, rowsum, _ = bl.bitlinear_quant_act(X, per_tensor=per_tensor)
    for e in range(E):
        mine = slice(at[e], at[e + 1])
        if at[e] == at[e + 1]:
            continue
        t = token[mine]
        u = bl.bitlinear_matmul(codes[t], gamma if per_tensor else gamma[t], rowsum[t], up[0][e], width, up[1][e:e + 1],
                                per_tensor)
        assert torch.equal(u, s["u"][mine])
        q, g2 = s["q2"][mine], s["g2"] if per_tensor else s["g2"][mine]
        y = bl.bitlinear_matmul(q, g2, q.sum(1, dtype=torch.int32), down[0][e], d, down[1][e:e + 1], per_tensor)
        assert torch.equal(y, s["y"][mine])
    # gradients, each step against autograd on what the step before it gave
    dY = (torch.randn(M, d, generator=torch.Generator().manual_seed(9)) * 1e-2).cuda()
    dX, dW1, dW2, dw = mixture_backward(bl, dY, X, ids, weights, up, down, "gelu", per_tensor, s)
    Wd, Xd = weights.double().requires_grad_(), X.double().requires_grad_()
    used, E1 = at[E], range(E)
    S1 = torch.stack([torch.from_numpy(unpack(bl, up[0][e], width, d)) for e in E1]).cuda().double()
    S2 = torch.stack([torch.from_numpy(unpack(bl, down[0][e], d, width)) for e in E1]).cuda().double()
    W1, W2 = (S1 * up[1].double().view(-1, 1, 1)).requires_grad_(), (S2 * down[1].double().view(-1, 1, 1)).requires_grad_()

    def through(value, quantised):  # straight-through: the quantised value, the value's gradient
        return value + (quantised - value).detach()

    xhat = torch.nn.functional.layer_norm(Xd, (d,), eps=1e-5)
    xq = through(xhat, codes.double() * (gamma.double() / 128).view(-1, 1))
    v = (s["check"].float() * s["scale"].repeat_interleave(128, 1)[:, :width]).double()
    parts = []
    for e in E1:
        mine = slice(at[e], at[e + 1])
        u = through(xq[token[mine]] @ W1[e].T, v[mine])
        h = torch.nn.functional.layer_norm(torch.nn.functional.gelu(u), (width,), eps=1e-5)
        hq = through(h, s["q2"][mine].double() * (s["g2"].double() if per_tensor else s["g2"][mine].double().view(-1, 1)) / 128)
        parts.append(hq @ W2[e].T)
    slots = torch.cat(parts + [torch.zeros(M * top_k - used, d, dtype=torch.float64, device="cuda")])
    has = (s["position"] >= 0).double()
    out = (slots[s["position"].long().clamp_min(0)] * (Wd * has).unsqueeze(2)).sum(1)
    assert float((Y.double() - out.detach()).norm()) <= 1e-5 * float(out.detach().norm()) + 1e-12  # fp32 at each of four steps
    out.backward(dY.double())
    # gradients pass two roundings to bf16 (2^-8 each at most, 2^-8 again with gammas of tokens): 1.2 % at the very most
    for got, ref in ((dX, Xd.grad), (dW1, W1.grad), (dW2, W2.grad), (dw, Wd.grad)):
        assert float((got.double() - ref).norm()) <= 3 * BF16 * float(ref.norm()) + 1e-12


@pytest.mark.parametrize("per_tensor", [False, True])
def test_mixture_with_a_marked_rectifier(bl, per_tensor):
    """The same network as with the plain rectifier, whose gradient reaches exactly the positive inputs of the function."""
    X, ids, weights, up, down = mixture(bl, 300, 2, 4, 256, 1056)
    Y, s = mixture_forward(bl, X, ids, weights, up, down, "relu_marked", per_tensor, True)
    assert torch.equal(Y, mixture_forward(bl, X, ids, weights, up, down, "relu", per_tensor, True)[0])
    used = int(s["offsets"][-1])
    dY = torch.randn(300, 256, device="cuda") * 1e-2
    dy, _ = bl.bitlinear_combine_backward(dY, s["y"], s["position"], weights)
    dx2, _ = bl.bitlinear_backward_ste_experts(dy, s["q2"], s["g2"], down[0], down[1], s["offsets"], per_tensor=per_tensor)
    du = bl.bitlinear_nonlinear_backward(dx2, s["check"], s["scale"], "relu_marked", rows=s["offsets"][4:])
    assert torch.equal(du[:used] != 0, s["u"][:used] > 0)
    dX, dW1, dW2, dw = mixture_backward(bl, dY, X, ids, weights, up, down, "relu_marked", per_tensor, s)
    ref = bl.bitlinear_backward_ste_experts(du, s["codes"], s["gamma"], up[0], up[1], s["offsets"], s["order"], 2, per_tensor)
    assert torch.equal(dW1, ref[1]) and torch.equal(dX, bl.bitlinear_layernorm_backward(
        bl.bitlinear_combine(ref[0], s["position"]), X))


def test_mixture_in_a_graph_with_other_work_between_replays(bl):
    """Forward and backward captured; replayed with new tokens and new choices, with eager calls and other streams' work
    between the replays; every replay is the eager result, bit for bit."""
    M, top_k, E, d, width = 70, 2, 4, 256, 512
    X, ids, weights, up, down = mixture(bl, M, top_k, E, d, width)
    dY = torch.randn(M, d, device="cuda") * 1e-2

    def step():
        Y, s = mixture_forward(bl, X, ids, weights, up, down, "silu", True, True)
        return Y, *mixture_backward(bl, dY, X, ids, weights, up, down, "silu", True, s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for r in range(4):
        X.copy_(torch.randn(M, d, device="cuda"))
        ids.copy_(gpu(choices(M, top_k, E, 100 + r, unrouted=[0.0, 0.5, 1.0, 0.1][r])))
        ref = step()
        torch.cuda.synchronize()
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert torch.equal(a, b)


def test_calls_follow_the_current_stream(bl):
    """Operands made on a side stream, used there without a synchronisation: the same results as on the default stream."""
    X, ids, weights, up, down = mixture(bl, 200, 2, 4, 256, 512, unrouted=0.0)
    ref, _ = mixture_forward(bl, X, ids, weights, up, down, "gelu", False, False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            late = torch.zeros_like(X)
            for _ in range(20):
                late.add_(1.0)
            late.copy_(X)
            y, _ = mixture_forward(bl, late, ids.clone(), weights, up, down, "gelu", False, False)
        side.synchronize()
        assert torch.equal(y, ref)
