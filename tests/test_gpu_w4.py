"""Products of a few rows with 4-bit weights (lq_w4_*) against the plain 64-bit implementation."""
import pytest
import torch

from tests import blocks_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def make(M, K, N, group, x="bf16", y="bf16", seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    codes = torch.randint(-7, 8, (N, K), generator=g, device="cuda", dtype=torch.int8)
    scales = normal(N, -(-K // group)) * 0.1  # of both signs
    X, dY = (normal(M, K) * 2 + 0.5).to(DT[x]), (normal(M, N) * 0.1).to(DT[y])
    return codes, scales, X, dY, normal(N)


def check_all(lq, cfg, packed, codes, scales, X, dY, bias, what=""):
    xt, yt = X.dtype, dY.dtype
    ref.check(lq.lq_w4_fwd(cfg, packed, X, bias), ref.w4_fwd(X, codes, scales, cfg.group, bias, yt), what + " forward")
    ref.check(lq.lq_w4_bwd(cfg, packed, dY), ref.w4_bwd(dY, codes, scales, cfg.group, xt), what + " gradient")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (40, 300), (33, 31), (5, 64), (160, 1152), (100, 2240)])
def test_pack_by_the_int_rule(lq, N, K, group):
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    W = torch.randn(N, K, generator=g, device="cuda") * 0.02
    W[:, : K // 3] = 0.0  # groups of zeros, and groups with some
    cfg = lq.make_w4_config(N, K, group)
    want_codes, want_scales = ref.w4_quantise(W.cpu(), group)
    for packed in (lq.lq_w4_pack(cfg, W), lq.lq_w4_pack(cfg, W, packed=torch.full((lq.lq_w4_sizes(cfg),), 0xFF, dtype=torch.uint8, device="cuda"))):
        codes, scales = lq.lq_w4_unpack(cfg, packed)
        assert torch.equal(codes.cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
    again = lq.lq_w4_pack_codes(cfg, codes, scales)
    assert torch.equal(again, packed)


def test_pack_groups_of_the_smallest_numbers(lq):
    """A group whose largest value is below 7 over the largest number: codes within one of the quotient, zeros exact."""
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    W = torch.randn(16, 128, generator=g, device="cuda")
    W[:, 5::7] = 0.0
    W = (W.double() * 2.0 ** -129).float()
    cfg = lq.make_w4_config(16, 128, 64)
    codes, scales = lq.lq_w4_unpack(cfg, lq.lq_w4_pack(cfg, W))
    amax = W.double().abs().view(16, 2, 64).amax(-1)
    assert not codes[:, 5::7].any()
    assert (codes.double() - W.double() * 7 / amax.repeat_interleave(64, 1)).abs().max() <= 1.0
    assert (scales.double() - amax / 7).abs().max() <= 2.0 ** -149


def test_codes_past_32_bits(lq):
    """More than 2^32 bytes of codes: the last channels, and the gradient with respect to some columns."""
    N, K, group = 2 ** 17 + 5, 2 ** 16, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    codes = torch.randint(-7, 8, (N, K), generator=g, device="cuda", dtype=torch.int8)
    scales = torch.randn(N, K // group, generator=g, device="cuda")
    cfg = lq.make_w4_config(N, K, group, "f32", "f32")
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    X, dY = torch.randn(1, K, generator=g, device="cuda"), torch.randn(1, N, generator=g, device="cuda")
    rows = torch.cat([torch.arange(40), torch.arange(N - 40, N)]).cuda()
    ref.check(lq.lq_w4_fwd(cfg, packed, X)[:, rows], ref.w4_fwd(X, codes[rows], scales[rows], group, None, torch.float32), "forward")
    dX = lq.lq_w4_bwd(cfg, packed, dY)
    for at in (0, K - 128):
        part = codes[:, at:at + 128].contiguous(), scales[:, at // group:at // group + 1].contiguous()
        ref.check(dX[:, at:at + 128], ref.w4_bwd(dY, *part, group, torch.float32), "gradient")


def test_codes_beyond_the_range(lq):
    codes = torch.arange(-128, 128, dtype=torch.int8, device="cuda").view(2, 128)
    cfg = lq.make_w4_config(2, 128, 32)
    got, _ = lq.lq_w4_unpack(cfg, lq.lq_w4_pack_codes(cfg, codes, torch.ones(2, 4, device="cuda")))
    assert torch.equal(got, codes.clamp(-7, 7))


@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("M,K,N,group", [(1, 1, 1, 32), (1, 128, 16, 128), (2, 130, 17, 64), (3, 1152, 100, 64), (1, 2240, 1153, 128), (16, 257, 40, 32), (17, 300, 50, 64),
                                         (31, 64, 33, 32), (33, 1000, 70, 128), (64, 96, 260, 32), (65, 136, 48, 64), (130, 520, 31, 32), (5, 65, 4608, 64),
                                         (4, 4608, 300, 64), (7, 40, 13441, 32)])
def test_sizes(lq, M, K, N, group, x, y):
    codes, scales, X, dY, bias = make(M, K, N, group, x, y, seed=M + K)
    cfg = lq.make_w4_config(N, K, group, x, y)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    check_all(lq, cfg, packed, codes, scales, X, dY, bias)
    ref.check(lq.lq_w4_fwd(cfg, packed, X), ref.w4_fwd(X, codes, scales, group, None, DT[y]), "without a bias")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N,x", [(40, 140, 3003, "bf16"), (40, 140, 10007, "bf16"), (40, 140, 25001, "bf16"), (70, 1100, 1000, "bf16"), (20, 1100, 2503, "f32"), (20, 1100, 5007, "f32"), (20, 1100, 7007, "f32"), (3, 1100, 14333, "f32"),
                                     (20, 140, 5007, "f32"), (20, 140, 10007, "f32"), (20, 140, 15001, "f32"), (16, 1100, 4090, "f32")])
def test_forms(lq, M, K, N, x, group):
    """One to four tiles to a workgroup, the last one with fewer, by four and eight wavefronts."""
    codes, scales, X, dY, bias = make(M, K, N, group, x, "f32", seed=N)
    cfg = lq.make_w4_config(N, K, group, x, "f32")
    check_all(lq, cfg, lq.lq_w4_pack_codes(cfg, codes, scales), codes, scales, X, dY, bias)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("pad,start", [(1, 0), (1, 1), (3, 2), (8, 0), (8, 3)])
def test_rows_that_start_anywhere(lq, pad, start, x):
    M, K, N, group = 5, 264, 70, 64
    codes, scales, X, dY, bias = make(M, K, N, group, x, x)
    cfg = lq.make_w4_config(N, K, group, x, x)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)

    def apart(t, fill=float("nan")):
        big = torch.full((M, t.shape[1] + pad), fill, dtype=t.dtype, device="cuda").flatten()
        big = torch.cat([big, big[:start]])[start:]
        v = big.as_strided((M, t.shape[1]), (t.shape[1] + pad, 1))
        v.copy_(t)
        return big, v
    _, Xs = apart(X)
    _, gs = apart(dY)
    ybig, Y = apart(torch.zeros_like(dY), 7.0)
    xbig, dX = apart(torch.zeros_like(X), 7.0)
    lq.lq_w4_fwd(cfg, packed, Xs, bias, Y=Y)
    lq.lq_w4_bwd(cfg, packed, gs, dX=dX)
    assert torch.equal(Y, lq.lq_w4_fwd(cfg, packed, X, bias)) and torch.equal(dX, lq.lq_w4_bwd(cfg, packed, dY))
    for big, cols in ((ybig, N), (xbig, K)):  # what lies between the rows stays
        at = torch.arange(big.numel(), device="cuda") % (cols + pad)
        assert (big[at >= cols] == 7.0).all()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 2, 6, 20, 70])
def test_a_row_does_not_depend_on_the_others(lq, M, x):
    K, N, group = 392, 100, 32
    codes, scales, X, dY, bias = make(M, K, N, group, x, x)
    cfg = lq.make_w4_config(N, K, group, x, x)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    Y, dX = lq.lq_w4_fwd(cfg, packed, X, bias), lq.lq_w4_bwd(cfg, packed, dY)
    assert torch.equal(Y, lq.lq_w4_fwd(cfg, packed, X, bias)) and torch.equal(dX, lq.lq_w4_bwd(cfg, packed, dY))
    if M < 2:
        return
    X2, dY2 = X.clone(), dY.clone()
    X2[1, 5], X2[1, 7], dY2[1, 3] = float("nan"), float("inf"), float("nan")
    Y2, dX2 = lq.lq_w4_fwd(cfg, packed, X2, bias), lq.lq_w4_bwd(cfg, packed, dY2)
    others = torch.arange(M, device="cuda") != 1
    assert torch.equal(Y[others], Y2[others]) and torch.equal(dX[others], dX2[others])
    assert torch.isnan(Y2[1]).all() and torch.isnan(dX2[1]).all()


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_infinities_give_what_the_formula_gives(lq, x):
    M, K, N, group = 3, 200, 60, 64
    codes, scales, X, dY, bias = make(M, K, N, group, x, "f32")
    cfg = lq.make_w4_config(N, K, group, x, "f32")
    X[0, 70], X[1, 3], X[1, 4] = float("inf"), float("-inf"), float("inf")
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    Y = lq.lq_w4_fwd(cfg, packed, X, bias)
    W = codes.double() * scales.double().repeat_interleave(group, 1)[:, :K]
    want = (X.double()[:, None, :] * W[None]).sum(-1) + bias.double()  # inf * 0 and inf - inf are not numbers
    bad = ~torch.isfinite(want)
    assert bad[:2].any() and not bad[2].any()
    assert torch.equal(Y.double()[bad].nan_to_num(nan=3.0), want[bad].nan_to_num(nan=3.0))
    assert torch.isfinite(Y[~bad]).all()


def test_strong_values_in_all_24_bits(lq):
    """fp32 rows whose strong channels cancel: what the small ones add is left, to the bits of fp32 sums."""
    K, N, group = 256, 32, 32
    codes = torch.ones(N, K, dtype=torch.int8, device="cuda")
    scales = torch.ones(N, K // group, device="cuda")
    X = torch.zeros(2, K, device="cuda")
    X[:, 0], X[:, 1], X[0, 2], X[1, 2] = 1.0 + 2.0 ** -23, -1.0, 2.0 ** -20, 3.0
    cfg = lq.make_w4_config(N, K, group, "f32", "f32")
    Y = lq.lq_w4_fwd(cfg, lq.lq_w4_pack_codes(cfg, codes, scales), X)
    # partial sums are at most 4: sums of three terms of 256 values each are off by (768 + 24) 2^-24 of the largest term at worst in general; here only a few values are not
    # zero, whose terms (8 bits each) add up without a rounding above 2^-22
    want = torch.tensor([2.0 ** -23 + 2.0 ** -20, 3.0 + 2.0 ** -23], device="cuda", dtype=torch.float64)
    assert ((Y.double() - want[:, None]).abs() <= 2.0 ** -22).all()


def test_empty_batch_and_workspace(lq):
    cfg = lq.make_w4_config(300, 200, 32)
    codes, scales, _, _, bias = make(1, 200, 300, 32)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    assert lq.lq_w4_fwd(cfg, packed, torch.zeros(0, 200, dtype=torch.bfloat16, device="cuda"), bias).shape == (0, 300)
    assert lq.lq_w4_bwd(cfg, packed, torch.zeros(0, 300, dtype=torch.bfloat16, device="cuda")).shape == (0, 200)
    with pytest.raises(lq.LqError) as e:
        lq.lq_w4_fwd(cfg, packed[:-256], torch.zeros(1, 200, dtype=torch.bfloat16, device="cuda"), bias)
    assert e.value.status == lq.LQ_ERR_BUFFER_TOO_SMALL


def test_captured_and_replayed_on_a_stream(lq):
    M, K, N, group = 2, 1152, 700, 64
    codes, scales, X, dY, bias = make(M, K, N, group, "bf16", "f32")
    cfg = lq.make_w4_config(N, K, group, "bf16", "f32")
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    Y, dX = torch.empty(M, N, device="cuda"), torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(lq.lq_w4_work_sizes(cfg, M), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        lq.lq_w4_fwd(cfg, packed, X, bias, Y=Y)
        lq.lq_w4_bwd(cfg, packed, dY, dX=dX, work=work)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            lq.lq_w4_fwd(cfg, packed, X, bias, Y=Y)
            lq.lq_w4_bwd(cfg, packed, dY, dX=dX, work=work)
    torch.cuda.synchronize()
    for k in range(4):
        _, _, X2, dY2, _ = make(M, K, N, group, "bf16", "f32", seed=10 + k)
        X.copy_(X2)
        dY.copy_(dY2)
        want = lq.lq_w4_fwd(cfg, packed, X2, bias), lq.lq_w4_bwd(cfg, packed, dY2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want[0]) and torch.equal(dX, want[1]), k


def normal24(rows, cols, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda")


FORMS = [(256, 32), (1100, 2007), (1100, 5007), (1100, 9007), (1100, 14333), (140, 3003), (140, 14333), (140, 30001), (4608, 300)]  # one to four tiles to a workgroup, by four and eight wavefronts


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K,N", FORMS)
def test_all_24_bits_of_rows(lq, K, N, group):
    """Strong channels that cancel leave what is 2^-18 of them to 2^-22 (a third term left out would cost 2^-18): every partial sum is a multiple of 2^-23 below 2 and so exact in 24 bits.  A row
    with one channel alone is that channel's value to the last bit, times a code that is a power of two, then times the scale with one rounding."""
    M = 3
    codes = torch.ones(N, K, dtype=torch.int8, device="cuda")
    cfg = lq.make_w4_config(N, K, group, "f32", "f32")
    packed = lq.lq_w4_pack_codes(cfg, codes, torch.ones(N, -(-K // group), device="cuda"))
    X = torch.zeros(M, K, device="cuda")
    strong = 1.0 + 2.0 ** -10 + 2.0 ** -18 + 2.0 ** -23
    for m, (a, b, c, d) in enumerate(((0, 1, 2, 3), (0, K - 1, K // 2, 5), (K - 2, K // 3, 7, 70))):
        X[m, a], X[m, b], X[m, c], X[m, d] = strong, -1.0, -(2.0 ** -10), 2.0 ** -20
    want = 2.0 ** -18 + 2.0 ** -20 + 2.0 ** -23
    assert ((lq.lq_w4_fwd(cfg, packed, X).double() - want).abs() <= 2.0 ** -22).all()
    scales = normal24(N, -(-K // group), 5) * 0.1
    codes = torch.tensor([1, -1, 2, -2, 4, -4], dtype=torch.int8, device="cuda")[torch.arange(N * K, device="cuda") % 6].view(N, K)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    at = torch.tensor([K - 1, K // 2, 3], device="cuda")
    X.zero_()
    X[torch.arange(M, device="cuda"), at] = normal24(1, M, 6)[0]
    got = lq.lq_w4_fwd(cfg, packed, X)
    for m in range(M):
        want = (X[m, at[m]].double() * codes[:, at[m]].double() * scales[:, at[m] // group].double()).float()
        assert torch.equal(got[m], want), m


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(2, 6912, 1152), (3, 359, 256), (16, 13441, 300), (5, 64, 64), (1, 33, 4608), (20, 2000, 130)])
def test_all_24_bits_of_gradients(lq, M, N, K, group):
    """The same of dY, in one launch and in parts of N; a bf16 dY times the scale is a number of 24 bits too."""
    codes = torch.ones(N, K, dtype=torch.int8, device="cuda")
    cfg = lq.make_w4_config(N, K, group, "f32", "f32")
    packed = lq.lq_w4_pack_codes(cfg, codes, torch.ones(N, -(-K // group), device="cuda"))
    dY = torch.zeros(M, N, device="cuda")
    strong = 1.0 + 2.0 ** -10 + 2.0 ** -18 + 2.0 ** -23
    for m in range(M):
        a, b, c, d = ((0, 1, 2, 3), (0, N - 1, N // 2, 5), (N - 2, N // 3, 7, 30))[m % 3]
        dY[m, a], dY[m, b], dY[m, c], dY[m, d] = strong, -1.0, -(2.0 ** -10), 2.0 ** -20
    want = 2.0 ** -18 + 2.0 ** -20 + 2.0 ** -23
    assert ((lq.lq_w4_bwd(cfg, packed, dY).double() - want).abs() <= 2.0 ** -22).all()
    scales = normal24(N, -(-K // group), 5) * 0.1
    codes = torch.tensor([1, -1, 2, -2, 4, -4], dtype=torch.int8, device="cuda")[torch.arange(N * K, device="cuda") % 6].view(N, K)
    at = (torch.arange(M, device="cuda") * 97 + 11) % N
    for y in ("f32", "bf16"):
        cfg = lq.make_w4_config(N, K, group, "f32", y)
        packed = lq.lq_w4_pack_codes(cfg, codes, scales)
        dY = torch.zeros(M, N, dtype=DT[y], device="cuda")
        dY[torch.arange(M, device="cuda"), at] = normal24(1, M, 6)[0].to(DT[y])
        got = lq.lq_w4_bwd(cfg, packed, dY)
        each = scales[at].repeat_interleave(group, 1)[:, :K]
        up = (dY[torch.arange(M, device="cuda"), at].double()[:, None] * each.double()).float()  # the one rounding
        assert torch.equal(got, (up.double() * codes[at].double()).float()), y


@pytest.mark.parametrize("M,K,N", [(2, 1152, 6912), (16, 2240, 13441), (3, 4608, 300), (40, 1100, 5007)])
def test_rounding_errors_of_random_rows(lq, M, K, N):
    """n sums of numbers of random signs are off by some sqrt(n) of a rounding of the result's size (in the 2-norm over all results), not by n: rows in one term of three would be off by 2^-9."""
    codes, scales, X, dY, _ = make(M, K, N, 64, "f32", "f32", seed=N)
    X = X - 0.5  # (no mean: results are of the size of a random sum)
    cfg = lq.make_w4_config(N, K, 64, "f32", "f32")
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    for got, (want, _), n in ((lq.lq_w4_fwd(cfg, packed, X), ref.w4_fwd(X, codes, scales, 64, None, torch.float32), K),
                              (lq.lq_w4_bwd(cfg, packed, dY), ref.w4_bwd(dY, codes, scales, 64, torch.float32), N)):
        assert float((got.double() - want).norm() / want.norm()) <= ref.U * (3 * n + 24) ** 0.5


def test_weights_of_another_layer_are_told(lq):
    """lq_w4_verify: another N, K or group, other memory, another kind of packed weights; the weights depend on nothing else of the configuration."""
    codes, scales, X, _, _ = make(2, 256, 512, 64)
    cfg = lq.make_w4_config(512, 256, 64)
    packed = lq.lq_w4_pack_codes(cfg, codes, scales)
    for x in ("bf16", "f32"):
        for y in ("bf16", "f32"):
            lq.lq_w4_verify(lq.make_w4_config(512, 256, 64, x, y), packed)
    lq.lq_w4_verify(cfg, lq.lq_w4_pack(cfg, torch.randn(512, 256, device="cuda")))
    same = [lq.make_w4_config(512, 256, 128), lq.make_w4_config(256, 512, 64), lq.make_w4_config(511, 256, 64), lq.make_w4_config(512, 255, 64), lq.make_w4_config(16, 128, 32)]
    for other in same:
        assert lq.lq_w4_sizes(other) <= packed.numel()
        with pytest.raises(lq.LqError) as e:
            lq.lq_w4_verify(other, packed)
        assert e.value.status == lq.LQ_ERR_STALE_BLOB
    for blob in (torch.zeros_like(packed), torch.full_like(packed, 0xFF), packed[256:].clone().resize_(packed.numel())):
        with pytest.raises(lq.LqError) as e:
            lq.lq_w4_verify(cfg, blob)
        assert e.value.status == lq.LQ_ERR_STALE_BLOB
    with pytest.raises(lq.LqError) as e:
        lq.lq_w4_verify(cfg, packed[:-256])
    assert e.value.status == lq.LQ_ERR_BUFFER_TOO_SMALL


@pytest.mark.parametrize("e", [-100, -109, -111, -118, -125, -130])
def test_rows_of_the_smallest_numbers(lq, e):
    """One channel to a row: the value itself from 2^-110 on; below, what three bf16 terms hold of it, which cut off less than 2^-133."""
    K, N, M = 256, 48, 16
    cfg = lq.make_w4_config(N, K, 64, "f32", "f32")
    packed = lq.lq_w4_pack_codes(cfg, torch.ones(N, K, dtype=torch.int8, device="cuda"), torch.ones(N, K // 64, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(-e)
    v = ((1 + torch.rand(M, generator=g, device="cuda").double()) * 2.0 ** e).float()
    X, dY, rows = torch.zeros(M, K, device="cuda"), torch.zeros(M, N, device="cuda"), torch.arange(M, device="cuda")
    X[rows, rows * 7], dY[rows, rows * 3] = v, v
    off = 0.0 if e >= -110 else 2.0 ** -133
    for got in (lq.lq_w4_fwd(cfg, packed, X), lq.lq_w4_bwd(cfg, packed, dY)):
        assert ((got.double() - v.double()[:, None]).abs() <= off).all()
