"""What the adapters' products keep of their numbers: cases made so that every sum is exact in fp32 and the answer is only what the last bits leave."""
import pytest
import torch

from tests.test_gpu_adapter import lq  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def triples(n, g):
    """Numbers a 2^16 + b 2^8 + c of 24 bits, as three bf16 integers each."""
    a, b, c = (torch.randint(lo, 256, (n,), generator=g).float() for lo in (128, 1, 1))
    return a, b, c


def cancelling(M, depth, width, R, slots, ids):
    """Left rows that pick one of 21 triples, a first factor whose rank 0 gives that number of 24 bits and rank 1 its negative without the last 8, a second factor that
    adds them up times a power of two: left, first (slots x R x depth), second (slots x width x R), what comes out (integers of 8 bits times powers of two)."""
    g = torch.Generator().manual_seed(M + R)
    n = 21
    first, second = torch.zeros(slots, R, depth), torch.zeros(slots, width, R)
    left, last = torch.zeros(M, depth), torch.zeros(slots, n)
    for s in range(slots):
        a, b, c = triples(n, g)
        last[s] = c
        for t, v in enumerate((a, b, c)):
            first[s, 0, t:3 * n:3] = v
            if t < 2:
                first[s, 1, t:3 * n:3] = -v
    pick = torch.arange(M) % n
    for t in range(3):
        left[torch.arange(M), 3 * pick + t] = 2.0 ** (16 - 8 * t)
    power = 2.0 ** (torch.arange(width) % 5 - 2)
    second[:, :, 0] = second[:, :, 1] = power
    want = torch.where((ids >= 0)[:, None], last[ids.clamp(min=0), pick][:, None] * power, torch.zeros(()))
    return left.bfloat16().cuda(), first.bfloat16().cuda(), second.bfloat16().cuda(), want.cuda()


def batch(M, slots, seed=0):
    return torch.randint(-1, slots, (M,), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("R", [8, 40, 72, 128])
@pytest.mark.parametrize("M,slots,N", [(150, 1, 64), (150, 3, 192), (130, 70, 1088)])
def test_all_bits_of_the_first_product_reach_the_output(lq, M, slots, N, R):  # noqa: F811
    ids = batch(M, slots)
    X, A, B, want = cancelling(M, 64, N, R, slots, ids)
    cfg = lq.make_adapter_config(N, 64, R, slots)
    ranks, scales = torch.full((slots,), R, dtype=torch.int32, device="cuda"), torch.ones(slots, device="cuda")
    Y = lq.lq_adapter_fwd(cfg, lq.lq_adapter_plan(slots, ids.int().cuda()), X, A, B, ranks, scales, torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(Y.float(), want)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("R", [8, 40, 72, 128])
@pytest.mark.parametrize("M,slots,K", [(150, 1, 64), (150, 3, 192), (130, 70, 1088)])
def test_all_bits_of_the_backwards_first_product_reach_dx(lq, M, slots, K, R, x):  # noqa: F811
    ids = batch(M, slots)
    dY, Bt, At, want = cancelling(M, 64, K, R, slots, ids)
    A, B = At.transpose(1, 2).contiguous(), Bt.transpose(1, 2).contiguous()
    cfg = lq.make_adapter_config(64, K, R, slots, x)
    ranks, scales = torch.full((slots,), R, dtype=torch.int32, device="cuda"), torch.ones(slots, device="cuda")
    X = torch.ones(M, K, dtype=torch.float32 if x == "f32" else torch.bfloat16, device="cuda")
    plan = lq.lq_adapter_plan(slots, ids.int().cuda())
    inter = torch.empty(lq.lq_adapter_sizes(cfg, M)[0], dtype=torch.uint8, device="cuda")
    lq.lq_adapter_fwd(cfg, plan, X, A, B, ranks, scales, dY, inter=inter)
    dX, _, _ = lq.lq_adapter_bwd(cfg, plan, X, A, B, ranks, scales, inter, dY)
    assert torch.equal(dX.float(), want)


@pytest.mark.parametrize("M,slots,K,N,R", [(1, 1, 64, 64, 8), (40, 1, 192, 64, 40), (3000, 1, 64, 64, 24), (30, 30, 128, 64, 8), (30, 30, 64, 64, 128)])
def test_all_bits_of_fp32_x_reach_da(lq, M, slots, K, N, R):  # noqa: F811
    """dA of adapters with one row that has a derivative: each value is one product of two numbers of 24 bits, whose terms after the first are as large as they come.
    It is rounded when the last of its terms' products is added (by at most 2^-23 of it, cut off or to nearest); what the additions before lose is below 2^-29."""
    g = torch.Generator().manual_seed(M + K)
    dY, X = torch.zeros(M, N), torch.zeros(M, K, dtype=torch.float64)
    first = torch.zeros(slots, N, R)
    ids = torch.arange(M) % slots
    value = torch.zeros(slots, R, dtype=torch.float64)
    for s in range(slots):
        a, b, c = triples(R, g)
        worst = torch.arange(R) % 2 == 0
        a, b, c = [torch.where(worst, torch.tensor(float(v)), t) for v, t in ((128, a), (255, b), (255, c))]
        first[s, :3] = torch.stack([a, b, c])
        value[s] = a.double() * 2 ** 16 + b.double() * 2 ** 8 + c.double()
        row = s  # the adapter's first
        dY[row, :3] = torch.tensor([2.0 ** 16, 2.0 ** 8, 1.0])
        x = torch.randint(2 ** 23, 2 ** 24, (K,), generator=g).double()
        x[::3] = 128 * 2 ** 16 + 255 * 2 ** 8 + 255
        X[row] = x * torch.where(torch.arange(K) % 5 == 0, -1.0, 1.0)
    cfg = lq.make_adapter_config(N, K, R, slots, "f32")
    pool = (torch.zeros(slots, R, K, dtype=torch.bfloat16, device="cuda"), first.bfloat16().cuda(), torch.full((slots,), R, dtype=torch.int32, device="cuda"),
            torch.ones(slots, device="cuda"))
    plan = lq.lq_adapter_plan(slots, ids.int().cuda())
    inter = torch.empty(lq.lq_adapter_sizes(cfg, M)[0], dtype=torch.uint8, device="cuda")
    Xg, dYg = X.float().cuda(), dY.bfloat16().cuda()
    lq.lq_adapter_fwd(cfg, plan, Xg, *pool, dYg, inter=inter)
    _, dA, _ = lq.lq_adapter_bwd(cfg, plan, Xg, *pool, inter, dYg)
    want = value[:, :, None] * X[:slots][:, None, :]
    off = (dA.double().cpu() - want).abs() / want.abs()
    assert float(off.max()) <= 2.0 ** -23 * (1 + 2.0 ** -5), float(off.max())
