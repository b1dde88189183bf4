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
