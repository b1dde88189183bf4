"""The forms of the adapters' products that only large or deep batches take, against the plain 64-bit implementation."""
import pytest
import torch

from tests import operators_ref as ref
from tests.operator_forms import DEEP, WIDE_BACKWARD, WIDE_FORWARD
from tests.test_gpu_adapter import compare, lq, make, pool, run  # noqa: F401  (lq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,N,R,slots", WIDE_FORWARD)
def test_forward_of_several_pieces(lq, M, K, N, R, slots):  # noqa: F811
    """Rows of every adapter, of one of rank 0 and of none; into another tensor with gaps between its rows, and in place."""
    d = make(M, K, N, R, slots, "bf16", seed=R, pad=8)
    cfg = lq.make_adapter_config(N, K, R, slots)
    plan = lq.lq_adapter_plan(slots, d["ids"])
    big = torch.full((M, N + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    Y = lq.lq_adapter_fwd(cfg, plan, d["X"], *pool(d), d["Yin"], Y=big[:, 16:N + 16])
    ref.check(Y, ref.adapter_fwd(d["X"], d["Yin"], *pool(d), d["ids"]), "Y")
    assert (big[:, :16] == 7).all() and (big[:, N + 16:] == 7).all()
    lq.lq_adapter_fwd(cfg, plan, d["X"], *pool(d), d["Yin"], Y=d["Yin"])
    assert torch.equal(d["Yin"], Y)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,R,slots", WIDE_BACKWARD)
def test_backward_of_several_pieces(lq, M, K, N, R, slots, x):  # noqa: F811
    d = make(M, K, N, R, slots, x, seed=R + 1, pad=8)
    a = run(lq, d, x)
    compare(d, a, what="several pieces")
    for p, q in zip(a, run(lq, d, x, in_place=True)):
        assert torch.equal(p, q)
    compare(d, run(lq, d, x, dxin=False), dxin=False, what="no dXin")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M,depth,R,slots", DEEP)
def test_deep_products_of_few_rows(lq, M, depth, R, slots, x):  # noqa: F811
    """Both factors' products: X A^T over `depth`, then dY B over it."""
    for K, N in ((depth, 128), (128, depth)):
        d = make(M, K, N, R, slots, x, seed=M, ranks="full")
        compare(d, run(lq, d, x), what=f"{K} -> {N}")


def test_offsets_past_32_bits_in_fp32(lq):  # noqa: F811
    """fp32 rows 2^20 values apart: bytes past 2^32 in X, dXin and dX."""
    M, K, N, R = 2200, 64, 128, 8
    d = make(M, K, N, R, 2, "f32", seed=7, ids=torch.arange(M) % 3)
    e = dict(d)
    for k in ("X", "dXin"):
        big = torch.empty((M << 20) + K, device="cuda").as_strided((M, K), (1 << 20, 1))
        big.copy_(d[k])
        e[k] = big
    cfg = lq.make_adapter_config(N, K, R, 2, "f32")
    plan = lq.lq_adapter_plan(2, e["ids"])
    inter = torch.empty(lq.lq_adapter_sizes(cfg, M)[0], dtype=torch.uint8, device="cuda")
    Y = lq.lq_adapter_fwd(cfg, plan, e["X"], *pool(e), e["Yin"], inter=inter)
    dX, dA, dB = lq.lq_adapter_bwd(cfg, plan, e["X"], *pool(e), inter, e["dY"], dXin=e["dXin"], dX=e["dXin"])
    compare(d, (Y, dX, dA, dB), what="far rows")
