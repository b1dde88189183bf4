"""A plan belongs to its number of rows and its pool: calls with another one, or with memory in which no plan was made, write nothing (the plans' rows and tiles would
lie elsewhere, and be read as numbers past the batch's)."""
import pytest
import torch

from tests import operators_ref as ref
from tests.test_gpu_adapter import compare, lq, make, pool, run  # noqa: F401  (lq is a fixture)

pytestmark = pytest.mark.gpu
BIG = 1 << 23  # bytes: a plan of any of the batches below


def _stale(lq, slots, M, plan):  # noqa: F811
    try:
        lq.lq_adapter_verify_plan(slots, M, plan)
    except lq.LqError as e:
        return e.status == lq.LQ_ERR_STALE_BLOB
    return False


def buffers(lq, cfg, d):  # noqa: F811
    M, K = d["X"].shape
    inter, work = lq.lq_adapter_sizes(cfg, M)
    five = dict(device="cuda")
    return dict(Y=torch.full((M, cfg.N), 5.0, dtype=torch.bfloat16, **five), inter=torch.full((inter,), 5, dtype=torch.uint8, **five),
                dX=torch.full((M, K), 5.0, dtype=d["X"].dtype, **five), dA=torch.full(d["A"].shape, 5.0, **five), dB=torch.full(d["B"].shape, 5.0, **five),
                work=torch.full((work,), 5, dtype=torch.uint8, **five))


def call(lq, cfg, d, plan, b):  # noqa: F811
    lq.lq_adapter_fwd(cfg, plan, d["X"], *pool(d), d["Yin"], Y=b["Y"], inter=b["inter"])
    lq.lq_adapter_bwd(cfg, plan, d["X"], *pool(d), b["inter"], d["dY"], dXin=d["dXin"], dX=b["dX"], dA=b["dA"], dB=b["dB"], work=b["work"])
    torch.cuda.synchronize()


# (rows, K, N, rank, slots) of the call; (rows, slots) of the plan in its buffer
@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,R,slots,made", [
    (200, 128, 192, 24, 4, (100, 4)), (100, 128, 192, 24, 4, (200, 4)), (200, 128, 192, 24, 4, (200, 7)), (130, 128, 1088, 40, 70, (130, 71)), (130, 128, 1088, 40, 70, (9000, 70)),
    (9000, 64, 128, 8, 3, (130, 3)), (9000, 64, 128, 8, 3, (9000, 2)), (1, 64, 64, 8, 1, (2, 1)), (40, 64, 128, 96, 300, (41, 300))])
def test_another_batchs_plan(lq, M, K, N, R, slots, made, x):  # noqa: F811
    d = make(M, K, N, R, slots, x, seed=M + slots)
    cfg = lq.make_adapter_config(N, K, R, slots, x)
    plan = torch.zeros(BIG, dtype=torch.uint8, device="cuda")
    ids = torch.arange(made[0], dtype=torch.int32, device="cuda") % made[1]
    lq.lq_adapter_plan(made[1], ids, plan=plan)
    lq.lq_adapter_verify_plan(made[1], made[0], plan)
    assert _stale(lq, slots, M, plan)
    b = buffers(lq, cfg, d)
    call(lq, cfg, d, plan, b)
    for k, t in b.items():
        assert (t == 5).all(), k
    lq.lq_adapter_plan(slots, d["ids"], plan=plan)  # the same buffer with the batch's own plan
    lq.lq_adapter_verify_plan(slots, M, plan)
    call(lq, cfg, d, plan, b)
    compare(d, [b[k] for k in ("Y", "dX", "dA", "dB")], what="after its own plan")


@pytest.mark.parametrize("fill", [0, 0xFF, 1])
def test_no_plan_at_all(lq, fill):  # noqa: F811
    d = make(300, 128, 192, 24, 5, "bf16", seed=1)
    cfg = lq.make_adapter_config(192, 128, 24, 5)
    plan = torch.full((BIG,), fill, dtype=torch.uint8, device="cuda")
    assert _stale(lq, 5, 300, plan)
    b = buffers(lq, cfg, d)
    call(lq, cfg, d, plan, b)
    for k, t in b.items():
        assert (t == 5).all(), k


def test_a_blob_of_another_kind(lq):  # noqa: F811
    """An activation blob has the same header with another kind."""
    d = make(300, 128, 192, 24, 5, "bf16", seed=1)
    cfg = lq.make_adapter_config(192, 128, 24, 5)
    icfg = lq.make_config(192, 128, 32, "int", 64, 8, 8)
    packed = lq.lq_pack_weights(icfg, torch.ones(192, 128, device="cuda"), torch.ones(192, 32, device="cuda"), torch.ones(32, 128, device="cuda"))
    blob = torch.zeros(BIG, dtype=torch.uint8, device="cuda")
    lq.lq_quantize_act(icfg, packed, d["X"], act=blob)
    assert _stale(lq, 5, 300, blob)
    b = buffers(lq, cfg, d)
    call(lq, cfg, d, blob, b)
    for k, t in b.items():
        assert (t == 5).all(), k
