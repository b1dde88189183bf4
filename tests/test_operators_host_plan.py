"""What the check of a plan refuses before it reads anything.  No device."""
from paper_2604_18117_amd import binding as lq

PTR, BIG = 1 << 20, 1 << 50


def test_verify_plan_arguments():
    f = lq.raw().lq_adapter_verify_plan
    need = lq.lq_adapter_plan_sizes(10, 4)
    for M, slots in ((-1, 4), ((1 << 24) + 1, 4), (10, 0), (10, 1025)):
        assert f(slots, M, PTR, BIG, None) == lq.LQ_ERR_SHAPE
    assert f(4, 10, None, BIG, None) == lq.LQ_ERR_NULL
    assert f(4, 10, PTR + 128, BIG, None) == lq.LQ_ERR_ALIGN
    assert f(4, 10, PTR, need - 1, None) == lq.LQ_ERR_BUFFER_TOO_SMALL
