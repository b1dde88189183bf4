"""The example's own checks.  No device: the batch is refused before anything is called."""
import pytest
import torch

from paper_2604_18117_amd import adapted_qkv as ex


@pytest.mark.parametrize("grouped", [None, 5, 2])
def test_a_batch_that_was_not_grouped_is_refused(monkeypatch, grouped):
    def nothing(*a, **k):
        raise AssertionError("reached the library")
    for name in ("lq_quantize_act", "lq_linear_lowrank_fwd", "lq_adapter_fwd", "lq_qk_norm_rope_fwd", "lq_qk_norm_rope_bwd", "lq_adapter_bwd"):
        monkeypatch.setattr(ex.lq, name, nothing)
    monkeypatch.setattr(ex.lq, "lq_adapter_plan", lambda *a, **k: None)
    m = object.__new__(ex.AdaptedQKV)
    m.dim, m.heads, m.head_dim = 16, 2, 8
    m.cfg = m.packed = m.act = m.plan = m.inter = m.work = m.A = m.B = m.ranks = m.scales = m.qk = m.wq = m.wk = m.inv_freq = None
    m.adapters = ex.lq.make_adapter_config(64, 64, 8, 2)
    m.rows = None
    if grouped is not None:
        m.group(torch.zeros(grouped, dtype=torch.int32))
    X, rows, pos = torch.zeros(3, 16), torch.zeros(3, 48), torch.zeros(3, 2)
    for call in (lambda: m.project(X), lambda: m(X, pos), lambda: m.backward(X, rows, pos, rows)):
        with pytest.raises(ValueError, match="3 rows"):
            call()


def test_a_plan_that_failed_is_none(monkeypatch):
    def fail(*a, **k):
        raise ex.lq.LqError(ex.lq.LQ_ERR_BUFFER_TOO_SMALL, "lq_adapter_plan")
    m = object.__new__(ex.AdaptedQKV)
    m.adapters, m.plan, m.rows = ex.lq.make_adapter_config(64, 64, 8, 2), None, 3
    monkeypatch.setattr(ex.lq, "lq_adapter_plan", fail)
    with pytest.raises(ex.lq.LqError):
        m.group(torch.zeros(4, dtype=torch.int32))
    assert m.rows is None
