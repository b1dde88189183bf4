"""Layouts of outputs between those of rows and of heads: what lies apart is taken, however it is interleaved, and inputs may repeat."""
import pytest
import torch

from tests.test_gpu_qk import EPS, lq, make  # noqa: F401  (lq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,H,ld,hs", [(3, 2, 16, 48), (2, 2, 64, 48), (3, 4, 80, 48), (4, 3, 48, 208), (1, 3, 0, 16), (5, 1, 16, 0), (6, 4, 64, 16), (6, 4, 16, 96)])
def test_interleaved_outputs(lq, M, H, ld, hs):  # noqa: F811
    """(3, 4, 80, 48): tokens at 0, 80, 160 and heads at 0, 48, 96, 144 values share none, though neither encloses the other."""
    D, pairs = 16, (4, 4)
    d = make(M, H, H, D, pairs, "bf16", seed=M + H)
    cfg = lq.make_qk_config(H, H, D, pairs, "half", True, EPS)
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    want = lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], *at)
    grads = lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"])
    big = [torch.full(((M - 1) * ld + (H - 1) * hs + D,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    out = [b.as_strided((M, H, D), (ld, hs, 1)) for b in big]
    lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], *at, qo=out[0], ko=out[1])
    lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"], dq=out[2], dk=out[3])
    for a, b in zip((*want, grads[0], grads[1]), out):
        assert torch.equal(a, b)


def test_a_key_head_shared_by_several(lq):  # noqa: F811
    """An expanded input (stride 0 over heads) with an output of its own for every head; the same tensor as output is refused."""
    M, H, D, pairs = 40, 4, 32, (8, 8)
    d = make(M, H, 1, D, pairs, "bf16", seed=2)
    k = d["k"].expand(M, H, D)
    cfg = lq.make_qk_config(H, H, D, pairs, "adjacent", True, EPS)
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    _, ko = lq.lq_qk_norm_rope_fwd(cfg, d["q"], k, *at)
    _, one = lq.lq_qk_norm_rope_fwd(lq.make_qk_config(H, 1, D, pairs, "adjacent", True, EPS), d["q"], d["k"], *at)
    assert torch.equal(ko, one.expand(M, H, D))
    for kw in (dict(ko=k), dict(ko=torch.empty_like(d["k"]).expand(M, H, D)), dict(qo=torch.empty(1, H, D, dtype=torch.bfloat16, device="cuda").expand(M, H, D))):
        with pytest.raises(lq.LqError) as e:
            lq.lq_qk_norm_rope_fwd(cfg, d["q"], k, *at, **kw)
        assert e.value.status == lq.LQ_ERR_SHAPE
