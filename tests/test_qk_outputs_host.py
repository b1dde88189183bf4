"""Outputs of the norm and rotation whose heads share values are refused (several threads would write them, in any order).  No device: what is refused launches nothing."""
import pytest

from paper_2604_18117_amd import binding as lq
from tests.test_operators_host import PTR, _qcfg, _qk


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("which", ["o0", "o1"])
@pytest.mark.parametrize("ld,hs", [(256, 0), (0, 64), (0, 0), (256, 63), (63, 640), (64, 64), (128, 64), (191, 64), (64, 128), (64, 639), (100, 164), (1 << 39, 32), (200, 720)])
def test_heads_that_share_values(ld, hs, which, bwd):
    """4 or 4 heads of 64 values, 10 tokens."""
    cfg = _qcfg(heads_k=4)
    assert _qk(cfg, bwd, **{which: (PTR, ld, hs)}) == lq.LQ_ERR_SHAPE


@pytest.mark.parametrize("bwd", [False, True])
def test_one_token_or_one_head(bwd):
    """The stride of a single one says nothing; the other one counts."""
    assert _qk(_qcfg(), bwd, M=1, o0=(PTR, 0, 63)) == lq.LQ_ERR_SHAPE
    assert _qk(_qcfg(heads_q=1, heads_k=1), bwd, o0=(PTR, 63, 0)) == lq.LQ_ERR_SHAPE
