"""Norm and rotation of batches large enough for several tokens to a workgroup, against the plain 64-bit implementation."""
import ctypes as C

import pytest
import torch

from tests import operators_ref as ref
from tests.operator_forms import TOKENS
from tests.test_gpu_qk import EPS, lq, make  # noqa: F401  (lq is a fixture)

pytestmark = pytest.mark.gpu


def check(d, out, grads, pairs, pairing, norm, kinds):
    for i, name in enumerate("qk"):
        if name not in kinds:
            continue
        x, w, dy = d[name], d["w" + name], d[f"d{name}o"]
        ref.check(out[i], ref.qk_fwd(x, w, d["pos"], d["inv_freq"], pairs, pairing, norm, EPS), name)
        # (a workgroup of the gradient adds up to 35 tokens of a head, 512 of them 64 at a time: below the 512 additions of the bound)
        dx, dw = ref.qk_bwd(x, w, d["pos"], d["inv_freq"], pairs, pairing, norm, EPS, dy)
        ref.check(grads[i], dx, "d" + name)
        if norm:
            ref.check(grads[2 + i], dw, "dw" + name)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "adjacent"])
@pytest.mark.parametrize("M,Hq,Hk,D,pairs,rows", TOKENS)
def test_several_tokens_to_a_workgroup(lq, M, Hq, Hk, D, pairs, rows, pairing, x):  # noqa: F811
    d = make(M, max(Hq, 1), max(Hk, 1), D, pairs, x, seed=M + D, pos_rows=rows, layout="fused" if M == 3000 else "dense")
    kinds = "q" * (Hq > 0) + "k" * (Hk > 0)
    for norm in (True, False):
        cfg = lq.make_qk_config(Hq, Hk, D, pairs, pairing, norm, EPS, x)
        a = [d["q"] if Hq else None, d["k"] if Hk else None]
        g = [d["dqo"] if Hq else None, d["dko"] if Hk else None]
        at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
        check(d, lq.lq_qk_norm_rope_fwd(cfg, *a, *at), lq.lq_qk_norm_rope_bwd(cfg, *a, *at, *g), pairs, pairing, norm, kinds)


def test_gradient_without_those_of_the_weights(lq):  # noqa: F811
    """Both dw NULL through the C ABI: the same dq and dk, no workspace."""
    M, H, D, pairs = 700, 3, 48, (12, 12)
    d = make(M, H, H, D, pairs, "bf16", seed=3)
    cfg = lq.make_qk_config(H, H, D, pairs, "half", True, EPS)
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    want = lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"])
    out = [torch.full((M, H, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    h = [C.byref(lq.lq_heads(t.data_ptr(), H * D, D)) for t in (d["q"], d["k"], d["dqo"], d["dko"], *out)]
    st = lq.raw().lq_qk_norm_rope_bwd(C.byref(cfg), h[0], h[1], at[0].data_ptr(), at[1].data_ptr(), at[2].data_ptr(), M, at[3].data_ptr(), h[2], h[3], h[4], h[5], None, None,
                                      M, None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == lq.LQ_OK
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_gradient_with_offsets_past_32_bits(lq, x):  # noqa: F811
    """Tokens 2^21 values apart, inputs and derivatives; dq and dk in place."""
    M, H, D, pairs = 1100, 2, 16, (4, 4)
    d = make(M, H, H, D, pairs, x, seed=1)
    cfg = lq.make_qk_config(H, H, D, pairs, "half", True, EPS, x)
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    far = []
    for a, b in (("q", "k"), ("dqo", "dko")):
        big = torch.empty((M << 21) + 64, dtype=d["q"].dtype, device="cuda")
        far += [big.as_strided((M, H, D), (1 << 21, D, 1)), big.as_strided((M, H, D), (1 << 21, D, 1), H * D)]
        far[-2].copy_(d[a])
        far[-1].copy_(d[b])
    want = lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"])
    got = lq.lq_qk_norm_rope_bwd(cfg, far[0], far[1], *at, far[2], far[3], dq=far[2], dk=far[3])
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    check(d, lq.lq_qk_norm_rope_fwd(cfg, far[0], far[1], *at), got, pairs, "half", True, "qk")


@pytest.mark.parametrize("M", [64, 256, 512, 4096])
def test_sums_of_the_weights_gradients_lose_little(lq, M):  # noqa: F811
    """Heads of ones have a norm of one, so that dw is the sum of the derivatives: 2^24, then ones.  An addition to 2^24 is off by at most 1; a value goes through at most
    8 of them in a workgroup, 8 of workgroups' sums in a share and 6 where the shares are joined."""
    cfg = lq.make_qk_config(1, 1, 2, (), "half", True, 1e-12, "f32")
    x, dy = torch.ones(M, 1, 2, device="cuda"), torch.ones(M, 1, 2, device="cuda")
    dy[0] = 2.0 ** 24
    _, _, dwq, dwk = lq.lq_qk_norm_rope_bwd(cfg, x, x, None, None, None, None, dy, dy)
    for dw in (dwq, dwk):
        assert float((dw.double() - (2.0 ** 24 + M - 1)).abs().max()) <= 8 + 8 + 6, dw
