"""Infinities in X, dY, Yin and dXin come out where the formulas have them.  All numbers are positive powers of two (scales of either sign), so that every finite sum is
exact, a product with an infinity is an infinity of a known sign, and the products' terms after the first are mostly zeros (zero times infinity is not a number)."""
import pytest
import torch

from tests.test_gpu_adapter import lq  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")


def powers(shape, lo, hi, g):
    return 2.0 ** torch.randint(lo, hi + 1, shape, generator=g, device="cuda").double()


def formulas(X, Yin, A, B, scales, ids, dY, dXin):
    Y, dX, dA, dB = Yin.clone(), dXin.clone(), torch.zeros_like(A), torch.zeros_like(B)
    for s in range(A.shape[0]):
        m = (ids == s).nonzero()[:, 0]
        if m.numel():
            T, dT = X[m] @ A[s].t(), dY[m] @ B[s]
            Y[m] += scales[s] * (T @ B[s].t())
            dX[m] += scales[s] * (dT @ A[s])
            dA[s], dB[s] = scales[s] * (dT.t() @ X[m]), scales[s] * (dY[m].t() @ T)
    return Y, dX, dA, dB


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,R,slots", [(70, 64, 64, 8, 2), (700, 192, 128, 40, 3), (60, 128, 1088, 72, 40), (300, 320, 64, 128, 1), (9, 64, 192, 24, 12)])
@pytest.mark.parametrize("where", ["X", "dY", "Yin", "dXin", "all"])
def test_infinities(lq, where, M, K, N, R, slots, x):  # noqa: F811
    g = torch.Generator(device="cuda")
    g.manual_seed(M + R)
    d = dict(X=powers((M, K), -1, 1, g), Yin=powers((M, N), -1, 1, g), dY=powers((M, N), -1, 0, g), dXin=powers((M, K), -1, 1, g))
    A, B = powers((slots, R, K), -1, 0, g), powers((slots, N, R), -1, 0, g)
    scales = powers((slots,), -1, 1, g) * torch.where(torch.arange(slots, device="cuda") % 2 == 1, -1.0, 1.0).double()
    ids = torch.arange(M, device="cuda") % (slots + 1) - 1  # (some of none)
    some = torch.randperm(M, generator=g, device="cuda")[:max(2, M // 50)]
    for k in ("X", "dY", "Yin", "dXin") if where == "all" else (where,):
        d[k][some, torch.randint(0, d[k].shape[1], (len(some),), generator=g, device="cuda")] = INF
    want = formulas(d["X"], d["Yin"], A, B, scales, ids, d["dY"], d["dXin"])
    dt = torch.float32 if x == "f32" else torch.bfloat16
    X, dXin, Yin, dY = d["X"].to(dt), d["dXin"].to(dt), d["Yin"].bfloat16(), d["dY"].bfloat16()
    cfg = lq.make_adapter_config(N, K, R, slots, x)
    plan = lq.lq_adapter_plan(slots, ids.int())
    pool = (A.bfloat16(), B.bfloat16(), torch.full((slots,), R, dtype=torch.int32, device="cuda"), scales.float())
    inter = torch.empty(lq.lq_adapter_sizes(cfg, M)[0], dtype=torch.uint8, device="cuda")
    got = [lq.lq_adapter_fwd(cfg, plan, X, *pool, Yin, inter=inter), *lq.lq_adapter_bwd(cfg, plan, X, *pool, inter, dY, dXin=dXin)]
    for name, a, b in zip(("Y", "dX", "dA", "dB"), got, want):
        same = (a == b.to(a.dtype)) | (torch.isnan(a) & torch.isnan(b))  # (Yin and the adapter's product of opposite infinities: not a number)
        assert same.all(), f"{name}: {int((~same).sum())} of {same.numel()} differ, {int(torch.isnan(a).sum())} not a number for {int(torch.isnan(b).sum())}"
