"""Gradients of the norms before and after a block where tensors are missing or not wanted, and where rows cannot be read four values at a time, at widths of one to five vectors a
lane and of several wavefronts: the kernels that these calls take are others than those of whole calls.  Against the plain 64-bit implementation."""
import ctypes as C

import pytest
import torch

from tests import blocks_ref as ref
from tests.test_gpu_block_norm import EPS, GRADS, backward, check_all, config, forward, make

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]
WIDTHS = [600, 883, 1021, 1152, 1153, 1279, 2239, 2240, 4607]
MISSING = [("dho",), ("dx",), ("y",), ("y", "dho"), ("y", "dx")]


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def cuts(M):
    return [2, M // 4, M // 4, M // 2 + 1, M - 3]


def gradients(d, post, pre, alpha):
    return ref.block_bwd(d["h"], d["y"], d["offsets"], d["gate"], d["scale"], d["w_post"], d["w_pre"], d["dho"], d["dx"], post, pre, EPS, alpha, d["h"].dtype,
                         d["yt"])


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "layer"), ("layer", "rms")])
@pytest.mark.parametrize("M", [50, 1300])
@pytest.mark.parametrize("D", WIDTHS)
def test_gradients_without_a_tensor(lq, D, M, post, pre, stream, branch):
    d = make(M, D, cuts(M), stream, branch, seed=D)
    cfg = config(lq, d, post, pre, 0.75)
    for keys in MISSING:
        e = dict(d, yt=d["y"].dtype, **{k: None for k in keys})
        keep = dict(dh=torch.full_like(d["h"], 7.0), dy=None if e["y"] is None else torch.full_like(d["y"], 7.0))
        got = dict(zip(GRADS, backward(lq, cfg, e, **keep)))
        want = gradients(e, post, pre, 0.75)
        rows = want["rows"]
        others = torch.ones(M, dtype=torch.bool, device="cuda")
        others[rows] = False
        for k in GRADS:
            if k in ("dh", "dy") and got[k] is not None:
                ref.check(got[k][rows], want[k], f"{k} without {keys}")
                assert (got[k][others] == 7.0).all(), (k, keys)
            elif k in want and got[k] is not None:
                ref.check(got[k], want[k], f"{k} without {keys}")
            elif got[k] is not None:
                assert (got[k] == 0).all(), (k, keys)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("D", [600, 1152, 1153, 2240])
@pytest.mark.parametrize("M", [50, 1300])
def test_gradients_that_are_not_wanted(lq, M, D, stream, branch):
    """dh, dy or sums left out, through the C interface."""
    d = make(M, D, cuts(M), stream, branch, seed=D)
    cfg = config(lq, d, "rms", "layer", 0.75)
    S = len(cuts(M)) - 1
    whole = dict(zip(GRADS, backward(lq, cfg, d, dh=torch.full_like(d["h"], 7.0), dy=torch.full_like(d["y"], 7.0))))
    p = lambda t: t.data_ptr()  # noqa: E731
    mod = lambda t: lq.lq_mod(None, 0) if t is None else lq.lq_mod(p(t), t.stride(0))  # noqa: E731
    work = torch.empty(lq.lq_block_work_sizes(cfg, M, S), dtype=torch.uint8, device="cuda")
    for left in (("dh",), ("dy",), ("dh", "dy"), ("dgate", "dscale", "dshift", "dw_post", "dw_pre"), ("dgate", "dw_pre"), ("dh", "dscale", "dshift", "dw_post")):
        o = {k: None if k in left else torch.full_like(t, 7.0) for k, t in whole.items()}
        out = lq.lq_block_grads(None if o["dh"] is None else p(o["dh"]), D, None if o["dy"] is None else p(o["dy"]), D, mod(o["dgate"]), mod(o["dscale"]), mod(o["dshift"]),
                                None if o["dw_post"] is None else p(o["dw_post"]), None if o["dw_pre"] is None else p(o["dw_pre"]))
        st = lq.raw().lq_block_norm_bwd(C.byref(cfg), p(d["h"]), D, p(d["y"]), D, p(d["offsets"]), S, C.byref(mod(d["gate"])), C.byref(mod(d["scale"])), p(d["w_post"]),
                                        p(d["w_pre"]), p(d["dho"]), D, p(d["dx"]), D, C.byref(out), M, p(work), work.numel(), torch.cuda.current_stream().cuda_stream)
        assert st == lq.LQ_OK
        want = gradients(dict(d, yt=d["y"].dtype), "rms", "layer", 0.75)
        for k, t in o.items():
            if t is None:
                continue
            if k in ("dh", "dy"):
                ref.check(t[want["rows"]], want[k], f"{k} without {left}")
                assert (t[:2] == 7.0).all() and (t[M - 3:] == 7.0).all(), (k, left)
            else:
                ref.check(t, want[k], f"{k} without {left}")


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms"), ("layer", "layer")])
@pytest.mark.parametrize("M", [50, 1300])
@pytest.mark.parametrize("D", [515, 770, 883, 1021, 1153, 1279, 1527, 2239, 3601, 10241])
def test_odd_widths(lq, D, M, post, pre, stream, branch):
    M = M if D < 4000 else min(M, 700)
    check_all(lq, make(M, D, cuts(M), stream, branch, seed=D), post, pre, alpha=0.75)


@pytest.mark.parametrize("stream,branch", TYPES)
@pytest.mark.parametrize("D", [1152, 2240])
def test_rows_at_odd_places(lq, D, stream, branch):
    """Rows of a width that is a multiple of four, one value from an aligned place: the kernels of any alignment with no row's end among four values."""
    M = 600
    d = make(M, D, cuts(M), stream, branch, seed=D)

    def moved(t):
        big = torch.full((M, D + 1), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 1:] = t
        return big[:, 1:]
    check_all(lq, dict(d, **{k: moved(d[k]) for k in ("h", "y", "dx", "dho")}), "rms", "layer", 0.75)


@pytest.mark.parametrize("mods", [("gate", "scale", "shift"), ()])
@pytest.mark.parametrize("D", [200, 1152, 1153])
@pytest.mark.parametrize("M", [40, 600])
def test_without_a_branch_there_is_no_residual_scale(lq, M, D, mods):
    """Without y the sum is h itself, whatever res_scale is, and the gradient with respect to h is not scaled either: the first norm of a model with the configuration of the others."""
    d = dict(make(M, D, cuts(M), "f32", "bf16", seed=D, mods=mods), y=None)
    cfg = lq.make_block_config(D, "rms", "layer", EPS, 0.5, "f32", "bf16")
    none, x = forward(lq, cfg, d)
    want = ref.block_fwd(d["h"], None, d["offsets"], d["gate"], d["scale"], d["shift"], d["w_post"], d["w_pre"], "rms", "layer", EPS, 1.0, torch.bfloat16)
    rows = want["rows"]
    assert none is None
    ref.check(x[rows], want["x"], "x")
    for keys in ((), ("dho",), ("dx",)):
        e = dict(d, yt=torch.bfloat16, **{k: None for k in keys})
        got, grads = dict(zip(GRADS, backward(lq, cfg, e))), gradients(e, "rms", "layer", 1.0)
        ref.check(got["dh"][rows], grads["dh"], f"dh without {keys}")
        assert got["dy"] is None and got["dgate"] is None and got["dw_post"] is None


def exact_rows(M, D, mean, seed):
    """fp32 rows of whole numbers whose sums, means and differences from the mean are all exact in 24 bits: M x D (a power of two, so that the mean is the sum times one), deviations
    around 1."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn(M, D, generator=g, device="cuda") * 1.5).round() + mean
    assert D & (D - 1) == 0 and float(x.abs().sum(1).max()) < 2 ** 24
    return x


@pytest.mark.parametrize("D", [256, 1024, 2048])
def test_variance_of_rows_with_a_large_mean(lq, D):
    """Differences from the mean being exact, 1 / deviation is off by half of what a sum of D squares can be in any order, (D + 8) 2^-24, and by the root, the division and the mean of the
    squares, 4 2^-24; the row by one product more, and its rounding.  (Squares less the mean's square are off by 4096^2 2^-24 of variances around 2.)"""
    M, e = 9, 2.0 ** -24
    rel = (0.5 * (D + 8) + 6) * e
    h, y = exact_rows(M, D, 4096.0, D), exact_rows(M, D, -4096.0, D + 1)

    def normed(x):
        x = x.double()
        x = x - x.mean(1, keepdim=True)
        r = 1.0 / (x.square().mean(1, keepdim=True) + EPS).sqrt()
        return x * r, r
    cfg = lq.make_block_config(D, "none", "layer", EPS, 1.0, "f32", "f32")
    (n, r), (p, ry) = normed(h), normed(y)
    _, x = lq.lq_block_norm_fwd(cfg, h)
    assert ((x.double() - n).abs() <= (rel + 2 * e) * n.abs()).all()
    both = lq.make_block_config(D, "layer", "none", EPS, 1.0, "f32", "f32")
    ho, _ = lq.lq_block_norm_fwd(both, torch.zeros_like(h), y)
    assert ((ho.double() - p).abs() <= (rel + 2 * e) * p.abs()).all()
    # gradients: of h through the first norm, of y through the second
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    d = torch.randn(M, D, generator=g, device="cuda")
    for name, got, v, s in (("dh", lq.lq_block_norm_bwd(cfg, h, None, dx=d)[0], n, r), ("dy", lq.lq_block_norm_bwd(both, torch.zeros_like(h), y, dho=d)[1], p, ry)):
        value, off = ref.norm_grad("layer", v, s, rel * v.abs(), torch.full_like(s, rel), d.double(), torch.zeros_like(v))
        ref.check(got, ref.rounded(value, off, torch.float32), name)
