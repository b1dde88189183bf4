"""Norms before and after a block with its gate, residual scale and modulation (lq_block_norm_fwd, lq_block_norm_bwd) against the plain 64-bit implementation."""
import pytest
import torch

from tests import blocks_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def make(M, D, offsets=None, stream="bf16", branch="bf16", weights=True, seed=0, mods=("gate", "scale", "shift")):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    S = 1 if offsets is None else len(offsets) - 1
    rows = normal(S, 6 * D) * 0.3
    d = dict(h=(normal(M, D) * 2 + 0.7).to(DT[stream]), y=(normal(M, D) + 0.2).to(DT[branch]), dx=(normal(M, D) * 0.1).to(DT[branch]),
             dho=(normal(M, D) * 0.1).to(DT[stream]), offsets=None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    d.update({k: rows[:, i * D:(i + 1) * D] if k in mods else None for i, k in enumerate(("shift", "scale", "gate"))})
    d["w_post"], d["w_pre"] = (1 + 0.2 * normal(D), 1 + 0.2 * normal(D)) if weights else (None, None)
    return d


def config(lq, d, post, pre, alpha=1.0):
    names = {v: k for k, v in DT.items()}
    return lq.make_block_config(d["h"].shape[1], post, pre, EPS, alpha, names[d["h"].dtype], names[d["y"].dtype])


def forward(lq, cfg, d, **kw):
    return lq.lq_block_norm_fwd(cfg, d["h"], d["y"], d["offsets"], d["gate"], d["scale"], d["shift"], d["w_post"], d["w_pre"], **kw)


def backward(lq, cfg, d, **kw):
    return lq.lq_block_norm_bwd(cfg, d["h"], d["y"], d["offsets"], d["gate"], d["scale"], d["w_post"], d["w_pre"], d["dho"], d["dx"], **kw)


GRADS = ("dh", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre")


def check_all(lq, d, post="none", pre="layer", alpha=1.0):
    cfg = config(lq, d, post, pre, alpha)
    M, D = d["h"].shape
    keep = [torch.full((M, D), 7.0, dtype=d[k].dtype, device="cuda") for k in ("h", "y", "h", "y")]
    ho, x = forward(lq, cfg, d, ho=keep[0], x=keep[1])
    want = ref.block_fwd(d["h"], d["y"], d["offsets"], d["gate"], d["scale"], d["shift"], d["w_post"], d["w_pre"], post, pre, EPS, alpha, d["y"].dtype)
    ref.check(ho[want["rows"]], want["ho"], "ho")
    ref.check(x[want["rows"]], want["x"], "x")
    got = dict(zip(GRADS, backward(lq, cfg, d, dh=keep[2], dy=keep[3])))
    grads = ref.block_bwd(d["h"], d["y"], d["offsets"], d["gate"], d["scale"], d["w_post"], d["w_pre"], d["dho"], d["dx"], post, pre, EPS, alpha, d["h"].dtype, d["y"].dtype)
    for k in GRADS:
        if got[k] is not None:
            ref.check(got[k][grads["rows"]] if k in ("dh", "dy") else got[k], grads[k], k)
    others = torch.ones(M, dtype=torch.bool, device="cuda")
    others[want["rows"]] = False
    for t in keep:  # rows of no sequence stay as they were
        assert (t[others] == 7.0).all()
    again = backward(lq, cfg, d)
    for k, t in zip(GRADS[2:], again[2:]):
        assert (t is None and got[k] is None) or torch.equal(t, got[k]), k
    return got


@pytest.mark.parametrize("stream,branch", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("none", "rms"), ("rms", "rms"), ("layer", "layer"), ("rms", "none"), ("none", "none")])
@pytest.mark.parametrize("D", [1, 7, 64, 264, 1152])
def test_norms_and_types(lq, D, post, pre, stream, branch):
    check_all(lq, make(37, D, [0, 5, 6, 30], stream, branch, seed=D), post, pre, alpha=0.75)


@pytest.mark.parametrize("D", [8, 250, 512, 513, 1024, 1032, 1500, 1537, 2240, 3000, 4100, 4608, 8200, 9000, 16383, 16384])
def test_widths(lq, D):
    check_all(lq, make(11, D, [0, 4, 4, 9], "f32", "bf16", seed=D), "rms", "layer")
    check_all(lq, make(3, D, None, "bf16", "bf16", weights=False, seed=D), "none", "layer")


@pytest.mark.parametrize("D", [72, 1152, 2240, 5000])
@pytest.mark.parametrize("M,offsets", [
    (1, None), (1, [0, 1]), (4, [0, 0, 4]), (9, [0, 9, 9]), (40, [0, 40]), (40, [3, 3, 10, 10, 10, 35]), (2000, [0, 1, 2, 1000, 1999]), (700, list(range(0, 701, 7))),
    (300, list(range(301))), (5000, [17, 2500, 4990]), (130, [130, 130]), (64, [0, 0, 0, 0])])
def test_sequences(lq, M, offsets, D):
    if M * D > 6e6:
        M, offsets = M // 4, [o // 4 for o in offsets]
    check_all(lq, make(M, D, offsets, seed=M), "none", "layer")


@pytest.mark.parametrize("stream,branch", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms"), ("layer", "none")])
@pytest.mark.parametrize("D", [33, 512, 1152, 1528, 2240, 3600, 4608, 12000])
def test_several_rows_to_a_workgroup(lq, D, post, pre, stream, branch):
    """Batches of more than 512 rows: several rows to a group of wavefronts, several groups and sequences to a workgroup."""
    M = 1300 if D < 4000 else 700
    check_all(lq, make(M, D, [3, M // 4, M // 4 + 1, M // 4 + 1, M // 2 + 7, M - 10], stream, branch, seed=D), post, pre, alpha=0.75)


@pytest.mark.parametrize("D", [200, 1152, 2240, 5000])
def test_several_rows_to_a_workgroup_in_place(lq, D):
    d = make(1100, D, [0, 20, 555, 1090], "bf16", "bf16")
    cfg = config(lq, d, "rms", "layer", 0.5)
    want = backward(lq, cfg, d, dh=d["dho"].clone(), dy=d["dx"].clone())
    e = dict(d, dho=d["dho"].clone(), dx=d["dx"].clone())
    for a, b in zip(backward(lq, cfg, e, dh=e["dho"], dy=e["dx"]), want):
        assert torch.equal(a, b)


def test_many_sequences(lq):
    g = torch.Generator()
    g.manual_seed(0)
    cuts = sorted(torch.randint(0, 9001, (4999,), generator=g).tolist())
    check_all(lq, make(9000, 40, [0] + cuts + [9000], "f32", "f32"), "layer", "rms")


@pytest.mark.parametrize("mods", [(), ("gate",), ("scale", "shift"), ("shift",)])
def test_parts_that_are_not_there(lq, mods):
    for weights in (False, True):
        d = make(50, 200, [0, 20, 50], mods=mods, weights=weights)
        check_all(lq, d, "rms", "layer")
    cfg = config(lq, d, "rms", "layer")
    # an output that is not wanted, a derivative that is not there
    ho, x = forward(lq, cfg, d, last=True)
    assert x is None and torch.equal(ho, forward(lq, cfg, d)[0])
    plain = dict(d, y=None)
    none, x = forward(lq, cfg, plain)
    want = ref.block_fwd(d["h"], None, d["offsets"], d["gate"], d["scale"], d["shift"], d["w_post"], d["w_pre"], "rms", "layer", EPS, 1.0, d["y"].dtype)
    assert none is None
    ref.check(x, want["x"], "x without a branch")
    for keys in (("dho",), ("dx",), ("y",), ("y", "dho"), ("y", "dx")):
        e = dict(d, **{k: None for k in keys})
        got = dict(zip(GRADS, backward(lq, cfg, e)))
        grads = ref.block_bwd(e["h"], e["y"], e["offsets"], e["gate"], e["scale"], e["w_post"], e["w_pre"], e["dho"], e["dx"], "rms", "layer", EPS, 1.0, e["h"].dtype,
                              d["y"].dtype)
        for k in GRADS:
            if k in grads:
                assert got[k] is None or not torch.isnan(got[k]).any()
                if got[k] is not None:
                    ref.check(got[k], grads[k], k)
            elif got[k] is not None:
                assert (got[k] == 0).all(), k  # (no derivative comes through that part)


@pytest.mark.parametrize("D", [64, 100, 1152, 2240])
def test_in_place(lq, D):
    d = make(60, D, [0, 20, 55], "bf16", "bf16")
    cfg = config(lq, d, "rms", "layer", 0.5)
    ho, x = forward(lq, cfg, d, ho=d["h"].clone(), x=d["y"].clone())
    e = dict(d, h=d["h"].clone(), y=d["y"].clone())
    forward(lq, cfg, e, ho=e["h"], x=e["y"])
    assert torch.equal(e["h"], ho) and torch.equal(e["y"], x)
    want = backward(lq, cfg, d, dh=d["dho"].clone(), dy=d["dx"].clone())
    e = dict(d, dho=d["dho"].clone(), dx=d["dx"].clone())
    got = backward(lq, cfg, e, dh=e["dho"], dy=e["dx"])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D,pad", [(64, 1), (64, 8), (1152, 4), (1152, 2240), (33, 3)])
def test_rows_that_lie_apart(lq, D, pad):
    M, S = 23, 3
    d = make(M, D, [0, 9, 9, 21], "f32", "bf16")
    cfg = config(lq, d, "layer", "rms")
    want, grads = forward(lq, cfg, d), backward(lq, cfg, d)

    def apart(t, rows, fill=float("nan")):
        big = torch.full((rows, D + pad), fill, dtype=t.dtype, device="cuda")
        big[:, pad:].copy_(t)
        return big[:, pad:]
    e = {k: apart(v, v.shape[0]) if v is not None and v.dim() == 2 else v for k, v in d.items()}
    outs = [apart(torch.full((n, D), 7.0, device="cuda").to(dt), n, 7.0) for n, dt in ((M, DT["f32"]), (M, DT["bf16"]), (M, DT["f32"]), (M, DT["bf16"]), (S, DT["f32"]), (S, DT["f32"]), (S, DT["f32"]))]
    ho, x = forward(lq, cfg, e, ho=outs[0], x=outs[1])
    got = backward(lq, cfg, e, **dict(zip(GRADS[:5], outs[2:])))
    # (other vectors of columns: another order of a row's sums)
    tol = {torch.bfloat16: 2.0 ** -7, torch.float32: 1e-5}
    for a, b in zip((ho, x) + tuple(got), tuple(want) + tuple(grads)):
        rows = slice(0, 21) if a.dim() == 2 and a.shape[0] == M else slice(None)
        assert torch.allclose(a[rows].double(), b[rows].double(), rtol=tol[a.dtype], atol=tol[a.dtype])
    for t in outs:
        whole = t._base if t._base is not None else t
        assert (whole[:, :pad] == 7.0).all()


@pytest.mark.parametrize("D", [136, 2240])
def test_not_a_number_stays_in_its_row(lq, D):
    d = make(50, D, [0, 10, 30, 48])
    cfg = config(lq, d, "rms", "layer")
    want, grads = forward(lq, cfg, d), backward(lq, cfg, d)
    e = {k: v.clone() if v is not None else None for k, v in d.items()}
    e["h"][12, 3], e["y"][13, 0], e["dx"][14, 5], e["h"][49, 1], e["dho"][49, 1] = float("nan"), float("inf"), float("nan"), float("nan"), float("nan")
    ho, x = forward(lq, cfg, e)
    got = backward(lq, cfg, e)
    fine = torch.ones(48, dtype=torch.bool, device="cuda")
    fine[12:15] = False
    assert torch.equal(ho[:48][fine], want[0][:48][fine]) and torch.equal(x[:48][fine], want[1][:48][fine])
    assert torch.isnan(x[12]).all() and torch.isnan(x[13]).all()
    for a, b in zip(got[:2], grads[:2]):
        assert torch.equal(a[:48][fine], b[:48][fine])
    for a, b in zip(got[2:5], grads[2:5]):
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and torch.isnan(a[1]).any()


@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_rows_of_one_value_and_zeros(lq, pre):
    """No variance (LayerNorm), no values: 1 / sqrt(eps) times nothing."""
    d = make(6, 96, [0, 3, 6], "f32", "f32", mods=("shift",), weights=False)
    d["h"][0], d["h"][1], d["h"][4] = 0.0, 5.0, -3e4
    d["y"].zero_()
    check_all(lq, d, "layer", pre)


def test_a_large_mean_keeps_the_variance(lq):
    """fp32 rows of mean 4096 and deviation 1: squares minus the mean's square would lose it."""
    d = make(8, 1152, None, "f32", "f32")
    d["h"] += 4096.0
    check_all(lq, d, "none", "layer")


def test_offsets_past_32_bits(lq):
    """Rows so far apart that their offsets pass 2^32 values."""
    D, M, far = 64, 3, (1 << 31) + 1024
    big = torch.zeros(2 * far + D, dtype=torch.bfloat16, device="cuda")
    d = make(M, D, [0, 1, 3])
    cfg = config(lq, d, "none", "rms")
    want, grads = forward(lq, cfg, d), backward(lq, cfg, d)

    def spread(t, at):
        v = big.as_strided((M, D), (far, 1), 0) if at == 0 else t
        v.copy_(t)
        return v
    e = dict(d, h=spread(d["h"], 0))
    ho, x = forward(lq, cfg, e, ho=e["h"])
    assert torch.equal(ho, want[0]) and torch.equal(x, want[1])
    big.zero_()
    e = dict(d, dx=spread(d["dx"], 0))
    got = backward(lq, cfg, e, dy=e["dx"])
    for a, b in zip(got, grads):
        assert torch.equal(a, b) if a is not None else b is None


def test_empty_batch(lq):
    d = make(0, 64, [0, 0, 0])
    cfg = config(lq, d, "rms", "layer")
    ho, x = forward(lq, cfg, d)
    assert ho.shape == x.shape == (0, 64)
    for t in backward(lq, cfg, d)[2:]:
        assert (t == 0).all()


def test_captured_and_replayed_on_a_stream(lq):
    M, D = 600, 1152
    d = make(M, D, [0, 100, 590])
    cfg = config(lq, d, "rms", "layer")
    keys = ("h", "y", "dx", "dho", "offsets")
    work = torch.empty(lq.lq_block_work_sizes(cfg, M, 2), dtype=torch.uint8, device="cuda")
    outs = [t.clone() for t in forward(lq, cfg, d)]
    grads = [t.clone() for t in backward(lq, cfg, d)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()

    def both():
        forward(lq, cfg, d, ho=outs[0], x=outs[1])
        backward(lq, cfg, d, **dict(zip(GRADS, grads)), work=work)
    with torch.cuda.stream(s):
        both()
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            both()
    torch.cuda.synchronize()
    for k in range(4):
        e = make(M, D, [0, 50 * k, 590], seed=20 + k)
        for key in keys:
            d[key].copy_(e[key])
        f = dict(d, **{key: e[key] for key in keys})
        want = list(forward(lq, cfg, f)) + list(backward(lq, cfg, f))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs + grads, want):
            a, b = (a[:590], b[:590]) if a.shape[0] == M else (a, b)
            assert torch.equal(a, b), k


def test_captured_without_a_call_before(lq):
    """Forms that nothing else calls: what a first call asks of the runtime is allowed in a capture."""
    d = make(700, 1021, [0, 333, 700], "f32", "f32")
    cfg = config(lq, d, "layer", "rms")
    outs = [torch.zeros_like(d["h"]) for _ in range(4)]
    sums = [torch.zeros(2, 1021, device="cuda") for _ in range(3)] + [torch.zeros(1021, device="cuda") for _ in range(2)]
    work = torch.empty(lq.lq_block_work_sizes(cfg, 700, 2), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        forward(lq, cfg, d, ho=outs[0], x=outs[1])
        backward(lq, cfg, d, **dict(zip(GRADS, outs[2:] + sums)), work=work)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs + sums, list(forward(lq, cfg, d)) + list(backward(lq, cfg, d))):
        assert torch.equal(a, b)


def test_offsets_that_do_not_rise_stay_in_bounds(lq):
    """What comes out then is not defined; nothing outside the rows is touched."""
    M, D = 40, 72
    for offsets in ([0, 30, 10, 40], [-5, 20, 90], [50, 60, 70], [0, -3, 2 ** 31 - 1]):
        d = make(M, D, offsets)
        cfg = config(lq, d, "rms", "layer")
        S = len(offsets) - 1
        big = torch.full((M + 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
        sums = torch.full((S + 2, D), 7.0, device="cuda")
        forward(lq, cfg, d, x=big[1:-1])
        assert (big[[0, -1]] == 7.0).all()
        backward(lq, cfg, d, dy=big[1:-1], dgate=sums[1:-1])
        assert (big[[0, -1]] == 7.0).all() and (sums[[0, -1]] == 7.0).all()


@pytest.mark.parametrize("M,offsets", [
    (12, [0, 5, 5, 12]), (4000, [0, 1000, 1000, 4000, 4000]),                       # weights' sums with those of the sequences
    (390, [3 * (i // 2) for i in range(261)]), (3000, [30 * (i - i % 3) // 3 for i in range(301)]),  # ... in a launch of their own
    (9, [0, 0, 9, 9, 9]), (0, [0, 0, 0])])
@pytest.mark.parametrize("D", [40, 1153])
def test_modulation_of_sequences_without_rows_is_not_used(lq, D, M, offsets):
    """Rows of modulation that belong to nothing (unused places of a batch of fixed size) may hold anything: their own gradients are zeros, and no other value sees them."""
    d = make(M, D, offsets, "f32", "bf16")
    cfg = config(lq, d, "rms", "layer")
    empty = (d["offsets"][1:] == d["offsets"][:-1])
    assert empty.any()
    want = [list(forward(lq, cfg, d)), list(backward(lq, cfg, d))]
    e = {k: v.clone() if k in ("gate", "scale", "shift") else v for k, v in d.items()}
    for k, v in (("gate", float("inf")), ("scale", float("nan")), ("shift", float("nan"))):
        e[k][empty] = v
    got = [list(forward(lq, cfg, e)), list(backward(lq, cfg, e))]
    inside = slice(offsets[0], offsets[-1])
    for a, b in zip(got[0] + got[1][:2], want[0] + want[1][:2]):
        assert torch.equal(a[inside], b[inside])
    for k, a, b in zip(GRADS[2:], got[1][2:], want[1][2:]):
        assert torch.equal(a, b), k
    for t in got[1][2:5]:
        assert (t[empty] == 0).all()


def test_gradients_of_sequences_without_rows_are_zeros_whatever_the_weights(lq):
    d = make(20, 72, [0, 8, 8, 20], "f32", "f32")
    cfg = config(lq, d, "rms", "layer")
    d["w_post"][3], d["w_pre"][5] = float("inf"), float("nan")
    for t in backward(lq, cfg, d)[2:5]:
        assert (t[1] == 0).all()
