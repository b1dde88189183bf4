"""Norm of queries and keys with the rotation by positions of several axes (lq_qk_norm_rope_fwd, lq_qk_norm_rope_bwd) against the plain 64-bit implementation."""
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make(M, Hq, Hk, D, pairs, x="bf16", seed=0, layout="dense", pos_rows=None, big=False):
    """layout: dense | fused (queries, keys and values in one row) | heads (heads outermost) | odd (heads D + 1 apart: no vector is aligned)."""
    g = _gen(seed)
    dt = torch.float32 if x == "f32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def heads(H):
        v = (normal(M, H, D) * 2).to(dt)
        if layout == "heads":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "odd":
            t = torch.zeros((M, H, D + 1), dtype=dt, device="cuda")
            t[..., 1:] = v
            return t[..., 1:]
        return v
    d = dict(q=heads(Hq), k=heads(Hk), dqo=(normal(M, Hq, D) * 0.1).to(dt), dko=(normal(M, Hk, D) * 0.1).to(dt))
    if layout == "fused":
        row = (normal(M, (Hq + 2 * Hk) * D) * 2).to(dt)
        d["row"] = row
        d["q"], d["k"] = row[:, :Hq * D].view(M, Hq, D), row[:, Hq * D:(Hq + Hk) * D].view(M, Hk, D)
    d["wq"], d["wk"] = 1 + 0.3 * normal(D), 1 + 0.3 * normal(D)
    rows = M if pos_rows is None else pos_rows
    d["pos"] = torch.randint(0, 64, (max(rows, 1), max(len(pairs), 1)), generator=g, device="cuda").float()
    if big:  # far positions, fractions, negative ones
        d["pos"] = d["pos"] * 12345.25 - 300000.5
    d["inv_freq"] = torch.cat([10000.0 ** (-torch.arange(p, dtype=torch.float64) / max(p, 1)) for p in pairs] + [torch.zeros(0, dtype=torch.float64)]).float().cuda()
    return d


def run(lq, d, cfg, **kw):
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    return lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], *at, **kw), lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"])


def compare(d, out, pairs, pairing, norm=True, what=""):
    (qo, ko), (dq, dk, dwq, dwk) = out
    for name, x, w, y, dy, dx, dw in (("q", d["q"], d["wq"], qo, d["dqo"], dq, dwq), ("k", d["k"], d["wk"], ko, d["dko"], dk, dwk)):
        ref.check(y, ref.qk_fwd(x, w, d["pos"], d["inv_freq"], pairs, pairing, norm, EPS), f"{what} {name}")
        want = ref.qk_bwd(x, w, d["pos"], d["inv_freq"], pairs, pairing, norm, EPS, dy)
        ref.check(dx, want[0], f"{what} d{name}")
        if norm:
            ref.check(dw, want[1], f"{what} dw{name}")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "adjacent"])
@pytest.mark.parametrize("M,Hq,Hk,D,pairs", [
    (1, 1, 1, 2, (1,)), (1, 16, 16, 72, (18, 18)), (3, 5, 2, 6, (1, 1)), (7, 3, 1, 50, (9, 8, 8)), (33, 20, 20, 112, (16, 20, 20)), (64, 2, 2, 256, (40, 40, 24, 24)),
    (65, 7, 7, 128, (64,)), (130, 12, 3, 96, (12, 12, 12)), (19, 4, 4, 254, (127,)), (21, 6, 6, 36, (5, 4)), (257, 70, 70, 32, (8, 8)), (40, 1, 9, 20, (3, 7)),
    (1100, 4, 2, 64, (16, 16)), (11, 3, 3, 160, (0, 80)), (5, 300, 2, 8, (2, 1))])
def test_forward_and_backward(lq, M, Hq, Hk, D, pairs, pairing, x):
    d = make(M, Hq, Hk, D, pairs, x, seed=M + D)
    cfg = lq.make_qk_config(Hq, Hk, D, pairs, pairing, True, EPS, x)
    compare(d, run(lq, d, cfg), pairs, pairing, what=f"{M} x ({Hq} + {Hk}) x {D} {pairs}")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["half", "adjacent"])
@pytest.mark.parametrize("layout", ["fused", "heads", "odd"])
@pytest.mark.parametrize("D,pairs", [(72, (18, 18)), (64, (8, 8, 8)), (18, (4, 5))])
def test_layouts(lq, D, pairs, layout, pairing, x):
    d = make(37, 6, 2, D, pairs, x, seed=D, layout=layout)
    cfg = lq.make_qk_config(6, 2, D, pairs, pairing, True, EPS, x)
    compare(d, run(lq, d, cfg), pairs, pairing, what=layout)
    # in place, where the values and what lies between the heads must stay as they are
    q, k = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t) for t in (d["q"], d["k"])]
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    want = [t.clone() for t in lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], *at)]
    if layout == "fused":
        row = d["row"].clone()
        q, k = row[:, :6 * D].view(37, 6, D), row[:, 6 * D:8 * D].view(37, 2, D)
        lq.lq_qk_norm_rope_fwd(cfg, q, k, *at, qo=q, ko=k)
        assert torch.equal(row[:, 8 * D:], d["row"][:, 8 * D:])
    else:
        lq.lq_qk_norm_rope_fwd(cfg, q, k, *at, qo=q, ko=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    g = [d["dqo"].clone(), d["dko"].clone()]
    first = lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"])
    again = lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, g[0], g[1], dq=g[0], dk=g[1])
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_output_between_heads_is_untouched(lq):
    d = make(29, 3, 3, 32, (8, 8), "bf16")
    cfg = lq.make_qk_config(3, 3, 32, (8, 8), "half", True, EPS)
    big = torch.full((29, 3, 48), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, _ = lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], d["wq"], d["wk"], d["pos"], d["inv_freq"], qo=big[..., 8:40])
    assert (big[..., :8] == 7).all() and (big[..., 40:] == 7).all()
    ref.check(qo, ref.qk_fwd(d["q"], d["wq"], d["pos"], d["inv_freq"], (8, 8), "half", True, EPS), "q")


@pytest.mark.parametrize("pairing", ["half", "adjacent"])
def test_without_norm_weights_or_rotation(lq, pairing):
    for x in ("bf16", "f32"):
        d = make(50, 4, 2, 40, (10, 10), x, seed=3)
        compare(d, run(lq, d, lq.make_qk_config(4, 2, 40, (10, 10), pairing, False, EPS, x)), (10, 10), pairing, norm=False, what="rotation alone")
        d["wq"] = d["wk"] = None
        compare(d, run(lq, d, lq.make_qk_config(4, 2, 40, (10, 10), pairing, True, EPS, x)), (10, 10), pairing, what="no weights")
        cfg = lq.make_qk_config(4, 2, 40, (), pairing, True, EPS, x)
        d["pos"] = d["inv_freq"] = None
        compare(d, run(lq, d, cfg), (), pairing, what="norm alone")


def test_positions_shared_by_equal_grids_and_far_ones(lq):
    d = make(60, 3, 3, 72, (18, 18), "f32", seed=5, pos_rows=20, big=True)
    cfg = lq.make_qk_config(3, 3, 72, (18, 18), "half", True, EPS, "f32")
    a = run(lq, d, cfg)
    compare(d, a, (18, 18), "half", what="grids")
    e = dict(d, pos=d["pos"].repeat(3, 1).contiguous())
    for p, q in zip(a[0], run(lq, e, cfg)[0]):
        assert torch.equal(p, q)


def test_rows_of_zeros_extremes_and_not_a_number(lq):
    """A head of zeros gives zeros and finite gradients; large and small heads stay in range; NaN and infinities stay in their head."""
    cfg = lq.make_qk_config(4, 2, 64, (16, 16), "half", True, EPS, "f32")
    d = make(9, 4, 2, 64, (16, 16), "f32", seed=8)
    clean = [t.clone() for t in run(lq, d, cfg)[0]]
    d["q"][2, 1] = 0.0
    d["q"][3, 0] *= 1e15
    d["k"][4, 1] *= 1e-15
    d["q"][5, 2, 7] = float("nan")
    d["q"][6, 3, 1] = float("inf")
    (qo, ko), (dq, dk, dwq, dwk) = run(lq, d, cfg)
    assert (qo[2, 1] == 0).all() and torch.isfinite(dq[2, 1]).all()
    ok = torch.ones((9, 4), dtype=torch.bool, device="cuda")
    ok[5, 2] = ok[6, 3] = False
    assert torch.isfinite(qo[ok]).all() and torch.isfinite(ko).all() and torch.isfinite(dq[ok]).all() and torch.isfinite(dk).all() and torch.isfinite(dwk).all()
    assert torch.isnan(qo[5, 2]).all()
    same = ok.clone()
    same[2, 1] = same[3, 0] = False
    assert torch.equal(qo[same], clean[0][same])


@pytest.mark.parametrize("which", ["q", "k"])
def test_queries_or_keys_alone_and_empty_batch(lq, which):
    d = make(31, 5, 5, 48, (12, 12), "bf16", seed=4)
    cfg = lq.make_qk_config(5 if which == "q" else 0, 5 if which == "k" else 0, 48, (12, 12), "adjacent", True, EPS)
    q, k = (d["q"], None) if which == "q" else (None, d["k"])
    dqo, dko = (d["dqo"], None) if which == "q" else (None, d["dko"])
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    out = lq.lq_qk_norm_rope_fwd(cfg, q, k, *at)
    i = 0 if which == "q" else 1
    assert out[1 - i] is None
    w = d["w" + which]
    ref.check(out[i], ref.qk_fwd(d[which], w, d["pos"], d["inv_freq"], (12, 12), "adjacent", True, EPS), which)
    grads = lq.lq_qk_norm_rope_bwd(cfg, q, k, *at, dqo, dko)
    want = ref.qk_bwd(d[which], w, d["pos"], d["inv_freq"], (12, 12), "adjacent", True, EPS, d["d" + which + "o"])
    ref.check(grads[i], want[0], "d" + which)
    ref.check(grads[2 + i], want[1], "dw" + which)
    assert (grads[3 - i] == 0).all()
    e = {k2: (v[:0] if k2 in ("q", "k", "dqo", "dko") else v) for k2, v in d.items()}
    cfg = lq.make_qk_config(5, 5, 48, (12, 12), "adjacent", True, EPS)
    (qo, ko), (dq, dk, dwq, dwk) = run(lq, e, cfg)
    assert qo.shape == (0, 5, 48) and (dwq == 0).all() and (dwk == 0).all()


def test_gradients_against_differences(lq):
    """Central differences of the 64-bit forward along random directions."""
    pairs = (6, 6)
    d = make(23, 3, 2, 32, pairs, "f32", seed=6)
    cfg = lq.make_qk_config(3, 2, 32, pairs, "half", True, EPS, "f32")
    _, (dq, dk, dwq, dwk) = run(lq, d, cfg)
    g = _gen(9)
    for x, w, dy, dx, dw in ((d["q"], d["wq"], d["dqo"], dq, dwq), (d["k"], d["wk"], d["dko"], dk, dwk)):
        def loss(x_, w_):
            return (ref.qk_fwd(x_, w_, d["pos"], d["inv_freq"], pairs, "half", True, EPS)[0] * dy.double()).sum()
        x64, w64, h = x.double(), w.double(), 1e-4
        v, vw = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64), torch.randn(w.shape, generator=g, device="cuda", dtype=torch.float64)
        want = ref.qk_bwd(x, w, d["pos"], d["inv_freq"], pairs, "half", True, EPS, dy)
        # (third derivatives of x / rms(x) over values of size 2, times h^2: below 1e-6 of the sum of the gradient's terms)
        for diff, grad, dirn, bound in (((loss(x64 + h * v, w64) - loss(x64 - h * v, w64)) / (2 * h), dx, v, want[0][1]),
                                        ((loss(x64, w64 + h * vw) - loss(x64, w64 - h * vw)) / (2 * h), dw, vw, want[1][1])):
            terms = float((grad.double() * dirn).abs().sum())
            assert abs(float((grad.double() * dirn).sum() - diff)) <= float((bound * dirn.abs()).sum()) + 1e-6 * terms


def test_deterministic_on_another_stream_and_in_a_graph(lq):
    d = make(3000, 16, 16, 72, (18, 18), "bf16", seed=2, layout="fused")
    cfg = lq.make_qk_config(16, 16, 72, (18, 18), "half", True, EPS)
    first = run(lq, d, cfg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = run(lq, d, cfg)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(first[0] + first[1], again[0] + again[1]):
        assert torch.equal(a, b)
    at = (d["wq"], d["wk"], d["pos"], d["inv_freq"])
    buf = [torch.zeros((3000, 16, 72), dtype=torch.bfloat16, device="cuda") for _ in range(4)] + [torch.zeros(72, device="cuda") for _ in range(2)]
    work = torch.zeros(lq.lq_qk_work_sizes(cfg, 3000), dtype=torch.uint8, device="cuda")

    def step():
        lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], *at, qo=buf[0], ko=buf[1])
        lq.lq_qk_norm_rope_bwd(cfg, d["q"], d["k"], *at, d["dqo"], d["dko"], dq=buf[2], dk=buf[3], dwq=buf[4], dwk=buf[5], work=work)
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 5, 6):
        e = make(3000, 16, 16, 72, (18, 18), "bf16", seed=seed, layout="fused")
        for k in ("row", "dqo", "dko", "wq", "wk", "pos"):
            d[k].copy_(e[k])
        eager = run(lq, d, cfg)
        for b in buf:
            b.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager[0] + eager[1], buf):
            assert torch.equal(a, b), seed


def test_offsets_past_32_bits(lq):
    """Tokens 2^21 values apart: the last ones start beyond 2^31 values."""
    M, H, D = 1100, 2, 16
    d = make(M, H, H, D, (4, 4), "bf16", seed=1)
    cfg = lq.make_qk_config(H, H, D, (4, 4), "half", True, EPS)
    big = torch.empty((M << 21) + 64, dtype=torch.bfloat16, device="cuda")
    q, k = big.as_strided((M, H, D), (1 << 21, D, 1)), big.as_strided((M, H, D), (1 << 21, D, 1), H * D)
    q.copy_(d["q"])
    k.copy_(d["k"])
    want = lq.lq_qk_norm_rope_fwd(cfg, d["q"], d["k"], d["wq"], d["wk"], d["pos"], d["inv_freq"])
    lq.lq_qk_norm_rope_fwd(cfg, q, k, d["wq"], d["wk"], d["pos"], d["inv_freq"], qo=q, ko=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    ref.check(q, ref.qk_fwd(d["q"], d["wq"], d["pos"], d["inv_freq"], (4, 4), "half", True, EPS), "q")
