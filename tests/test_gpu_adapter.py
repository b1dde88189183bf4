"""Low-rank adapters of many requests (lq_adapter_plan, lq_adapter_fwd, lq_adapter_bwd) against the plain 64-bit implementation."""
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _strided(t, pad):
    """The same rows, `pad` values further apart; what lies between holds a pattern."""
    if not pad:
        return t.contiguous()
    big = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def _untouched(t):
    """The values between the rows of a _strided tensor still hold their pattern."""
    big = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))
    return bool((big[:, t.shape[1]:] == 7.0).all())


def make(M, K, N, R, slots, x="f32", seed=0, ids=None, pad=0, ranks="mixed", garbage=True):
    g = _gen(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    dt = torch.float32 if x == "f32" else torch.bfloat16
    d = dict(A=(normal(slots, R, K) * K ** -0.5).bfloat16(), B=(normal(slots, N, R) * 0.2).bfloat16())
    d["scales"] = torch.rand(slots, generator=g, device="cuda") * 3 - 1
    r = torch.randint(0, R + 1, (slots,), generator=g, device="cuda", dtype=torch.int32) if ranks == "mixed" else torch.full((slots,), R, dtype=torch.int32, device="cuda")
    if ranks == "mixed":
        r[0] = R
        if slots > 2:
            r[1], r[2] = 0, max(1, R - 3)
        if slots > 4:
            r[3], r[4] = R + 9, -2          # taken as R and 0
    d["ranks"] = r
    if garbage:                             # what lies beyond an adapter's rank is not looked at
        j = torch.arange(R, device="cuda")
        out = j[None, :] >= r.clamp(0, R)[:, None]
        d["A"][out[:, :, None].expand_as(d["A"])] = float("nan")
        d["B"][out[:, None, :].expand_as(d["B"])] = float("inf")
    if ids is None:
        ids = torch.randint(-1, slots + 1, (M,), generator=g, device="cuda")  # -1 and slots: none
    elif isinstance(ids, int):
        ids = torch.full((M,), ids, device="cuda")
    d["ids"] = ids.to(torch.int32).cuda()
    d["X"], d["Yin"] = _strided(normal(M, K).to(dt), pad), _strided(normal(M, N).bfloat16(), pad)
    d["dY"], d["dXin"] = _strided((normal(M, N) * 0.1).bfloat16(), pad), _strided((normal(M, K) * 0.1).to(dt), pad)
    return d


def pool(d):
    return d["A"], d["B"], d["ranks"], d["scales"]


def run(lq, d, x="f32", in_place=False, dxin=True):
    M, K = d["X"].shape
    slots, R, _ = d["A"].shape
    N = d["B"].shape[1]
    cfg = lq.make_adapter_config(N, K, R, slots, x)
    plan = lq.lq_adapter_plan(slots, d["ids"])
    inter_b, work_b = lq.lq_adapter_sizes(cfg, M)
    inter = torch.full((inter_b,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN patterns: nothing is read before it is written)
    work = torch.full((work_b,), 0xFF, dtype=torch.uint8, device="cuda")
    pad = d["X"].stride(0) - K if M > 1 else 0
    Yin = d["Yin"].clone() if not pad else _strided(d["Yin"], pad)
    Y = Yin if in_place else _strided(torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda"), pad)
    Y = lq.lq_adapter_fwd(cfg, plan, d["X"], *pool(d), Yin, Y=Y, inter=inter)
    dXin = (d["dXin"].clone() if not pad else _strided(d["dXin"], pad)) if dxin else None
    dX = dXin if in_place and dxin else _strided(torch.full((M, K), float("nan"), dtype=d["X"].dtype, device="cuda"), pad)
    dA = torch.full(d["A"].shape, float("nan"), device="cuda")
    dB = torch.full(d["B"].shape, float("nan"), device="cuda")
    dX, dA, dB = lq.lq_adapter_bwd(cfg, plan, d["X"], *pool(d), inter, d["dY"], dXin=dXin, dX=dX, dA=dA, dB=dB, work=work)
    if pad:
        assert _untouched(Y) and _untouched(dX)
    return Y, dX, dA, dB


def compare(d, out, dxin=True, what=""):
    Y, dX, dA, dB = out
    ref.check(Y, ref.adapter_fwd(d["X"], d["Yin"], *pool(d), d["ids"]), what + " Y")
    want = ref.adapter_bwd(d["X"], d["dXin"] if dxin else None, *pool(d), d["ids"], d["dY"])
    for k, t in (("dX", dX), ("dA", dA), ("dB", dB)):
        ref.check(t, want[k], f"{what} {k}")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,R,slots", [
    (1, 64, 64, 8, 1), (2, 1152, 1152, 16, 4), (15, 64, 128, 24, 3), (16, 192, 320, 40, 2), (17, 128, 64, 128, 1), (63, 256, 192, 72, 6),
    (64, 320, 64, 104, 2), (65, 64, 448, 32, 1), (130, 1152, 192, 64, 64), (300, 512, 640, 48, 8), (1025, 192, 320, 16, 5), (2500, 128, 192, 80, 3),
    (700, 64, 64, 8, 1024), (4099, 64, 128, 96, 33), (150, 192, 320, 48, 9), (24, 64, 832, 128, 1), (240, 1152, 64, 24, 10), (241, 128, 192, 16, 10)])
def test_forward_and_backward(lq, M, K, N, R, slots, x):
    d = make(M, K, N, R, slots, x, seed=M + R)
    compare(d, run(lq, d, x), what=f"{M} x {K} -> {N} rank {R} slots {slots}")


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_a_full_layer(lq, x):
    """The fused QKV width, requests of uneven length, one adapter over most of the batch (several groups of its gradients' sums)."""
    M = 3001
    ids = torch.cat([torch.full((2400,), 1), torch.full((1,), 0), torch.full((400,), -1), torch.full((200,), 2)])
    d = make(M, 1152, 3456, 32, 4, x, seed=5, ids=ids, ranks="full")
    compare(d, run(lq, d, x), what="full layer")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[65, 65, 65, 129, 1, 64, 0, 65, 193], [0, 0, 129, 0, 65, 66, 127, 128, 65, 0], [700], [64, 64, 1]])
def test_a_few_adapters_of_a_large_pool(lq, counts, x):
    """Adapters whose last tile holds a single row, next to each other: their gradients' parts stay apart."""
    ids = torch.repeat_interleave(torch.arange(len(counts)) + 3, torch.tensor(counts))
    d = make(len(ids), 128, 192, 24, 100, x, seed=sum(counts), ids=ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(1))], ranks="full")
    compare(d, run(lq, d, x), what=f"counts {counts}")


@pytest.mark.parametrize("rank", [8, 128])
@pytest.mark.parametrize("ids", [-1, 0, 2, 3])
def test_one_adapter_for_all_rows(lq, ids, rank):
    """No row has an adapter; all have the first; the last; a number past the pool's."""
    d = make(200, 128, 192, rank, 3, "bf16", seed=ids + 9, ids=ids, ranks="full", garbage=False)
    out = run(lq, d, "bf16")
    compare(d, out, what=f"ids {ids}")
    if ids in (-1, 3):
        assert torch.equal(out[0], d["Yin"]) and torch.equal(out[1], d["dXin"])
    for s in range(3):
        assert (s == ids) == bool((out[2][s] != 0).any()) == bool((out[3][s] != 0).any())


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_strides_in_place_and_no_incoming_gradient(lq, x):
    d = make(133, 128, 192, 24, 5, x, seed=3, pad=24)
    a = run(lq, d, x)
    compare(d, a, what="strided")
    b = run(lq, d, x, in_place=True)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    compare(d, run(lq, d, x, dxin=False), dxin=False, what="no dXin")


def test_rows_do_not_depend_on_each_other(lq):
    """A row's output is the same bits whatever else is in the batch and wherever it stands."""
    d = make(777, 576, 320, 40, 6, "bf16", seed=4)
    Y, dX, _, _ = run(lq, d, "bf16")
    g = _gen(8)
    for n in (1, 5, 64, 500):
        pick = torch.randperm(777, generator=g, device="cuda")[:n]
        e = dict(d, **{k: d[k][pick].contiguous() for k in ("X", "Yin", "dY", "dXin", "ids")})
        Y2, dX2, _, _ = run(lq, e, "bf16")
        assert torch.equal(Y2, Y[pick]) and torch.equal(dX2, dX[pick]), n


@pytest.mark.parametrize("R", [8, 40, 96, 128])
def test_many_adapters_of_few_rows(lq, R):
    """Enough adapters for the form with a wavefront per 128 columns (one of them with more than 16 rows, some with none), with the other form's bits."""
    M, K, N, slots = 130, 128, 1088, 70
    g = _gen(R)
    ids = torch.randint(-1, slots, (M,), generator=g, device="cuda")
    ids[:40] = 7
    d = make(M, K, N, R, slots, "bf16", seed=R, ids=ids, pad=8)
    cfg = lq.make_adapter_config(N, K, R, slots)
    Y = lq.lq_adapter_fwd(cfg, lq.lq_adapter_plan(slots, d["ids"]), d["X"], *pool(d), d["Yin"])
    ref.check(Y, ref.adapter_fwd(d["X"], d["Yin"], *pool(d), d["ids"]), "Y")
    one = make(40, K, N, R, 8, "bf16", ids=7, garbage=False)
    e = dict(one, X=d["X"][:40], Yin=d["Yin"][:40], A=d["A"][:8].contiguous(), B=d["B"][:8].contiguous(), ranks=d["ranks"][:8].contiguous(), scales=d["scales"][:8].contiguous())
    alone = lq.lq_adapter_fwd(lq.make_adapter_config(N, K, R, 8), lq.lq_adapter_plan(8, one["ids"]), e["X"], *pool(e), e["Yin"])
    assert torch.equal(alone, Y[:40])
    inplace = _strided(d["Yin"], 8)
    lq.lq_adapter_fwd(cfg, lq.lq_adapter_plan(slots, d["ids"]), d["X"], *pool(d), inplace, Y=inplace)
    assert torch.equal(inplace, Y) and _untouched(inplace)


def test_not_a_number_stays_in_its_row(lq):
    """Infinities and NaN in rows without an adapter are carried over as they are and reach nothing else; in rows with one they reach that adapter alone."""
    d = make(300, 128, 192, 24, 4, "f32", seed=6, ranks="full", garbage=False)
    clean = [t.clone() for t in run(lq, d, "f32")]
    none = ((d["ids"] < 0) | (d["ids"] >= 4)).nonzero()[:, 0]
    one = (d["ids"] == 2).nonzero()[:1, 0]
    assert none.numel() > 3 and one.numel() == 1
    e = {k: v.clone() for k, v in d.items()}
    for rows in (none[:3], one):
        e["X"][rows] = float("nan")
        e["Yin"][rows, ::3] = float("inf")
        e["dY"][rows, 5] = float("-inf")
        e["dXin"][rows, 1] = float("nan")
    Y, dX, dA, dB = run(lq, e, "f32")
    assert torch.equal(Y[none].view(torch.int16), e["Yin"][none].view(torch.int16)) and torch.equal(dX[none].view(torch.int32), e["dXin"][none].view(torch.int32))
    rest = torch.ones(300, dtype=torch.bool, device="cuda")
    rest[none[:3]] = rest[one] = False
    assert torch.equal(Y[rest], clean[0][rest]) and torch.equal(dX[rest], clean[1][rest])
    for s in (0, 1, 3):
        assert torch.equal(dA[s], clean[2][s]) and torch.equal(dB[s], clean[3][s])
    assert torch.isnan(Y[one]).all() and torch.isnan(dA[2]).any()


@pytest.mark.parametrize("M,slots", [(1, 1), (63, 5), (1000, 1024), (1025, 3), (8192, 1024), (8193, 64), (20011, 1024), (40000, 2)])
def test_plans_of_every_size(lq, M, slots):
    """Batches on both sides of the plan's forms: every row's output is its own adapter's, with runs of one adapter and single rows mixed."""
    g = _gen(M + slots)
    ids = torch.randint(-1, slots, (M,), generator=g, device="cuda")
    ids[M // 3: M // 2] = slots - 1
    d = make(M, 64, 64, 8, slots, "bf16", seed=M, ids=ids, ranks="full", garbage=False)
    cfg = lq.make_adapter_config(64, 64, 8, slots)
    Y = lq.lq_adapter_fwd(cfg, lq.lq_adapter_plan(slots, d["ids"]), d["X"], *pool(d), d["Yin"])
    A, B = d["A"].double(), d["B"].double()
    own = ids.clamp(min=0)
    T = (d["X"].double()[:, None, :] * A[own]).sum(-1)
    delta = (T[:, None, :] * B[own]).sum(-1) * d["scales"].double()[own, None] * (ids >= 0)[:, None]
    Tabs = (d["X"].double().abs()[:, None, :] * A[own].abs()).sum(-1)
    off = ((72 * ref.U * Tabs + 2.0 ** -16 * T.abs())[:, None, :] * B[own].abs()).sum(-1) * d["scales"].double().abs()[own, None] * (1 + 30 * ref.U)
    want = d["Yin"].double() + delta
    off = off + 30 * ref.U * (Tabs[:, None, :] * B[own].abs()).sum(-1) * d["scales"].double().abs()[own, None] + 4 * ref.U * d["Yin"].double().abs()
    ref.check(Y, (want, off + ref.ROUND[torch.bfloat16] * (want.abs() + off)), f"{M} rows, {slots} adapters")


def test_empty_batch(lq):
    d = make(0, 128, 64, 8, 3, "bf16", ids=torch.zeros(0))
    Y, dX, dA, dB = run(lq, d, "bf16")
    assert Y.shape == (0, 64) and dX.shape == (0, 128)
    assert (dA == 0).all() and (dB == 0).all()


def test_gradients_against_differences(lq):
    """sum(dY * Y) is linear in each of X, A and B: its difference quotient, taken in 64 bits along a random direction, is the gradient's inner product."""
    d = make(190, 128, 192, 16, 3, "f32", seed=11, ranks="full", garbage=False)
    _, dX, dA, dB = run(lq, d, "f32", dxin=False)

    def loss(**kw):
        e = dict(d, **kw)
        return (ref.adapter_fwd(e["X"], e["Yin"], e["A"], e["B"], e["ranks"], e["scales"], e["ids"])[0] * d["dY"].double()).sum()
    want = ref.adapter_bwd(d["X"], None, *pool(d), d["ids"], d["dY"])
    g = _gen(12)
    for key, grad in (("X", dX), ("A", dA), ("B", dB)):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-3
        diff = (loss(**{key: d[key].double() + h * v}) - loss(**{key: d[key].double() - h * v})) / (2 * h)
        assert abs(float((grad.double() * v).sum() - diff)) <= float((want["d" + key][1] * v.abs()).sum()) + 1e-9 * abs(float(diff)), key


def test_deterministic_on_another_stream_and_in_a_graph(lq):
    d = make(900, 320, 448, 64, 7, "bf16", seed=2)
    first = [t.clone() for t in run(lq, d, "bf16")]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = run(lq, d, "bf16")
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    cfg = lq.make_adapter_config(448, 320, 64, 7, "bf16")
    inter_b, work_b = lq.lq_adapter_sizes(cfg, 900)
    buf = dict(plan=torch.zeros(lq.lq_adapter_plan_sizes(900, 7), dtype=torch.uint8, device="cuda"), inter=torch.zeros(inter_b, dtype=torch.uint8, device="cuda"),
               work=torch.zeros(work_b, dtype=torch.uint8, device="cuda"), Y=torch.zeros_like(d["Yin"]), dX=torch.zeros_like(d["X"]),
               dA=torch.zeros(d["A"].shape, device="cuda"), dB=torch.zeros(d["B"].shape, device="cuda"))

    def step():
        lq.lq_adapter_plan(7, d["ids"], plan=buf["plan"])
        lq.lq_adapter_fwd(cfg, buf["plan"], d["X"], *pool(d), d["Yin"], Y=buf["Y"], inter=buf["inter"])
        lq.lq_adapter_bwd(cfg, buf["plan"], d["X"], *pool(d), buf["inter"], d["dY"], dXin=d["dXin"], dX=buf["dX"], dA=buf["dA"], dB=buf["dB"], work=buf["work"])
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 21, 22):
        e = make(900, 320, 448, 64, 7, "bf16", seed=seed)
        for k in d:
            d[k].copy_(e[k])
        eager = [t.clone() for t in run(lq, d, "bf16")]
        for k in ("Y", "dX", "dA", "dB"):
            buf[k].fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, k in zip(eager, ("Y", "dX", "dA", "dB")):
            assert torch.equal(a, buf[k]), (seed, k)


def test_offsets_past_32_bits(lq):
    """Rows 2^20 values apart: the last ones start beyond 2^31 values."""
    M, K, N, R = 2200, 64, 128, 8
    d = make(M, K, N, R, 2, "bf16", seed=7, ids=torch.arange(2200) % 3)
    far = {}
    for k, cols in (("X", K), ("Yin", N), ("dY", N), ("dXin", K)):
        big = torch.empty((M << 20) + cols, dtype=torch.bfloat16, device="cuda").as_strided((M, cols), (1 << 20, 1))
        big.copy_(d[k])
        far[k] = big
    e = dict(d, **far)
    cfg = lq.make_adapter_config(N, K, R, 2, "bf16")
    plan = lq.lq_adapter_plan(2, e["ids"])
    inter = torch.empty(lq.lq_adapter_sizes(cfg, M)[0], dtype=torch.uint8, device="cuda")
    Y = lq.lq_adapter_fwd(cfg, plan, e["X"], *pool(e), e["Yin"], Y=e["Yin"], inter=inter)
    dX, dA, dB = lq.lq_adapter_bwd(cfg, plan, e["X"], *pool(e), inter, e["dY"], dXin=e["dXin"], dX=e["dXin"])
    compare(d, (Y, dX, dA, dB), what="far rows")


def test_beside_a_quantised_projection(lq):
    """The path as it is used: activation step and forward of the quantised layer, then the adapters in place on its output."""
    g = _gen(1)
    M, K, N = 190, 256, 320
    cfg = lq.make_config(N, K, 32, "int", 64, 8, 8)
    W = torch.randn((N, K), generator=g, device="cuda") * 0.02
    packed = lq.lq_pack_weights(cfg, W, torch.randn((N, 32), generator=g, device="cuda") * 1e-3, torch.randn((32, K), generator=g, device="cuda") * 1e-3)
    d = make(M, K, N, 16, 4, "bf16", seed=13)
    Y = lq.lq_linear_lowrank_fwd(cfg, packed, lq.lq_quantize_act(cfg, packed, d["X"]), M)
    d["Yin"] = Y.clone()
    acfg = lq.make_adapter_config(N, K, 16, 4)
    out = lq.lq_adapter_fwd(acfg, lq.lq_adapter_plan(4, d["ids"]), d["X"], *pool(d), Y, Y=Y)
    assert out is Y or out.data_ptr() == Y.data_ptr()
    ref.check(Y, ref.adapter_fwd(d["X"], d["Yin"], *pool(d), d["ids"]), "in place on the projection's output")
