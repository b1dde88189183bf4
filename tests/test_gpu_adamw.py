"""The AdamW step over many tensors (lq_adamw_step) against the plain 64-bit formulas; states in 8 bits against their rule, element by element."""
import pytest
import torch

from tests import blocks_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def make(lq, cfg, sizes, master=False, seed=0, start=0):
    """Tensors in one buffer of each kind, `start` values from its start and from each other."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    total = sum(sizes) + (len(sizes) + 1) * start + 16
    dts = [DT["f32" if c == lq.LQ_F32 else "bf16"] for c in (cfg.p_dtype, cfg.g_dtype)]

    def spread(t):
        out, at = [], start
        for n in sizes:
            out.append(t[at:at + n])
            at += n + start
        return out
    w = torch.randn(total, generator=g, device="cuda") * 0.1
    d = dict(p=spread(w.to(dts[0])), g=spread((torch.randn(total, generator=g, device="cuda") * torch.exp(torch.randn(total, generator=g, device="cuda")) * 1e-2).to(dts[1])),
             master=spread(w.clone()) if master else None)
    if cfg.state_bits == 32:
        d["m"], d["v"] = spread(torch.randn(total, generator=g, device="cuda") * 1e-3), spread(torch.rand(total, generator=g, device="cuda") * 1e-4)
        d["scales"] = None
    else:
        d["m"] = spread((torch.randn(total, generator=g, device="cuda") * 50).to(torch.float8_e4m3fn))
        d["v"] = spread((torch.rand(total, generator=g, device="cuda") * 400 + 0.01).to(torch.float8_e4m3fn))
        d["scales"] = [torch.exp2(torch.randint(-24, -14, ((n + 255) // 256, 2), generator=g, device="cuda").float()) for n in sizes]
    return d


def step(lq, cfg, d, lr, t, **kw):
    lq.lq_adamw_step(cfg, d["p"], d["g"], d["m"], d["v"], lr, t, scales=d["scales"], masters=d["master"], **kw)


def copy(d):
    return {k: None if v is None else [t.clone() for t in v] for k, v in d.items()}


SIZES = [1, 3, 255, 256, 257, 1000, 5, 0, 70000, 12]


@pytest.mark.parametrize("p,g,master", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "f32", True), ("bf16", "bf16", False), ("f32", "f32", True)])
@pytest.mark.parametrize("start", [0, 4, 1])
@pytest.mark.parametrize("t", [1, 2, 1000])
def test_states_in_32_bits(lq, t, start, p, g, master):
    cfg = lq.make_adamw_config(p, g, 32, **HYPER)
    d = make(lq, cfg, SIZES, master, seed=t, start=start)
    e = copy(d)
    step(lq, cfg, d, 1e-2, t)
    for i in range(len(SIZES)):
        want = ref.adamw(e["master"][i] if master else e["p"][i], e["g"][i], e["m"][i], e["v"][i], 1e-2, t, 0.9, 0.999, 1e-8, 0.01)
        ref.check(d["m"][i], want["m"], f"m {i}")
        ref.check(d["v"][i], want["v"], f"v {i}")
        value, off = want["p"]
        ref.check(d["p"][i], (value, off + ref.ROUND[DT[p]] * (value.abs() + off)), f"p {i}")
        if master:
            ref.check(d["master"][i], want["p"], f"master {i}")
            assert torch.equal(d["p"][i], d["master"][i].to(DT[p]))
        assert torch.equal(d["g"][i], e["g"][i])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("start", [1, 5])
def test_what_lies_between_the_tensors_stays(lq, bits, start):
    """A buffer of each kind with marks between its tensors."""
    cfg = lq.make_adamw_config("bf16", "f32", bits, **HYPER)
    d = make(lq, cfg, SIZES, True, start=start)
    bases = {k: d[k][0]._base for k in ("p", "m", "v", "master")}
    inside = torch.zeros(bases["p"].numel(), dtype=torch.bool, device="cuda")
    at = start
    for n in SIZES:
        inside[at:at + n] = True
        at += n + start
    before = {k: b.clone() for k, b in bases.items()}
    step(lq, cfg, d, 1e-2, 3)
    for k, b in bases.items():
        a, c = b.view(torch.uint8 if b.element_size() == 1 else torch.int16 if b.element_size() == 2 else torch.int32), before[k].view(
            torch.uint8 if b.element_size() == 1 else torch.int16 if b.element_size() == 2 else torch.int32)
        assert torch.equal(a[~inside], c[~inside]), k


def eight_bit_rule(cfg, e, lr, t, masters):
    """One step by the rule, every operation an fp32 one rounded by itself, on the CPU."""
    b1, b2 = cfg.beta1, cfg.beta2
    f = torch.float32
    out, at = [], 0
    total = sum((p.numel() + 255) // 256 * 256 for p in e["p"])
    bits_m, bits_v = ref.random_bits(cfg.seed, t, total)
    for i, p in enumerate(e["p"]):
        n = p.numel()
        blocks = (n + 255) // 256

        def padded(x):
            return torch.nn.functional.pad(x.cpu().to(f), (0, blocks * 256 - n)).view(blocks, 256)
        sc = e["scales"][i].cpu()
        g = padded(e["g"][i])
        m, r = padded(e["m"][i]) * sc[:, :1], padded(e["v"][i]) * sc[:, 1:]
        v = r * r
        m = m * torch.tensor(b1, dtype=f) + g * torch.tensor(1 - b1, dtype=f)
        v = v * torch.tensor(b2, dtype=f) + g * torch.tensor(1 - b2, dtype=f) * g
        root = v.double().sqrt().to(f)  # (torch's own fp32 root on the CPU is not the nearest number; that of the 64-bit one is)
        w = slice(at, at + blocks * 256)
        at += blocks * 256
        sm, sv = ref.power_scale(m.abs().amax(1)) if blocks else m.new_ones(0), ref.power_scale(root.amax(1)) if blocks else m.new_ones(0)
        em = torch.copysign(ref.e4m3_random(m.abs() / sm[:, None], bits_m[w].view(blocks, 256)).to(f), m)
        ev = ref.e4m3_random(root / sv[:, None], bits_v[w].view(blocks, 256)).to(f)
        ev = torch.where(v > 0, ev.clamp(min=2.0 ** -9), ev)
        out.append((em.flatten()[:n], ev.flatten()[:n], torch.stack([sm, sv], 1)))
    return out


@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("seed,t", [(0, 1), (12345, 7), (2 ** 32 - 1, 2 ** 31 - 1)])
def test_states_in_8_bits(lq, seed, t, start):
    cfg = lq.make_adamw_config("f32", "f32", 8, seed=seed, **HYPER)
    sizes = SIZES + [300] * 140  # more than a launch's tensors
    d = make(lq, cfg, sizes, seed=3, start=start)
    e = copy(d)
    step(lq, cfg, d, 1e-2, t)
    for i, (m, v, sc) in enumerate(eight_bit_rule(cfg, e, 1e-2, t, False)):
        assert torch.equal(d["scales"][i].cpu(), sc), f"scales {i}"
        assert torch.equal(d["m"][i].cpu().float(), m), f"m {i}"
        assert torch.equal(d["v"][i].cpu().float(), v), f"v {i}"
        n = sizes[i]
        each = e["scales"][i].repeat_interleave(256, 0)[:n].double()
        want = ref.adamw(e["p"][i], e["g"][i], e["m"][i].double() * each[:, 0], (e["v"][i].double() * each[:, 1]) ** 2, 1e-2, t, 0.9, 0.999, 1e-8, 0.01)
        # (the states that come in are products of E4M3 elements and a power of two, squared: off by 2^-24 at most, as v's own sum allows)
        value, off = want["p"]
        ref.check(d["p"][i], (value, off * 1.2 + ref.ROUND[torch.float32] * value.abs()), f"p {i}")


def test_rounding_keeps_the_mean(lq):
    """The same state and gradient under many seeds: the mean of what is held is the value, up to five deviations of the mean."""
    n, tries = 1 << 16, 64
    cfg0 = lq.make_adamw_config("f32", "f32", 8, **HYPER)
    d0 = make(lq, cfg0, [n], seed=5)
    ms, vs = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for seed in range(tries):
        cfg = lq.make_adamw_config("f32", "f32", 8, seed=seed * 7919, **HYPER)
        d = copy(d0)
        step(lq, cfg, d, 0.0, 10)
        each = d["scales"][0].repeat_interleave(256, 0).double()
        ms += d["m"][0].double() * each[:, 0]
        vs += d["v"][0].double() * each[:, 1]
    each = d0["scales"][0].repeat_interleave(256, 0).double()
    m = 0.9 * d0["m"][0].double() * each[:, 0] + 0.1 * d0["g"][0].double()
    root = (0.999 * (d0["v"][0].double() * each[:, 1]) ** 2 + 0.001 * d0["g"][0].double() ** 2).sqrt()
    for got, want, sc in ((ms, m, d["scales"][0][:, 0]), (vs, root, d["scales"][0][:, 1])):
        unit = torch.exp2(torch.floor(torch.log2((want.abs() / sc.repeat_interleave(256).double()).clamp(min=2.0 ** -6)))) / 8 * sc.repeat_interleave(256).double()
        far = (got / tries - want) / unit  # a try is off by less than a step, its deviation at most half of one
        assert float(far.mean().abs()) <= 5 * 0.5 / (n * tries) ** 0.5
        assert float(far.abs().max()) <= 6 * 0.5 / tries ** 0.5  # (6 deviations: 65536 values)


def test_a_value_that_does_not_change_is_held_as_it_was(lq):
    """beta = 0 for neither: without a gradient and with betas next to 1 the average moves by less than its rounding, and stays at its mean; zeros stay zeros."""
    cfg = lq.make_adamw_config("f32", "f32", 8, beta1=0.9, beta2=0.999)
    p = torch.ones(1000, device="cuda")
    m, v, scales = lq.adamw_states(cfg, p)
    for t in range(1, 4):
        lq.lq_adamw_step(cfg, [p], [torch.zeros(1000, device="cuda")], [m], [v], 1e-2, t, scales=[scales])
    assert (m.float() == 0).all() and (v.float() == 0).all() and (scales == 1).all() and (p == 1).all()


def test_a_root_above_zero_is_not_held_as_zero(lq):
    cfg = lq.make_adamw_config("f32", "f32", 8)
    g = torch.full((512,), 1e-12, device="cuda")
    g[0] = g[300] = 1e3
    p = torch.zeros(512, device="cuda")
    m, v, scales = lq.adamw_states(cfg, p)
    lq.lq_adamw_step(cfg, [p], [g], [m], [v], 1e-3, 1, scales=[scales])
    assert (v.float() >= 2.0 ** -9).all()


def test_a_gradient_that_is_not_finite(lq):
    for bits in (32, 8):
        cfg = lq.make_adamw_config("f32", "f32", bits, **HYPER)
        d = make(lq, cfg, [1000])
        e = copy(d)
        d["g"][0][300] = float("nan")
        d["g"][0][700] = float("inf")
        step(lq, cfg, d, 1e-2, 5)
        step(lq, cfg, e, 1e-2, 5)
        fine = torch.ones(1000, dtype=torch.bool, device="cuda")
        fine[[300, 700]] = False
        assert torch.equal(d["p"][0][fine], e["p"][0][fine]) and not torch.isfinite(d["p"][0][[300, 700]]).any()
        if bits == 8:  # the states of its 256 values are not numbers, and are seen to be
            sc = torch.isnan(d["scales"][0]).all(1)
            assert sc.tolist() == [False, True, True, False]
            assert torch.equal(d["m"][0].float()[:256], e["m"][0].float()[:256])


@pytest.mark.parametrize("bits", [32, 8])
def test_the_same_step_by_device_numbers_and_in_a_graph(lq, bits):
    cfg = lq.make_adamw_config("bf16", "bf16", bits, **HYPER)
    sizes = [1000, 256, 70000, 3]
    d = make(lq, cfg, sizes, True)
    e = copy(d)
    lr, t, gs = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            step(lq, cfg, d, lr, t, grad_scale=gs)
    torch.cuda.synchronize()
    for k in range(1, 5):
        lr.fill_(1e-2 / k)
        t.fill_(k * k)
        gs.fill_(1.0 / k)
        graph.replay()
        scaled = dict(e, g=[(x.float() * (1.0 / k)) for x in e["g"]])
        cfg2 = lq.make_adamw_config("bf16", "f32", bits, **HYPER)
        step(lq, cfg2, scaled, float(lr), k * k)
        torch.cuda.synchronize()
        for key in ("p", "master", "m", "v", "scales"):
            for a, b in zip(d[key] or [], e[key] or []):
                assert torch.equal(a.float(), b.float()), (k, key)


def test_repeated_steps_follow_the_formula(lq):
    """Twenty steps of changing gradients: 64-bit averages, each step off by what one step allows and what the steps before left."""
    cfg = lq.make_adamw_config(**HYPER)
    p = torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    m, v, _ = lq.adamw_states(cfg, p)
    want = [p.double(), m.double(), v.double()]
    for t in range(1, 21):
        g = torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(t)) + 0.1
        r = ref.adamw(want[0], g, want[1], want[2], 1e-2, t, 0.9, 0.999, 1e-8, 0.01)
        want = [r[k][0] for k in ("p", "m", "v")]
        lq.lq_adamw_step(cfg, [p], [g], [m], [v], 1e-2, t)
    for got, w in zip((p, m, v), want):  # relative errors of a step are at most 20 * 2^-24, the averages forget them
        assert (got.double() - w).abs().max() <= 20 * 20 * 2.0 ** -24 * w.abs().max()


def test_overlapping_tensors_are_refused(lq):
    cfg = lq.make_adamw_config()
    t = [torch.zeros(100, device="cuda") for _ in range(4)]
    for lists in (([t[0], t[0]], [t[1]] * 2, [t[2], t[2].clone()], [t[3], t[3].clone()]), ([t[0][:60], t[0][50:]], [t[1][:60], t[1][50:]], [t[2][:60], t[2][60:].new_zeros(50)], [t[3][:60], t[3].new_zeros(50)]),
                  ([t[0]], [t[1]], [t[2]], [t[2]])):
        before = [x.clone() for x in t]
        with pytest.raises(lq.LqError) as e:
            lq.lq_adamw_step(cfg, *lists, 1e-3, 1)
        assert e.value.status == lq.LQ_ERR_SHAPE
        assert all(torch.equal(a, b) for a, b in zip(t, before))
    lq.lq_adamw_step(cfg, [], [], [], [], 1e-3, 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_values_past_32_bits(lq, bits):
    """A tensor of more than 2^31 values: its end as a short tensor's (states in 32 bits), or next to it (in 8 bits, whose rounding goes by a value's place)."""
    n, end = 2 ** 31 + 300, 812
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    cfg = lq.make_adamw_config("bf16", "bf16", bits)
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p[-end:], g[-end:] = torch.randn(end, generator=gen, device="cuda").bfloat16(), torch.randn(end, generator=gen, device="cuda").bfloat16()
    short, grad = p[-end:].clone(), g[-end:].clone()
    m, v, scales = lq.adamw_states(cfg, p)
    sm, sv, ss = lq.adamw_states(cfg, short)
    for params, grads, a, b, s in ((p, g, m, v, scales), (short, grad, sm, sv, ss)):
        lq.lq_adamw_step(cfg, [params], [grads], [a], [b], 1e-2, 1, scales=None if s is None else [s])
    assert torch.equal(p[-end:], short) and not p[:end].any()
    if bits == 32:
        assert torch.equal(m[-end:], sm) and torch.equal(v[-end:], sv) and not m[:end].float().any()
    else:
        last = scales[-4:].repeat_interleave(256, 0)[:end]  # (the end begins with a block, at 2^31 - 512)
        for k, (t, want) in enumerate(((m, 0.1 * grad.double()), (v, (0.001 * grad.double().square()).sqrt()))):
            got = t[-end:].double() * last[:, k]
            assert (got - want).abs().max() <= 2.0 ** -3 * want.abs().max() * 1.01


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,decay", [(1e-4, 0.01), (1e-5, 0.01), (3e-4, 0.1), (1e-3, 1e-5), (1e-2, 0.5)])
def test_weight_decay_keeps_small_factors(lq, lr, decay, bits):
    """lr weight_decay down to 1e-8: what is taken from a parameter is that part of it, to the bits of fp32, before the one rounding of the result.  lr and weight_decay are rounded, and their
    product, and its product with the parameter (4 e, e = 2^-24); the step's own part is off by 14 e of itself and 5 e of the sizes that its average is made of."""
    e, n, t = 2.0 ** -24, 70001, 7
    cfg = lq.make_adamw_config("f32", "f32", bits, weight_decay=decay)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for device_lr in (False, True):
        for size in (0.0, 1e-3):
            p, g = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda") * size
            m, v, scales = lq.adamw_states(cfg, p)
            old = p.double()
            lq.lq_adamw_step(cfg, [p], [g], [m], [v], torch.full((1,), lr, device="cuda") if device_lr else lr, t, scales=None if scales is None else [scales])
            mean = 0.1 * g.double() / (1 - 0.9 ** t)
            step = lr * mean / ((0.001 * g.double().square() / (1 - 0.999 ** t)).sqrt() + 1e-8)
            want = old - lr * decay * old - step
            off = ref.SLACK * e * (4 * lr * decay * old.abs() + 20 * step.abs())
            bad = ~((p.double() - want).abs() <= off + e * (want.abs() + off))
            assert not bad.any(), (device_lr, size, int(bad.sum()))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.01])
def test_parameters_that_are_infinite_stay_so(lq, decay, bits):
    """Masked places of a parameter, with gradients of zero."""
    cfg = lq.make_adamw_config("f32", "f32", bits, weight_decay=decay)
    p = torch.ones(300, device="cuda")
    p[5], p[290] = float("-inf"), float("inf")
    m, v, scales = lq.adamw_states(cfg, p)
    lq.lq_adamw_step(cfg, [p], [torch.zeros_like(p)], [m], [v], 1e-2, 1, scales=None if scales is None else [scales])
    assert float(p[5]) == float("-inf") and float(p[290]) == float("inf") and torch.isfinite(p).sum() == 298


def roots_at_a_step(count, seed, t, c2):
    """fp32 gradients g for which the cut part of the nearest root of v = fl(fl(g c2) g), beside the random number that its place is rounded with, decides by its last bit: (g, codes that
    a right root gives, how many of them go up).  In every second place the root's lowest 20 bits and the random number make 2^20, in the others 2^20 - 1."""
    _, bits = ref.random_bits(seed, t, count)
    f, i32 = torch.float32, torch.int32
    gen = torch.Generator().manual_seed(seed)
    top = torch.randint(0, 8, (count,), generator=gen)           # mantissa's first three bits
    e = torch.randint(-5, 8, (count,), generator=gen)            # roots in [2^-5, 2^8): E4M3's normal numbers
    up = torch.arange(count) % 2 == 0
    low = (2 ** 20 - bits - (~up).long()).clamp(min=0)
    low = torch.where(low > 2 ** 20 - 1, torch.zeros_like(low), low)
    root = (((e + 127) << 23) | (top << 20) | low).to(i32).view(f)
    c = torch.tensor(c2, dtype=f)
    near = (root.double() / float(c) ** 0.5).to(f)
    g, hit = torch.zeros(count, dtype=f), torch.zeros(count, dtype=torch.bool)
    for k in range(-6, 7):  # the gradient whose v has this nearest root
        x = (near.view(i32) + k).view(f)
        r = (x * c * x).double().sqrt().to(f)
        found = (r == root) & ~hit
        g, hit = torch.where(found, x, g), hit | found
    g = torch.where(hit, g, torch.ones_like(g))
    r = (g * c * g).double().sqrt().to(f)
    return g, r, bits, hit, up


@pytest.mark.parametrize("size", [0, -40, 40, -52, 52])
@pytest.mark.parametrize("c2", [1.0, 0.25 + 2.0 ** -7, 0.001])
def test_roots_are_the_nearest_numbers(lq, c2, size):
    """The held root of v where its last bit decides which way it is rounded: a root that is one bit too small is seen in one half of the places, one that is too large in the other.  Gradients
    times 2^size, which the blocks' scales take up."""
    blocks, seed, t = 2000, 77, 3
    n = blocks * 256
    cfg = lq.make_adamw_config("f32", "f32", 8, beta1=0.0, beta2=1.0 - c2, seed=seed)
    c2 = 1.0 - cfg.beta2
    g, root, bits, hit, up = roots_at_a_step(n, seed, t, c2)
    assert float(hit.double().mean()) > 0.4 and float((hit & up).double().mean()) > 0.15 and float((hit & ~up).double().mean()) > 0.15
    last = g.view(blocks, 256)[:, -1]
    last.copy_((torch.full((blocks,), 448.0, dtype=torch.float64) / c2 ** 0.5 * 0.99).float())  # a large value: every block's scale is 1
    root = (g * torch.tensor(c2, dtype=torch.float32) * g).double().sqrt().float()
    p = torch.zeros(n, device="cuda")
    m, v, scales = lq.adamw_states(cfg, p)
    lq.lq_adamw_step(cfg, [p], [g.cuda() * 2.0 ** size], [m], [v], 1e-3, t, scales=[scales])
    assert (scales[:, 1] == 2.0 ** size).all()
    assert torch.equal(v.float().cpu().double(), ref.e4m3_random(root, bits))
