"""The operators around a block run together: modulation from 4-bit weights, the block before added and normalised, their gradients, the AdamW step; each step against its plain
form on what the step before left, and a training step captured and replayed."""
import pytest
import torch

from tests import blocks_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    from paper_2604_18117_amd import binding
    return binding


def normal(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape: torch.randn(shape, generator=g, device="cuda")


@pytest.mark.parametrize("images,side,dim,emb", [(3, 6, 256, 256), (2, 5, 100, 33), (1, 1, 1152, 1152)])
def test_entrance(lq, images, side, dim, emb):
    """The example's entrance, forward and backward, with rows of no image behind the last."""
    from paper_2604_18117_amd import adapted_qkv as ex
    rnd, M = normal(0), images * side * side
    offsets = torch.arange(images + 1, dtype=torch.int32, device="cuda") * side * side
    enter = ex.Entrance(rnd(3 * dim, emb) * 0.05, offsets, rnd(3 * dim))
    codes, scales = lq.lq_w4_unpack(enter.cfg, enter.packed)
    e, h0, y, dh0, dx0 = rnd(images, emb), *(rnd(M + 2, dim).bfloat16() for _ in range(4))
    h, X = h0.clone(), torch.zeros_like(h0)
    assert enter(e, h, y, X)[1] is X
    ref.check(enter.mod, ref.w4_fwd(e, codes, scales, 64, enter.bias, torch.float32), "modulation")
    gate, scale, shift = enter.parts(enter.mod)
    want = ref.block_fwd(h0, y, offsets, gate, scale, shift, None, None, "none", "layer", enter.norm.eps, 1.0, X.dtype)
    ref.check(h[:M], want["ho"], "stream")
    ref.check(X[:M], want["x"], "rows")
    assert torch.equal(h[M:], h0[M:]) and not X[M:].any()
    # gradients, in the place of what comes in
    dh, dx = dh0.clone(), dx0.clone()
    _, _, demb = enter.backward(h, y, dh, dx)
    grads = ref.block_bwd(h, y, offsets, gate, scale, None, None, dh0, dx0, "none", "layer", enter.norm.eps, 1.0, h.dtype, y.dtype)
    ref.check(dh[:M], grads["dh"], "dh")
    ref.check(dx[:M], grads["dy"], "dy")
    assert torch.equal(dh[M:], dh0[M:]) and torch.equal(dx[M:], dx0[M:])
    dmod = torch.cat(lq.lq_block_norm_bwd(enter.norm, h, y, offsets, gate, scale, dho=dh0, dx=dx0)[2:5], 1)
    for k, name in enumerate(("dgate", "dscale", "dshift")):
        ref.check(dmod[:, k * dim:(k + 1) * dim], grads[name], name)
    ref.check(demb, ref.w4_bwd(dmod, codes, scales, 64, torch.float32), "demb")


class Fit:
    """Embeddings and the two norms' weights learn to give wanted rows: all of a step on one stream, the step's number on the device."""

    def __init__(self, lq, bits, images=3, rows=21, dim=200, emb=72):
        rnd, M = normal(1), images * rows
        self.lq, self.dim = lq, dim
        self.offsets = torch.arange(images + 1, dtype=torch.int32, device="cuda") * rows
        self.cfg = lq.make_w4_config(3 * dim, emb, 64, "f32", "f32")
        self.packed = lq.lq_w4_pack(self.cfg, rnd(3 * dim, emb) * 0.05)
        self.norm = lq.make_block_config(dim, "rms", "layer", h_dtype="f32", y_dtype="bf16")
        self.h, self.y, self.want = rnd(M, dim), rnd(M, dim).bfloat16(), rnd(M, dim).bfloat16()
        self.params = [rnd(images, emb), torch.ones(dim, device="cuda"), torch.ones(dim, device="cuda")]
        self.adamw = lq.make_adamw_config(state_bits=bits, weight_decay=0.01, seed=7)
        self.m, self.v, self.scales = map(list, zip(*(lq.adamw_states(self.adamw, p) for p in self.params)))
        self.number = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.mod, self.dmod = torch.empty(images, 3 * dim, device="cuda"), torch.empty(images, 3 * dim, device="cuda")
        self.ho, self.x = torch.empty_like(self.h), torch.empty_like(self.y)
        self.dh, self.dy = torch.empty_like(self.h), torch.empty_like(self.y)
        self.grads = [torch.empty_like(p) for p in self.params]
        self.work = torch.empty(lq.lq_block_work_sizes(self.norm, M, images), dtype=torch.uint8, device="cuda")
        self.w4_work = torch.empty(lq.lq_w4_work_sizes(self.cfg, images), dtype=torch.uint8, device="cuda")

    def parts(self, t):
        return [t[:, k * self.dim:(k + 1) * self.dim] for k in range(3)]

    def gradients(self):
        lq, (e, w_post, w_pre), (de, dw_post, dw_pre) = self.lq, self.params, self.grads
        (gate, scale, shift), (dgate, dscale, dshift) = self.parts(self.mod), self.parts(self.dmod)
        lq.lq_w4_fwd(self.cfg, self.packed, e, Y=self.mod)
        lq.lq_block_norm_fwd(self.norm, self.h, self.y, self.offsets, gate, scale, shift, w_post, w_pre, ho=self.ho, x=self.x)
        lq.lq_block_norm_bwd(self.norm, self.ho, self.y, self.offsets, gate, scale, w_post, w_pre, dx=self.x - self.want, dh=self.dh, dy=self.dy, dgate=dgate,
                             dscale=dscale, dshift=dshift, dw_post=dw_post, dw_pre=dw_pre, work=self.work)
        lq.lq_w4_bwd(self.cfg, self.packed, self.dmod, dX=de, work=self.w4_work)

    def step(self):
        self.number += 1
        self.gradients()
        self.lq.lq_adamw_step(self.adamw, self.params, self.grads, self.m, self.v, 1e-2, self.number, scales=None if self.scales[0] is None else self.scales)

    def state(self):
        return [t.clone() for t in self.params] + [t.view(torch.uint8).clone() for t in self.m + self.v] + [t.clone() for t in self.scales if t is not None]


def rows_64(fit, e, w_post, w_pre):
    """The formulas' rows in 64 bits."""
    codes, scales = fit.lq.lq_w4_unpack(fit.cfg, fit.packed)
    mod = e.double() @ ref.w4_weights(codes, scales, 64).t()
    gate, scale, shift = (t[ref.rows_of(fit.offsets, fit.h.shape[0], fit.h.device)] for t in fit.parts(mod))
    y, eps = fit.y.double(), fit.norm.eps
    h = fit.h.double() + gate * w_post.double() * y / (y.square().mean(1, keepdim=True) + eps).sqrt()
    c = h - h.mean(1, keepdim=True)
    return c / (c.square().mean(1, keepdim=True) + eps).sqrt() * w_pre.double() * (1 + scale) + shift


def test_gradients_of_the_run_against_differences(lq):
    """Of 0.5 sum (x - want)^2 along a random direction of all three parameters at once.  x and x - want are rounded to bf16, each by 2^-8 of its value, so that the sum of
    (x - want) times the change of x is off by at most 2^-8 of the sum of (|x| + |x - want|) |change|; all else is fp32 and adds less than as much again."""
    fit = Fit(lq, 32)
    fit.gradients()
    rnd, s, want = normal(5), 1e-6, fit.want.double()
    d = [rnd(*p.shape).double() for p in fit.params]
    got = sum((g.double() * q).sum() for g, q in zip(fit.grads, d))
    above, below = (rows_64(fit, *(p.double() + t * q for p, q in zip(fit.params, d))) for t in (s, -s))
    slope = 0.5 * ((above - want).square() - (below - want).square()).sum() / (2 * s)
    change, x = ((above - below) / (2 * s)).abs(), (above + below) / 2
    bound = 2 * 2.0 ** -8 * ((x.abs() + (x - want).abs()) * change).sum()
    assert (got - slope).abs() <= bound, (float(got), float(slope), float(bound))


@pytest.mark.parametrize("bits", [32, 8])
def test_training_step_captured_and_replayed(lq, bits):
    """The whole step as one graph, replayed with eager work of another fit between the replays: every state as after eager steps."""
    eager, fit = Fit(lq, bits), Fit(lq, bits)
    first = eager.state()
    eager.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fit.step()
        assert all(torch.equal(a, b) for a, b in zip(fit.state(), eager.state()))
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fit.step()
    for _ in range(4):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(fit.state(), eager.state()))
    assert int(fit.number) == 5 and all(not torch.equal(a, b) for a, b in zip(eager.params, first))


def test_steps_follow_the_formula(lq):
    """Three steps, each against the formula's from the gradients that were there (the bound of a step, and the parameter's rounding)."""
    fit = Fit(lq, 32)
    for t in range(1, 4):
        before = [(p.clone(), m.clone(), v.clone()) for p, m, v in zip(fit.params, fit.m, fit.v)]
        fit.step()
        for (p, m, v), g, p1, m1, v1 in zip(before, fit.grads, fit.params, fit.m, fit.v):
            want = ref.adamw(p, g, m, v, 1e-2, t, 0.9, 0.999, 1e-8, 0.01)
            for name, got in (("p", p1), ("m", m1), ("v", v1)):
                value, off = want[name]
                ref.check(got, (value, off + 2.0 ** -24 * (value.abs() + off)), f"{name} of step {t}")


@pytest.mark.parametrize("given", [False, True])
def test_entrance_with_two_batches_under_way(lq, given):
    """Two calls before their gradients: each backward takes the modulation of its own call."""
    from paper_2604_18117_amd import adapted_qkv as ex
    images, rows, dim, emb = 3, 11, 100, 48
    rnd, M = normal(2), images * rows
    enter = ex.Entrance(rnd(3 * dim, emb) * 0.05, torch.arange(images + 1, dtype=torch.int32, device="cuda") * rows, rnd(3 * dim))
    batches = []
    for _ in range(2):
        e, h, y, dh, dx = rnd(images, emb), *(rnd(M, dim).bfloat16() for _ in range(4))
        mod = torch.empty(images, 3 * dim, device="cuda") if given else None
        h0 = h.clone()
        enter(e, h, y, mod=mod)
        batches.append((e, h0, h, y, dh, dx, enter.mod))
        assert not given or enter.mod is mod
    with pytest.raises(ValueError):  # whose?
        enter.backward(batches[0][2], batches[0][3], batches[0][4].clone(), batches[0][5].clone())
    got = []
    for _, _, h, y, dh, dx, mod in reversed(batches):
        got.insert(0, enter.backward(h, y, dh.clone(), dx.clone(), mod=mod))
        with pytest.raises(ValueError):  # the other call's is not the last one
            enter.backward(h, y, dh.clone(), dx.clone())
    for (e, h0, h, y, dh, dx, mod), have in zip(batches, got):
        alone = ex.Entrance(torch.zeros(3 * dim, emb, device="cuda"), enter.offsets, enter.bias)
        alone.packed = enter.packed
        again = h0.clone()
        alone(e, again, y)
        assert torch.equal(again, h) and torch.equal(alone.mod, mod)
        for _ in range(2):
            for a, b in zip(have, alone.backward(again, y, dh.clone(), dx.clone())):
                assert torch.equal(a, b)
    with pytest.raises(ValueError):  # a call's modulation without a call
        ex.Entrance(torch.zeros(3 * dim, emb, device="cuda"), enter.offsets).backward(h, y, dh, dx)
