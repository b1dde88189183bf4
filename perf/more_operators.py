"""What the operators around the quantised projections of a transformer block are measured with: the product of a few rows with 4-bit weights and group
scales (the conditioning vector's layers; forward, gradient), the norms before and after a block with its gate, residual scale and modulation for each
sequence (forward, gradient), and an AdamW step over many tensors with states in 32 or in 8 bits.

Widths and token counts are those of the repository's layers (`paper_2604_18117_amd.workloads`: a 1152-wide and a 2240-wide transformer, two images of 64 x 64
patches, 300 tokens of a prompt), from one row to the batches of its benchmark.  `own` chooses between the framework's operators and their plain form.
"""
import math
import random

import torch

own = False

_BLOCK = 256            # values of an 8-bit state that share a scale
_BETAS = (0.9, 0.999)
_ADAM_EPS, _DECAY, _LR = 1e-8, 0.01, 1e-4
_NORM_EPS = 1e-6


def _w4(name, kind, M, K, N, group, x="bf16", y="bf16", bias=True):
    """x, y: types of the rows that go in and come out (the gradient goes from y's to x's)."""
    return dict(name=name, kind=kind, M=M, K=K, N=N, group=group, x=x, y=y, bias=bias)


def _block(name, kind, M, D, seqs, post="none", pre="layer", stream="bf16", branch="bf16", weights=False, tail=0, alpha=1.0):
    """post, pre: norm of the branch's output before it is added, norm of the sum for the next block ("none", "rms", "layer").  weights: the norms have them.
    tail: rows behind the last sequence (of a padded batch), which stay as they are.  alpha: scale of the residual."""
    return dict(name=name, kind=kind, M=M, D=D, seqs=seqs, post=post, pre=pre, stream=stream, branch=branch, weights=weights, tail=tail, alpha=alpha)


def _adamw(name, sizes, bits, p="f32", master=False, g="f32"):
    """sizes: "count x values" of tensors, joined by "+"."""
    return dict(name=name, kind="adamw", sizes=sizes, bits=bits, p=p, master=master, g=g)


def listed():
    return [
        # a timestep's features into the conditioning vector's first layer: the smallest product
        _w4("w4_timestep", "w4", 1, 256, 1152, 64, x="f32", y="f32"),
        # six vectors of modulation of the 1152-wide transformer for the two images of a batch
        _w4("w4_modulation1152", "w4", 2, 1152, 6912, 64, y="f32"),
        # the expansion of the 2240-wide transformer for single tokens of 64 requests
        _w4("w4_tokens2240", "w4", 64, 2240, 11200, 64),
        # gradient of the conditioning vectors through the modulation's layer
        _w4("w4_modulation1152_grad", "w4_grad", 2, 1152, 6912, 64, y="f32"),
        # ... and of 16 vectors through that of the 2240-wide transformer
        _w4("w4_modulation2240_grad", "w4_grad", 16, 2240, 13440, 128, y="f32"),
        # one token between two blocks
        _block("block_token", "block", 1, 1152, 1, stream="f32"),
        # two images of 64 x 64 patches of the 1152-wide transformer
        _block("block_image", "block", 8192, 1152, 2),
        # ragged sequences of the 2240-wide transformer, a norm on both sides of the block, padded batch: the largest
        _block("block_sandwich2240", "block", 16384, 2240, 7, post="rms", pre="rms", stream="f32", weights=True, tail=113),
        # the gradient of the image batch
        _block("block_image_grad", "block_grad", 8192, 1152, 2),
        # ... and of prompts of a few requests, 32-bit, a norm on both sides
        _block("block_prompt_grad", "block_grad", 300, 1152, 7, post="rms", pre="layer", stream="f32", branch="f32", weights=True, tail=5),
        # the adapters of one fused QKV layer (four of rank 32): bf16 factors with 32-bit masters
        _adamw("adamw_adapters", "4x36864+4x110592", 32, p="bf16", master=True),
        # adapters of rank 32 on the linears of 28 blocks of the 1152-wide transformer, and small vectors beside them, states in 8 bits
        _adamw("adamw_blocks8", "112x36864+28x110592+28x147456+56x1152+5x37", 8),
    ]


def _log(rng, lo, hi, mul=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / mul)) * mul))


def draw(rng):
    kind = rng.choices(["w4", "w4_grad", "block", "block_grad", "adamw"], [25, 15, 25, 20, 15])[0]
    if kind.startswith("w4"):
        K, N = _log(rng, 64, 4608, rng.choice([1, 8, 64])), _log(rng, 64, 13440, rng.choice([1, 8, 64]))
        M = _log(rng, 1, 64 if kind == "w4" else 16)
        d = _w4("", kind, M, K, N, rng.choice([32, 64, 128]), x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.5)
    elif kind.startswith("block"):
        D = _log(rng, 48, 4608, rng.choice([1, 8, 32, 64]))
        M = _log(rng, 1, 16384)
        M = max(1, min(M, int((16384 * 2240.0 if kind == "block" else 8192 * 1152.0) / D)))
        stream = rng.choice(["bf16", "f32"])
        d = _block("", kind, M, D, _log(rng, 1, max(1, min(64, M))), post=rng.choice(["none", "none", "rms", "layer"]), pre=rng.choice(["layer", "rms"]), stream=stream,
                   branch="bf16" if stream == "bf16" else rng.choice(["bf16", "f32"]), weights=rng.random() < 0.5,
                   tail=rng.randint(0, M // 8) if rng.random() < 0.3 else 0, alpha=rng.choice([1.0, 1.0, 0.5]))
    else:
        room, parts = 12e6, []
        for _ in range(rng.randint(1, 4)):
            n = _log(rng, 1, 4000000)
            count = _log(rng, 1, max(1, int(min(200, room / n))))
            if count * n <= room:
                room -= count * n
                parts.append("%dx%d" % (count, n))
        p = rng.choice(["f32", "bf16"])
        d = _adamw("", "+".join(parts or ["1x1152"]), rng.choice([32, 8]), p=p, master=p == "bf16" and rng.random() < 0.7, g=rng.choice(["f32", "bf16"]))
    del d["name"]
    return d


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---- inputs ------------------------------------------------------------------------------------

def _w4_inputs(case, seed):
    g = _generator(seed)
    M, K, N, G = case["M"], case["K"], case["N"], -(-case["K"] // case["group"])
    W = torch.randn(N, K, generator=g, device="cuda") * 0.02
    # symmetric 4-bit codes, a scale for each group along K: the largest magnitude becomes 7
    groups = torch.nn.functional.pad(W, (0, G * case["group"] - K)).view(N, G, case["group"])
    scales = groups.abs().amax(-1) / 7
    codes = (groups / scales[:, :, None]).round().clamp(-7, 7).view(N, -1)[:, :K].to(torch.int8).contiguous()
    s = dict(codes=codes, scales=scales)
    if case["kind"] == "w4":
        x = torch.randn(M, K, generator=g, device="cuda")
        s["X"] = (x * torch.sigmoid(x)).to(_type(case["x"]))  # what an activation leaves: mostly small negative and some larger positive values
        s["bias"] = torch.randn(N, generator=g, device="cuda") * 0.02 if case["bias"] else None
    else:
        s["dY"] = (torch.randn(M, N, generator=g, device="cuda") * 1e-2).to(_type(case["y"]))
    return s


def _block_inputs(case, seed):
    g, rng = _generator(seed), random.Random(seed)
    M, D, S = case["M"], case["D"], case["seqs"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    rows = M - case["tail"]
    cuts = sorted(rng.randint(0, rows) for _ in range(S - 1)) if S > 2 else [rows // 2] * (S - 1)  # (two: equal images)
    h = normal(M, D) * 2.0 + 0.3
    h[:, torch.randperm(D, generator=g, device="cuda")[: max(1, D // 100)]] *= 8.0  # strong channels of the residual stream
    mod = normal(S, 6 * D) * 0.3  # shift, scale, gate of two blocks, side by side as their layer gives them
    s = dict(offsets=torch.tensor([0] + cuts + [rows], dtype=torch.int32).cuda(), h=h.to(_type(case["stream"])), y=normal(M, D).to(_type(case["branch"])),
             shift=mod[:, :D], scale=mod[:, D:2 * D], gate=mod[:, 2 * D:3 * D])
    s["w_post"] = 1.0 + 0.2 * normal(D) if case["weights"] and case["post"] != "none" else None
    s["w_pre"] = 1.0 + 0.2 * normal(D) if case["weights"] and case["pre"] != "none" else None
    if case["kind"] == "block_grad":  # h is then the sum that the forward left
        s["dx"], s["dho"] = (normal(M, D) * 1e-2).to(_type(case["branch"])), (normal(M, D) * 1e-2).to(_type(case["stream"]))
    return s


def _counts(case):
    return [int(n) for part in case["sizes"].split("+") for c, n in [part.split("x")] for _ in range(int(c))]


def _padded(n):
    return -(-n // _BLOCK) * _BLOCK


def _power_scale(amax):
    """The smallest power of two that brings amax to 448, the largest value of E4M3, or below; 1 for 0."""
    bits = amax.contiguous().view(torch.int32)
    e = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()  # its exponent's field
    return torch.where(amax > 0, (e.clamp(min=1) << 23).view(torch.float32), 1.0)


def _adamw_inputs(case, seed):
    """All tensors lie in one buffer of each kind, every one from a multiple of 256 on (what is between them is zero and stays it)."""
    g, rng = _generator(seed), random.Random(seed)
    counts = _counts(case)
    total = sum(map(_padded, counts))
    inside = torch.zeros(total, dtype=torch.bool)
    starts, at = [], 0
    for n in counts:
        starts.append(at)
        inside[at:at + n] = True
        at += _padded(n)
    inside = inside.cuda()

    def normal(scale):
        return torch.randn(total, generator=g, device="cuda") * scale * inside
    p = normal(0.05)
    s = dict(counts=counts, starts=starts, master=p if case["master"] else None, p=p.to(_type(case["p"])), t=rng.randint(20, 2000), seed=seed & 0xFFFF)
    size = torch.exp(torch.randn(total, generator=g, device="cuda"))  # sizes of the gradients differ from value to value
    s["g"] = (normal(1e-3) * size).to(_type(case["g"]))
    m, root = normal(4e-4) * size, size * 1e-3 * inside
    if case["bits"] == 32:
        s.update(m=m, v=root * root)
    else:
        mb, rb = m.view(-1, _BLOCK), root.view(-1, _BLOCK)
        scales = torch.stack([_power_scale(mb.abs().amax(1)), _power_scale(rb.amax(1))], 1)
        s.update(m=(mb / scales[:, :1]).to(torch.float8_e4m3fn).view(-1), v=(rb / scales[:, 1:]).to(torch.float8_e4m3fn).view(-1), scales=scales)
    return s


def _inputs(case, seed):
    make = _w4_inputs if case["kind"].startswith("w4") else _adamw_inputs if case["kind"] == "adamw" else _block_inputs
    return dict(make(case, seed), case=case, kind=case["kind"])


def prepare(case, seed):
    """The inputs; for the framework's operators also the packed weights, configurations, workspaces and outputs that a program keeps."""
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2604_18117_amd import binding as lq
    s["lq"] = lq
    if case["kind"].startswith("w4"):
        M = case["M"]
        cfg = lq.make_w4_config(case["N"], case["K"], case["group"], case["x"], case["y"])
        s.update(cfg=cfg, packed=lq.lq_w4_pack_codes(cfg, s["codes"], s["scales"]))
        if case["kind"] == "w4":
            s["Y"] = torch.empty(M, case["N"], dtype=_type(case["y"]), device="cuda")
        else:
            s.update(dX=torch.empty(M, case["K"], dtype=_type(case["x"]), device="cuda"), work=torch.empty(lq.lq_w4_work_sizes(cfg, M), dtype=torch.uint8, device="cuda"))
    elif case["kind"] == "adamw":
        def views(t):
            return None if t is None else [t[a:a + n] for a, n in zip(s["starts"], s["counts"])]
        s["cfg"] = lq.make_adamw_config(case["p"], case["g"], case["bits"], _BETAS[0], _BETAS[1], _ADAM_EPS, _DECAY, s["seed"])
        s["lists"] = [views(s[k]) for k in ("p", "g", "m", "v")]
        s["masters"] = views(s["master"])
        s["scale_list"] = [s["scales"][a // _BLOCK:(a + _padded(n)) // _BLOCK] for a, n in zip(s["starts"], s["counts"])] if case["bits"] == 8 else None
    else:
        M, D, S = case["M"], case["D"], case["seqs"]
        cfg = lq.make_block_config(D, case["post"], case["pre"], _NORM_EPS, case["alpha"], case["stream"], case["branch"])
        s.update(cfg=cfg, out=[torch.zeros_like(s["h"]), torch.zeros_like(s["y"])])
        if case["kind"] == "block_grad":
            s["dmod"] = torch.empty(S, 6 * D, device="cuda")
            s["dw"] = [None if s[k] is None else torch.empty(D, device="cuda") for k in ("w_post", "w_pre")]
            s["work"] = torch.empty(lq.lq_block_work_sizes(cfg, M, S), dtype=torch.uint8, device="cuda")
    return s


# ---- the framework's operators ---------------------------------------------------------------

def _run_own(s):
    lq, cfg = s["lq"], s["cfg"]
    if s["kind"] == "w4":
        return lq.lq_w4_fwd(cfg, s["packed"], s["X"], s["bias"], Y=s["Y"])
    if s["kind"] == "w4_grad":
        return lq.lq_w4_bwd(cfg, s["packed"], s["dY"], dX=s["dX"], work=s["work"])
    if s["kind"] == "block":
        ho, x = lq.lq_block_norm_fwd(cfg, s["h"], s["y"], s["offsets"], s["gate"], s["scale"], s["shift"], s["w_post"], s["w_pre"], ho=s["out"][0], x=s["out"][1])
        return dict(ho=ho, x=x)
    if s["kind"] == "block_grad":
        D, d = s["case"]["D"], s["dmod"]
        grads = lq.lq_block_norm_bwd(cfg, s["h"], s["y"], s["offsets"], s["gate"], s["scale"], s["w_post"], s["w_pre"], s["dho"], s["dx"], dh=s["out"][0],
                                     dy=s["out"][1], dgate=d[:, 2 * D:3 * D], dscale=d[:, D:2 * D], dshift=d[:, :D], dw_post=s["dw"][0], dw_pre=s["dw"][1],
                                     work=s["work"])
        return dict(zip(("dh", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre"), grads))
    s["t"] += 1
    lq.lq_adamw_step(cfg, *s["lists"], _LR, s["t"], scales=s["scale_list"], masters=s["masters"])
    return {k: s[k] for k in ("p", "master", "m", "v", "scales") if s.get(k) is not None}


# ---- their plain form ------------------------------------------------------------------------

def _plain_w4(s):
    case = s["case"]
    W = s["codes"].float() * s["scales"].repeat_interleave(case["group"], 1)[:, :case["K"]]
    if s["kind"] == "w4_grad":
        return (s["dY"].float() @ W).to(_type(case["x"]))
    y = s["X"].float() @ W.t()
    return (y if s["bias"] is None else y + s["bias"]).to(_type(case["y"]))


def _rows(s):
    """Sequence of each row, which rows have one, and the rows of each as a matrix of zeros and ones."""
    row = torch.arange(s["case"]["M"], device="cuda")
    past = row[:, None] >= s["offsets"][1:]
    seq = past.sum(1)
    has = (seq < s["case"]["seqs"])[:, None]
    return seq.clamp(max=s["case"]["seqs"] - 1), has, (torch.arange(s["case"]["seqs"], device="cuda")[:, None] == seq).float()


def _plain_norm(kind, x):
    """(the normalised rows, 1 / deviation)"""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _NORM_EPS)
    return x * r, r


def _plain_norm_grad(kind, n, r, dn):
    if kind == "none":
        return dn
    g = dn - n * (dn * n).mean(-1, keepdim=True)
    if kind == "layer":
        g = g - dn.mean(-1, keepdim=True)
    return r * g


def _weighted(x, w):
    return x if w is None else x * w


def _plain_block(s):
    case = s["case"]
    seq, has, _ = _rows(s)
    p = _weighted(_plain_norm(case["post"], s["y"].float())[0], s["w_post"])
    ho = case["alpha"] * s["h"].float() + s["gate"][seq] * p
    x = _weighted(_plain_norm(case["pre"], ho)[0], s["w_pre"]) * (1.0 + s["scale"][seq]) + s["shift"][seq]
    return dict(ho=(ho * has).to(s["h"].dtype), x=(x * has).to(s["y"].dtype))


def _plain_block_grad(s):
    case = s["case"]
    seq, has, member = _rows(s)
    n, r = _plain_norm(case["pre"], s["h"].float())
    ny, ry = _plain_norm(case["post"], s["y"].float())
    dx = s["dx"].float() * has
    q = member @ (dx * n)  # for each sequence
    dho = s["dho"].float() * has + _plain_norm_grad(case["pre"], n, r, _weighted(dx * (1.0 + s["scale"][seq]), s["w_pre"]))
    t = member @ (dho * ny)
    dy = _plain_norm_grad(case["post"], ny, ry, _weighted(dho * s["gate"][seq], s["w_post"]))
    out = dict(dh=(case["alpha"] * dho).to(s["h"].dtype), dy=dy.to(s["y"].dtype), dgate=_weighted(t, s["w_post"]), dscale=_weighted(q, s["w_pre"]), dshift=member @ dx)
    if s["w_post"] is not None:
        out["dw_post"] = (s["gate"] * t).sum(0)
    if s["w_pre"] is not None:
        out["dw_pre"] = ((1.0 + s["scale"]) * q).sum(0)
    return out


def _random_bits(s, n):
    """Two 20-bit numbers for each place of the buffers, from the seed, the step and the place: products of 32-bit numbers (wrapped) and shifts."""
    def shift(x, k):  # of 32 bits without a sign
        return (x >> k) & ((1 << (32 - k)) - 1)
    key = (s["seed"] * 0x9E3779B1 + s["t"] * 0x6A09E667) & 0xFFFFFFFF
    h = torch.arange(n, dtype=torch.int32, device="cuda") ^ (key - (1 << 32) if key >> 31 else key)
    h = h * (0x9E3779B1 - (1 << 32))
    h = (h ^ shift(h, 16)) * 0x6A09E667
    h = (h ^ shift(h, 15)) * (0xBB67AE85 - (1 << 32))
    h = h ^ shift(h, 16)
    other = h * 0x3C6EF373
    return h & 0xFFFFF, shift(other, 12)


def _round_e4m3(x, bits):
    """x (0 <= x <= 448) to one of the E4M3 values next to it, the upper one with the probability that keeps the mean.  Below 2^-6 they are 2^-9 apart, as they are
    from 2^-6 to 2^-5."""
    small = (x < 0.015625).float() * 0.015625
    return (((x + small).view(torch.int32) + bits) & ~0xFFFFF).view(torch.float32) - small


def _encode(x, bits):
    """(elements, their blocks' scales)"""
    mag = x.abs().view(-1, _BLOCK)
    scale = _power_scale(mag.amax(1))
    q = _round_e4m3((mag / scale[:, None]).view(-1), bits)
    return torch.copysign(q, x), scale


def _plain_adamw(s):
    case, (b1, b2) = s["case"], _BETAS
    s["t"] += 1
    g = s["g"].float()
    p = (s["p"] if s["master"] is None else s["master"]).float()
    m, v = s["m"].float(), s["v"].float()
    if case["bits"] == 8:
        each = s["scales"].repeat_interleave(_BLOCK, 0)
        m, v = m * each[:, 0], (v * each[:, 1]) ** 2
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * (1.0 - b2) * g
    p = p * (1.0 - _LR * _DECAY) - _LR * (m / (1.0 - b1 ** s["t"])) / (torch.sqrt(v / (1.0 - b2 ** s["t"])) + _ADAM_EPS)
    if case["bits"] == 8:
        bits_m, bits_v = _random_bits(s, m.numel())
        m, sm = _encode(m, bits_m)
        r, sv = _encode(torch.sqrt(v), bits_v)
        r = torch.where(v > 0, r.clamp(min=2.0 ** -9), r)  # a root that is not zero is not held as zero
        m, v, s["scales"] = m.to(torch.float8_e4m3fn), r.to(torch.float8_e4m3fn), torch.stack([sm, sv], 1)
    s["m"], s["v"], s["p"] = m, v, p.to(s["p"].dtype)
    if s["master"] is not None:
        s["master"] = p
    return {k: s[k] for k in ("p", "master", "m", "v", "scales") if s.get(k) is not None}


def run(s):
    if own:
        return _run_own(s)
    if s["kind"].startswith("w4"):
        return _plain_w4(s)
    return _plain_adamw(s) if s["kind"] == "adamw" else _plain_block(s) if s["kind"] == "block" else _plain_block_grad(s)


def _bytes_of(name):
    return 4.0 if name == "f32" else 2.0


def work(case):
    if case["kind"].startswith("w4"):
        M, K, N = case["M"], case["K"], case["N"]
        b = N * K / 2.0 + 4.0 * N * -(-K // case["group"]) + M * (K * _bytes_of(case["x"]) + N * _bytes_of(case["y"])) + (4.0 * N if case["kind"] == "w4" and case["bias"] else 0.0)
        return {"bytes": b, "flops": 2.0 * M * N * K}
    if case["kind"] == "adamw":
        n = float(sum(_counts(case)))
        p = 2.0 * _bytes_of(case["p"]) if not case["master"] else _bytes_of(case["p"]) + 8.0  # (with a 32-bit master the small copy is written only)
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / _BLOCK
        return {"bytes": n * (p + _bytes_of(case["g"]) + state), "flops": 14.0 * n}
    n = float(case["M"] - case["tail"]) * case["D"]
    hb, yb = _bytes_of(case["stream"]), _bytes_of(case["branch"])
    norms = sum({"none": 0.0, "rms": 3.0, "layer": 5.0}[case[k]] for k in ("post", "pre"))
    if case["kind"] == "block":
        return {"bytes": n * 2.0 * (hb + yb) + 12.0 * case["seqs"] * case["D"], "flops": n * (5.0 + norms)}
    return {"bytes": n * 3.0 * (hb + yb) + 20.0 * case["seqs"] * case["D"], "flops": n * (12.0 + 3.0 * norms)}


# ---- from the definitions, in 64 bits ----------------------------------------------------------

def _exact_w4(s):
    f = torch.float64
    G = s["scales"].shape[1]
    group, K = s["case"]["group"], s["case"]["K"]
    parts = []
    if s["kind"] == "w4":
        Y = torch.zeros(s["X"].shape[0], s["codes"].shape[0], dtype=f, device="cuda")
        for k in range(G):  # group by group: its product, times its scales
            a = slice(k * group, min(K, (k + 1) * group))
            Y += torch.matmul(s["X"][:, a].to(f), s["codes"][:, a].to(f).transpose(0, 1)) * s["scales"][:, k].to(f)
        return Y if s["bias"] is None else Y + s["bias"].to(f)
    for k in range(G):
        a = slice(k * group, min(K, (k + 1) * group))
        parts.append(torch.matmul(s["dY"].to(f) * s["scales"][:, k].to(f), s["codes"][:, a].to(f)))
    return torch.cat(parts, 1)


def _exact_norm(kind, x):
    if kind == "none":
        return x
    mean = x.sum(-1, keepdim=True) / x.shape[-1] if kind == "layer" else 0.0
    return (x - mean) / (((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1] + _NORM_EPS).sqrt()


def _exact_block(s):
    """Sequence by sequence; the gradients by differentiating the definition."""
    f, case = torch.float64, s["case"]
    train = s["kind"] == "block_grad"
    at = s["offsets"].tolist()
    one = torch.ones(case["D"], dtype=f, device="cuda")
    w_post, w_pre = (one if s[k] is None else s[k].to(f) for k in ("w_post", "w_pre"))
    first, second = torch.zeros(s["h"].shape, dtype=f, device="cuda"), torch.zeros(s["y"].shape, dtype=f, device="cuda")
    dgate, dscale, dshift = (torch.zeros(case["seqs"], case["D"], dtype=f, device="cuda") for _ in range(3))
    dw_post, dw_pre = torch.zeros_like(one), torch.zeros_like(one)
    for q in range(case["seqs"]):
        a = slice(at[q], at[q + 1])
        if a.start >= a.stop:
            continue
        h, y, gate, scale, shift = s["h"][a].to(f), s["y"][a].to(f), s["gate"][q].to(f), s["scale"][q].to(f), s["shift"][q].to(f)
        if not train:
            first[a] = case["alpha"] * h + gate * (w_post * _exact_norm(case["post"], y))
            second[a] = _exact_norm(case["pre"], first[a]) * w_pre * (scale + 1) + shift
            continue
        with torch.enable_grad():
            ins = [t.detach().clone().requires_grad_() for t in (h, scale, shift, w_pre)]
            x = _exact_norm(case["pre"], ins[0]) * ins[3] * (ins[1] + 1) + ins[2]
            through, ds, db, dw = torch.autograd.grad(x, ins, s["dx"][a].to(f))
            up = through + s["dho"][a].to(f)
            ins = [t.detach().clone().requires_grad_() for t in (y, gate, w_post)]
            dy, dg, dv = torch.autograd.grad(ins[1] * (ins[2] * _exact_norm(case["post"], ins[0])), ins, up)
        first[a], second[a] = case["alpha"] * up, dy
        dgate[q], dscale[q], dshift[q] = dg, ds, db
        dw_pre += dw
        dw_post += dv
    if not train:
        return dict(ho=first, x=second)
    out = dict(dh=first, dy=second, dgate=dgate, dscale=dscale, dshift=dshift)
    if s["w_post"] is not None:
        out["dw_post"] = dw_post
    if s["w_pre"] is not None:
        out["dw_pre"] = dw_pre
    return out


def _exact_adamw(s):
    """One step; states in 8 bits have no exact value (they are rounded at random)."""
    f = torch.float64
    t, eight = s["t"] + 1, s["case"]["bits"] == 8
    m, v = s["m"].to(f), s["v"].to(f)
    if eight:
        m = (m.view(-1, _BLOCK) * s["scales"][:, 0].to(f).unsqueeze(1)).flatten()
        v = (v.view(-1, _BLOCK) * s["scales"][:, 1].to(f).unsqueeze(1)).flatten().square()
    g = s["g"].to(f)
    m, v = m + (1 - _BETAS[0]) * (g - m), v + (1 - _BETAS[1]) * (g.square() - v)
    old = (s["p"] if s["master"] is None else s["master"]).to(f)
    new = old - _LR * _DECAY * old - _LR * m / (1 - _BETAS[0] ** t) / ((v / (1 - _BETAS[1] ** t)).sqrt() + _ADAM_EPS)
    out = dict(p=new)
    if s["master"] is not None:
        out["master"] = new
    out.update(m=None if eight else m, v=None if eight else v)
    if eight:
        out["scales"] = None
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_w4(s) if s["kind"].startswith("w4") else _exact_adamw(s) if s["kind"] == "adamw" else _exact_block(s)
