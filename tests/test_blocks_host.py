"""Host side of the products with 4-bit weights, the norms before and after a block and the AdamW step: what they refuse, before anything is launched, through the C ABI and
through the binding; what they do when a launch fails; the plain implementations that the GPU tests compare with, against differences.  No device."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest
import torch

from paper_2604_18117_amd import binding as lq
from tests import blocks_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 20       # aligned, never dereferenced by host code
BIG = 1 << 50


def _wcfg(**kw):
    c = lq.make_w4_config(100, 200, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _w4(name, cfg=None, **kw):
    a = dict(packed=PTR, packed_bytes=BIG, X=PTR, ldx=200, bias=PTR, Y=PTR, ldy=100, M=10, W=PTR, codes=PTR, scales=PTR, work=PTR, work_bytes=BIG)
    assert set(kw) <= set(a)
    a.update(kw)
    raw, c = lq.raw(), C.byref(_wcfg() if cfg is None else cfg)
    if name == "pack":
        return raw.lq_w4_pack(c, a["W"], a["packed"], a["packed_bytes"], None)
    if name == "pack_codes":
        return raw.lq_w4_pack_codes(c, a["codes"], a["scales"], a["packed"], a["packed_bytes"], None)
    if name == "unpack":
        return raw.lq_w4_unpack(c, a["packed"], a["packed_bytes"], a["codes"], a["scales"], None)
    if name == "fwd":
        return raw.lq_w4_fwd(c, a["packed"], a["packed_bytes"], a["X"], a["ldx"], a["bias"], a["Y"], a["ldy"], a["M"], None)
    return raw.lq_w4_bwd(c, a["packed"], a["packed_bytes"], a["Y"], a["ldy"], a["X"], a["ldx"], a["M"], a["work"], a["work_bytes"], None)


W4_CALLS = ["pack", "pack_codes", "unpack", "fwd", "bwd"]


@pytest.mark.parametrize("name", W4_CALLS)
def test_w4_arguments(name):
    for field, value, status in (("N", 0, "SHAPE"), ("N", (1 << 18) + 1, "SHAPE"), ("K", 0, "SHAPE"), ("K", (1 << 16) + 1, "SHAPE"), ("group", 16, "SHAPE"), ("group", 0, "SHAPE"),
                                 ("x_dtype", 2, "UNSUPPORTED"), ("y_dtype", -1, "UNSUPPORTED"), ("flags", 1, "UNSUPPORTED")):
        want, n = getattr(lq, "LQ_ERR_" + status), C.c_size_t(0)
        assert _w4(name, _wcfg(**{field: value})) == want
        assert lq.raw().lq_w4_sizes(C.byref(_wcfg(**{field: value})), C.byref(n)) == lq.raw().lq_w4_work_sizes(C.byref(_wcfg(**{field: value})), 3, C.byref(n)) == want
    assert _w4(name, packed=None) == lq.LQ_ERR_NULL and _w4(name, packed=PTR + 128) == lq.LQ_ERR_ALIGN
    assert _w4(name, packed_bytes=lq.lq_w4_sizes(_wcfg()) - 1) == lq.LQ_ERR_BUFFER_TOO_SMALL
    if name == "pack":
        assert _w4(name, W=None) == lq.LQ_ERR_NULL and _w4(name, W=PTR + 2) == lq.LQ_ERR_ALIGN
    if name == "pack_codes":
        assert _w4(name, codes=None) == _w4(name, scales=None) == lq.LQ_ERR_NULL
    if name in ("pack_codes", "unpack"):
        assert _w4(name, scales=PTR + 1) == lq.LQ_ERR_ALIGN
    if name == "unpack":
        assert _w4(name, codes=None, scales=None) == lq.LQ_OK
    if name in ("fwd", "bwd"):
        assert _w4(name, X=None) == _w4(name, Y=None) == lq.LQ_ERR_NULL
        assert _w4(name, X=PTR + 1) == _w4(name, Y=PTR + 1) == _w4(name, _wcfg(x_dtype=lq.LQ_F32), X=PTR + 2) == lq.LQ_ERR_ALIGN
        assert _w4(name, ldx=199) == _w4(name, ldy=99) == _w4(name, ldx=(1 << 22) + 1) == _w4(name, ldy=(1 << 22) + 1) == _w4(name, M=-1) == _w4(name, M=(1 << 14) + 1) == lq.LQ_ERR_SHAPE
        assert _w4(name, M=0, X=None, Y=None, packed=None) == lq.LQ_OK
    if name == "fwd":
        assert _w4(name, bias=PTR + 2) == lq.LQ_ERR_ALIGN
    if name == "bwd":
        big = _wcfg(N=4096)
        need = lq.lq_w4_work_sizes(big, 10)
        assert need > 0 and _w4(name, big, ldy=4096, work_bytes=need - 1) == lq.LQ_ERR_BUFFER_TOO_SMALL
        assert _w4(name, big, ldy=4096, work=None) == lq.LQ_ERR_NULL and _w4(name, big, ldy=4096, work=PTR + 64) == lq.LQ_ERR_ALIGN


def test_w4_verify_arguments():
    f, c = lq.raw().lq_w4_verify, C.byref(_wcfg())
    assert f(None, PTR, BIG, None) == f(c, None, BIG, None) == lq.LQ_ERR_NULL
    assert f(c, PTR + 128, BIG, None) == lq.LQ_ERR_ALIGN and f(c, PTR, lq.lq_w4_sizes(_wcfg()) - 1, None) == lq.LQ_ERR_BUFFER_TOO_SMALL
    assert f(C.byref(_wcfg(group=16)), PTR, BIG, None) == lq.LQ_ERR_SHAPE and f(C.byref(_wcfg(flags=1)), PTR, BIG, None) == lq.LQ_ERR_UNSUPPORTED


def _bcfg(**kw):
    c = lq.make_block_config(64, "rms", "layer", h_dtype="f32")
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _block(bwd, cfg=None, **kw):
    a = dict(h=PTR, ldh=64, y=PTR, ldy=64, offsets=PTR, S=3, gate=(PTR, 64), scale=(PTR, 64), shift=(PTR, 64), w_post=PTR, w_pre=PTR, ho=PTR, ldho=64, x=PTR, ldx=64, M=10,
             dho=PTR, lddho=64, dx=PTR, lddx=64, dh=PTR, lddh=64, dy=PTR, lddy=64, dgate=(PTR, 64), dscale=(PTR, 64), dshift=(PTR, 64), dw_post=PTR, dw_pre=PTR, work=PTR,
             work_bytes=BIG)
    assert set(kw) <= set(a)
    a.update(kw)
    c = C.byref(_bcfg() if cfg is None else cfg)
    mod = {k: None if a[k] is None else C.byref(lq.lq_mod(*a[k])) for k in ("gate", "scale", "shift")}
    if not bwd:
        return lq.raw().lq_block_norm_fwd(c, a["h"], a["ldh"], a["y"], a["ldy"], a["offsets"], a["S"], mod["gate"], mod["scale"], mod["shift"], a["w_post"], a["w_pre"], a["ho"],
                                          a["ldho"], a["x"], a["ldx"], a["M"], None)
    out = lq.lq_block_grads(a["dh"], a["lddh"], a["dy"], a["lddy"], lq.lq_mod(*a["dgate"]), lq.lq_mod(*a["dscale"]), lq.lq_mod(*a["dshift"]), a["dw_post"], a["dw_pre"])
    return lq.raw().lq_block_norm_bwd(c, a["ho"], a["ldho"], a["y"], a["ldy"], a["offsets"], a["S"], mod["gate"], mod["scale"], a["w_post"], a["w_pre"], a["dho"], a["lddho"],
                                      a["dx"], a["lddx"], C.byref(out), a["M"], a["work"], a["work_bytes"], None)


@pytest.mark.parametrize("bwd", [False, True])
def test_block_configuration(bwd):
    n = C.c_size_t(0)
    for kw, status in ((dict(dim=0), "SHAPE"), (dict(dim=16385), "SHAPE"), (dict(post=3), "UNSUPPORTED"), (dict(pre=-1), "UNSUPPORTED"), (dict(h_dtype=2), "UNSUPPORTED"),
                       (dict(h_dtype=lq.LQ_BF16, y_dtype=lq.LQ_F32), "UNSUPPORTED"), (dict(flags=1), "UNSUPPORTED"), (dict(eps=0.0), "UNSUPPORTED"),
                       (dict(eps=float("nan")), "UNSUPPORTED"), (dict(res_scale=float("inf")), "UNSUPPORTED"), (dict(res_scale=float("nan")), "UNSUPPORTED")):
        want = getattr(lq, "LQ_ERR_" + status)
        assert _block(bwd, _bcfg(**kw)) == want and _block(bwd, _bcfg(**kw), M=0) == want
        assert lq.raw().lq_block_work_sizes(C.byref(_bcfg(**kw)), 10, 3, C.byref(n)) == want
    assert lq.raw().lq_block_work_sizes(C.byref(_bcfg(post=0, pre=0, eps=0.0)), 10, 3, C.byref(n)) == lq.LQ_OK
    for kw in (dict(M=-1), dict(M=(1 << 24) + 1), dict(S=0), dict(S=(1 << 20) + 1), dict(offsets=None)):
        assert _block(bwd, **kw) == lq.LQ_ERR_SHAPE


@pytest.mark.parametrize("bwd", [False, True])
def test_block_arguments(bwd):
    rows = dict(h="ldh", y="ldy", ho="ldho", x="ldx") if not bwd else dict(ho="ldho", y="ldy", dho="lddho", dx="lddx", dh="lddh", dy="lddy")
    for name, ld in rows.items():
        assert _block(bwd, **{name: PTR + 1}) == lq.LQ_ERR_ALIGN
        assert _block(bwd, **{ld: 63}) == _block(bwd, **{ld: 1 << 40}) == lq.LQ_ERR_SHAPE
    for name in ("gate", "scale") + (("dgate", "dscale", "dshift") if bwd else ("shift",)):
        assert _block(bwd, **{name: (PTR + 2, 64)}) == lq.LQ_ERR_ALIGN
        assert _block(bwd, **{name: (PTR, 63)}) == _block(bwd, **{name: (PTR, 1 << 40)}) == lq.LQ_ERR_SHAPE
    for name in ("offsets", "w_post", "w_pre") + (("dw_post", "dw_pre") if bwd else ()):
        assert _block(bwd, **{name: PTR + 2}) == lq.LQ_ERR_ALIGN
    if not bwd:
        assert _block(bwd, h=None) == _block(bwd, y=None) == _block(bwd, ho=None) == _block(bwd, y=None, ho=None, x=None) == lq.LQ_ERR_NULL
        assert _block(bwd, M=0, h=None, y=None, x=None) == lq.LQ_OK
    else:
        assert _block(bwd, dho=None, dx=None) == _block(bwd, ho=None) == _block(bwd, y=None) == _block(bwd, work=None) == lq.LQ_ERR_NULL
        assert _block(bwd, y=None, dy=None, dgate=(None, 0)) == lq.LQ_ERR_NULL  # dw_post is left
        assert _block(bwd, work=PTR + 64) == lq.LQ_ERR_ALIGN
        assert _block(bwd, work_bytes=lq.lq_block_work_sizes(_bcfg(), 10, 3) - 1) == lq.LQ_ERR_BUFFER_TOO_SMALL
        assert _block(bwd, M=0, work=None) == lq.LQ_ERR_NULL  # (gradients of no rows are written, too)


def _adamw(cfg=None, count=None, args=None, **kw):
    base = dict(p=PTR, master=None, grad=2 * PTR, m=3 * PTR, v=4 * PTR, scales=5 * PTR, n=1000)
    second = {k: v + 8192 if v and k != "n" else v for k, v in base.items()}
    assert set(kw) <= set(base)
    base.update(kw)
    table = (lq.lq_adamw_tensor * 2)(lq.lq_adamw_tensor(**base), lq.lq_adamw_tensor(**second))
    args = lq.lq_adamw_args(1e-3, 1, None, None, None) if args is None else args
    return lq.raw().lq_adamw_step(C.byref(lq.make_adamw_config() if cfg is None else cfg), table, 2 if count is None else count, C.byref(args), None)


def test_adamw_arguments():
    raw = lq.raw()
    for kw in (dict(p_dtype=2), dict(g_dtype=-1), dict(state_bits=16), dict(flags=1), dict(reserved=1), dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=0.0), dict(eps=1e-31),
               dict(weight_decay=-1.0), dict(weight_decay=float("nan"))):
        c = lq.make_adamw_config()
        for k, v in kw.items():
            setattr(c, k, v)
        assert _adamw(c) == _adamw(c, count=0) == lq.LQ_ERR_UNSUPPORTED, kw
    for a, status in ((lq.lq_adamw_args(1e-3, 0, None, None, None), "SHAPE"), (lq.lq_adamw_args(1e-3, 1 << 31, None, None, None), "SHAPE"),
                      (lq.lq_adamw_args(float("nan"), 1, None, None, None), "UNSUPPORTED"), (lq.lq_adamw_args(float("inf"), 1, None, None, None), "UNSUPPORTED"),
                      (lq.lq_adamw_args(0, 1, PTR + 1, None, None), "ALIGN"), (lq.lq_adamw_args(0, 0, None, PTR + 2, None), "ALIGN"),
                      (lq.lq_adamw_args(0, 1, None, None, PTR + 1), "ALIGN")):
        assert _adamw(args=a) == getattr(lq, "LQ_ERR_" + status)
    eight = lq.make_adamw_config(state_bits=8)
    for name in ("p", "grad", "m", "v"):
        assert _adamw(**{name: None}) == lq.LQ_ERR_NULL
        assert _adamw(**{name: 7 * PTR + 1}) == lq.LQ_ERR_ALIGN
    assert _adamw(eight, scales=None) == lq.LQ_ERR_NULL and _adamw(eight, scales=PTR + 1) == lq.LQ_ERR_ALIGN and _adamw(master=7 * PTR + 2) == lq.LQ_ERR_ALIGN
    assert _adamw(n=-1) == _adamw(n=1 << 32) == _adamw(count=-1) == _adamw(count=65537) == lq.LQ_ERR_SHAPE
    # what is written lies apart: p over its neighbour, a state over a parameter, a master over a state, scales over scales
    assert _adamw(n=3000) == _adamw(m=PTR + 3996) == _adamw(v=3 * PTR) == _adamw(master=4 * PTR + 8192 + 3996) == lq.LQ_ERR_SHAPE
    assert _adamw(eight, scales=5 * PTR + 8192 - 16) == lq.LQ_ERR_SHAPE
    a = lq.lq_adamw_args(1e-3, 1, None, None, None)
    assert raw.lq_adamw_step(None, None, 0, C.byref(a), None) == raw.lq_adamw_step(C.byref(eight), None, 0, None, None) == lq.LQ_ERR_NULL
    assert raw.lq_adamw_step(C.byref(eight), None, 1, C.byref(a), None) == lq.LQ_ERR_NULL and raw.lq_adamw_step(C.byref(eight), None, 0, C.byref(a), None) == lq.LQ_OK


def test_binding_checks_its_arguments():
    """CPU tensors, other types and shapes raise as in the binding's other calls, before the library is reached."""
    bf = torch.bfloat16
    wcfg, bcfg, acfg = lq.make_w4_config(16, 32, 32), lq.make_block_config(32), lq.make_adamw_config()
    blob, X, Y, h = torch.zeros(4096, dtype=torch.uint8), torch.zeros(2, 32, dtype=bf), torch.zeros(2, 16, dtype=bf), torch.zeros(2, 32, dtype=bf)
    t = torch.zeros(10)
    for call in (lambda: lq.lq_w4_pack(wcfg, torch.zeros(16, 32)), lambda: lq.lq_w4_pack_codes(wcfg, torch.zeros(16, 32, dtype=torch.int8), torch.zeros(16, 1)),
                 lambda: lq.lq_w4_unpack(wcfg, blob), lambda: lq.lq_w4_fwd(wcfg, blob, X), lambda: lq.lq_w4_fwd(wcfg, blob, X, None, Y=Y),
                 lambda: lq.lq_w4_bwd(wcfg, blob, Y), lambda: lq.lq_block_norm_fwd(bcfg, h, h), lambda: lq.lq_block_norm_fwd(bcfg, h, None, None, ho=h),
                 lambda: lq.lq_block_norm_fwd(bcfg, h, h, last=True, x=h), lambda: lq.lq_block_norm_bwd(bcfg, h, h, dx=h), lambda: lq.lq_block_norm_bwd(bcfg, h, h),
                 lambda: lq.lq_block_norm_fwd(bcfg, h, h, torch.zeros(1, dtype=torch.int32)), lambda: lq.lq_adamw_step(acfg, [t], [t], [t], [t], 1e-3, 1),
                 lambda: lq.lq_adamw_step(acfg, [t], [], [t], [t], 1e-3, 1), lambda: lq.lq_adamw_step(lq.make_adamw_config(state_bits=8), [t], [t], [t], [t], 1e-3, 1)):
        with pytest.raises(AssertionError):
            call()
    for bad in (lambda: lq.make_w4_config(1, 1, 32, "f16"), lambda: lq.make_block_config(8, "other"), lambda: lq.make_adamw_config("f16")):
        with pytest.raises(KeyError):
            bad()
    for cfg in (lq.make_w4_config(1, 1, 5), lq.make_w4_config(0, 1, 32)):
        with pytest.raises(lq.LqError):
            lq.lq_w4_sizes(cfg)
    c = lq._call
    assert c.w4_fwd(wcfg, blob, X, None, Y) == c.w4_bwd(wcfg, blob, Y, X, blob) == c.w4_fwd(bcfg, blob, X, None, Y) == c.w4_fwd() == -1
    assert c.block_norm_fwd(bcfg, h, h, None, None, None, None, None, None, h, h, False) == c.block_norm_fwd(bcfg, None, *[None] * 9, False) == -1
    assert c.block_norm_bwd(bcfg, *[None] * 17) == c.block_norm_bwd(bcfg) == -1
    assert c.adamw_step(acfg, [t], [t], [t], [t], 1e-3, 1, None, None, None) == c.adamw_step(acfg, 3, [t], [t], [t], 1e-3, 1, None, None, None) == -1
    assert c.adamw_step(acfg, [t], [t], [t, t], [t], 1e-3, 1, None, None, None) == c.adamw_step(acfg, [None], [t], [t], [t], 1, 1, None, None, None) == -1
    assert not C.pythonapi.PyErr_Occurred()


@pytest.mark.parametrize("status", [lq.LQ_OK, lq.LQ_ERR_DEVICE])
def test_a_call_is_submitted_once(monkeypatch, status):
    wcfg, bcfg, acfg = lq.make_w4_config(16, 32, 32), lq.make_block_config(32), lq.make_adamw_config()
    x = torch.zeros(4)
    calls = {"w4_fwd": lambda: lq.lq_w4_fwd(wcfg, x, x, x, Y=x), "w4_bwd": lambda: lq.lq_w4_bwd(wcfg, x, x, dX=x, work=x),
             "block_norm_fwd": lambda: lq.lq_block_norm_fwd(bcfg, x, x, ho=x, x=x), "block_norm_bwd": lambda: lq.lq_block_norm_bwd(bcfg, x, x, dx=x, dh=x, dy=x, work=x),
             "adamw_step": lambda: lq.lq_adamw_step(acfg, [x], [x], [x], [x], 1e-3, 1)}
    for name, call in calls.items():
        made = []
        monkeypatch.setattr(lq._call, name, lambda *a: made.append("native") or status)
        monkeypatch.setattr(lq._lib, "lq_" + name, lambda *a: made.append("ctypes") or lq.LQ_OK)
        if status == lq.LQ_OK:
            call()
        else:
            with pytest.raises(lq.LqError) as e:
                call()
            assert e.value.status == status
        assert made == ["native"], name


CHILD = r"""
import ctypes as C, json, sys
fake = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
fake.fake_launched.restype = C.c_char_p
fake.fake_threads.restype = C.c_double
lib = C.CDLL(sys.argv[2])
V, Z, L, I, F, D = C.c_void_p, C.c_size_t, C.c_int64, C.c_int32, C.c_float, C.c_double
class W4(C.Structure):
    _fields_ = [("N", L), ("K", L)] + [(k, I) for k in ("group", "x", "y", "flags")]
class Block(C.Structure):
    _fields_ = [(k, I) for k in ("dim", "post", "pre", "h", "y", "flags")] + [("eps", F), ("res", F)]
class Mod(C.Structure):
    _fields_ = [("p", V), ("ld", L)]
class Grads(C.Structure):
    _fields_ = [("dh", V), ("lddh", L), ("dy", V), ("lddy", L), ("g", Mod * 3), ("wp", V), ("wr", V)]
class Adam(C.Structure):
    _fields_ = [(k, I) for k in ("p", "g", "bits", "flags")] + [(k, D) for k in ("b1", "b2", "eps", "wd")] + [("seed", I), ("r", I)]
class Tensor(C.Structure):
    _fields_ = [(k, V) for k in ("p", "master", "g", "m", "v", "s")] + [("n", L)]
class Args(C.Structure):
    _fields_ = [("lr", D), ("t", L)] + [(k, V) for k in "abc"]
P, B = V(1 << 20), Z(1 << 60)
def call(name, a):
    if name.startswith("w4"):
        N, K, group, x, y, M = a
        c = C.byref(W4(N, K, group, x, y, 0))
        if name == "w4_pack": return lib.lq_w4_pack(c, P, P, B, None)
        if name == "w4_unpack": return lib.lq_w4_unpack(c, P, B, P, P, None)
        if name == "w4_fwd": return lib.lq_w4_fwd(c, P, B, P, L(K), P, P, L(N), L(M), None)
        return lib.lq_w4_bwd(c, P, B, P, L(N), P, L(K), L(M), P, B, None)
    if name.startswith("block"):
        dim, post, pre, h, y, S, M, odd = a
        c = C.byref(Block(dim, post, pre, h, y, 0, 1e-6, 1.0))
        m, ld, X = C.byref(Mod(1 << 20, dim)), L(dim + odd), P
        if name == "block_fwd":
            return lib.lq_block_norm_fwd(c, X, ld, X, ld, P, I(S), m, m, m, P, P, X, ld, X, ld, L(M), None)
        one = Mod(1 << 20, dim)
        g = Grads(1 << 20, dim + odd, 1 << 20, dim + odd, (Mod * 3)(one, one, one), 1 << 20, 1 << 20)
        return lib.lq_block_norm_bwd(c, X, ld, X, ld, P, I(S), m, m, P, P, X, ld, X, ld, C.byref(g), L(M), P, B, None)
    bits, sizes = a
    at, ts = 1 << 20, []
    for n in sizes:
        t = []
        for k in range(6):
            t.append(at)
            at += (4 * n + 511) // 256 * 256
        ts.append(Tensor(t[0], None, t[2], t[3], t[4], t[5], n))
    return lib.lq_adamw_step(C.byref(Adam(0, 0, bits, 0, 0.9, 0.999, 1e-8, 0, 0, 0)), (Tensor * len(ts))(*ts), I(len(ts)), C.byref(Args(1e-3, 1, None, None, None)), None)
out = []
for name, a, failing in json.loads(sys.argv[3]):
    fake.fake_reset(failing, 0, 0)
    st = call(name, a)
    n = fake.fake_launches()
    out.append([st, [fake.fake_launched(i).decode() for i in range(min(n, 256))], [fake.fake_threads(i) for i in range(min(n, 256))]])
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    fake = str(tmp_path_factory.mktemp("fake") / "libfake_hip.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "tests", "fake_hip.c"), "-o", fake], check=True)

    def go(jobs):
        r = subprocess.run([sys.executable, "-c", CHILD, fake, os.path.join(ROOT, "paper_2604_18117_amd", "liblq.so"), json.dumps(jobs)], capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout)
    return go


CALLS = [("w4_pack", (100, 200, 32, 1, 1, 0)), ("w4_unpack", (100, 200, 64, 1, 1, 0)), ("w4_fwd", (6912, 1152, 64, 1, 0, 2)), ("w4_bwd", (6912, 1152, 64, 1, 0, 2)),
         ("block_fwd", (1152, 1, 2, 1, 1, 2, 8192, 0)), ("block_bwd", (1152, 1, 2, 1, 1, 2, 8192, 0)), ("block_bwd", (33, 0, 1, 0, 0, 5, 0, 1)), ("adamw", (8, [1000] * 250))]


@pytest.mark.parametrize("name,args", CALLS)
def test_nothing_is_launched_after_a_failed_launch(run, name, args):
    (st, names, _), = run([(name, args, -1)])
    assert st == 0 and names
    for k, (st, got, _) in enumerate(run([(name, args, k) for k in range(len(names))])):
        assert st == 6 and got == names[:k + 1], (k, got)


def test_launches_stay_below_two_to_the_32_threads(run):
    """The largest calls that are not refused."""
    jobs = [("w4_pack", (1 << 18, 1 << 16, 32, 1, 1, 0), -1), ("w4_fwd", (1 << 18, 1 << 16, 32, 0, 1, 1 << 14), -1), ("w4_bwd", (1 << 18, 1 << 16, 32, 0, 1, 1 << 14), -1),
            ("w4_bwd", (1 << 18, 1, 32, 0, 1, 1 << 14), -1), ("block_fwd", (16384, 1, 2, 0, 0, 1 << 20, 1 << 24, 0), -1), ("block_fwd", (1, 1, 2, 0, 0, 1, 1 << 24, 0), -1),
            ("block_fwd", (16383, 1, 2, 0, 0, 1 << 20, 1 << 24, 1), -1), ("block_bwd", (16384, 1, 2, 0, 0, 1 << 20, 1 << 24, 0), -1), ("adamw", (32, [(1 << 32) - 1] * 3), -1),
            ("adamw", (8, [1 << 20] * 200), -1)]
    for job, (st, names, threads) in zip(jobs, run(jobs)):
        assert st == 0 and names and max(threads) < 2.0 ** 32, (job[:1], list(zip(names, threads)))


def test_adamw_launches_of_120_tensors(run):
    """... fewer where they are more than 2^33 values, or lie so far apart that steps of an element pass 32 bits."""
    big = (1 << 32) - 1
    for sizes, launches in (([5], 1), ([5] * 64, 1), ([5] * 65, 1), ([5] * 120, 1), ([5] * 121, 2), ([5] * 300, 3), ([0] * 200 + [5] * 120, 1), ([0] * 10, 0), ([5, 0] * 130, 2), ([5] * 240, 2),
                            ([big], 1), ([big, 5], 2), ([1 << 28] * 3, 1), ([1 << 28] * 12, 4)):  # (here tensors of 2^28 lie 6 GB from each other, 2^32 steps are 16)
        (st, names, _), = run([("adamw", (32, sizes), -1)])
        assert st == 0 and len(names) == launches, (sizes[:4], len(names))


# ---- the plain implementations, against differences --------------------------------------------

def _difference(f, t, direction, step=1e-6):
    return float(f(t + step * direction) - f(t - step * direction)) / (2 * step)


@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "layer"), ("layer", "rms"), ("rms", "none")])
def test_the_plain_block_gradient_against_differences(post, pre):
    g = torch.Generator().manual_seed(3)
    M, D, alpha, eps = 7, 12, 0.75, 1e-3
    offsets = torch.tensor([0, 3, 3, 6], dtype=torch.int32)  # (the last row has no sequence)

    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)
    t = dict(h=normal(M, D), y=normal(M, D), gate=normal(3, D), scale=normal(3, D), shift=normal(3, D), w_post=1 + 0.3 * normal(D), w_pre=1 + 0.3 * normal(D))
    dho, dx = normal(M, D), normal(M, D)

    def loss(**kw):
        a = dict(t, **kw)
        out = ref.block_fwd(a["h"], a["y"], offsets, a["gate"], a["scale"], a["shift"], a["w_post"], a["w_pre"], post, pre, eps, alpha, torch.float64)
        r = out["rows"]
        return (out["ho"][0] * dho[r]).sum() + (out["x"][0] * dx[r]).sum()
    fwd = ref.block_fwd(t["h"], t["y"], offsets, t["gate"], t["scale"], t["shift"], t["w_post"], t["w_pre"], post, pre, eps, alpha, torch.float64)
    ho = torch.zeros(M, D, dtype=torch.float64)
    ho[fwd["rows"]] = fwd["ho"][0]
    grads = ref.block_bwd(ho, t["y"], offsets, t["gate"], t["scale"], t["w_post"], t["w_pre"], dho, dx, post, pre, eps, alpha, torch.float64, torch.float64)
    for k, name in (("h", "dh"), ("y", "dy"), ("gate", "dgate"), ("scale", "dscale"), ("shift", "dshift"), ("w_post", "dw_post"), ("w_pre", "dw_pre")):
        got = grads[name][0]
        if k in ("h", "y"):
            full = torch.zeros(M, D, dtype=torch.float64)
            full[grads["rows"]] = got
            got = full
        for _ in range(3):
            d = normal(*t[k].shape)
            want = _difference(lambda v: loss(**{k: v}), t[k], d)
            # central differences: the third derivative times 1e-12, and rounding 1e-16 over 1e-6 of sums of about 100
            assert abs(float((got * d).sum()) - want) <= 1e-7 * (1 + abs(want)), (k, want)


def test_the_rounding_rule_of_the_8_bit_states():
    """The plain rule hits E4M3's numbers alone, both neighbours and no other, with shares that keep the mean."""
    x = torch.cat([torch.linspace(0, 0.05, 200), torch.linspace(0.05, 448, 400)])
    bits = torch.arange(0, 1 << 20, 4099)
    q = ref.e4m3_random(x[:, None], bits[None, :])
    assert torch.equal(q.float().to(torch.float8_e4m3fn).double(), q)
    step = torch.exp2(torch.floor(torch.log2(x.double().clamp(min=2.0 ** -6)))) / 8
    assert ((q - x[:, None]).abs() < step[:, None]).all()
    assert ((q.mean(1) - x).abs() <= step * 2 / bits.numel()).all()
    for amax, want in ((0.0, 1.0), (448.0, 1.0), (448.1, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (1e-3, 2.0 ** -18)):
        assert float(ref.power_scale(torch.tensor(amax))) == want
    a, b = ref.random_bits(7, 3, 1 << 16)
    for r in (a, b, a ^ b):  # uniform: mean within 5 deviations of the middle, neighbours not alike
        u = r.double() / 2 ** 20 - 0.5
        assert abs(float(u.mean())) <= 5 * (1 / 12) ** 0.5 / 256
        assert abs(float((u[1:] * u[:-1]).mean())) <= 5 / 12 / 256


def test_workspaces_serve_smaller_batches():
    for N, K, group in ((100, 64, 32), (6912, 1152, 64), (13440, 2240, 128), (64, 4608, 64), (700, 128, 128)):
        cfg = lq.make_w4_config(N, K, group)
        sizes = [lq.lq_w4_work_sizes(cfg, M) for M in range(0, 2200)]
        assert sizes == sorted(sizes) and sizes[0] == 0
    for dim in (63, 1152, 2240, 5000, 16384):
        cfg = lq.make_block_config(dim)
        for S in (1, 7):
            sizes = [lq.lq_block_work_sizes(cfg, M, S) for M in [*range(0, 1100), 2000, 4096, 8191, 8192, 8193, 2 ** 24]]
            assert sizes == sorted(sizes)
            assert sizes <= [lq.lq_block_work_sizes(cfg, M, S + 1) for M in [*range(0, 1100), 2000, 4096, 8191, 8192, 8193, 2 ** 24]]
