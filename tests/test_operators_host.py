"""Host side of the operators around a projection (adapters, norm and rotation of queries and keys): what they refuse, before anything is launched, through
the C ABI and through the binding; what they do when a launch fails.  No device."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest
import torch

from paper_2604_18117_amd import binding as lq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 20       # aligned, never dereferenced by host code
BIG = 1 << 50


def _acfg(**kw):
    c = lq.make_adapter_config(128, 192, 16, 4, "bf16")
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _fwd(cfg=None, **kw):
    a = dict(plan=PTR, plan_bytes=BIG, A=PTR, B=PTR, ranks=PTR, scales=PTR, X=PTR, ldx=192, Yin=PTR, ldyin=128, Y=PTR, ldy=128, M=100, inter=PTR, inter_bytes=BIG)
    assert set(kw) <= set(a)
    a.update(kw)
    pool = lq.lq_adapter_pool(a["A"], a["B"], a["ranks"], a["scales"])
    return lq.raw().lq_adapter_fwd(C.byref(_acfg() if cfg is None else cfg), a["plan"], a["plan_bytes"], C.byref(pool), a["X"], a["ldx"], a["Yin"], a["ldyin"],
                                   a["Y"], a["ldy"], a["M"], a["inter"], a["inter_bytes"], None)


def _bwd(cfg=None, **kw):
    a = dict(plan=PTR, plan_bytes=BIG, A=PTR, B=PTR, ranks=PTR, scales=PTR, X=PTR, ldx=192, inter=PTR, inter_bytes=BIG, dY=PTR, lddy=128, dXin=PTR, lddxin=192,
             dX=PTR, lddx=192, dA=PTR, dB=PTR, M=100, work=PTR, work_bytes=BIG)
    assert set(kw) <= set(a)
    a.update(kw)
    pool = lq.lq_adapter_pool(a["A"], a["B"], a["ranks"], a["scales"])
    return lq.raw().lq_adapter_bwd(C.byref(_acfg() if cfg is None else cfg), a["plan"], a["plan_bytes"], C.byref(pool), a["X"], a["ldx"], a["inter"],
                                   a["inter_bytes"], a["dY"], a["lddy"], a["dXin"], a["lddxin"], a["dX"], a["lddx"], a["dA"], a["dB"], a["M"], a["work"],
                                   a["work_bytes"], None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("field,value,status", [
    ("N", 100, "SHAPE"), ("N", 0, "SHAPE"), ("N", 1 << 23, "SHAPE"), ("K", 96, "SHAPE"), ("rank", 0, "SHAPE"), ("rank", 12, "SHAPE"), ("rank", 136, "SHAPE"),
    ("slots", 0, "SHAPE"), ("slots", 1025, "SHAPE"), ("x_dtype", 2, "UNSUPPORTED"), ("flags", 1, "UNSUPPORTED")])
def test_adapter_configuration(call, field, value, status):
    cfg = _acfg(**{field: value})
    want = getattr(lq, "LQ_ERR_" + status)
    assert call(cfg, M=0) == want and call(cfg) == want
    n = C.c_size_t(0)
    assert lq.raw().lq_adapter_sizes(C.byref(cfg), 10, C.byref(n), None) == want


def test_a_few_rows_over_a_large_pool_need_little_memory():
    """Only adapters of more than 64 rows have parts of their gradients' sums: none here, then at most two for every 64 rows."""
    cfg, rp = _acfg(N=1152, K=1152, rank=32, slots=1024), 32
    part = 32 * (1152 + 1152) * 4
    assert lq.lq_adapter_sizes(cfg, 64)[1] == 64 * rp * 4
    assert lq.lq_adapter_sizes(cfg, 1000)[1] <= 1000 * rp * 4 + 256 + 2 * 16 * part + 256


def test_adapter_pools_beyond_a_launch():
    assert _fwd(_acfg(N=1 << 22, K=1 << 22, rank=128, slots=16), M=0) == lq.LQ_ERR_UNSUPPORTED
    assert _fwd(M=-1) == lq.LQ_ERR_SHAPE and _bwd(M=(1 << 24) + 1) == lq.LQ_ERR_SHAPE


@pytest.mark.parametrize("name,call", [("X", _fwd), ("Yin", _fwd), ("Y", _fwd), ("plan", _fwd), ("inter", _fwd), ("A", _fwd), ("B", _fwd), ("ranks", _fwd), ("scales", _fwd),
                                       ("X", _bwd), ("dY", _bwd), ("dX", _bwd), ("dA", _bwd), ("dB", _bwd), ("plan", _bwd), ("inter", _bwd), ("work", _bwd), ("A", _bwd)])
def test_adapter_pointers(name, call):
    assert call(**{name: None}) == lq.LQ_ERR_NULL
    assert call(**{name: PTR + 2}) == lq.LQ_ERR_ALIGN
    if name in ("plan", "inter", "work"):
        assert call(**{name: PTR + 128}) == lq.LQ_ERR_ALIGN
        need = {"plan": lq.lq_adapter_plan_sizes(100, 4), "inter": lq.lq_adapter_sizes(_acfg(), 100)[0], "work": lq.lq_adapter_sizes(_acfg(), 100)[1]}[name]
        assert call(**{name + "_bytes": need - 1}) == lq.LQ_ERR_BUFFER_TOO_SMALL


@pytest.mark.parametrize("name,call,cols", [("ldx", _fwd, 192), ("ldyin", _fwd, 128), ("ldy", _fwd, 128), ("ldx", _bwd, 192), ("lddy", _bwd, 128), ("lddx", _bwd, 192),
                                            ("lddxin", _bwd, 192)])
def test_adapter_strides(name, call, cols):
    assert call(**{name: cols - 8}) == lq.LQ_ERR_SHAPE
    assert call(**{name: (1 << 22) + 8}) == lq.LQ_ERR_SHAPE
    assert call(**{name: cols + 4}) == lq.LQ_ERR_ALIGN
    if name in ("ldx", "lddx", "lddxin"):   # 4 fp32 values are 16 bytes
        assert call(_acfg(x_dtype=lq.LQ_F32), **{name: cols + 2}) == lq.LQ_ERR_ALIGN


def test_adapter_plan_and_empty_batches():
    raw, n = lq.raw(), C.c_size_t(0)
    assert raw.lq_adapter_plan_sizes(10, 4, None) == lq.LQ_ERR_NULL
    for M, slots in ((-1, 4), ((1 << 24) + 1, 4), (10, 0), (10, 1025)):
        assert raw.lq_adapter_plan_sizes(M, slots, C.byref(n)) == lq.LQ_ERR_SHAPE
        assert raw.lq_adapter_plan(slots, PTR, M, PTR, BIG, None) == lq.LQ_ERR_SHAPE
    assert raw.lq_adapter_plan(4, None, 10, PTR, BIG, None) == lq.LQ_ERR_NULL
    assert raw.lq_adapter_plan(4, PTR, 10, None, BIG, None) == lq.LQ_ERR_NULL
    assert raw.lq_adapter_plan(4, PTR + 1, 10, PTR, BIG, None) == lq.LQ_ERR_ALIGN
    assert raw.lq_adapter_plan(4, PTR, 10, PTR + 16, BIG, None) == lq.LQ_ERR_ALIGN
    assert raw.lq_adapter_plan(4, PTR, 10, PTR, lq.lq_adapter_plan_sizes(10, 4) - 1, None) == lq.LQ_ERR_BUFFER_TOO_SMALL
    # an empty forward looks at no buffer; an empty backward still has the gradients to clear
    assert _fwd(M=0, X=None, Yin=None, Y=None, plan=None, inter=None, A=None) == lq.LQ_OK
    assert _bwd(M=0, dA=None) == lq.LQ_ERR_NULL and _bwd(M=0, dB=PTR + 4) == lq.LQ_ERR_ALIGN


def _qcfg(**kw):
    c = lq.make_qk_config(4, 2, 64, (8, 8), "half", True, 1e-6)
    pairs = kw.pop("pairs", None)
    if pairs is not None:
        c.pairs = (C.c_int32 * 4)(*pairs)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _qk(cfg=None, bwd=False, **kw):
    a = dict(q=(PTR, 256, 64), k=(PTR, 128, 64), g0=(PTR, 256, 64), g1=(PTR, 128, 64), o0=(PTR, 256, 64), o1=(PTR, 128, 64), wq=PTR, wk=PTR, pos=PTR, pos_rows=10,
             inv_freq=PTR, M=10, dwq=PTR, dwk=PTR, work=PTR, work_bytes=BIG)
    assert set(kw) <= set(a)
    a.update(kw)
    h = {k: None if a[k] is None else C.byref(lq.lq_heads(*a[k])) for k in ("q", "k", "g0", "g1", "o0", "o1")}
    cfg = C.byref(_qcfg() if cfg is None else cfg)
    if not bwd:
        return lq.raw().lq_qk_norm_rope_fwd(cfg, h["q"], h["k"], a["wq"], a["wk"], a["pos"], a["pos_rows"], a["inv_freq"], h["o0"], h["o1"], a["M"], None)
    return lq.raw().lq_qk_norm_rope_bwd(cfg, h["q"], h["k"], a["wq"], a["wk"], a["pos"], a["pos_rows"], a["inv_freq"], h["g0"], h["g1"], h["o0"], h["o1"], a["dwq"],
                                        a["dwk"], a["M"], a["work"], a["work_bytes"], None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(heads_q=-1), "SHAPE"), (dict(heads_q=0, heads_k=0), "SHAPE"), (dict(heads_q=4096), "SHAPE"), (dict(heads_q=2 ** 31 - 1), "SHAPE"), (dict(head_dim=63), "SHAPE"),
    (dict(head_dim=0), "SHAPE"), (dict(head_dim=258), "SHAPE"), (dict(axes=5), "SHAPE"), (dict(axes=1), "SHAPE"), (dict(pairs=(30, 8, 0, 0)), "SHAPE"),
    (dict(pairs=(-1, 8, 0, 0)), "SHAPE"), (dict(axes=4, pairs=(2 ** 30, 2 ** 30, 2 ** 30, 2 ** 30)), "SHAPE"), (dict(pairing=2), "UNSUPPORTED"), (dict(norm=2), "UNSUPPORTED"),
    (dict(dtype=5), "UNSUPPORTED"), (dict(flags=1), "UNSUPPORTED"), (dict(eps=0.0), "UNSUPPORTED"), (dict(eps=float("nan")), "UNSUPPORTED")])
def test_qk_configuration(kw, status, bwd):
    want = getattr(lq, "LQ_ERR_" + status)
    assert _qk(_qcfg(**kw), bwd) == want and _qk(_qcfg(**kw), bwd, M=0) == want
    n = C.c_size_t(0)
    assert lq.raw().lq_qk_work_sizes(C.byref(_qcfg(**kw)), 10, C.byref(n)) == want


@pytest.mark.parametrize("bwd", [False, True])
def test_qk_arguments(bwd):
    names = ("q", "k", "o0", "o1") + (("g0", "g1") if bwd else ())
    for name in names:
        assert _qk(None, bwd, **{name: None}) == lq.LQ_ERR_NULL
        assert _qk(None, bwd, **{name: (None, 256, 64)}) == lq.LQ_ERR_NULL
        assert _qk(None, bwd, **{name: (PTR + 1, 256, 64)}) == lq.LQ_ERR_ALIGN
        assert _qk(None, bwd, **{name: (PTR, -1, 64)}) == lq.LQ_ERR_SHAPE
        assert _qk(None, bwd, **{name: (PTR, 256, 1 << 40)}) == lq.LQ_ERR_SHAPE
    assert _qk(None, bwd, pos=None) == _qk(None, bwd, inv_freq=None) == lq.LQ_ERR_NULL
    assert _qk(None, bwd, pos_rows=0) == lq.LQ_ERR_SHAPE
    assert _qk(None, bwd, pos=PTR + 2) == _qk(None, bwd, wq=PTR + 2) == lq.LQ_ERR_ALIGN
    assert _qk(None, bwd, M=-1) == _qk(None, bwd, M=(1 << 24) + 1) == lq.LQ_ERR_SHAPE
    if bwd:
        assert _qk(None, True, dwq=None) == _qk(None, True, dwk=None) == lq.LQ_ERR_NULL
        assert _qk(None, True, work=None) == lq.LQ_ERR_NULL
        assert _qk(None, True, work=PTR + 64) == _qk(None, True, dwq=PTR + 2) == lq.LQ_ERR_ALIGN
        assert _qk(None, True, work_bytes=lq.lq_qk_work_sizes(_qcfg(), 10) - 1) == lq.LQ_ERR_BUFFER_TOO_SMALL
    else:
        assert _qk(M=0, q=None, pos=None) == lq.LQ_OK


def test_binding_checks_its_arguments():
    """CPU tensors, other types and shapes raise as in the binding's other calls, before the library is reached."""
    bf, f = torch.bfloat16, torch.float32
    cfg = lq.make_adapter_config(128, 192, 16, 2)
    X, Yin = torch.zeros(4, 192, dtype=bf), torch.zeros(4, 128, dtype=bf)
    A, B, ranks, scales = torch.zeros(2, 16, 192, dtype=bf), torch.zeros(2, 128, 16, dtype=bf), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    blob = torch.zeros(1 << 16, dtype=torch.uint8)
    qcfg = lq.make_qk_config(2, 2, 16, (4, 4))
    q = torch.zeros(3, 2, 16, dtype=bf)
    w, pos, freq = torch.ones(16), torch.zeros(3, 2), torch.ones(8)
    for call in (lambda: lq.lq_adapter_plan(2, torch.zeros(4, dtype=torch.int32), plan=blob),
                 lambda: lq.lq_adapter_plan(2, torch.zeros(4, dtype=torch.int64)),
                 lambda: lq.lq_adapter_fwd(cfg, blob, X, A, B, ranks, scales, Yin, Y=Yin, inter=blob),
                 lambda: lq.lq_adapter_fwd(cfg, blob, X.to(f), A, B, ranks, scales, Yin),
                 lambda: lq.lq_adapter_bwd(cfg, blob, X, A, B, ranks, scales, blob, Yin),
                 lambda: lq.lq_qk_norm_rope_fwd(qcfg, q, q, w, w, pos, freq, qo=q, ko=q),
                 lambda: lq.lq_qk_norm_rope_bwd(qcfg, q, q, w, w, pos, freq, q, q)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(lq.LqError) as e:
        lq.lq_adapter_plan_sizes(10, 0)
    assert e.value.status == lq.LQ_ERR_SHAPE
    with pytest.raises(ValueError):
        lq.make_qk_config(1, 1, 16, (1, 1, 1, 1, 1))
    with pytest.raises(KeyError):
        lq.make_qk_config(1, 1, 16, (1,), "other")
    assert lq._call.adapter_fwd(cfg, blob, X, A, B, ranks, scales, Yin, Yin, blob) == -1
    assert lq._call.qk_norm_rope_fwd(qcfg, q, q, w, w, pos, freq, q, q) == -1 and lq._call.qk_norm_rope_fwd(cfg, q, q, w, w, pos, freq, q, q) == -1
    assert lq._call.adapter_plan(2.0, blob, blob) == -1 and lq._call.adapter_bwd() == -1 and lq._call.qk_norm_rope_bwd(qcfg, None) == -1
    assert not C.pythonapi.PyErr_Occurred()


@pytest.mark.parametrize("status", [lq.LQ_OK, lq.LQ_ERR_DEVICE])
def test_a_call_is_submitted_once(monkeypatch, status):
    cfg, qcfg = lq.make_adapter_config(128, 192, 16, 2), lq.make_qk_config(2, 2, 16, (4, 4))
    x = torch.zeros(4)
    calls = {"adapter_plan": lambda: lq.lq_adapter_plan(2, x, plan=x), "adapter_fwd": lambda: lq.lq_adapter_fwd(cfg, x, x, x, x, x, x, x, Y=x, inter=x),
             "adapter_bwd": lambda: lq.lq_adapter_bwd(cfg, x, x, x, x, x, x, x, x, x, x, x, x, x),
             "qk_norm_rope_fwd": lambda: lq.lq_qk_norm_rope_fwd(qcfg, x, x, x, x, x, x, qo=x, ko=x),
             "qk_norm_rope_bwd": lambda: lq.lq_qk_norm_rope_bwd(qcfg, x, x, x, x, x, x, x, x, x, x, x, x, x)}
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
V, Z, L, I, F = C.c_void_p, C.c_size_t, C.c_int64, C.c_int32, C.c_float
class Cfg(C.Structure):
    _fields_ = [("N", L), ("K", L)] + [(k, I) for k in ("rank", "slots", "x", "flags")]
class Pool(C.Structure):
    _fields_ = [(k, V) for k in "ABrs"]
class Qk(C.Structure):
    _fields_ = [(k, I) for k in ("q", "k", "d", "axes")] + [("pairs", I * 4)] + [(k, I) for k in ("pairing", "norm", "dtype", "flags")] + [("eps", F)]
class H(C.Structure):
    _fields_ = [("p", V), ("ld", L), ("hs", L)]
P, B = V(1 << 20), Z(1 << 60)
def call(name, a):
    if name == "plan":
        slots, M = a
        return lib.lq_adapter_plan(I(slots), P, L(M), P, B, None)
    if name in ("fwd", "bwd"):
        N, K, rank, slots, x, M = a
        c, p = Cfg(N, K, rank, slots, x, 0), Pool(1 << 20, 1 << 20, 1 << 20, 1 << 20)
        if name == "fwd":
            return lib.lq_adapter_fwd(C.byref(c), P, B, C.byref(p), P, L(K), P, L(N), P, L(N), L(M), P, B, None)
        return lib.lq_adapter_bwd(C.byref(c), P, B, C.byref(p), P, L(K), P, B, P, L(N), P, L(K), P, L(K), P, P, L(M), P, B, None)
    q, k, d, pairs, pairing, norm, dtype, M = a
    c = Qk(q, k, d, len(pairs), (I * 4)(*pairs), pairing, norm, dtype, 0, 1e-6)
    h, g = H(1 << 20, q * d, d), H(1 << 20, k * d, d)
    q, k = C.byref(h), C.byref(g)
    if name == "qk":
        return lib.lq_qk_norm_rope_fwd(C.byref(c), q, k, P, P, P, L(M), P, q, k, L(M), None)
    return lib.lq_qk_norm_rope_bwd(C.byref(c), q, k, P, P, P, L(M), P, q, k, q, k, P, P, L(M), P, B, None)
out = []
for name, a, failing in json.loads(sys.argv[3]):
    fake.fake_reset(failing, 0, 0)
    st = call(name, a)
    n = fake.fake_launches()
    out.append([st, [fake.fake_launched(i).decode() for i in range(n)], [fake.fake_threads(i) for i in range(n)]])
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


CALLS = [("plan", (4, 5000)), ("plan", (4, 7)), ("fwd", (3456, 1152, 32, 4, 1, 5000)), ("fwd", (1152, 1152, 16, 4, 0, 2)), ("bwd", (3456, 1152, 32, 4, 1, 5000)),
         ("bwd", (1152, 1152, 104, 4, 0, 90)), ("bwd", (128, 64, 8, 3, 1, 0)), ("qk", (16, 16, 72, (18, 18), 0, 1, 1, 900)), ("qk_bwd", (16, 16, 72, (18, 18), 0, 1, 1, 900)),
         ("qk_bwd", (3, 1, 50, (9,), 1, 1, 0, 4))]


@pytest.mark.parametrize("name,args", CALLS)
def test_nothing_is_launched_after_a_failed_launch(run, name, args):
    (st, names, _), = run([(name, args, -1)])
    assert st == 0 and names
    for k, (st, got, _) in enumerate(run([(name, args, k) for k in range(len(names))])):
        assert st == 6 and got == names[:k + 1], (k, got)


def test_launches_stay_below_two_to_the_32_threads(run):
    """The largest batches and pools that are not refused."""
    jobs = [("plan", (1024, 1 << 24), -1), ("fwd", (1 << 16, 64, 128, 256, 1, 1 << 24), -1), ("fwd", (1 << 22, 1 << 22, 128, 3, 0, 1 << 24), -1), ("bwd", (1 << 22, 1 << 22, 128, 3, 1, 1 << 24), -1), ("bwd", (1 << 16, 1 << 16, 128, 255, 0, 1 << 20), -1),
            ("bwd", (1 << 18, 1 << 18, 8, 1023, 1, 1000), -1), ("bwd", (1 << 22, 64, 128, 4, 1, 1 << 14), -1), ("qk", (2048, 2048, 256, (128,), 0, 1, 1, 1 << 24), -1),
            ("qk_bwd", (1, 1, 2, (1,), 1, 1, 1, 1 << 24), -1)]
    for job, (st, names, threads) in zip(jobs, run(jobs)):
        assert st == 0 and names and max(threads) < 2.0 ** 32, (job, list(zip(names, threads)))
