"""The host checks of the feed-forward operators: what is refused before anything is launched (no GPU needed)."""
import copy
import ctypes
import gc
import os
import pickle
import subprocess
import weakref

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 256          # never dereferenced: every call below fails on the host, or has nothing to do


@pytest.fixture(scope="module")
def B():
    from paper_2410_13056_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2410_13056_amd import build
        build.build()
    binding.lib()
    return binding


def test_structures_have_the_headers_layout(B, tmp_path):
    fields = {"cmpq_int8_job": (B.Int8Job, ["x_codes", "gated", "bias", "activation", "residual", "ldr", "Y", "ldy", "status"]),
              "cmpq_epilogue_job": (B.EpilogueJob, ["bias", "times", "times_bias", "residual", "out", "m", "activation"]),
              "cmpq_int8_feed_forward_job": (B.Int8FeedForwardJob, ["add", "gain", "Y", "eps", "m", "d_ff", "gate_up_codes", "down_scale",
                                                                     "activation", "hidden_dtype", "status"]),
              "cmpq_norm_job": (B.NormJob, ["add", "gain", "S", "Y", "codes", "scale", "m", "eps", "status"])}
    lines = ['#include <stdio.h>', '#include "cmpq.h"', "int main(void) {"]
    for name, (_, names) in fields.items():
        lines.append(f'printf("%zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {n}));' for n in names] + ['printf("\\n");']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.check_call(["gcc", "-std=c99", f"-I{ROOT}/include", str(src), "-o", str(exe)])
    got = subprocess.check_output([str(exe)], text=True).splitlines()
    for line, (struct, names) in zip(got, fields.values()):
        assert [int(v) for v in line.split()] == [ctypes.sizeof(struct)] + [getattr(struct, n).offset for n in names]


def _rows(p=FAKE, ld=64, dtype=0):
    return p, ld, dtype


NONE = (None, 0, 0)


def test_product_jobs(B):
    good = dict(X=FAKE, x_dtype=0, m=4, d_in=8, ldx=8, codes=FAKE, scale=FAKE, d_out=8, Y=FAKE, y_dtype=1, ldy=8)
    run = lambda ws=FAKE, n=1 << 30, **k: B.lib().cmpq_int8_product_job(ctypes.byref(B.Int8Job(**{**good, **k})), ws, n, None)
    coded = dict(X=None, x_codes=FAKE, x_scale=FAKE)
    for bad in (dict(X=None), dict(codes=None), dict(scale=None), dict(Y=None), dict(x_dtype=3), dict(y_dtype=-1), dict(m=-1), dict(d_in=0),
                dict(d_out=-1), dict(activation=5), dict(activation=-1), dict(codes=FAKE + 8), dict(bias=FAKE, bias_dtype=3),
                dict(residual=FAKE, r_dtype=3, ldr=8), dict(up_bias=FAKE), {**coded, "x_codes": None}, {**coded, "x_scale": None},
                {**coded, "x_codes": FAKE + 8}):
        assert run(**bad) == -1, bad
    for bad in (dict(ldx=7), dict(ldy=7), dict(residual=FAKE, ldr=7), dict(d_in=131073, ldx=131073), dict(m=1 << 24),
                dict(gated=1, d_out=1 << 23, ldy=1 << 23), dict(d_out=1 << 24, ldy=1 << 24), {**coded, "d_in": 131073}):
        assert run(**bad) == -2, bad
    assert run(ws=None) == run(ws=FAKE + 16) == run(n=256) == -5
    for kind in ({}, dict(gated=1), coded):
        assert run(m=0, **kind) == run(d_out=0, **kind) == 0
    assert B.lib().cmpq_int8_product_job(None, FAKE, 1 << 30, None) == -1


def test_gated_weights(B):
    L = B.lib()
    assert [B.int8_gated_rows(n) for n in (0, 1, 16, 17, 28672)] == [0, 32, 32, 64, 57344]
    assert B.int8_gated_rows(-1) == B.int8_gated_rows(1 << 23) == 0
    prep = lambda g=FAKE, u=FAKE, dt=0, o=8, i=8, lg=8, lu=8, c=FAKE, s=FAKE: L.cmpq_int8_prepare_gated(g, u, dt, o, i, lg, lu, c, s, None, None)
    assert prep(g=None) == prep(u=None) == prep(c=None) == prep(s=None) == prep(dt=3) == prep(o=-1) == prep(i=-1) == prep(c=FAKE + 8) == -1
    assert prep(lg=7) == prep(lu=7) == prep(i=131073, lg=131073, lu=131073) == prep(o=1 << 23) == -2
    assert prep(o=0) == prep(i=0) == 0


def test_epilogue_jobs(B):
    def run(m=4, d=64, act=1, **k):
        f = {n: NONE for n in ("Y", "bias", "times", "times_bias", "residual", "out")}
        f.update(Y=_rows(), out=_rows())
        f.update(k)
        return B.lib().cmpq_epilogue(ctypes.byref(B.EpilogueJob(*f["Y"], *f["bias"], *f["times"], *f["times_bias"], *f["residual"],
                                                                *f["out"], m, d, act)), None)
    for bad in (dict(m=-1), dict(d=-1), dict(act=5), dict(act=-1), dict(Y=NONE), dict(out=NONE), dict(Y=_rows(dtype=3)), dict(bias=_rows(dtype=3)),
                dict(times_bias=_rows()), dict(residual=_rows(dtype=-1)), dict(out=_rows(dtype=7))):
        assert run(**bad) == -1, bad
    for bad in (dict(Y=_rows(ld=63)), dict(out=_rows(ld=63)), dict(times=_rows(ld=63)), dict(residual=_rows(ld=63)), dict(m=1 << 24),
                dict(d=1 << 24, Y=_rows(ld=1 << 24), out=_rows(ld=1 << 24))):
        assert run(**bad) == -2, bad
    assert run(m=0) == run(d=0) == 0 and B.lib().cmpq_epilogue(None, None) == -1


def test_norm_jobs(B):
    def run(codes=None, scale=None, m=4, d=64, eps=1e-6, **k):
        f = {n: NONE for n in ("X", "add", "gain", "S", "Y")}
        f.update(X=_rows(), Y=_rows() if codes is None else NONE)
        f.update(k)
        return B.lib().cmpq_rms_norm(ctypes.byref(B.NormJob(*f["X"], *f["add"], *f["gain"], *f["S"], *f["Y"], codes, scale, m, d, eps, None)), None)
    for bad in (dict(m=-1), dict(d=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40), dict(X=NONE),
                dict(Y=NONE), dict(codes=FAKE, scale=FAKE, Y=_rows()), dict(codes=FAKE), dict(codes=FAKE + 8, scale=FAKE), dict(X=_rows(dtype=3)),
                dict(add=_rows(dtype=-1)), dict(gain=_rows(dtype=4)), dict(S=_rows(dtype=4)), dict(Y=_rows(dtype=4))):
        assert run(**bad) == -1, bad
    for bad in (dict(X=_rows(ld=63)), dict(add=_rows(ld=63)), dict(S=_rows(ld=63)), dict(Y=_rows(ld=63)), dict(m=1 << 24),
                dict(codes=FAKE, scale=FAKE, d=131073, X=_rows(ld=131073))):
        assert run(**bad) == -2, bad
    assert run(m=0) == run(m=0, codes=FAKE, scale=FAKE) == 0 and B.lib().cmpq_rms_norm(None, None) == -1


def test_feed_forward_jobs(B):
    def job(m=4, d=64, d_ff=96, eps=1e-6, gc=FAKE, gs=FAKE, dc=FAKE, ds=FAKE, act=1, hidden=0, **k):
        f = {n: NONE for n in ("X", "add", "gain", "Y")}
        f.update(X=_rows(), Y=_rows())
        f.update(k)
        return B.Int8FeedForwardJob(*f["X"], *f["add"], *f["gain"], *f["Y"], eps, m, d, d_ff, gc, gs, dc, ds, act, hidden, None)
    run = lambda ws=FAKE, n=1 << 40, **k: B.lib().cmpq_int8_feed_forward(ctypes.byref(job(**k)), ws, n, None)
    for bad in (dict(m=-1), dict(d=0), dict(d_ff=0), dict(eps=0.0), dict(gc=None), dict(gs=None), dict(dc=None), dict(ds=None), dict(act=9),
                dict(hidden=3), dict(X=NONE), dict(Y=NONE), dict(X=_rows(dtype=3)), dict(Y=_rows(dtype=3)), dict(add=_rows(dtype=5)),
                dict(gain=_rows(dtype=-1)), dict(gc=FAKE + 8), dict(dc=FAKE + 8)):
        assert run(**bad) == -1, bad
    for bad in (dict(m=1 << 24), dict(d=131073, X=_rows(ld=131073), Y=_rows(ld=131073)), dict(d_ff=131073), dict(X=_rows(ld=63)),
                dict(Y=_rows(ld=63)), dict(add=_rows(ld=63))):
        assert run(**bad) == -2, bad
    size = lambda **k: B.lib().cmpq_int8_feed_forward_workspace(ctypes.byref(job(**k)))
    need = size()
    assert need % 256 == 0 and size(add=_rows()) >= need + 4 * 64 * 2 and size(hidden=1) > need and size(m=0) >= 256
    assert run(ws=None) == run(ws=FAKE + 16) == run(n=need - 1) == -5 and run(m=0) == run(m=0, X=NONE[:2] + (0,), Y=NONE) == 0
    assert size(m=-1) == size(d_ff=131073) == size(hidden=7) == 0
    assert B.lib().cmpq_int8_feed_forward(None, FAKE, 1 << 40, None) == -1 and B.lib().cmpq_int8_feed_forward_workspace(None) == 0


# ---- the Python side, on host tensors with the library's part left out ---------------------------------

@pytest.fixture
def S(B, monkeypatch):
    from paper_2410_13056_amd import serving
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(B, "_device", lambda: -1)                       # where host tensors say that they are
    monkeypatch.setattr(B, "_stream", lambda: 0)

    class Library:
        def __init__(self, real):
            self.real = real

        def __getattr__(self, name):
            if name in ("cmpq_int8_weight_bytes", "cmpq_int8_feed_forward_workspace", "cmpq_int8_gated_rows", "cmpq_workspace_bytes", "cmpq_strerror"):
                return getattr(self.real, name)
            return lambda *args: 0
    monkeypatch.setattr(B, "_lib", Library(B.lib()))
    return serving


class _Workspace:
    buf = torch.empty(0, dtype=torch.uint8)


def _weight(S, B, d_in=64, d_out=24, gated=False):
    rows = B.int8_gated_rows(d_out) if gated else d_out
    return (S.Int8GatedWeight if gated else S.Int8Weight)(d_in, d_out, torch.zeros(B.int8_weight_bytes(rows, d_in), dtype=torch.int8), torch.ones(rows))


def test_tensors_that_do_not_fit_are_refused(S, B):
    ws, X, z = _Workspace(), torch.zeros((3, 64)), torch.zeros
    for w, call, bias in ((_weight(S, B), S.int8_product, "bias"), (_weight(S, B, gated=True), S.int8_gated_product, "gate_bias")):
        ok = {bias: z(24), "residual": z((3, 24)), "activation": "silu"}
        assert call(w, X, ws, **ok).shape == (3, 24)
        for bad in ({bias: z(23)}, {bias: z((24, 1))}, {bias: z(48)[::2]}, {"residual": z((3, 23))}, {"residual": z((2, 24))},
                    {"residual": z((24, 3)).t()}, {"out": z((3, 23))}, {"out": z((4, 24))}, {"activation": "tanh"}, {"activation": 1},
                    {"status": z(1)}):
            with pytest.raises(ValueError):
                call(w, X, ws, **{**ok, **bad})
        for bad in ({bias: z(24, dtype=torch.int32)}, {"residual": z((3, 24), dtype=torch.float64)}, {"out_dtype": torch.int32}):
            with pytest.raises(TypeError):
                call(w, X, ws, **{**ok, **bad})
        with pytest.raises(ValueError):
            call(w, z((3, 63)), ws, **ok)
        with pytest.raises(ValueError):
            call(w, S.Int8Rows(3, 63, z(B.int8_weight_bytes(3, 63), dtype=torch.int8), z(3)), ws, **ok)
    with pytest.raises(ValueError):
        S.int8_gated_product(_weight(S, B, gated=True), X, ws, gate_bias=z(24), up_bias=z(24).half())
    with pytest.raises(ValueError):
        S.prepare_int8_gated(z((24, 64)), z((24, 64)).half())
    with pytest.raises(ValueError):
        S.prepare_int8_gated(z((24, 64)), z((23, 64)))
    gate_up, down, norm = _weight(S, B, 64, 24, True), _weight(S, B, 24, 64), S.RmsNorm(z(64))
    assert S.feed_forward_block(X, norm, gate_up, down, ws, add=X.half()).shape == (3, 64)
    for bad in (dict(norm=S.RmsNorm(z(63))), dict(add=z((3, 63))), dict(down=_weight(S, B, 24, 63)), dict(down=_weight(S, B, 23, 64)),
                dict(gate_up=_weight(S, B, 63, 24, True)), dict(activation="tanh")):
        with pytest.raises(ValueError):
            S.feed_forward_block(**{**dict(X=X, norm=norm, gate_up=gate_up, down=down, ws=ws), **bad})
    with pytest.raises(TypeError):
        S.feed_forward_block(X, norm, gate_up, down, ws, hidden_dtype=torch.float64)
    for bad in (dict(bias=z(63)), dict(times=z((3, 63))), dict(times_bias=z(64), times=z((2, 64))), dict(residual=z(64)), dict(out=z((3, 65))),
                dict(activation="swish")):
        with pytest.raises(ValueError):
            S.epilogue(X, **bad)
    for bad in (dict(weight=z(63)), dict(add=z((3, 63))), dict(sum_out=z((2, 64)), add=X), dict(out=z((3, 63))), dict(out=z((64, 3)).t())):
        with pytest.raises(ValueError):
            S.rms_norm(X, **bad)
    with pytest.raises(TypeError):
        S.rms_norm(X, add=X.double())
    with pytest.raises(ValueError):
        S.rms_norm(X, out=S._empty_rows(z((2, 64))))
    with pytest.raises(ValueError):
        S.int8_rows(X, out=S._empty_rows(z((2, 64))))


def test_host_tensors_and_other_devices_are_refused(B):
    class Elsewhere:
        is_cuda, shape, dtype = True, (3,), torch.float16

        def is_contiguous(self):
            return True

        def get_device(self):
            return 1

        def data_ptr(self):
            return FAKE
    for t, why in ((torch.zeros(3), "device tensors"), (Elsewhere(), "current device")):
        with pytest.raises(ValueError, match=why):
            B._vector(t, 3, 0, "bias")
    with pytest.raises(ValueError, match="device tensors"):
        B._matrix(torch.zeros((3, 4)), 3, 4, 0, "X")
    with pytest.raises(ValueError):
        B._flags(torch.zeros(1, dtype=torch.int32), 0)
    assert B._vector(Elsewhere(), 3, 1, "bias") == (FAKE, 0, B.F16)


def test_layers_and_workspaces_of_another_device_are_refused(S, B, monkeypatch):
    class Elsewhere:
        class buf:
            get_device = staticmethod(lambda: 1)
    X, layers = torch.zeros((3, 64)), (_weight(S, B, 64, 24, True), _weight(S, B, 24, 64))
    rows = S.rms_norm(X, coded=True)
    calls = [lambda ws, x: S.int8_gated_product(layers[0], x, ws), lambda ws, x: S.int8_product(_weight(S, B), x, ws, activation="relu")]
    for call in calls:
        for x in (X, rows):
            with pytest.raises(ValueError, match="current device"):
                call(Elsewhere(), x)
    with pytest.raises(ValueError, match="current device"):
        S.feed_forward_block(X, S.RmsNorm(), *layers, Elsewhere())
    monkeypatch.setattr(B, "_device", lambda: 0)
    for call in calls + [lambda ws, x: S.rms_norm(X, out=rows), lambda ws, x: S.epilogue(X)]:
        with pytest.raises(ValueError):
            call(_Workspace(), rows)


def test_outputs_have_the_types_asked_for(S, B):
    ws, X, A = _Workspace(), torch.zeros((3, 64), dtype=torch.bfloat16), torch.zeros((3, 64))
    rows = S.rms_norm(X, coded=True)
    assert isinstance(rows, S.Int8Rows) and (rows.rows, rows.dim) == (3, 64)
    assert S.int8_product(_weight(S, B), rows, ws).dtype == torch.float16
    assert S.int8_product(_weight(S, B), X, ws, bias=torch.zeros(24)).dtype == torch.bfloat16
    assert S.int8_gated_product(_weight(S, B, gated=True), rows, ws, out_dtype=torch.float32).dtype == torch.float32
    norm, total = S.rms_norm(X, add=A, out_dtype=torch.float16)
    assert norm.dtype == torch.float16 and total.dtype == torch.bfloat16
    assert S.rms_norm(X, add=A, sum_out=A)[1] is A
    assert S.epilogue(A, out_dtype=torch.float16).dtype == torch.float16 and S.epilogue(A, out=A) is A
    assert S.epilogue(A) is A and S.epilogue(A, out_dtype=A.dtype) is A and S.epilogue(A, activation="relu") is not A
    for bad in (A.t(), A.double(), A[0]):
        with pytest.raises((ValueError, TypeError)):
            S.epilogue(bad)


def test_objects_are_copied_and_give_their_memory_back(S, B):
    for make in (lambda: S._empty_rows(torch.zeros((5, 64))), lambda: _weight(S, B, gated=True)):
        thing = make()
        thing.codes.zero_()
        for other in (copy.deepcopy(thing), pickle.loads(pickle.dumps(thing))):
            assert type(other) is type(thing) and torch.equal(other.codes, thing.codes) and other.codes.data_ptr() != thing.codes.data_ptr()
        scale = thing.scale.clone()
        thing.scale = scale
        assert scale.data_ptr() in (getattr(thing._args, "_scale", 0), getattr(thing._args, "scale", 0))
        thing.scale = scale[:-1]
        with pytest.raises(ValueError):
            thing._args
        held = weakref.ref(thing.codes)
        del thing, other
        gc.collect()
        assert held() is None
