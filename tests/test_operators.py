"""The operators' boundary on the host: layouts, refusals (before any HIP call), workspace sizes, the binding."""
import ctypes
import os
import re

import pytest

from paper_2008_11849_amd import sparsert as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, Q, S, T, V = (0x1000000 * i for i in range(1, 6))   # addresses that are only looked at


@pytest.mark.parametrize("name,struct", [("sparsert_norm", sp._Norm), ("sparsert_dequant", sp._Dequant), ("sparsert_adapter_set", sp._AdapterSet)])
def test_descriptors_match_the_header(name, struct):
    text = open(os.path.join(ROOT, "include", "sparsert.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, re.S).group(1), flags=re.S)
    fields = []
    for kind, names in re.findall(r"(int32_t|float)\s+([^;]+);", body):
        for item in names.split(","):
            m = re.match(r"\s*(\w+)(?:\[(\d+)\])?\s*$", item)
            fields.append((m.group(1), kind, int(m.group(2) or 1)))
    at = 0
    assert len(fields) == len(struct._fields_)
    for (n, kind, count), (name_, type_) in zip(fields, struct._fields_):
        base = type_._type_ if hasattr(type_, "_length_") else type_
        assert n == name_ and getattr(struct, n).offset == at and ctypes.sizeof(type_) == 4 * count
        assert base is (ctypes.c_float if kind == "float" else ctypes.c_int32)
        at += 4 * count
    assert ctypes.sizeof(struct) == at


def refused(status, text, call, *args):
    with pytest.raises(sp.SparseRTError) as e:
        call(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


def norm(**kw):
    a = dict(K=8, N=16, dtype=sp.F16)
    a.update(kw)
    return sp.RmsNorm(**a)


@pytest.mark.parametrize("kw,status,text", [
    (dict(K=0), sp.EINVAL, "positive"), (dict(N=-1), sp.EINVAL, "positive"), (dict(batch=-1), sp.EINVAL, "batch"), (dict(batch=65536), sp.EINVAL, "batch"),
    (dict(dtype=sp.I8), sp.EINVAL, "dtype"), (dict(dtype=7), sp.EINVAL, "dtype"), (dict(out_dtype=sp.F32), sp.EINVAL, "out_dtype"),
    (dict(eps=0.0), sp.EINVAL, "eps"), (dict(eps=-1.0), sp.EINVAL, "eps"), (dict(eps=float("nan")), sp.EINVAL, "eps"), (dict(eps=float("inf")), sp.EINVAL, "eps"),
    (dict(ldx=15), sp.EINVAL, "ldx"), (dict(ldh=-1), sp.EINVAL, "ldh"), (dict(ldy=1), sp.EINVAL, "ldy"),
    (dict(K=1 << 20, ldx=1 << 10), sp.EUNSUPPORTED, "2 GiB"), (dict(K=2 ** 31 - 1, N=2 ** 31 - 1), sp.EUNSUPPORTED, "2^28"),
    (dict(K=1 << 28, N=1), sp.EUNSUPPORTED, "2^28"), (dict(K=1, N=1 << 28), sp.EUNSUPPORTED, "2^28")])
def test_norm_descriptors_that_are_refused(kw, status, text):
    refused(status, text, sp.rms_norm, norm(**kw), P, 0, 0, 0, Q)
    refused(status, text, norm(**kw).workspace_bytes)


def test_norm_calls_that_are_refused():
    f16, i8 = norm(), norm(out_dtype=sp.I8)
    for args, text in (((0, 0, 0, 0, Q), "NULL"), ((P, 0, 0, 0, 0), "NULL"), ((P, 0, 0, 0, Q, S), "scale"), ((P + 8, 0, 0, 0, Q), "16-byte"),
                       ((P, Q + 2, 0, 0, Q), "16-byte"), ((P, 0, 0, S + 4, Q), "16-byte"), ((P, 0, 0, 0, Q + 1), "16-byte"), ((P, 0, S + 2, 0, Q), "4-byte"),
                       ((P, 0, 0, Q, Q), "two buffers")):
        refused(sp.EINVAL, text, sp.rms_norm, f16, *args)
    refused(sp.EINVAL, "scale", sp.rms_norm, i8, P, 0, 0, 0, Q, 0)
    refused(sp.EINVAL, "4-byte", sp.rms_norm, i8, P, 0, 0, 0, Q, S + 1)
    refused(sp.EINVAL, "Y may be X", sp.rms_norm, i8, P, 0, 0, 0, P, S)
    refused(sp.EINVAL, "Y may be R", sp.rms_norm, i8, P, Q, 0, 0, Q, S)
    refused(sp.EINVAL, "Y may be X", sp.rms_norm, norm(ldx=17), P, 0, 0, 0, P)
    refused(sp.EINVAL, "Y may be R", sp.rms_norm, norm(ldh=17), P, Q, 0, 0, Q)
    refused(sp.EINVAL, "H may be X", sp.rms_norm, norm(ldh=17), P, 0, 0, P, Q)
    reserved = norm()
    reserved.fields.reserved[1] = 1
    refused(sp.EINVAL, "reserved", sp.rms_norm, reserved, P, 0, 0, 0, Q)
    assert sp.raw.sparsert_rms_norm(None, P, None, None, None, Q, None, None, 0, None) == sp.EINVAL
    size = ctypes.c_size_t()
    assert sp.raw.sparsert_rms_norm_workspace(None, ctypes.byref(size)) == sp.EINVAL
    assert sp.raw.sparsert_rms_norm_workspace(norm().handle, None) == sp.EINVAL
    split = norm(K=8192, N=64)
    need = split.workspace_bytes()
    assert need > 0
    refused(sp.EINVAL, "smaller", sp.rms_norm, split, P, 0, 0, 0, Q, 0, T, need - 1)
    refused(sp.EINVAL, "16-byte", sp.rms_norm, split, P, 0, 0, 0, Q, 0, T + 4, need)


@pytest.mark.parametrize("kw,status,text", [
    (dict(M=0), sp.EINVAL, "positive"), (dict(N=0), sp.EINVAL, "positive"), (dict(batch=70000), sp.EINVAL, "batch"), (dict(dtype=sp.I8), sp.EINVAL, "dtype"),
    (dict(ldc=15), sp.EINVAL, "ldc"), (dict(ldy=15), sp.EINVAL, "ldy"), (dict(M=1 << 20, ldc=512), sp.EUNSUPPORTED, "2 GiB"),
    (dict(M=1, N=1 << 28), sp.EUNSUPPORTED, "2^28")])
def test_dequantize_descriptors_that_are_refused(kw, status, text):
    a = dict(M=8, N=16)
    a.update(kw)
    refused(status, text, sp.dequantize, sp.Dequantize(**a), P, Q, S, T)


def test_dequantize_calls_that_are_refused():
    d = sp.Dequantize(8, 16)
    for args, text in (((0, 0, 0, Q), "NULL"), ((P, 0, 0, 0), "NULL"), ((P + 4, 0, 0, Q), "16-byte"), ((P, 0, 0, Q + 8), "16-byte"), ((P, S + 1, 0, Q), "4-byte"),
                       ((P, 0, S + 2, Q), "4-byte")):
        refused(sp.EINVAL, text, sp.dequantize, d, *args)
    refused(sp.EINVAL, "Y may be C", sp.dequantize, sp.Dequantize(8, 16, dtype=sp.F16), P, 0, 0, P)
    refused(sp.EINVAL, "Y may be C", sp.dequantize, sp.Dequantize(8, 16, ldy=17), P, 0, 0, P)
    d.fields.reserved[0] = -1
    refused(sp.EINVAL, "reserved", sp.dequantize, d, P, 0, 0, Q)
    assert sp.raw.sparsert_dequantize(None, P, None, None, Q, None) == sp.EINVAL


def adapter_set(**kw):
    a = dict(M=8, K=24, N=16, rank=4, count=3, dtype=sp.F16)
    a.update(kw)
    return sp.Adapters(**a)


@pytest.mark.parametrize("kw,status,text", [
    (dict(M=0), sp.EINVAL, "positive"), (dict(K=-3), sp.EINVAL, "positive"), (dict(N=0), sp.EINVAL, "positive"), (dict(batch=-2), sp.EINVAL, "batch"),
    (dict(rank=0), sp.EINVAL, "rank"), (dict(rank=257), sp.EINVAL, "rank"), (dict(count=0), sp.EINVAL, "count"), (dict(dtype=sp.I8), sp.EINVAL, "dtype"),
    (dict(x_dtype=sp.F32), sp.EINVAL, "x_dtype"), (dict(ldx=15), sp.EINVAL, "ldx"), (dict(ldc=15), sp.EINVAL, "ldc"), (dict(ldy=15), sp.EINVAL, "ldy"),
    (dict(M=1 << 20, N=1024), sp.EUNSUPPORTED, "2 GiB"), (dict(K=1 << 24, rank=256, N=1), sp.EUNSUPPORTED, "2 GiB"),
    (dict(M=1, K=1, N=1 << 26, batch=64), sp.EUNSUPPORTED, "tokens"), (dict(M=1 << 28, K=1, N=1), sp.EUNSUPPORTED, "2^28"),
    (dict(M=1, K=1 << 28, N=1), sp.EUNSUPPORTED, "2^28"), (dict(M=1, K=1, N=1 << 28, x_dtype=sp.I8), sp.EUNSUPPORTED, "2^28")])
def test_adapter_sets_that_are_refused(kw, status, text):
    refused(status, text, adapter_set(**kw).workspace_bytes)
    refused(status, text, sp.adapters, adapter_set(**kw), P, P, P, P, 0, Q, 0, 0, S, T, 1 << 40)


def test_adapters_calls_that_are_refused():
    d = adapter_set()
    need = d.workspace_bytes()
    assert need > 0
    good = [P, P, P, P, 0, Q, 0, 0, S, T, need]
    for at, value, text in ((0, 0, "NULL"), (1, 0, "NULL"), (2, 0, "NULL"), (3, 0, "NULL"), (5, 0, "NULL"), (8, 0, "NULL"), (9, 0, "NULL"),
                            (0, P + 8, "16-byte"), (1, P + 2, "16-byte"), (2, P + 4, "16-byte"), (5, Q + 1, "16-byte"), (8, S + 8, "16-byte"), (9, T + 4, "16-byte"),
                            (3, P + 2, "4-byte"), (4, P + 1, "4-byte"), (6, P, "scales"), (7, P, "scales"), (10, need - 1, "smaller"), (10, 0, "smaller"),
                            (8, P, "overlaps"), (9, S, "overlaps")):
        args = list(good)
        args[at] = value
        refused(sp.EINVAL, text, sp.adapters, d, *args)
    i8 = adapter_set(x_dtype=sp.I8)
    refused(sp.EINVAL, "4-byte", sp.adapters, i8, P, P, P, P, 0, Q, P + 1, 0, S, T, i8.workspace_bytes())
    refused(sp.EINVAL, "Y may be C", sp.adapters, i8, P, P, P, P, 0, Q, 0, 0, Q, T, i8.workspace_bytes())
    pitch = adapter_set(ldy=17)
    refused(sp.EINVAL, "Y may be C", sp.adapters, pitch, P, P, P, P, 0, Q, 0, 0, Q, T, pitch.workspace_bytes())
    d.fields.reserved[2] = 5
    refused(sp.EINVAL, "reserved", sp.adapters, d, *good)
    assert sp.raw.sparsert_adapters(None, P, P, P, P, None, Q, None, None, S, T, 1 << 30, None) == sp.EINVAL
    size = ctypes.c_size_t()
    assert sp.raw.sparsert_adapters_workspace(None, ctypes.byref(size)) == sp.EINVAL
    assert sp.raw.sparsert_adapters_workspace(adapter_set().handle, None) == sp.EINVAL


def test_more_workgroups_than_a_launch_can_have_are_refused():
    refused(sp.EUNSUPPORTED, "workgroups", sp.rms_norm, sp.RmsNorm(1, (1 << 28) - 1, dtype=sp.F32), P, 0, 0, 0, Q, 0, 0, 0)
    refused(sp.EUNSUPPORTED, "workgroups", sp.adapters, adapter_set(M=1, K=1, N=(1 << 28) - 1), P, P, P, P, 0, Q, 0, 0, S, T, 1 << 40)
    refused(sp.EUNSUPPORTED, "workgroups", sp.adapters, adapter_set(M=1, K=200, N=1 << 22, rank=256), P, P, P, P, 0, Q, 0, 0, S, T, 1 << 40)
    refused(sp.EUNSUPPORTED, "workgroups", sp.adapters, adapter_set(M=(1 << 28) - 1, K=8, N=1, rank=1), P, P, P, P, 0, Q, 0, 0, S, 0, 0)


@pytest.mark.parametrize("source", ["norm.hip", "dequantize.hip", "adapters.hip"])
def test_wide_stores_have_no_scalar_offset(source, tmp_path):
    """Behind a buffer store of 12 or 16 bytes with a scalar offset the compiler leaves no room before the data registers are written anew."""
    import subprocess
    import __graft_entry__ as entry
    flags = [a for a in entry.hipcc_command(str(tmp_path / "kernels.s")) if not a.startswith(entry.CSRC) and a not in ("-shared", "-fPIC", "-ldl")]
    subprocess.run(flags + ["--offload-device-only", "-S", os.path.join(entry.CSRC, source)], check=True, capture_output=True)
    for store in re.findall(r"^\s+buffer_store_dwordx[34] (.*)", (tmp_path / "kernels.s").read_text(), re.M):
        assert re.fullmatch(r"v\[\d+:\d+\], (v\d+|off), s\[\d+:\d+\], 0( .*)?", store.split(";")[0].strip()), store


def _outcome(call, args, kw):
    try:
        return call(*args, **kw)
    except Exception as e:
        return type(e).__name__, re.sub(r"\b_(rms_norm|dequantize|adapters)", r"\1", str(e)), getattr(e, "status", None)


@pytest.mark.parametrize("which", ["rms_norm", "dequantize", "adapters"])
def test_operator_calls_take_the_same_arguments_as_ctypes_does(which):
    """Every call ends in the library's argument checks: an address is null or off its alignment."""
    fast, general = getattr(sp, which), getattr(sp, "_" + which)
    made, words = {"rms_norm": (norm(), [P, 0, 0, 0, Q + 1, 0, 0, 0]), "dequantize": (sp.Dequantize(8, 16), [P, 0, 0, Q + 1]),
                   "adapters": (adapter_set(), [P, P, P, P, 0, Q, 0, 0, S + 1, T, 1 << 20])}[which]

    class Wide:
        handle = ctypes.c_void_p(made.handle)

    class Closed:
        handle = None

    forms = [((made, *words), {}), ((made, *words, 0), {}), ((made, *words, None), {}), ((made, *words, 7), {}), ((made, *words), {"stream": 0}),
             ((made, None, *words[1:]), {}), ((Wide, *words), {}), ((Closed, *words), {}), ((made, ctypes.c_void_p(P), *words[1:]), {}),
             ((made, *words[:-1], True), {}), ((made, -16, *words[1:]), {}), ((made, 2 ** 64 + 16, *words[1:]), {}), ((made, *words, "s"), {}), ((made, 1.5, *words[1:]), {}),
             ((made, *words[:2]), {}), ((), {}), ((made, *words, 0, 0), {}), ((made, *words), {"streem": 0}), ((None, *words), {}), ((made.handle, *words), {})]
    refused_ = 0
    for args, kw in forms:
        want = _outcome(general, args, kw)
        assert _outcome(fast, args, kw) == want, (args, kw)
        refused_ += want is not None and want[0] == "SparseRTError"
    assert refused_ >= 10


def test_operators_work_without_the_c_functions():
    import subprocess
    import sys
    code = """
import sys
sys.modules["paper_2008_11849_amd._fastcall"] = None   # what an import finds that was not built
from paper_2008_11849_amd import sparsert as sp
assert sp.rms_norm is sp._rms_norm and sp.dequantize is sp._dequantize and sp.adapters is sp._adapters
for call, made, args in ((sp.rms_norm, sp.RmsNorm(8, 16), (0, 0, 0, 0, 0)), (sp.dequantize, sp.Dequantize(8, 16), (0, 0, 0, 0)),
                         (sp.adapters, sp.Adapters(8, 8, 16, 4, 2), (0,) * 11)):
    try:
        call(made, *args, stream=0)
    except sp.SparseRTError as e:
        assert e.status == sp.EINVAL
    else:
        raise SystemExit("not refused")
"""
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]


@pytest.mark.skipif(sp._fastcall is None, reason="built without the Python headers")
def test_the_operators_are_called_through_the_c_functions():
    assert sp.rms_norm is sp._fastcall.rms_norm and sp.dequantize is sp._fastcall.dequantize and sp.adapters is sp._fastcall.adapters
