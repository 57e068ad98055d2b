"""Every kernel that an operator's call can take, on the GPU: calls of the sizes that take it, against plain statements in 64 bits.

Which kernels a call takes is read from a capture of it, so that a change of the rules that choose shows here."""
import ctypes
import re

import numpy as np
import pytest

import operators_ref as plain
from test_gpu_operators import (DEV, KIND, AdaptersCall, Wide, adapters_case, at, norm_case, run_norm, sp, stream, torch, vector)

pytestmark = pytest.mark.gpu

SOMEWHERE = [0x7f0000000000 + (i << 40) for i in range(8)]   # addresses for calls that are captured and not run


class _Node(ctypes.Structure):
    """hipKernelNodeParams"""
    _fields_ = [("block", ctypes.c_uint32 * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint32 * 3),
                ("params", ctypes.c_void_p), ("shared", ctypes.c_uint32)]


def kernels(call):
    """The (mangled) names of the kernels that a call launches, in their order.  They do not run."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    hip, handle, count = sp.raw, ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(handle, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(handle, nodes, ctypes.byref(count)) == 0
    name = hip.hipKernelNameRefByPtr
    name.restype, name.argtypes = ctypes.c_char_p, [ctypes.c_void_p, ctypes.c_void_p]
    names = []
    for n in nodes:
        p = _Node()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(n), ctypes.byref(p)) == 0
        names.append(name(p.func, None).decode())
    return names


def named(kernel, types, *values):
    """A kernel's name with these template arguments, up to the last of them that is given."""
    return kernel + "I" + "".join(types) + "".join("Lb%dE" % v if isinstance(v, bool) else "Li%dE" % v for v in values)


LETTER = {np.dtype(np.float32): "f", np.dtype(np.float16): "DF16_", np.dtype(np.int8): "a", np.dtype(np.int32): "i"}


# ---------------------------------------------------------------- norm

def norm_kernels(K, N, batch, dtype, out, split):
    d = sp.RmsNorm(K, N, dtype=KIND[np.dtype(dtype)], out_dtype=KIND[np.dtype(out)], batch=batch)
    x, r, g, h, y, scale, ws, _ = SOMEWHERE
    return kernels(lambda: sp.rms_norm(d, x, r, g, h, y, scale if out == np.int8 else 0, *((ws, d.workspace_bytes()) if split else (0, 0)), stream()))


def norm_both(K, N, batch, dtype, split, kernel, *values, pads=(0, 0, 0), last=(), inplace=""):
    """A call with a result of its own type and one to int8; the kernels' names and results."""
    x, r, g = norm_case(np.random.default_rng(K + N), K, N, dtype, batch)
    for out in (dtype, np.int8):
        got = norm_kernels(K, N, batch, dtype, out, split)
        if split:
            assert named("norm_sums_kernel", [LETTER[np.dtype(dtype)]], out == np.int8, *values) in got[0] and len(got) == 2
        else:
            assert len(got) == 1
        assert named(kernel, [LETTER[np.dtype(dtype)]], out == np.int8, *values, *last) in got[-1], got
        if out == np.int8 and "y=" in inplace:
            continue
        y, scale, h = run_norm(split, x, r, g, out, pads=pads, inplace=inplace)
        plain.check_norm(y, scale, h, x, r, g, 1e-5)


def pads_of(N):
    return (0, 0, 0) if N % 8 == 0 else (5, 3, 9)


# Columns of a lane, lanes of a strip, tokens, batch.  A workgroup takes 1024 / lanes rows in a pass.
ONE = [(np.float16, 1, 1, 1, 1), (np.float16, 1, 2, 2, 1), (np.float16, 1, 4, 3, 2), (np.float16, 1, 8, 5, 1), (np.float16, 4, 1, 17, 1), (np.float16, 8, 1, 136, 1), (np.float16, 8, 1, 131, 2),
       (np.float16, 8, 2, 4101, 1), (np.float16, 8, 4, 8200, 1), (np.float16, 8, 8, 8195, 2),
       (np.float32, 1, 1, 1, 1), (np.float32, 1, 2, 2, 1), (np.float32, 1, 4, 3, 2), (np.float32, 4, 1, 18, 1), (np.float32, 4, 1, 136, 1), (np.float32, 4, 2, 2051, 1), (np.float32, 4, 4, 4104, 1),
       (np.float32, 4, 8, 4099, 2)]


@pytest.mark.parametrize("passes", [1, 2, 4, 8, 0])
@pytest.mark.parametrize("dtype,V,L,N,batch", ONE)
def test_norms_as_one_kernel(dtype, V, L, N, batch, passes):
    """1 to 8 passes stay in registers; 0: more, four of them at a time, fetched twice."""
    rows = 1024 // L
    K = {1: rows * 2 // 3, 2: 2 * rows - 1, 4: 3 * rows, 8: 7 * rows + 5, 0: 8 * rows + 1}[passes]
    norm_both(K, N, batch, dtype, False, "norm_kernel", V, L, passes or 4, passes > 0, pads=pads_of(N))


# FAR: the sum is not to stay in the caches, from 100 MB on.
SPLIT = [(np.float16, 1, 2, 8524, 1, 1, False), (np.float16, 1, 2, 8301, 2, 1, False), (np.float16, 1, 4, 4099, 3, 1, False), (np.float16, 1, 8, 4097, 7, 1, False),
         (np.float16, 8, 1, 6397, 8, 1, False), (np.float16, 8, 2, 5680, 13, 1, False), (np.float16, 8, 4, 5001, 30, 2, False), (np.float16, 8, 8, 4096, 45, 1, False),
         (np.float16, 8, 16, 2900, 2051, 1, False), (np.float16, 8, 16, 2900, 1041, 2, False), (np.float16, 8, 16, 4100, 3600, 1, True), (np.float16, 8, 16, 5125, 2901, 1, True),
         (np.float32, 1, 2, 8232, 1, 1, False), (np.float32, 1, 2, 8301, 2, 1, False), (np.float32, 1, 4, 4099, 3, 1, False), (np.float32, 4, 1, 8195, 4, 1, False), (np.float32, 4, 2, 5681, 7, 1, False),
         (np.float32, 4, 4, 3559, 13, 1, False), (np.float32, 4, 8, 4096, 45, 1, False), (np.float32, 4, 16, 4000, 1001, 1, False), (np.float32, 4, 16, 8200, 1000, 1, True),
         (np.float32, 4, 16, 4100, 1001, 2, True)]


@pytest.mark.parametrize("dtype,V,L,K,N,batch,far", SPLIT)
def test_norms_as_two_kernels(dtype, V, L, K, N, batch, far):
    norm_both(K, N, batch, dtype, True, "norm_results_kernel", V, L, pads=pads_of(N), last=(far,))


@pytest.mark.parametrize("inplace", ["h=r", "h=r y=x", "h=x y=r"])
@pytest.mark.parametrize("dtype,V,K,N", [(np.float16, 8, 5125, 2901), (np.float32, 4, 4099, 2002)])
def test_norms_beyond_the_caches_in_place(dtype, V, K, N, inplace):
    norm_both(K, N, 1, dtype, True, "norm_results_kernel", V, 16, pads=(3, 3, 3), last=(True,), inplace=inplace)


# ---------------------------------------------------------------- dequantisation

@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("V,L,N", [(1, 1, 1), (1, 4, 2), (1, 4, 3), (4, 1, 4), (4, 4, 5), (4, 4, 16), (4, 16, 17), (4, 16, 63), (4, 64, 65), (4, 64, 260)])
def test_dequantisations(V, L, N, dtype):
    rng = np.random.default_rng(N)
    for M in (1, 256 // L * 4, 1025):
        d = sp.Dequantize(M, N, dtype=KIND[np.dtype(dtype)], batch=2, ldc=N + 1, ldy=N + 3)
        got = kernels(lambda: sp.dequantize(d, *SOMEWHERE[:4], stream()))
        assert len(got) == 1 and named("dequantize_kernel", [LETTER[np.dtype(dtype)]], V, L) in got[0], got
        c = rng.integers(-20000, 20000, (2, M, N)).astype(np.int32)
        row, col = rng.uniform(1e-4, 1e-3, M).astype(np.float32), rng.uniform(0.01, 0.1, (2, N)).astype(np.float32)
        C, Y, R, S = Wide(c.shape, N + 1, np.int32, c), Wide(c.shape, N + 3, dtype), vector(row), vector(col)
        sp.dequantize(d, C.at, at(R), at(S), Y.at, stream())
        torch.cuda.synchronize()
        plain.check_dequantize(Y.read(), c, row, col)


# ---------------------------------------------------------------- adapters

KINDS = ["f16", "f32", "i8f16", "i8f32"]


def adapter_kernels(M, K, N, rank, count, kind, batch=1):
    w = sp.F32 if kind in ("f32", "i8f32") else sp.F16
    d = sp.Adapters(M, K, N, rank, count, dtype=w, x_dtype=sp.I8 if kind.startswith("i8") else w, batch=batch)
    return kernels(lambda: sp.adapters(d, *SOMEWHERE[:4], 0, SOMEWHERE[4], 0, 0, SOMEWHERE[5], SOMEWHERE[6], d.workspace_bytes(), stream()))


def types_of(kind):
    w = "f" if kind in ("f32", "i8f32") else "DF16_"
    return ["a" if kind.startswith("i8") else w, w], ["i" if kind.startswith("i8") else w, w]


def adapters_checked(M, K, N, rank, count, kind, index):
    call = AdaptersCall(adapters_case(np.random.default_rng(M + N + rank), M, K, N, rank, count, kind, index=index), pads=(0, 0, 0) if N % 2 == 0 else (1, 2, 3))
    call.run()
    y = call.read()
    call.check(y)
    call.run()
    assert call.read().tobytes() == y.tobytes()


# Blocks of 16 ranks (1, 2 and 4 are built), and whether rows of `down` and of `up` are of whole 16 bytes in either type.
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("blocks,whole_k,whole_rank,M,K,N,rank,count,index", [
    (1, True, True, 300, 64, 3300, 8, 1, "runs"), (1, False, False, 301, 67, 3301, 10, 1, "runs"), (1, True, True, 1030, 512, 1100, 16, 2, "tokens"),
    (2, True, True, 270, 264, 2300, 24, 2, "runs"), (2, False, False, 271, 269, 2301, 29, 1, "tokens"), (4, True, True, 512, 520, 1300, 64, 3, "tokens"),
    (4, False, False, 517, 523, 1303, 63, 2, "runs"), (4, True, False, 512, 520, 1301, 34, 2, "runs")])
def test_adapters_in_tiles(blocks, whole_k, whole_rank, M, K, N, rank, count, index, kind):
    shrink, expand = types_of(kind)
    got = adapter_kernels(M, K, N, rank, count, kind)
    assert len(got) == 2 and named("shrink_tiles_kernel", shrink, blocks, whole_k) in got[0] and named("expand_tiles_kernel", expand, blocks, whole_rank) in got[1], got
    adapters_checked(M, K, N, rank, count, kind, index)


# Tokens of a wave (1, 2, 4), of a group (1: fewer than eight tokens).
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("each,group,whole_k,whole_rank,M,K,N,rank,count,index", [
    (1, 1, True, True, 300, 520, 5, 16, 3, "tokens"), (1, 1, False, False, 301, 515, 7, 13, 3, "tokens"), (1, 8, True, True, 300, 1024, 40, 16, 3, "tokens"),
    (1, 8, False, False, 301, 1029, 41, 21, 3, "tokens"), (2, 8, True, True, 4096, 8, 130, 16, 2, "runs"), (2, 8, False, False, 4100, 9, 131, 13, 2, "tokens"),
    (4, 8, True, True, 4096, 16, 200, 16, 2, "runs"), (4, 8, False, False, 4101, 9, 201, 13, 2, "tokens")])
def test_adapters_token_by_token(each, group, whole_k, whole_rank, M, K, N, rank, count, index, kind):
    shrink, expand = types_of(kind)
    got = adapter_kernels(M, K, N, rank, count, kind)
    assert len(got) == 2 and named("shrink_tokens_kernel", shrink, group, whole_k) in got[0] and named("expand_tokens_kernel", expand, each, whole_rank) in got[1], got
    adapters_checked(M, K, N, rank, count, kind, index)


# No tiles: ranks above 64, and in half odd ones below 8.
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,K,N,rank,count,index", [(1030, 520, 1100, 65, 2, "runs"), (520, 520, 1101, 128, 2, "runs"), (600, 300, 700, 256, 3, "tokens"), (1001, 1001, 1000, 255, 1, "runs"),
                                                    (2050, 64, 1500, 3, 1, "runs"), (2051, 65, 1501, 7, 2, "tokens"), (1030, 1030, 2500, 5, 1, "runs")])
def test_adapters_of_many_tokens_without_tiles(M, K, N, rank, count, index, kind):
    if rank > 64 or rank * (2 if kind.endswith("f16") else 4) % 4:
        assert all("tokens_kernel" in k for k in adapter_kernels(M, K, N, rank, count, kind))
    adapters_checked(M, K, N, rank, count, kind, index)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("K,rank,whole", [(1024, 8, True), (771, 13, False)])
def test_adapters_of_a_single_token(K, rank, whole, kind):
    (x, w), (c, _) = types_of(kind)
    got = adapter_kernels(300, K, 1, rank, 3, kind, 2)
    assert len(got) == 1 and named("one_token_kernel", [x, c, w], whole) in got[0], got
    s = adapters_case(np.random.default_rng(K), 300, K, 1, rank, 3, kind, 2)
    s["index"][:] = [[2], [0]]
    call = AdaptersCall(s)
    call.run()
    call.check(call.read())


def test_names_of_kernels_are_read():
    """The names above are compared with what a capture says: it names the kernel of a call whose kernel is known."""
    got = norm_kernels(1024, 1, 1, np.float16, np.float16, False)
    assert len(got) == 1 and re.match(r"_ZN8sparsert\d+norm_kernelI", got[0])
