"""The operators around the products on the GPU, against plain statements of them in 64 bits (operators_ref.py)."""
import numpy as np
import pytest

import operators_ref as plain
from oracle import ref
from paper_2008_11849_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2008_11849_amd import sparsert as sp  # noqa: E402

DEV = "cuda:0"
KIND = {np.dtype(np.float32): sp.F32, np.dtype(np.float16): sp.F16, np.dtype(np.int8): sp.I8}
POISON = {np.dtype(np.float32): np.nan, np.dtype(np.float16): np.nan, np.dtype(np.int8): 113, np.dtype(np.int32): 1234567891}


def stream():
    return torch.cuda.current_stream().cuda_stream


class Wide:
    """[batch, rows, ld] on the GPU of which the first N columns are the operand; the others hold a poison value."""

    def __init__(self, shape, ld, dtype, values=None):
        self.N, self.dtype = shape[-1], np.dtype(dtype)
        host = np.full(shape[:-1] + (ld,), POISON[self.dtype], dtype=dtype)
        if values is not None:
            host[..., :self.N] = values
        self.before, self.t = host, torch.from_numpy(host).to(DEV)
        self.at = self.t.data_ptr()

    def read(self):
        """The operand; what is behind it has to be as it was."""
        got = self.t.cpu().numpy()
        assert got[..., self.N:].tobytes() == self.before[..., self.N:].tobytes()
        return got[..., :self.N]


def vector(v, dtype=np.float32):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=dtype)).to(DEV)


def at(t):
    return 0 if t is None else t.data_ptr()


# ---------------------------------------------------------------- norm

def norm_case(rng, K, N, dtype, batch=1, residual=True, gamma=True):
    x = rng.standard_normal((batch, K, N)).astype(dtype)
    r = (3 * rng.standard_normal((batch, K, N))).astype(dtype) if residual else None
    g = rng.uniform(-1.5, 1.5, K).astype(np.float32) if gamma else None
    return x, r, g


class Scratch:
    """A workspace of NaN, with 64 bytes behind it that are not its own."""

    def __init__(self, need):
        self.need, self.t = need, torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)

    def args(self):
        return (self.t.data_ptr(), self.need) if self.need else (0, 0)

    def check(self):
        assert (self.t[self.need:].cpu().numpy() == 255).all()


@pytest.fixture(params=["one kernel", "workspace"])
def way(request):
    """Norms without a workspace, and with one, which splits long columns over two kernels."""
    return request.param == "workspace"


def run_norm(way, x, r, g, out, eps=1e-5, pads=(0, 0, 0), keep=True, inplace=""):
    """Returns (y, scale, h).  pads: of X, of R and H, of Y.  inplace: "h=r", "h=x", "y=x", "y=r" in any combination."""
    b, K, N = x.shape
    X = Wide(x.shape, N + pads[0], x.dtype, x)
    R = Wide(x.shape, N + pads[1], x.dtype, r) if r is not None else None
    H = R if "h=r" in inplace else X if "h=x" in inplace else Wide(x.shape, N + pads[1], x.dtype) if keep else None
    Y = X if "y=x" in inplace else R if "y=r" in inplace else Wide(x.shape, N + pads[2], out)
    scale = torch.full((b, N), -7.0, device=DEV) if np.dtype(out) == np.int8 else None
    G = vector(g) if g is not None else None
    d = sp.RmsNorm(K, N, dtype=KIND[x.dtype], out_dtype=KIND[np.dtype(out)], eps=eps, batch=b, ldx=N + pads[0], ldh=N + pads[1], ldy=N + pads[2])
    ws = Scratch(d.workspace_bytes())
    sp.rms_norm(d, X.at, R.at if R else 0, at(G), H.at if H else 0, Y.at, at(scale), *(ws.args() if way else (0, 0)), stream())
    torch.cuda.synchronize()
    ws.check()
    if not inplace:
        assert X.t.cpu().numpy().tobytes() == X.before.tobytes()
    return Y.read(), None if scale is None else scale.cpu().numpy(), H.read() if H else None


@pytest.mark.parametrize("out", ["same", "int8"])
@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("N", [1, 2, 3, 7, 8, 9, 16, 31, 33, 64, 65, 130, 517])
def test_norm_at_the_edges_of_its_strips(N, dtype, out, way):
    rng = np.random.default_rng(N)
    for K in (1, 2, 63, 64, 65, 257, 1027):
        x, r, g = norm_case(rng, K, N, dtype, batch=1 if N > 100 else 2)
        y, scale, h = run_norm(way, x, r, g, dtype if out == "same" else np.int8, pads=(0, 0, 0) if K % 2 else (5, 3, 9))
        plain.check_norm(y, scale, h, x, r, g, 1e-5)


@pytest.mark.parametrize("out", ["same", "int8"])
@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("K,N,batch", [(4096, 4, 1), (4096, 40, 1), (8192, 24, 1), (8200, 17, 2), (16385, 5, 1), (40000, 3, 1), (5000, 1030, 1), (130, 5003, 1)])
def test_norm_of_long_columns_and_many_tokens(K, N, batch, dtype, out, way):
    x, r, g = norm_case(np.random.default_rng(K), K, N, dtype, batch)
    y, scale, h = run_norm(way, x, r, g, dtype if out == "same" else np.int8, pads=(8, 8, 8) if N % 8 == 0 else (0, 1, 2))
    plain.check_norm(y, scale, h, x, r, g, 1e-5)


@pytest.mark.parametrize("out", ["same", "int8"])
@pytest.mark.parametrize("residual,gamma,keep", [(False, True, False), (True, False, False), (False, False, True), (True, True, False), (False, True, True)])
def test_norm_without_residual_weights_or_sum(residual, gamma, keep, out, way):
    rng = np.random.default_rng(3)
    for dtype, K, N in ((np.float16, 300, 70), (np.float32, 9000, 20)):
        x, r, g = norm_case(rng, K, N, dtype, residual=residual, gamma=gamma)
        y, scale, h = run_norm(way, x, r, g, dtype if out == "same" else np.int8, keep=keep)
        plain.check_norm(y, scale, h, x, r, g, 1e-5)


@pytest.mark.parametrize("inplace", ["h=r", "h=x", "y=x", "y=r", "h=r y=x", "h=x y=r"])
@pytest.mark.parametrize("K,N", [(200, 19), (1027, 96), (9001, 21)])
def test_norm_in_place(K, N, inplace, way):
    rng = np.random.default_rng(K)
    for dtype in (np.float16, np.float32):
        x, r, g = norm_case(rng, K, N, dtype, batch=2)
        y, _, h = run_norm(way, x, r, g, dtype, pads=(3, 3, 3), inplace=inplace)
        plain.check_norm(y, None, h, x, r, g, 1e-5)


@pytest.mark.parametrize("K", [70, 2000, 9000])
def test_norm_of_columns_with_zeros_infinities_and_undefined_values(K, way):
    rng = np.random.default_rng(4)
    for dtype in (np.float16, np.float32):
        x, _, g = norm_case(rng, K, 24, dtype, residual=False)
        x[0, :, 3] = 0
        x[0, :, 4] = np.finfo(dtype).smallest_subnormal
        x[0, 5, 7], x[0, K - 1, 9], x[0, K // 2, 15] = np.inf, np.nan, -np.inf
        y, _, _ = run_norm(way, x, None, g, dtype)
        sound = [n for n in range(24) if n not in (7, 9, 15)]
        plain.check_norm(y[..., sound], None, None, x[..., sound], None, g, 1e-5)
        assert np.isnan(y[0, :, 9]).all() and np.isnan(y[0, 5, 7]) and np.isnan(y[0, K // 2, 15])
        others = np.delete(y[0, :, 7], 5)
        assert (others == 0).all()                 # 1 / infinity
        q, scale, _ = run_norm(way, x, None, g, np.int8)
        plain.check_norm(q[..., sound], scale[..., sound], None, x[..., sound], None, g, 1e-5)
        assert (q[0, :, 3] == 0).all() and scale[0, 3] == 0
        for n in (7, 9, 15):
            assert (q[0, :, n] == 0).all() and np.isnan(scale[0, n])
    x = np.full((1, 90, 9), 1e-3, dtype=np.float32)
    g = np.ones(90, dtype=np.float32)
    x[0, 4, 2], g[8] = 1e25, np.nan                # squares beyond binary32; an undefined weight
    q, scale, _ = run_norm(way, x, None, g, np.int8)
    assert (q == 0).all() and np.isnan(scale).all()
    g[8] = 1.0
    q, scale, _ = run_norm(way, x, None, g, np.int8)
    assert np.isnan(scale[0, 2]) and (q[0, :, 2] == 0).all() and np.isfinite(np.delete(scale[0], 2)).all()


def test_norm_ties_go_to_the_even_integer(way):
    v = np.zeros((1, 8, 4), dtype=np.float32)
    v[0, :, 0] = [127, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]
    v[0, :, 1] = -v[0, :, 0]
    q, scale, _ = run_norm(way, v, None, None, np.int8)
    assert q[0, :, 0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126] and q[0, :, 1].tolist() == [-127, 0, -2, -2, 0, 2, 2, -126]


# ---------------------------------------------------------------- dequantize

@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("M,N,batch,pads", [(1, 1, 1, (0, 0)), (3, 7, 2, (0, 1)), (64, 64, 1, (0, 0)), (65, 129, 1, (3, 0)), (7, 1000, 3, (8, 8)), (1000, 9, 1, (0, 7)),
                                            (333, 2048, 1, (0, 0)), (130, 4093, 1, (4, 4)), (5003, 16, 1, (16, 0)), (2, 300001, 1, (0, 0))])
def test_dequantize(M, N, batch, pads, dtype):
    rng = np.random.default_rng(M + N)
    c = rng.integers(-20000, 20000, (batch, M, N)).astype(np.int32)
    c.reshape(-1)[:1] = 2 ** 31 - 1
    row, col = rng.uniform(1e-4, 1e-3, M).astype(np.float32), rng.uniform(0.01, 0.1, (batch, N)).astype(np.float32)
    row[0] = 1e-9
    for use_row, use_col in ((True, True), (False, True), (True, False)):
        C, Y = Wide(c.shape, N + pads[0], np.int32, c), Wide(c.shape, N + pads[1], dtype)
        r, k = vector(row) if use_row else None, vector(col) if use_col else None
        with np.errstate(over="ignore"):
            want = plain.dequantize(c, row if use_row else None, col if use_col else None)
        if dtype == np.float16 and np.abs(want).max() > 60000:
            continue
        sp.dequantize(sp.Dequantize(M, N, dtype=KIND[np.dtype(dtype)], batch=batch, ldc=N + pads[0], ldy=N + pads[1]), C.at, at(r), at(k), Y.at, stream())
        torch.cuda.synchronize()
        plain.check_dequantize(Y.read(), c, row if use_row else None, col if use_col else None)


def test_dequantize_in_place_and_of_undefined_scales():
    rng = np.random.default_rng(1)
    c = rng.integers(-20000, 20000, (2, 70, 131)).astype(np.int32)
    col = rng.uniform(0.01, 0.1, (2, 131)).astype(np.float32)
    col[1, 77] = np.nan
    c[1, 3, 77] = 0
    C, k = Wide(c.shape, 140, np.int32, c), vector(col)
    sp.dequantize(sp.Dequantize(70, 131, batch=2, ldc=140, ldy=140), C.at, 0, at(k), C.at, stream())
    torch.cuda.synchronize()
    y = C.read().view(np.float32)
    assert np.isnan(y[1, :, 77]).all()
    y, c, col = y.copy(), c, col.copy()
    y[1, :, 77], c[1, :, 77], col[1, 77] = 0, 0, 1
    plain.check_dequantize(y, c, None, col)


# ---------------------------------------------------------------- adapters

def adapters_case(rng, M, K, N, rank, count, kind, batch=1, index="tokens"):
    w = np.float32 if kind in ("f32", "i8f32") else np.float16
    s = {"down": (rng.standard_normal((count, rank, K)) / np.sqrt(K)).astype(w), "up": (rng.standard_normal((count, M, rank)) / np.sqrt(rank)).astype(w),
         "alpha": rng.uniform(0.25, 2, count).astype(np.float32), "row": None, "col": None}
    if kind.startswith("i8"):
        s["x"] = rng.integers(-127, 128, (batch, K, N)).astype(np.int8)
        s["c"] = rng.integers(-20000, 20000, (batch, M, N)).astype(np.int32)
        s["row"], s["col"] = rng.uniform(1e-4, 1e-3, M).astype(np.float32), rng.uniform(0.01, 0.03, (batch, N)).astype(np.float32)
    else:
        s["x"], s["c"] = rng.standard_normal((batch, K, N)).astype(w), rng.standard_normal((batch, M, N)).astype(w)
    if index == "tokens":
        s["index"] = rng.integers(-1, count, (batch, N)).astype(np.int32)
    else:   # runs of tokens of ragged lengths
        s["index"] = np.sort(rng.integers(-1, count, (batch, N)).astype(np.int32), axis=1)
    return s


class AdaptersCall:
    """The operands of a call on the GPU; run() launches it, read() is its result."""

    def __init__(self, s, pads=(0, 0, 0), inplace=False):
        (self.b, self.K, self.N), self.M = s["x"].shape, s["c"].shape[1]
        self.s, self.w = s, s["down"].dtype
        N = self.N
        self.X, self.C = Wide(s["x"].shape, N + pads[0], s["x"].dtype, s["x"]), Wide(s["c"].shape, N + pads[1], s["c"].dtype, s["c"])
        self.Y = self.C if inplace else Wide(s["c"].shape, N + pads[2], self.w)
        self.v = {k: None if s[k] is None else torch.from_numpy(np.ascontiguousarray(s[k])).to(DEV) for k in ("down", "up", "index", "alpha", "row", "col")}
        self.d = sp.Adapters(self.M, self.K, N, s["down"].shape[1], s["down"].shape[0], dtype=KIND[self.w], x_dtype=KIND[s["x"].dtype], batch=self.b,
                             ldx=N + pads[0], ldc=N + pads[1], ldy=N + pads[2])
        need = self.d.workspace_bytes()
        self.ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)     # (NaN where floats lie; the last 64 bytes are not its own)
        self.need = need

    def run(self):
        v = self.v
        sp.adapters(self.d, self.X.at, at(v["down"]), at(v["up"]), at(v["index"]), at(v["alpha"]), self.C.at, at(v["row"]), at(v["col"]), self.Y.at,
                    self.ws.data_ptr(), self.need, stream())

    def read(self):
        torch.cuda.synchronize()
        assert (self.ws[self.need:].cpu().numpy() == 255).all()
        y = self.Y.read()
        return y if y.dtype == self.w else y.view(self.w)

    def check(self, y):
        plain.check_adapters(y, *(self.s[k] for k in ("x", "down", "up", "index", "alpha", "c", "row", "col")))


@pytest.mark.parametrize("kind", ["f16", "f32", "i8f16", "i8f32"])
@pytest.mark.parametrize("N", [1, 2, 5, 15, 16, 17, 31, 32, 33, 63, 65, 130, 257])
def test_adapters_at_the_edges_of_their_tiles(N, kind):
    rng = np.random.default_rng(N)
    for M, K, rank, count in ((1, 1, 1, 1), (16, 32, 16, 3), (33, 31, 5, 2), (70, 65, 17, 4), (130, 257, 33, 6), (64, 1027, 64, 2)):
        call = AdaptersCall(adapters_case(rng, M, K, N, rank, count, kind, batch=2 if N < 40 else 1), pads=(0, 0, 0) if rank % 2 == 0 else (5, 3, 9))
        call.run()
        call.check(call.read())


@pytest.mark.parametrize("kind", ["f16", "f32", "i8f16"])
@pytest.mark.parametrize("M,K,N,rank,count,index", [
    (1024, 4096, 1, 8, 2, "tokens"), (512, 4096, 3, 16, 40, "tokens"), (300, 2048, 48, 16, 32, "tokens"), (520, 768, 1000, 16, 9, "runs"), (96, 8192, 70, 8, 5, "runs"),
    (70, 300, 40, 100, 3, "tokens"), (70, 300, 40, 256, 3, "runs"), (2048, 70, 33, 129, 2, "tokens"), (64, 128, 4099, 4, 100, "tokens"), (4099, 96, 20, 12, 3, "runs")])
def test_adapters_of_real_sizes(M, K, N, rank, count, index, kind):
    call = AdaptersCall(adapters_case(np.random.default_rng(M + N), M, K, N, rank, count, kind, index=index), pads=(0, 8, 8) if N % 8 == 0 else (1, 2, 0))
    call.run()
    y = call.read()
    call.check(y)
    call.run()
    assert call.read().tobytes() == y.tobytes()     # the same operands, the same bits


# A single token is one kernel, without workspace, up to 65536 elements of an adapter's `down` (16384 where K is odd in its 16 bytes) and rank 64.
@pytest.mark.parametrize("kind", ["f16", "f32", "i8f16", "i8f32"])
@pytest.mark.parametrize("M,K,rank,batch", [
    (64, 4096, 16, 1), (65, 4104, 16, 1), (63, 4095, 3, 2), (1, 1024, 64, 1), (129, 1023, 16, 3), (200, 1024, 63, 1), (200, 1023, 17, 1), (7, 600, 61, 1), (70, 7, 5, 4), (5, 3, 64, 1),
    (1030, 256, 64, 1), (64, 256, 65, 1), (3, 1, 2, 70), (300, 12000, 4, 1), (90, 515, 33, 2)])
def test_adapters_of_one_token(M, K, rank, batch, kind):
    rng = np.random.default_rng(M + K + rank)
    s = adapters_case(rng, M, K, 1, rank, 3, kind, batch)
    s["index"][0] = 2
    for pads in ((0, 0, 0), (6, 1, 3)):
        call = AdaptersCall(s, pads=pads)
        for _ in range(2):
            call.run()
            call.check(call.read())


@pytest.mark.parametrize("kind", ["f16", "f32", "i8f32"])
def test_one_token_is_computed_from_its_own_column_and_adapter_alone(kind):
    rng = np.random.default_rng(5)
    M, K, rank, batch = 70, 203, 13, 8
    s = adapters_case(rng, M, K, 1, rank, 4, kind, batch)
    s["index"][:, 0] = [0, 1, -1, 4, 0, np.iinfo(np.int32).min, 2, 0]
    if kind != "i8f32":
        s["x"][1, :, 0], s["x"][2, 5, 0], s["x"][3, K - 1, 0] = np.nan, np.nan, np.inf     # of token 1 alone; tokens 2 and 3 have no adapter
    s["down"][2, rank - 1, K - 1], s["up"][2, M - 1, rank - 1] = np.inf, np.nan            # of token 6 alone
    s["down"][3], s["up"][3] = np.nan, np.nan                                              # of none
    sound = [0, 4, 7] + ([1] if kind == "i8f32" else [])
    clean = {k: None if v is None else v.copy() for k, v in s.items()}
    for k in ("x", "down", "up"):
        clean[k] = np.where(np.isfinite(clean[k]), clean[k], 0).astype(clean[k].dtype)
    got, want = (AdaptersCall(v, pads=(1, 1, 1)) for v in (s, clean))
    got.run()
    want.run()
    a, b = got.read(), want.read()
    want.check(b)
    assert got.need == 0
    assert np.array_equal(a[sound], b[sound]) and not np.isfinite(a[6]).all()
    none = [2, 3, 5]
    assert np.array_equal(a[none], b[none])
    if kind != "i8f32":
        assert np.array_equal(a[none], s["c"][none]) and not np.isfinite(a[1]).any()


@pytest.mark.parametrize("kind", ["f16", "i8f32"])
def test_one_token_needs_no_workspace_and_is_captured(kind):
    s = adapters_case(np.random.default_rng(11), 130, 512, 1, 16, 3, kind, 2)
    s["index"][:] = 1
    call = AdaptersCall(s)
    call.run()
    y = call.read()
    call.check(y)
    v = call.v

    def without():
        sp.adapters(call.d, call.X.at, at(v["down"]), at(v["up"]), at(v["index"]), at(v["alpha"]), call.C.at, at(v["row"]), at(v["col"]), call.Y.at, 0, 0, stream())

    without()
    assert call.read().tobytes() == y.tobytes()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        without()
    for i in range(3):
        v["index"][0, 0] = i      # the graph reads what lies there when it runs
        graph.replay()
        s["index"][0, 0] = i
        call.check(call.read())


# Calls whose tokens would read more weights than their tiles of 64 share go to the matrix cores: over 34 MB with one adapter, 4 MB more for each other one, twice that in single precision.
@pytest.mark.parametrize("kind", ["f16", "f32", "i8f16", "i8f32"])
@pytest.mark.parametrize("M,K,N,rank,count,batch,index", [
    (520, 512, 1100, 64, 3, 1, "runs"), (517, 513, 1101, 64, 2, 1, "runs"), (500, 600, 1500, 64, 40, 1, "tokens"), (530, 600, 1063, 33, 3, 1, "tokens"),
    (300, 270, 2050, 4, 1, 2, "runs"), (301, 263, 4103, 6, 2, 1, "runs"), (1030, 264, 1200, 24, 2, 1, "tokens"), (700, 1300, 450, 20, 1, 3, "runs"),
    (17, 9, 10303, 64, 1, 1, "runs"), (3, 1025, 1130, 40, 1, 1, "tokens"), (2100, 8, 700, 62, 1, 1, "runs"), (64, 4100, 257, 57, 2, 1, "runs"), (1000, 1000, 64, 64, 1, 5, "runs"),
    (900, 900, 65, 64, 1, 5, "tokens")])
def test_adapters_of_many_tokens(M, K, N, rank, count, batch, index, kind):
    call = AdaptersCall(adapters_case(np.random.default_rng(M + N), M, K, N, rank, count, kind, batch, index), pads=(0, 0, 0) if N % 2 == 0 else (1, 2, 3))
    call.run()
    y = call.read()
    call.check(y)
    call.run()
    assert call.read().tobytes() == y.tobytes()


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_many_tokens_are_computed_from_their_own_column_and_adapter_alone(kind):
    rng = np.random.default_rng(18)
    N = 1100
    s = adapters_case(rng, 520, 514, N, 63, 4, kind)
    s["index"][0, :] = np.where(np.arange(N) < 300, np.arange(N) // 150, np.arange(N) % 7 - 2)     # runs, then requests of a token each, some without adapter
    s["index"][0, 700:800] = -1
    s["index"][0, 800:900] = np.where(np.arange(100) % 2, 4, np.iinfo(np.int32).min)
    clean = {k: None if v is None else v.copy() for k, v in s.items()}
    hurt = [0, 150, 331, 1099]
    s["index"][0, 331], clean["index"][0, 331] = 1, 1
    s["x"][0, 513, 0], s["x"][0, 5, 150], s["x"][0, 0, 331], s["x"][0, 77, 1099] = np.nan, np.inf, -np.inf, np.nan
    s["index"][0, 1099], clean["index"][0, 1099] = 0, 0
    s["down"][3, 62, 513], s["up"][3, 519, 62] = np.inf, np.nan                # the last weights of adapter 3, which is the last
    s["down"][2, 0, 0] = np.nan
    got, want = (AdaptersCall(v, pads=(1, 1, 1)) for v in (s, clean))
    got.run()
    want.run()
    want.check(want.read())
    sound = ~np.isin(s["index"][0], (2, 3))
    sound[hurt] = False
    a, b = got.read(), want.read()
    assert np.array_equal(a[..., sound], b[..., sound])
    assert not np.isfinite(a[0][:, hurt]).any()
    none = (s["index"][0] < 0) | (s["index"][0] >= 4)
    assert none.sum() > 200 and np.array_equal(a[..., none], s["c"][..., none])


@pytest.mark.parametrize("kind", ["f16", "f32", "i8f32"])
def test_adapters_of_many_tokens_in_place(kind):
    rng = np.random.default_rng(19)
    s = adapters_case(rng, 530, 512, 1101, 64, 2, kind, index="runs")
    s["alpha"] = None
    call = AdaptersCall(s, pads=(3, 2, 2), inplace=True)
    call.run()
    call.check(call.read())


def test_many_tokens_keep_large_and_small_inner_values():
    rng = np.random.default_rng(20)
    s = adapters_case(rng, 520, 512, 1100, 64, 1, "f16")
    s["index"][:] = 0
    s["x"] *= np.float16(1500.0)
    s["down"] = (s["down"].astype(np.float32) * 60).astype(np.float16)
    s["up"] = (s["up"].astype(np.float32) * 1e-3).astype(np.float16)
    s["x"][0, :, ::3] = (s["x"][0, :, ::3].astype(np.float32) * 1e-9).astype(np.float16)      # tokens of very different sizes side by side
    s["x"][0, :, 7] = 0
    assert np.abs(s["down"][0].astype(np.float64) @ s["x"][0].astype(np.float64)).max() > 70000
    call = AdaptersCall(s)
    call.run()
    call.check(call.read())


@pytest.mark.parametrize("kind", ["f16", "f32", "i8f16"])
def test_adapters_where_no_token_has_one_and_where_the_index_names_none(kind):
    rng = np.random.default_rng(2)
    for N in (1, 40, 200):
        s = adapters_case(rng, 90, 100, N, 8, 3, kind)
        for index in (np.full((1, N), -1), np.full((1, N), 3), np.where(np.arange(N) % 3 == 0, np.iinfo(np.int32).min, np.iinfo(np.int32).max)[None], np.arange(N)[None] % 7 - 2):
            s["index"] = index.astype(np.int32)
            call = AdaptersCall(s, pads=(1, 1, 1))
            call.run()
            y = call.read()
            call.check(y)
            if kind != "i8f16":
                none = (index[0] < 0) | (index[0] >= 3)
                assert np.array_equal(y[..., none], s["c"][..., none])


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_adapters_in_place_and_without_factors(kind):
    rng = np.random.default_rng(6)
    for M, K, N in ((70, 130, 45), (257, 64, 300)):
        s = adapters_case(rng, M, K, N, 8, 3, kind, batch=2)
        s["alpha"] = None
        call = AdaptersCall(s, pads=(2, 4, 4), inplace=True)
        call.run()
        call.check(call.read())
    s = adapters_case(rng, 70, 130, 45, 8, 3, "i8f32", batch=2)
    s["row"] = None
    call = AdaptersCall(s, inplace=True)
    call.run()
    call.check(call.read())
    s["row"], s["col"] = np.ones(70, dtype=np.float32), None
    call = AdaptersCall(s)
    call.run()
    call.check(call.read())


@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("N", [40, 3, 300])
def test_a_token_is_computed_from_its_own_column_and_adapter_alone(kind, N):
    rng = np.random.default_rng(8)
    s = adapters_case(rng, 70, 130, N, 20, 4, kind)
    s["index"][0, :] = np.arange(N) % 5 - 1
    clean = {k: None if v is None else v.copy() for k, v in s.items()}
    s["x"][0, 5, 1], s["x"][0, 129, 2] = np.inf, np.nan          # the tokens of adapters 0 and 1
    s["down"][3, 19, 129] = np.nan                                # adapter 3
    s["up"][3, 69, 0] = np.inf
    s["alpha"][2] = 0.5
    clean["alpha"][2] = 0.5
    call = AdaptersCall(s)
    call.run()
    got = call.read()
    call = AdaptersCall(clean)
    call.run()
    want = call.read()
    touched = np.zeros(N, dtype=bool)
    touched[[1, 2]] = True
    touched |= s["index"][0] == 3
    assert np.array_equal(got[..., ~touched], want[..., ~touched])
    assert not np.isfinite(got[0, :, 1]).any() and not np.isfinite(got[0, :, 2]).any()


def test_adapters_keep_large_and_small_inner_values():
    """t beyond half's range and far below it: it is kept in binary32."""
    rng = np.random.default_rng(9)
    s = adapters_case(rng, 70, 200, 40, 8, 3, "f16")
    s["x"] *= np.float16(2000.0)
    s["down"] = (s["down"].astype(np.float32) * 40).astype(np.float16)
    s["up"] = (s["up"].astype(np.float32) * 1e-3).astype(np.float16)
    t = np.abs(s["down"][0].astype(np.float64) @ s["x"][0].astype(np.float64))
    assert t.max() > 70000
    call = AdaptersCall(s)
    call.run()
    call.check(call.read())
    s["x"] = (s["x"].astype(np.float32) * 1e-7).astype(np.float16)
    call = AdaptersCall(s)
    call.run()
    call.check(call.read())


# ---------------------------------------------------------------- together, streams, graphs, far offsets

def chain(N, seed, batch=1, K=256, M=320):
    """norm -> int8 product -> adapters with the product's scales; returns (launch, check)."""
    rng = np.random.default_rng(seed)
    x, r, g = norm_case(rng, K, N, np.float16, batch)
    csr = synth.int8_csr(M, K, 0.9, seed)
    plan = sp.inspect(csr.row_ptr, csr.col_idx, csr.vals, M, K, N, batch=batch)
    X, R, G = Wide(x.shape, N, np.float16, x), Wide(x.shape, N, np.float16, r), vector(g)
    H, Q = Wide(x.shape, N, np.float16), Wide(x.shape, N, np.int8)
    scale, C = torch.zeros((batch, N), device=DEV), torch.zeros((batch, M, N), dtype=torch.int32, device=DEV)
    s = adapters_case(rng, M, K, N, 8, 3, "i8f16", batch)
    a = AdaptersCall(s)
    D = torch.zeros((batch, M, N), device=DEV)
    d, dq = sp.RmsNorm(K, N, dtype=sp.F16, out_dtype=sp.I8, eps=1e-5, batch=batch), sp.Dequantize(M, N, batch=batch)
    nws = Scratch(d.workspace_bytes())

    def launch():
        st, v = stream(), a.v
        sp.rms_norm(d, X.at, R.at, at(G), H.at, Q.at, at(scale), *nws.args(), st)
        sp.spmm(plan, Q.at, C.data_ptr(), st)
        sp.dequantize(dq, C.data_ptr(), at(v["row"]), at(scale), D.data_ptr(), st)
        sp.adapters(a.d, Q.at, at(v["down"]), at(v["up"]), at(v["index"]), at(v["alpha"]), C.data_ptr(), at(v["row"]), at(scale), a.Y.at, a.ws.data_ptr(), a.need, st)

    def check():
        torch.cuda.synchronize()
        q, sc, c = Q.read(), scale.cpu().numpy(), C.cpu().numpy()
        plain.check_norm(q, sc, H.read(), x, r, g, 1e-5)
        for b in range(batch):
            assert np.array_equal(c[b].astype(np.float64), ref.spmm(M, K, N, csr.row_ptr, csr.col_idx, csr.vals, q[b])[0])
        plain.check_dequantize(D.cpu().numpy(), c, s["row"], sc)
        plain.check_adapters(a.Y.read(), q, s["down"], s["up"], s["index"], s["alpha"], c, s["row"], sc)

    def clear():
        for t in (H.t, Q.t, scale, C, D, a.Y.t):
            t.zero_()
        a.ws[:a.need] = 255
        nws.t.fill_(255)

    launch.keep = plan
    return launch, check, clear


@pytest.mark.parametrize("N,batch", [(1, 1), (24, 3), (128, 1), (517, 1)])
def test_an_int8_layer_with_adapters(N, batch):
    launch, check, _ = chain(N, 20 + N, batch)
    launch()
    check()


def test_layers_on_two_streams_at_once():
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    layers = [chain(200, 31), chain(70, 32)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (launch, _, _) in zip(streams, layers):
            with torch.cuda.stream(st):
                launch()
    torch.cuda.synchronize()
    for _, check, _ in layers:
        check()


def test_two_captured_layers_replayed_between_eager_work():
    layers = [chain(200, 41), chain(3, 42)]
    graphs = []
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for launch, _, _ in layers:
            launch()
    torch.cuda.synchronize()
    for launch, _, _ in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            launch()
        graphs.append(g)
    eager = chain(96, 43)
    for _ in range(4):
        for (_, check, clear), g in zip(layers, graphs):
            clear()
            eager[0]()
            g.replay()
            eager[0]()
            check()
            eager[1]()


def test_problems_whose_offsets_pass_32_bits():
    """Batches of wide pitch: the last problem begins beyond 2^32 elements; only the columns that are looked at are filled in."""
    K, N, batch, ld = 1021, 24, 5, 1_050_000
    rng = np.random.default_rng(5)
    x, r, g = norm_case(rng, K, N, np.float16, batch)
    X = torch.zeros((batch, K, ld), dtype=torch.float16, device=DEV)
    H, Q = torch.zeros_like(X), torch.zeros((batch, K, ld), dtype=torch.int8, device=DEV)
    X[..., :N], H[..., :N] = torch.from_numpy(x).to(DEV), torch.from_numpy(r).to(DEV)
    G, scale = vector(g), torch.zeros((batch, N), device=DEV)
    d = sp.RmsNorm(K, N, dtype=sp.F16, out_dtype=sp.I8, eps=1e-5, batch=batch, ldx=ld, ldh=ld, ldy=ld)
    nws = Scratch(d.workspace_bytes())
    sp.rms_norm(d, X.data_ptr(), H.data_ptr(), at(G), H.data_ptr(), Q.data_ptr(), at(scale), *nws.args(), stream())
    torch.cuda.synchronize()
    nws.check()
    q, sc = Q[..., :N].cpu().numpy(), scale.cpu().numpy()
    plain.check_norm(q, sc, H[..., :N].cpu().numpy(), x, r, g, 1e-5)
    del H
    M, ldc = 509, 1_050_000
    s = adapters_case(rng, M, K, N, 8, 3, "i8f16", batch)
    C, Y = torch.zeros((batch, M, ldc), dtype=torch.int32, device=DEV), torch.zeros((batch, M, ldc), dtype=torch.float16, device=DEV)
    C[..., :N] = torch.from_numpy(s["c"]).to(DEV)
    v = {k: torch.from_numpy(s[k]).to(DEV) for k in ("down", "up", "index", "alpha", "row")}
    a = sp.Adapters(M, K, N, 8, 3, dtype=sp.F16, x_dtype=sp.I8, batch=batch, ldx=ld, ldc=ldc, ldy=ldc)
    ws = torch.empty(a.workspace_bytes(), dtype=torch.uint8, device=DEV)
    sp.adapters(a, Q.data_ptr(), at(v["down"]), at(v["up"]), at(v["index"]), at(v["alpha"]), C.data_ptr(), at(v["row"]), at(scale), Y.data_ptr(), at(ws), ws.numel(), stream())
    torch.cuda.synchronize()
    plain.check_adapters(Y[..., :N].cpu().numpy(), q, s["down"], s["up"], s["index"], s["alpha"], s["c"], s["row"], sc)
    assert not Y[..., N:N + 64].any()
    sp.dequantize(sp.Dequantize(M, N, dtype=sp.F16, batch=batch, ldc=ldc, ldy=ldc), C.data_ptr(), at(v["row"]), at(scale), Y.data_ptr(), stream())
    torch.cuda.synchronize()
    plain.check_dequantize(Y[..., :N].cpu().numpy(), s["c"], s["row"], sc)


def test_an_adapter_beyond_4_gib_of_weights():
    count, rank, K, M, N = 70, 256, 131072, 40, 20
    down = torch.zeros((count, rank, K), dtype=torch.float16, device=DEV)      # 4.7 GB, the last adapter behind 2^32 bytes
    rng = np.random.default_rng(5)
    s = adapters_case(rng, M, K, N, rank, 1, "f16")
    down[count - 1] = torch.from_numpy(s["down"][0]).to(DEV)
    up = torch.zeros((count, M, rank), dtype=torch.float16, device=DEV)
    up[count - 1] = torch.from_numpy(s["up"][0]).to(DEV)
    index = np.where(np.arange(N) % 2, count - 1, 3).astype(np.int32)[None]
    X, C, I = torch.from_numpy(s["x"]).to(DEV), torch.from_numpy(s["c"]).to(DEV), torch.from_numpy(index).to(DEV)
    Y = torch.full_like(C, float("nan"))
    a = sp.Adapters(M, K, N, rank, count, dtype=sp.F16)
    ws = torch.empty(a.workspace_bytes(), dtype=torch.uint8, device=DEV)
    sp.adapters(a, at(X), at(down), at(up), at(I), 0, at(C), 0, 0, at(Y), at(ws), ws.numel(), stream())
    torch.cuda.synchronize()
    plain.check_adapters(Y.cpu().numpy(), s["x"], s["down"], s["up"], np.where(index == count - 1, 0, -1), None, s["c"], None, None)


# ---------------------------------------------------------------- infinities are those of the formula, whichever kernels a call takes

def column(s, n):
    """Token n of a call in 64 bits, product by product: its result and the sum of the terms' sizes, [M] each."""
    x, c = s["x"][0, :, n].astype(np.float64), s["c"][0, :, n].astype(np.float64)
    if s["x"].dtype == np.int8:
        x, c = x * float(s["col"][0, n]), c * s["row"].astype(np.float64) * float(s["col"][0, n])
    a = s["index"][0, n]
    if not 0 <= a < s["down"].shape[0]:
        return c, np.abs(c)
    down, up = s["down"][a].astype(np.float64), s["up"][a].astype(np.float64) * float(s["alpha"][a])
    with np.errstate(invalid="ignore"):
        return c + (up * (down * x).sum(axis=1)).sum(axis=1), np.abs(c) + (np.abs(up) * (np.abs(down * x)).sum(axis=1)).sum(axis=1)


def check_columns(y, s, tokens):
    K, rank = s["x"].shape[1], s["down"].shape[1]
    for n in tokens:
        want, size = column(s, n)
        got, known = y[0, :, n].astype(np.float64), np.isfinite(want)
        # (as in check_adapters: K and rank terms to a sum, factors and additions)
        bound = size[known] * (K + rank + 16) * plain.U + plain.store_bound(want[known], y.dtype)
        assert (np.abs(got[known] - want[known]) <= bound * 1.001).all(), n
        assert np.array_equal(got[~known], want[~known], equal_nan=True), (n, got[~known], want[~known])


# 3 and 40 tokens go one by one, 1100 in tiles on the matrix cores.
@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("N", [1, 3, 40, 1100])
@pytest.mark.parametrize("rank", [10, 20, 40])
def test_infinite_activations_beside_fewer_ranks_than_a_block(rank, N, kind):
    """Every t of the token is infinite; ranks that the adapter does not have are no terms."""
    rng = np.random.default_rng(rank + N)
    s = adapters_case(rng, 600, 512, N, rank, 2, kind)
    s["down"], s["up"] = np.abs(s["down"]) + s["down"].dtype.type(0.01), np.abs(s["up"]) + s["up"].dtype.type(0.01)
    s["index"][0, :] = np.arange(N) * 2 // N
    hurt = sorted({0, N // 2, N - 1})
    for i, n in enumerate(hurt):
        s["x"][0, 100 + 50 * i, n] = (np.inf, -np.inf, np.inf)[i]
    call = AdaptersCall(s)
    call.run()
    y = call.read()
    assert np.isinf(y[0][:, hurt]).all()
    check_columns(y, s, sorted({*hurt, *(n + 1 for n in hurt[:-1] if n + 1 < N)}))


def selecting(s, rng):
    """Makes t_j of adapter a the token's x in row 3 j + a, as it is."""
    s["down"][:] = 0
    for a in range(s["down"].shape[0]):
        for j in range(s["down"].shape[1]):
            s["down"][a, j, 3 * j + a] = 1


@pytest.mark.parametrize("kind", ["f16", "i8f16", "f32"])
@pytest.mark.parametrize("N", [1, 3, 40, 1100])
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_an_infinite_inner_value_beside_large_ones(rank, N, kind):
    """One t is infinite; the others, beyond half's range and of the other sign, are finite."""
    rng = np.random.default_rng(rank + N)
    s = adapters_case(rng, 600, 512, N, rank, 2, kind)
    selecting(s, rng)
    s["index"][0, :] = np.arange(N) * 2 // N
    w = s["down"].dtype.type
    s["down"][:, 0, :2], s["down"][0, 1, 3], s["down"][1, 1, 4] = 0, 60000, 60000
    s["down"][:, 0, 2] = np.inf
    s["x"][0, 2, :] = np.where(np.arange(N) % 2, 1, -1)
    s["x"][0, 3:5, :] = np.where(np.arange(N) % 2, 50, -50)
    if s["col"] is not None:
        s["col"][:] = 0.5
    s["up"] = (np.abs(s["up"]) * w(0.01) + w(0.001)) * np.where(np.arange(rank) == 0, 1, -1).astype(w)
    assert abs(column(s, 0)[1]).max() == np.inf
    call = AdaptersCall(s)
    call.run()
    y = call.read()
    assert np.isinf(y).all()
    check_columns(y, s, sorted({0, N // 3, N // 2, N - 1}))


@pytest.mark.parametrize("kind", ["f16", "i8f16", "f32", "i8f32"])
@pytest.mark.parametrize("N", [1, 3, 40, 1100])
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_infinite_weights_of_up(rank, N, kind):
    """Whatever t they meet: one that half holds, ones that it rounds up and down, one far under the token's largest, none."""
    rng = np.random.default_rng(rank + N)
    M = 600
    s = adapters_case(rng, M, 512, N, rank, 2, kind)
    selecting(s, rng)
    s["index"][0, :] = np.arange(N) * 2 // N
    s["alpha"][:] = 1.0
    special = [1.0, 0.3, -0.7, 0.0, 2.0 ** -24] if s["x"].dtype != np.int8 else [100, 33, -77, 0, 1]
    rows, j = [0, 17, 18, M - 1], rank - 2
    hurt = [n for n in (0, 1, 2, N // 2, N // 2 + 1, N // 2 + 2, N - 3, N - 2, N - 1) if 0 <= n < N]
    for i, n in enumerate(hurt):
        a = s["index"][0, n]
        s["x"][0, 3 * j + a, n] = special[(i + rank // 8 + N) % 5]
        if s["x"].dtype != np.int8 and i % 2:
            s["x"][0, a, n] = 60000.0          # the token's largest
    s["up"][:, :, 0] *= s["up"].dtype.type(1e-3)
    s["up"][:, rows[:3], j] = np.array([np.inf, -np.inf, np.inf])
    s["up"][:, rows[2], j + 1] = -np.inf
    s["up"][1, rows[3], j] = np.inf
    call = AdaptersCall(s)
    call.run()
    y = call.read()
    check_columns(y, s, sorted({*hurt, N // 3}))
    others = np.delete(np.arange(M), rows)
    plain.check_adapters(y[:, others], s["x"], s["down"], s["up"][:, others], s["index"], s["alpha"], s["c"][:, others], None if s["row"] is None else s["row"][others], s["col"])


@pytest.mark.parametrize("K,N", [(2, 4000), (8192, 256), (8192, 3)])
def test_norm_factor_is_rounded_once(K, N, way):
    """Columns of a one, whose result is the factor, and a number that makes the mean of the squares exact; eps is lost beside it."""
    x = np.zeros((1, K, N), dtype=np.float32)
    x[0, 0, :], x[0, K - 1, :] = 1, np.arange(1, N + 1) / 64
    y, _, _ = run_norm(way, x, None, None, np.float32, eps=1e-30)
    want = 1 / np.sqrt((1 + x[0, K - 1, :].astype(np.float64) ** 2) / K)
    # one rounding; what is behind it is of the order of its square
    assert (np.abs(y[0, 0, :] - want) <= want * plain.U * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("K", [90, 9000])
def test_norm_of_a_floating_column_whose_squares_overflow(K, way):
    x = np.full((1, K, 20), 1e-3, dtype=np.float32)
    x[0, 4, 2], x[0, 5, 3], x[0, 6, 3] = 1e25, np.inf, 1e25
    y, _, _ = run_norm(way, x, None, None, np.float32)
    sound = [n for n in range(20) if n not in (2, 3)]
    plain.check_norm(y[..., sound], None, None, x[..., sound], None, None, 1e-5)
    assert (y[0, :, 2] == 0).all() and np.isnan(y[0, 5, 3]) and (np.delete(y[0, :, 3], 5) == 0).all()
