"""A NaN without an activation stays one, through every kernel, and on into the gradients."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2407_19644_amd as ubp                                      # noqa: E402
from gpu_util import _TORCH, from_device, to_device                    # noqa: E402
from layer_util import layer                                           # noqa: E402
from synthetic import decode_f64, encode, make_activations             # noqa: E402
from test_linear_gpu import CASES, bound, run_linear                   # noqa: E402
from test_parity_gpu import FUSED_CASES                                # noqa: E402

name = lambda c: "k%d-%s-%s" % (c[0], "x".join(map(str, c[1])), c[2])   # noqa: E731


def inputs(case):
    """A layer with a token of NaN, and a bias with a NaN, an Inf of either sign; (what is not finite is left out of X64)."""
    kernel, (M, K, N, bh, bw, d), dtype = case
    blocks, W, Wd = layer(M, K, bh, bw, d, dtype, seed=5 * M + K)
    X = make_activations(K, N, M + N, dtype, "normal")
    token = N // 2
    X[:, token] = 0x7fc0 if dtype == "bf16" else np.nan
    X64 = decode_f64(X, dtype)
    assert np.isnan(X64[:, token]).all()
    X64[:, token] = 0.0
    bias = np.random.default_rng(M + N).standard_normal(M).astype(np.float32)
    bias[[0, M // 2, M - 1]] = np.nan, -np.inf, np.inf
    p = ubp.pack(W, dtype, bh, bw, blocks, device=torch.cuda.current_device())
    return p, Wd, X, X64, token, bias


def compare(Y, p, Wd, X64, token, bias, R64, activation, y_dtype, lo, hi):
    M, N = Y.shape
    b = np.zeros(M) if bias is None else bias.astype(np.float64)
    finite = np.isfinite(b)
    r = np.zeros((M, N)) if R64 is None else R64
    rest = np.arange(N) != token
    f = {None: lambda v: v, "relu": lambda v: np.fmax(v, 0.0), "clamp": lambda v: np.fmin(np.fmax(v, lo), hi)}[activation]
    z = Wd @ X64 + np.where(finite, b, 0.0)[:, None]
    want = f(z) + r
    tol = bound(Wd, X64, want, z, R64, y_dtype)
    ok = finite[:, None] & rest[None, :]
    assert (np.abs(Y - want)[ok] <= tol[ok]).all()
    for i in np.flatnonzero(~finite):
        v = f(b[i])
        if np.isfinite(v):
            assert (np.abs(Y[i, rest] - (v + r[i, rest])) <= tol[i, rest] + 2.0 ** -8 * (abs(v) + np.abs(r[i, rest]))).all()
        else:
            assert np.array_equal(Y[i, rest], np.full(N - 1, v), equal_nan=True), (i, v)
    # the token of NaN: every row that keeps weights
    rows = (Wd != 0).any(1)
    if activation is None:
        assert np.isnan(Y[rows, token]).all()
    else:
        assert (np.abs(Y[rows, token] - (f(np.nan) + r[rows, token])) <= 2.0 ** -7 * (abs(lo) + np.abs(r[rows, token]))).all()


@pytest.mark.parametrize("case", CASES, ids=name)
def test_linear(case):
    p, Wd, X, X64, token, bias = inputs(case)
    (M, N), dtype = (Wd.shape[0], X.shape[1]), case[2]
    plan = ubp.Plan(kernel=case[0]) if case[0] else None
    lo, hi = -0.5, 0.75
    for y_dtype in sorted({dtype, "f32"}):
        R = encode((2 * np.random.default_rng(M).standard_normal((M, N))).astype(np.float32), y_dtype)
        R64 = decode_f64(R, y_dtype)
        for activation in (None, "relu", "clamp"):
            for with_bias, with_r in ((True, True), (False, True), (True, False)):
                Y = run_linear(p, X, dtype, y_dtype, bias if with_bias else None, activation, lo, hi, R if with_r else None, plan=plan)
                compare(Y, p, Wd, X64, token, bias if with_bias else None, R64 if with_r else None, activation, y_dtype, lo, hi)
    p.free()


@pytest.mark.parametrize("case", FUSED_CASES, ids=name)
def test_fused_product(case):
    p, Wd, X, X64, token, bias = inputs(case)
    (M, N), dtype = (Wd.shape[0], X.shape[1]), case[2]
    plan = ubp.Plan(kernel=case[0]) if case[0] else None
    lo, hi = -0.5, 0.75
    x, b = to_device(X, dtype), torch.from_numpy(bias).cuda()
    for y_dtype in sorted({dtype, "f32"}):
        for activation in (None, "relu", "clamp"):
            y = torch.full((M, N), 7.0, dtype=_TORCH[y_dtype], device="cuda")
            ubp.spmm_fused(p, x.data_ptr(), N, N, y.data_ptr(), N, y_dtype, b.data_ptr(), activation, lo, hi,
                           torch.cuda.current_stream().cuda_stream, plan)
            torch.cuda.synchronize()
            assert p.device_error() == 0
            compare(from_device(y, y_dtype), p, Wd, X64, token, bias, None, activation, y_dtype, lo, hi)
    p.free()


@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_nan_reaches_the_gradients(dtype, activation):
    """X -> Z = W X + b -> G, db -> dW: a token of NaN is one in G, and so are db and dW of the rows that keep weights."""
    case = (0, (96, 200, 300, 8, 4, 0.25), dtype)
    p, Wd, X, X64, token, _ = inputs(case)
    M, N = Wd.shape[0], X.shape[1]
    rows = (Wd != 0).any(1)
    bias = torch.linspace(-1, 1, M, device="cuda")
    x, dy = to_device(X, dtype), to_device(make_activations(M, N, 5, dtype, "normal"), dtype)
    z, g = torch.zeros_like(dy), torch.zeros_like(dy)
    db = torch.zeros(M, device="cuda")
    dv = torch.zeros(M * N, device="cuda")
    n = ubp.weight_grad_workspace(p, N)
    ws = torch.zeros(n + 16, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    ubp.spmm_fused(p, x.data_ptr(), N, N, z.data_ptr(), N, dtype, bias.data_ptr(), stream=st)
    ubp.linear_grad(p, dy.data_ptr(), N, z.data_ptr(), N, N, g.data_ptr(), N, db.data_ptr(), activation, stream=st)
    ubp.weight_grad(p, g.data_ptr(), N, x.data_ptr(), N, N, dv.data_ptr(), False, ws.data_ptr(), n, st)
    torch.cuda.synchronize()
    G = from_device(g, dtype)
    rest = np.arange(N) != token
    assert np.isfinite(G[:, rest]).all() and np.isnan(G[rows, token]).all()
    assert np.isnan(db.cpu().numpy()[rows]).all()
    kept = p.indices.size * 32                                             # values of a block of 8 x 4
    assert torch.isnan(dv[:kept]).all() and (dv[kept:] == 0).all()
    p.free()
