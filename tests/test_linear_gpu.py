"""ubp_linear: bias, every activation and the residual through every kernel, against float64."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2407_19644_amd as ubp                                      # noqa: E402
from gpu_util import _TORCH, from_device, to_device                    # noqa: E402
from layer_util import act, half_step, layer                           # noqa: E402
from synthetic import decode_f64, encode, make_activations             # noqa: E402

ACTS = (None, "relu", "clamp", "gelu", "gelu_tanh", "silu")


def run_linear(p, X, dtype, y_dtype, bias, activation, lo=0.0, hi=0.0, R=None, ldr=None, r_off=0, ldy=None, plan=None):
    """Y as float64; R (encoded M x N) lies at column r_off of rows of ldr elements whose other elements are NaN."""
    M = p.info(0)
    K, N = X.shape
    ldx = N if plan is None or plan.kernel != 6 else (N + 7) // 8 * 8     # (kernel 6 takes aligned rows)
    Xd = torch.zeros((K, ldx), dtype=_TORCH[dtype], device="cuda")
    Xd[:, :N] = to_device(X, dtype)
    ldy = max(ldy or N, ldx) if ldx == N else ldx + 24
    Yd = torch.full((M, ldy), float("nan"), dtype=_TORCH[y_dtype], device="cuda")
    bd = None if bias is None else torch.from_numpy(bias).cuda()
    rp, ldr = None, ldr or N
    if R is not None:
        buf = torch.full((M, ldr + r_off), float("nan"), dtype=_TORCH[y_dtype], device="cuda")
        flat = buf.view(-1)[r_off:r_off + M * ldr].view(M, ldr)
        flat[:, :N] = to_device(R, y_dtype)
        rp = flat.data_ptr()
    ubp.linear(p, Xd.data_ptr(), ldx, N, Yd.data_ptr(), ldy, y_dtype, None if bd is None else bd.data_ptr(), activation, lo, hi, rp,
               ldr, torch.cuda.current_stream().cuda_stream, plan)
    torch.cuda.synchronize()
    assert p.device_error() == 0
    Y = from_device(Yd, y_dtype)
    assert np.isnan(Y[:, N:]).all(), "wrote beyond column N"
    return Y[:, :N]


def bound(Wd, Xd, want, z, R, y_dtype):
    """Largest distance of a right result: the sum of n products in fp32 (n 2^-24 of the sum of magnitudes, twice that where
    matrix instructions add in steps of their own), the activation's slope (below 1.13) and its own error (v times a
    distribution function that is within 4e-7), an addition, and the rounding to Y's type."""
    n = (Wd != 0).sum(1, keepdims=True) + 2
    dz = 2 * n * 2.0 ** -24 * (np.abs(Wd) @ np.abs(Xd)) + np.abs(z) * 2.0 ** -23
    before = 1.13 * dz + 4e-7 * np.abs(z) + 2.0 ** -24 * (np.abs(want) + (0 if R is None else np.abs(R)))
    return (before + half_step(np.abs(want) + before, y_dtype)) * 1.01 + 1e-37


CASES = [  # kernel, (M, K, N, bh, bw, density), dtype
    (1, (70, 45, 67, 3, 1, 0.4), "f32"), (1, (64, 64, 196, 4, 4, 0.5), "f32"), (1, (40, 1400, 132, 4, 4, 0.2), "f32"),
    (1, (96, 300, 256, 4, 4, 0.25), "f16"), (1, (33, 40, 35, 5, 3, 0.3), "bf16"),
    (2, (130, 600, 1000, 16, 16, 0.15), "bf16"), (2, (33, 40, 129, 5, 3, 0.3), "f16"),
    (4, (200, 256, 328, 8, 8, 0.2), "f16"), (4, (50, 100, 72, 4, 4, 0.3), "bf16"), (5, (160, 1024, 264, 4, 4, 0.25), "bf16"),
    (6, (300, 2500, 192, 16, 32, 0.1), "bf16"), (6, (130, 600, 1000, 16, 16, 0.15), "f16"), (6, (130, 600, 131, 16, 16, 0.15), "bf16"),
    (7, (160, 320, 520, 4, 4, 0.45), "f16"), (8, (130, 600, 333, 16, 16, 0.15), "f16"), (8, (160, 1024, 264, 4, 4, 0.25), "bf16"),
    (8, (47, 90, 1, 4, 4, 0.2), "bf16"), (9, (160, 1024, 263, 4, 4, 0.25), "bf16"), (9, (100, 200, 201, 8, 8, 0.2), "f16"),
    (0, (256, 2048, 1, 16, 16, 0.1), "bf16"), (0, (256, 2048, 128, 16, 16, 0.1), "bf16"), (0, (64, 64, 3, 4, 4, 0.5), "f32"),
    (0, (40, 50, 33, 4, 4, 0.0), "f16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "k%d-%s-%s" % (c[0], "x".join(map(str, c[1])), c[2]))
def test_linear(case):
    kernel, (M, K, N, bh, bw, d), dtype = case
    blocks, W, Wd = layer(M, K, bh, bw, d, dtype, seed=5 * M + K)
    X = make_activations(K, N, M + N, dtype, "normal")
    X64 = decode_f64(X, dtype)
    rng = np.random.default_rng(M + N)
    bias = rng.standard_normal(M).astype(np.float32)
    p = ubp.pack(W, dtype, bh, bw, blocks, device=torch.cuda.current_device())
    plan = ubp.Plan(kernel=kernel) if kernel else None
    lo, hi = -0.5, 0.75
    for y_dtype in sorted({dtype, "f32"}):
        R = encode((2 * rng.standard_normal((M, N))).astype(np.float32), y_dtype)
        R64 = decode_f64(R, y_dtype)
        for i, a in enumerate(ACTS):
            for with_bias, with_r in ((True, True), (False, True), (True, False)):
                if (with_bias, with_r) == (False, True) and a not in (None, "silu"):
                    continue
                z = Wd @ X64 + (bias.astype(np.float64)[:, None] if with_bias else 0.0)
                want = act(a, z, lo, hi) + (R64 if with_r else 0.0)
                # the residual's rows at another pitch and alignment for every activation
                ldr, off = (N + (0, 3, 8, 1, 16, 24)[i], (0, 1, 8, 0, 3, 0)[i]) if with_r else (N, 0)
                Y = run_linear(p, X, dtype, y_dtype, bias if with_bias else None, a, lo, hi, R if with_r else None, ldr, off,
                               ldy=N + (24 if i == 2 else 0), plan=plan)
                tol = bound(Wd, X64, want, z, R64 if with_r else None, y_dtype)
                assert np.isfinite(Y).all()
                assert (np.abs(Y - want) <= tol).all(), (a, with_bias, with_r, y_dtype, float((np.abs(Y - want) / tol).max()))
    p.free()


def test_linear_without_the_new_parts_is_the_fused_product():
    M, K, N = 130, 600, 264
    blocks, W, _ = layer(M, K, 16, 16, 0.15, "bf16", 9)
    X = make_activations(K, N, 3, "bf16", "normal")
    p = ubp.pack(W, "bf16", 16, 16, blocks, device=torch.cuda.current_device())
    bias = np.linspace(-1, 1, M).astype(np.float32)
    Xd, bd = to_device(X, "bf16"), torch.from_numpy(bias).cuda()
    for a in (None, "relu"):
        out = [torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        st = torch.cuda.current_stream().cuda_stream
        ubp.spmm_fused(p, Xd.data_ptr(), N, N, out[0].data_ptr(), N, "bf16", bd.data_ptr(), a, stream=st)
        ubp.linear(p, Xd.data_ptr(), N, N, out[1].data_ptr(), N, "bf16", bd.data_ptr(), a, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1])
    p.free()


def test_activations_over_their_range():
    """Every binade of v, both signs, far tails: one weight of 1 per row, so that v is X itself."""
    v = np.concatenate([[0.0], np.logspace(-30, 30, 2000), np.linspace(0, 20, 3001)])
    v = np.concatenate([v, -v]).astype(np.float32)
    N = v.size
    W = np.eye(4, dtype=np.float32)
    p = ubp.pack(W, "f32", 1, 1, np.asarray([[i, i] for i in range(4)], np.int32), device=torch.cuda.current_device())
    X = np.tile(v, (4, 1))
    for a in ("gelu", "gelu_tanh", "silu"):
        Y = run_linear(p, X, "f32", "f32", None, a)
        z = X.astype(np.float64)
        with np.errstate(over="ignore"):
            want = act(a, z)
        # v (F(v) + 4e-7), and a tail that is right to itself: exp's argument, up to z^2 / 2 or 100, rounds by 2^-24 of itself
        tail = np.abs(want) * (1e-6 + 2.0 ** -22 * np.minimum(z * z / 2 + np.abs(z), 120.0))
        tol = np.minimum(4e-7 * np.abs(z), tail) + 1e-36
        assert (np.abs(Y - want) <= tol).all(), (a, float((np.abs(Y - want) / tol).max()), float(z[0, (np.abs(Y - want) / tol)[0].argmax()]))
    p.free()


def test_not_finite_values():
    W = np.eye(3, dtype=np.float32)
    p = ubp.pack(W, "f32", 1, 1, np.asarray([[i, i] for i in range(3)], np.int32), device=torch.cuda.current_device())
    X = np.zeros((3, 4), np.float32)
    X[0] = [np.inf, -np.inf, np.nan, 3e38]
    R = np.ones((3, 4), np.float32)
    R[1, 1], R[2, 2] = np.nan, np.inf
    for a in ("gelu", "gelu_tanh", "silu"):
        Y = run_linear(p, X, "f32", "f32", None, a, R=R)
        assert np.isposinf(Y[0, 0]) and np.isnan(Y[0, 1]) and np.isnan(Y[0, 2]) and Y[0, 3] == np.float32(3e38)
        assert np.isnan(Y[1, 1]) and np.isposinf(Y[2, 2])
        rest = np.ones((3, 4), bool)
        rest[0], rest[1, 1], rest[2, 2] = False, False, False
        assert (Y[rest] == 1.0).all()
    Y = run_linear(p, X, "f32", "f32", None, "relu", R=R)
    assert Y[0, 2] == 1.0                                                # (a NaN becomes the lower bound)
    p.free()


def test_captured_linear_replays():
    M, K, N = 96, 200, 40
    blocks, W, Wd = layer(M, K, 8, 8, 0.2, "bf16", 4)
    p = ubp.pack(W, "bf16", 8, 8, blocks, device=torch.cuda.current_device())
    X = to_device(make_activations(K, N, 1, "bf16", "normal"), "bf16")
    R = to_device(make_activations(M, N, 2, "bf16", "normal"), "bf16")
    Y = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    b = torch.linspace(-1, 1, M, device="cuda")

    def call(out):
        ubp.linear(p, X.data_ptr(), N, N, out.data_ptr(), N, "bf16", b.data_ptr(), "silu", residual_ptr=R.data_ptr(), ldr=N,
                   stream=torch.cuda.current_stream().cuda_stream)

    ubp.spmm_prepare(p, X.data_ptr(), N, N, Y.data_ptr(), N, "bf16")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(Y)
    for i in range(3):
        X.copy_(to_device(make_activations(K, N, 10 + i, "bf16", "normal"), "bf16"))
        Y.zero_()
        g.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(Y)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, Y)
    p.free()


def test_linear_refusals():
    M, K, N = 64, 64, 40
    blocks, W, _ = layer(M, K, 4, 4, 0.3, "f16", 2)
    p = ubp.pack(W, "f16", 4, 4, blocks, device=torch.cuda.current_device())
    X = torch.zeros((K, N), dtype=torch.float16, device="cuda")
    both = torch.full((M, 2 * N + 8), 7.0, dtype=torch.float16, device="cuda")
    Y = both[:, :N]

    def call(code, **kw):
        a = dict(X=X.data_ptr(), ldx=N, N=N, Y=Y.data_ptr(), ldy=both.shape[1], y="f16")
        extra = {k: kw.pop(k) for k in list(kw) if k not in a}
        a.update(kw)
        if code is None:
            ubp.linear(p, a["X"], a["ldx"], a["N"], a["Y"], a["ldy"], a["y"], **extra)
            torch.cuda.synchronize()
            return
        before = both.clone()
        with pytest.raises(ubp.UBPError) as e:
            ubp.linear(p, a["X"], a["ldx"], a["N"], a["Y"], a["ldy"], a["y"], **extra)
        torch.cuda.synchronize()
        assert e.value.code == code and torch.equal(before, both)

    ld = both.shape[1]
    call(1, residual_ptr=Y.data_ptr(), ldr=ld)                            # in place
    call(1, residual_ptr=Y.data_ptr() + 2, ldr=ld)                        # a column further
    call(1, residual_ptr=Y.data_ptr() + 2 * (N - 1), ldr=ld)
    call(1, residual_ptr=Y.data_ptr() + 2 * (ld - N + 1), ldr=ld)         # reaches into the next row of Y
    call(1, residual_ptr=Y.data_ptr() + 2 * N, ldr=ld + 8)                # another pitch in the same rows
    call(1, residual_ptr=X.data_ptr(), ldr=N - 1)
    call(1, activation="clamp", lo=1.0, hi=-1.0)
    call(1, activation="clamp", lo=float("nan"), hi=1.0)
    call(1, y="bf16", activation="silu")
    call(4, activation="silu", plan=ubp.Plan(kernel=3))
    call(4, activation="silu", plan=ubp.Plan(kernel=7, sub_stripes=3))
    with pytest.raises(KeyError):
        call(1, activation="swish")
    call(None, residual_ptr=both[:, N:].data_ptr(), ldr=ld)               # beside Y in the same rows
    assert (both[:, :N] == 7.0).all() and (both[:, N:] == 7.0).all()
    call(None, residual_ptr=both[:, N + 8:].data_ptr(), ldr=ld, activation="silu")
    call(None, N=0, residual_ptr=Y.data_ptr(), ldr=ld)                    # nothing to do
    p.free()


def test_linear_on_a_host_only_handle():
    blocks, W, _ = layer(16, 16, 4, 4, 0.3, "f16", 2)
    p = ubp.pack(W, "f16", 4, 4, blocks)
    with pytest.raises(ubp.UBPError) as e:
        ubp.linear(p, 16, 8, 8, 1024, 8, "f16", activation="silu")
    assert e.value.code == 1
