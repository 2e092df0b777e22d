"""The bias's gradient of rows of any length."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2407_19644_amd as ubp                                      # noqa: E402
from layer_util import act_slope                                       # noqa: E402
from test_train_gpu import DEV, guards_intact, handle, stream, workspace   # noqa: E402

_T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("M,N,dtype", [(1024, 1 << 18, "bf16"), (1031, (1 << 17) + 5, "f32"), (2, (1 << 24) + 5, "bf16"), (1, (1 << 23) + 3, "f32"),
                                       (1023, 70001, "f16")])
def test_bias_gradient_of_long_rows(M, N, dtype):
    """Rows of one value each: what a long fp32 sum drops is dropped to one side at every addition, so that a sum of n terms one
    after the other is off by up to n 2^-25 of itself."""
    t = _T[dtype]
    z = torch.linspace(0.3, 2.9, M, device=DEV).to(t)
    d = torch.linspace(1.9, 0.7, M, device=DEV).to(t)
    Z, G = z[:, None].expand(M, N).contiguous(), d[:, None].expand(M, N).contiguous()
    db = torch.full((M,), float("nan"), device=DEV)
    p = handle(M, 8, dtype)
    n = ubp.linear_grad_workspace(p, N)
    ws, wp = workspace(n)
    ubp.linear_grad(p, G.data_ptr(), N, Z.data_ptr(), N, N, G.data_ptr(), N, db.data_ptr(), "silu", workspace_ptr=wp, workspace_bytes=n,
                    stream=stream())
    torch.cuda.synchronize()
    assert guards_intact(ws, n)
    z64, d64 = z.double().cpu().numpy(), d.double().cpu().numpy()
    want = N * d64 * act_slope("silu", z64)
    # a value of G: the slope within 4e-7 and the roundings of z and of the product.  The sum: 8 neighbours, trees over 64 lanes and 4
    # wavefronts, 18 roundings; where more is added one after the other, what an addition drops is kept (24 with that)
    tol = N * np.abs(d64) * (4e-7 + 2.0 ** -23 * (1 + np.abs(z64))) + 24 * 2.0 ** -24 * np.abs(want)
    err = np.abs(db.cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())
    p.free()


@pytest.mark.parametrize("bad,want", [((np.inf,), np.inf), ((-np.inf,), -np.inf), ((np.inf, -np.inf), np.nan), ((np.nan,), np.nan)])
@pytest.mark.parametrize("M,N", [(3, 300), (2, 20001), (1024, 9000)])
def test_bias_gradient_of_values_that_are_not_finite(M, N, bad, want):
    p = handle(M, 8, "f32")
    dY = torch.ones((M, N), device=DEV)
    for k, v in enumerate(bad):
        dY[1, 7 + (N // 2) * k] = v
    G, db = torch.empty_like(dY), torch.empty(M, device=DEV)
    n = ubp.linear_grad_workspace(p, N)
    ws, wp = workspace(n)
    ubp.linear_grad(p, dY.data_ptr(), N, None, 0, N, G.data_ptr(), N, db.data_ptr(), None, workspace_ptr=wp, workspace_bytes=n, stream=stream())
    torch.cuda.synchronize()
    db = db.cpu().numpy()
    assert np.array_equal(db[1], np.float32(want), equal_nan=True)
    assert (np.delete(db, 1) == N).all()
    p.free()
