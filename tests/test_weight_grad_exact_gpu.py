"""Weight gradients over many tokens: whole numbers, exact, and the same bits at every pitch."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2407_19644_amd as ubp                                      # noqa: E402
from layer_util import value_cells                                     # noqa: E402
from synthetic import select_blocks                                    # noqa: E402
from test_train_gpu import DEV, guards_intact, handle, stream, workspace   # noqa: E402

_T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# M, K, N, bh, bw, density: one range of tokens is N / 256 of them at least, and more where the layer has regions of its own.
# A range takes its exponents for 512 tokens at once: the first and the last two layers do so several times.
EXACT = [(24, 16, 300001, 4, 4, 0.5), (24, 16, 34000, 4, 4, 0.5), (64, 80, 34017, 8, 8, 0.4), (1100, 1000, 20011, 16, 16, 0.25),
         (2048, 1024, 4999, 16, 16, 0.3)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", EXACT, ids=lambda c: "-".join(map(str, c)))
def test_weight_grad_of_many_tokens_is_exact(case, dtype):
    """Whole numbers whose sums of magnitudes stay below 2^24: every sum is exact in fp32, in any order, so that no token may be
    missing.  X in 4 bits times a power of two per 32 tokens: a checkpoint holds it exactly, with exponents of all sizes.
    At every pitch and alignment, and from a checkpoint, the same."""
    M, K, N, bh, bw, d = case
    blocks = select_blocks(M, K, bh, bw, d, seed=M + K)
    rows, cols = (torch.from_numpy(a).cuda() for a in value_cells(blocks, bh, bw))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M + N)
    t, G32 = _T[dtype], (N + 31) // 32
    g = torch.randint(-1, 2, (M, N), generator=gen, device=DEV, dtype=torch.int32)
    x = torch.randint(-15, 16, (K, N), generator=gen, device=DEV, dtype=torch.int32)
    x = x << torch.randint(0, 4, (K, G32), generator=gen, device=DEV, dtype=torch.int32).repeat_interleave(32, 1)[:, :N]
    want = (g.double() @ x.double().t())[rows, cols]                        # (exact in 64 bits)
    assert float((g.abs().double() @ x.abs().double().t()).max()) < 2.0 ** 24
    p = handle(M, K, dtype, blocks, bh, bw)
    n = ubp.weight_grad_workspace(p, N)
    ws, wp = workspace(n)

    def place(a, kind, ld, off):
        buf = torch.full((a.shape[0] * ld + off + 64,), 113, dtype=kind, device=DEV)
        view = buf[off:off + a.shape[0] * ld].view(a.shape[0], ld)[:, :a.shape[1]]
        view.copy_(a)
        return view

    for pad_g, pad_x, off in ((0, 0, 0), (-N % 16, -N % 16 + 16, 0), (1, 3, 1), (5, 8, 3)):
        gv, xv = place(g, t, N + pad_g, off), place(x, t, N + pad_x, off)
        q, s = place(torch.zeros_like(x), torch.uint8, N + pad_x, off), place(torch.zeros((K, G32)), torch.uint8, G32 + off, off)
        back = torch.zeros((K, N), dtype=t, device=DEV)
        ubp.checkpoint_save(p, xv.data_ptr(), N + pad_x, N, q.data_ptr(), N + pad_x, s.data_ptr(), G32 + off, stream())
        ubp.checkpoint_load(p, q.data_ptr(), N + pad_x, s.data_ptr(), G32 + off, N, back.data_ptr(), N, stream())
        assert torch.equal(back, xv)
        for saved in (False, True):
            dv = torch.full((rows.numel(),), float("nan"), device=DEV)
            if saved:
                ubp.weight_grad_checkpoint(p, gv.data_ptr(), N + pad_g, q.data_ptr(), N + pad_x, s.data_ptr(), G32 + off, N, dv.data_ptr(),
                                           False, wp, n, stream())
            else:
                ubp.weight_grad(p, gv.data_ptr(), N + pad_g, xv.data_ptr(), N + pad_x, N, dv.data_ptr(), False, wp, n, stream())
            torch.cuda.synchronize()
            assert guards_intact(ws, n)
            wrong = int((dv.double() != want).sum())
            assert wrong == 0, (pad_g, pad_x, off, saved, wrong)
    p.free()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", [(256, 600, 4096, 4, 4, 0.25), (130, 600, 1001, 16, 16, 0.15), (24, 16, 34000, 4, 4, 0.5)], ids=lambda c: "-".join(map(str, c)))
def test_weight_grad_has_the_same_bits_at_every_pitch(case, dtype):
    """One kernel, ranges and order for all pitches and alignments, and for a checkpoint and the values that it gives."""
    M, K, N, bh, bw, d = case
    blocks = select_blocks(M, K, bh, bw, d, seed=M + K)
    p = handle(M, K, dtype, blocks, bh, bw)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M + N)
    t, G32 = _T[dtype], (N + 31) // 32
    g, x = (torch.randn(r, N, generator=gen, device=DEV).to(t) for r in (M, K))
    q, s = torch.zeros((K, N), dtype=torch.uint8, device=DEV), torch.zeros((K, G32), dtype=torch.uint8, device=DEV)
    ubp.checkpoint_save(p, x.data_ptr(), N, N, q.data_ptr(), N, s.data_ptr(), G32, stream())
    ubp.checkpoint_load(p, q.data_ptr(), N, s.data_ptr(), G32, N, x.data_ptr(), N, stream())
    n = ubp.weight_grad_workspace(p, N)
    ws, wp = workspace(n)

    def place(a, ld, off):
        buf = torch.full((a.shape[0] * ld + off + 64,), 113, dtype=a.dtype, device=DEV)
        view = buf[off:off + a.shape[0] * ld].view(a.shape[0], ld)[:, :a.shape[1]]
        view.copy_(a)
        return view

    out = []
    for ldg, ldx, off in ((N, N, 0), (N + 3, N + 5, 7), (-(-N // 16) * 16, -(-N // 16) * 16 + 16, 0)):
        gv, xv, qv = place(g, ldg, off), place(x, ldx, off), place(q, ldx, off)
        for saved in (False, True):
            dv = torch.full((blocks.shape[0] * bh * bw,), float("nan"), device=DEV)
            if saved:
                ubp.weight_grad_checkpoint(p, gv.data_ptr(), ldg, qv.data_ptr(), ldx, s.data_ptr(), G32, N, dv.data_ptr(), False, wp, n, stream())
            else:
                ubp.weight_grad(p, gv.data_ptr(), ldg, xv.data_ptr(), ldx, N, dv.data_ptr(), False, wp, n, stream())
            torch.cuda.synchronize()
            out.append(dv)
    assert torch.isfinite(out[0]).all()
    for dv in out[1:]:
        assert torch.equal(dv, out[0])
    p.free()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [31, 200, 20001])
def test_a_checkpoint_keeps_not_finite_values_in_their_columns(N, dtype):
    """An Inf or NaN in X is a NaN in the checkpoint, and in the weights' gradients of its own column alone."""
    M, K = 64, 96
    blocks = select_blocks(M, K, 8, 8, 0.4, seed=5)
    cols = torch.from_numpy(value_cells(blocks, 8, 8)[1]).cuda()
    p = handle(M, K, dtype, blocks, 8, 8)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    t, G32 = _T[dtype], (N + 31) // 32
    g, x = (torch.randn(r, N, generator=gen, device=DEV).to(t) for r in (M, K))
    x[11, N - 1], x[40, 0], x[95, N // 2] = float("nan"), float("inf"), float("-inf")
    q, s = torch.zeros((K, N), dtype=torch.uint8, device=DEV), torch.zeros((K, G32), dtype=torch.uint8, device=DEV)
    n = ubp.weight_grad_workspace(p, N)
    ws, wp = workspace(n)
    ubp.checkpoint_save(p, x.data_ptr(), N, N, q.data_ptr(), N, s.data_ptr(), G32, stream())
    out = []
    for clean in (False, True):
        if clean:                                                          # (the group's other values do not depend on them)
            q[11, N - 1] = q[40, 0] = q[95, N // 2] = 0
        dv = torch.full((cols.numel(),), 3.0, device=DEV)
        ubp.weight_grad_checkpoint(p, g.data_ptr(), N, q.data_ptr(), N, s.data_ptr(), G32, N, dv.data_ptr(), False, wp, n, stream())
        torch.cuda.synchronize()
        out.append(dv)
    touched = (cols == 11) | (cols == 40) | (cols == 95)
    assert touched.any() and torch.isnan(out[0][touched]).all()
    assert torch.equal(out[0][~touched], out[1][~touched]) and torch.isfinite(out[1]).all()
    p.free()


def test_calls_of_two_launches_are_captured_and_replayed():
    """Sums over many tokens take a second launch: the bias's gradient of few rows, and the weights', added to what is there."""
    M, K, N, dtype = 40, 64, 20001, "bf16"
    blocks = select_blocks(M, K, 4, 4, 0.4, seed=5)
    nv, G32 = blocks.shape[0] * 16, (N + 31) // 32
    p = handle(M, K, dtype, blocks, 4, 4)
    t = _T[dtype]
    new = lambda *shape, d=t: torch.zeros(shape, dtype=d, device=DEV)      # noqa: E731
    X, dY, Z, G = new(K, N), new(M, N), new(M, N), new(M, N)
    Q, S = new(K, N, d=torch.uint8), new(K, G32, d=torch.uint8)
    n, m = ubp.weight_grad_workspace(p, N), ubp.linear_grad_workspace(p, N)
    assert n > 0 and m > 0
    wn, wm = new(n, d=torch.uint8), new(m, d=torch.uint8)
    ubp.weight_grad_prepare(p)

    def step(db, dv):
        st = stream()
        ubp.checkpoint_save(p, X.data_ptr(), N, N, Q.data_ptr(), N, S.data_ptr(), G32, st)
        ubp.linear_grad(p, dY.data_ptr(), N, Z.data_ptr(), N, N, G.data_ptr(), N, db.data_ptr(), "gelu", workspace_ptr=wm.data_ptr(),
                        workspace_bytes=m, stream=st)
        ubp.weight_grad_checkpoint(p, G.data_ptr(), N, Q.data_ptr(), N, S.data_ptr(), G32, N, dv.data_ptr(), False, wn.data_ptr(), n, st)
        ubp.weight_grad(p, G.data_ptr(), N, X.data_ptr(), N, N, dv.data_ptr(), True, wn.data_ptr(), n, st)

    db, dv = new(M, d=torch.float32), new(nv, d=torch.float32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(db, dv)
    for seed in range(3):
        torch.manual_seed(seed)
        for a in (X, dY, Z):
            a.copy_(torch.randn_like(a))
        wn.fill_(0xA5)
        wm.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        eager = new(M, d=torch.float32), new(nv, d=torch.float32)
        step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(db, eager[0]) and torch.equal(dv, eager[1]) and dv.abs().max() > 0 and torch.isfinite(dv).all()
    p.free()
