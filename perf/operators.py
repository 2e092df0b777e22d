"""Operators of a pruned linear layer's training step and of its serving form, and how they are timed.

linear       Y = act(W X + b) + R with block-pruned W (act: relu, gelu, gelu_tanh, silu or none).
linear_grad  G = dY * act'(Z) for the pre-activations Z, and db = the sums of G's rows.
checkpoint   X to 8 bits (e4m3, a power of two per 32 neighbouring tokens of a row) and back to its type.
weight_grad  dW at the kept weights alone, sums over the tokens of G and X, X in its type or as a checkpoint.

Matrices have a feature per row and a token per column.  The order of weight_grad's output is the packed handle's: blocks by
(start row, column), in a block columns first, the weight of row i in slot i mod bh.
"""
import math

import numpy as np
import torch

own = False

_T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _case(name, op, M, K, N, dtype, block=(4, 4), density=0.25, act="none", bias=False, res=False, ckpt=False):
    return {"name": name, "op": op, "M": M, "K": K, "N": N, "dtype": dtype, "bh": block[0], "bw": block[1],
            "density": density, "act": act, "bias": bias, "res": res, "ckpt": ckpt}


def listed():
    return [
        # one token through a pruned projection: what serving does for every layer and token; latency
        _case("linear, 1 token, 4096 x 4096", "linear", 4096, 4096, 1, "bf16", (16, 16), 0.10, "silu", True, True),
        # a small layer with small blocks and an ordinary number of tokens
        _case("linear, 1568 tokens, 960 x 160", "linear", 960, 160, 1568, "f16", (4, 4), 0.30, "gelu", True, True),
        # the largest layer, a batch of training or prefill
        _case("linear, 8192 tokens, 4096 x 4096", "linear", 4096, 4096, 8192, "bf16", (16, 16), 0.10, "silu", True, True),
        # backward of the small layer's epilogue
        _case("linear_grad, 1568 tokens, 960 rows", "linear_grad", 960, 160, 1568, "f16", (4, 4), 0.30, "gelu", True),
        # backward of the largest layer's epilogue
        _case("linear_grad, 8192 tokens, 4096 rows", "linear_grad", 4096, 4096, 8192, "bf16", (16, 16), 0.10, "silu", True),
        # inputs of the small layer, kept in 8 bits
        _case("checkpoint, 1568 tokens, 160 rows", "checkpoint", 960, 160, 1568, "f16", (4, 4), 0.30),
        # a ragged number of tokens: rows start at any alignment, the last group is short
        _case("checkpoint, 12543 tokens, 2304 rows", "checkpoint", 256, 2304, 12543, "bf16", (4, 4), 0.25),
        # inputs of the largest layer
        _case("checkpoint, 8192 tokens, 4096 rows", "checkpoint", 4096, 4096, 8192, "bf16", (16, 16), 0.10),
        # fp32 training of a tiny layer; latency
        _case("weight_grad, 196 tokens, 64 x 64", "weight_grad", 64, 64, 196, "f32", (4, 4), 0.50),
        # small layer, ragged number of tokens, inputs as they were
        _case("weight_grad, 1567 tokens, 960 x 160", "weight_grad", 960, 160, 1567, "f16", (4, 4), 0.30),
        # small blocks, many tokens, inputs from the checkpoint
        _case("weight_grad, 12544 tokens, 256 x 2304", "weight_grad", 256, 2304, 12544, "bf16", (4, 4), 0.25, ckpt=True),
        # the largest layer, inputs from the checkpoint
        _case("weight_grad, 8192 tokens, 4096 x 4096", "weight_grad", 4096, 4096, 8192, "bf16", (16, 16), 0.10, ckpt=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("linear", "linear_grad", "checkpoint", "weight_grad"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    block = rng.choice(((4, 4), (8, 8), (16, 16), (4, 1), (16, 4)))
    top = 1024 if dtype == "f32" else 4096
    M, K = spread(64, top), spread(64, top)
    N = spread(1, 2048 if dtype == "f32" else 8192)
    if op in ("linear_grad", "checkpoint"):
        N = max(N, 16)
    # (as many blocks as the largest listed layer has, at most half of them again)
    density = min(rng.uniform(0.05, 0.35), 10000.0 * block[0] * block[1] / (M * K))
    c = _case("", op, M, K, N, dtype, block, density, rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")),
              rng.random() < 0.8, rng.random() < 0.6, rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _blocks(case, seed):
    """Blocks at arbitrary origins that share no cell, as many as the density says: uniform origins, drawn anew on a collision."""
    M, K, bh, bw = case["M"], case["K"], case["bh"], case["bw"]
    want = int(math.floor(M * K * case["density"] / (bh * bw) + 1e-9))
    rng = np.random.default_rng(seed)
    taken = np.zeros((M, K), dtype=bool)
    out = []
    for _ in range(200):
        rows = rng.integers(0, M - bh + 1, 2 * want + 8).tolist()
        cols = rng.integers(0, K - bw + 1, 2 * want + 8).tolist()
        for r, c in zip(rows, cols):
            if len(out) == want:
                break
            cells = taken[r:r + bh, c:c + bw]
            if not cells.any():
                cells[...] = True
                out.append((r, c))
    out.sort()
    return np.asarray(out, dtype=np.int32).reshape(-1, 2)


def _value_cells(blocks, bh, bw):
    """Rows and columns of the kept weights in the packed order."""
    s = np.arange(bh)[None, None, :]
    q = np.arange(bw)[None, :, None]
    r = blocks[:, 0].astype(np.int64)[:, None, None]
    c = blocks[:, 1].astype(np.int64)[:, None, None]
    rows = r + (s - r) % bh + 0 * q
    cols = c + q + 0 * s
    return rows.reshape(-1), cols.reshape(-1)


def _inputs(case, seed):
    """What both forms are given, on the GPU, from the seed alone."""
    M, K, N, t = case["M"], case["K"], case["N"], _T[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * scale

    x = {}
    op = case["op"]
    if op in ("linear", "weight_grad"):
        x["blocks"] = _blocks(case, seed)
    if op == "linear":
        cells = _value_cells(x["blocks"], case["bh"], case["bw"])
        kept = torch.zeros(M, K, device="cuda")
        kept[torch.from_numpy(cells[0]).cuda(), torch.from_numpy(cells[1]).cuda()] = 1.0
        x["W"] = (normal(M, K, scale=math.sqrt(2.0 / (K * case["density"]))) * kept).to(t)
        x["X"] = normal(K, N).to(t)
        x["b"] = normal(M, scale=0.5) if case["bias"] else None
        x["R"] = normal(M, N, scale=2.0).to(t) if case["res"] else None
    elif op == "linear_grad":
        x["dY"] = normal(M, N, scale=0.01).to(t)
        x["Z"] = normal(M, N, scale=1.5).to(t)
    elif op == "checkpoint":
        # activations: rows of different size, few large values
        x["X"] = (normal(K, N) * torch.exp(normal(K, 1)) * torch.where(normal(K, N) > 3.0, 8.0, 1.0)).to(t)
    else:
        x["G"] = normal(M, N, scale=0.01).to(t)
        X = normal(K, N).to(t)
        if case["ckpt"]:
            q, e = _to_e4m3(X.float())
            x["Q"] = q.to(torch.float8_e4m3fn).view(torch.uint8)
            x["S"] = (e + 127).to(torch.uint8)
        else:
            x["X"] = X
    return x


# ------------------------------------------------------------------ plain form: 32 bits, elementary operations
def _groups(N):
    return (N + 31) // 32


def _times_power(x, e):
    """x * 2^e for whole e in -254 .. 254, in two factors that are exact (pow of the GPU need not be)."""
    half = torch.div(e.int(), 2, rounding_mode="floor")
    for part in (half, e.int() - half):
        x = x * ((part + 127) << 23).view(torch.float32)
    return x


def _to_e4m3(x):
    """x in 32 bits -> the e4m3 values and the exponents of the groups of 32."""
    K, N = x.shape
    padded = torch.nn.functional.pad(x, (0, _groups(N) * 32 - N)).view(K, -1, 32)
    m, e = torch.frexp(padded.abs().amax(dim=2))
    e = torch.where(m <= 0.875, e - 9, e - 8)          # smallest e with amax <= 448 * 2^e
    e = torch.where(m == 0, torch.full_like(e, -127), e).clamp(min=-127)
    y = _times_power(padded, -e[:, :, None])
    step = (torch.frexp(y.abs())[1] - 4).clamp(min=-9)
    return _times_power(torch.round(_times_power(y, -step)), step).view(K, -1)[:, :N], e


def _from_e4m3(q, e, t):
    K, N = q.shape
    return _times_power(q, e.repeat_interleave(32, dim=1)[:, :N]).to(t)


def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return z * 0.5 * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if name == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3.0 * 0.044715 * z * z)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain(state):
    case, x = state["case"], state["x"]
    t = _T[case["dtype"]]
    op = case["op"]
    if op == "linear":
        z = torch.matmul(x["W"].float(), x["X"].float())
        if x["b"] is not None:
            z = z + x["b"][:, None]
        y = _act(case["act"], z)
        if x["R"] is not None:
            y = y + x["R"].float()
        return y.to(t)
    if op == "linear_grad":
        g = x["dY"].float() * _act_slope(case["act"], x["Z"].float())
        return (g.to(t), g.sum(dim=1)) if case["bias"] else g.to(t)
    if op == "checkpoint":
        q, e = _to_e4m3(x["X"].float())
        return _from_e4m3(q, e, t)
    X = x["X"].float() if "X" in x else _from_e4m3(x["Q"].view(torch.float8_e4m3fn).float(), x["S"].int() - 127, t).float()
    return torch.matmul(x["G"].float(), X.t()).reshape(-1)[state["at"]]


# ------------------------------------------------------------------ the framework's calls
def _pack(case, W, blocks):
    import paper_2407_19644_amd as ubp
    host = W.cpu()
    host = host.view(torch.uint16).numpy() if case["dtype"] == "bf16" else host.numpy()
    return ubp.pack(host, case["dtype"], case["bh"], case["bw"], blocks, device=torch.cuda.current_device())


def _own(state):
    import paper_2407_19644_amd as ubp
    case, x, p = state["case"], state["x"], state["packed"]
    N, d = case["N"], case["dtype"]
    stream = torch.cuda.current_stream().cuda_stream
    op = case["op"]
    if op == "linear":
        ubp.linear(p, x["X"].data_ptr(), N, N, state["Y"].data_ptr(), N, d,
                   bias_ptr=None if x["b"] is None else x["b"].data_ptr(), activation=case["act"],
                   residual_ptr=None if x["R"] is None else x["R"].data_ptr(), ldr=N, stream=stream)
        return state["Y"]
    ws, ws_bytes = state["ws"].data_ptr(), state["ws"].numel()
    if op == "linear_grad":
        ubp.linear_grad(p, x["dY"].data_ptr(), N, x["Z"].data_ptr(), N, N, state["G"].data_ptr(), N,
                        dbias_ptr=state["db"].data_ptr() if case["bias"] else None, activation=case["act"],
                        workspace_ptr=ws, workspace_bytes=ws_bytes, stream=stream)
        return (state["G"], state["db"]) if case["bias"] else state["G"]
    if op == "checkpoint":
        ubp.checkpoint_save(p, x["X"].data_ptr(), N, N, state["Q"].data_ptr(), N, state["S"].data_ptr(), _groups(N),
                            stream=stream)
        ubp.checkpoint_load(p, state["Q"].data_ptr(), N, state["S"].data_ptr(), _groups(N), N, state["X"].data_ptr(), N,
                            stream=stream)
        return state["X"]
    if case["ckpt"]:
        ubp.weight_grad_checkpoint(p, x["G"].data_ptr(), N, x["Q"].data_ptr(), N, x["S"].data_ptr(), _groups(N), N,
                                   state["dW"].data_ptr(), workspace_ptr=ws, workspace_bytes=ws_bytes, stream=stream)
    else:
        ubp.weight_grad(p, x["G"].data_ptr(), N, x["X"].data_ptr(), N, N, state["dW"].data_ptr(), workspace_ptr=ws,
                        workspace_bytes=ws_bytes, stream=stream)
    return state["dW"]


def prepare(case, seed):
    M, K, N, t, op = case["M"], case["K"], case["N"], _T[case["dtype"]], case["op"]
    x = _inputs(case, seed)
    state = {"case": case, "x": x}
    if not own:
        if op == "weight_grad":
            rows, cols = _value_cells(x["blocks"], case["bh"], case["bw"])
            state["at"] = torch.from_numpy(rows * K + cols).cuda()
        return state
    import paper_2407_19644_amd as ubp
    # the layer's handle; where an operator looks at no weight, one without blocks carries the layer's sizes and type
    W = x["W"] if op == "linear" else torch.zeros(M, K, dtype=t)
    p = state["packed"] = _pack(case, W, x["blocks"] if "blocks" in x else np.zeros((0, 2), dtype=np.int32))
    if op == "linear":
        state["Y"] = torch.empty(M, N, dtype=t, device="cuda")
        ubp.spmm_prepare(p, x["X"].data_ptr(), N, N, state["Y"].data_ptr(), N, case["dtype"])
    elif op == "linear_grad":
        state["G"] = torch.empty(M, N, dtype=t, device="cuda")
        state["db"] = torch.empty(M, dtype=torch.float32, device="cuda")
        state["ws"] = torch.empty(max(ubp.linear_grad_workspace(p, N), 16), dtype=torch.uint8, device="cuda")
    elif op == "checkpoint":
        state["Q"] = torch.empty(K, N, dtype=torch.uint8, device="cuda")
        state["S"] = torch.empty(K, _groups(N), dtype=torch.uint8, device="cuda")
        state["X"] = torch.empty(K, N, dtype=t, device="cuda")
        state["ws"] = torch.empty(16, dtype=torch.uint8, device="cuda")
    else:
        state["dW"] = torch.empty(len(x["blocks"]) * case["bh"] * case["bw"], dtype=torch.float32, device="cuda")
        state["ws"] = torch.empty(max(ubp.weight_grad_workspace(p, N), 16), dtype=torch.uint8, device="cuda")
    return state


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def _kept(case):
    return int(math.floor(case["M"] * case["K"] * case["density"] / (case["bh"] * case["bw"]) + 1e-9)) * case["bh"] * case["bw"]


def work(case):
    M, K, N, size, op = case["M"], case["K"], case["N"], _SIZE[case["dtype"]], case["op"]
    kept = _kept(case)
    eight = K * N + K * _groups(N)
    if op == "linear":
        outputs = 2 if case["res"] else 1
        return {"bytes": kept * size + K * N * size + outputs * M * N * size + (4 * M if case["bias"] else 0), "flops": 2 * kept * N}
    if op == "linear_grad":
        return {"bytes": 3 * M * N * size + (4 * M if case["bias"] else 0), "flops": 10 * M * N}
    if op == "checkpoint":
        return {"bytes": 2 * K * N * size + 2 * eight, "flops": 4 * K * N}
    return {"bytes": M * N * size + (eight if case["ckpt"] else K * N * size) + 4 * kept, "flops": 2 * kept * N}


# ------------------------------------------------------------------ the definitions in 64 bits
def _e4m3_values():
    """The 127 finite e4m3 values that are not negative: 3 bits of fraction, exponents -6 .. 8, below them multiples of 2^-9."""
    v = [k * 2.0 ** -9 for k in range(8)]
    for e in range(-6, 9):
        v += [(8 + k) * 2.0 ** (e - 3) for k in range(8)]
    return v[:-1]                                       # (the last code is NaN; 448 is the largest)


def _power64(s):
    return ((s.long() + 1023) << 52).view(torch.float64)


def exact(case, seed):
    x = _inputs(case, seed)
    op, act, N = case["op"], case["act"], case["N"]
    f64 = torch.float64
    if op in ("linear", "linear_grad"):
        if op == "linear":
            z = x["W"].to(f64) @ x["X"].to(f64)
            if x["b"] is not None:
                z += x["b"].to(f64).unsqueeze(1)
        else:
            z = x["Z"].to(f64)
        a = math.sqrt(2.0 / math.pi)
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        sig = torch.sigmoid(z)
        th = torch.sigmoid(2.0 * a * (z + 0.044715 * z ** 3))     # (1 + tanh u) / 2
        if op == "linear":
            y = {"none": z, "relu": torch.where(z > 0, z, 0.0), "gelu": z * phi, "gelu_tanh": z * th, "silu": z * sig}[act]
            return y if x["R"] is None else y + x["R"].to(f64)
        slope = {"none": torch.ones_like(z), "relu": torch.where(z > 0, 1.0, 0.0).to(f64),
                 "gelu": phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
                 "gelu_tanh": th + 2.0 * a * z * th * (1.0 - th) * (1.0 + 0.134145 * z ** 2),
                 "silu": sig + z * sig * (1.0 - sig)}[act]
        g = x["dY"].to(f64) * slope
        return (g, g.sum(1)) if case["bias"] else g
    if op == "checkpoint":
        X = x["X"].to(f64)
        table = torch.tensor(_e4m3_values(), dtype=f64, device="cuda")
        out = torch.empty_like(X)
        # groups, some rows at a time
        for r in range(0, X.shape[0], 512):
            rows = X[r:r + 512]
            top = torch.stack([rows[:, c:c + 32].abs().amax(1) for c in range(0, N, 32)], 1)
            s = torch.ceil(torch.log2(torch.clamp(top / 448.0, min=2.0 ** -300)))
            s = torch.where(top > 448.0 * _power64(s), s + 1, torch.where(top <= 448.0 * _power64(s - 1), s - 1, s)).clamp(min=-127)
            scale = _power64(s).repeat_interleave(32, 1)[:, :N]
            y = rows.abs() / scale
            hi = torch.searchsorted(table, y).clamp(max=len(table) - 1)
            lo = (hi - 1).clamp(min=0)
            up, down = table[hi] - y, y - table[lo]
            code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
            out[r:r + 512] = torch.sign(rows) * table[code] * scale
        return out.to(_T[case["dtype"]]).to(f64)
    if "X" in x:
        X = x["X"].to(f64)
    else:
        code = (x["Q"] & 127).long()
        table = torch.tensor(_e4m3_values() + [float("nan")], dtype=f64, device="cuda")
        X = torch.where(x["Q"] >= 128, -1.0, 1.0) * table[code]
        X *= _power64(x["S"].long() - 127).repeat_interleave(32, 1)[:, :N]
        X = X.to(_T[case["dtype"]]).to(f64)
    dense = x["G"].to(f64) @ X.t()
    bh, bw = case["bh"], case["bw"]
    out = torch.empty(len(x["blocks"]), bw, bh, dtype=f64, device="cuda")
    start = torch.from_numpy(x["blocks"].astype(np.int64)).cuda()
    for i in range(bh):
        row = start[:, 0] + i
        for q in range(bw):
            out[torch.arange(len(start), device="cuda"), q, row % bh] = dense[row, start[:, 1] + q]
    return out.reshape(-1)
