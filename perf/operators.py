"""The layers around a chunk's gradient and the orthogonalised update, as they are measured.

`listed()` and `draw()` give cases of three families, `prepare()` the tensors that a training or serving program has in hand,
`run()` one pass:

  norm           an RMSNorm or LayerNorm layer: forward (output and per-token statistics) or backward (input gradient and the
                 fp32 gradients of scale and shift)
  linear         y = act(x W^T + bias) + residual: forward (with the pre-activation where a backward pass follows) or backward
                 (gradient of the pre-activation, of the bias in fp32, of the input)
  orthogonalize  Newton-Schulz steps on a matrix, the result in the matrix' own type
  muon           momentum, the steps on it, and the update of a chunk of whole rows: fp32 master and momentum, bf16 weights

With `own` false `run` is the plain form in elementary torch operations, in 32 bits, rounded once at the end; with `own` true it
calls the library.  `exact()` is the definition in 64 bits.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
DEV = "cuda"
STEPS = 5
NS_EPS = 1e-7
NORM_EPS = 1e-5
MUON = dict(lr=0.02, momentum=0.95, weight_decay=0.01)
COEF_A, COEF_B, COEF_C = 3.4445, -4.7750, 2.0315


def _norm(way, kind, dtype, tokens, width):
    return dict(op="norm", way=way, kind=kind, dtype=dtype, tokens=tokens, width=width)


def _linear(way, dtype, tokens, n_in, out, act, residual=False, keep=False, pad=0):
    """keep: the forward pass also writes the pre-activation; pad: extra columns of the buffers that x, y, dy are views of."""
    return dict(op="linear", way=way, dtype=dtype, tokens=tokens, n_in=n_in, out=out, act=act, residual=residual, keep=keep, pad=pad)


def listed():
    return [
        # one token of a serving loop through an RMSNorm: nothing but latency
        dict(_norm("forward", "rmsnorm", "bf16", 1, 4096), name="norm_one_token"),
        # the norm in front of an 8B-shaped block's projections at a training batch of 4096 tokens
        dict(_norm("forward", "layernorm", "bf16", 4096, 4096), name="norm_forward"),
        # its backward pass over 8192 tokens: input gradient, both vectors' gradients
        dict(_norm("backward", "layernorm", "bf16", 8192, 4096), name="norm_backward"),
        # full precision, odd width and token count
        dict(_norm("backward", "rmsnorm", "f32", 1021, 2907), name="norm_backward_odd_f32"),
        # one token through an 8B-shaped up projection: the weights are read once
        dict(_linear("forward", "bf16", 1, 4096, 14336, "silu"), name="linear_one_token"),
        # the same projection in training: bias and GELU in the epilogue, pre-activation kept
        dict(_linear("forward", "bf16", 1024, 4096, 14336, "gelu", keep=True), name="linear_up_gelu"),
        # the down projection onto the residual stream, sizes without 16-byte rows
        dict(_linear("forward", "bf16", 1001, 2907, 2705, "none", residual=True), name="linear_ragged_residual"),
        # backward pass of the up projection at 4096 tokens
        dict(_linear("backward", "bf16", 4096, 4096, 14336, "gelu"), name="linear_up_backward"),
        # the smallest full-precision layer, backward
        dict(_linear("backward", "f32", 256, 512, 1024, "relu"), name="linear_small_f32_backward"),
        # a square projection's update in 16 bits
        dict(op="orthogonalize", dtype="bf16", rows=4096, cols=4096, name="orthogonalize_square_bf16"),
        # a key projection as one chunk: fp32 steps, few rows
        dict(op="muon", rows=1024, cols=4096, name="muon_key_projection"),
        # 32 Mi elements, 8192 whole rows of an up projection
        dict(op="muon", rows=8192, cols=4096, name="muon_up_projection_rows"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "orthogonalize", "muon"])
    if op == "norm":
        width = rng.choice([1, 8, 64])
        width *= _log_int(rng, 64 // width, 16384 // width)
        return _norm(rng.choice(["forward", "backward"]), rng.choice(["rmsnorm", "layernorm"]), rng.choice(["f32", "bf16", "bf16"]),
                     min(_log_int(rng, 1, 16384), (64 << 20) // width), width)
    if op == "linear":
        dtype = rng.choice(["f32", "bf16", "bf16", "bf16"])
        unit = rng.choice([1, 8, 64])
        n_in, out = unit * _log_int(rng, 64 // unit, 14336 // unit), unit * _log_int(rng, 64 // unit, 14336 // unit)
        tokens = _log_int(rng, 1, 8192)
        most = 2e11 if dtype == "bf16" and unit > 1 else 2e10
        tokens = max(1, min(tokens, int(most / (n_in * out))))
        way = rng.choice(["forward", "backward"])
        return _linear(way, dtype, tokens, n_in, out, rng.choice(["none", "relu", "gelu", "silu"]),
                       residual=way == "forward" and rng.random() < 0.5, keep=way == "forward" and rng.random() < 0.5,
                       pad=rng.choice([0, 0, 64]))
    unit = rng.choice([1, 8, 64])
    rows, cols = unit * _log_int(rng, 64 // unit, 8192 // unit), unit * _log_int(rng, 64 // unit, 8192 // unit)
    while min(rows, cols) ** 2 * max(rows, cols) > 8192 * 4096 * 4096:
        rows, cols = rows // 2 // unit * unit, cols // 2 // unit * unit
    if op == "orthogonalize":
        return dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16"]), rows=rows, cols=cols)
    return dict(op=op, rows=rows, cols=cols)


# ------------------------------------------------------------------ inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _view(t, dtype, pad):
    """t as rows of a wider buffer."""
    buf = torch.empty(t.shape[0], t.shape[1] + pad, dtype=dtype, device=DEV)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _update_like(gen, rows, cols):
    """A gradient's shape of spectrum: half of the energy in a few directions, the rest spread."""
    rank = max(1, min(rows, cols) // 64)
    low = _randn(gen, rows, rank) @ _randn(gen, rank, cols) / math.sqrt(rank)
    return (low + _randn(gen, rows, cols)) * 1e-3


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    if op == "norm":
        T, n, dt = case["tokens"], case["width"], DTYPES[case["dtype"]]
        x = _randn(gen, T, n) * (1 + 0.5 * _randn(gen, n).abs()) + 0.3 * _randn(gen, n)    # channels of different size and mean
        s = dict(case=case, x=x.to(dt), w=(1 + 0.1 * _randn(gen, n)).to(dt), y=torch.empty(T, n, dtype=dt, device=DEV),
                 stats=torch.empty(T, 2, device=DEV))
        s["b"] = (0.1 * _randn(gen, n)).to(dt) if case["kind"] == "layernorm" else None
        if case["way"] == "backward":
            s["dy"] = (1e-3 * _randn(gen, T, n)).to(dt)
            s["dw"], s["db"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            xf = s["x"].double()                                                          # the forward pass left its statistics
            mean = xf.mean(1) if case["kind"] == "layernorm" else torch.zeros(T, dtype=torch.float64, device=DEV)
            var = (xf - mean[:, None]).square().mean(1)
            s["stats"][:, 0] = mean
            s["stats"][:, 1] = (var + NORM_EPS).rsqrt()
        return s
    if op == "linear":
        T, n_in, out, dt, pad = case["tokens"], case["n_in"], case["out"], DTYPES[case["dtype"]], case["pad"]
        s = dict(case=case, W=(_randn(gen, out, n_in) / math.sqrt(n_in)).to(dt), bias=(0.1 * _randn(gen, out)).to(dt))
        if case["way"] == "forward":
            s["x"] = _view(_randn(gen, T, n_in), dt, pad)
            s["res"] = _view(_randn(gen, T, out), dt, pad) if case["residual"] else None
            s["y"] = _view(torch.zeros(T, out, device=DEV), dt, pad)
            s["z"] = torch.empty(T, out, dtype=dt, device=DEV) if case["keep"] else None
        else:
            s["dy"], s["z"] = _view(1e-3 * _randn(gen, T, out), dt, pad), _randn(gen, T, out).to(dt)
            s["dz"] = torch.empty(T, out, dtype=dt, device=DEV) if case["act"] != "none" else None
            s["dx"] = _view(torch.zeros(T, n_in, device=DEV), dt, pad)
            s["db"] = torch.empty(out, device=DEV)
        return s
    rows, cols = case["rows"], case["cols"]
    u = _update_like(gen, rows, cols)
    if op == "orthogonalize":
        return dict(case=case, g=u.to(DTYPES[case["dtype"]]), o=torch.empty(rows, cols, dtype=DTYPES[case["dtype"]], device=DEV))
    master = 0.02 * _randn(gen, rows, cols)
    return dict(case=case, g=u, m=4 * _update_like(gen, rows, cols), master=master, W=master.bfloat16(),
                scale=max(1.0, rows / cols) ** 0.5)


# ------------------------------------------------------------------ the library's calls
def _workspace(s, need):
    """Kept from pass to pass beside the tensors it serves, as a training loop keeps it."""
    if need and s.get("ws") is None:
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s.get("ws")


def _run_own(s):
    from paper_2605_21177_amd import binding as B
    case = s["case"]
    op = case["op"]
    if op == "norm":
        layer = B.make_norm(B.LAYERNORM if case["kind"] == "layernorm" else B.RMSNORM, s["x"], s["w"], s["b"], NORM_EPS)
        if case["way"] == "forward":
            B.chunkft_norm_forward(layer, s["y"], s["stats"])
            return _norm_out(s, s["y"], s["stats"])
        ws = _workspace(s, B.chunkft_norm_workspace_bytes(layer))
        shift = case["kind"] == "layernorm"
        B.chunkft_norm_backward(layer, s["stats"], s["dy"], s["y"], dw=s["dw"], db=s["db"] if shift else None, ws=ws)
        return dict(dx=s["y"], dw=s["dw"], **({"db": s["db"]} if shift else {}))
    if op == "linear":
        act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}[case["act"]]
        if case["way"] == "forward":
            layer = B.make_linear(s["x"], s["W"], bias=s["bias"], activation=act, residual=s["res"])
            ws = _workspace(s, B.chunkft_linear_workspace_bytes(layer))
            B.chunkft_linear_forward(layer, s["y"], Z=s["z"], ws=ws)
            return dict(y=s["y"], **({"z": s["z"]} if case["keep"] else {}))
        layer = B.make_linear(None, s["W"], activation=act, tokens=case["tokens"])
        ws = _workspace(s, B.chunkft_linear_workspace_bytes(layer, backward=True))
        B.chunkft_linear_backward(layer, s["dy"], Z=s["z"], dZ=s["dz"], dX=s["dx"], db=s["db"], ws=ws)
        return dict(dx=s["dx"], db=s["db"], **({"dz": s["dz"]} if case["act"] != "none" else {}))
    if op == "orthogonalize":
        ws = _workspace(s, B.chunkft_orthogonalize_workspace_bytes(B.BF16 if case["dtype"] == "bf16" else B.F32, *s["g"].shape))
        B.chunkft_orthogonalize(s["g"], s["o"], steps=STEPS, eps=NS_EPS, ws=ws)
        return s["o"]
    hp = B.muon_hparams(**MUON, scale=s["scale"], steps=STEPS, eps=NS_EPS, nesterov=True, precision=B.F32)
    ws = _workspace(s, B.chunkft_orthogonalize_workspace_bytes(B.F32, *s["g"].shape))
    B.chunkft_muon_chunk(s["g"], s["master"], s["m"], s["W"], case["rows"], case["cols"], hp, ws=ws)
    return dict(master=s["master"], m=s["m"], W=s["W"])


# ------------------------------------------------------------------ plain forms
def _norm_out(s, y, stats):
    """An RMSNorm has no mean: only the second column says something."""
    return dict(y=y, rstd=stats[:, 1], **({"mean": stats[:, 0]} if s["case"]["kind"] == "layernorm" else {}))


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _newton_schulz(u):
    """In 64 bits inside the 32-bit form where only the norm is summed; wide: the products are the small side's."""
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (x.double().square().sum().sqrt() + NS_EPS).float()
    for _ in range(STEPS):
        a = x @ x.t()
        x = COEF_A * x + (COEF_B * a + COEF_C * (a @ a)) @ x
    return x.t() if tall else x


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        x, w, layernorm = s["x"].float(), s["w"].float(), case["kind"] == "layernorm"
        if case["way"] == "forward":
            mean = x.mean(1, keepdim=True) if layernorm else torch.zeros_like(x[:, :1])
            rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + NORM_EPS).sqrt()
            y = (x - mean) * rstd * w
            y = y + s["b"].float() if layernorm else y
            return _norm_out(s, y.to(s["x"].dtype), torch.cat([mean, rstd], 1))
        mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
        dy = s["dy"].float()
        xh = (x - mean) * rstd if layernorm else x * rstd
        h = dy * w
        dx = h - xh * (h * xh).mean(1, keepdim=True)
        dx = (dx - h.mean(1, keepdim=True) if layernorm else dx) * rstd
        return dict(dx=dx.to(s["x"].dtype), dw=(dy * xh).sum(0), **({"db": dy.sum(0)} if layernorm else {}))
    if op == "linear":
        W = s["W"].float()
        if case["way"] == "forward":
            z = s["x"].float() @ W.t() + s["bias"].float()
            y = _act(z, case["act"])
            y = y + s["res"].float() if case["residual"] else y
            return dict(y=y.to(s["W"].dtype), **({"z": z.to(s["W"].dtype)} if case["keep"] else {}))
        dy = s["dy"].float()
        dz = dy * _act_slope(s["z"].float(), case["act"]) if case["act"] != "none" else dy
        out = dict(dx=(dz @ W).to(s["W"].dtype), db=dz.sum(0))
        return dict(out, dz=dz.to(s["W"].dtype)) if case["act"] != "none" else out
    if op == "orthogonalize":
        return _newton_schulz(s["g"].float()).to(s["g"].dtype)
    s["m"].mul_(MUON["momentum"]).add_(s["g"])
    o = _newton_schulz(s["g"] + MUON["momentum"] * s["m"])
    s["master"].sub_(MUON["lr"] * (s["scale"] * o + MUON["weight_decay"] * s["master"]))
    s["W"].copy_(s["master"])
    return dict(master=s["master"], m=s["m"], W=s["W"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "norm":
        cells, s = case["tokens"] * case["width"], SIZE[case["dtype"]]
        if case["way"] == "forward":
            return dict(bytes=2 * cells * s + 2 * case["width"] * s + 8 * case["tokens"], flops=8 * cells)
        return dict(bytes=3 * cells * s + case["width"] * (s + 8) + 8 * case["tokens"], flops=14 * cells)
    if op == "linear":
        T, n_in, out, s = case["tokens"], case["n_in"], case["out"], SIZE[case["dtype"]]
        wide = 1 + case["residual"] + case["keep"] if case["way"] == "forward" else 1 if case["act"] == "none" else 3
        return dict(bytes=s * (T * n_in + out * n_in + wide * T * out + out), flops=2 * T * n_in * out)
    r, c = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    flops = STEPS * (3 * r * r * c + r * r * r)          # the Gram matrix and its square are symmetric: half of each
    return dict(bytes=r * c * (2 * SIZE[case["dtype"]] if op == "orthogonalize" else 4 * 5 + 2), flops=flops)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point() and k not in ("y", "o", "dx", "ws")}
    op = case["op"]
    if op == "norm":
        n, layernorm = case["width"], case["kind"] == "layernorm"
        if case["way"] == "forward":
            mu = d["x"].sum(1) / n if layernorm else torch.zeros(case["tokens"], dtype=torch.float64, device=DEV)
            centred = d["x"] - mu.unsqueeze(1)
            r = torch.rsqrt((centred * centred).sum(1) / n + NORM_EPS)
            y = torch.einsum("tn,t,n->tn", centred, r, d["w"])
            if layernorm:
                return dict(y=y + d["b"], rstd=r, mean=mu)
            return dict(y=y, rstd=r)
        mu, r = d["stats"].unbind(1)
        xh = (d["x"] - mu.unsqueeze(1)) * r.unsqueeze(1) if layernorm else d["x"] * r.unsqueeze(1)
        h = d["dy"] * d["w"]
        along = (h * xh).sum(1, keepdim=True) / n
        flat = h.sum(1, keepdim=True) / n if layernorm else 0.0
        out = dict(dx=r.unsqueeze(1) * (h - flat - xh * along), dw=(d["dy"] * xh).sum(0))
        return dict(out, db=d["dy"].sum(0)) if layernorm else out
    if op == "linear":
        if case["way"] == "forward":
            z = torch.addmm(d["bias"], d["x"], d["W"].t())
            y = {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z * torch.sigmoid(z),
                 "gelu": lambda: torch.special.ndtr(z) * z}[case["act"]]()
            y = y + d["res"] if case["residual"] else y
            return dict(y=y, z=z) if case["keep"] else dict(y=y)
        if case["act"] == "none":
            return dict(dx=torch.mm(d["dy"], d["W"]), db=d["dy"].sum(0))
        z = d["z"]
        if case["act"] == "relu":
            slope = torch.where(z > 0, 1.0, 0.0).double()
        elif case["act"] == "gelu":
            slope = torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        dz = d["dy"] * slope
        return dict(dx=torch.mm(dz, d["W"]), db=dz.sum(0), dz=dz)

    def orthogonal(u):
        x = u / (torch.linalg.matrix_norm(u) + NS_EPS)
        eye = torch.eye(min(u.shape), dtype=torch.float64, device=DEV)
        for _ in range(STEPS):
            gram = x.t() @ x if u.shape[0] > u.shape[1] else x @ x.t()
            poly = COEF_A * eye + gram @ (COEF_B * eye + COEF_C * gram)
            x = x @ poly if u.shape[0] > u.shape[1] else poly @ x
        return x

    if op == "orthogonalize":
        return orthogonal(d["g"])
    m = MUON["momentum"] * d["m"] + d["g"]
    o = orthogonal(d["g"] + MUON["momentum"] * m)
    master = d["master"] - MUON["lr"] * (s["scale"] * o + MUON["weight_decay"] * d["master"])
    return dict(master=master, m=m, W=master)
