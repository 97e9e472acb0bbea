"""The layers under autograd, and the operators together as a training step uses them: a pre-norm block (LayerNorm, up projection with
bias and GELU, down projection with bias onto the residual stream) whose chunk crosses its tensors, against torch's own autograd
in 64 bits, and against differences.

Bounds on a gradient's relative Frobenius error: a product of K terms in fp32 is off by at most K 2^-24 |A||B|, about K^1.5 2^-24 of
the product of random factors; the chain has seven products of at most 600 terms or sums of as many: 7 x 600^1.5 x 2^-24 = 6e-3 for
fp32, and for bf16 the dozen tensors that are rounded to 8 bits on the way add 12 x 2^-9 (a rounding's root mean square is half its
bound) = 2.4e-2."""

import pytest
import torch

from paper_2605_21177_amd import autograd as A
from paper_2605_21177_amd import binding as B

import gpu_harness as H
from layers_harness import DEV, act64

pytestmark = pytest.mark.gpu

BOUND = {torch.float32: 6e-3, torch.bfloat16: 6e-3 + 2.4e-2}
D, FF = 264, 520
SHAPES = dict(w=(D,), b=(D,), W1=(FF, D), b1=(FF,), W2=(D, FF), b2=(D,))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    H.require_gpu()


def _params(seed, dtype):
    gen = torch.Generator().manual_seed(seed)
    p = {k: 0.1 * torch.randn(*s, generator=gen) for k, s in SHAPES.items()}
    p["w"] += 1
    return {k: v.to(dtype) for k, v in p.items()}


def _data(seed, dtype, lead=(3, 70)):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(*lead, D, generator=gen).to(dtype), (1e-2 * torch.randn(*lead, D, generator=gen)).to(dtype)


def _block(x, p, s):
    h = A.chunk_norm(x, p["w"], p["b"], B.LAYERNORM, 1e-5, s.get("w"), s.get("b"))
    h = A.chunk_linear(h, p["W1"], s.get("W1"), bias=p["b1"], bias_seg=s.get("b1"), activation=B.ACT_GELU)
    return A.chunk_linear(h, p["W2"], s.get("W2"), bias=p["b2"], bias_seg=s.get("b2"), residual=x)


def _block64(x, p):
    mean = x.mean(-1, keepdim=True)
    h = (x - mean) / ((x - mean).square().mean(-1, keepdim=True) + 1e-5).sqrt() * p["w"] + p["b"]
    return act64(h @ p["W1"].t() + p["b1"], "gelu") @ p["W2"].t() + p["b2"] + x


def _grads64(x, R, p):
    leaves = {k: v.double().requires_grad_() for k, v in p.items()}
    xd = x.double().requires_grad_()
    y = _block64(xd, leaves)
    (y * R.double()).sum().backward()
    return y.detach(), xd.grad, {k: v.grad.reshape(-1) for k, v in leaves.items()}


def _off(got, ref):
    return float((got.detach().double().cpu().reshape(-1) - ref.reshape(-1)).norm() / ref.norm())


def _part(k):
    n = torch.Size(SHAPES[k]).numel()
    return n // 5 + 1, n - n // 7


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_gradients_over_two_micro_batches(dtype):
    p = _params(1, dtype)
    dev = {k: v.to(DEV) for k, v in p.items()}
    segs = {k: A.ChunkSegment(*_part(k), torch.full((_part(k)[1] - _part(k)[0],), 9.0, device=DEV)) for k in SHAPES}
    total = {}
    for seed in (2, 3):
        x, R = _data(seed, dtype)
        xd = x.to(DEV).requires_grad_()
        y = _block(xd, dev, segs)
        (y.float() * R.to(DEV).float()).sum().backward()
        y64, dx64, g64 = _grads64(x, R, p)
        assert y.shape == x.shape and _off(y, y64) <= BOUND[dtype]
        assert _off(xd.grad, dx64) <= BOUND[dtype]
        for k in SHAPES:
            total[k] = total.get(k, 0) + g64[k][slice(*_part(k))]
    for k, seg in segs.items():
        assert seg.micro_batches == 2 and _off(seg.g, total[k]) <= BOUND[dtype], k


def test_only_what_is_active_is_computed_and_the_input_needs_no_gradient():
    p = {k: v.to(DEV) for k, v in _params(4, torch.float32).items()}
    x, R = _data(5, torch.float32)
    for active in SHAPES:
        seg = A.ChunkSegment(*_part(active), torch.empty(_part(active)[1] - _part(active)[0], device=DEV))
        y = _block(x.to(DEV), p, {active: seg, "W1" if active != "W1" else "W2": A.ChunkSegment(0, 0)})
        (y * R.to(DEV)).sum().backward()
        ref = _grads64(x, R, {k: v.cpu() for k, v in p.items()})[2][active][slice(*_part(active))]
        assert _off(seg.g, ref) <= BOUND[torch.float32], active
    with torch.no_grad():
        y2 = _block(x.to(DEV), p, {})
    assert not y2.requires_grad and torch.equal(y2, y.detach())
    assert not _block(x.to(DEV), p, {}).requires_grad


def test_directional_differences():
    """(L(x + h d) - L(x - h d)) / 2h against the gradient along d, fp32: the difference is off by its own h^2 term and by the
    loss's rounding over h; with h = 1e-2 and |L| of a few units, 1e-3 of the gradient's size covers both."""
    p = {k: v.to(DEV) for k, v in _params(6, torch.float32).items()}
    x, R = (t.to(DEV) for t in _data(7, torch.float32))
    xd = x.clone().requires_grad_()
    (_block(xd, p, {}).double() * R.double()).sum().backward()
    gen = torch.Generator().manual_seed(8)
    for _ in range(3):
        d = torch.randn(x.shape, generator=gen).to(DEV)
        loss = lambda t: (_block(t, p, {}).double() * R.double()).sum()  # noqa: E731
        with torch.no_grad():
            slope = float((loss(x + 1e-2 * d) - loss(x - 1e-2 * d)) / 2e-2)
        along = float((xd.grad.double() * d.double()).sum())
        assert abs(slope - along) <= 1e-3 * float(xd.grad.norm() * d.norm()) / d.numel() ** 0.5 + 1e-3 * abs(along)


def test_one_step_with_every_update():
    """Orthogonalised update on whole rows of W1, AdamW on a part of W2 and on the vectors, all inside backward; the gradients come from a
    plain pass on the same data, the updates from the calls by themselves: the same bits."""
    dtype = torch.bfloat16
    p = {k: v.to(DEV) for k, v in _params(9, dtype).items()}
    x, R = (t.to(DEV) for t in _data(10, dtype))
    spans = {k: _part(k) for k in SHAPES}
    spans["W1"] = (8 * D, 408 * D)
    plain = {k: A.ChunkSegment(*s, torch.empty(s[1] - s[0], device=DEV)) for k, s in spans.items()}
    (_block(x, p, plain).float() * R.float()).sum().backward()
    adam, muon = B.hparams(1e-2, 0.9, 0.999, 1e-8, 0.01, 1), B.muon_hparams(0.02, 0.9, 0.01, scale=1.5)
    want, fused = {}, {}
    for k, (b, e) in spans.items():
        master = p[k].view(-1)[b:e].float()
        w = p[k].view(-1)[b:e].clone()
        m, v = torch.zeros_like(master), torch.zeros_like(master)
        if k == "W1":
            fused[k] = A.ChunkSegment(b, e, master=master.clone(), m=m.clone(), hp=muon)
            ws = torch.empty(B.chunkft_orthogonalize_workspace_bytes(B.F32, 400, D), dtype=torch.uint8, device=DEV)
            B.chunkft_muon_chunk(plain[k].g, master, m, w, 400, D, muon, ws=ws)
        else:
            fused[k] = A.ChunkSegment(b, e, master=master.clone(), m=m.clone(), v=v.clone(), hp=adam)
            B.chunkft_adamw_chunk(plain[k].g, master, m, v, w, e - b, adam)
        want[k] = master, m, w
    before = {k: v.clone() for k, v in p.items()}
    (_block(x, p, fused).float() * R.float()).sum().backward()
    torch.cuda.synchronize()
    for k, (b, e) in spans.items():
        master, m, w = want[k]
        assert torch.equal(fused[k].master, master) and torch.equal(fused[k].m, m) and torch.equal(p[k].view(-1)[b:e], w), k
        assert torch.equal(p[k].view(-1)[:b], before[k].view(-1)[:b]) and torch.equal(p[k].view(-1)[e:], before[k].view(-1)[e:]), k
    snapshot = {k: v.clone() for k, v in p.items()}
    with pytest.raises(RuntimeError, match="one micro-batch"):
        (_block(x, p, fused).float() * R.float()).sum().backward()
    torch.cuda.synchronize()
    assert all(torch.equal(p[k], snapshot[k]) for k in p)
    with pytest.raises(ValueError, match="whole rows"):
        seg = A.ChunkSegment(3, D + 3, master=torch.zeros(D, device=DEV), m=torch.zeros(D, device=DEV), hp=muon)
        (_block(x, p, {"W1": seg}).float() * R.float()).sum().backward()


def test_mixed_segments_of_one_norm():
    """A plain part of the scale in its second micro-batch beside a fused part of the shift: one call writes both kinds."""
    x, R = (t.to(DEV) for t in _data(11, torch.float32))
    p = _params(12, torch.float32)
    w, b = p["w"].to(DEV), p["b"].to(DEV)
    seg_w = A.ChunkSegment(3, 200, torch.empty(197, device=DEV))
    loss = lambda s: (A.chunk_norm(x, w, b, B.LAYERNORM, 1e-5, seg_w, s) * R).sum()  # noqa: E731
    loss(None).backward()
    once = seg_w.g.clone()
    master = b[5:9].clone()
    seg_b = A.ChunkSegment(5, 9, master=master, m=torch.zeros(4, device=DEV), v=torch.zeros(4, device=DEV), hp=B.hparams(0.1, 0.9, 0.999, 1e-8, 0.0, 1))
    loss(seg_b).backward()
    torch.cuda.synchronize()
    assert torch.equal(seg_w.g, once + once) and seg_w.micro_batches == 2
    # the first AdamW step is lr g / (|g| + eps): the sign of the gradient
    g = R.double().reshape(-1, D).sum(0)[5:9].cpu()
    step = (p["b"][5:9] - master.cpu()).double()
    assert torch.allclose(step, 0.1 * g / (g.abs() + 1e-8), atol=1e-5)
    assert torch.equal(b[5:9], master)


def test_no_tokens():
    p = {k: v.to(DEV) for k, v in _params(13, torch.bfloat16).items()}
    segs = {k: A.ChunkSegment(*_part(k), torch.full((_part(k)[1] - _part(k)[0],), 7.0, device=DEV)) for k in SHAPES}
    x = torch.empty(0, 5, D, dtype=torch.bfloat16, device=DEV).requires_grad_()
    y = _block(x, p, segs)
    assert y.shape == x.shape
    y.float().sum().backward()
    assert x.grad.shape == x.shape and all(bool((s.g == 0).all()) and s.micro_batches == 1 for s in segs.values())


def test_strided_inputs_and_gradients():
    p = {k: v.to(DEV) for k, v in _params(14, torch.float32).items()}
    x, R = _data(15, torch.float32, (4, 30))
    ref_y, ref_dx, _ = _grads64(x, R, {k: v.cpu() for k, v in p.items()})
    turned = x.transpose(0, 1).contiguous().to(DEV).requires_grad_()        # [30, 4, D], seen as [4, 30, D]
    y = _block(turned.transpose(0, 1), p, {})
    (y.transpose(1, 2) * R.to(DEV).transpose(1, 2)).sum().backward()
    assert _off(y, ref_y) <= BOUND[torch.float32]
    assert _off(turned.grad.transpose(0, 1), ref_dx) <= BOUND[torch.float32]


def test_captured_step_beside_a_living_eager_graph():
    """Forward and backward of the block in a graph, on a side stream, while an eager graph over the same parameters and segments is
    alive; replayed with eager work between, each replay against the eager result."""
    dtype = torch.bfloat16
    p = {k: v.to(DEV) for k, v in _params(16, dtype).items()}
    x, R = (t.to(DEV) for t in _data(17, dtype))
    new = lambda: {k: A.ChunkSegment(*_part(k), torch.zeros(_part(k)[1] - _part(k)[0], device=DEV)) for k in SHAPES}  # noqa: E731
    segs, captured = new(), new()

    def step(s):
        for seg in s.values():
            seg.reset()
        y = _block(x, p, s)
        y.backward(R)
        return y.detach()

    step(captured)                                                           # what sets itself up on first use
    alive = _block(x, p, segs)                                               # not yet backward
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = step(captured)
    alive.backward(R)
    for _ in range(3):
        for seg in captured.values():
            seg.g.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = step(segs)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        for k in SHAPES:
            assert torch.equal(captured[k].g, segs[k].g), k
        x.mul_(0.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_expanded_gradients_inputs_and_residuals(dtype):
    """Rows that share their memory: the gradient behind a sum over the tokens, an input and a residual that are one row repeated,
    and a layer of one output, whose gradient behind a sum is one number repeated."""
    p = _params(18, dtype)
    dev = {k: v.to(DEV) for k, v in p.items()}
    x, R = _data(19, dtype, (1, 1))
    row, R = x[0], R[0, 0]
    xd = row.to(DEV).requires_grad_()
    y = _block(xd.expand(9, D), dev, {})
    (y.sum(0) * R.to(DEV)).sum().backward()
    ref_y, ref_dx, _ = _grads64(row, 9 * R, p)
    assert y.shape == (9, D) and _off(y[3], ref_y) <= BOUND[dtype]
    assert _off(xd.grad, ref_dx) <= 2 * BOUND[dtype]                       # nine equal rows summed in the type: eight roundings more
    W, b = dev["W1"][:1].contiguous(), dev["b1"][:1].contiguous()
    seg, bias_seg = (A.ChunkSegment(0, n, torch.empty(n, device=DEV)) for n in (D, 1))
    xs = torch.randn(40, D, generator=torch.Generator().manual_seed(20)).to(dtype)
    xd = xs.to(DEV).requires_grad_()
    A.chunk_linear(xd, W, seg, bias=b, bias_seg=bias_seg).sum().backward()
    assert torch.equal(xd.grad, W.expand(40, D)) and float(bias_seg.g) == 40.0
    assert _off(seg.g, xs.double().sum(0)) <= BOUND[dtype]
