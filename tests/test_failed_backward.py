"""A backward pass that fails and is repeated (no GPU: the library's calls are replaced by products of torch, the first of them, or an
allocation, fails): the repeated pass leaves the gradient that a pass without a failure leaves."""

import pytest
import torch

from paper_2605_21177_amd import autograd as A
from paper_2605_21177_amd import binding as B


class Library:
    """What the layers call, on the CPU; `fail` names the call that fails the next time."""

    def __init__(self, monkeypatch):
        self.fail, self.made = None, []
        for name in ("make_layer", "make_linear", "make_norm"):
            monkeypatch.setattr(B, name, getattr(self, name))
        for name in ("chunk_wgrad", "wgrad_adamw_fused", "muon_chunk", "adamw_chunk", "linear_forward", "linear_backward", "norm_forward", "norm_backward"):
            monkeypatch.setattr(B, "chunkft_" + name, self._call(name))
        for name in ("linear", "norm", "orthogonalize"):
            monkeypatch.setattr(B, f"chunkft_{name}_workspace_bytes", lambda *a, **k: 16)
        monkeypatch.setattr(A.ChunkSegment, "workspace", self._allocation("workspace", lambda seg, layer: None))
        monkeypatch.setattr(A, "_scratch", self._allocation("scratch", lambda need, device: None))

    def _failing(self, name, error):
        if self.fail == name:
            self.fail = None
            raise error
        self.made.append(name)

    def _call(self, name):
        def call(*a, **k):
            self._failing(name, B.ChunkFTError(B.ERR_HIP, name))
            return getattr(self, name)(*a, **k)
        return call

    def _allocation(self, name, then):
        def call(*a):
            self._failing(name, torch.OutOfMemoryError(name))
            return then(*a)
        return call

    def make_layer(self, kind, X, dY, out, n_in, split_k=0):
        return dict(X=X, dY=dY)

    def make_linear(self, X, W, bias=None, activation=0, residual=None, tokens=None):
        return dict(X=X, W=W, bias=bias)

    def make_norm(self, kind, X, w=None, b=None, eps=1e-5):
        return dict(X=X)

    def _into(self, g, value, accumulate):
        if g is not None:
            g.add_(value) if accumulate else g.copy_(value)

    def chunk_wgrad(self, layer, begin, end, g, accumulate=False, ws=None):
        self._into(g, (layer["dY"].t() @ layer["X"]).reshape(-1)[begin:end], accumulate)

    def wgrad_adamw_fused(self, layer, begin, end, W, master, m, v, hp, ws=None):
        m.add_((layer["dY"].t() @ layer["X"]).reshape(-1)[begin:end])

    def muon_chunk(self, g, master, m, W, rows, cols, hp, w_dtype=None, ws=None):
        m.add_(g)

    def adamw_chunk(self, g, master, m, v, W, n, hp, w_dtype=None):
        m.add_(g)

    def linear_forward(self, layer, Y, Z=None, ws=None):
        Y.copy_(layer["X"] @ layer["W"].t() + layer["bias"])

    def linear_backward(self, layer, dY, Z=None, dZ=None, dX=None, db=None, b_range=None, accumulate=False, ws=None):
        if dX is not None:
            dX.copy_(dY @ layer["W"])
        if db is not None:
            self._into(db, dY.sum(0)[b_range[0]:b_range[1]], accumulate)

    def norm_forward(self, layer, Y, stats):
        Y.copy_(layer["X"])

    def norm_backward(self, layer, stats, dY, dX, dw=None, w_range=None, db=None, b_range=None, accumulate=False, ws=None):
        for g, span, value in ((dw, w_range, (dY * layer["X"]).sum(0)), (db, b_range, dY.sum(0))):
            if g is not None:
                self._into(g, value[span[0]:span[1]], accumulate)


@pytest.fixture
def library(monkeypatch):
    return Library(monkeypatch)


T, IN, OUT = 5, 4, 6
ADAM = dict(hp=B.hparams(0.1, 0.9, 0.999, 1e-8, 0.0, 1))


def _segment(kind, begin, end):
    n = end - begin
    if kind == "plain":
        return A.ChunkSegment(begin, end, torch.full((n,), 77.0))
    state = dict(master=torch.zeros(n), m=torch.zeros(n))
    return A.ChunkSegment(begin, end, **state, **(dict(hp=B.muon_hparams(0.1)) if kind == "muon" else dict(v=torch.zeros(n), **ADAM)))


def _result(seg):
    return seg.m if seg.fused else seg.g


def _data(seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(T, IN, generator=gen), torch.randn(OUT, IN, generator=gen), torch.randn(OUT, generator=gen), torch.randn(T, OUT, generator=gen)


def _twice(library, step, failing, segs):
    """One pass that fails (with everything as it was), then the same pass."""
    library.fail = failing
    before = [_result(s).clone() for s in segs], [s.micro_batches for s in segs]
    with pytest.raises((torch.OutOfMemoryError, B.ChunkFTError)):
        step()
    assert library.fail is None
    assert [s.micro_batches for s in segs] == before[1]
    assert all(torch.equal(_result(s), b) for s, b in zip(segs, before[0]))
    step()


@pytest.mark.parametrize("kind,failing", [("plain", "workspace"), ("plain", "chunk_wgrad"), ("adam", "workspace"), ("adam", "wgrad_adamw_fused"),
                                          ("muon", "workspace"), ("muon", "scratch"), ("muon", "chunk_wgrad"), ("muon", "muon_chunk")])
def test_products_of_torch(library, kind, failing):
    x, W, _, R = _data(1)
    seg = _segment(kind, IN, 3 * IN)
    step = lambda: (A.chunk_linear(x.requires_grad_(), W, seg) * R).sum().backward()  # noqa: E731
    want = (R.t() @ x.detach()).reshape(-1)[IN:3 * IN]
    _twice(library, step, failing, [seg])
    assert seg.micro_batches == 1 and torch.allclose(_result(seg), want)
    if kind == "plain":                                       # the second micro-batch, with a failure too, adds to the first
        _twice(library, step, failing, [seg])
        assert seg.micro_batches == 2 and torch.allclose(seg.g, 2 * want)
    else:
        with pytest.raises(RuntimeError, match="one micro-batch"):
            step()


@pytest.mark.parametrize("bias_kind", ["plain", "adam"])
@pytest.mark.parametrize("kind,failing", [("plain", "workspace"), ("adam", "workspace"), ("muon", "workspace"), ("muon", "scratch"), ("plain", "linear_backward")])
def test_bias_and_weight_of_a_layer(library, kind, bias_kind, failing):
    """The weight's allocations fail before the bias has been touched."""
    x, W, b, R = _data(2)
    seg, bias_seg = _segment(kind, 0, 2 * IN), _segment(bias_kind, 1, 5)
    step = lambda: (A.chunk_linear(x, W, seg, bias=b, bias_seg=bias_seg) * R).sum().backward()  # noqa: E731
    if failing == "scratch":
        inner = step

        def step():
            # the forward pass has a workspace of its own: the failure is the backward pass's
            f, library.fail = library.fail, None
            y = (A.chunk_linear(x, W, seg, bias=b, bias_seg=bias_seg) * R).sum()
            library.fail = f
            y.backward()
    _twice(library, step, failing, [seg, bias_seg])
    assert torch.allclose(_result(seg), (R.t() @ x).reshape(-1)[:2 * IN]) and torch.allclose(_result(bias_seg), R.sum(0)[1:5])
    assert seg.micro_batches == bias_seg.micro_batches == 1


def test_second_micro_batch_of_a_layer(library):
    x, W, b, R = _data(3)
    seg, bias_seg = _segment("plain", 0, 2 * IN), _segment("plain", 0, OUT)
    step = lambda: (A.chunk_linear(x, W, seg, bias=b, bias_seg=bias_seg) * R).sum().backward()  # noqa: E731
    step()
    _twice(library, step, "workspace", [seg, bias_seg])
    assert torch.allclose(seg.g, 2 * (R.t() @ x).reshape(-1)[:2 * IN]) and torch.allclose(bias_seg.g, 2 * R.sum(0))


@pytest.mark.parametrize("failing", ["norm_backward", "scratch"])
def test_norm(library, failing):
    x, _, _, _ = _data(4)
    w, b, R = torch.ones(IN), torch.zeros(IN), torch.randn(T, IN, generator=torch.Generator().manual_seed(5))
    seg, bias_seg = _segment("plain", 0, 3), _segment("adam", 1, 4)
    step = lambda: (A.chunk_norm(x, w, b, B.LAYERNORM, seg=seg, bias_seg=bias_seg) * R).sum().backward()  # noqa: E731
    _twice(library, step, failing, [seg, bias_seg])
    assert torch.allclose(seg.g, (R * x).sum(0)[:3]) and torch.allclose(bias_seg.m, R.sum(0)[1:4])


def test_an_update_that_is_refused_is_not_counted(library):
    x, _, _, _ = _data(6)
    w, seg = torch.ones(IN), _segment("adam", 0, IN)
    step = lambda: A.chunk_norm(x, w, seg=seg).sum().backward()  # noqa: E731
    _twice(library, step, "adamw_chunk", [seg])
    assert seg.micro_batches == 1 and torch.allclose(seg.m, x.sum(0))


@pytest.mark.parametrize("kind,failing", [("plain", "chunk_wgrad"), ("adam", "wgrad_adamw_fused"), ("muon", "muon_chunk")])
def test_a_refused_weight_gradient_leaves_the_bias_to_be_written_again(library, kind, failing):
    x, W, b, R = _data(7)
    seg, bias_seg = _segment(kind, 0, 2 * IN), _segment("plain", 0, OUT)
    step = lambda: (A.chunk_linear(x, W, seg, bias=b, bias_seg=bias_seg) * R).sum().backward()  # noqa: E731
    library.fail = failing
    with pytest.raises(B.ChunkFTError):
        step()
    assert seg.micro_batches == bias_seg.micro_batches == 0
    step()
    assert torch.allclose(_result(seg), (R.t() @ x).reshape(-1)[:2 * IN]) and torch.allclose(bias_seg.g, R.sum(0))


@pytest.mark.parametrize("fused_first", [True, False])
def test_a_refused_update_of_one_vector_leaves_the_other_to_be_written_again(library, fused_first):
    x, _, _, _ = _data(8)
    w, b, R = torch.ones(IN), torch.zeros(IN), torch.randn(T, IN, generator=torch.Generator().manual_seed(9))
    segs = [_segment("adam", 0, IN), _segment("plain", 0, IN)]
    seg, bias_seg = segs if fused_first else segs[::-1]
    step = lambda: (A.chunk_norm(x, w, b, B.LAYERNORM, seg=seg, bias_seg=bias_seg) * R).sum().backward()  # noqa: E731
    library.fail = "adamw_chunk"
    with pytest.raises(B.ChunkFTError):
        step()
    assert seg.micro_batches == bias_seg.micro_batches == 0
    step()
    assert torch.allclose(_result(seg), (R * x).sum(0)) and torch.allclose(_result(bias_seg), R.sum(0))
