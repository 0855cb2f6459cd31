"""The dense operators record nothing for autograd: a tensor that requires a
gradient, or carries a forward-mode tangent, is refused instead of losing it.
The refusal comes first of all checks, so most of it needs no GPU."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2412_00119_amd import dense as D

X = torch.ones(4, 8)
V, R = torch.ones(8), torch.ones(4)
IDX = torch.zeros((4, 1), dtype=torch.int32)

CALLS = {
    "norm x": (X, lambda t: D.norm_quant(t, V, X)),
    "norm weight": (V, lambda t: D.norm_quant(X, t, X)),
    "norm residual": (X, lambda t: D.norm_quant(X, V, t)),
    "rows x": (X, lambda t: D.quantize_rows(t)),
    "backward dy": (X, lambda t: D.norm_quant_backward(t, X, R, V, X)),
    "backward h": (X, lambda t: D.norm_quant_backward(X, t, R, V, X)),
    "backward rstd": (R, lambda t: D.norm_quant_backward(X, X, t, V, X)),
    "backward weight": (V, lambda t: D.norm_quant_backward(X, X, R, t, X)),
    "backward dh": (X, lambda t: D.norm_quant_backward(X, X, R, V, t)),
    "distill z": (X, lambda t: D.distill(t, IDX, X[:, :1], 1.0, R, R)),
    "distill t": (X[:, :1], lambda t: D.distill(X, IDX, t, 1.0, R, R)),
    "distill lse": (R, lambda t: D.distill(X, IDX, X[:, :1], 1.0, t, R)),
    "distill weight": (R, lambda t: D.distill(X, IDX, X[:, :1], 1.0, R, t)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused_while_gradients_are_recorded(name):
    t, call = CALLS[name]
    t = t.clone().requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        call(t)
    with torch.no_grad(), pytest.raises(ValueError) as e:   # as far as the next check: nothing here is on the GPU
        call(t)
    assert "gradient" not in str(e.value)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tangents_are_refused(name):
    t, call = CALLS[name]
    with fwd.dual_level():
        dual = fwd.make_dual(t.clone(), torch.ones_like(t))
        with pytest.raises(ValueError, match="requires a gradient"):
            call(dual)


@pytest.mark.gpu
def test_layer_row_scale_is_refused():
    layer = D.QLinear(torch.ones((5, 8), dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"))
    q, scale = torch.ones((2, 8), dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="requires a gradient"):
        layer(q, scale)
    with torch.no_grad():
        assert (layer(q, scale) == 8).all()


@pytest.mark.gpu
def test_layer_from_parameters_is_made_of_constants():
    w = torch.nn.Parameter(torch.randn(5, 8, generator=torch.Generator().manual_seed(0)).cuda())
    bias = torch.nn.Parameter(torch.ones(5, device="cuda"))
    layer = D.QLinear.from_weight(w, bias)
    assert not layer.scale.requires_grad and not layer.bias.requires_grad
    q = torch.ones((2, 8), dtype=torch.int8, device="cuda")
    same = D.QLinear(*D.quantize_rows(w.detach()), bias.detach())
    assert torch.equal(layer(q), same(q)) and not layer(q).requires_grad


@pytest.mark.gpu
def test_chained_by_hand():
    """What the message says: the gradient of detached logits, given back to them.  dz is within 512 roundings
    (test_gpu_dense.check_distill), and a gradient of the head adds four of them times |a| <= 4."""
    g = torch.Generator().manual_seed(1)
    a, head = torch.randn(4, 8, generator=g).clamp(-4, 4), torch.randn(8, 6, generator=g)
    idx, t = torch.tensor([[1, 2]] * 4, dtype=torch.int32), torch.randn(4, 2, generator=g)
    on_gpu = head.cuda().requires_grad_()
    logits = a.cuda() @ on_gpu
    logits.backward(D.distill(logits.detach(), idx.cuda(), t.cuda())[1])
    want = head.double().requires_grad_()
    p = torch.zeros(4, 6, dtype=torch.float64).scatter(1, idx.long(), torch.softmax(t.double(), 1))
    (-p * torch.log_softmax(a.double() @ want, 1)).sum().backward()
    assert ((on_gpu.grad.cpu().double() - want.grad).abs() <= 4 * 4 * 512 * 2.0 ** -24).all()


def test_layer_of_what_is_no_tensor():
    w = torch.ones((4, 8), dtype=torch.int8)
    for call in (lambda: D.QLinear(w, None), lambda: D.QLinear(None, R), lambda: D.QLinear(w, 1.0), lambda: D.QLinear.from_weight(None),
                 lambda: D.QLinear.from_weight([[1.0]])):
        with pytest.raises((TypeError, ValueError)):   # (ValueError: w is not on the GPU)
            call()
