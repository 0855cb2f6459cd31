"""A layer's tensors are attributes that a program can replace: one that fits is
used, one that does not is refused on the host, before anything is launched."""
import pytest
import torch

from paper_2412_00119_amd import dense as D

pytestmark = pytest.mark.gpu

N, K = 40, 100


def make():
    g = torch.Generator().manual_seed(1)
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8).cuda()
    q = torch.randint(-128, 128, (3, K), generator=g, dtype=torch.int8).cuda()
    return D.QLinear(w, torch.ones(N, device="cuda"), torch.zeros(N, device="cuda")), w, q


BAD = {
    "scale-short": ("scale", lambda t: torch.ones(N - 1, device="cuda")),
    "scale-long-within-the-padding": ("scale", lambda t: torch.ones(64, device="cuda")),
    "scale-long": ("scale", lambda t: torch.ones(1000, device="cuda")),
    "scale-bf16": ("scale", lambda t: t.bfloat16()),
    "scale-cpu": ("scale", lambda t: t.cpu()),
    "scale-strided": ("scale", lambda t: torch.ones(2 * N, device="cuda")[::2]),
    "scale-none": ("scale", lambda t: None),
    "bias-short": ("bias", lambda t: torch.ones(1, device="cuda")),
    "bias-f16": ("bias", lambda t: t.half()),
    "bias-cpu": ("bias", lambda t: t.cpu()),
    "bias-matrix": ("bias", lambda t: t[None, :]),
    "packed-short": ("packed", lambda t: t[:-1]),
    "packed-empty": ("packed", lambda t: t[:0]),
    "packed-int8": ("packed", lambda t: t.view(torch.int8)),
    "packed-cpu": ("packed", lambda t: t.cpu()),
    "packed-strided": ("packed", lambda t: torch.stack([t, t], 1)[:, 0]),
    "packed-none": ("packed", lambda t: None),
    "more-inputs": ("n_in", lambda v: 129),
    "more-outputs": ("n_out", lambda v: 65),
    "no-outputs": ("n_out", lambda v: 0),
    "negative-outputs": ("n_out", lambda v: -1),
    "outputs-past-32-bits": ("n_out", lambda v: 2 ** 32 + N),
}


@pytest.mark.parametrize("case", sorted(BAD))
def test_layer_refuses_a_tensor_that_does_not_fit(case):
    layer, _, q = make()
    name, change = BAD[case]
    setattr(layer, name, change(getattr(layer, name)))
    with pytest.raises((ValueError, TypeError)):
        layer(q, None, torch.float32)


def test_layer_uses_a_tensor_that_fits():
    layer, w, q = make()
    whole = (q.cpu().long() @ w.cpu().long().t()).float()
    layer.scale, layer.bias = torch.full((N,), 2.0, device="cuda"), torch.full((N,), 3.0, device="cuda")
    assert torch.equal(layer(q, None, torch.float32).cpu(), whole * 2 + 3)
    layer.bias = None
    layer.packed = D.QLinear(w.flip(0), layer.scale).packed
    assert torch.equal(layer(q, None, torch.float32).cpu(), whole.flip(1) * 2)
