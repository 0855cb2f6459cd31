"""Every kernel of the 8-bit product on random bytes, equal to the last bit."""
import pytest
import torch

from paper_2412_00119_amd import dense as D

from gpu_common import note
from product_shapes import ALIGNED, RAGGED
from test_gpu_dense import BF16, F16, F32, gen, int8, product_ref, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,m,k,pad,lead", ALIGNED + RAGGED)
def test_kernels(n, m, k, pad, lead):
    note(f"product {n}x{k}+{pad}x{m} from {lead}")
    g = gen(n + 3 * m + 7 * k + lead)
    q, w = int8(g, n, k), int8(g, m, k)
    scale, ws, bias = torch.rand(n, generator=g) + 0.1, (torch.rand(m, generator=g) + 0.1) / 100, torch.randn(m, generator=g)
    dq, dscale = rows(q, pad, lead), scale.cuda()
    assert dq.data_ptr() % 16 == lead % 16
    layer, plain = D.QLinear(w.cuda(), ws.cuda(), bias.cuda()), D.QLinear(w.cuda(), ws.cuda())
    whole = product_ref(q, w, None, torch.ones(m), None, F32)   # exact; the scales and the bias are applied below
    one = whole * scale[:, None] * ws[None, :]
    assert torch.equal(layer(dq, dscale, F32).cpu(), one + bias[None, :])
    assert torch.equal(layer(dq, dscale, BF16).cpu(), (one + bias[None, :]).to(BF16))
    assert torch.equal(plain(dq, dscale, F16).cpu(), one.to(F16))
    assert torch.equal(plain(dq, None, BF16).cpu(), (whole * ws[None, :]).to(BF16))


@pytest.mark.parametrize("n,m", [(3001, 2999), (1003, 4107), (523, 4101), (2047, 1021), (20, 8200)])
@pytest.mark.parametrize("k,lead", [(336, 0), (333, 1)])
def test_kernels_write_nothing_else(n, m, k, lead):
    """Outputs with wider rows: what lies between and behind them stays."""
    from paper_2412_00119_amd import bmlp as B
    note(f"product {n}x{k}x{m}, wide rows")
    g = gen(n + k)
    q, w = rows(int8(g, n, k), 0, lead), int8(g, m, k).cuda()
    layer, ldo = D.QLinear(w, torch.ones(m, device="cuda")), m + 7
    want = layer(q, None, F32)
    out = torch.full((n + 1, ldo), 5.0, device="cuda")
    st = B.lib().bmlp_qlinear(0, n, m, k, q.data_ptr(), k, None, layer.packed.data_ptr(), layer.scale.data_ptr(), None,
                              out.data_ptr(), ldo, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert torch.equal(out[:n, :m], want) and (out[:n, m:] == 5).all() and (out[n] == 5).all()
