"""The norm's statistics where squares leave the 32-bit range: rows far below 1
with an eps below their mean square, and rows of zeros with eps = 0."""
import pytest
import torch

from paper_2412_00119_amd import dense as D

from gpu_common import note
from test_gpu_dense import BF16, EPS32, F16, F32, check_norm, gen, rows

pytestmark = pytest.mark.gpu

# the rows' sizes: the squares of the first ones are below 2^-149 or subnormal, or become so when divided by K
POWERS = (-116, -110, -101, -90, -80, -76, -74, -70, -66, -63, -62, -60, -56, -51, -50, -49, -48, -40, -20, 0, 40, 60)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 1e-38, 1e-33, 2.0 ** -101, 2.0 ** -100, 1e-25])
@pytest.mark.parametrize("k", [5, 700, 4096, 65536])
def test_small_rows(dtype, eps, k):
    """Within the bounds of check_norm: what a square may lose to the range's end (2^-150 of a sum that is above 2^-101, up
    to 2^16 times: 2^-33) is far below its roundings."""
    note(f"small rows {dtype} eps {eps} {k}")
    g = gen(k)
    size = torch.tensor([2.0 ** p for p in POWERS], dtype=torch.float32)[:, None]
    n = len(POWERS)
    x = (torch.randn(n, k, generator=g).clamp(-8, 8) * size).to(dtype)
    x[:, 0] = (1.5 * size[:, 0]).to(dtype)            # no row smaller than its size by chance
    r = (torch.randn(n, k, generator=g).clamp(-8, 8) * size).to(dtype)
    r[:, 0] = 0
    w = 1 + 0.3 * torch.rand(k, generator=g)
    check_norm(x, w, r, eps, D.norm_quant(rows(x), w.cuda(), rows(r), eps, values=True))
    check_norm(x, None, None, eps, D.norm_quant(rows(x), None, None, eps, values=True))


@pytest.mark.parametrize("k", [16384, 65536])
def test_constant_small_rows(k):
    """Constant rows, for which every square is lost alike: 1.3e-19 (its square is a normal number), 2e-20 and 1e-21."""
    x = torch.tensor([1.3e-19, 2e-20, 1e-21, 1e-30])[:, None].expand(4, k).contiguous()
    got = D.norm_quant(x.cuda(), None, None, 0.0, values=True)
    check_norm(x, None, None, 0.0, got)
    torch.testing.assert_close(got.y.cpu(), torch.ones(4, k), rtol=100 * EPS32, atol=0)
    assert (got.q == 127).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("k", [7, 300, 5000])
def test_zero_rows_without_eps(dtype, k):
    """A row of zeros at eps = 0: everything of it is 0, and its gradient adds nothing to dweight."""
    note(f"zero rows {dtype} {k}")
    g = gen(k)
    x, dy, dh = (torch.randn(6, k, generator=g).to(dtype) for _ in range(3))
    x[1], x[4] = 0, 0
    w = (1 + 0.3 * torch.rand(k, generator=g)).to(dtype)
    got = D.norm_quant(x.cuda(), w.cuda(), None, 0.0, values=True)
    for i in (1, 4):
        assert got.rstd[i] == 0 and got.scale[i] == 0 and (got.q[i] == 0).all() and (got.y[i] == 0).all()
    keep = [0, 2, 3, 5]
    check_norm(x[keep], w, None, 0.0, D.NormQuant(*(None if v is None else v[keep] for v in got)))
    for add in (None, dh.cuda()):
        dx, dw = D.norm_quant_backward(dy.cuda(), x.cuda(), got.rstd, w.cuda(), add)
        want = dy[keep].cuda(), x[keep].cuda(), got.rstd[keep]
        kx, kw = D.norm_quant_backward(*want, w.cuda(), None if add is None else add[keep])
        assert torch.equal(dx[keep], kx) and kx.isfinite().all()
        assert torch.equal(dx[[1, 4]], torch.zeros_like(dx[:2]) if add is None else add[[1, 4]])
        terms = dy[keep].double() * x[keep].double() * got.rstd[keep].double().cpu()[:, None]
        assert ((dw.double().cpu() - terms.sum(0)).abs() <= 8 * EPS32 * terms.abs().sum(0)).all()


def test_rows_below_the_smallest_root_mean_square():
    """At or below 2^-118, with eps = 0: rstd = 0 and scale = 0, as above the squares' range (where the last row's t is not
    finite either, so that its scale is NaN)."""
    x = torch.tensor([2.0 ** -125, 2.0 ** -119, 2.0 ** -117, 2.0 ** 127])[:, None].expand(4, 64).contiguous()
    w = torch.full((64,), 2.0 ** 20)
    got = D.norm_quant(x.cuda(), w.cuda(), None, 0.0, values=True)
    assert (got.rstd[[0, 1, 3]] == 0).all() and (got.scale[:2] == 0).all() and (got.y[:2] == 0).all()
    assert got.scale[3].isnan() and got.y[3].isnan().all() and (got.q[3] == 0).all()
    assert got.rstd[2] == 2.0 ** 117 and (got.y[2] - 2.0 ** 20).abs().max() <= 3 * EPS32 * 2.0 ** 20
