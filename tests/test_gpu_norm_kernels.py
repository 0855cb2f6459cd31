"""Every shape of the norm's kernels, by the number of 16-byte vectors in a row
(each range between two powers of two has a shape of its own at most), with as
many rows as give every work-group several turns; and the calls in place."""
import pytest
import torch

from paper_2412_00119_amd import bmlp as B
from paper_2412_00119_amd import dense as D

from gpu_common import note
from test_gpu_dense import BF16, EPS32, F16, F32, HALF_STEP, SMALLEST, check_norm, gen, norm_back_ref, rows

pytestmark = pytest.mark.gpu

VEC = {F32: 4, BF16: 8, F16: 8}
# vectors of a row -> rows that a work-group of the backward takes at a time, at most
RANGES = {50: 16, 64: 16, 100: 8, 128: 8, 200: 4, 256: 4, 400: 2, 512: 2, 700: 1, 1024: 1, 1500: 1, 2048: 1, 3000: 1, 4096: 1,
          6000: 1, 8192: 1, 12000: 1, 16384: 1}

SHAPES = [(t, v) for t in VEC for v in sorted(RANGES) if v * VEC[t] <= 65536]


def width(dtype, vecs, cut):
    """A row of that many vectors, the last one short by `cut` elements."""
    return vecs * VEC[dtype] - cut


@pytest.mark.parametrize("dtype,vecs", SHAPES)
@pytest.mark.parametrize("cut", [0, 3])
def test_forward_shapes(dtype, vecs, cut):
    k = width(dtype, vecs, cut)
    note(f"norm {dtype} 5x{k}")
    g = gen(vecs + cut)
    x, r = torch.randn(5, k, generator=g).to(dtype), torch.randn(5, k, generator=g).to(dtype)
    w = (1 + 0.3 * torch.randn(k, generator=g)).to(dtype if cut else F32)
    check_norm(x, w, r, 1e-6, D.norm_quant(rows(x, cut), w.cuda(), rows(r), 1e-6, values=True))


@pytest.mark.parametrize("dtype,vecs", SHAPES)
@pytest.mark.parametrize("cut", [0, 3])
def test_gradient_shapes(dtype, vecs, cut):
    """Three turns and a part of one for every work-group (256 of them at most).  A row's sum: at most 64 elements a thread,
    6 joins, 16 waves and 4 roundings a term; a column's: 4 rows, 16 of a work-group, 16 partial sums and 16 waves, and 3
    a term: below 160 eps of the sums of magnitudes, plus one rounding to the type.  The 64-bit formula runs on the GPU."""
    k = width(dtype, vecs, cut)
    n = 3 * 256 * RANGES[vecs] + 5 * RANGES[vecs] + 1
    note(f"norm gradient {dtype} {n}x{k}")
    g = torch.Generator(device="cuda").manual_seed(vecs + cut)
    make = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    h, dy, dh = (make(n, k).to(dtype) for _ in range(3))
    w = (1 + 0.3 * make(k)).to(dtype if cut else F32)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    for add in (dh, None):
        dx, dw = D.norm_quant_backward(dy, h, rstd, w, add)
        step = max(1, (1 << 25) // k)
        sum_dw, sum_size = torch.zeros(k, dtype=torch.float64, device="cuda"), torch.zeros(k, dtype=torch.float64, device="cuda")
        for a in range(0, n, step):
            part = slice(a, a + step)
            want, size, wdw, wsize = norm_back_ref(dy[part], h[part], rstd[part], w, None if add is None else add[part])
            bound = 160 * EPS32 * size + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype]
            assert ((dx[part].double() - want).abs() <= bound).all(), a
            sum_dw += wdw
            sum_size += wsize
        assert ((dw.double() - sum_dw).abs() <= 160 * EPS32 * sum_size).all()


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k", [(5, 3), (20, 77), (3000, 130), (600, 2051), (600, 4099), (600, 9001), (520, 20003), (260, 40001)])
def test_gradient_in_place(dtype, n, k):
    """dx over dy, and over dh: the same bits as into a matrix of its own."""
    note(f"norm gradient in place {dtype} {n}x{k}")
    g = torch.Generator(device="cuda").manual_seed(k)
    h, dy, dh = (torch.randn((n, k), generator=g, device="cuda").to(dtype) for _ in range(3))
    w = torch.randn(k, generator=g, device="cuda")
    rstd = torch.rand(n, generator=g, device="cuda") + 0.5
    want, want_dw = D.norm_quant_backward(dy, h, rstd, w, dh)
    size = B.lib().bmlp_norm_quant_backward_workspace_bytes(n, k)
    ws, code = torch.empty(size, dtype=torch.uint8, device="cuda"), D.TYPES[dtype]
    for over in ("dy", "dh"):
        t = {"dy": dy.clone(), "dh": dh.clone()}
        dw = torch.empty(k, device="cuda")
        st = B.lib().bmlp_norm_quant_backward(code, n, k, t["dy"].data_ptr(), k, h.data_ptr(), k, rstd.data_ptr(), w.data_ptr(), 0,
                                              t["dh"].data_ptr(), k, t[over].data_ptr(), k, dw.data_ptr(), ws.data_ptr(), size,
                                              stream())
        assert st == 0
        assert torch.equal(t[over], want) and torch.equal(dw, want_dw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [3, 77, 513, 2051, 4099, 9001, 20003, 40001])
@pytest.mark.parametrize("over", ["x", "residual"])
def test_forward_in_place(dtype, k, over):
    """The sum written over x or over the residual: the same bits as into a matrix of its own."""
    n = 300
    note(f"norm over {over} {dtype} {n}x{k}")
    g = torch.Generator(device="cuda").manual_seed(k)
    x, r = (torch.randn((n, k), generator=g, device="cuda").to(dtype) for _ in range(2))
    want = D.norm_quant(x, None, r)
    q, sc = torch.empty_like(want.q), torch.empty_like(want.scale)
    h = x if over == "x" else r
    st = B.lib().bmlp_norm_quant(D.TYPES[dtype], n, k, x.data_ptr(), k, r.data_ptr(), k, None, 0, 1e-6, q.data_ptr(), k,
                                 sc.data_ptr(), None, h.data_ptr(), k, None, 0, stream())
    assert st == 0
    assert torch.equal(h, want.h) and torch.equal(q, want.q) and torch.equal(sc, want.scale)
