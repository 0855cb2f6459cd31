"""The distillation without a gradient, with a teacher's logits in every type, and
with padding entries, whose row has no looser bound anywhere."""
import pytest
import torch

from paper_2412_00119_amd import dense as D

from gpu_common import note
from test_gpu_dense import BF16, CLASSES, EPS32, F16, F32, HALF_STEP, SMALLEST, check_distill, distill_ref, gen, sample

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,c,k", CLASSES)
def test_loss_only(n, c, k, dtype, rest):
    """The loss is within check_distill's bound, and the bits are those of the call with a gradient."""
    note(f"loss only {n}x{c} top {k} {dtype} rest={rest}")
    z, idx, t, lse = sample(n, c, k, dtype, n + c + k, rest)
    w = torch.rand(n, generator=gen(c)) + 0.5 if c % 2 else None
    args = z.cuda(), idx.cuda(), t.cuda(), 1.0, None if lse is None else lse.cuda(), None if w is None else w.cuda()
    loss, none = D.distill(*args, grad=False)
    assert none is None
    check_distill(z, idx, t, 1.0, lse, w, (loss, None))
    assert torch.equal(loss, D.distill(*args)[0])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("t_dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,c,k", [(5, 100, 7), (3, 1027, 64), (2, 3001, 65), (2, 6002, 9), (2, 12003, 300), (2, 30001, 64),
                                   (1, 60007, 33), (1, 140001, 100)])
def test_teacher_types(n, c, k, dtype, t_dtype):
    note(f"distill {n}x{c} top {k} {dtype}, teacher {t_dtype}")
    z, idx, t, lse = sample(n, c, k, dtype, c, True)
    check_distill(z, idx, t.to(t_dtype), 1.0, lse)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,c,k", [(6, 40, 8), (5, 1001, 70), (4, 5000, 30), (3, 33333, 64)])
def test_padding_entries(n, c, k, dtype, rest):
    """check_distill's bound, with the error of p allowed only at classes that are listed."""
    note(f"padding {n}x{c} top {k} {dtype} rest={rest}")
    z, idx, t, lse = sample(n, c, k, dtype, c + k, rest)
    idx[0, 1:] = -1
    idx[1, ::2] = -1
    idx[2, k // 2:] = c + 5
    if rest:
        ent = torch.where((idx >= 0) & (idx < c), t, torch.full_like(t, -float("inf")))
        lse = torch.logsumexp(ent, 1) + 0.3
    loss, dz = D.distill(z.cuda(), idx.cuda(), t.cuda(), 1.0, None if lse is None else lse.cuda())
    want, grad = distill_ref(z, idx, t, 1.0, lse)
    tol = 512 * EPS32
    assert ((loss.cpu().double() - want).abs() <= tol * 64).all()
    bound = tol * torch.softmax(z.double(), 1) + HALF_STEP[dtype] * grad.abs() + SMALLEST[dtype]
    for i in range(n):
        for v in idx[i].tolist():
            if 0 <= v < c:
                bound[i, v] += tol
    assert ((dz.cpu().double() - grad).abs() <= bound).all()
