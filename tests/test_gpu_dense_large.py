"""More work than the 2^32 threads that a launch may hold: it is spread over
several launches."""
import pytest
import torch

from paper_2412_00119_amd import dense as D

from gpu_common import note

pytestmark = pytest.mark.gpu


def test_more_outputs_than_a_launch_takes():
    """2^30 + 33 outputs of one input: the packed weights (64 bytes an output, 69 GB) have more 16-byte chunks, and the
    product more tiles times threads, than one launch takes.  Compared whole, to the last bit."""
    n, m = 3, 2 ** 30 + 33
    note(f"product {n}x1x{m}")
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randint(-128, 128, (m, 1), generator=g, device="cuda", dtype=torch.int8)
    ws, bias = torch.rand(m, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    q, scale = torch.tensor([[3], [-128], [127]], dtype=torch.int8, device="cuda"), torch.tensor([0.5, 0.3, 2.0], device="cuda")
    layer = D.QLinear(w, ws, bias)
    out = layer(q, scale, torch.float32)
    del layer.packed
    for a in range(0, m, 2 ** 27):
        b = min(a + 2 ** 27, m)
        for i in range(n):
            want = w[a:b, 0].float() * float(q[i, 0]) * scale[i] * ws[a:b] + bias[a:b]
            assert torch.equal(out[i, a:b], want)
        note(f"columns up to {b} of {m}")
    del layer, out, w, ws, bias, want
    torch.cuda.empty_cache()
