"""Rows of logits and of their gradient that alternate in memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, V, gap", [(7, 100, 0), (5, 3000, 1), (300, 3000, 0), (2, 40000, 3)])
def test_halves_of_wider_rows(rows, V, gap):
    """Logits before or behind their gradient in one buffer, and one above the other: the bits of separate buffers on the same grid."""
    import paper_1708_02983_amd as hip
    gen = torch.Generator(device="cuda").manual_seed(V)
    width = (2 * V + gap + 7) // 4 * 4
    idx = torch.randint(0, V, (rows, 9), generator=gen, device="cuda", dtype=torch.int32)
    val = torch.randn(rows, 9, generator=gen, device="cuda")
    logits = torch.randn(rows, V, generator=gen, device="cuda")
    for at, to in ((0, V + gap), (V + gap, 0)):
        alone = torch.empty(rows, width, device="cuda")
        alone[:, at:at + V] = logits
        loss, grad = hip.easgd_distill(alone[:, at:at + V], idx, val)
        buf = torch.full((rows, width), 3.0, device="cuda")
        buf[:, at:at + V] = logits
        l, _ = hip.easgd_distill(buf[:, at:at + V], idx, val, dlogits=buf[:, to:to + V])
        assert torch.equal(l, loss) and torch.equal(buf[:, to:to + V], grad) and torch.equal(buf[:, at:at + V], logits)
        both = torch.full((2 * rows, V), 3.0, device="cuda")
        both[:rows] = logits
        l, _ = hip.easgd_distill(both[:rows], idx, val, dlogits=both[rows:])
        assert torch.allclose(l, loss, rtol=1e-5) and torch.allclose(both[rows:], grad, atol=1e-6) and torch.equal(both[:rows], logits)
