"""What the gated-delta layer's Python wrappers do with tensors beyond their numbers."""
import pytest
import torch

from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _calls():
    """Every wrapper, as (function, tensor arguments, others)."""
    g = torch.Generator(device=DEV).manual_seed(1)

    def r(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    gates = -r(2, 5, 2).abs(), r(2, 5, 2).sigmoid()
    slots = torch.tensor([1, 0], dtype=torch.int32, device=DEV)
    return [
        (P.delta, (r(2, 5, 1, 8), r(2, 5, 1, 8), r(2, 5, 2, 8)) + gates + (r(2, 2, 8, 8),), {}),
        (P.delta_step, (r(2, 1, 8), r(2, 1, 8), r(2, 2, 8), gates[0][:, 0].contiguous(),
                        gates[1][:, 0].contiguous(), r(3, 2, 8, 8)), dict(slots=slots)),
        (P.conv, (r(2, 5, 16), r(16, 4), r(16), r(2, 3, 16)), {}),
        (P.conv_step, (r(2, 16), r(16, 4), r(16), r(3, 3, 16)), dict(slots=slots)),
        (P.score_tokens, (r(4, 100),), dict(top=3))]


@pytest.mark.parametrize("which", range(5))
def test_a_gradient_that_would_be_lost_is_refused(which):
    fn, tensors, kw = _calls()[which]
    for i in range(len(tensors)):
        args = [t.clone().requires_grad_(j == i) for j, t in enumerate(tensors)]
        with pytest.raises(ValueError, match="no backward pass"):
            fn(*args, **kw)
        with torch.no_grad():
            out = fn(*args, **kw)
        ref = fn(*[t.clone() for t in tensors], **kw)
        for a, b in zip(out if isinstance(out, tuple) else (out,), ref if isinstance(ref, tuple) else (ref,)):
            assert (a is None and b is None) or (torch.equal(a, b) and not a.requires_grad)
