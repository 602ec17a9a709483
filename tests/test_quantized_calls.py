"""Calls on a relayed cache held in 8 or 4 bits: what they refuse."""
import pytest
import torch

import paper_2604_13349_b200 as P


# ---- gradients ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
def test_scales_that_require_a_gradient_are_refused(bits, which):
    host = P.quantized_cache(1, 2, 10, 64, bits, device="cpu")
    leaf = host._replace(**{which: getattr(host, which).clone().requires_grad_()})
    x = torch.zeros(1, 2, 3, 64)
    for call in (lambda: P.attend_quantized(x, leaf), lambda: P.read_quantized(leaf), lambda: P.write_quantized(leaf, x, x)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on a device"):        # the next check: tensors of the host
            call()
