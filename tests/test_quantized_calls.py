"""Calls on a relayed cache held in 8 or 4 bits: what they refuse."""
import pytest
import torch

import paper_2604_13349_b200 as P

BF16 = torch.bfloat16


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


# ---- outputs ---------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_outputs_of_another_number_of_dimensions_are_refused():
    cache = P.quantized_cache(1, 2, 10, 64)
    q = torch.zeros(1, 2, 3, 64, dtype=BF16, device="cuda")
    for out in (torch.zeros(2, 3, 64, dtype=BF16, device="cuda"), torch.zeros(64, dtype=BF16, device="cuda"), torch.zeros((), dtype=BF16, device="cuda"),
                torch.zeros(1, 1, 2, 3, 64, dtype=BF16, device="cuda")):
        with pytest.raises(ValueError, match="out"):
            P.attend_quantized(q, cache, out=out)
        with pytest.raises(ValueError, match="k_out"):
            P.read_quantized(cache, k_out=out, v_out=out)
        with pytest.raises(ValueError, match="k_values"):
            P.write_quantized(cache, q, q, k_values=out, v_values=out)
    for name in ("k", "v", "k_scale", "v_scale"):
        with pytest.raises(ValueError, match="cache"):
            P.read_quantized(cache._replace(**{name: getattr(cache, name)[0]}))
        with pytest.raises(ValueError, match="cache"):
            P.read_quantized(cache._replace(**{name: getattr(cache, name).reshape(-1)[0]}))
