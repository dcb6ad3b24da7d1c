"""The 4-bit head (rpd_quant_*) at its edges: activations of any size under a norm.  Bounds as in test_quant_head.py."""
import pytest
import torch

import paper_2609_36452_gb300 as rpd
from test_quant_head import TYPES, check, head_of, make

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")


@gpu
@needs_gpu
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30, 1e30])
@pytest.mark.parametrize("d,rows,V", [(192, 5, 260), (192, 20, 260), (192, 20, 5003), (1001, 16, 600), (5000, 33, 5003)])
@pytest.mark.parametrize("x", ["bf16", "f16"])
def test_normalised_rows_of_any_magnitude(d, rows, V, x, eps):
    """Rows whose squares leave fp32 on either side, rows whose elements span the type's range, one largest element
    alone, and rows of zeros (0 with any eps > 0; no number without one, as by the formula)."""
    c = make(d, V, rows, 64, True, True, x=x, pad=3 if d % 8 else 0)
    c["eps"] = eps
    low, high = (-132, 126) if x == "bf16" else (-24, 15)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    part = 0.5 + 0.5 * torch.rand(rows, d, device="cuda", generator=gen).double()
    sign = torch.where(torch.rand(rows, d, device="cuda", generator=gen) < 0.5, -1.0, 1.0).double()
    power = torch.linspace(low, high, rows, device="cuda").round().double()
    c["x"].copy_((part * sign * torch.exp2(power)[:, None]).to(TYPES[x]))
    c["x"][2] = torch.exp2(torch.linspace(low, high, d, device="cuda").round().double()).to(TYPES[x])
    c["x"][3] = 0
    c["x"][3, 77] = torch.finfo(TYPES[x]).max
    zero = 1
    c["x"][zero] = 0
    c["gain"].copy_((0.5 + 0.5 * torch.rand(d, device="cuda", generator=gen)).to(TYPES[x]))  # g x stays finite
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=eps)
    torch.cuda.synchronize()
    if eps:
        assert (c["out"][zero] == 0).all()
    else:
        assert torch.isnan(c["out"][zero]).all()
        c["out"][zero] = 0
        # the rest against the definition, with another row in the zeros' place
        c["x"][zero] = c["x"][0]
        c["out"][zero] = c["out"][0]
    check(c)
    h.close()
