"""The 8-bit head with scales at the ends of their documented range, 2^-100 and 2^100, for rows of any size."""
import pytest
import torch

import paper_2609_36452_gb300 as rpd

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")


@gpu
@needs_gpu
@pytest.mark.parametrize("rows", [1, 130])
@pytest.mark.parametrize("shift,size", [(100, 2.0 ** -20), (100, 2.0 ** -100), (-100, 1.0), (-100, 2.0 ** 100)])
def test_longest_rows_at_the_ends_of_scales(shift, size, rows):
    """32768 columns of the largest codes: a sum relative to the row's largest number is below 2^25 2^100, and its logit is that times
    the number.  Every step is a power of two times 448 or 7 / 4 of one, so that sums of 32768 are exact."""
    d, V = 32768, 130
    x = torch.full((rows, d), 1.75 * size, device="cuda").bfloat16()
    codes = torch.full((V, d), 448.0, device="cuda").to(torch.float8_e4m3fn)
    scales = torch.full((2, d // 128), 2.0 ** shift, device="cuda")
    out = torch.empty(rows, V, device="cuda")
    h = rpd.Fp8Head(d, V)
    h.set_weights(codes, scales)
    h.logits(x, out)
    torch.cuda.synchronize()
    want = 1.75 * size * 448.0 * d * 2.0 ** shift
    # the activations' scale, 1.75 size / 448, its products with the block's sum and the additions of 256 of these are rounded
    assert 2.0 ** -126 < want < 2.0 ** 127
    assert ((out.double() - want).abs() <= (2 + 256) * 2.0 ** -24 * want).all()


@gpu
@needs_gpu
def test_blocks_of_small_activations():
    """A block whose sx sw is 2^-126 of the row's largest number and more counts in full, also where nothing else does."""
    d, V = 256, 128
    x = torch.ones(3, d, device="cuda").bfloat16()
    x[:, 128:] = 2.0 ** -16
    codes = torch.zeros(V, d, device="cuda").to(torch.float8_e4m3fn)
    codes[:, 128:] = torch.ones(V, 128, device="cuda").to(torch.float8_e4m3fn)
    out = torch.empty(3, V, device="cuda")
    h = rpd.Fp8Head(d, V)
    h.set_weights(codes, torch.full((1, 2), 2.0 ** -100, device="cuda"))
    h.logits(x, out)
    torch.cuda.synchronize()
    want = 128 * 2.0 ** -116
    assert ((out.double() - want).abs() <= 4 * 2.0 ** -24 * want).all()
