"""Sampling under limits (rpd_sample) at the ends of its ranges, against a sort in 64 bits.  Tokens, numbers and masks have to be
equal, probabilities as close as in test_sample.py."""
import pytest
import torch

import paper_2609_36452_gb300 as rpd
from test_sample import INF, NAN, TYPES, gen, gpu, logits, needs_gpu, run_and_check

# from where the largest logit less 54 octaves of weights still is an fp32 number to the largest temperature there is
HOT = [7e28, 1e29, 1e33, 1e35, 3e36, 1.2e37, 2e37, 3e38, INF]


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", HOT)
@pytest.mark.parametrize("masked", [False, True])
def test_tokens_without_weight_have_none_however_hot(masked, T, kind):
    """Rows of which vectors do not hold every token, logits of -infinity and tokens that are not allowed: at T = infinity each of
    the others weighs the same and these nothing."""
    rows, V, g = 12, 50021, gen(3)
    z = logits(rows, V, kind, 8)
    on = torch.rand(rows, V, generator=g) < 0.67 if masked else None
    z[4:8][torch.rand(4, V, generator=g) < 0.1] = -INF
    z[8:, ::5] = torch.finfo(TYPES[kind]).min
    if masked:
        z[:, 1::7][~on[:, 1::7]] = NAN
    u = [0.0, 0.01, 0.5, 1 - 2.0 ** -24] * 3
    p = [0.9, 0.3, 0.999, 0.02] * 3
    for kw in (dict(), dict(p=p), dict(p=p, m=[1e-9] * rows), dict(m=[1e-9] * rows), dict(k=[30, 3000, 20000, 0] * 3), dict(k=[1000] * rows, p=p)):
        run_and_check(z, u, [T] * rows, on=on, stride=V + 5 if masked else V, **kw)


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1000, 5001, 152064])
@pytest.mark.parametrize("T", HOT)
def test_logits_as_large_as_the_temperature(T, V, kind):
    """Weights that differ although no temperature is larger: logits over all that the type has, beside its ends, and around 0."""
    rows, g = 9, gen(V)
    t, most = min(T, 1.44e37), torch.finfo(TYPES[kind]).max
    z = 1.5 * t * torch.randn(rows, V, generator=g, dtype=torch.float64)
    z[3:6] = 0.999 * most * (2 * torch.rand(3, V, generator=g, dtype=torch.float64) - 1)
    z[6] = z[6] - most
    z[7] = z[7].abs() - most
    z[8] = most - z[8].abs()
    z = z.clamp(-most, most).to(TYPES[kind])
    z[1, 100:200] = -INF
    u = [0.0, 0.3, 0.97] * 3
    p = [0.9, 0.5, 0.99] * 3
    for kw in (dict(), dict(p=p), dict(p=p, m=[1e-4] * rows), dict(m=[1e-4] * rows), dict(k=[30, 300, V // 2] * 3, p=p)):
        run_and_check(z, u, [T] * rows, stride=V + 1, **kw)


@gpu
@needs_gpu
@pytest.mark.parametrize("V,count,limits", [
    (5000, 40, "k"), (5000, 500, "k"), (5000, 1000, "k"), (5000, 2048, "k"), (900, 600, "k"), (2000, 1500, "k"), (300, 300, ""), (1024, 1000, ""),
    (5000, 40, "m"), (5000, 500, "m"), (5000, 1500, "m"), (126464, 2048, "k"), (126464, 1500, "m")])
def test_light_tokens_beside_a_heavy_one(V, count, limits):
    """Probabilities of tokens of 2^-21 of the sum altogether.  Sums are in units of 2^-54 of the largest weight, lists of more than 512
    tokens in units of 2^-52: a token's weight is one of them off at most (a weight that is a product of 32-bit numbers is cut off to
    whole units: rows whose other tokens overflow a bin, 126464 of them here; one made in 64 bits is rounded), and their
    sum, of which the quotient is taken, count of them.  Weights themselves are right to 2^-30, the quotient to 2^-29, and half of
    fp32's eps comes with the result."""
    rows, g = 40, gen(V + count)
    T = 0.5 + torch.rand(rows, generator=g)
    light = 2.0 ** -21 / count * torch.exp2(torch.rand(rows, count, generator=g, dtype=torch.float64) - 0.5)
    z = torch.full((rows, V), -60.0)
    z[:, :count] = (T.double()[:, None] * torch.log(light)).float()
    z[:, 7] = 0.0
    z = z[:, torch.randperm(V, generator=g)]
    u = 1 - 2.0 ** -24 * torch.tensor([1.0, 2.0, 3.0, 4.0]).repeat(rows // 4)
    w = torch.where(z < -50.0, 0.0, torch.exp(z.double() / T.double()[:, None]))
    if not limits:
        w = torch.exp(z.double() / T.double()[:, None])
    dev = z.cuda()
    token, status = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    prob = torch.zeros(rows, device="cuda")
    rpd.sample(dev, u.cuda(), token, status, temperature=T.cuda(), out_prob=prob,
               top_k=torch.full((rows,), count, dtype=torch.int32, device="cuda") if limits == "k" else None,
               min_p=torch.full((rows,), 2.0 ** -50, device="cuda") if limits == "m" else None)
    assert (status == 0).all()
    want = w.gather(1, token.long().cpu()[:, None])[:, 0] / w.sum(1)
    assert (want < 2.0 ** -20 / count).all()
    off = (prob.cpu().double() - want).abs()
    unit = 2.0 ** -54 if count <= 512 else 2.0 ** -52
    most = want * (2.0 ** -24 + 2.0 ** -28 + count * unit) + unit
    assert (off <= most).all(), float((off / most).max())


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,V", [(1, 65536), (24, 70001), (5, 130000)])
def test_few_rows_under_top_p(rows, V, kind):
    """Eight CTAs a row: top-p's tokens from one to thousands, likely ones beside each other, in one CTA's slice or over all of them."""
    g = gen(V)
    for spread, peaks in ((0.3, 6), (1.5, 6), (2.5, 1), (1.0, 300), (1.0, 900)):
        z = logits(rows, V, kind, V + peaks, spread=spread, peaks=peaks)
        z[::3, 100:100 + 2 * peaks] = (8 + 2 * torch.randn(len(z[::3]), 2 * peaks, generator=g)).to(z.dtype)
        for low, high in ((0.2, 0.9), (0.9, 0.999), (0.9999, 1.0)):
            p = (low + (high - low) * torch.rand(rows, generator=g)).tolist()
            T = (0.5 + torch.rand(rows, generator=g)).tolist()
            u = torch.rand(rows, generator=g).tolist()
            run_and_check(z, u, T, None, p, None, stride=V + 3)
            run_and_check(z, u, T, None, p, [10.0 ** -i for i in range(rows)] if rows < 24 else None)


@gpu
@needs_gpu
@pytest.mark.parametrize("V", [300, 1500, 5000, 70001])
def test_zeros_of_either_sign(V):
    """A number, limits and a temperature of -0 are 0."""
    z = logits(6, V, "f32", V)
    u, zero = [-0.0] * 6, [-0.0] * 6
    for kw in (dict(), dict(p=[0.9] * 6), dict(k=[20] * 6), dict(k=[20] * 6, p=[0.9] * 6), dict(k=[V // 2 + 1] * 6), dict(m=[0.1] * 6), dict(p=zero),
               dict(k=[20] * 6, p=zero), dict(m=zero), dict(T=zero), dict(p=[0.999] * 6, T=[4.0] * 6)):
        run_and_check(z, u, **kw)
    run_and_check(z, [0.3, 0.99, 0.0] * 2, p=zero, m=zero)
