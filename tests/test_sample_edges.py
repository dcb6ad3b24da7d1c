"""Sampling under limits (rpd_sample) at the ends of its ranges, against a sort in 64 bits.  Tokens, numbers and masks have to be
equal, probabilities as close as in test_sample.py."""
import pytest
import torch
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
