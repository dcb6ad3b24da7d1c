"""Verification of drafted tokens (rpd_verify) at its edges: variates and probabilities at the ends of their
ranges, sizes beyond 32 bits.  Decisions are held against the definition in 64 bits, with test_verify.py's bounds."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2609_36452_gb300 as rpd
from test_verify import Case, args_of

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")


def read_singly(c):
    """The case's variates moved to where no vector of them lies beside one of the logits."""
    e = torch.full((c.B, c.V + 4), math.nan, device="cuda")[:, 1:c.V + 1]
    e.copy_(c.noise)
    c.noise = e


def reject_all(c):
    """Drafts that the target is far less likely to draw than the draft model."""
    q, p = c.draft.double(), torch.where(c.on[:, :c.D], c.target[:, :c.D].double(), -math.inf)
    t = c.temperature.double().view(-1, 1, 1)
    gain = torch.softmax(q / t, 2) - torch.softmax(p / t, 2)
    c.tokens = gain.argmax(2).int()
    c.uniform.fill_(1 - 2.0 ** -24)


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("bad", [-1e-6, -0.0, 0.0, -math.inf, math.nan])
def test_tokens_without_an_excess_never_win(dtype, single, bad):
    """After a rejection against a draft model: variates that would win, or that are no variates, at all the
    tokens that the target is not more likely to draw than the draft model, masked ones among them."""
    c = Case(6, 1, 1016, dtype, True, allowed=True)
    reject_all(c)
    t = c.temperature.double().view(-1, 1)
    p = torch.softmax(torch.where(c.on[:, 0], c.target[:, 0].double(), -math.inf) / t, 1)
    q = torch.softmax(c.draft[:, 0].double() / t, 1)
    none = p * (1 + 2.0 ** -12) < q  # below the draft model's by more than either is off
    assert (none & c.on[:, 0]).any(1).all() and (none & ~c.on[:, 0]).any(1).all() and (~none).any(1).all()
    c.noise[none] = bad
    if single:
        read_singly(c)
    got = c.run()
    assert (got["accepted"] == 0).all() and (got["status"] == 0).all()
    token = torch.tensor(got["token"][:, 0], device="cuda").long()
    assert not none[torch.arange(6, device="cuda"), token].any()
    c.noise = torch.where(none, math.inf, c.noise)  # (weights of 0: for the definition, any variate)
    c.check(got)


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("kind", ["all", "others", "excess", "sample"])
def test_a_variate_of_minus_zero_is_zero(dtype, single, kind):
    """-0 is not negative (-log(1 - u) gives it at u = 0): it wins as 0 does, the lowest of several."""
    c = Case(4, 0 if kind == "sample" else 1, 1016, dtype, kind in ("all", "excess"))
    if kind == "excess":
        reject_all(c)
    elif kind == "others":
        c.tokens = c.target[:, :1].float().argmin(2).int()
        c.uniform.fill_(1 - 2.0 ** -24)
    else:
        c.uniform.fill_(0.0)
    row = 1 if kind == "all" else 0
    t = c.temperature.double().view(-1, 1)
    w = torch.softmax(c.target[:, row].double() / t, 1)
    if kind == "excess":
        w = w - torch.softmax(c.draft[:, 0].double() / t, 1)
    best = w.topk(2, 1).indices.sort(1).values  # the two that are surely worth something
    if kind == "others":
        assert not (best == c.tokens.long()).any()
    c.noise.scatter_(1, best, -0.0)
    c.noise[0, best[0, 0]] = 0.0  # the two zeros tie
    if single:
        read_singly(c)
    got = c.run()
    assert got["token"][:, row].tolist() == best[:, 0].tolist()
    assert (got["status"] == 0).all() and (got["accepted"] == row).all()


@pytest.mark.parametrize("shape", [((1 << 32) + 1, 1, 1), (1, (1 << 32) + 1, 1), (1, 1, (1 << 32) + 1), (1 << 31, 1, 1)])
def test_sizes_beyond_32_bits_are_refused(shape):
    """Of 2^32 + 1 sequences, drafts or tokens the C ABI would see one."""
    z = torch.zeros(1, 1, 1).expand(shape)
    with pytest.raises(rpd.RpdError, match="32 bits") as e:
        rpd.verify(z, None, None, None, None, None, None)
    assert e.value.code == rpd.RPD_ERR_UNSUPPORTED


def test_as_many_rows_as_promised_are_taken():
    """2^26 rows of logits and no more: drafts' rows count too."""
    for kw, ok in ((dict(B=1 << 26, D=0), True), (dict(B=(1 << 26) + 1, D=0), False), (dict(B=1 << 24, D=3), True),
                   (dict(B=(1 << 24) + 1, D=3), False), (dict(B=1 << 23, D=3, draft=4096), True),
                   (dict(B=1 << 24, D=2, draft=4096), False)):
        a = args_of(target=None, **kw)  # what comes after the sizes is refused in any case
        want = rpd.RPD_ERR_INVALID_ARGUMENT if ok else rpd.RPD_ERR_UNSUPPORTED
        assert rpd.rpd_verify(ctypes.byref(a), 4096, 1 << 60, None) == want, kw


@gpu
@needs_gpu
def test_the_most_rows():
    """2^26 sequences of one token, and 2^25 of one draft each, which is accepted."""
    for B, D in ((1 << 26, 0), (1 << 25, 1)):
        target = torch.zeros(1, 1, 2, device="cuda").expand(B, D + 1, 2)
        tokens = torch.zeros(B, D, dtype=torch.int32, device="cuda")
        uniform = torch.full((B, D), 0.25, device="cuda")
        noise = torch.tensor([[1.0, 2.0]], device="cuda").expand(B, 2)
        o = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, D + 1), (B,))]
        rpd.verify(target, tokens, uniform, noise, *o)
        assert (o[0] == D).all() and (o[1] == 0).all() and (o[2] == 0).all()
        del target, tokens, uniform, noise, o
        torch.cuda.empty_cache()


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("draft", [True, False])
def test_probabilities_down_to_the_smallest_number(dtype, draft):
    """Drafts whose probability lies between 2^-149 and 2^-126: it is what the definition says to half of fp32's smallest
    number (and the tolerance of the value), and u = 0 accepts them."""
    c = Case(16, 1, 700, dtype, draft, spread=0.5)
    c.temperature.fill_(0.5)
    c.tokens.fill_(33)
    c.target[:, 0, 33] = c.target[:, 0].amax(1) - torch.linspace(38, 46, 16, device="cuda").to(c.dtype)
    if draft:
        c.draft[:, 0, 33] = c.draft[:, 0].amax(1) - 40
    c.uniform.fill_(0.0)
    got = c.run()
    assert (got["accepted"] == 1).all() and (got["status"] == 0).all()
    p = torch.softmax(c.target[:, 0].double() / 0.5, 1)[:, 33].cpu().numpy()
    assert (p < 2.0 ** -110).all() and (p > 2.0 ** -149).all() and (p < 2.0 ** -126).any()
    x = c.target[:, 0, 33].double() - c.target[:, 0].double().amax(1)
    bound = c.tolerance(x.cpu().numpy() * 2 / math.log(2)) * p + 2.0 ** -150
    assert (abs(got["prob"][:, 0].astype(float) - p) <= bound).all()
    c.check(got)


@gpu
@needs_gpu
@pytest.mark.parametrize("D", [0, 2])
def test_temperatures_beyond_their_bounds_count_as_these(D):
    """Infinite and huge temperatures over logits that span all of fp32, and vanishing ones: the same as at the largest and
    the smallest that count, probabilities, verdicts and draws alike, so that the probabilities still add up to 1."""
    runs = []
    most, least = 1 / math.log(2) * 1e37, 1 / math.log(2) * 1e-30
    for T in ((math.inf, 1e38, 2e37, 1e-40, 1e-33, 1e-30), (1e38, math.inf, math.inf, 1e-31, 1e-42, 1e-32)):
        c = Case(6, D, 700, "f32", False)
        c.target[:, :, ::2] = torch.finfo(torch.float32).min
        c.target[:, :, 1::2] *= 1e36
        c.target[3:] = (c.target[3:] / 1e36).clamp(min=-4).round() * 1e-30
        c.temperature.copy_(torch.tensor(T))
        c.tokens.fill_(7)
        runs.append(c.run())
        c.temperature.copy_(torch.tensor((most,) * 3 + (least,) * 3))
        c.check(runs[-1])
    for k in runs[0]:
        assert (runs[0][k] == runs[1][k]).all(), k
    assert (runs[0]["status"] == 0).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_error_of_the_probabilities(dtype):
    """Relative errors of the drafts' probabilities: the roundings of z - m, of 1 / T and of their product move the
    exponent, and so the value, by 3 * 2^-24 |x|; exp2f is right to 2^-22, the quotient to 2^-24.  The sum: ex2's
    2^-22, and a term's exponent, three times rounded, |x| of which the weights of the sum average; its
    additions have no common sign."""
    c = Case(16, 8, 50021, dtype, False, seed=4)
    c.tokens = torch.where(torch.rand(16, 8, device="cuda") < 0.5, c.target[:, :8].float().argmax(2).int(), c.tokens)
    got = c.run()
    t = c.temperature.double().view(-1, 1, 1)
    z = c.target[:, :8].double()
    p = torch.softmax(z / t, 2)
    x = (z - z.amax(2, keepdim=True)) / t
    mean = (p * x.abs()).sum(2)  # |x| of the terms as the sum weighs them
    at = c.tokens.long().unsqueeze(2)
    p, x = p.gather(2, at).squeeze(2), x.gather(2, at).squeeze(2).abs()
    chain = (50021 / 256 + 64) ** 0.5
    bound = (3 * x + 5 + 4 + 3 * mean + chain) * 2.0 ** -24
    off = (torch.tensor(got["prob"], device="cuda").double() / p - 1).abs()
    print(f"off {off.max().item():.3g}, of the bound {(off / bound).max().item():.3g}")
    assert (off <= bound).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("draft", [None, False, True])
def test_a_tie_anywhere_in_the_row_goes_to_the_lowest_index(dtype, single, draft):
    """Two tokens with the same logits and the same variate, by far the smallest of the row: wherever they lie, and whatever
    the largest logits of their parts of the row are."""
    B, V = 150, 6008
    c = Case(B, 0 if draft is None else 1, V, dtype, draft, spread=4.0, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(9)
    pair = torch.rand(B, V, device="cuda", generator=gen).topk(2, 1).indices.sort(1).values
    row = 0
    c.temperature.fill_(1.0)
    if draft is not None:
        row = 1 if draft else 0  # behind an accepted draft, or in a rejected one's place
        c.uniform.fill_(0.0 if draft else 1 - 2.0 ** -24)
        c.tokens = c.target[:, :1].float().argmin(2).int()
    below = 6 * torch.rand(B, 1, device="cuda", generator=gen)  # at least e^-6 2^27 in the race, others at most 100
    c.target[:, row].scatter_(1, pair, (c.target[:, row].float().amax(1, keepdim=True) - below).to(c.dtype).expand(B, 2))
    c.noise.clamp_(min=0.01)
    c.noise.scatter_(1, pair, (2.0 ** -28 * (1 + torch.rand(B, 1, device="cuda", generator=gen))).expand(B, 2))
    if single:
        read_singly(c)
    got = c.run()
    assert (got["status"] == 0).all() and (got["accepted"] == row).all()
    assert got["token"][:, row].tolist() == pair[:, 0].tolist()


@gpu
@needs_gpu
def test_drafts_drawn_under_the_target_s_mask():
    """A draft model that drew under a mask, its other logits at -infinity: the first token that a sequence yields is a draw
    from the masked target; 20000 sequences, every frequency within five standard deviations."""
    B, V = 20000, 6
    g = torch.Generator(device="cuda").manual_seed(11)
    dev = dict(device="cuda", generator=g)
    on = torch.tensor([True, False, True, True, False, True], device="cuda")
    z = torch.tensor([0.0, 5.0, -1.0, 1.0, math.nan, 0.5], device="cuda")
    y = torch.where(on, torch.randn(V, **dev), -math.inf)
    c = Case(2, 1, V)
    c.B, c.on = B, on.expand(B, 2, V)
    c.pack()
    c.target, c.draft, c.temperature = z.expand(B, 2, V), y.expand(B, 1, V), None
    e = torch.empty(B, V, device="cuda").exponential_(generator=g)
    c.tokens = (y - e.log()).argmax(1).int().view(B, 1)
    c.uniform = torch.rand(B, 1, **dev)
    c.noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    got = c.run()
    assert (got["status"] == 0).all()
    p = torch.softmax(torch.where(on, z, -math.inf).double(), 0).cpu().numpy()
    first = np.bincount(got["token"][:, 0], minlength=V) / B
    assert (abs(first - p) <= 5 * (p * (1 - p) / B) ** 0.5).all(), (first, p)
