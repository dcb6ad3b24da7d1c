"""Verification of drafted tokens (rpd_verify) at its edges: variates and probabilities at the ends of their
ranges, sizes beyond 32 bits.  Decisions are held against the definition in 64 bits, with test_verify.py's bounds."""
import ctypes
import math

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
