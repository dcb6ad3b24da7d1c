"""Verification of drafted tokens (rpd_verify): refusals (no GPU), and every decision against the
definition in 64 bits.

Tolerance.  A probability is 2^((z - m) c) / s in fp32.  z - m, c and their product are rounded once each,
which moves the exponent by 3 * 2^-24 |x| (x = (z - m) c, in powers of two) and the value by ln 2 times that;
ex2 is right to 2^-22, the sum s has that error of its terms (the heavy ones, with |x| below 30, to
(4 + 63) * 2^-24) and one rounding for every addition of a chain of at most V / 256 + 64 terms, and a
division is one more: in all (2.1 |x| + V / 256 + 140) * 2^-24 of the value.  A draft's verdict, and the race for
the next token, may differ from the definition's only where the two sides lie closer than their errors."""
import ctypes
import math
import threading

import numpy as np
import pytest
import torch

import paper_2609_36452_gb300 as rpd

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------ refusals

def args_of(**kw):
    """A rpd_verify_args of made-up addresses: refused before any of them is used."""
    a = rpd.RpdVerifyArgs()
    for k in ("target", "tokens", "temperature", "uniform", "noise", "out_accepted", "out_token", "out_status"):
        setattr(a, k, 4096)
    a.B, a.D, a.V, a.type = 2, 3, 100, rpd.RPD_TYPE_F32
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), "INVALID_ARGUMENT"), (dict(D=-1), "INVALID_ARGUMENT"), (dict(V=0), "INVALID_ARGUMENT"),
    (dict(type=7), "INVALID_ARGUMENT"), (dict(D=1025), "UNSUPPORTED"), (dict(V=(1 << 24) + 1), "UNSUPPORTED"),
    (dict(B=1 << 27), "UNSUPPORTED"), (dict(target=None), "INVALID_ARGUMENT"), (dict(tokens=None), "INVALID_ARGUMENT"),
    (dict(out_token=None), "INVALID_ARGUMENT"), (dict(temperature=None, noise=None), "INVALID_ARGUMENT"),
    (dict(temperature=None, uniform=None), "INVALID_ARGUMENT"), (dict(target_row_stride=-1), "INVALID_ARGUMENT"),
    (dict(noise_stride=-1), "INVALID_ARGUMENT"), (dict(target=4098), "INVALID_ARGUMENT"),
    (dict(lengths=4098), "INVALID_ARGUMENT"), (dict(type=rpd.RPD_TYPE_BF16, draft=4097), "INVALID_ARGUMENT")])
def test_bad_arguments_are_refused(kw, code):
    a = args_of(**kw)
    got = rpd.rpd_verify(ctypes.byref(a), 4096, 1 << 40, None)
    assert got == getattr(rpd, "RPD_ERR_" + code)
    assert rpd.rpd_last_error() != b""


def test_small_or_crooked_workspace_is_refused():
    a = args_of()
    need = rpd.rpd_verify_workspace(2, 3)
    assert need > 0 and rpd.rpd_verify_workspace(-1, 3) == -1
    assert rpd.rpd_verify(ctypes.byref(a), 4096, need - 1, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_verify(ctypes.byref(a), 4104, need, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_verify(ctypes.byref(a), None, need, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_verify(None, 4096, need, None) == rpd.RPD_ERR_INVALID_ARGUMENT


def test_no_sequences_is_a_no_op():
    a = args_of(B=0, target=None, tokens=None, out_token=None, out_accepted=None, out_status=None)
    assert rpd.rpd_verify(ctypes.byref(a), None, 0, None) == rpd.RPD_OK


def test_binding_refuses_host_tensors():
    z = torch.zeros(1, 2, 10)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(rpd.RpdError, match="CUDA"):
        rpd.verify(z, i, z[0, :1, :1], z[0, :1], i[0], i, i[0])
    with pytest.raises(rpd.RpdError, match="target"):
        rpd.verify(None, i, z, z, i, i, i)


# ------------------------------------------------------------------------------ the definition

class Case:
    """Inputs on the GPU and the definition of the answer in 64 bits (numpy)."""

    def __init__(self, B, D, V, dtype="f32", draft=True, greedy=0, ragged=False, allowed=False, pad=0, seed=0,
                 spread=2.0):
        g = torch.Generator(device="cuda").manual_seed(1000 + seed)
        dev = dict(device="cuda", generator=g)
        T = TYPES[dtype]
        self.B, self.D, self.V, self.dtype = B, D, V, T
        whole = torch.full((B, D + 1, V + pad), float("nan"), dtype=T, device="cuda")
        self.target = whole[:, :, :V]
        z = spread * torch.randn(B, D + 1, V, **dev)
        self.target.copy_(z)
        self.draft = None
        self.tokens = torch.randint(0, V, (B, D), dtype=torch.int32, **dev)
        self.temperature = 0.5 + torch.rand(B, **dev)
        if greedy:
            self.temperature[::greedy] = 0
        if draft:
            self.draft = torch.full((B, D, V + pad), float("nan"), dtype=T, device="cuda")[:, :, :V]
            self.draft.copy_(z[:, :D] + 0.7 * torch.randn(B, D, V, **dev))
            if D:
                e = torch.empty(B, D, V, device="cuda").exponential_(generator=g)
                t = self.temperature.clamp(min=0.05).view(B, 1, 1)
                self.tokens = (self.draft.float() / t - e.log()).argmax(2).int()
        elif D:
            self.tokens = torch.where(torch.rand(B, D, **dev) < 0.7, z[:, :D].argmax(2), self.tokens.long()).int()
        self.lengths = torch.randint(0, D + 1, (B,), dtype=torch.int32, **dev) if ragged else None
        self.uniform = torch.rand(B, D, **dev)
        self.noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
        self.on = torch.ones(B, D + 1, V, dtype=torch.bool, device="cuda")
        self.allowed = None
        if allowed:
            self.on = torch.rand(B, D + 1, V, **dev) < 0.6
            self.on[:, :, V // 2] = True
            self.pack()
            self.target[~self.on] = torch.tensor([math.inf, math.nan, -math.inf, 3e38], device="cuda").to(T)[
                torch.randint(0, 4, (int((~self.on).sum()),), **dev)]

    def pack(self):
        words = (self.V + 31) // 32
        bits = torch.nn.functional.pad(self.on, (0, words * 32 - self.V)).view(self.B, self.D + 1, words, 32)
        w = (bits.long() << torch.arange(32, device="cuda")).sum(-1)
        self.allowed = torch.where(w >= 1 << 31, w - (1 << 32), w).int()

    def run(self, **kw):
        o = self.outputs = dict(
            out_accepted=torch.full((self.B + 1,), -9, dtype=torch.int32, device="cuda"),
            out_token=torch.full((self.B + 1, self.D + 1), -9, dtype=torch.int32, device="cuda"),
            out_status=torch.full((self.B + 1,), -9, dtype=torch.int32, device="cuda"),
            out_prob=torch.full((self.B + 1, self.D), -9.0, device="cuda"))
        given = dict(draft=self.draft, lengths=self.lengths, temperature=self.temperature, allowed=self.allowed)
        given.update(kw)
        rpd.verify(self.target, self.tokens, self.uniform, self.noise, *[
            o[k][:self.B] for k in ("out_accepted", "out_token", "out_status", "out_prob")], **given)
        torch.cuda.synchronize()
        for v in o.values():  # what lies behind the last sequence stays as it was
            assert (v[self.B:] == -9).all()
        return {k[4:]: v[:self.B].cpu().numpy() for k, v in o.items()}

    def tolerance(self, x):
        return (2.1 * np.abs(x) + self.V / 256 + 140) * 2.0 ** -24

    def row(self, logits, on, T):
        """Probabilities in 64 bits and the bound of their relative error; None without a distribution."""
        z = np.where(on, logits.double().cpu().numpy(), -np.inf)
        top = z.max()
        if not np.isfinite(top):
            return None
        if T == 0:
            p = np.zeros(self.V)
            p[np.argmax(z)] = 1
            return p, np.zeros(self.V)
        x = (z - top) / T * math.log2(math.e)
        p = np.exp2(x)
        return p / p.sum(), self.tolerance(np.where(np.isfinite(x), x, 0))

    def check(self, got):
        """Follows the decisions that were made and asks whether the definition allows each."""
        temps = self.temperature.double().cpu().numpy() if self.temperature is not None else np.ones(self.B)
        on_all, tokens = self.on.cpu().numpy(), self.tokens.cpu().numpy()
        uniform, exactly = self.uniform.double().cpu().numpy(), 0
        for b in range(self.B):
            n = self.D if self.lengths is None else int(self.lengths[b])
            acc, row, T = int(got["accepted"][b]), got["token"][b], temps[b]
            assert 0 <= acc <= n
            assert (row[:acc] == tokens[b, :acc]).all() and (row[acc + 1:] == -1).all()
            assert (got["prob"][b, n:] == 0).all()
            ended = False
            for i in range(n + 1):
                pr = self.row(self.target[b, i], on_all[b, i], T)
                x = int(tokens[b, i]) if i < n else -1
                inside = 0 <= x < self.V
                px, pe = (pr[0][x], pr[1][x]) if pr is not None and inside else (0.0, 0.0)
                if i < n:
                    assert abs(got["prob"][b, i] - px) <= pe * px + 1e-37, (b, i, got["prob"][b, i], px)
                if ended:
                    continue
                if i == acc and row[acc] == -1:  # the sequence ends without a distribution
                    assert got["status"][b] == rpd.RPD_ERR_INVALID_ARGUMENT
                    qr = self.row(self.draft[b, i], np.ones(self.V, bool), T) if self.draft is not None and T > 0 and i < n else ()
                    assert pr is None or qr is None
                    ended = True
                    continue
                assert pr is not None
                w, err = pr[0].copy(), pr[0] * pr[1]
                if i < n:
                    qx, qe = 1.0, 0.0
                    if T > 0 and self.draft is not None:
                        q, qerr = self.row(self.draft[b, i], np.ones(self.V, bool), T)
                        qx, qe = (q[x], qerr[x]) if inside else (0.0, 0.0)
                    if i < acc:
                        ok = px > 0 if T == 0 else uniform[b, i] * qx * (1 - qe) < px * (1 + pe)
                        assert ok, (b, i, "accepted")
                        continue
                    ok = px == 0 if T == 0 else uniform[b, i] * qx * (1 + qe) >= px * (1 - pe)
                    assert ok, (b, i, "rejected")
                    if T > 0:
                        if self.draft is not None:
                            err = err + q * qerr
                            w = np.maximum(w - q, 0)
                        elif inside:
                            w[x] = err[x] = 0
                ended = True
                assert got["status"][b] == rpd.RPD_OK
                v = int(row[acc])
                assert 0 <= v < self.V and on_all[b, i, v]
                if T == 0:
                    assert v == np.argmax(w)
                    exactly += 1
                    continue
                e = self.noise[b].double().cpu().numpy()
                with np.errstate(divide="ignore", invalid="ignore"):
                    score = np.where(w > 0, w / e, 0.0)
                    low = np.where(w - err > 0, (w - err) / e, 0.0)
                exactly += v == np.argmax(score)
                assert (w[v] + err[v]) / e[v] * (1 + 2.0 ** -21) >= low.max(), (b, v, np.argmax(score))
            assert ended
        return exactly


# ------------------------------------------------------------------------------ decisions

SHAPES = [
    # B, D, V, dtype, draft, greedy, ragged, allowed, pad
    (1, 0, 1, "f32", False, 0, False, False, 0),
    (1, 1, 1, "bf16", True, 0, False, False, 1),
    (1, 0, 7, "f16", False, 0, False, True, 0),
    (2, 1, 8, "f32", True, 0, False, False, 0),
    (3, 2, 31, "bf16", False, 2, True, True, 3),
    (4, 3, 33, "f16", True, 0, True, True, 0),
    (1, 3, 4096, "f32", True, 0, False, False, 0),
    (5, 4, 1000, "bf16", True, 1, False, False, 0),
    (9, 5, 1001, "f16", True, 3, True, True, 5),
    (8, 4, 2048, "f32", False, 4, True, False, 8),
    (3, 33, 515, "bf16", True, 0, True, False, 1),
    (64, 5, 3000, "bf16", True, 8, True, False, 0),
    (33, 0, 5000, "f32", False, 5, False, True, 2),
    (1, 257, 300, "f32", False, 0, False, False, 0),
    (1, 1024, 40, "bf16", True, 0, False, True, 0),
    (40, 3, 2000, "f16", True, 7, True, False, 0),
    (200, 0, 900, "f32", False, 9, False, False, 1),
    (2, 5, 50021, "bf16", True, 0, False, True, 3),
    (1, 5, 126464, "bf16", True, 0, False, False, 0),
    (3, 2, 152064, "f32", True, 0, False, False, 0),
    (2, 1, 126464, "f16", False, 0, False, True, 8),
]


@gpu
@needs_gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(int(v) if isinstance(v, bool) else v) for v in s))
def test_decisions_match_the_definition(shape):
    c = Case(*shape)
    exactly = c.check(c.run())
    assert exactly >= c.B - 1  # near ties are rare


@gpu
@needs_gpu
@pytest.mark.parametrize("draft", [True, False])
def test_accepted_and_next_tokens_are_distributed_like_the_target(draft):
    """The first token that a sequence yields is a draw from the target, whatever the draft model:
    20000 sequences over the same small rows; every frequency within five standard deviations."""
    B, V = 20000, 6
    g = torch.Generator(device="cuda").manual_seed(7)
    dev = dict(device="cuda", generator=g)
    z, y = torch.tensor([0.0, 1.0, -1.0, 2.0, 0.5, -3.0], device="cuda"), torch.randn(V, **dev)
    c = Case(2, 1, V, draft=draft)
    c.B, c.on = B, torch.ones(B, 2, V, dtype=torch.bool, device="cuda")
    c.target = z.expand(B, 2, V)
    c.draft = y.expand(B, 1, V) if draft else None
    c.temperature = None
    e = torch.empty(B, V, device="cuda").exponential_(generator=g)
    c.tokens = ((y - e.log()).argmax(1) if draft else torch.randint(0, V, (B,), **dev)).int().view(B, 1)
    c.uniform = torch.rand(B, 1, **dev)
    c.noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    got = c.run()
    p = torch.softmax(z.double(), 0).cpu().numpy()
    first = np.bincount(got["token"][:, 0], minlength=V) / B
    assert (np.abs(first - p) < 5 * np.sqrt(p * (1 - p) / B)).all(), (first, p)


@gpu
@needs_gpu
def test_ties_go_to_the_lowest_index():
    c = Case(2, 1, 4000, "bf16", False, 1)  # greedy
    c.target.fill_(1.0)
    c.tokens.fill_(0)
    got = c.run()
    assert (got["accepted"] == 1).all() and (got["token"] == 0).all()
    c.temperature.fill_(1.0)
    c.noise.fill_(0.25)  # a race in which all are equal, after a rejection of token 0
    c.uniform.fill_(0.5)
    got = c.run()
    assert (got["accepted"] == 0).all() and (got["token"][:, 0] == 1).all()
    c.noise[:, 777:] = 0.0  # a variate of 0 wins, the lowest of several
    assert (c.run()["token"][:, 0] == 777).all()
    c.noise.fill_(float("nan"))
    c.noise[:, 3] = 2.0  # variates that are no numbers, or negative, never win
    c.noise[:, 4] = -1.0
    assert (c.run()["token"][:, 0] == 3).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("greedy", [0, 1])
def test_rows_without_a_distribution(dtype, greedy):
    """A sequence ends, with a status, at a row that is empty or holds a NaN or +infinity; other
    sequences go on."""
    c = Case(8, 3, 700, dtype, True, greedy)
    c.uniform.fill_(0.0)  # with these every draft is accepted
    if greedy:
        for b in range(8):
            c.tokens[b] = c.target[b, :3].float().argmax(1).int()
    c.target[1, 0] = -math.inf
    c.target[2, 1, 5] = math.nan
    c.target[3, 3, 699] = math.inf
    c.target[4, 2] = math.nan
    lowest = torch.finfo(TYPES[dtype]).min
    c.target[5, 1] = lowest  # the type's lowest value is a value: all equal
    c.tokens[5, 1] = 0
    c.target[7, 0, 1:] = -math.inf  # one token is left
    c.tokens[7, 0] = 0
    got = c.run()
    assert got["status"].tolist() == [0, 1, 1, 1, 1, 0, 0, 0]
    assert got["accepted"].tolist() == [3, 0, 1, 3, 2, 3, 3, 3]
    for b, i in ((1, 0), (2, 1), (3, 3), (4, 2)):
        assert got["token"][b, i] == -1
    # rows of the draft model
    if not greedy:
        d = Case(4, 3, 700, dtype, True)
        d.uniform.fill_(0.0)
        d.draft[1, 1] = -math.inf
        d.draft[2, 0, 3] = math.nan
        got = d.run()
        assert got["status"].tolist() == [0, 1, 1, 0] and got["accepted"].tolist() == [3, 1, 0, 3]
        d.check(got)
    # masks that leave a row empty
    m = Case(3, 2, 333, dtype, False, greedy, allowed=True)
    m.on[1, 0] = False
    m.pack()
    got = m.run()
    assert got["status"][1] == 1 and got["accepted"][1] == 0 and got["token"][1].tolist() == [-1, -1, -1]
    assert got["prob"][1, 0] == 0
    m.on[1, 0, 0] = True  # (the row itself is checked on the other sequences)
    assert got["status"][0] == 0 and got["status"][2] == 0


@gpu
@needs_gpu
def test_bad_lengths_temperatures_and_tokens_end_a_sequence_not_the_call():
    c = Case(7, 4, 600, "f32", True, ragged=True)
    c.lengths.copy_(torch.tensor([4, -1, 5, 2, 4, 4, 1 << 30], dtype=torch.int32))
    c.temperature[3], c.temperature[4] = -1.0, math.nan
    c.tokens[0, 1], c.tokens[5, 0] = 600, -7
    got = c.run()
    assert got["status"].tolist()[1:5] == [1, 1, 1, 1] and got["status"][6] == 1
    assert got["status"][0] == 0 and got["status"][5] == 0
    for b in (1, 2, 3, 4, 6):
        assert got["accepted"][b] == 0 and (got["token"][b] == -1).all() and (got["prob"][b] == 0).all()
    assert got["accepted"][0] <= 1 and got["accepted"][5] == 0
    n = Case(2, 1, 100, "f32", False, 2)  # sequence 0 is greedy, sequence 1 needs variates that are not there
    n.noise = None
    got = n.run()
    assert got["status"].tolist() == [0, 1]


@gpu
@needs_gpu
def test_nothing_drafted():
    """D = 0: rows that are empty or hold no number, offsets of logits that grow along the row, lengths that are
    not 0, and temperatures, as with drafts."""
    c = Case(9, 0, 777, "bf16", False, allowed=True)
    c.temperature.copy_(torch.tensor([1.0, 0.0, 1.0, 0.0, 1.0, 1e-30, math.inf, -1.0, 1.0]))
    c.target[2, 0, 776] = math.nan
    c.on[2, 0, 776] = True
    c.target[3, 0, 5] = math.inf
    c.on[3, 0, 5] = True
    c.on[4] = False
    c.target[5, 0, 388] = 1000.0
    c.pack()
    c.lengths = torch.tensor([0, 0, 0, 0, 0, 0, 0, 0, 1], dtype=torch.int32, device="cuda")
    got = c.run()
    assert got["status"].tolist() == [0, 0, 1, 1, 1, 0, 0, 1, 1]
    assert (got["accepted"] == 0).all() and got["token"][5, 0] == 388
    assert (got["token"][got["status"] == 1] == -1).all()
    d = Case(3, 0, 60000, "f32", False)
    d.target += torch.linspace(-300, 300, 60000, device="cuda")  # the maximum rises in every thread's part
    d.check(d.run())
    d.target.copy_(d.target.flip(2))
    d.check(d.run())


@gpu
@needs_gpu
def test_extreme_temperatures():
    c = Case(4, 2, 900, "f32", True)
    c.temperature.copy_(torch.tensor([1e-30, 1e30, math.inf, 1e-6], device="cuda"))
    c.target[:, :, 17] = 30.0  # one largest logit: a vanishing temperature leaves it alone
    c.draft[:, :, 17] = 30.0
    c.draft[:, :, 20] = -math.inf
    c.target[1, :, 21] = -math.inf
    c.tokens[:] = 17
    got = c.run()
    assert (got["status"] == 0).all()
    for b in (0, 3):
        assert got["accepted"][b] == 2 and got["token"][b].tolist() == [17, 17, 17]
        assert (got["prob"][b] == 1).all()
    np.testing.assert_allclose(got["prob"][2], 1 / 900, rtol=1e-4)  # equal shares
    np.testing.assert_allclose(got["prob"][1], 1 / 899, rtol=1e-4)


@gpu
@needs_gpu
def test_greedy_reads_neither_random_numbers_nor_drafts():
    c = Case(4, 3, 1200, "bf16", True, 1)
    c.draft.fill_(math.nan)
    c.uniform.fill_(math.nan)
    c.noise.fill_(math.nan)
    a = c.run()
    c.check(a)
    c.uniform = c.noise = None
    b = c.run(draft=None)
    for k in a:
        assert np.array_equal(a[k], b[k])


@gpu
@needs_gpu
def test_strides_and_shared_rows():
    """Logits whose sequences and rows lie anywhere, and a target row that all share."""
    base = Case(3, 2, 1000, "f16", True)
    want = base.run()
    t = torch.full((3, 3, 1007), math.nan, dtype=torch.float16, device="cuda").transpose(0, 1)[:, :, 3:1003]
    t.copy_(base.target)
    d = torch.full((2, 3, 1001), math.nan, dtype=torch.float16, device="cuda").transpose(0, 1)[:, :, 1:]
    d.copy_(base.draft)
    e = torch.full((3, 1003), math.nan, device="cuda")[:, 3:]
    e.copy_(base.noise)
    base.target, base.draft, base.noise = t, d, e
    got = base.run()
    assert np.array_equal(got["token"], want["token"]) and np.array_equal(got["accepted"], want["accepted"])
    np.testing.assert_allclose(got["prob"], want["prob"], rtol=1e-5)
    base.check(got)


@gpu
@needs_gpu
def test_offsets_beyond_32_bits():
    far = (1 << 31) + 16
    c = Case(2, 0, 500, "bf16", False)
    want = c.run()
    t = torch.zeros(far + 500, dtype=torch.bfloat16, device="cuda").as_strided((2, 1, 500), (far, 500, 1))
    t.copy_(c.target)
    c.target = t
    assert np.array_equal(c.run()["token"], want["token"])


@gpu
@needs_gpu
def test_graphs_streams_and_repeats_agree():
    """Two captured graphs with workspaces of their own on two streams at once; new inputs in the same
    buffers are the ones that count."""
    c = Case(6, 4, 20000, "bf16", True, 3, True)
    want = c.run()
    outs, graphs = [], []
    for _ in range(2):
        o = [torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, 5, dtype=torch.int32, device="cuda"),
             torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, 4, device="cuda")]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                rpd.verify(c.target, c.tokens, c.uniform, c.noise, *o, draft=c.draft, lengths=c.lengths,
                           temperature=c.temperature)
        outs.append(o)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in outs:
        for k, v in zip(("accepted", "token", "status", "prob"), o):
            assert np.array_equal(v.cpu().numpy(), want[k])
    fresh = Case(6, 4, 20000, "bf16", True, 3, True, seed=1)
    for k in ("target", "draft", "tokens", "uniform", "noise", "lengths", "temperature"):
        getattr(c, k).copy_(getattr(fresh, k))
    graphs[0].replay()
    torch.cuda.synchronize()
    c.check({k: v.cpu().numpy() for k, v in zip(("accepted", "token", "status", "prob"), outs[0])})
    del graphs


@gpu
@needs_gpu
def test_threads_and_streams_without_workspaces_given():
    """Calls of several threads on the default stream, one of them with a head in between, and one's on a
    stream of its own: each works in a workspace that no other call is using."""
    cases = [Case(5, 4, 20011, "bf16", True, 2, True, seed=s) for s in range(3)]
    want = [c.run() for c in cases]
    V, d = 3001, 256
    head = rpd.QuantHead(d, V, 64)
    head.set_weights(torch.randint(0, 256, (V, d // 2), dtype=torch.uint8, device="cuda"),
                     torch.rand(V, d // 64, device="cuda").bfloat16())
    x = torch.randn(20, d, device="cuda").bfloat16()
    logits = torch.empty(20, V, device="cuda")
    head.logits(x, logits)
    want_logits = logits.clone()
    own, failures = torch.cuda.Stream(), []

    def work(c, want, stream, with_head):
        try:
            o = [torch.zeros(40, *shape, dtype=t, device="cuda") for shape, t in (
                ((5,), torch.int32), ((5, 5), torch.int32), ((5,), torch.int32), ((5, 4), torch.float32))]
            y = torch.zeros(40, 20, V, device="cuda")
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for i in range(40):
                    rpd.verify(c.target, c.tokens, c.uniform, c.noise, *[t[i] for t in o], draft=c.draft,
                               lengths=c.lengths, temperature=c.temperature)
                    if with_head:
                        head.logits(x, y[i])
            torch.cuda.synchronize()
            for k, t in zip(("accepted", "token", "status", "prob"), o):
                assert all(np.array_equal(r, want[k]) for r in t.cpu().numpy()), k
            assert not with_head or all(torch.equal(r, want_logits) for r in y)
        except BaseException as e:
            failures.append(e)

    threads = [threading.Thread(target=work, args=(c, w, s, h)) for c, w, s, h in zip(
        cases, want, (torch.cuda.default_stream(), torch.cuda.default_stream(), own), (False, True, False))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    head.close()
    assert not failures, failures


@gpu
@needs_gpu
def test_head_then_verification():
    """The two operators together, as a decoder runs them: a 4-bit draft head proposes a token behind every
    position, the target's 4-bit head reads out its hidden states, the drafts are verified, on one stream
    and in one captured graph."""
    B, D, d, V = 3, 4, 256, 5000
    g = torch.Generator(device="cuda").manual_seed(3)
    dev = dict(device="cuda", generator=g)

    def head(seed):
        gg = torch.Generator(device="cuda").manual_seed(seed)
        h = rpd.QuantHead(d, V, 64)
        h.set_weights(torch.randint(0, 256, (V, d // 2), dtype=torch.uint8, device="cuda", generator=gg),
                      (torch.rand(V, d // 64, device="cuda", generator=gg) * 0.02 + 0.02).bfloat16())
        return h

    target_head, draft_head = head(1), head(1)
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    hidden = torch.randn(B, D + 1, d, **dev).bfloat16()
    guess = (hidden[:, :D].float() + 0.2 * torch.randn(B, D, d, **dev)).bfloat16().contiguous()
    c = Case(B, D, V, "bf16", True)
    c.target = torch.zeros(B, D + 1, V, dtype=torch.bfloat16, device="cuda")
    c.draft = torch.zeros(B, D, V, dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, D + 1, dtype=torch.int32, device="cuda"),
            torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, D, device="cuda")]

    def step():
        draft_head.logits(guess.view(B * D, d), c.draft.view(B * D, V), gain=gain)
        c.tokens.copy_(c.draft.argmax(2))
        target_head.logits(hidden.view(-1, d), c.target.view(-1, V), gain=gain)
        rpd.verify(c.target, c.tokens, c.uniform, c.noise, *outs, draft=c.draft, temperature=c.temperature)

    step()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]
    got = {k: v.cpu().numpy() for k, v in zip(("accepted", "token", "status", "prob"), outs)}
    c.check(got)
    assert got["accepted"].sum() > 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for o in outs:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, outs):
        assert torch.equal(a, b)
    target_head.close()
    draft_head.close()
