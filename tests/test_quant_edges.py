"""The 4-bit head (rpd_quant_*) at its edges: activations of any size under a norm, the accuracy that is promised, calls
that fail or give up.  Where not said otherwise, bounds are those of test_quant_head.py."""
import ctypes

import pytest
import torch

import paper_2609_36452_gb300 as rpd
from test_quant_head import TYPES, check, head_of, make, reference, weights

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


def rounding_steps(d, group, norm):
    """The error of a logit in units of 2^-23 of the logits' norm, as the root of a sum of squares.  A group is summed in
    n = group / 16 steps, the sum after step i having i / n of the variance of a group's: each cuts off at most 2^-23 of it.
    The m = d / group groups are added up with a rounding of at most half of that each.  The group's scale and the two
    factors round a logit three times more; rho, under a norm, is a chain of 40 roundings of at most half of that each."""
    n, m = group // 16, -(-d // group)
    inside = sum(i / n for i in range(1, n + 1))
    outside = sum(i / m for i in range(1, m + 1)) / 4
    return (inside + outside + 3 / 4 + (40 / 4 if norm else 0)) ** 0.5


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V", [(1, 4096), (16, 4096), (20, 20000), (64, 20000), (128, 20000)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_error_in_units_of_the_logits_norm(rows, V, group, zeros, norm):
    """At d = 4096 the fp32 logits' error lies below what fp32 sums of exact products may leave, relative to the logits'
    norm: weights rounded to 16 bits, group sums in 16 bits (both some 10^-3) or operands that the tensor core
    lines up worse (1.7e-6 with groups of 128) lie above it."""
    c = make(4096, V, rows, group, zeros, norm, seed=group + rows)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    y, _ = reference(c)
    off = (c["out"].double() - y).norm() / y.norm()
    print(f"off {off.item():.3g}")
    assert off <= rounding_steps(4096, group, norm) * 2.0 ** -23
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V", [(3, 600), (20, 600), (20, 5003)])
@pytest.mark.parametrize("x", ["bf16", "f16"])
def test_small_elements_beside_a_large_one(rows, V, x):
    """A row's largest element meets weights of 0: what is 2^-28 of it and more enters exactly, and a smaller one is off by
    at most 2^-39 of the largest."""
    d, group = 256, 64
    c = make(d, V, rows, group, True, False, x=x)
    c["zeros"].fill_(5)
    c["codes"][:, 32] = 0x55  # columns 64 and 65
    c["scales"].fill_(1.0)
    top = 2.0 ** 100 if x == "bf16" else 2.0 ** 15
    gen = torch.Generator(device="cuda").manual_seed(rows)
    small = (1 + torch.rand(rows, d, device="cuda", generator=gen)).to(TYPES[x]).double()
    if x == "bf16":
        small *= top * 2.0 ** -28
    else:  # (fp16 has nothing smaller that is exact)
        small = (small * 2.0 ** -13).to(TYPES[x]).double()
    small[:, 64:66] = 0
    for j in range(2):
        xs = small.clone() if j == 0 or x == "f16" else small * 2.0 ** -9
        xs[:, 64] = top
        c["x"].copy_(xs.to(TYPES[x]))
        assert torch.equal(c["x"].double(), xs)
        h = head_of(c)
        h.logits(c["x"], c["out"])
        torch.cuda.synchronize()
        w = weights(c)
        assert (w[:, 64:66] == 0).all()
        y = xs @ w.t()
        xs[:, 64] = 0
        # the sums' own roundings, of sums of the sizes of the small products alone
        bound = (group / 16 + d / group + 28) * 2.0 ** -23 * (xs.abs() @ w.abs().t())
        if j and x == "bf16":
            bound += 2.0 ** -39 * top * w.abs().sum(1)
        assert ((c["out"].double() - y).abs() <= bound).all()
        h.close()


def test_wait_limits_of_no_head_are_refused():
    assert rpd.rpd_quant_set_wait_limit(None, 5000) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_quant_inject_stall(None, 1) == rpd.RPD_ERR_INVALID_ARGUMENT


@gpu
@needs_gpu
@pytest.mark.parametrize("d,V,rows,group,zeros", [(384, 5003, 20, 128, False), (1024, 40003, 64, 128, True),
                                                  (1024, 40003, 128, 32, True), (8192, 3000, 33, 64, False)])
def test_a_wait_that_runs_out_leaves_nan_and_a_usable_head(d, V, rows, group, zeros):
    """A role of the kernel for many rows that never gets its copies: every other one gives up within the limit, in
    one unit of matrix rows and in several."""
    c = make(d, V, rows, group, zeros, True, pad=8)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    before = c["out"].clone()
    for bad in (0, -5, 999, 60000001):
        with pytest.raises(rpd.RpdError) as e:
            h.set_wait_limit(bad)
        assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    h.set_wait_limit(2000)
    h.inject_stall()
    for _ in range(2):
        h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    few = torch.zeros(8, V, device="cuda")
    h.logits(c["x"][:8], few, gain=c["gain"], eps=c["eps"])  # (the other kernel has no such waits)
    torch.cuda.synchronize()
    assert torch.isnan(c["out"]).all() and torch.isfinite(few).all()
    assert (c["buffer"][rows:] == 77).all() and (c["buffer"][:, V:] == 77).all()
    h.inject_stall(False)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    assert torch.equal(c["out"], before)
    h.close()


class Capture:
    """A stream under capture in the global mode, by the driver's own calls; `blocking`: one that the legacy default stream
    waits for.  What ends it says whether it was still sound."""

    def __init__(self, blocking):
        self.cu = ctypes.CDLL("libcuda.so.1")
        self.stream, self.graph = ctypes.c_void_p(), ctypes.c_void_p()
        assert self.cu.cuStreamCreate(ctypes.byref(self.stream), 0 if blocking else 1) == 0
        assert self.cu.cuStreamBeginCapture_v2(self.stream, 0) == 0

    def end(self):
        rc = self.cu.cuStreamEndCapture(self.stream, ctypes.byref(self.graph))
        if rc == 0:
            self.cu.cuGraphDestroy(self.graph)
        self.cu.cuStreamDestroy_v2(self.stream)
        return rc


@gpu
@needs_gpu
@pytest.mark.parametrize("rows", [3, 20])
def test_weights_are_set_and_heads_closed_while_another_stream_is_captured(rows):
    c, c2 = make(256, 5003, rows, 64, False, True), make(256, 5003, rows, 64, True, True, seed=1)
    h, other = head_of(c), head_of(c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (torch.cuda.default_stream(), side):
        for case in (c2, c):
            capture = Capture(blocking=False)
            try:
                with torch.cuda.stream(stream):
                    h.set_weights(case["codes"], case["scales"], case["zeros"])
                if other.handle:
                    other.close()
            finally:
                rc = capture.end()
            assert rc == 0  # (neither call has ended it)
            h.logits(case["x"], case["out"], gain=case["gain"], eps=case["eps"])
            torch.cuda.synchronize()
            check(case)
    h.close()


@gpu
@needs_gpu
def test_a_refused_call_leaves_the_weights_and_no_error_behind():
    """The legacy default stream cannot be asked for anything while a stream that it waits for is being captured: the call
    fails, the weights stay, and the next call does not report the failure again."""
    c, c2 = make(256, 1000, 5, 64, False, True), make(256, 1000, 5, 64, True, True, seed=1)
    h = head_of(c)
    torch.cuda.synchronize()
    capture = Capture(blocking=True)
    try:
        with pytest.raises(rpd.RpdError) as e:
            h.set_weights(c2["codes"], c2["scales"], c2["zeros"])
    finally:
        capture.end()
    assert e.value.code == rpd.RPD_ERR_CUDA
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    h.set_weights(c2["codes"], c2["scales"], c2["zeros"])
    h.logits(c2["x"], c2["out"], gain=c2["gain"], eps=c2["eps"])
    torch.cuda.synchronize()
    check(c2)
    h.close()


@gpu
@needs_gpu
def test_new_weights_where_there_is_no_room_for_two_layouts():
    """2.4 GB of weights on a device with some 1 GB left: the old ones are freed first; a head that has none fails,
    and works once there is room."""
    c = make(1024, 1 << 22, 2, 32, False, False, out="bf16")
    h, empty = head_of(c), rpd.QuantHead(1024, 1 << 22, 32)
    ref, zeros = c["out"].clone(), torch.full((1 << 22, 32), 8, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    filler = torch.empty(torch.cuda.mem_get_info()[0] - (1200 << 20), dtype=torch.uint8, device="cuda")
    assert torch.cuda.mem_get_info()[0] < 1300 << 20
    with pytest.raises(rpd.RpdError) as e:
        empty.set_weights(c["codes"], c["scales"])
    assert e.value.code == rpd.RPD_ERR_OUT_OF_MEMORY
    h.logits(c["x"], c["out"])
    ref.copy_(c["out"])
    h.set_weights(c["codes"], c["scales"], zeros)
    c["out"].zero_()
    h.logits(c["x"], c["out"])
    torch.cuda.synchronize()
    assert torch.equal(c["out"], ref)
    del filler
    torch.cuda.empty_cache()
    empty.set_weights(c["codes"], c["scales"])
    c["out"].zero_()
    empty.logits(c["x"], c["out"])
    torch.cuda.synchronize()
    assert torch.equal(c["out"], ref)
    h.close()
    empty.close()


@pytest.mark.parametrize("d,V,group", [((1 << 32) + 64, 100, 32), (64, (1 << 32) + 100, 32), (64, 100, (1 << 32) + 32),
                                       (64, 1 << 31, 32)])
def test_sizes_beyond_32_bits_make_no_head(d, V, group):
    with pytest.raises(rpd.RpdError, match="32 bits") as e:
        rpd.QuantHead(d, V, group)
    assert e.value.code == rpd.RPD_ERR_UNSUPPORTED


@gpu
@needs_gpu
def test_rows_beyond_32_bits_are_refused():
    """2^32 + 1 rows of which the C ABI would see one."""
    c = make(64, 40, 1, 32, False, False)
    h = head_of(c)
    for rows in ((1 << 32) + 1, 1 << 31):
        with pytest.raises(rpd.RpdError) as e:
            h.logits(c["x"].expand(rows, 64), c["out"].expand(rows, 40))
        assert e.value.code == rpd.RPD_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert (c["buffer"] == 77).all()
    h.close()
