"""The 4-bit head (rpd_quant_*): refusals (no GPU), and its logits against the definition in 64 bits.

Tolerance.  A logit is a sum over groups of s sum (q - z) u.  The bound is that of s (sum q u - z sum u), a form with
larger sums: the products are exact in fp32, and a group is summed in fp32 in steps of 16 columns (the tensor core may
cut its addends off instead of rounding them: 2^-23 of the sum S of the sizes s (q + z) |u| for every step), the groups'
sums are added up in fp32, as are the sums of u, and at most 16 partial sums are joined.  A logit sees at most
group / 16 + d / group + 28 such roundings.  The activations enter as fp16 numbers scaled by a power of two; the bound
takes them for exact down to 2^-24 of the row's largest, and smaller ones for off by at most 2^-35 of it.  The
kernels sum (q - z) u and are exact down to 2^-28, with 2^-39 below: test_quant_edges.py holds them to that.  The
factor rho is right to 48 * 2^-24 (a chain of at most 40 additions under a square root, rsqrtf's two last places and
a division).  The logit itself is rounded once to the type of the output, by half of its eps or of its smallest
subnormal."""
import ctypes
import os
import threading

import pytest
import torch

import paper_2609_36452_gb300 as rpd

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_SUBNORMAL = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


# ------------------------------------------------------------------------------ refusals

@pytest.mark.parametrize("d,V,group,code", [(0, 16, 32, "INVALID_ARGUMENT"), (64, 0, 32, "INVALID_ARGUMENT"),
                                            (64, 16, 16, "UNSUPPORTED"), (64, 16, 100, "UNSUPPORTED"),
                                            (32769, 16, 32, "UNSUPPORTED"), (64, (1 << 24) + 1, 32, "UNSUPPORTED")])
def test_create_refuses_bad_shapes(d, V, group, code):
    assert not rpd.rpd_quant_create(d, V, group)
    assert rpd.rpd_last_error() != b""


def test_null_head_is_refused():
    assert rpd.rpd_quant_set_weights(None, None, None, 0, None, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_quant_logits(None, None, 0, 0, 1, None, ctypes.c_float(0), None, 0, 0, None, 0,
                                None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_quant_workspace(None, 1) == -1
    rpd.rpd_quant_destroy(None)


def test_create_without_gpu_fails_cleanly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(rpd.RpdError):
        rpd.QuantHead(64, 256, 32)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    """The row checks of the binding, which come before any call into the library."""
    t = torch.zeros(3, 8, dtype=torch.bfloat16)
    with pytest.raises(rpd.RpdError, match="CUDA"):
        rpd._rows_arg(t, "x", (torch.bfloat16,), (3, 8))
    with pytest.raises(rpd.RpdError, match="required"):
        rpd._rows_arg(None, "x", (torch.bfloat16,), (3, 8))


@gpu
@needs_gpu
def test_refusals_with_a_head():
    E = rpd.RpdError
    h = rpd.QuantHead(64, 100, 32)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full((2, 100), 7.0, device="cuda")
    with pytest.raises(E) as e:
        h.logits(x, out)
    assert e.value.code == rpd.RPD_ERR_NO_HEAD
    codes = torch.zeros(100, 32, dtype=torch.uint8, device="cuda")
    scales = torch.ones(100, 2, dtype=torch.bfloat16, device="cuda")
    for bad in ((codes.cpu(), scales, None), (codes, scales.float(), None), (codes[:, :31], scales, None),
                (codes, scales[:50], None), (codes, scales, scales), (codes.int(), scales, None)):
        with pytest.raises(E):
            h.set_weights(*bad)
    h.set_weights(codes, scales)
    for kw in (dict(x=x.float()), dict(x=x[:, :63]), dict(x=x.cpu()), dict(out=out[:1]), dict(out=out.int()),
               dict(gain=torch.zeros(64, dtype=torch.float16, device="cuda")),
               dict(gain=torch.zeros(63, dtype=torch.bfloat16, device="cuda")),
               dict(x=torch.zeros(64, 2, dtype=torch.bfloat16, device="cuda").t()),
               dict(x=x[:1].expand(2, 64)),  # rows that overlap
               dict(gain=torch.ones(64, dtype=torch.bfloat16, device="cuda"), eps=float("nan")),
               dict(gain=torch.ones(64, dtype=torch.bfloat16, device="cuda"), eps=-1.0)):
        with pytest.raises(E) as e:
            h.logits(**dict(dict(x=x, out=out), **kw))
        assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert (out == 7).all()
    h.logits(x[:0], out[:0])  # nothing to do
    h.close()


@gpu
@needs_gpu
def test_workspace_refusals_and_weights_under_capture():
    c = make(256, 5003, 40, 64, False, False)
    h = head_of(c)
    need = rpd.rpd_quant_workspace(h.handle, 40)
    assert need > 0 and rpd.rpd_quant_workspace(h.handle, 16) == 0 and rpd.rpd_quant_workspace(h.handle, -1) == -1
    ws = torch.zeros(need + 256, dtype=torch.uint8, device="cuda")
    for bad in (ws[:need - 1], ws[8:], ws.cpu(), ws.int()):
        with pytest.raises(rpd.RpdError) as e:
            h.logits(c["x"], c["out"], workspace=bad)
        assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_quant_logits(h.handle, c["x"].data_ptr(), 0, 256, 40, None, 0.0, c["out"].data_ptr(), 2, 5003, None, 0,
                                None) == rpd.RPD_ERR_INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert (c["buffer"] == 77).all()
    ws.fill_(0xFF)  # whatever the workspace holds
    h.logits(c["x"], c["out"], workspace=ws)
    torch.cuda.synchronize()
    check(c)
    # new weights wait for the device, which a capture forbids: refused, and the old ones stay
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c["out"].zero_()
        with pytest.raises(rpd.RpdError) as e:
            h.set_weights(c["codes"], c["scales"])
        h.logits(c["x"], c["out"])
    assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    g.replay()
    torch.cuda.synchronize()
    check(c)
    del g
    h.close()


# ------------------------------------------------------------------------------ numerics

def make(d, V, rows, group, zeros, norm, x="bf16", out="f32", scale="bf16", pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = dict(device="cuda", generator=g)
    groups = -(-d // group)
    c = dict(d=d, V=V, rows=rows, group=group, outtype=out,
             codes=torch.randint(0, 256, (V, (d + 1) // 2), dtype=torch.uint8, **dev),
             scales=((torch.rand(V, groups, **dev) - 0.3) * 0.02).to(TYPES[scale]),
             zeros=torch.randint(0, 16, (V, groups), dtype=torch.uint8, **dev) if zeros else None,
             gain=(1 + 0.2 * torch.randn(d, **dev)).to(TYPES[x]) if norm else None, eps=1e-5)
    whole = torch.randn(rows, d + pad, **dev).to(TYPES[x])
    whole[:, d:] = float("nan")  # what lies between the rows is nobody's business
    c["x"] = whole[:, :d]
    c["buffer"] = torch.full((rows + 2, V + pad), 77.0, dtype=TYPES[out], device="cuda")
    c["out"] = c["buffer"][:rows, :V]
    return c


def weights(c, sign=-1):
    """(q - z) s, or the sizes (q + z) |s|, in 64 bits, [V][d]."""
    k = torch.arange(c["d"], device="cuda")
    byte = c["codes"][:, k // 2].long()
    q = torch.where(k % 2 == 0, byte & 15, byte >> 4)
    z = 8 if c["zeros"] is None else c["zeros"][:, k // c["group"]].long()
    s = c["scales"][:, k // c["group"]].double()
    return (q - z).double() * s if sign < 0 else (q + z).double() * s.abs()


def reference(c):
    """Logits in 64 bits and the bound of the kernel's error."""
    u, rho = c["x"].double(), 1.0
    if c["gain"] is not None:
        rho = ((u * u).mean(1, keepdim=True) + c["eps"]).rsqrt()
        u = (c["x"].float() * c["gain"].float()).to(c["x"].dtype).double()
    w = weights(c)
    y = (u @ w.t()) * rho
    sizes = weights(c, 1)
    size = (u.abs() @ sizes.t()) * rho
    steps = c["group"] / 16 + c["d"] / c["group"] + 28
    bound = steps * 2.0 ** -23 * size + 48 * 2.0 ** -24 * y.abs()
    bound += 2.0 ** -35 * u.abs().amax(1, keepdim=True) * rho * sizes.sum(1)
    bound += torch.finfo(TYPES[c["outtype"]]).eps / 2 * (y.abs() + bound) + HALF_SUBNORMAL[c["outtype"]]
    return y, bound


def head_of(c):
    h = rpd.QuantHead(c["d"], c["V"], c["group"])
    h.set_weights(c["codes"], c["scales"], c["zeros"])
    return h


def check(c, out=None):
    y, bound = reference(c)
    err = ((c["out"] if out is None else out).double() - y).abs()
    assert torch.isfinite(err).all()
    worst = (err / bound).max().item()
    assert worst <= 1, worst
    if out is None:  # nothing around the logits has been touched
        assert (c["buffer"][c["rows"]:] == 77).all() and (c["buffer"][:, c["V"]:] == 77).all()


SHAPES = [
    # d, V, rows, group, zeros, norm, x, out, scale, pad
    (1, 1, 1, 32, False, False, "bf16", "f32", "bf16", 0),
    (2, 3, 2, 128, True, True, "f16", "f16", "f16", 1),
    (31, 16, 3, 32, True, False, "bf16", "f32", "f16", 0),
    (33, 17, 8, 32, False, True, "bf16", "bf16", "bf16", 0),
    (64, 15, 9, 64, True, True, "bf16", "f32", "bf16", 8),
    (65, 255, 16, 64, False, False, "f16", "f32", "bf16", 3),
    (128, 256, 1, 128, False, True, "bf16", "f32", "bf16", 0),
    (129, 257, 17, 128, True, True, "bf16", "bf16", "bf16", 0),
    (200, 1000, 33, 128, True, False, "f16", "f16", "f16", 5),
    (256, 4096, 1, 32, False, True, "bf16", "f32", "bf16", 0),
    (1001, 5003, 13, 32, True, False, "f16", "f16", "f16", 3),
    (1001, 5003, 70, 64, True, True, "bf16", "f32", "f16", 3),
    (3584, 2432, 5, 64, True, True, "bf16", "bf16", "f16", 0),
    (4096, 15872, 20, 128, True, True, "bf16", "bf16", "bf16", 0),
    (4096, 2500, 16, 128, False, False, "bf16", "f32", "bf16", 0),
    (4096, 2433, 128, 128, False, True, "bf16", "bf16", "bf16", 0),
    (4096, 999, 129, 32, True, True, "f16", "f32", "f16", 8),
    (8192, 300, 14, 64, False, True, "bf16", "f32", "bf16", 0),
    (8192, 300, 100, 64, True, True, "bf16", "f32", "bf16", 0),
    (256, 5000, 20, 32, False, True, "bf16", "f32", "bf16", 0),
    (700, 5000, 40, 32, True, True, "f16", "f32", "f16", 3),
    (700, 4900, 100, 64, False, False, "bf16", "f32", "f16", 8),
    (129, 4865, 17, 128, True, True, "bf16", "bf16", "bf16", 0),
    (200, 4877, 33, 128, False, False, "f16", "f16", "f16", 5),
    (1254, 1022, 80, 64, True, False, "bf16", "f32", "f16", 0),
    (20000, 513, 40, 128, False, True, "bf16", "f32", "bf16", 0),
    (32768, 40, 35, 32, False, True, "f16", "f32", "bf16", 0),
    (32768, 40, 3, 128, True, True, "bf16", "f32", "bf16", 0),
    (32767, 33, 2, 32, False, False, "f16", "f32", "f16", 1),
]


@gpu
@needs_gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(int(v) if isinstance(v, bool) else v) for v in s))
def test_logits_match_the_definition(shape):
    c = make(*shape)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("V,rows", [(700, r) for r in list(range(1, 20)) + [
    24, 31, 32, 33, 47, 48, 49, 63, 64, 65, 96, 127, 128, 130, 257]] + [(4999, r) for r in (
        9, 16, 17, 18, 24, 31, 32, 33, 47, 48, 49, 63, 64, 65, 96, 127, 128, 130, 257)] + [(1022, r) for r in (
            32, 33, 38, 39, 64, 65, 80, 96, 127, 128, 129, 130)])
def test_every_row_count(V, rows):
    """Small heads, whose rows run side by side, and larger ones, by the kernel for many rows."""
    c = make(384, V, rows, 128, True, True, seed=rows)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    h.close()


@gpu
@needs_gpu
def test_millions_of_rows():
    """More passes than a grid has places in its second and third dimension (65535)."""
    c = make(8, 5, 65536 * 64 + 17, 32, True, True)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V", [(2, 130), (40, 130), (40, 5003)])
def test_one_column_at_a_time_lands_in_its_place(rows, V):
    """Unit activations read single columns of the matrix: every code, scale and zero point in place,
    exactly (one product, no sum)."""
    c = make(97, V, rows, 32, True, False, seed=5)
    w = weights(c)
    h = head_of(c)
    for first in range(0, 97, rows):
        c["x"].zero_()
        k = torch.arange(first, min(97, first + rows), device="cuda")
        c["x"][torch.arange(len(k), device="cuda"), k] = 1
        h.logits(c["x"], c["out"])
        assert torch.equal(c["out"][:len(k)].double(), w[:, k].t())
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V", [(3, 300), (33, 300), (33, 5003)])
def test_a_row_that_is_not_finite_stays_alone(rows, V):
    c = make(256, V, rows, 64, False, True)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    before = c["out"].clone()
    c["x"][1, 7] = float("nan")
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    keep = [r for r in range(rows) if r != 1]
    assert torch.equal(c["out"][keep], before[keep])
    assert torch.isnan(c["out"][1]).all()
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V", [(5, 260), (20, 260), (20, 5003)])
@pytest.mark.parametrize("x", ["bf16", "f16"])
def test_rows_of_any_magnitude(rows, V, x):
    """Activations from the type's smallest to its largest numbers, rows of zeros, and rows whose elements
    span its range: a power of two a row brings them into the tensor core's."""
    c = make(192, V, rows, 64, True, False, x=x)
    low, high = (-120, 100) if x == "bf16" else (-20, 8)
    power = torch.linspace(low, high, rows, device="cuda").round()
    c["x"].copy_((torch.randn(rows, 192, device="cuda").double() * torch.exp2(power.double())[:, None]).to(TYPES[x]))
    c["x"][1] = 0
    c["x"][2] = torch.exp2(torch.linspace(low, high, 192, device="cuda").round()).to(TYPES[x])
    c["x"][3] = 0
    c["x"][3, 77] = torch.finfo(TYPES[x]).max
    h = head_of(c)
    c["scales"].mul_(2.0 ** -10)
    h.set_weights(c["codes"], c["scales"], c["zeros"])
    h.logits(c["x"], c["out"])
    torch.cuda.synchronize()
    assert (c["out"][1] == 0).all()
    check(c)
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows", [4, 50])
def test_graphs_streams_and_repeats_agree(rows):
    """Two graphs captured from one head and replayed on two streams at once, a plain call on a third,
    and a repeated call all give the same bits; weights set anew are the ones that are used."""
    c = make(1024, 3000, rows, 128, True, True)
    h = head_of(c)
    outs = [torch.zeros_like(c["out"]) for _ in range(4)]
    h.logits(c["x"], outs[0], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c, outs[0])
    graphs = []
    for o in outs[1:3]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                h.logits(c["x"], o, gain=c["gain"], eps=c["eps"])
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for o in outs[1:]:
        o.zero_()
    torch.cuda.synchronize()
    for s, g in zip(streams, graphs):
        with torch.cuda.stream(s):
            for _ in range(5):
                g.replay()
    with torch.cuda.stream(streams[2]):
        h.logits(c["x"], outs[3], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    del graphs
    c2 = make(1024, 3000, rows, 128, False, True, seed=9)
    h.set_weights(c2["codes"], c2["scales"], c2["zeros"])
    h.logits(c2["x"], c2["out"], gain=c2["gain"], eps=c2["eps"])
    torch.cuda.synchronize()
    check(c2)
    h.close()


@gpu
@needs_gpu
def test_threads_share_a_head():
    c = make(512, 2000, 6, 64, False, True)
    h = head_of(c)
    outs = [torch.zeros(6, 2000, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    errors = []

    def work(o):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    h.logits(c["x"], o, gain=c["gain"], eps=c["eps"])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(o,)) for o in outs]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not errors
    for o in outs:
        check(c, o)
    h.close()


@gpu
@needs_gpu
def test_offsets_beyond_32_bits():
    """Rows of activations and of logits that lie more than 2^32 bytes apart."""
    far = (1 << 31) + 8
    c = make(64, 40, 2, 32, False, False)
    h = head_of(c)
    xs = torch.zeros(far + 64, dtype=torch.bfloat16, device="cuda").as_strided((2, 64), (far, 1))
    xs.copy_(c["x"])
    out = torch.zeros(far + 40, dtype=torch.float16, device="cuda").as_strided((2, 40), (far, 1))
    h.logits(xs, out)
    near = torch.zeros(2, 40, dtype=torch.float16, device="cuda")
    h.logits(c["x"], near)
    assert torch.equal(out, near)
    h.close()
