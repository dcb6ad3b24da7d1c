"""The 8-bit head (rpd_fp8_*) and its quantiser: refusals (no GPU), and results against the definition in 64 bits.

Codes and scales of the quantiser are exact: one fp32 division each and one rounding, which torch does alike.

Tolerance of the logits.  With S the sum of the sizes sw sx |qw qx| of a logit's terms: products of two codes are
exact; the tensor core adds a block of 128 in four steps and may cut its addends off at 2^-23 of the sum so far; the
two scales' product, the multiply-add and the sum over blocks are fp32 (half of 2^-23 each); a tile that several
workers shared has at most 16 partial sums.  So (4 + d / 128 + 16 + 2) 2^-23 S.  The scales relative to a power of
two are exact.  The factor rho is right to 48 * 2^-24 (a chain of at most 40 additions under a square root, rsqrtf's two
last places and a division).  The logit itself is rounded once, by half of its type's eps or smallest subnormal."""
import ctypes
import threading

import pytest
import torch

import paper_2609_36452_gb300 as rpd

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_SUBNORMAL = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


# ------------------------------------------------------------------------------ refusals

@pytest.mark.parametrize("d,V", [(0, 16), (64, 0), (-1, 5), (32769, 16), (64, (1 << 24) + 1), (1 << 30, 1 << 30)])
def test_create_refuses_bad_shapes(d, V):
    assert not rpd.rpd_fp8_create(d, V)
    assert rpd.rpd_last_error() != b""


def test_null_head_is_refused():
    bad = rpd.RPD_ERR_INVALID_ARGUMENT
    assert rpd.rpd_fp8_set_weights(None, None, None, None) == bad
    assert rpd.rpd_fp8_logits(None, None, 0, 0, 1, None, ctypes.c_float(0), None, 0, 0, None, 0, None) == bad
    assert rpd.rpd_fp8_workspace(None, 1) == -1
    assert rpd.rpd_fp8_set_wait_limit(None, 5000) == bad and rpd.rpd_fp8_inject_stall(None, 1) == bad
    rpd.rpd_fp8_destroy(None)


def test_quantise_refusals():
    q = rpd.rpd_fp8_quantize
    assert q(None, 0, 8, 2, 8, 1, None, 8, None, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert q(16, 9, 8, 2, 8, 1, 16, 8, 16, None) == rpd.RPD_ERR_INVALID_ARGUMENT      # type
    assert q(16, 0, 8, -2, 8, 1, 16, 8, 16, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert q(16, 0, 8, 2, 8, 64, 16, 8, 16, None) == rpd.RPD_ERR_UNSUPPORTED
    assert q(16, 0, 7, 2, 8, 1, 16, 8, 16, None) == rpd.RPD_ERR_INVALID_ARGUMENT      # rows overlap
    assert q(16, 0, 8, 2, 8, 1, 16, 7, 16, None) == rpd.RPD_ERR_INVALID_ARGUMENT
    assert q(17, 0, 8, 2, 8, 1, 16, 8, 16, None) == rpd.RPD_ERR_INVALID_ARGUMENT      # alignment
    assert q(None, 0, 8, 0, 8, 1, None, 8, None, None) == rpd.RPD_OK                  # nothing to do
    host = torch.zeros(2, 8, dtype=torch.bfloat16)
    assert q(host.data_ptr(), 0, 8, 2, 8, 1, host.data_ptr(), 8, host.data_ptr(), None) == rpd.RPD_ERR_INVALID_ARGUMENT
    for bad in (dict(x=torch.zeros(3)), dict(x=None), dict(block_rows=2), dict()):  # the last one: host tensors
        with pytest.raises(rpd.RpdError):
            rpd.quantize_fp8(**dict(dict(x=host, codes=torch.zeros(2, 8, dtype=torch.uint8), scales=torch.zeros(2, 1)), **bad))


# ------------------------------------------------------------------------------ definition

def to_codes(x, high):
    """fp32 scales and e4m3 codes (as numbers) of a matrix by the definition."""
    x = x.float()
    rows, cols = x.shape
    R, C = -(-rows // high), -(-cols // 128)
    t = torch.nn.functional.pad(x, (0, C * 128 - cols, 0, R * high - rows)).view(R, high, C, 128)
    scale = t.abs().amax((1, 3))
    scale = scale / torch.full_like(scale, 448.0)
    by = torch.where(scale > 0, scale, torch.ones_like(scale))[:, None, :, None].expand_as(t).contiguous()
    q = (t / by).clamp(-448, 448).to(torch.float8_e4m3fn).view(R * high, C * 128)[:rows, :cols]
    return q, scale


def rows_apart(rows, cols, pad, dtype, fill=0.0):
    buffer = torch.full((rows, cols + pad), fill, dtype=dtype, device="cuda")
    return buffer, buffer[:, :cols]


def make(d, V, rows, norm, x="bf16", out="f32", pad=0, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * d + V + rows)
    dev = dict(device="cuda", generator=g)
    c = dict(d=d, V=V, rows=rows, x_type=x, out_type=out)
    c["codes"] = (112 * torch.randn(V, d, **dev)).clamp(-448, 448).to(torch.float8_e4m3fn)
    c["scales"] = (torch.rand(-(-V // 128), -(-d // 128), **dev) + 0.5) * 2e-4
    _, c["x"] = rows_apart(rows, d, pad, TYPES[x])
    strong = 1 + 6 * (torch.rand(d, **dev) < 0.02).float()
    c["x"].copy_(size * torch.randn(rows, d, **dev) * strong)
    c["gain"] = (1 + 0.2 * torch.randn(d, **dev)).to(TYPES[x]) if norm else None
    c["buffer"], c["out"] = rows_apart(rows, V, pad, TYPES[out], 77.0)
    c["eps"] = 1e-6
    return c


def head_of(c):
    h = rpd.Fp8Head(c["d"], c["V"])
    h.set_weights(c["codes"], c["scales"])
    return h


def expected(c):
    """Logits and S in 64 bits."""
    x, rho = c["x"], 1.0
    u = x.float()
    if c["gain"] is not None:
        u = (u * c["gain"].float()).to(x.dtype).float()
        rho = ((x.double() ** 2).mean(1, keepdim=True) + c["eps"]).rsqrt()
    q, scale = to_codes(u, 1)
    u = q.double() * scale.double().repeat_interleave(128, 1)[:, :c["d"]]
    w = c["scales"].double().repeat_interleave(128, 0)[:c["V"]].repeat_interleave(128, 1)[:, :c["d"]] * c["codes"].double()
    return (u @ w.t()) * rho, (u.abs() @ w.abs().t()) * rho


def check(c):
    y, S = expected(c)
    tol = (4 + -(-c["d"] // 128) + 18) * 2.0 ** -23 * S + 48 * 2.0 ** -24 * y.abs()
    eps = torch.finfo(TYPES[c["out_type"]]).eps / 2
    tol = tol + eps * (y.abs() + tol) + HALF_SUBNORMAL[c["out_type"]]
    off = (c["out"].double() - y).abs()
    assert (off <= tol).all(), (float((off / tol).max()), int((~(off <= tol)).sum()))
    assert (c["buffer"][:, c["V"]:] == 77).all()


CASES = [
    (1, 1, 1, False, "bf16", "f32", 0), (64, 256, 1, True, "bf16", "f32", 0), (128, 128, 3, False, "f16", "f16", 0),
    (130, 257, 5, True, "bf16", "bf16", 1), (1001, 5003, 13, False, "f16", "f16", 3), (256, 4096, 1, True, "bf16", "f32", 0),
    (4096, 4096, 1, True, "bf16", "f32", 0), (4096, 1000, 33, True, "f16", "f32", 8), (640, 38913, 2, False, "bf16", "f32", 0),
    (512, 39168, 128, True, "bf16", "bf16", 0), (32768, 300, 2, True, "bf16", "f32", 0),
    (256, 4096, 129, True, "bf16", "f32", 0), (384, 1000, 300, False, "f16", "bf16", 1), (520, 20000, 257, True, "bf16", "f32", 0),
    (1024, 19713, 512, True, "bf16", "f16", 0), (128, 50021, 1024, False, "bf16", "bf16", 8), (100, 100, 2000, True, "f16", "f32", 3),
]


@gpu
@needs_gpu
@pytest.mark.parametrize("d,V,rows,norm,x,out,pad", CASES)
def test_logits(d, V, rows, norm, x, out, pad):
    c = make(d, V, rows, norm, x, out, pad)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    first = c["out"].clone()
    c["out"].fill_(5)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])  # the same sums in the same order
    torch.cuda.synchronize()
    assert torch.equal(first, c["out"])
    h.close()


QUANTISED = [(1, 1, 0), (1, 128, 0), (5, 127, 1), (16, 4096, 0), (17, 1001, 3), (128, 384, 0), (129, 130, 0), (700, 1000, 8), (3, 8192, 5)]


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,cols,pad", QUANTISED)
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("high", [1, 128])
def test_quantise(rows, cols, pad, kind, high):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    _, x = rows_apart(rows, cols, pad, TYPES[kind])
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g) * 3)
    x[:, :128] *= 1e-3
    x[rows // 2:, 128:256] = 0  # blocks of nothing
    buffer = torch.full((rows, cols + pad), 0x55, dtype=torch.uint8, device="cuda")
    codes = buffer[:, :cols]
    scales = torch.full((-(-rows // high), -(-cols // 128)), -1.0, device="cuda")
    rpd.quantize_fp8(x, codes.view(torch.float8_e4m3fn) if not pad else codes, scales, block_rows=high)
    torch.cuda.synchronize()
    q, s = to_codes(x, high)
    assert torch.equal(scales, s)
    assert torch.equal(codes.contiguous().view(torch.float8_e4m3fn).float(), q.float())
    assert (buffer[:, cols:] == 0x55).all()
