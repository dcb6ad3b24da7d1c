"""The 8-bit head and sampling where they can go wrong: waits that run out, weights set again, streams and threads and captured
graphs, magnitudes, refusals with a head, and a run of the operators together.  Tolerances as in test_fp8_head.py."""
import threading

import pytest
import torch

import paper_2609_36452_gb300 as rpd
from test_fp8_head import TYPES, check, expected, head_of, make, to_codes

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")


@gpu
@needs_gpu
def test_refusals_with_a_head():
    h = rpd.Fp8Head(64, 100)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full((2, 100), 7.0, device="cuda")
    with pytest.raises(rpd.RpdError) as e:
        h.logits(x, out)
    assert e.value.code == rpd.RPD_ERR_NO_HEAD
    codes = torch.zeros(100, 64, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.ones(1, 1, device="cuda")
    for bad in ((codes.cpu(), scales), (codes, scales.half()), (codes[:, :63], scales), (codes, torch.ones(2, 1, device="cuda")),
                (codes.float(), scales)):
        with pytest.raises(rpd.RpdError):
            h.set_weights(*bad)
    h.set_weights(codes.view(torch.uint8), scales)
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(x=x.float()), dict(x=x[:, :63]), dict(x=x.cpu()), dict(out=out[:1]), dict(out=out.int()), dict(gain=gain.half()),
               dict(gain=gain[:63]), dict(x=x[:1].expand(2, 64)), dict(gain=gain, eps=float("nan")), dict(gain=gain, eps=-1.0),
               dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(rpd.RpdError) as e:
            h.logits(**dict(dict(x=x, out=out), **kw))
        assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    for bad in (999, 60000001):
        with pytest.raises(rpd.RpdError):
            h.set_wait_limit(bad)
    torch.cuda.synchronize()
    assert (out == 7).all()
    h.logits(x[:0], out[:0])  # nothing to do
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out.zero_()
        with pytest.raises(rpd.RpdError) as e:
            h.set_weights(codes, scales)
        assert e.value.code == rpd.RPD_ERR_INVALID_ARGUMENT
    h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("rows", [3, 128, 300])
def test_waits_that_run_out_leave_nan_and_a_usable_head(rows):
    c = make(640, 60000, rows, True)
    h = head_of(c)
    h.set_wait_limit(2000)
    h.inject_stall(True)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    assert c["out"].isnan().all()
    h.inject_stall(False)
    h.set_wait_limit(2000000)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)


@gpu
@needs_gpu
def test_workspace_of_any_content_and_weights_set_again():
    c = make(256, 5003, 40, False)
    h = head_of(c)
    need = rpd.rpd_fp8_workspace(h.handle, 40)
    assert need > 0 and rpd.rpd_fp8_workspace(h.handle, 0) == 0 and rpd.rpd_fp8_workspace(h.handle, -1) == -1
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    h.logits(c["x"], c["out"], workspace=ws[:need])
    torch.cuda.synchronize()
    check(c)
    assert (ws[need:] == 0xFF).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.logits(c["x"], c["out"], workspace=ws[:need])
    other = make(256, 5003, 40, False, seed=7)
    h.set_weights(other["codes"], other["scales"])  # the captured call has the new weights
    c["codes"], c["scales"] = other["codes"], other["scales"]
    for _ in range(3):
        c["buffer"].fill_(77)
        ws.fill_(0x7F)
        g.replay()
        torch.cuda.synchronize()
        check(c)


@gpu
@needs_gpu
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("norm", [False, True])
def test_magnitudes(size, norm):
    """Rows whose squares leave fp32 and whose scales are far from 1; a row of zeros, as a batch is padded with."""
    c = make(384, 700, 5, norm, size=size)
    c["x"][2] = 0
    c["scales"].fill_(1.0 if norm else min(1e20, 1 / size))
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    if norm:
        x = c["x"].double()
        rho = ((x ** 2).mean(1, keepdim=True) + c["eps"]).rsqrt()
        u = (c["x"].float() * c["gain"].float()).to(c["x"].dtype)
    else:
        rho, u = 1.0, c["x"]
    q, s = to_codes(u, 1)
    u = q.double() * s.double().repeat_interleave(128, 1)[:, :384]
    w = c["codes"].double() * c["scales"].double().repeat_interleave(128, 0)[:700].repeat_interleave(128, 1)[:, :384]
    y, S = (u @ w.t()) * rho, (u.abs() @ w.abs().t()) * rho
    tol = 25 * 2.0 ** -23 * S + 48 * 2.0 ** -24 * y.abs() + 2.0 ** -149
    assert ((c["out"].double() - y).abs() <= tol).all()
    assert (c["out"][2] == 0).all()


@gpu
@needs_gpu
def test_rows_of_every_count_between_tiles():
    c = make(300, 3000, 400, True, out="bf16")
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    whole = c["out"].clone()
    for n in (1, 2, 7, 8, 9, 24, 25, 31, 32, 33, 127, 128, 129, 255, 256, 257, 383, 399):
        c["out"].fill_(3)
        h.logits(c["x"][:n], c["out"][:n], gain=c["gain"], eps=c["eps"])
        torch.cuda.synchronize()
        # another division of the work: sums in another order
        part = dict(c, rows=n, x=c["x"][:n], out=c["out"][:n], buffer=c["buffer"][:n])
        check(part)
        assert (c["out"][n:] == 3).all()
    assert whole.isfinite().all()


@gpu
@needs_gpu
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [25, 128, 200])
def test_rows_of_logits_at_any_address(rows, out):
    """Strides and first columns of every alignment, V that ends anywhere in a tile; what lies around the logits stays."""
    for V in (1, 63, 128, 193, 383, 513):
        c = make(200, V, rows, True, out=out)
        h = head_of(c)
        for apart in range(9):
            for first in (0, 1, 2, 4, 8):
                buffer = torch.full((rows + 2, first + V + apart), 77.0, dtype=TYPES[out], device="cuda")
                c["out"] = buffer[:rows, first:first + V]
                c["buffer"] = buffer[:, first:]
                h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
                torch.cuda.synchronize()
                if apart == first == 0:
                    check(c)
                    want = c["out"].clone()
                assert torch.equal(c["out"], want), (V, apart, first)
                assert (buffer[:, :first] == 77).all() and (buffer[:, first + V:] == 77).all(), (V, apart, first)
                assert (buffer[rows:] == 77).all(), (V, apart, first)
        h.close()


@gpu
@needs_gpu
@pytest.mark.parametrize("more,out,pad", [(1, "bf16", 0), (24, "f32", 1), (25, "f16", 2), (200, "bf16", 5)])
def test_more_rows_than_a_launch_takes(more, out, pad):
    most = 1 << 14
    c = make(130, 70, most + more, True, out=out, pad=pad)
    h = head_of(c)
    h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])
    torch.cuda.synchronize()
    check(c)
    whole = c["out"].clone()
    for rows in (slice(0, most), slice(most, None)):
        c["out"].fill_(3)
        h.logits(c["x"][rows], c["out"][rows], gain=c["gain"], eps=c["eps"])
        torch.cuda.synchronize()
        assert torch.equal(c["out"][rows], whole[rows])
    h.close()


@gpu
@needs_gpu
def test_two_streams_and_threads():
    cases = [make(512, 20000, r, True, seed=r) for r in (5, 200)]
    h = head_of(cases[0])
    for c in cases:
        c["codes"], c["scales"] = cases[0]["codes"], cases[0]["scales"]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()

    def work(c, s):
        with torch.cuda.stream(s):
            for _ in range(20):
                h.logits(c["x"], c["out"], gain=c["gain"], eps=c["eps"])

    threads = [threading.Thread(target=work, args=a) for a in zip(cases, streams)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    for c in cases:
        check(c)


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_quantise_strides_and_magnitudes(kind):
    for high in (1, 128):
        x = torch.randn(200, 700, device="cuda") * torch.logspace(-40, 30, 200, device="cuda")[:, None]
        x[5], x[7, 3], x[9, :] = 0, -1e-42, 448 * 2.0 ** -20
        x = x.to(TYPES[kind])
        buffer = torch.full((200, 1400), 0x55, dtype=torch.uint8, device="cuda")
        codes, scales = buffer[:, 3:703], torch.empty(-(-200 // high), 6, device="cuda")
        rpd.quantize_fp8(x, codes, scales, block_rows=high)
        torch.cuda.synchronize()
        q, s = to_codes(x, high)
        assert torch.equal(scales, s)
        assert torch.equal(codes.contiguous().view(torch.float8_e4m3fn).float(), q.float())
        assert (buffer[:, :3] == 0x55).all() and (buffer[:, 703:] == 0x55).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("high", [1, 128])
@pytest.mark.parametrize("cols", [8, 127, 128, 300, 384])
def test_codes_at_any_address(cols, high):
    """First columns and strides of every alignment; what lies around the codes stays."""
    rows = 150
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(cols)).cuda().bfloat16()
    want = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(-(-rows // high), -(-cols // 128), device="cuda")
    rpd.quantize_fp8(x, want, scales, block_rows=high)
    q, s = to_codes(x.float(), high)
    assert torch.equal(want, q.view(torch.uint8)) and torch.equal(scales, s)
    for first in range(9):
        for apart in range(5):
            buffer = torch.full((rows + 2, first + cols + apart), 0x55, dtype=torch.uint8, device="cuda")
            again = torch.zeros_like(scales)
            rpd.quantize_fp8(x, buffer[:rows, first:first + cols], again, block_rows=high)
            assert torch.equal(buffer[:rows, first:first + cols], want) and torch.equal(again, scales), (first, apart)
            assert (buffer[:, :first] == 0x55).all() and (buffer[:, first + cols:] == 0x55).all() and (buffer[rows:] == 0x55).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("high", [1, 128])
def test_zeros_keep_their_sign(high, kind):
    x = torch.tensor([0.0, -0.0, 1.5, -1e-6, 1e-6, -2.0, -0.0, 0.0]).repeat(130, 20).to(TYPES[kind]).cuda()
    x[:, 128:] *= 0.0  # a block of zeros of both signs
    q, s = to_codes(x, high)
    codes = torch.full((130, 160), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(s.shape, device="cuda")
    rpd.quantize_fp8(x, codes, scales, block_rows=high)
    assert torch.equal(codes, q.view(torch.uint8)) and torch.equal(scales, s)


@gpu
@needs_gpu
def test_quantise_every_quotient_of_8_bit_mantissas():
    """All pairs of bf16 mantissas as a block's largest number and another one: where ties are."""
    m = torch.arange(128, 256, device="cuda").float()
    for shift in range(0, 12):
        x = torch.zeros(128, 128, device="cuda")
        x[:, 0] = m * 2.0 ** shift
        x = torch.cat([x[:, :1], (m[None, :127]).expand(128, 127)], 1)
        x = torch.where(x > x[:, :1], x / 2, x).to(torch.bfloat16)
        codes, scales = torch.empty(128, 128, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(128, 1, device="cuda")
        rpd.quantize_fp8(x, codes, scales)
        q, s = to_codes(x, 1)
        assert torch.equal(scales, s) and torch.equal(codes.float(), q.float())


@gpu
@needs_gpu
def test_operators_together_in_a_graph():
    """Weights to 8 bits, a target's rows through the head, their likely tokens, and drafts verified among these: captured once,
    and replayed with new activations."""
    d, V, B, D = 320, 9001, 3, 4
    g = torch.Generator(device="cuda").manual_seed(0)
    dev = dict(device="cuda", generator=g)
    w = (torch.randn(V, d, **dev) * 0.05).bfloat16()
    codes, scales = torch.empty(V, d, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(-(-V // 128), -(-d // 128), device="cuda")
    rpd.quantize_fp8(w, codes, scales, block_rows=128)
    h = rpd.Fp8Head(d, V)
    h.set_weights(codes, scales)
    rows = B * (D + 1)
    x = torch.randn(rows, d, **dev).bfloat16()
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    z = torch.empty(rows, V, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    token, status, kept = i32(rows), i32(rows), i32(rows)
    mask = i32(rows, -(-V // 32))
    u = torch.rand(rows, **dev)
    top_p = torch.full((rows,), 0.8, device="cuda")
    tokens, uniform, noise = i32(B, D), torch.rand(B, D, **dev), torch.empty(B, V, device="cuda").exponential_(generator=g)
    accepted, out_token, out_status = i32(B), i32(B, D + 1), i32(B)

    def calls():
        h.logits(x, z, gain=gain)
        rpd.sample(z, u, token, status, top_p=top_p, out_kept=kept, out_allowed=mask)
        tokens.copy_(token.view(B, D + 1)[:, :D])
        rpd.verify(z.view(B, D + 1, V), tokens, uniform, noise, accepted, out_token, out_status, allowed=mask)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        x.copy_(torch.randn(rows, d, **dev).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (z, token, kept, mask, accepted, out_token)]
        c = dict(x=x, gain=gain, eps=1e-6, codes=codes, scales=scales, d=d, V=V, out=z, out_type="f32", buffer=z)
        check(c)
        assert (status == 0).all() and (out_status == 0).all()
        bits = ((mask[:, :, None] >> torch.arange(32, device="cuda")) & 1).flatten(1)[:, :V].bool()
        assert (bits.sum(1) == kept).all() and bits.gather(1, token[:, None].long()).all()
        p = torch.softmax(z.double(), 1)
        inside = (p * bits).sum(1)
        edge = torch.where(bits, p, 2.0).amin(1)
        assert (inside >= 0.8 - 1e-9).all() and (inside - edge < 0.8 + 1e-9).all()
        assert bits.view(B, D + 1, V).gather(2, out_token[:, :1, None].long().clamp(min=0)).all()
        x2 = x.clone()
        calls()  # the same outside of the graph
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (z, token, kept, mask, accepted, out_token))) and torch.equal(x, x2)


@gpu
@needs_gpu
def test_sampling_on_streams_and_rows_that_are_shared():
    z = torch.randn(1, 40000, device="cuda").mul_(3)
    u = torch.linspace(0, 0.999, 64, device="cuda")
    outs = []
    for s in [torch.cuda.Stream() for _ in range(4)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            token, status = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
            rpd.sample(z.expand(64, 40000), u, token, status)
            outs.append((token, status))
    torch.cuda.synchronize()
    w = torch.exp(z[0].double() - z[0].double().max())
    order = torch.sort(z[0], descending=True, stable=True).indices
    total = w[order].cumsum(0)
    want = order[(total[None] <= u.double()[:, None] * total[-1]).sum(1)]
    for token, status in outs:
        assert (status == 0).all() and torch.equal(token.long(), want)


@gpu
@needs_gpu
def test_sampling_beyond_32_bits():
    """The last row begins behind 2^32 bytes and 2^31 elements."""
    V, stride = 1000, 1 << 28
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 20 GB")
    base = torch.zeros(9 * stride + V, dtype=torch.bfloat16, device="cuda")
    z = base.as_strided((10, V), (stride, 1))
    z.copy_(torch.randn(10, V, device="cuda"))
    z[9, 123] = 50
    token, status, kept = (torch.zeros(10, dtype=torch.int32, device="cuda") for _ in range(3))
    rpd.sample(z, torch.full((10,), 0.5, device="cuda"), token, status, top_p=torch.full((10,), 0.9, device="cuda"), out_kept=kept)
    torch.cuda.synchronize()
    assert (status == 0).all() and int(token[9]) == 123 and int(kept[9]) == 1
