"""Sampling under limits (rpd_sample): refusals (no GPU), and tokens, numbers and masks against a sort in 64 bits.

Whole numbers have to be equal.  That a border of a running sum falls between the kernel's and the reference's sums,
which differ by some 2^-40 of it, has a chance of 10^-6 a row, and the inputs are fixed.  A probability is rounded to fp32
(half of its eps) from a weight that is right to 2^-30, relative."""
import ctypes

import pytest
import torch

import paper_2609_36452_gb300 as rpd

gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF, NAN = float("inf"), float("nan")
BAD = rpd.RPD_ERR_INVALID_ARGUMENT


# ------------------------------------------------------------------------------ refusals

def args(**kw):
    a = rpd.RpdSampleArgs(*([16] * 12), 8, rpd.RPD_TYPE_F32, 2, 8)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), BAD), (dict(V=0), BAD), (dict(type=7), BAD), (dict(V=(1 << 24) + 1), rpd.RPD_ERR_UNSUPPORTED),
    (dict(rows=(1 << 26) + 1), rpd.RPD_ERR_UNSUPPORTED), (dict(logits=None), BAD), (dict(out_token=None), BAD),
    (dict(out_status=None), BAD), (dict(uniform=None, temperature=None), BAD), (dict(row_stride=-8), BAD),
    (dict(logits=18), BAD), (dict(top_k=18), BAD), (dict(out_allowed=17), BAD), (dict(), BAD)])  # the last: no such memory
def test_refusals(kw, code):
    assert rpd.rpd_sample(ctypes.byref(args(**kw)), None) == code
    assert rpd.rpd_last_error() != b""


def test_null_and_nothing():
    assert rpd.rpd_sample(None, None) == BAD
    assert rpd.rpd_sample(ctypes.byref(args(rows=0)), None) == rpd.RPD_OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    z, i = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for bad in (dict(logits=z), dict(logits=z[0]), dict(logits=None), dict(logits=torch.zeros(2, 0))):
        with pytest.raises(rpd.RpdError):
            rpd.sample(bad["logits"], torch.zeros(2), i, i)


# ------------------------------------------------------------------------------ definition

def reference(z, u, T, k, p, m, on):
    """One row in 64 bits: token, status, kept, probability, kept tokens."""
    V = z.shape[0]
    bad = (-1, BAD, 0, 0.0, torch.zeros(V, dtype=torch.bool))
    z = z.double()
    finite = torch.isfinite(z) & on
    if not finite.any() or (on & ~(z < INF)).any() or not T >= 0 or (T > 0 and not 0 <= u < 1) or p != p or not m <= 1:
        return bad
    z = torch.where(finite, z, torch.full_like(z, -INF))
    z, order = torch.sort(z, descending=True, stable=True)
    n = int(finite.sum())
    if T == 0:
        kept, w = 1, torch.ones(1, dtype=torch.float64)
    else:
        T = min(max(T, 1.45e-30), 1.44e37)
        w = torch.exp((z[:n] - z[0]) / T)
        kept = min(n, k) if k > 0 else n
        if p < 1:
            before = w[:kept].cumsum(0) - w[:kept]
            kept = max(1, int((before < p * w[:kept].sum()).sum()))
        if m > 0:
            kept = min(kept, int((w >= m).sum()))
        w = w[:kept]
    place = int((w.cumsum(0) <= (u if T > 0 else 0.0) * w.sum()).sum())
    mask = torch.zeros(V, dtype=torch.bool)
    mask[order[:kept]] = True
    return int(order[place]), 0, kept, float(w[place] / w.sum()), mask


def unpack(words, V):
    return ((words[:, None] >> torch.arange(32)) & 1).flatten()[:V] == 1


def pack(on):
    rows, V = on.shape
    words = -(-V // 32)
    on = torch.nn.functional.pad(on, (0, words * 32 - V)).view(rows, words, 32)
    word = (on.long() << torch.arange(32)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int()


def run_and_check(z, u=None, T=None, k=None, p=None, m=None, on=None, stride=None):
    """z [rows][V] on the CPU; limits as lists."""
    rows, V = z.shape
    buffer = torch.full((rows, stride or V), NAN, dtype=z.dtype)
    buffer[:, :V] = z
    dev = buffer.cuda()
    f = lambda x, d: None if x is None else torch.tensor(x, dtype=d).cuda()  # noqa: E731
    out = {n: torch.full((rows,), -7, dtype=torch.int32, device="cuda") for n in ("token", "status", "kept")}
    prob = torch.full((rows,), -7.0, device="cuda")
    bits = torch.full((rows, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    rpd.sample(dev[:, :V], f(u, torch.float32), out["token"], out["status"], temperature=f(T, torch.float32), top_k=f(k, torch.int32),
               top_p=f(p, torch.float32), min_p=f(m, torch.float32), allowed=None if on is None else pack(on).cuda(), out_kept=out["kept"],
               out_prob=prob, out_allowed=bits)
    torch.cuda.synchronize()
    got = {n: t.cpu() for n, t in out.items()}
    prob, bits = prob.cpu(), bits.cpu()
    one = lambda x, r, d: d if x is None else float(torch.tensor(x[r], dtype=torch.float32))  # noqa: E731
    for r in range(rows):
        want = reference(z[r], one(u, r, 0.0), one(T, r, 1.0), k[r] if k else 0, one(p, r, 1.0), one(m, r, 0.0),
                         torch.ones(V, dtype=torch.bool) if on is None else on[r])
        assert (int(got["token"][r]), int(got["status"][r]), int(got["kept"][r])) == want[:3], r
        assert abs(float(prob[r]) - want[3]) <= (2.0 ** -24 + 2.0 ** -29) * want[3] + 1e-45, r
        full = unpack(bits[r], bits.shape[1] * 32)
        assert torch.equal(full[:V], want[4]) and not full[V:].any(), r
    return got


def gen(seed):
    return torch.Generator().manual_seed(seed)


def logits(rows, V, kind, seed, spread=1.5, peaks=6):
    g = gen(seed)
    z = spread * torch.randn(rows, V, generator=g)
    at = torch.randint(0, V, (rows, peaks), generator=g)
    z.scatter_(1, at, 9 + 2.5 * torch.randn(rows, peaks, generator=g))
    return z.to(TYPES[kind])


LIMITS = [dict(), dict(k=40), dict(p=0.9), dict(m=0.05), dict(k=200, p=0.95, m=0.01), dict(k=3000, p=0.99), dict(p=0.97, m=1e-4),
          dict(p=0.999, T=2.5), dict(T=3.0), dict(k=1), dict(p=0.0), dict(m=1.0), dict(p=1.0, m=1e-30, T=0.3), dict(k=1 << 30)]


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("limit", LIMITS, ids=str)
@pytest.mark.parametrize("rows,V,stride", [(3, 1, None), (2, 7, 11), (3, 33, None), (5, 1000, 1003), (3, 4096, None), (2, 50021, 50026)])
def test_limits(rows, V, stride, limit, kind):
    z = logits(rows, V, kind, V + rows)
    u = torch.rand(rows, generator=gen(5)).tolist()
    run_and_check(z, u, [limit.get("T", 0.8)] * rows, [limit["k"]] * rows if "k" in limit else None,
                  [limit["p"]] * rows if "p" in limit else None, [limit["m"]] * rows if "m" in limit else None, stride=stride)


@gpu
@needs_gpu
@pytest.mark.parametrize("rows,V,kind", [(1, 126464, "bf16"), (40, 126464, "bf16"), (3, 152064, "f32"), (2, 1500001, "f32"), (1, 5000011, "bf16"), (300, 5000, "f16"), (160, 30000, "f32")])
def test_sizes(rows, V, kind):
    g = gen(V)
    z = logits(rows, V, kind, rows)
    on = torch.rand(rows, V, generator=g) < 0.6
    z[(torch.rand(rows, V, generator=g) < 0.01) & ~on] = NAN
    z[(torch.rand(rows, V, generator=g) < 0.01) & ~on] = INF
    r = lambda lo, hi: (lo + (hi - lo) * torch.rand(rows, generator=g)).tolist()  # noqa: E731
    k = torch.randint(0, 400, (rows,), generator=g).tolist()
    T = r(0.4, 1.5)
    T[0] = 0.0
    run_and_check(z, r(0, 1), T, k, r(0.5, 1.05), r(-0.01, 0.02), on)
    run_and_check(z, r(0, 1), r(0.4, 1.5), None, r(0.5, 1.05), None, on)


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [31, 257, 512, 513, 1025, 2047, 2048, 2049])
def test_short_rows(V, kind):
    g = gen(V)
    for stride in (V, V + 3):
        z = logits(24, V, kind, V, spread=0.7, peaks=1)
        on = torch.rand(24, V, generator=g) < 0.8
        on[0], on[1] = False, True
        z[2:5, ::3] = -INF
        z[(torch.rand(24, V, generator=g) < 0.1) & ~on] = NAN
        z[5] = torch.finfo(TYPES[kind]).min
        u = torch.rand(24, generator=g).tolist()
        k = torch.randint(V // 2, V + 2, (24,), generator=g).tolist()
        p = torch.rand(24, generator=g).tolist()
        for kw in (dict(), dict(p=p), dict(k=k), dict(k=k, p=p, m=[1e-3] * 24), dict(p=p, m=[1e-2] * 24), dict(p=[0.999] * 24, T=[3.0] * 24),
                   dict(p=[-INF] * 24, m=[-INF] * 24)):
            run_and_check(z, u, on=on, stride=stride, **kw)


@gpu
@needs_gpu
@pytest.mark.parametrize("V", [5, 2048, 40000, 152064])
def test_equal_logits_and_exact_borders(V):
    z = torch.full((8, V), 3.25)
    z[4:] = torch.tensor([1.0, 2.0]).repeat(V)[:V]
    u = [0.0, 0.5, 0.25, 1 - 2.0 ** -24] * 2
    run_and_check(z, u)
    run_and_check(z, u, p=[0.5, 0.25, 0.75, 1.0] * 2)
    run_and_check(z, u, k=[1, 2, 3, V - 1] * 2, p=[0.5, 0.5, 0.5, 0.5] * 2)
    run_and_check(z.to(torch.bfloat16), u, T=[100.0] * 8, m=[0.99] * 8)


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_masked_places_and_rows_without_tokens(kind):
    V = 3001
    z = logits(12, V, kind, 1)
    on = torch.rand(12, V, generator=gen(2)) < 0.5
    z[0, :] = -INF                       # no finite logit
    on[1, :] = False                     # no token
    z[2, 17], on[2, 17] = NAN, True
    z[3, 17], on[3, 17] = INF, True
    z[4, 17], on[4, 17] = NAN, False     # anything may be there
    z[5, :], z[5, 9], on[5, 9] = -INF, -4.0, True    # one token
    z[6, ~on[6]] = torch.finfo(TYPES[kind]).min
    on[6, :] = True                      # the type's lowest value in place of a mask
    z[7, :] = torch.finfo(TYPES[kind]).min           # and everywhere
    z[8, ::2], z[8, 1::2] = 0.0, -0.0    # equal
    z[9, :], on[9, :] = torch.finfo(TYPES[kind]).max, True
    z[10, 5], on[10, 5] = torch.finfo(TYPES[kind]).max, True
    u = [0.3] * 12
    for kw in (dict(), dict(p=[0.9] * 12), dict(k=[2000] * 12), dict(k=[1800] * 12, p=[0.9999] * 12), dict(m=[0.01] * 12), dict(T=[0.0] * 12)):
        run_and_check(z, u, on=on, **kw)


@gpu
@needs_gpu
def test_bad_numbers_end_in_a_status():
    z = logits(9, 500, "f32", 3)
    u = [0.5, -0.1, 1.0, NAN, 0.5, 0.5, 0.5, 0.5, 0.5]
    T = [1.0, 1.0, 1.0, 1.0, -1.0, NAN, 1.0, 1.0, 1.0]
    p = [0.9] * 6 + [NAN, 0.9, -3.0]
    m = [0.1] * 7 + [1.5, NAN]
    got = run_and_check(z, u, T, None, p, m)
    assert got["status"].tolist() == [0] + [BAD] * 8
    run_and_check(z, None, [0.0] * 9)


@gpu
@needs_gpu
@pytest.mark.parametrize("T", [1e-38, 1e-6, 1e-3, 0.05, 30.0, 1e4, 3e38, INF])
@pytest.mark.parametrize("at", [0.0, 1e4, -1e6, 1e-20])
def test_temperatures_and_offsets(T, at):
    z = logits(4, 5000, "f32", 7) + at
    z[3] = z[3].sign() * z[3].abs() ** 3
    run_and_check(z, [0.1, 0.5, 0.9, 0.99], [T] * 4, None, [0.7, 0.9, 0.999, 1.0], None)
    run_and_check(z, [0.1, 0.5, 0.9, 0.99], [T] * 4, [10, 100, 1000, 4999], None, [0.0, 0.5, 1e-6, 0.0])


@gpu
@needs_gpu
def test_random_rows():
    """Many rows of every kind at once: a border that is off by one shows here first."""
    g = gen(11)
    for i in range(6):
        rows, V = 200, int(torch.randint(1000, 30000, (1,), generator=g))
        z = logits(rows, V, ["f32", "bf16", "f16"][i % 3], 100 + i, spread=[1.5, 0.3, 4.0][i // 2])
        r = lambda lo, hi: (lo + (hi - lo) * torch.rand(rows, generator=g)).tolist()  # noqa: E731
        run_and_check(z, r(0, 1), r(0.3, 3.0), torch.randint(0, V, (rows,), generator=g).tolist() if i % 2 else None, r(0.3, 1.1),
                      (10 ** (-6 * torch.rand(rows, generator=g))).tolist() if i > 2 else None)


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_draws_from_the_tail(kind):
    """Tokens that weigh 2^-24 of the sum and less.  Units of 2^-54 of the largest weight, cut off, take 152064 / 2 of them, 2^-37.8, at
    most; weights that are 2^-31 off take 2^-35.3 if all of a tail of 0.05 were off alike.  Together less than 2^-35 of the sum."""
    rows, V = 197, 152064
    z = logits(rows, V, kind, 41, spread=1.0).cuda()
    T = (0.4 + 0.6 * torch.rand(rows, generator=gen(42))).float().cuda()
    zd, order = torch.sort(z.double(), dim=1, descending=True, stable=True)
    C = torch.exp((zd - zd[:, :1]) / T.double()[:, None]).cumsum(1)
    S = C[:, -1]
    token, status = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    for seed in range(20):
        u = (1 - 0.02 * torch.rand(rows, generator=gen(100 + seed))).float().clamp(max=1 - 2.0 ** -24).cuda()
        rpd.sample(z, u, token, status, temperature=T)
        at = (order == token[:, None]).int().argmax(1)
        with_it = C.gather(1, at[:, None])[:, 0]
        before = torch.where(at > 0, C.gather(1, (at - 1).clamp(min=0)[:, None])[:, 0], torch.zeros_like(S))
        target = u.double() * S
        assert (status == 0).all()
        assert (target < with_it + 2.0 ** -35 * S).all() and (target > before - 2.0 ** -35 * S).all()


@gpu
@needs_gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_min_p_at_its_border(kind):
    """Logits one step of the type above and below the largest one plus T ln min_p, for many min_p."""
    rows, V = 64, 300
    g = gen(21)
    m = torch.cat([torch.exp(-20 * torch.rand(60, generator=g)), torch.tensor([1.0, 1e-38, 1e-44, 2.0 ** -20])]).float()
    T = 0.5 + torch.rand(rows, generator=g).float()
    top = 10 + torch.rand(rows, generator=g)
    z = torch.full((rows, V), -300.0, dtype=TYPES[kind])
    z[:, 0] = top.to(z.dtype)
    for r in range(rows):
        edge = (z[r, 0].double() + T[r].double() * torch.log(m[r].double())).to(z.dtype)
        step = edge
        for i in range(1, 40):
            z[r, i] = step
            step = torch.nextafter(step.float(), torch.tensor(100.0)).to(z.dtype) if kind == "f32" else step + abs(step) * 2.0 ** -7
        step = edge
        for i in range(40, 80):
            z[r, i] = step
            step = torch.nextafter(step.float(), torch.tensor(-1000.0)).to(z.dtype) if kind == "f32" else step - abs(step) * 2.0 ** -7
    z = torch.minimum(z, z[:, :1])
    run_and_check(z, [0.999] * rows, T.tolist(), None, None, m.tolist())
    run_and_check(z, [0.999] * rows, T.tolist(), [70] * rows, None, m.tolist())
    run_and_check(z, [0.5] * rows, T.tolist(), [V + 5] * rows, [0.9] * rows, m.tolist())
