"""Performance cases of the 8-bit head, of the quantiser that makes its operands, and of sampling.

A case of op "fp8" is the readout of `rows` hidden states through a matrix of e4m3 codes with a scale for
every 128 x 128 of them; the call rounds the activations to e4m3 with a scale for every 128 columns of a row:

    d, V        columns and rows of the matrix (hidden size, vocabulary entries)
    rows        activations;  norm: RMSNorm with a gain before the product
    x, out      types of the activations and of the logits
    pad         elements between the rows of x and of the logits beyond their length

A case of op "blocks" brings a matrix to e4m3 with a scale for every 128 columns of `high` rows:

    rows, cols, x, pad;  high: 1 (activations) or 128 (weights)

A case of op "sample" draws a token from every row of logits by one given random number:

    V, rows, x, pad as above
    k           largest top-k of a row, rows have between 1 and k (0: no limit)
    p, minp     top-p and min-p of the rows, spread by a twentieth (0: none)
    temp        middle of the rows' temperatures
    greedy      of every `greedy` rows one has temperature 0 (0: none)
    allowed     a bit mask of allowed tokens for every row
    bits        the kept tokens are returned as such a mask too (what a verification of drafts takes)
"""
import math

import torch

own = False

LLADA = {"d": 4096, "V": 126464}
DREAM = {"d": 3584, "V": 152064}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
MOST = 448.0  # e4m3's largest number


def _fp8(name, d, V, rows, norm, x="bf16", out="f32", pad=0):
    c = dict(op="fp8", d=d, V=V, rows=rows, norm=norm, x=x, out=out, pad=pad)
    return dict(c, name=name) if name else c


def _blocks(name, rows, cols, high, x="bf16", pad=0):
    c = dict(op="blocks", rows=rows, cols=cols, high=high, x=x, pad=pad)
    return dict(c, name=name) if name else c


def _sample(name, V, rows, x, k=0, p=0.0, minp=0.0, temp=0.8, greedy=0, allowed=False, bits=False, pad=0):
    c = dict(op="sample", V=V, rows=rows, x=x, k=k, p=p, minp=minp, temp=temp, greedy=greedy, allowed=allowed,
             bits=bits, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small drafter's head, one token: launch and latency, nothing else
        _fp8("fp8_tiny", 256, 4096, 1, True),
        # one token through a large head: what autoregressive decoding does at every step
        _fp8("fp8_token", **LLADA, rows=1, norm=True),
        # odd everything: columns, rows, strides that no vector load fits
        _fp8("fp8_odd", 1001, 50021, 13, False, x="f16", out="f16", pad=3),
        # a serving batch, a token each (or a block of 32 positions with its 4 window layers)
        _fp8("fp8_batch", **LLADA, rows=128, norm=True, out="bf16"),
        # all rows of a first step: 256 positions of 4 window layers
        _fp8("fp8_window", **DREAM, rows=1024, norm=True, out="bf16"),
        # activations of a serving batch
        _blocks("blocks_rows", 128, 4096, 1),
        # a bf16 head on its way to 8 bits
        _blocks("blocks_head", LLADA["V"], LLADA["d"], 128),
        # one sequence over a small vocabulary: launch and latency
        _sample("sample_tiny", 4096, 1, "f32", k=40),
        # one user's next token
        _sample("sample_one", LLADA["V"], 1, "bf16", p=0.95),
        # a serving batch whose users ask for different things, some for the likeliest token, under a grammar's mask
        _sample("sample_batch", LLADA["V"], 128, "bf16", k=100, p=0.95, minp=0.02, greedy=8, allowed=True),
        # rows of a target model whose drafts are verified under top-p: 16 sequences of 32 drafts
        _sample("sample_rows", DREAM["V"], 528, "f32", p=0.9, bits=True),
        # hot, unfiltered, odd vocabulary and strides: nearly every token is likely
        _sample("sample_hot", 50021, 7, "f16", temp=3.0, pad=5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _most(name):
    return next(work(k) for k in listed() if k["name"] == name)


def draw(rng):
    """Heads: the two models' or any of d 64..8192 and V 256..152064, 1..1024 rows, every type, with and without
    norm.  Blocks: 1..131072 rows of 64..8192 columns.  Sampling: V 256..152064, 1..1024 rows, every type and
    option.  No case moves or computes more than the largest listed one of its kind."""
    kind = rng.random()
    if kind < 0.42:
        pick = rng.random()
        head = LLADA if pick < 0.25 else DREAM if pick < 0.4 else {
            "d": _log_int(rng, 64, 8192), "V": _log_int(rng, 256, 152064)}
        c = _fp8(None, head["d"], head["V"], _log_int(rng, 1, 1024), rng.random() < 0.6, rng.choice(["bf16", "bf16", "f16"]),
                 rng.choice(["f32", "bf16", "f16"]), rng.choice([0, 0, 8, 1, 3]))
        while c["V"] * c["d"] > DREAM["V"] * DREAM["d"]:
            c["V"] = c["V"] // 2 + 1
        most = _most("fp8_window")
        while (work(c)["bytes"] > most["bytes"] or work(c)["flops"] > most["flops"]) and c["rows"] > 1:
            c["rows"] = c["rows"] // 2
        return c
    if kind < 0.55:
        c = _blocks(None, _log_int(rng, 1, 131072), _log_int(rng, 64, 8192), rng.choice([1, 128]),
                    rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 8, 1, 3]))
        most = _most("blocks_head")["bytes"]
        while work(c)["bytes"] > most:
            c["rows"] = c["rows"] // 2
        return c
    c = _sample(None, rng.choice([LLADA["V"], DREAM["V"], _log_int(rng, 256, 152064)]), _log_int(rng, 1, 1024),
                rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, _log_int(rng, 1, 4096)]),
                rng.choice([0.0, 0.95, rng.uniform(0.06, 1.0)]), rng.choice([0.0, 0.0, rng.uniform(0.001, 0.3)]),
                rng.choice([0.7, 1.0, math.exp(rng.uniform(math.log(0.3), math.log(3.0)))]), rng.choice([0, 0, 1, 4]),
                rng.random() < 0.3, rng.random() < 0.3, rng.choice([0, 0, 8, 1]))
    most = _most("sample_rows")["bytes"]
    while work(c)["bytes"] > most:
        c["rows"] = c["rows"] // 2
    return c


# ------------------------------------------------------------------------------- inputs

def _rows_with(rows, cols, pad, dtype):
    """A matrix whose rows lie cols + pad elements apart."""
    return torch.zeros(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _dev(seed):
    return dict(device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _fp8_inputs(c, seed):
    """Codes spread as those of normal weights whose block's largest is 448, scales that differ from block to
    block, and hidden states with a few strong channels, as a transformer's last layer has."""
    d, V, R = c["d"], c["V"], c["rows"]
    dev = _dev(seed)
    s = {"codes": torch.empty(V, d, dtype=torch.float8_e4m3fn, device="cuda"), "gain": None,
         "scales": (torch.rand(-(-V // 128), -(-d // 128), **dev) * 1.5 + 0.5) * (0.02 / 112),
         "x": _rows_with(R, d, c["pad"], TYPES[c["x"]]), "out": _rows_with(R, V, c["pad"], TYPES[c["out"]])}
    for v in range(0, V, 32768):
        part = s["codes"][v:v + 32768]
        part.copy_((112 * torch.randn(part.shape, **dev)).clamp(-MOST, MOST))
    if c["norm"]:
        s["gain"] = (1 + 0.1 * torch.randn(d, **dev)).to(TYPES[c["x"]])
    strong = 1 + 6 * (torch.rand(d, **dev) < 0.01).float()
    s["x"].copy_(torch.randn(R, d, **dev) * strong)
    return s


def _blocks_inputs(c, seed):
    """A head's weights, or hidden states with a few strong channels."""
    R, cols = c["rows"], c["cols"]
    dev = _dev(seed)
    s = {"x": _rows_with(R, cols, c["pad"], TYPES[c["x"]]),
         "codes": torch.empty(R, cols, dtype=torch.float8_e4m3fn, device="cuda"),
         "scales": torch.empty(-(-R // c["high"]), -(-cols // 128), device="cuda")}
    strong = 0.02 if c["high"] > 1 else 1 + 6 * (torch.rand(cols, **dev) < 0.01).float()
    for r in range(0, R, 32768):
        part = s["x"][r:r + 32768]
        part.copy_(torch.randn(part.shape, **dev) * strong)
    return s


def _sample_inputs(c, seed):
    """Logits with a handful of likely tokens over a broad floor; a third of the tokens is not allowed where there
    is a mask, and logits in such places hold anything, infinities and NaN too.  Rows ask for different limits."""
    V, R = c["V"], c["rows"]
    dev = _dev(seed)
    s = {"logits": _rows_with(R, V, c["pad"], TYPES[c["x"]]), "uniform": torch.rand(R, **dev),
         "temperature": c["temp"] * (0.75 + 0.5 * torch.rand(R, **dev)), "top_k": None, "top_p": None, "min_p": None,
         "allowed": None}
    if c["greedy"]:
        s["temperature"][::c["greedy"]] = 0
    if c["k"]:
        s["top_k"] = torch.randint(1, c["k"] + 1, (R,), dtype=torch.int32, **dev)
    if c["p"]:
        s["top_p"] = c["p"] - 0.05 * torch.rand(R, **dev)
    if c["minp"]:
        s["min_p"] = c["minp"] * (0.95 + 0.05 * torch.rand(R, **dev))
    words = -(-V // 32)
    if c["allowed"]:
        s["allowed"] = torch.empty(R, words, dtype=torch.int32, device="cuda")
    for r in range(0, R, 64):
        n = min(64, R - r)
        z = 1.5 * torch.randn(n, V, **dev)
        at = torch.randint(0, V, (n, 6), **dev)
        z.scatter_(1, at, 11.0 + 2.5 * torch.randn(n, 6, **dev))
        if c["allowed"]:
            on = torch.rand(n, V, **dev) < 0.67
            on.scatter_(1, at, True)
            junk = torch.rand(n, V, **dev)
            z = torch.where(on | (junk > 0.01), z, torch.where(junk < 0.005, math.inf, math.nan))
            s["allowed"][r:r + n] = _pack(on)
        s["logits"][r:r + n] = z.to(TYPES[c["x"]])
    return s


def _pack(on):
    """Truth values [rows][V] as bits, 32 to a word."""
    words = -(-on.shape[1] // 32)
    on = torch.nn.functional.pad(on, (0, words * 32 - on.shape[1])).view(on.shape[0], words, 32)
    word = (on.long() << torch.arange(32, device=on.device)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int()


_INPUTS = {"fp8": _fp8_inputs, "blocks": _blocks_inputs, "sample": _sample_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "fp8" and own:
        import paper_2609_36452_gb300 as rpd
        s["head"] = rpd.Fp8Head(case["d"], case["V"])
        s["head"].set_weights(s["codes"], s["scales"])
    if case["op"] == "sample":
        R = case["rows"]
        s["out_token"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["out_status"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["out_kept"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["out_prob"] = torch.zeros(R, device="cuda")
        s["out_allowed"] = None
        if case["bits"]:
            s["out_allowed"] = torch.zeros(R, -(-case["V"] // 32), dtype=torch.int32, device="cuda")
    s["case"] = case
    return s


# ------------------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        import paper_2609_36452_gb300 as rpd
    if case["op"] == "fp8":
        if own:
            s["head"].logits(s["x"], s["out"], gain=s["gain"], eps=EPS)
        else:
            _plain_fp8(s)
        return s["out"]
    if case["op"] == "blocks":
        if own:
            rpd.quantize_fp8(s["x"], s["codes"], s["scales"], block_rows=case["high"])
        else:
            for r in range(0, case["rows"], 16384):
                q, scale = _plain_quantize(s["x"][r:r + 16384].float(), case["high"])
                s["codes"][r:r + 16384] = q
                s["scales"][r // case["high"]:r // case["high"] + scale.shape[0]] = scale
        return {"codes": s["codes"], "scales": s["scales"]}
    if not own:
        return _plain_sample(s)
    rpd.sample(s["logits"], s["uniform"], s["out_token"], s["out_status"], temperature=s["temperature"],
               top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], allowed=s["allowed"], out_kept=s["out_kept"],
               out_prob=s["out_prob"], out_allowed=s["out_allowed"])
    out = {"token": s["out_token"], "status": s["out_status"], "kept": s["out_kept"], "prob": s["out_prob"]}
    return dict(out, allowed=s["out_allowed"]) if case["bits"] else out


def _plain_quantize(x, high):
    """e4m3 codes and scales of a float32 matrix in blocks of high x 128."""
    rows, cols = x.shape
    R, C = -(-rows // high), -(-cols // 128)
    t = torch.nn.functional.pad(x, (0, C * 128 - cols, 0, R * high - rows)).view(R, high, C, 128)
    scale = t.abs().amax((1, 3))
    scale = scale / torch.full_like(scale, MOST)  # (divided by a number, torch multiplies by its reciprocal)
    q = (t / torch.where(scale > 0, scale, 1.0)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(R * high, C * 128)[:rows, :cols], scale


def _plain_fp8(s):
    c = s["case"]
    d, V = c["d"], c["V"]
    u, factor = s["x"].float(), 1.0
    if s["gain"] is not None:
        factor = torch.rsqrt(u.square().mean(1, keepdim=True) + EPS)
        u = (u * s["gain"].float()).to(s["x"].dtype).float()
    q, scale = _plain_quantize(u, 1)
    u = q.float() * scale.repeat_interleave(128, 1)[:, :d]
    for v in range(0, V, 32768):
        part = s["codes"][v:v + 32768]
        w = s["scales"][v // 128:v // 128 + 256].repeat_interleave(128, 0)[:part.shape[0]]
        w = part.float() * w.repeat_interleave(128, 1)[:, :d]
        s["out"][:, v:v + 32768] = ((u @ w.t()) * factor).to(s["out"].dtype)


def _plain_sample(s):
    """In chunks of rows: sorted, summed in 64 bits, cut off, drawn."""
    c, outs = s["case"], []
    V, R = c["V"], c["rows"]
    at = torch.arange(V, device="cuda")
    for r in range(0, R, 64):
        rows = slice(r, min(r + 64, R))
        z = s["logits"][rows].float()
        if s["allowed"] is not None:
            z = torch.where((s["allowed"][rows][:, at // 32] >> (at % 32)) & 1 == 1, z, -math.inf)
        z, order = torch.sort(z, dim=1, descending=True, stable=True)
        T = s["temperature"][rows].double()[:, None]
        kept = torch.isfinite(z) & ((T > 0) | (at == 0))
        if s["top_k"] is not None:
            kept &= at < s["top_k"][rows][:, None]
        w = torch.exp((z.double() - z[:, :1].double()) / torch.where(T > 0, T, 1.0)) * kept
        if s["top_p"] is not None:
            before = w.cumsum(1) - w
            kept &= (before < s["top_p"][rows].double()[:, None] * w.sum(1, keepdim=True)) | (at == 0)
        if s["min_p"] is not None:
            kept &= w >= s["min_p"][rows].double()[:, None]
        w = w * kept
        total = w.cumsum(1)
        mass = total[:, -1:]
        place = (total <= s["uniform"][rows].double()[:, None] * mass).sum(1, keepdim=True)
        out = {"token": order.gather(1, place)[:, 0].int(),
               "status": torch.zeros(z.shape[0], dtype=torch.int32, device="cuda"),
               "kept": kept.sum(1).int(), "prob": (w.gather(1, place) / mass)[:, 0].float()}
        if c["bits"]:
            out["allowed"] = _pack(torch.zeros_like(kept).scatter_(1, order, kept))
        outs.append(out)
    return {k: torch.cat([o[k] for o in outs]) for k in outs[0]}


# ------------------------------------------------------------------- what a pass has to do

def work(case):
    c = case
    if c["op"] == "fp8":
        d, V, R = c["d"], c["V"], c["rows"]
        return {"bytes": float(V * d + 4 * (-(-V // 128)) * (-(-d // 128)) + 2 * R * d + R * V * SIZE[c["out"]]
                               + (2 * d if c["norm"] else 0)),
                "flops": 2.0 * R * d * V}
    if c["op"] == "blocks":
        n = c["rows"] * c["cols"]
        return {"bytes": float(n * (SIZE[c["x"]] + 1) + 4 * (-(-c["rows"] // c["high"])) * (-(-c["cols"] // 128))),
                "flops": 3.0 * n}
    n, words = c["rows"] * c["V"], -(-c["V"] // 32)
    masks = (1 if c["allowed"] else 0) + (1 if c["bits"] else 0)
    return {"bytes": float(n * SIZE[c["x"]] + masks * c["rows"] * words * 4 + 36 * c["rows"]), "flops": 6.0 * n}


# ---------------------------------------------------------------------------- 64-bit results

def exact(case, seed):
    return {"fp8": _exact_fp8, "blocks": _exact_blocks, "sample": _exact_sample}[case["op"]](case, seed)


def _e4m3(x):
    """The nearest e4m3 number (ties to the even one) of numbers up to 448, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_codes(x, high):
    """What the operator holds a matrix as: the scale and the quotient are fp32 numbers by its definition (a
    quotient in 64 bits, rounded to them, is the right one)."""
    x = x.double()
    q = torch.empty_like(x)
    scales = torch.zeros(-(-x.shape[0] // high), -(-x.shape[1] // 128), dtype=torch.float64, device=x.device)
    for j in range(scales.shape[1]):
        cols = x[:, j * 128:j * 128 + 128]
        top = cols.abs().max(1).values
        for i in range(scales.shape[0]) if high > 1 else ():
            top[i * high:i * high + high] = top[i * high:i * high + high].max()
        scale = (top / MOST).float().double()
        scales[:, j] = scale[::high]
        scale = torch.where(scale == 0, torch.ones_like(scale), scale)
        q[:, j * 128:j * 128 + 128] = _e4m3((cols / scale[:, None]).float().double())
    return q, scales


def _exact_blocks(c, seed):
    x = _blocks_inputs(c, seed)["x"]
    codes = torch.empty(x.shape, dtype=torch.float32, device="cuda")  # e4m3 numbers, exactly
    scales = []
    for r in range(0, c["rows"], 16384):
        q, scale = _exact_codes(x[r:r + 16384], c["high"])
        codes[r:r + 16384] = q
        scales.append(scale)
    return {"codes": codes, "scales": torch.cat(scales)}


def _exact_fp8(c, seed):
    s = _fp8_inputs(c, seed)
    x = s["x"].double()
    u = x
    if c["norm"]:  # the product's operand is rounded to the activations' type, the factor is not
        u = (s["x"].float() * s["gain"].float()).to(s["x"].dtype).double()
    q, scale = _exact_codes(u, 1)
    column = torch.arange(c["d"], device="cuda") // 128
    u = q * scale[:, column]
    out = torch.empty(c["rows"], c["V"], dtype=torch.float64, device="cuda")
    for v in range(0, c["V"], 8192):
        part = s["codes"][v:v + 8192].float().double()
        row = torch.arange(v, v + part.shape[0], device="cuda") // 128
        out[:, v:v + 8192] = torch.einsum("rk,vk->rv", u, part * s["scales"].double()[row][:, column])
    if c["norm"]:
        out /= ((x * x).sum(1) / c["d"] + EPS).sqrt()[:, None]
    return out


def _exact_sample(c, seed):
    """Row by row from the distinct logits and how often each occurs: whole tokens of a value, then the tokens of
    the value at a border by their index."""
    s = _sample_inputs(c, seed)
    V, R = c["V"], c["rows"]
    out = {"token": torch.empty(R, dtype=torch.int32), "status": torch.zeros(R, dtype=torch.int32),
           "kept": torch.empty(R, dtype=torch.int32), "prob": torch.empty(R, dtype=torch.float64)}
    masks = []
    bit = torch.arange(32, device="cuda")
    ones = torch.ones(R, device="cuda")
    temps, uniform = s["temperature"].tolist(), s["uniform"].double().tolist()
    top_p = (ones if s["top_p"] is None else s["top_p"]).double().tolist()
    min_p = (0 * ones if s["min_p"] is None else s["min_p"]).double().tolist()
    top_k = [V] * R if s["top_k"] is None else s["top_k"].tolist()
    for r in range(R):
        z = s["logits"][r].double()
        on = torch.isfinite(z)
        if c["allowed"]:
            on &= ((s["allowed"][r][:, None] >> bit) & 1).flatten()[:V] != 0
        values, counts = torch.unique(z[on], return_counts=True)
        values, counts = values.flip(0), counts.flip(0)
        ends = counts.cumsum(0)
        T, limit = temps[r], min(top_k[r], int(ends[-1]))
        if T == 0:
            limit = 1
        w = torch.exp((values - values[0]) / (T if T > 0 else 1.0))

        def mass_of(n):  # of the first n tokens
            i = int((ends < n).sum())
            return float((w[:i] * counts[:i]).sum()) + float(w[i]) * (n - (int(ends[i - 1]) if i else 0))

        def reach(target, most, strictly):  # the first token at which the sum is `target` (or more than that)
            sums = (w * counts).cumsum(0)
            i = int(((sums <= target) if strictly else (sums < target)).sum())
            if i >= len(w):
                return most
            before, rest = (int(ends[i - 1]), target - float(sums[i - 1])) if i else (0, target)
            steps = rest / float(w[i])
            return min(most, before + max(1, math.floor(steps) + 1 if strictly else math.ceil(steps)))

        def token_at(n):  # index of the n-th token
            i = int((ends < n).sum())
            return int(torch.nonzero(on & (z == values[i]))[n - 1 - (int(ends[i - 1]) if i else 0), 0]), float(w[i])

        n = limit
        if top_p[r] < 1:
            n = min(n, reach(top_p[r] * mass_of(limit), limit, False))
        above = int(counts[w >= min_p[r]].sum())
        n = max(1, min(n, above))
        mass = mass_of(n)
        token, weight = token_at(reach(uniform[r] * mass, n, True))
        out["token"][r], out["kept"][r], out["prob"][r] = token, n, weight / mass
        if c["bits"]:
            last, _ = token_at(n)
            edge = z[last]
            on &= (z > edge) | ((z == edge) & (torch.arange(V, device="cuda") <= last))
            weights = torch.nn.functional.pad(on, (0, -V % 32)).view(-1, 32).double() @ torch.exp2(bit.double())
            masks.append(torch.where(weights >= 2.0 ** 31, weights - 2.0 ** 32, weights).to(torch.int32))
    return dict(out, allowed=torch.stack(masks)) if c["bits"] else out
