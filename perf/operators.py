"""Performance cases of the 4-bit head and of the verification of drafted tokens.

A case of op "quant" is one product of `rows` activations with a 4-bit matrix:

    d, V        columns and rows of the matrix (hidden size, vocabulary entries)
    rows        activations;  group: columns that share a scale (and a zero point)
    zeros       stored zero points (else 8);  norm: RMSNorm with a gain before the product
    x, out, scale   types of the activations, the logits and the scales
    pad         elements between the rows of x and of the logits beyond their length

A case of op "verify" is one decision over B sequences of at most D drafted tokens:

    V, B, D     vocabulary entries, sequences, most drafts of one
    dtype       of the target's and the draft model's logits
    draft       a draft model's logits are there (else the drafts were chosen outright)
    greedy      of every `greedy` sequences one has temperature 0 (0: none)
    ragged      sequences have different numbers of drafts
    allowed     a bit mask of allowed tokens for every row of the target
    pad         elements between rows of logits beyond V
"""
import math

import torch

own = False

LLADA = {"d": 4096, "V": 126464}
DREAM = {"d": 3584, "V": 152064}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


def _quant(name, d, V, rows, group, zeros, norm, x="bf16", out="f32", scale="bf16", pad=0):
    c = dict(op="quant", d=d, V=V, rows=rows, group=group, zeros=zeros, norm=norm, x=x, out=out,
             scale=scale, pad=pad)
    return dict(c, name=name) if name else c


def _verify(name, V, B, D, dtype, draft, greedy=0, ragged=False, allowed=False, pad=0):
    c = dict(op="verify", V=V, B=B, D=D, dtype=dtype, draft=draft, greedy=greedy, ragged=ragged,
             allowed=allowed, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small drafter's head, one token: launch and latency, nothing else
        _quant("quant_tiny", 256, 4096, 1, 32, False, True),
        # one token through a large head: what autoregressive decoding does at every step
        _quant("quant_token", **LLADA, rows=1, group=128, zeros=False, norm=True),
        # five sequences of another model, finer groups with zero points
        _quant("quant_five", **DREAM, rows=5, group=64, zeros=True, norm=True, out="bf16", scale="f16"),
        # odd everything: columns, rows, strides that no vector load fits
        _quant("quant_odd", 1001, 50021, 13, 32, True, False, x="f16", out="f16", scale="f16", pad=3),
        # the last steps of a decode: 5 positions of 4 window layers
        _quant("quant_tail", **LLADA, rows=20, group=128, zeros=True, norm=True, out="bf16"),
        # a block of 32 positions, all of its 4 window layers
        _quant("quant_block", **LLADA, rows=128, group=128, zeros=False, norm=True, out="bf16"),
        # one sequence over a small vocabulary: launch and latency
        _verify("verify_tiny", 4096, 1, 3, "f32", True),
        # one user's sequence, a draft model's five tokens
        _verify("verify_one", LLADA["V"], 1, 5, "bf16", True),
        # a serving batch whose sequences have drafted between 0 and 5 tokens, some decoded greedily
        _verify("verify_batch", LLADA["V"], 64, 5, "bf16", True, greedy=8, ragged=True),
        # blocks of 32 committed positions checked by another model, 32-bit logits
        _verify("verify_block", DREAM["V"], 16, 32, "f32", False),
        # nothing drafted: a batch samples its next tokens under a grammar's mask
        _verify("verify_sample", LLADA["V"], 128, 0, "bf16", False, allowed=True),
        # odd vocabulary and strides, greedy and sampled sequences mixed
        _verify("verify_odd", 50021, 7, 9, "f16", True, greedy=3, ragged=True, allowed=True, pad=5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """4-bit heads: the two models' or any of d 64..8192 and V 256..152064, 1..128 rows, every
    group, type and zero point, with and without norm.  Verification: V 256..152064, 1..256
    sequences of 0..32 drafts, every type and option.  No case moves or computes more than the
    largest listed one of its kind."""
    if rng.random() < 0.5:
        pick = rng.random()
        head = LLADA if pick < 0.25 else DREAM if pick < 0.4 else {
            "d": _log_int(rng, 64, 8192), "V": _log_int(rng, 256, 152064)}
        c = _quant(None, head["d"], head["V"], _log_int(rng, 1, 128), rng.choice([32, 64, 128]),
                   rng.random() < 0.5, rng.random() < 0.6, rng.choice(["bf16", "bf16", "f16"]),
                   rng.choice(["f32", "bf16", "f16"]), rng.choice(["bf16", "f16"]),
                   rng.choice([0, 0, 8, 1, 3]))
        while c["V"] * c["d"] > LLADA["V"] * LLADA["d"] * 1.02:
            c["V"] = c["V"] // 2 + 1
        most = next(work(k)["bytes"] for k in listed() if k["name"] == "quant_block")
        while work(c)["bytes"] > most and c["rows"] > 1:
            c["rows"] = c["rows"] // 2
        return c
    c = _verify(None, rng.choice([LLADA["V"], DREAM["V"], _log_int(rng, 256, 152064)]),
                _log_int(rng, 1, 256), rng.choice([0, 1, 2, 3, 4, 5, 7, 8, 12, 16, 32]),
                rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.6,
                rng.choice([0, 0, 1, 4]), rng.random() < 0.5, rng.random() < 0.3,
                rng.choice([0, 0, 8, 1]))
    most = next(work(k)["bytes"] for k in listed() if k["name"] == "verify_block")
    while work(c)["bytes"] > most:
        c["B"] = c["B"] // 2
    return c


# ------------------------------------------------------------------------------- inputs

def _rows_with(rows, cols, pad, dtype):
    """A matrix whose rows lie cols + pad elements apart."""
    return torch.zeros(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _quant_inputs(c, seed):
    """Codes around the middle of their range, scales that differ from group to group, zero points
    around 8, and hidden states with a few strong channels, as a transformer's last layer has."""
    d, V, R = c["d"], c["V"], c["rows"]
    dev = dict(device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
    groups = -(-d // c["group"])
    s = {"codes": torch.randint(0, 256, (V, (d + 1) // 2), dtype=torch.uint8, **dev),
         "scales": (torch.rand(V, groups, **dev) * 0.012 + 0.002).to(TYPES[c["scale"]]), "zeros": None,
         "gain": None, "x": _rows_with(R, d, c["pad"], TYPES[c["x"]]),
         "out": _rows_with(R, V, c["pad"], TYPES[c["out"]])}
    if c["zeros"]:
        s["zeros"] = torch.randint(5, 12, (V, groups), dtype=torch.uint8, **dev)
    if c["norm"]:
        s["gain"] = (1 + 0.1 * torch.randn(d, **dev)).to(TYPES[c["x"]])
    strong = 1 + 6 * (torch.rand(d, **dev) < 0.01).float()
    s["x"].copy_(torch.randn(R, d, **dev) * strong)
    return s


def _lengths(c):
    """Numbers of drafts, without their order: D, or spread over 0..D."""
    return [(b * (c["D"] + 1) // c["B"]) if c["ragged"] else c["D"] for b in range(c["B"])]


def _verify_inputs(c, seed):
    """Target logits with a handful of likely tokens over a broad floor; the draft model's are the
    target's with noise; drafts are drawn from the draft model (or taken as the target's best or
    second best token); a third of the tokens is not allowed where there is a mask, and logits in
    such places hold anything, infinities and NaN too."""
    V, B, D = c["V"], c["B"], c["D"]
    cpu = torch.Generator().manual_seed(seed)
    dev = dict(device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
    order = torch.randperm(B, generator=cpu)
    lengths = torch.tensor(_lengths(c), dtype=torch.int32)[order]
    temperature = 0.6 + 0.6 * torch.rand(B, generator=cpu)
    if c["greedy"]:
        temperature[::c["greedy"]] = 0
    dtype = TYPES[c["dtype"]]
    s = {"target": torch.zeros(B, D + 1, V + c["pad"], dtype=dtype, device="cuda")[:, :, :V],
         "draft": None, "allowed": None,
         "tokens": torch.zeros(B, D, dtype=torch.int32, device="cuda"),
         "lengths": lengths.cuda() if c["ragged"] else None, "temperature": temperature.cuda(),
         "uniform": torch.rand(B, D, **dev),
         "noise": torch.empty(B, V, device="cuda").exponential_(generator=dev["generator"])}
    if c["draft"]:
        s["draft"] = torch.zeros(B, D, V + c["pad"], dtype=dtype, device="cuda")[:, :, :V]
    words = (V + 31) // 32
    if c["allowed"]:
        bits = torch.zeros(B, D + 1, words * 32, dtype=torch.bool, device="cuda")
        s["allowed"] = torch.empty(B, D + 1, words, dtype=torch.int32, device="cuda")
    for b in range(B):
        z = 1.5 * torch.randn(D + 1, V, **dev)
        at = torch.randint(0, V, (D + 1, 6), **dev)
        z.scatter_(1, at, 11.0 + 2.5 * torch.randn(D + 1, 6, **dev))
        if c["draft"]:
            y = (z[:D] + 0.5 * torch.randn(D, V, **dev)).to(dtype)
            s["draft"][b] = y
            drawn = y.float() / max(float(temperature[b]), 0.05)
            drawn -= torch.empty(D, V, device="cuda").exponential_(generator=dev["generator"]).log()
            s["tokens"][b] = drawn.argmax(1).int()
        elif D:
            best = z[:D].topk(2, 1).indices
            second = torch.rand(D, **dev) < 0.05
            s["tokens"][b] = torch.where(second, best[:, 1], best[:, 0]).int()
        if c["allowed"]:
            on = torch.rand(D + 1, V, **dev) < 0.67
            on.scatter_(1, at, True)
            junk = torch.rand(D + 1, V, **dev)
            z = torch.where(on | (junk > 0.01), z, torch.where(junk < 0.005, math.inf, math.nan))
            bits[b, :, :V] = on
        s["target"][b] = z.to(dtype)
    if c["allowed"]:
        weight = torch.tensor([1 << i for i in range(32)], device="cuda")
        for b in range(B):
            word = (bits[b].view(D + 1, words, 32).long() * weight).sum(-1)
            s["allowed"][b] = torch.where(word >= 1 << 31, word - (1 << 32), word).int()
    return s


def prepare(case, seed):
    if case["op"] == "quant":
        s = _quant_inputs(case, seed)
        if own:
            import paper_2609_36452_gb300 as rpd
            s["head"] = rpd.QuantHead(case["d"], case["V"], case["group"])
            s["head"].set_weights(s["codes"], s["scales"], s["zeros"])
    else:
        s = _verify_inputs(case, seed)
        B, D = case["B"], case["D"]
        s["out_accepted"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["out_token"] = torch.zeros(B, D + 1, dtype=torch.int32, device="cuda")
        s["out_status"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["out_prob"] = torch.zeros(B, D, device="cuda")
    s["case"] = case
    return s


# ------------------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if case["op"] == "quant":
        if own:
            s["head"].logits(s["x"], s["out"], gain=s["gain"], eps=EPS)
        else:
            _plain_quant(s)
        return s["out"]
    if not own:
        return _plain_verify(s)
    import paper_2609_36452_gb300 as rpd
    rpd.verify(s["target"], s["tokens"], s["uniform"], s["noise"], s["out_accepted"], s["out_token"],
               s["out_status"], out_prob=s["out_prob"], draft=s["draft"], lengths=s["lengths"],
               temperature=s["temperature"], allowed=s["allowed"])
    return {"accepted": s["out_accepted"], "token": s["out_token"], "status": s["out_status"],
            "prob": s["out_prob"]}


def _plain_quant(s):
    c = s["case"]
    d, V, group = c["d"], c["V"], c["group"]
    u, scale = s["x"].float(), 1.0
    if s["gain"] is not None:
        scale = torch.rsqrt(u.square().mean(1, keepdim=True) + EPS)
        u = (u * s["gain"].float()).to(s["x"].dtype).float()
    for v in range(0, V, 32768):
        packed = s["codes"][v:v + 32768]
        q = torch.stack((packed & 15, packed >> 4), 2).flatten(1)[:, :d].float()
        zero = 8.0 if s["zeros"] is None else \
            s["zeros"][v:v + 32768].float().repeat_interleave(group, 1)[:, :d]
        w = (q - zero) * s["scales"][v:v + 32768].float().repeat_interleave(group, 1)[:, :d]
        s["out"][:, v:v + 32768] = ((u @ w.t()) * scale).to(s["out"].dtype)


def _lowest_argmax(x):
    at = torch.arange(x.shape[-1], device=x.device)
    return torch.where(x == x.amax(-1, keepdim=True), at, x.shape[-1]).amin(-1)


def _softmax(z, T):
    """Probabilities at temperature T ([B], 0: all at the largest logit), or zeros where a row has
    no finite logit."""
    z = z - z.amax(-1, keepdim=True)
    hot = torch.zeros_like(z).scatter_(-1, _lowest_argmax(z).clamp(max=z.shape[-1] - 1).unsqueeze(-1), 1.0)
    T = T.view(-1, 1, 1)
    e = torch.exp(z / torch.where(T > 0, T, 1.0))
    return torch.where(T > 0, e / e.sum(-1, keepdim=True), hot)


def _plain_verify(s):
    c = s["case"]
    V, B, D = c["V"], c["B"], c["D"]
    z = s["target"].float()
    if s["allowed"] is not None:
        at = torch.arange(V, device="cuda")
        z = torch.where((s["allowed"][..., at // 32] >> (at % 32)) & 1 == 1, z, -math.inf)
    p = _softmax(z, s["temperature"])
    n = torch.full((B,), D, device="cuda") if s["lengths"] is None else s["lengths"].long()
    seq, pos = torch.arange(B, device="cuda"), torch.arange(D + 1, device="cuda")
    tokens = s["tokens"].long()
    live = pos[:D] < n[:, None]
    px = p[:, :D].gather(2, tokens.unsqueeze(2)).squeeze(2)
    if s["draft"] is not None:
        q = _softmax(s["draft"].float(), s["temperature"])
    else:
        q = torch.zeros(B, D, V, device="cuda").scatter_(2, tokens.unsqueeze(2), 1.0)
    qx = q.gather(2, tokens.unsqueeze(2)).squeeze(2)
    greedy = (s["temperature"] == 0)[:, None]
    ok = torch.where(greedy, px > 0, s["uniform"] * qx < px) & live
    accepted = ok.int().cumprod(1).sum(1)
    chosen = p[seq, accepted]
    rejected = (accepted < n) & ~greedy[:, 0]
    if D:
        left = (chosen - q[seq, accepted.clamp(max=D - 1)]).clamp(min=0)
        chosen = torch.where(rejected[:, None], left, chosen)
    best = torch.where(greedy, chosen, chosen / s["noise"])
    nxt = _lowest_argmax(best)
    token = torch.where(pos < accepted[:, None], torch.nn.functional.pad(tokens, (0, 1)), -1)
    token[seq, accepted] = nxt
    return {"accepted": accepted.int(), "token": token.int(),
            "status": torch.zeros(B, dtype=torch.int32, device="cuda"), "prob": torch.where(live, px, 0.0)}


# ------------------------------------------------------------------- what a pass has to do

def work(case):
    c = case
    if c["op"] == "quant":
        d, V, R, groups = c["d"], c["V"], c["rows"], -(-c["d"] // c["group"])
        return {"bytes": float(V * ((d + 1) // 2) + V * groups * (3 if c["zeros"] else 2)
                               + 2 * R * d + R * V * SIZE[c["out"]] + (2 * d if c["norm"] else 0)),
                "flops": 2.0 * R * d * V}
    n, V = sum(_lengths(c)), c["V"]
    rows = n + c["B"]
    elements = (rows + (n if c["draft"] else 0)) * V
    return {"bytes": float(elements * SIZE[c["dtype"]] + (rows * ((V + 31) // 32) * 4 if c["allowed"] else 0)
                           + c["B"] * V * 4 + 20 * rows),
            "flops": 4.0 * elements}


# ---------------------------------------------------------------------------- 64-bit results

def exact(case, seed):
    return _exact_quant(case, seed) if case["op"] == "quant" else _exact_verify(case, seed)


def _exact_quant(c, seed):
    s = _quant_inputs(c, seed)
    x = s["x"].double()
    u = x
    if c["norm"]:  # the product's operand is rounded to the activations' type, the factor is not
        u = (s["x"].float() * s["gain"].float()).to(s["x"].dtype).double()
    out = torch.empty(c["rows"], c["V"], dtype=torch.float64, device="cuda")
    column = torch.arange(c["d"], device="cuda")
    for v in range(0, c["V"], 8192):
        byte = s["codes"][v:v + 8192][:, column // 2].long()
        code = torch.where(column % 2 == 0, byte % 16, byte // 16)
        group = column // c["group"]
        zero = s["zeros"][v:v + 8192][:, group].long() if c["zeros"] else 8
        w = (code - zero).double() * s["scales"][v:v + 8192][:, group].double()
        out[:, v:v + 8192] = torch.einsum("rk,vk->rv", u, w)
    if c["norm"]:
        out /= ((x * x).sum(1) / c["d"] + EPS).sqrt()[:, None]
    return out


def _exact_verify(c, seed):
    s = _verify_inputs(c, seed)
    V, B, D = c["V"], c["B"], c["D"]
    accepted = torch.zeros(B, dtype=torch.int32)
    token = torch.full((B, D + 1), -1, dtype=torch.int32)
    prob = torch.zeros(B, D, dtype=torch.float64)
    count = s["lengths"].tolist() if c["ragged"] else [D] * B
    drafts, temps, uniform = s["tokens"].tolist(), s["temperature"].tolist(), s["uniform"].tolist()
    bit = torch.arange(32, device="cuda")

    def first(x):
        return int(torch.nonzero(x == x.max())[0, 0])

    def dist(row, T, words=None):
        row = row.double()
        if words is not None:
            on = ((words[:, None] >> bit) & 1).flatten()[:V] != 0
            row = torch.where(on, row, torch.full_like(row, -math.inf))
        if T == 0:
            hot = torch.zeros(V, dtype=torch.float64, device="cuda")
            hot[first(row)] = 1
            return hot
        return torch.softmax(row / T, 0)

    for b in range(B):
        n, T, stop, left = count[b], temps[b], None, None
        for i in range(n + 1):
            p = dist(s["target"][b, i], T, None if s["allowed"] is None else s["allowed"][b, i])
            if i == n:
                if stop is None:
                    stop, left = n, p
                break
            x = drafts[b][i]
            prob[b, i] = p[x]
            if stop is not None:
                continue
            q = torch.zeros_like(p)
            if T > 0 and c["draft"]:
                q = dist(s["draft"][b, i], T)
            elif T > 0:
                q[x] = 1
            if (float(p[x]) > 0) if T == 0 else uniform[b][i] * float(q[x]) < float(p[x]):
                token[b, i] = x
                accepted[b] += 1
            else:
                stop, left = i, (p - q).clamp(min=0)
        token[b, stop] = first(left if T == 0 else left / s["noise"][b].double())
    return {"accepted": accepted, "token": token, "status": torch.zeros(B, dtype=torch.int32), "prob": prob}
