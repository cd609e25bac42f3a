"""Performance cases of a mixture-of-experts layer's other operators: the whole layer for a few tokens, projections in 8-bit
floating point with a scale for each block of 128, what brings rows of activations into that form, and the activation
between two projections.

A case names the operator ("op"):

    moe        logits [T, E] and activations -> the k experts of each token, each a sub-bit feed-forward block (activation,
               with a gate or without, between its projections), weighted and summed
    scaled     rows of e4m3 values with a scale for each 128 of a row, times e4m3 weights with a scale for each 128 x 128
               of them; one projection for all rows, or rows grouped by expert
    quantise   rows into that form, behind an activation or as they are, in their order or by an index
    activate   f(gate) * up, or f(up)

Projections of the mixture are 1x1 layers of the library: alpha * (W x), W of +1 and -1, one tau-bit index per vector of 8
input channels into a codebook of 2^tau such vectors.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_E4M3 = torch.float8_e4m3fn
_LEAST = 2.0 ** -70   # of a block's scale


def _moe(T, E, k, c_in, hidden, c_out, tau, fn, gated, act, out, normalise, masked):
    return {"op": "moe", "T": T, "E": E, "k": k, "c_in": c_in, "hidden": hidden, "c_out": c_out, "tau": tau, "fn": fn, "gated": gated, "act": act,
            "out": out, "normalise": normalise, "masked": masked}


def _scaled(R, E, c_in, c_out, out, skew):
    return {"op": "scaled", "R": R, "E": E, "c_in": c_in, "c_out": c_out, "out": out, "skew": skew}


def _quantise(R, C, act, fn, gated, repeat):
    return {"op": "quantise", "R": R, "C": C, "act": act, "fn": fn, "gated": gated, "repeat": repeat}


def _activate(R, C, act, out, fn, gated):
    return {"op": "activate", "R": R, "C": C, "act": act, "out": out, "fn": fn, "gated": gated}


def listed():
    return [
        # one token of one conversation: latency, and the bits of two experts
        {"name": "moe_1token", **_moe(1, 8, 2, 4096, 4096, 4096, 5, "silu", True, "bf16", "bf16", True, 0.0)},
        # a few conversations, odd sizes, no gate, sums that go on in fp32, experts switched off
        {"name": "moe_ragged", **_moe(5, 60, 3, 1096, 1000, 1003, 7, "gelu", False, "f16", "f32", False, 0.1)},
        # a batch of conversations over many small experts, one token each
        {"name": "moe_batch", **_moe(64, 64, 4, 2048, 1024, 2048, 5, "silu", True, "bf16", "bf16", True, 0.0)},
        # one token through one projection
        {"name": "scaled_1row", **_scaled(1, 1, 4096, 4096, "bf16", 0.0)},
        # a batch of conversations through one wide projection
        {"name": "scaled_batch", **_scaled(48, 1, 4096, 8192, "bf16", 0.0)},
        # a batch of conversations, a few rows for each of many experts, some without any
        {"name": "scaled_experts", **_scaled(256, 64, 2048, 2048, "bf16", 1.0)},
        # uneven experts, sizes that end inside blocks and tiles, fp32 outputs
        {"name": "scaled_ragged", **_scaled(2042, 16, 1104, 1003, "f32", 1.5)},
        # a prompt
        {"name": "scaled_prompt", **_scaled(4096, 1, 4096, 8192, "bf16", 0.0)},
        # one token's activations
        {"name": "quantise_1row", **_quantise(1, 4096, "bf16", "none", False, 1)},
        # a prompt between the two projections of a feed-forward block; an odd number of rows
        {"name": "quantise_prompt", **_quantise(8191, 4096, "bf16", "silu", True, 1)},
        # a batch between the two projections, odd columns, fp32 sums of the first
        {"name": "activate_batch", **_activate(256, 1003, "f32", "f16", "gelu", False)},
        # a prompt
        {"name": "activate_prompt", **_activate(8191, 8192, "bf16", "bf16", "silu", True)},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the same ranges, no larger than the largest listed."""
    op = rng.choice(["moe", "moe", "moe", "scaled", "scaled", "scaled", "quantise", "activate"])
    act = rng.choice(["bf16", "f16"])
    fn = rng.choice(["silu", "gelu", "relu"])
    if op == "moe":
        E, c_in, hidden, c_out = rng.choice([4, 8, 16, 60, 64]), 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 512), _log(rng, 64, 4096)
        if E * hidden * (c_in + c_out) > 1 << 28:
            E, c_in, hidden = min(E, 8), min(c_in, 2048), min(hidden, 2048)
        return _moe(_log(rng, 1, 64), E, rng.choice([1, 2, 4]), c_in, hidden, c_out, rng.randint(3, 8), fn, rng.random() < 0.7, act,
                    rng.choice([act, act, "f32"]), rng.random() < 0.7, rng.choice([0.0, 0.0, 0.2]))
    if op == "scaled":
        E, R = rng.choice([1, 1, 1, 8, 16, 60]), _log(rng, 1, 4096)
        c_in, c_out = 16 * _log(rng, 8, 256), _log(rng, 64, 8192)
        if E > 1:
            c_in, c_out = min(c_in, 2048), min(c_out, 2048)
        return _scaled(R, E, c_in, c_out, rng.choice(["bf16", "f16", "f32"]), 0.0 if E == 1 else rng.choice([0.0, 0.5, 1.5]))
    R, C = _log(rng, 1, 8191), _log(rng, 64, 4096)
    if op == "quantise":
        fn = rng.choice(["none", fn])
        return _quantise(R, C, rng.choice(["f32", act]), fn, fn != "none" and rng.random() < 0.7, rng.choice([1, 1, 2]) if R < 4000 else 1)
    return _activate(R, C, rng.choice(["f32", act]), rng.choice(["f32", act]), fn, rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------------- inputs

def _weights(g, E, c_in, c_out, tau):
    """Codebooks of different 8-bit codes, uniform indices, scales about 1 / sqrt(c_in) (outputs of the size of the inputs)."""
    codes = torch.rand(E, 256, generator=g, device="cuda").argsort(1)[:, : 1 << tau].contiguous()
    idx = torch.randint(0, 1 << tau, (E, c_out, c_in // 8), generator=g, device="cuda", dtype=torch.uint8 if tau < 8 else torch.int16)
    alpha = (0.5 + torch.rand(E, c_out, generator=g, device="cuda")) / math.sqrt(c_in)
    return codes, idx, alpha


def _decoded(codes, idx):
    """+1 / -1 as int8 [E, c_out, c_in]: element j of a vector is bit 7 - j of its code."""
    bit = 7 - torch.arange(8, device="cuda")
    signs = (((codes[:, :, None] >> bit) & 1) * 2 - 1).to(torch.int8)
    E, c_out, G = idx.shape
    w = torch.gather(signs, 1, idx.reshape(E, c_out * G, 1).long().expand(-1, -1, 8))
    return w.reshape(E, c_out, G * 8)


def _stored(codes, idx, alpha, tau):
    """The stored form of each projection: codes, LSB-first stream of tau-bit indices, scales, as host arrays."""
    E = idx.shape[0]
    bits = (idx.reshape(E, -1)[:, :, None].to(torch.int16) >> torch.arange(tau, device="cuda", dtype=torch.int16)) & 1
    bits = torch.nn.functional.pad(bits.reshape(E, -1).to(torch.uint8), (0, -(bits.shape[1] * tau) % 8))
    stream = (bits.reshape(E, -1, 8) << torch.arange(8, device="cuda", dtype=torch.uint8)).sum(2).to(torch.uint8)
    return codes.cpu().numpy().astype(np.uint16), stream.cpu().numpy(), alpha.cpu().numpy()


def _blocks(x):
    """[..., C] as [..., blocks, 128], zeros behind C."""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % 128)).reshape(*x.shape[:-1], -1, 128)


def _to_e4m3(x):
    """Rows [..., C] in fp32 as e4m3 and a scale for each 128 of a row."""
    b = _blocks(x)
    scale = (b.abs().amax(-1) / torch.full((), 448.0, device="cuda")).clamp(min=_LEAST)   # (by a number: a product with 1 / 448)
    return (b / scale[..., None]).to(_E4M3).flatten(-2)[..., : x.shape[-1]].contiguous(), scale


def _weights_e4m3(g, E, c_in, c_out):
    """Normal weights as e4m3 and a scale for each 128 x 128; blocks of different sizes."""
    w = torch.randn(E, c_out, c_in, generator=g, device="cuda") / math.sqrt(c_in)
    nb, nk = -(-c_in // 128), -(-c_out // 128)
    w = torch.nn.functional.pad(w, (0, 128 * nb - c_in, 0, 128 * nk - c_out)).reshape(E, nk, 128, nb, 128)
    w = w * (0.25 + 1.5 * torch.rand(E, nk, 1, nb, 1, generator=g, device="cuda"))
    scale = w.abs().amax((2, 4)) / 448.0
    q = (w / scale[:, :, None, :, None]).to(_E4M3).reshape(E, nk * 128, nb * 128)[:, :c_out, :c_in].contiguous()
    return q, scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    op = case["op"]
    if op == "moe":
        T, E, act = case["T"], case["E"], _TYPES[case["act"]]
        logits = 1.5 * torch.randn(T, E, generator=g, device="cuda")
        if case["masked"]:
            off = torch.rand(T, E, generator=g, device="cuda") < case["masked"]
            off |= torch.rand(T, 1, generator=g, device="cuda") < case["masked"]   # a padded token
            logits = logits.masked_fill(off, -math.inf)
        s["logits"] = logits
        s["x"] = torch.randn(T, case["c_in"], generator=g, device="cuda").to(act)
        s["up"] = _weights(g, E, case["c_in"], case["hidden"], case["tau"])
        s["gate"] = _weights(g, E, case["c_in"], case["hidden"], case["tau"]) if case["gated"] else None
        s["down"] = _weights(g, E, case["hidden"], case["c_out"], case["tau"])
        return s
    if op == "scaled":
        R, E = case["R"], case["E"]
        s["x"], s["xs"] = _to_e4m3(torch.randn(R, case["c_in"], generator=g, device="cuda"))
        s["w"], s["ws"] = _weights_e4m3(g, E, case["c_in"], case["c_out"])
        favour = torch.softmax(case["skew"] * torch.randn(E, generator=g, device="cuda"), 0)
        who = torch.multinomial(favour, R, replacement=True, generator=g)
        counts = (who[:, None] == torch.arange(E, device="cuda")[None, :]).sum(0)
        s["sizes"] = counts.tolist()
        s["offsets"] = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).to(torch.int32)
        return s
    R, C, act = case["R"], case["C"], _TYPES[case["act"]]
    s["up"] = torch.randn(R, C, generator=g, device="cuda").to(act)
    s["gate"] = (1.5 * torch.randn(R, C, generator=g, device="cuda")).to(act) if case["gated"] else None
    if op == "quantise":
        n = case["repeat"] * R
        s["rows"] = torch.randperm(n, generator=g, device="cuda").remainder(R).to(torch.int32) if case["repeat"] > 1 else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "moe":
        s["out"] = torch.empty(case["T"], case["c_out"], dtype=_TYPES[case["out"]], device="cuda")
    elif op == "scaled":
        s["out"] = torch.empty(case["R"], case["c_out"], dtype=_TYPES[case["out"]], device="cuda")
        s["place"] = _places(s["sizes"])
    elif op == "activate":
        s["out"] = torch.empty(case["R"], case["C"], dtype=_TYPES[case["out"]], device="cuda")
    if own:
        import paper_2110_09195_b200 as snn
        s["snn"] = snn
        if op == "quantise":
            s["out"] = snn.alloc_quantised(case["repeat"] * case["R"], case["C"])
        elif op == "scaled":
            s["handle"] = snn.SnnConvScaled(s["w"], s["ws"])
            del s["w"], s["ws"]
        if op in ("quantise", "activate", "moe"):
            s["fn"] = {"none": snn.FN_NONE, "relu": snn.FN_RELU, "silu": snn.FN_SILU, "gelu": snn.FN_GELU}[case["fn"]]
        if op == "moe":
            for name in ("up", "gate", "down"):
                if s[name] is not None:
                    s[name] = _experts(snn, *s[name], case["tau"])
            s["handle"] = snn.SnnConvMoe(s["up"], s["down"], gate=s["gate"], fn=s["fn"])
    elif op == "moe":
        for name in ("up", "gate", "down"):
            if s[name] is not None:
                codes, idx, alpha = s[name]
                s[name] = _decoded(codes, idx), alpha
    return s


def _experts(snn, codes, idx, alpha, tau):
    codes, stream, alpha = _stored(codes, idx, alpha, tau)
    layers = [snn.SnnConv(idx.shape[2] * 8, idx.shape[1], tau, codes[e], stream[e], alpha[e], pad=0, act_type=snn.ACT_F16, ksize=1)
              for e in range(len(codes))]
    experts = snn.SnnConvExperts(layers)
    for layer in layers:
        layer.destroy()
    return experts


def _places(sizes):
    """Where row i stands in a table [E, largest size]: the experts' rows side by side, padded."""
    counts = torch.tensor(sizes, device="cuda")
    expert = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), counts)
    start = torch.repeat_interleave(torch.cumsum(counts, 0) - counts, counts)
    return expert * max(sizes) + torch.arange(len(expert), device="cuda") - start


# ------------------------------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        snn = s["snn"]
        if op == "moe":
            return s["handle"].forward(s["x"], s["logits"], case["k"], normalise=case["normalise"], out=s["out"])
        if op == "scaled":
            return s["handle"].forward(s["x"], s["xs"], offsets=s["offsets"] if case["E"] > 1 else None, out=s["out"])
        if op == "quantise":
            return snn.quantise(s["up"], gate=s["gate"], fn=s["fn"], rows=s["rows"], out=s["out"])
        return snn.activate(s["up"], gate=s["gate"], fn=s["fn"], out=s["out"])
    return {"moe": _plain_moe, "scaled": _plain_scaled, "quantise": _plain_quantise, "activate": _plain_activate}[op](s)


def _activation(fn, x):
    if fn == "silu":
        return x / (1 + torch.exp(-x))
    if fn == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return x.clamp(min=0) if fn == "relu" else x


def _between(fn, gate, up):
    return _activation(fn, up) if gate is None else _activation(fn, gate) * up


def _plain_moe(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    logits = s["logits"]
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    e = torch.where(logits == -math.inf, torch.zeros_like(logits), torch.exp(logits - top[:, :1].clamp(min=-3e38)))
    chosen = torch.gather(e, 1, ids[:, :k])
    total = chosen.sum(1, keepdim=True) if case["normalise"] else e.sum(1, keepdim=True)
    w = torch.where(chosen > 0, chosen / total, torch.zeros_like(chosen))
    ids = ids[:, :k]
    x = s["x"].float()
    if T * k < E:   # the chosen experts' weights, by token and choice
        flat = ids.reshape(-1)
        x = x.repeat_interleave(k, 0)[:, None, :]

        def through(name, v):
            return torch.bmm(v, s[name][0][flat].float().transpose(1, 2)) * s[name][1][flat][:, None, :]
    else:           # all tokens through all experts
        x = x.expand(E, T, -1)

        def through(name, v):
            return torch.bmm(v, s[name][0].float().transpose(1, 2)) * s[name][1][:, None, :]
    h = _between(case["fn"], None if s["gate"] is None else through("gate", x), through("up", x))
    y = through("down", h)
    if T * k < E:
        return (y.reshape(T, k, -1) * w[:, :, None]).sum(1).to(s["out"].dtype)
    share = ((ids[:, :, None] == torch.arange(E, device="cuda")).float() * w[:, :, None]).sum(1)   # [T, E]
    return (y * share.T[:, :, None]).sum(0).to(s["out"].dtype)


def _plain_scaled(s):
    case = s["case"]
    E, cap = case["E"], max(s["sizes"])
    c_in, c_out = case["c_in"], case["c_out"]
    x = s["x"].float() * s["xs"].repeat_interleave(128, 1)[:, :c_in]
    w = s["w"].float() * s["ws"].repeat_interleave(128, 1)[:, :c_out].repeat_interleave(128, 2)[:, :, :c_in]
    if E == 1:
        return (x @ w[0].T).to(s["out"].dtype)
    table = torch.zeros(E * cap, c_in, device="cuda")
    table[s["place"]] = x
    return torch.bmm(table.reshape(E, cap, -1), w.transpose(1, 2)).reshape(E * cap, -1)[s["place"]].to(s["out"].dtype)


def _plain_quantise(s):
    h = _between(s["case"]["fn"], None if s["gate"] is None else s["gate"].float(), s["up"].float())
    return _to_e4m3(h if s["rows"] is None else h[s["rows"].long()])


def _plain_activate(s):
    return _between(s["case"]["fn"], None if s["gate"] is None else s["gate"].float(), s["up"].float()).to(s["out"].dtype)


# ------------------------------------------------------------------------------------------------------- costs, oracle

def work(case):
    """Each input read once (projections in their stored form, of the experts that rows can go to), each output written once."""
    op = case["op"]
    if op == "moe":
        T, E, k, c_in, hidden, c_out = (case[n] for n in ("T", "E", "k", "c_in", "hidden", "c_out"))
        first = 2 if case["gated"] else 1

        def stored(c, n):
            return c * n // 8 * case["tau"] / 8 + 4 * n + (2 << case["tau"])
        return {"bytes": T * (c_in * 2 + 4 * E + c_out * _SIZE[case["out"]]) + min(E, T * k) * (first * stored(c_in, hidden) + stored(hidden, c_out)),
                "flops": 2 * T * k * hidden * (first * c_in + c_out)}
    if op == "scaled":
        R, E, c_in, c_out = (case[n] for n in ("R", "E", "c_in", "c_out"))
        nb, nk = -(-c_in // 128), -(-c_out // 128)
        return {"bytes": R * (c_in + 4 * nb + c_out * _SIZE[case["out"]]) + min(R, E) * (c_in * c_out + 4 * nb * nk), "flops": 2 * R * c_in * c_out}
    R, C, reads = case["R"], case["C"], 2 if case["gated"] else 1
    if op == "quantise":
        n = R * case["repeat"]
        return {"bytes": R * C * reads * _SIZE[case["act"]] + n * (C + 4 * -(-C // 128)) + (4 * n if case["repeat"] > 1 else 0), "flops": 6 * n * C}
    return {"bytes": R * C * (reads * _SIZE[case["act"]] + _SIZE[case["out"]]), "flops": 6 * R * C}


def _signs64(codes, idx):
    """+1 / -1 in 64 bits of one projection, element by element from the codes."""
    code = codes[idx.long()]                                            # [c_out, G]
    parts = [torch.where((code // (1 << (7 - j))) % 2 == 1, 1.0, -1.0).double() for j in range(8)]
    return torch.stack(parts, 2).reshape(idx.shape[0], -1)


def _fn64(fn, v):
    if fn == "silu":
        return v * torch.sigmoid(v)
    if fn == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
    return torch.maximum(v, torch.zeros_like(v)) if fn == "relu" else v


def _middle64(s):
    up = s["up"].double()
    return _fn64(s["case"]["fn"], up) if s["gate"] is None else _fn64(s["case"]["fn"], s["gate"].double()) * up


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "activate":
        return _middle64(s)
    if op == "quantise":
        h = _middle64(s)
        if s["rows"] is not None:
            h = h[s["rows"].long()]
        values, scales = torch.empty_like(h), []
        for lo in range(0, h.shape[1], 128):
            part = h[:, lo:lo + 128]
            scale = torch.clamp(part.abs().max(1).values / 448, min=_LEAST)
            # by the scale as it is kept, and rounded to 32 bits before it is to 8: 16-bit values often lie on a border
            q = (part / scale.float().double()[:, None]).float().double()
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            values[:, lo:lo + 128] = torch.round(q / step) * step
            scales.append(scale)
        return values, torch.stack(scales, 1)
    if op == "scaled":
        ends = np.cumsum(s["sizes"])
        out = torch.empty(case["R"], case["c_out"], dtype=torch.float64, device="cuda")
        for e, (end, size) in enumerate(zip(ends, s["sizes"])):
            if size:
                part = slice(int(end) - size, int(end))
                total = torch.zeros(size, case["c_out"], dtype=torch.float64, device="cuda")
                for b, lo in enumerate(range(0, case["c_in"], 128)):
                    dot = s["x"][part, lo:lo + 128].double() @ s["w"][e, :, lo:lo + 128].double().T
                    of_row = s["ws"][e, :, b].double()[torch.arange(case["c_out"], device="cuda") // 128]
                    total += dot * s["xs"][part, b].double()[:, None] * of_row[None, :]
                out[part] = total
        return out
    T, E, k = case["T"], case["E"], case["k"]
    logits = s["logits"].double().cpu().numpy()
    by_expert = [[] for _ in range(E)]
    for t in range(T):
        able = [e for e in range(E) if logits[t, e] > -math.inf]
        best = sorted(able, key=lambda e: (-logits[t, e], e))[:k]
        if best:
            top = logits[t, best[0]]
            total = math.fsum(math.exp(logits[t, e] - top) for e in (best if case["normalise"] else able))
            for e in best:
                by_expert[e].append((t, math.exp(logits[t, e] - top) / total))
    out = torch.zeros(T, case["c_out"], dtype=torch.float64, device="cuda")
    for e in range(E):
        if by_expert[e]:
            tokens = torch.tensor([t for t, _ in by_expert[e]], device="cuda")
            shares = torch.tensor([w for _, w in by_expert[e]], dtype=torch.float64, device="cuda")

            def through(name, v):
                codes, idx, alpha = s[name]
                return (v @ _signs64(codes[e], idx[e]).T) * alpha[e].double()
            x = s["x"][tokens].double()
            up = through("up", x)
            h = _fn64(case["fn"], up) if s["gate"] is None else _fn64(case["fn"], through("gate", x)) * up
            out[tokens] += shares[:, None] * through("down", h)
    return out
