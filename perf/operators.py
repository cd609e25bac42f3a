"""Performance cases of the operators around sub-bit projections of language models: routing tokens to experts, the
experts' products with weights stored as tau-bit indices, the weighted sum of their outputs, and low-rank adapters of
many requests beside one shared projection.

A projection is the 1x1 layer of the library: out = alpha * (W x), W of +1 and -1, stored as one tau-bit index per
vector of 8 input channels into a codebook of 2^tau such vectors.  A case names the operator ("op"):

    route     logits [T, E] -> the k experts of each token, their weights, and the order of the rows by expert
    experts   rows grouped by expert, each through its own expert's projection; "gather": the rows are named by an
              index into the tokens, as in front of a first projection; else they lie in order, as in front of a second
    combine   the rows' outputs back in the order of the tokens, weighted and summed
    adapters  one projection for all rows, plus scale * B (A x) with the adapter of each row's request

Activations, adapters and outputs are in the types of serving (fp16, bf16; fp32 outputs where sums go on).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _route(T, E, k, act, normalise, masked):
    return {"op": "route", "T": T, "E": E, "k": k, "act": act, "normalise": normalise, "masked": masked}


def _experts(T, E, k, c_in, c_out, tau, act, out, gather, skew):
    return {"op": "experts", "T": T, "E": E, "k": k, "c_in": c_in, "c_out": c_out, "tau": tau, "act": act, "out": out,
            "gather": gather, "skew": skew}


def _combine(T, E, k, C, act, out, masked):
    return {"op": "combine", "T": T, "E": E, "k": k, "C": C, "act": act, "out": out, "masked": masked}


def _adapters(R, c_in, c_out, tau, n, rank, run, act, out):
    return {"op": "adapters", "R": R, "c_in": c_in, "c_out": c_out, "tau": tau, "n": n, "rank": rank, "run": run,
            "act": act, "out": out}


def listed():
    return [
        # one token of one conversation: the smallest call there is
        {"name": "route_1token", **_route(1, 64, 2, "bf16", True, 0.0)},
        # a long prompt over many experts, some of them switched off; an odd number of tokens
        {"name": "route_prompt", **_route(8191, 128, 8, "f32", False, 0.1)},
        # one token through its two experts: the first projection of a feed-forward block
        {"name": "experts_1token", **_experts(1, 8, 2, 4096, 4096, 5, "bf16", "bf16", True, 0.5)},
        # a batch of conversations, one token each: few rows for each of many experts, some without any
        {"name": "experts_batch", **_experts(64, 64, 4, 2048, 2048, 5, "bf16", "bf16", True, 1.0)},
        # a prompt through the first projection, rows gathered by the router's order
        {"name": "experts_prompt", **_experts(4096, 8, 2, 2048, 8192, 5, "bf16", "bf16", True, 0.5)},
        # odd sizes, uneven experts, sums that go on in fp32, rows already in order: a second projection
        {"name": "experts_ragged", **_experts(1021, 16, 2, 1096, 1003, 7, "f16", "f32", False, 1.5)},
        # a batch of conversations: what the experts gave, back in order
        {"name": "combine_batch", **_combine(64, 64, 4, 2048, "bf16", "bf16", 0.0)},
        # a prompt
        {"name": "combine_prompt", **_combine(8191, 64, 4, 4096, "bf16", "bf16", 0.1)},
        # one token of one request with its adapter
        {"name": "adapters_1token", **_adapters(1, 4096, 4096, 5, 8, 16, 1, "bf16", "bf16")},
        # a batch of requests, one token each, every one with an adapter of its own choice
        {"name": "adapters_batch", **_adapters(48, 4096, 4096, 5, 64, 16, 1, "bf16", "bf16")},
        # prompts of several requests side by side
        {"name": "adapters_prompt", **_adapters(4096, 4096, 4096, 5, 8, 32, 700, "bf16", "bf16")},
        # an uneven mix of short prompts, odd sizes, fp32 outputs
        {"name": "adapters_ragged", **_adapters(333, 1000, 1157, 8, 5, 8, 23, "f16", "f32")},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the same ranges, no larger than the largest listed."""
    op = rng.choice(["route", "experts", "experts", "combine", "adapters", "adapters"])
    act = rng.choice(["bf16", "f16"])
    masked = rng.choice([0.0, 0.0, 0.1, 0.3])
    if op == "route":
        E = rng.choice([4, 8, 16, 60, 64, 128, 256])
        return _route(_log(rng, 1, 8191), E, min(E, rng.choice([1, 2, 4, 6, 8])), rng.choice(["f32", "bf16", "f16"]),
                      rng.random() < 0.5, masked)
    if op == "combine":
        return _combine(_log(rng, 1, 6000), rng.choice([8, 16, 64]), rng.choice([1, 2, 4, 8]), _log(rng, 64, 4096),
                        rng.choice(["f32", "bf16", "f16"]), rng.choice(["f32", "bf16", "f16"]), masked)
    c_in, c_out, tau = 8 * _log(rng, 8, 512), _log(rng, 64, 4096), rng.randint(3, 8)
    out = rng.choice([act, act, "f32"])
    if op == "experts":
        E = rng.choice([4, 8, 16, 60])
        return _experts(_log(rng, 1, 3000), E, rng.choice([1, 2, 4]), c_in, c_out, tau, act, out, rng.random() < 0.5,
                        rng.choice([0.0, 0.5, 1.5]))
    return _adapters(_log(rng, 1, 4000), c_in, c_out, tau, rng.choice([1, 3, 8, 16]), rng.choice([8, 16, 32, 64]),
                     _log(rng, 1, 900), act, out)


# ------------------------------------------------------------------------------------------------------- inputs

def _rows_by_expert(ids, E):
    """Stable order of the (token, choice) pairs by expert: ids [T, k] with -1 for no expert -> counts, rows, slots."""
    T, k = ids.shape
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    order = torch.sort(key, stable=True).indices
    counts = (key[:, None] == torch.arange(E, device=ids.device)[None, :]).sum(0)
    total = counts.sum()
    place = torch.arange(T * k, device=ids.device)
    rows = torch.where(place < total, order // k, torch.full_like(order, -1))
    slots = torch.empty_like(order)
    slots[order] = place
    slots = torch.where(flat < 0, torch.full_like(slots, -1), slots).reshape(T, k)
    return counts, rows, slots


def _choices(g, T, E, k, skew, masked=0.0):
    """k different experts for each token, some experts asked for more often than others; the last choices of a share
    of the tokens dropped (id -1)."""
    favour = skew * torch.randn(E, generator=g, device="cuda")
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    ids = torch.topk(favour[None, :] + noise, k, dim=1).indices
    if masked:
        drop = torch.rand(T, 1, generator=g, device="cuda") < masked
        keep = torch.randint(0, k, (T, 1), generator=g, device="cuda")
        ids = torch.where(drop & (torch.arange(k, device="cuda")[None, :] >= keep), torch.full_like(ids, -1), ids)
    return ids.to(torch.int32)


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


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    act = _TYPES[case["act"]]
    s = {"case": case}
    if case["op"] == "route":
        logits = 1.5 * torch.randn(case["T"], case["E"], generator=g, device="cuda")
        if case["masked"]:
            off = torch.rand(case["T"], case["E"], generator=g, device="cuda") < case["masked"]
            off |= torch.rand(case["T"], 1, generator=g, device="cuda") < case["masked"] / 50   # a padded token
            logits = logits.masked_fill(off, -math.inf)
        s["logits"] = logits.to(act)
        return s
    if case["op"] == "combine":
        ids = _choices(g, case["T"], case["E"], case["k"], 1.0, case["masked"])
        _, _, slots = _rows_by_expert(ids, case["E"])
        w = torch.rand(case["T"], case["k"], generator=g, device="cuda")
        s["weights"] = torch.where(ids < 0, torch.zeros_like(w), w / w.sum(1, keepdim=True))
        s["slots"] = slots.to(torch.int32)
        s["y"] = torch.randn(case["T"] * case["k"], case["C"], generator=g, device="cuda").to(act)
        return s
    c_in, c_out, tau = case["c_in"], case["c_out"], case["tau"]
    E = case["E"] if case["op"] == "experts" else 1
    s["codes"], s["idx"], s["alpha"] = _weights(g, E, c_in, c_out, tau)
    if case["op"] == "experts":
        ids = _choices(g, case["T"], E, case["k"], case["skew"])
        counts, rows, _ = _rows_by_expert(ids, E)
        s["sizes"] = counts.tolist()
        s["offsets"] = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).to(torch.int32)
        s["rows"] = rows.to(torch.int32) if case["gather"] else None
        n = case["T"] if case["gather"] else case["T"] * case["k"]
        s["x"] = torch.randn(n, c_in, generator=g, device="cuda").to(act)
        return s
    n, rank, R = case["n"], case["rank"], case["R"]
    s["x"] = torch.randn(R, c_in, generator=g, device="cuda").to(act)
    # runs of rows of one request each; one in eight without an adapter
    request = torch.arange(R, device="cuda") // case["run"]
    pick = torch.randint(0, 8 * n, (int(request[-1]) + 1,), generator=g, device="cuda")
    s["adapter"] = torch.where(pick % 8 == 7, torch.full_like(pick, -1), pick // 8)[request].to(torch.int32)
    s["a"] = (torch.randn(n, rank, c_in, generator=g, device="cuda") / math.sqrt(c_in)).to(act)
    s["b"] = (torch.randn(n, c_out, rank, generator=g, device="cuda") / math.sqrt(rank)).to(act)
    s["scale"] = 0.25 + torch.rand(n, generator=g, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    out = _TYPES[case["out"]] if "out" in case else None
    if op == "combine":
        s["out"] = torch.empty(case["T"], case["C"], dtype=out, device="cuda")
    elif op == "experts":
        s["out"] = torch.empty(case["T"] * case["k"], case["c_out"], dtype=out, device="cuda")
        s["place"] = _places(s["sizes"])
    elif op == "adapters":
        s["out"] = torch.empty(case["R"], case["c_out"], dtype=out, device="cuda")
    if own:
        import paper_2110_09195_b200 as snn
        s["snn"] = snn
        if op == "route":
            s["out"] = snn.alloc_route(case["T"], case["E"], case["k"])
        if op in ("experts", "adapters"):
            codes, stream, alpha = _stored(s["codes"], s["idx"], s["alpha"], case["tau"])
            layers = [snn.SnnConv(case["c_in"], case["c_out"], case["tau"], codes[e], stream[e], alpha[e], pad=0,
                                  act_type=snn.ACT_F16, ksize=1) for e in range(len(codes))]
            s["handle"] = snn.SnnConvExperts(layers) if op == "experts" else snn.SnnConvAdapters(layers[0])
            for layer in layers:
                layer.destroy()
    if op in ("experts", "adapters"):
        if not own:
            s["w"] = _decoded(s["codes"], s["idx"])
        del s["codes"], s["idx"]
    return s


def _places(sizes):
    """Where row i stands in a table [E, largest size]: the experts' rows side by side, padded."""
    cap = max(sizes)
    counts = torch.tensor(sizes, device="cuda")
    expert = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), counts)
    start = torch.repeat_interleave(torch.cumsum(counts, 0) - counts, counts)
    return expert * cap + torch.arange(len(expert), device="cuda") - start


# ------------------------------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        snn = s["snn"]
        if op == "route":
            return tuple(snn.route(s["logits"], case["k"], normalise=case["normalise"], out=s["out"]))
        if op == "combine":
            return snn.combine(s["y"], s["slots"], s["weights"], out=s["out"])
        if op == "experts":
            return s["handle"].forward(s["x"], s["offsets"], rows=s["rows"], out=s["out"])
        return s["handle"].forward(s["x"], s["adapter"], s["a"], s["b"], s["scale"], out=s["out"])
    return {"route": _plain_route, "combine": _plain_combine, "experts": _plain_experts, "adapters": _plain_adapters}[op](s)


def _plain_route(s):
    case = s["case"]
    E, k = case["E"], case["k"]
    logits = s["logits"].float()
    logits = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    largest = top[:, :1]
    rise = torch.where(logits == largest, torch.zeros_like(logits), logits - largest)
    e = torch.where(logits == -math.inf, torch.zeros_like(logits), torch.exp(rise))
    chosen = torch.gather(e, 1, ids[:, :k])
    total = chosen.sum(1, keepdim=True) if case["normalise"] else e.sum(1, keepdim=True)
    weights = torch.where(chosen > 0, chosen / total, torch.zeros_like(chosen))
    ids = torch.where(top[:, :k] == -math.inf, torch.full_like(ids[:, :k], -1), ids[:, :k]).to(torch.int32)
    counts, rows, slots = _rows_by_expert(ids, E)
    offsets = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0))
    return ids, weights, offsets.to(torch.int32), rows.to(torch.int32), slots.to(torch.int32)


def _plain_combine(s):
    y = s["y"].float()[s["slots"].clamp(min=0).long()]                 # [T, k, C]
    w = torch.where(s["slots"] < 0, torch.zeros_like(s["weights"]), s["weights"])
    return (y * w[:, :, None]).sum(1).to(s["out"].dtype)


def _plain_experts(s):
    x = s["x"].float() if s["rows"] is None else s["x"].float()[s["rows"].long()]
    E, cap = len(s["sizes"]), max(s["sizes"])
    table = torch.zeros(E * cap, x.shape[1], device="cuda")
    table[s["place"]] = x
    y = torch.bmm(table.reshape(E, cap, -1), s["w"].float().transpose(1, 2)) * s["alpha"][:, None, :]
    return y.reshape(E * cap, -1)[s["place"]].to(s["out"].dtype)


def _plain_adapters(s):
    case = s["case"]
    n, rank, R = case["n"], case["rank"], case["R"]
    x = s["x"].float()
    y = (x @ s["w"][0].float().T) * s["alpha"][0]
    mine = (s["adapter"][:, None] == torch.arange(n, device="cuda")[None, :]).float() * s["scale"][None, :]
    h = (x @ s["a"].float().reshape(n * rank, -1).T).reshape(R, n, rank) * mine[:, :, None]
    y = y + h.reshape(R, n * rank) @ s["b"].float().permute(0, 2, 1).reshape(n * rank, -1)
    return y.to(s["out"].dtype)


# ------------------------------------------------------------------------------------------------------- costs, oracle

def work(case):
    """Each input read once (projections in their stored form, of the experts that rows can go to), each output written once."""
    op = case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * _SIZE[case["act"]] + T * k * 16 + 4 * (E + 1), "flops": 4 * T * E}
    if op == "combine":
        T, k, C = case["T"], case["k"], case["C"]
        return {"bytes": T * k * (C * _SIZE[case["act"]] + 8) + T * C * _SIZE[case["out"]], "flops": 2 * T * k * C}
    c_in, c_out = case["c_in"], case["c_out"]
    stored = c_in * c_out // 8 * case["tau"] / 8 + 4 * c_out + (2 << case["tau"])
    if op == "experts":
        R = case["T"] * case["k"]
        read = (case["T"] * c_in * 2 + 4 * R) if case["gather"] else R * c_in * 2
        return {"bytes": read + min(case["E"], R) * stored + R * c_out * _SIZE[case["out"]] + 4 * (case["E"] + 1),
                "flops": 2 * R * c_in * c_out}
    R, n, rank = case["R"], case["n"], case["rank"]
    used = min(n, -(-R // case["run"]))
    return {"bytes": R * c_in * 2 + stored + used * rank * (c_in + c_out) * 2 + R * (c_out * _SIZE[case["out"]] + 4),
            "flops": 2 * R * c_in * c_out + 2 * R * rank * (c_in + c_out)}


def _signs64(codes, idx):
    """+1 / -1 in 64 bits of one projection, element by element from the codes."""
    code = codes[idx.long()]                                            # [c_out, G]
    parts = [torch.where((code // (1 << (7 - j))) % 2 == 1, 1.0, -1.0).double() for j in range(8)]
    return torch.stack(parts, 2).reshape(idx.shape[0], -1)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        logits = s["logits"].double().cpu().numpy()
        weights, ids = np.zeros((T, k)), np.full((T, k), -1, dtype=np.int32)
        by_expert = [[] for _ in range(E)]
        for t in range(T):
            able = [e for e in range(E) if logits[t, e] > -math.inf]
            if not able:
                continue
            best = sorted(able, key=lambda e: (-logits[t, e], e))[:k]
            over = best if case["normalise"] else able
            top = logits[t, best[0]]
            total = math.fsum(math.exp(logits[t, e] - top) for e in over)
            for j, e in enumerate(best):
                ids[t, j], weights[t, j] = e, math.exp(logits[t, e] - top) / total
                by_expert[e].append((t, j))
        offsets, rows, slots = np.zeros(E + 1, np.int32), np.full(T * k, -1, np.int32), np.full((T, k), -1, np.int32)
        i = 0
        for e in range(E):
            for t, j in by_expert[e]:
                rows[i], slots[t, j] = t, i
                i += 1
            offsets[e + 1] = i
        return tuple(torch.from_numpy(v) for v in (ids, weights, offsets, rows, slots))
    if op == "combine":
        out = torch.zeros(case["T"], case["C"], dtype=torch.float64, device="cuda")
        for j in range(case["k"]):
            have = (s["slots"][:, j] >= 0).nonzero()[:, 0]
            out[have] += s["weights"][have, j].double()[:, None] * s["y"][s["slots"][have, j].long()].double()
        return out
    if op == "experts":
        ends = np.cumsum(s["sizes"])
        out = torch.zeros(case["T"] * case["k"], case["c_out"], dtype=torch.float64, device="cuda")
        for e, (end, size) in enumerate(zip(ends, s["sizes"])):
            if size:
                part = slice(int(end) - size, int(end))
                x = s["x"][part] if s["rows"] is None else s["x"][s["rows"][part].long()]
                out[part] = (x.double() @ _signs64(s["codes"][e], s["idx"][e]).T) * s["alpha"][e].double()
        return out
    out = (s["x"].double() @ _signs64(s["codes"][0], s["idx"][0]).T) * s["alpha"][0].double()
    for a in range(case["n"]):
        mine = (s["adapter"] == a).nonzero()[:, 0]
        if len(mine):
            h = s["x"][mine].double() @ s["a"][a].double().T
            out[mine] += s["scale"][a].double() * (h @ s["b"][a].double().T)
    return out
