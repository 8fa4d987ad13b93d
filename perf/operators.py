"""Operators next to the quantized linear, as cases that can be timed and compared.

Four operators, in three kinds of case:

  epilogue  the quantized linear with what follows it in a block (bias, activation or gate, residual) in
            its epilogue: fp16 activations in, fp16 results out
  route     the router of a layer of experts: scores, a bias for balance, groups of experts, top-k,
            weights, and the lists of rows per expert that the experts' products read
  experts   one of the two products of a layer of experts with mixed-precision weights: "up" takes the
            tokens' activations to the gated hidden rows of their experts, "down" the hidden rows back,
            followed by the weighted sum of every token's rows and the residual

Weights are the codes, scales and zero points that the library's pack_weights takes, held per expert in the
original channel order.  `own` says whose computation `run` is: the plain form in torch, or the library's.
"""
import math

import numpy as np
import torch

own = False

# the largest experts and the most pairs of activation and weight that a case has
MOST_WEIGHTS = 64 * 2816 * 4096
MOST_MACS = 2048 * 28672 * 4096
GROUP = 128


def listed():
    return [
        # one token: the output projection of a block of synth.LLAMA3_8B with the block's residual, where launches count
        {"name": "token_o_residual", "kind": "epilogue", "M": 1, "K": 4096, "N": 4096, "share": 0.1, "grouped": False,
         "bias": False, "act": "none", "gated": False, "residual": True},
        # a decode batch through the gated up projection of that block: the weight stream
        {"name": "batch16_gate_up", "kind": "epilogue", "M": 16, "K": 4096, "N": 28672, "share": 0.1, "grouped": False,
         "bias": False, "act": "silu", "gated": True, "residual": False},
        # a short ragged prompt through the long down projection with bias and residual, scales per group of 128 on both sides
        {"name": "ragged333_down", "kind": "epilogue", "M": 333, "K": 14336, "N": 4096, "share": 0.2, "grouped": True,
         "bias": True, "act": "none", "gated": False, "residual": True},
        # a chunk of a prompt through the gated up projection: the largest product
        {"name": "prompt2048_gate_up", "kind": "epilogue", "M": 2048, "K": 4096, "N": 28672, "share": 0.1, "grouped": False,
         "bias": False, "act": "silu", "gated": True, "residual": False},
        # one token of a served sequence: a launch or two
        {"name": "route_token", "kind": "route", "T": 1, "E": 64, "k": 4, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "group_score": "max", "renormalize": True, "scale": 1.0, "half": False, "padded": False},
        # a decode batch, padded, with sigmoid scores, a balancing bias and groups of experts
        {"name": "route_batch_groups", "kind": "route", "T": 61, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "group_score": "top2", "renormalize": True, "scale": 2.5, "half": False, "padded": True},
        # a long prompt
        {"name": "route_prompt", "kind": "route", "T": 16384, "E": 128, "k": 8, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "group_score": "max", "renormalize": True, "scale": 1.0, "half": True, "padded": False},
        # one token through its four experts, up and down: the stream of four experts' weights
        {"name": "token_up", "kind": "experts", "way": "up", "T": 1, "E": 64, "k": 4, "K": 4096, "N": 2816, "share": 0.1,
         "grouped": False, "act": "silu", "bias": False, "residual": False},
        {"name": "token_down", "kind": "experts", "way": "down", "T": 1, "E": 64, "k": 4, "K": 1408, "N": 4096, "share": 0.1,
         "grouped": False, "act": "none", "bias": False, "residual": True},
        # a serving batch of an odd size, a few rows for every expert, scales per group of 128 on both sides
        {"name": "batch53_up", "kind": "experts", "way": "up", "T": 53, "E": 64, "k": 4, "K": 4096, "N": 2816, "share": 0.1,
         "grouped": True, "act": "silu", "bias": False, "residual": False},
        # a chunk of a prompt: hundreds of rows for an expert, up and down
        {"name": "prompt4096_up", "kind": "experts", "way": "up", "T": 4096, "E": 64, "k": 4, "K": 4096, "N": 2816, "share": 0.1,
         "grouped": False, "act": "silu", "bias": False, "residual": False},
        {"name": "prompt4096_down", "kind": "experts", "way": "down", "T": 4096, "E": 64, "k": 4, "K": 1408, "N": 4096, "share": 0.1,
         "grouped": False, "act": "none", "bias": False, "residual": True},
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["epilogue", "route", "experts", "experts"])
    share, grouped = rng.choice([0.0, 0.05, 0.1, 0.1, 0.2, 0.5]), rng.random() < 0.3
    if kind == "route":
        size, groups = rng.choice([(1, 1), (1, 1), (4, 8), (16, 4), (32, 8), (20, 8)])
        E = size * groups if groups > 1 else rng.randint(8, 256)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(10, E // groups * top_groups))
        return {"kind": kind, "T": _spread(rng, 1, 16384 * 128 // max(E, 128)), "E": E, "k": k, "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups, "group_score": rng.choice(["max", "top2"]),
                "renormalize": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5]), "half": rng.random() < 0.5, "padded": rng.random() < 0.5}
    if kind == "epilogue":
        gated = rng.random() < 0.5
        K = GROUP * _spread(rng, 4, 224)
        N = _spread(rng, 64, min(28672, 2048 * 57344 // K))
        N += N % 2
        return {"kind": kind, "M": _spread(rng, 1, min(8192, MOST_MACS // (K * N))), "K": K, "N": N, "share": share, "grouped": grouped,
                "bias": rng.random() < 0.5, "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"] if gated else ["none", "none", "relu", "silu", "gelu", "gelu_tanh"]),
                "gated": gated, "residual": rng.random() < 0.5}
    way = rng.choice(["up", "down"])
    K = GROUP * _spread(rng, 4, 40)
    N = 2 * _spread(rng, 64, 2560)
    E = rng.randint(4, max(4, min(64, MOST_WEIGHTS // (K * N))))
    k = rng.randint(1, min(8, E))
    return {"kind": kind, "way": way, "T": _spread(rng, 1, min(8192, 4096 * 4 * 2816 * 4096 // (k * K * N))), "E": E, "k": k, "K": K, "N": N,
            "share": share, "grouped": grouped, "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh"]) if way == "up" else "none",
            "bias": rng.random() < 0.3, "residual": way == "down" and rng.random() < 0.7}


# ---- inputs -------------------------------------------------------------------------------------

def _gated(case):
    return case["gated"] if case["kind"] == "epilogue" else case["way"] == "up"


def _codes(W, eight, grouped):
    """Codes (int8), scales (fp16) and zero points of weights [N, K]: channels of `eight` symmetric in 8 bits
    (zero point 0, a scale per channel or per group), the others asymmetric in 4 bits with groups of 128."""
    N, K = W.shape
    g = W.float().view(N, K // GROUP, GROUP)
    lo, hi = g.amin(2).clamp(max=0), g.amax(2).clamp(min=0)
    top = g.abs().amax(2)
    if not grouped:
        top = top.amax(1, keepdim=True).expand(-1, K // GROUP)
    s = torch.where(eight[:, None], top / 127, (hi - lo) / 15).half()
    s = torch.where(s == 0, torch.ones_like(s), s)
    z = torch.where(eight[:, None], torch.zeros_like(lo), torch.round(-lo / s.float()).clamp(0, 15))
    q = torch.round(g / s.float()[..., None])
    q = torch.where(eight[:, None, None], q.clamp(-127, 127), (q + z[..., None]).clamp(0, 15))
    return q.view(N, K).to(torch.int8), s, z.to(torch.uint8)


def _weights(case, E, gen):
    """E layers of N x K: codes in channel order, and which channels have 8 bits (an uneven number of them over
    the experts, the way a choice over all of a model's channels leaves it; gate and up of a pair alike)."""
    K, N, pair = case["K"], case["N"], 2 if _gated(case) else 1
    q = torch.empty((E, N, K), dtype=torch.int8, device="cuda")
    s = torch.empty((E, N, K // GROUP), dtype=torch.float16, device="cuda")
    z = torch.empty((E, N, K // GROUP), dtype=torch.uint8, device="cuda")
    eight = torch.zeros((E, N), dtype=torch.bool, device="cuda")
    for e in range(E):
        W = torch.randn((N, K), generator=gen, device="cuda", dtype=torch.float16) * 0.02
        W[torch.randperm(N, generator=gen, device="cuda")[: max(1, N // 64)]] *= 4.0
        n8 = int(case["share"] * (N // pair) * (1 if E == 1 else 0.5 + e / (E - 1)))
        widest = W.abs().amax(1).view(-1, pair).amax(1).topk(n8).indices
        eight[e].view(-1, pair)[widest] = True
        q[e], s[e], z[e] = _codes(W, eight[e], case["grouped"])
    return {"q": q, "s": s, "z": z}, eight


def _pack(mx, weights, eight, grouped, e):
    q, s, z = weights["q"][e], weights["s"][e], weights["z"][e]
    a, b = eight[e].nonzero().view(-1), (~eight[e]).nonzero().view(-1)
    K = q.shape[1]
    s8 = s[a] if grouped else s[a, :1].contiguous()
    return mx.pack_weights(q[a] if len(a) else None, s8 if len(a) else None, q[b].to(torch.uint8) if len(b) else None,
                           s[b] if len(b) else None, z[b] if len(b) else None, torch.cat([a, b]).to(torch.int32), K, GROUP if grouped else None)


def _activations(M, K, hidden, gen):
    """N(0, 1) with one input channel in 100 twenty times as large, or, hidden, products of two normal values."""
    x = torch.randn((M, K), generator=gen, device="cuda", dtype=torch.float16)
    if hidden:
        return x * torch.randn((M, K), generator=gen, device="cuda", dtype=torch.float16)
    x[:, torch.randperm(K, generator=gen, device="cuda")[: max(1, K // 100)]] *= 20.0
    return x


def _logits(T, E, gen):
    """N(0, 1) around every expert's own mean: some experts are asked often, some seldom."""
    return torch.randn((T, E), generator=gen, device="cuda") + 0.5 * torch.randn(E, generator=gen, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    half = lambda *size: torch.randn(size, generator=gen, device="cuda", dtype=torch.float16)
    if own:
        import paper_2412_14590_amd as mx
        state["mx"] = mx
    if case["kind"] == "route":
        T, E = case["T"], case["E"]
        logits = _logits(T, E, gen)
        state["logits"] = logits.half() if case["half"] else logits
        state["bias"] = 0.1 * torch.randn(E, generator=gen, device="cuda") if case["bias"] else None
        # a padded batch: about one token in ten is none
        state["mask"] = torch.rand(T, generator=gen, device="cuda") < 0.9 if case["padded"] else None
        return state
    if case["kind"] == "epilogue":
        M, K, N = case["M"], case["K"], case["N"]
        weights, eight = _weights(case, 1, gen)
        state.update(weights=weights, x=_activations(M, K, False, gen), bias=half(N) if case["bias"] else None,
                     residual=half(M, N // 2 if _gated(case) else N) if case["residual"] else None)
        if own:   # the layer as a model holds it
            state["layer"] = _pack(mx, weights, eight, case["grouped"], 0)
        return state
    T, E, k, K, N = (case[n] for n in ("T", "E", "k", "K", "N"))
    weights, eight = _weights(case, E, gen)
    weight, ids = _logits(T, E, gen).softmax(1).topk(k, 1)
    route = _lists(ids.to(torch.int32), E)
    route["weights"] = weight / weight.sum(1, keepdim=True)
    up = case["way"] == "up"
    state.update(weights=weights, route=route, x=_activations(T if up else T * k, K, not up, gen), bias=half(E, N) if case["bias"] else None,
                 residual=half(T, N) if case["residual"] else None)
    if own:   # the experts and the route as a model holds them
        state["layer"] = mx.pack_experts([_pack(mx, weights, eight, case["grouped"], e) for e in range(E)])
        state["plan"] = mx.Route(**route)
    return state


# ---- the plain form -------------------------------------------------------------------------------

def _lists(ids, E):
    """The assignments t k + j sorted by their experts: where every expert's begin, the sorted list (-1 behind the
    last), and every assignment's place in it (-1 for none)."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.long, device=ids.device).index_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([counts.new_zeros(1), counts[:E].cumsum(0)]).to(torch.int32)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=ids.device)
    return {"ids": ids, "offsets": offsets, "rows": torch.where(key[order] < E, order, -1).to(torch.int32),
            "slots": torch.where(key < E, place, -1).to(torch.int32).view(ids.shape)}


def _route(case, logits, bias, mask):
    T, E, k = case["T"], case["E"], case["k"]
    lowest = float("-inf")
    l = logits.double()   # 64 bits: two experts of nearly the same score keep their order
    able = l > lowest
    if mask is not None:
        able = able & mask[:, None]
    if case["score"] == "softmax":
        p = torch.exp(l - l.amax(1, keepdim=True))
        score = p / p.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-l))
    choice = score if bias is None else score + bias.double()
    choice = torch.where(able, choice, lowest)
    if case["groups"] > 1:
        best = choice.view(T, case["groups"], -1).sort(2, descending=True).values
        of_group = best[:, :, 0]
        if case["group_score"] == "top2" and best.shape[2] > 1:
            of_group = of_group + torch.where(best[:, :, 1] > lowest, best[:, :, 1], 0)
        chosen = of_group.sort(dim=1, descending=True, stable=True).indices[:, : case["top_groups"]]
        kept = torch.zeros_like(of_group, dtype=torch.bool).scatter_(1, chosen, True)
        choice = torch.where(kept.repeat_interleave(E // case["groups"], 1), choice, lowest)
    value, ids = choice.sort(dim=1, descending=True, stable=True)
    value, ids = value[:, :k], ids[:, :k]
    taken = value > lowest
    w = torch.where(taken, score.gather(1, ids), 0)
    if case["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0)
    out = _lists(torch.where(taken, ids, -1).to(torch.int32), E)
    out["weights"] = (w * case["scale"]).float()
    return out


def _quantized(x, grouped):
    """Activations as the values that their int8 codes stand for, one scale per token or per token and group."""
    M, K = x.shape
    v = x.float().view(M, -1, GROUP if grouped else K)
    s = (v.abs().amax(2, keepdim=True) / 127).half().float()
    s = torch.where(s == 0, 1.0, s)
    return (torch.round(v / s).clamp(-127, 127) * s).view(M, K)


def _values(weights, which):
    """Weights [n, N, K] of the layers `which`, as the values that their codes stand for."""
    q, s, z = weights["q"][which], weights["s"][which], weights["z"][which]
    v = (q.view(*s.shape, GROUP).float() - z[..., None].float()) * s[..., None].float()
    return v.view(q.shape)


def _act(name, v):
    if name == "relu":
        return v.clamp(min=0)
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _finish(case, v, residual):
    """Activation (of the gates, even channels, times the odd ones) and residual."""
    v = _act(case["act"], v[..., 0::2]) * v[..., 1::2] if _gated(case) else _act(case["act"], v)
    return v if residual is None else v + residual.float()


def _experts(case, state):
    """Rows in the order of the route: those of an expert against its weights, by one product over all experts that
    have rows, each padded to the longest."""
    route, k = state["route"], case["k"]
    rows = route["rows"].long()
    expert = route["ids"].reshape(-1).long()[rows]
    x = _quantized(state["x"], case["grouped"])
    x = x[rows // k] if case["way"] == "up" else x
    active, at = torch.unique(expert, return_inverse=True)   # (sorted, as the rows are)
    within = torch.arange(rows.numel(), device=rows.device) - route["offsets"].long()[expert]
    padded = x.new_zeros((active.numel(), int(within.max()) + 1, case["K"]))
    padded[at, within] = x
    v = torch.bmm(padded, _values(state["weights"], active).transpose(1, 2).contiguous())[at, within]
    if state["bias"] is not None:
        v = v + state["bias"].float()[expert]
    return _finish(case, v, None).half()


def _combine(case, state, y):
    route = state["route"]
    v = (y.float()[route["slots"].long()] * route["weights"][..., None]).sum(1)
    return (v if state["residual"] is None else v + state["residual"].float()).half()


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    group = GROUP if case.get("grouped") else None
    if case["kind"] == "route":
        if own:
            r = state["mx"].route_experts(state["logits"], case["k"], score=case["score"], bias=state["bias"], mask=state["mask"],
                                          groups=case["groups"], top_groups=case["top_groups"], group_score=case["group_score"],
                                          renormalize=case["renormalize"], scale=case["scale"])
            return {"ids": r.ids, "weights": r.weights, "offsets": r.offsets, "rows": r.rows, "slots": r.slots}
        return _route(case, state["logits"], state["bias"], state["mask"])
    if case["kind"] == "epilogue":
        if own:
            return state["mx"].linear_fp16_epilogue(state["x"], state["layer"], bias=state["bias"], activation=case["act"], gated=case["gated"],
                                                    residual=state["residual"], act_group=group)
        v = _quantized(state["x"], case["grouped"]) @ _values(state["weights"], slice(0, 1))[0].t()
        if state["bias"] is not None:
            v = v + state["bias"].float()
        return _finish(case, v, state["residual"]).half()
    up = case["way"] == "up"
    if own:
        mx = state["mx"]
        y = mx.experts_linear_fp16(state["x"], state["layer"], state["plan"], bias=state["bias"], activation=case["act"], gated=up, gather=up,
                                   act_group=group)
        return y if up else mx.experts_combine(y, state["plan"], residual=state["residual"])
    y = _experts(case, state)
    return y if up else _combine(case, state, y)


# ---- what a pass cannot do without ------------------------------------------------------------------

def _layer_bytes(case, share):
    """Half a byte per 4-bit weight and 2.5 bytes per group of 128, a byte per 8-bit weight and 2 per scale, 4 per channel."""
    K, N = case["K"], case["N"]
    n8, ng = int(share * N), K // GROUP
    return (N - n8) * (K / 2 + 2.5 * ng) + n8 * (K + 2 * (ng if case["grouped"] else 1)) + 4 * N


def work(case):
    if case["kind"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * (2 if case["half"] else 4) + 16 * T * k + 4 * (E + 1) + (4 * E if case["bias"] else 0) + (T if case["padded"] else 0),
                "flops": 4 * T * E}
    K, N = case["K"], case["N"]
    Nout = N // 2 if _gated(case) else N
    if case["kind"] == "epilogue":
        M = case["M"]
        return {"bytes": _layer_bytes(case, case["share"]) + 2 * M * K + 2 * M * Nout * (2 if case["residual"] else 1) + (2 * N if case["bias"] else 0),
                "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    R = T * k
    busy = E * (1 - (1 - k / E) ** T)   # experts that have a row, were all equally likely
    # the rows' lists; down: the rows again in the sum, which a kernel over both need not write out
    nbytes = busy * (_layer_bytes(case, case["share"]) + (2 * N if case["bias"] else 0)) + 2 * K * (T if case["way"] == "up" else R) + 4 * R + 4 * (E + 1)
    nbytes += 2 * R * Nout if case["way"] == "up" else 2 * T * N * (2 if case["residual"] else 1) + 8 * R
    return {"bytes": nbytes, "flops": 2 * R * N * K + (0 if case["way"] == "up" else 2 * R * N)}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------

def _exact_quantized(x, group):
    """Codes and scales of the definition (scale = fp16 of the largest magnitude over 127), and their products."""
    v = x.double().reshape(x.shape[0], x.shape[1] // group, group)
    s = (torch.max(v.max(2).values, -v.min(2).values) / 127.0).to(torch.float16).double()
    s[s == 0] = 1.0
    return (torch.clamp(torch.round(v / s.unsqueeze(2)), -127, 127) * s.unsqueeze(2)).reshape(x.shape)


def _exact_rows(case, x, weights, e, bias):
    q, s, z = (weights[n][e].double() for n in ("q", "s", "z"))
    w = (q - z.repeat_interleave(GROUP, 1)) * s.repeat_interleave(GROUP, 1)
    v = torch.matmul(x, w.T.contiguous())
    if bias is not None:
        v += bias.double()
    a = v[:, ::2] if _gated(case) else v
    name = case["act"]
    if name == "relu":
        a = torch.relu(a)
    elif name == "silu":
        a = a * torch.sigmoid(a)
    elif name == "gelu":
        a = a * torch.special.ndtr(a)
    elif name == "gelu_tanh":
        a = a * torch.sigmoid(math.sqrt(8 / math.pi) * (a + 0.044715 * a ** 3))
    return a * v[:, 1::2] if _gated(case) else a


def _exact_route(case, logits, bias, mask):
    l = logits.double().cpu().numpy()
    b = np.zeros(case["E"]) if bias is None else bias.double().cpu().numpy()
    on = np.ones(len(l), bool) if mask is None else mask.cpu().numpy()
    T, E, k, size = case["T"], case["E"], case["k"], case["E"] // case["groups"]
    if case["score"] == "softmax":
        s = np.exp(l - np.logaddexp.reduce(l, axis=1)[:, None])
    else:
        s = np.exp(-np.logaddexp(0, -l))
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    c = s + b
    top = np.sort(c.reshape(T, case["groups"], size), axis=2)
    group = top[:, :, -1] + (top[:, :, -2] if case["group_score"] == "top2" and size > 1 else 0)
    for t in np.nonzero(on)[0]:
        experts = np.arange(E)
        if case["groups"] > 1:
            best = np.argsort(-group[t], kind="stable")[: case["top_groups"]]
            experts = np.sort(np.concatenate([np.arange(j * size, (j + 1) * size) for j in best]))
        ids[t] = experts[np.argsort(-c[t, experts], kind="stable")[:k]]
        w[t] = s[t, ids[t]]
        if case["renormalize"]:
            w[t] /= w[t].sum()
    per = [np.nonzero(ids.reshape(-1) == e)[0] for e in range(E)]
    order = np.concatenate(per)
    rows, slots = np.full(T * k, -1, np.int32), np.full(T * k, -1, np.int32)
    rows[: len(order)] = order
    slots[order] = np.arange(len(order))
    return {"ids": ids, "weights": w * case["scale"], "offsets": np.cumsum([0] + [len(p) for p in per]).astype(np.int32), "rows": rows,
            "slots": slots.reshape(T, k)}


def exact(case, seed):
    state = prepare(case, seed)
    bias, residual = state["bias"], state.get("residual")
    if case["kind"] == "route":
        return _exact_route(case, state["logits"], bias, state["mask"])
    x = _exact_quantized(state["x"], GROUP if case["grouped"] else case["K"])
    if case["kind"] == "epilogue":
        y = _exact_rows(case, x, state["weights"], 0, bias)
        return y if residual is None else y + residual.double()
    route, k = state["route"], case["k"]
    starts = route["offsets"].tolist()
    order = route["rows"].long()
    N = case["N"]
    y = torch.zeros((len(order), N // 2 if _gated(case) else N), dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        a, b = starts[e], starts[e + 1]
        if b > a:
            y[a:b] = _exact_rows(case, x[order[a:b] // k] if case["way"] == "up" else x[a:b], state["weights"], e, None if bias is None else bias[e])
    if case["way"] == "up":
        return y
    total = torch.zeros((case["T"], N), dtype=torch.float64, device="cuda") if residual is None else residual.double()
    total.index_add_(0, order // k, y * route["weights"].double().reshape(-1)[order].unsqueeze(1))
    return total
