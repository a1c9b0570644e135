"""What the operators for mixtures of many experts, and for 4-bit experts, are measured by.

A case is one pass through one operator, of one of four kinds:

  route      scores, group-limited top-k selection, gates and the grouping of the (token, slot) pairs by expert
  route_bwd  the gradient of the logits, from those of the gates (and of the scores)
  quant      a tensor to microscaled 4-bit floats (MXFP4: e2m1 values, one power of two for 32 of them) and back: the
             values that the 4 bits stand for.  axis 1: blocks along the rows, as activations are quantised; axis 0:
             along the columns, as the expert weights [E, K, N] are, whose products sum over K
  layer      the feed-forward layer of 4-bit experts: token rows and SwiGLU activations are quantised on the way,
             the products take 4-bit operands, the gates weigh the experts' outputs

`own` False: elementary torch operations in 32 bits (64 for the scores, which are compared with each other); True: the
framework's entry points.
"""
import math
from types import SimpleNamespace

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32                                     # elements that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of e2m1, by code
TINY = 1e-20                                   # added to the sum that gates are divided by


def route_case(kind, T, E, k, groups=1, keep=1, score="sigmoid", gscore="top2", bias=True, renorm=True, scale=1.0, dtype="f32",
               dscores=False):
    return dict(kind=kind, T=T, E=E, k=k, groups=groups, keep=keep, score=score, gscore=gscore, bias=bias, renorm=renorm, scale=scale,
                dtype=dtype, dscores=dscores)


def layer_case(T, d, f, E, k, residual=False):
    return dict(kind="layer", T=T, d=d, f=f, E=E, k=k, dtype="bf16", residual=residual)


def listed():
    cases = {
        # one decoding step of 16 sequences: nothing but latency
        "route_decode_16": route_case("route", 16, 64, 8, groups=8, keep=4, scale=2.5),
        # a prompt of an odd length, experts in four groups of 15, softmax scores of bf16 logits, no bias
        "route_prompt_301": route_case("route", 301, 60, 6, groups=4, keep=2, score="softmax", gscore="max", bias=False, renorm=False,
                                       dtype="bf16"),
        # the training batch of the benchmark (four sequences), 256 experts in 8 groups
        "route_train_16384": route_case("route", 16384, 256, 8, groups=8, keep=4, scale=2.5),
        # its gradient
        "route_bwd_16384": route_case("route_bwd", 16384, 256, 8, groups=8, keep=4, scale=2.5),
        # one ragged sequence of a softmax router whose scores carry a loss of their own
        "route_bwd_4001": route_case("route_bwd", 4001, 64, 4, score="softmax", gscore="max", bias=False, dtype="bf16", dscores=True),
        # the rows of a short prompt
        "quant_rows_301": dict(kind="quant", batch=1, rows=301, cols=4096, axis=1, dtype="bf16"),
        # a stack of experts' up-projections, once per model
        "quant_experts": dict(kind="quant", batch=4, rows=4096, cols=11008, axis=0, dtype="bf16"),
        # one token: the weights of two experts are read for a row each
        "layer_decode_1": layer_case(1, 4096, 11008, 4, 2, residual=True),
        # a decoding step of 64 sequences, 32 split experts of width 1376: about 16 rows each, all weights read
        "layer_decode_64_split": layer_case(64, 4096, 1376, 32, 8, residual=True),
        # a prompt of an odd length: about 150 rows an expert
        "layer_prompt_301": layer_case(301, 4096, 11008, 4, 2),
        # four sequences through split experts: 4096 rows each, short sums
        "layer_16384_split": layer_case(16384, 4096, 1376, 32, 8),
        # four sequences through the 7B-shaped layer
        "layer_16384": layer_case(16384, 4096, 11008, 4, 2),
    }
    return [dict(name=name, **case) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for; never more work than the largest of its kind."""
    what = rng.choice(["route", "route", "route_bwd", "quant", "layer", "layer", "layer"])
    if what in ("route", "route_bwd"):
        groups = rng.choice([1, 1, 2, 4, 8, 8, 16])
        per = _log_int(rng, max(1, 4 // groups), 256 // groups)
        E, keep = groups * per, rng.randint(1, groups)
        k = rng.randint(1, min(8, keep * per))
        renorm = rng.random() < 0.7 and (k > 1 or what == "route")     # the only gate, renormalised, is a constant: no gradient
        return route_case(what, _log_int(rng, 1, 16384), E, k, groups, keep, rng.choice(["sigmoid", "softmax"]), rng.choice(["top2", "max"]),
                          rng.random() < 0.6, renorm, rng.choice([1.0, 2.5]), rng.choice(["f32", "f32", "bf16"]),
                          what == "route_bwd" and rng.random() < 0.4)
    if what == "quant":
        axis, dtype = rng.randint(0, 1), rng.choice(["bf16", "bf16", "f32"])
        batch = rng.choice([1, 1, 2, 4])
        blocked, other = BLOCK * _log_int(rng, 1, 344), _log_int(rng, 1, 16384)
        most = 4 * 4096 * 11008 // (batch * (2 if dtype == "f32" else 1))
        other = max(1, min(other, most // blocked))
        return dict(kind="quant", batch=batch, rows=blocked if axis == 0 else other, cols=other if axis == 0 else blocked, axis=axis,
                    dtype=dtype)
    E = rng.choice([1, 4, 4, 8, 16, 32, 33, 64])
    k = rng.randint(1, min(E, 8))
    d, f = BLOCK * _log_int(rng, 2, 128), BLOCK * _log_int(rng, 2, 344)
    f = min(f, BLOCK * max(1, 4 * 4096 * 11008 // (E * d * BLOCK)))
    T = min(_log_int(rng, 1, 16384), max(1, 32768 * 4096 * 11008 // (k * d * f)), max(1, 131072 // k))
    return layer_case(T, d, f, E, k, rng.random() < 0.5)


# ---- inputs --------------------------------------------------------------------------------------------------


def _randn(shape, seed, stream):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed * 7919 + stream), device="cuda")


def _logits(c, seed):
    # rows of unit mean square through a router of N(0, 0.02^2) weights 4096 deep
    return _randn((c["T"], c["E"]), seed, 1).mul_(1.28).to(DTYPES[c["dtype"]])


def _bias(c, seed):
    return _randn((c["E"],), seed, 2).mul_(0.05) if c["bias"] else None


def _encode(x):
    """[..., K] -> codes [..., K/2] (the element of the lower index in the low half of a byte) and scale bytes [..., K/32], as
    uint8: the format that the 4-bit experts are kept in."""
    rows, K = x.shape[:-1], x.shape[-1]
    v = x.float().reshape(*rows, K // BLOCK, BLOCK)
    byte = ((v.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp_(min=0)
    v = v * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)       # exact: a power of two
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code | (v < 0).to(torch.uint8) << 3).reshape(*rows, K // 2, 2)
    return code[..., 0] | code[..., 1] << 4, byte.to(torch.uint8)


def _scale_rows(byte):
    """Scale rows are padded with zeros to a multiple of 16 bytes."""
    return torch.nn.functional.pad(byte, (0, -byte.shape[-1] % 16)).contiguous()


def _experts(E, K, N, seed, stream):
    """N(0, 1/K) experts that drifted from one seed by a tenth, quantised along K: codes [E, N, K/2], scale rows."""
    base, codes, scales = _randn((N, K), seed, stream), [], []
    for e in range(E):
        w = (base + 0.1 * _randn((N, K), seed, stream + 1 + e)).mul_(K ** -0.5).bfloat16()
        c, s = _encode(w)
        codes.append(c)
        scales.append(_scale_rows(s))
    return torch.stack(codes), torch.stack(scales)


def _group(idx, E):
    """The stable grouping of the (token, slot) pairs by expert: counts, offsets, perm, inv_pos."""
    flat = idx.reshape(-1).long()
    perm = torch.sort(flat, stable=True).indices
    counts = (flat.unsqueeze(1) == torch.arange(E, device=idx.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(perm.numel(), device=perm.device)
    return counts.int(), offsets.int(), perm.int(), inv.int().reshape(idx.shape)


def prepare(case, seed):
    c = dict(case)
    s = dict(case=c)
    kind, dtype = c["kind"], DTYPES[c["dtype"]]
    if kind in ("route", "route_bwd"):
        s["logits"], s["bias"] = _logits(c, seed), _bias(c, seed)
    if kind == "route_bwd":
        # a routing of these logits, as a forward pass left it
        r = _plain_route(s)
        s["topk_idx"], s["gates"] = r["topk_idx"], r["gates"]
        s["dgates"] = _randn((c["T"], c["k"]), seed, 3).mul_(0.1)
        s["dscores"] = _randn((c["T"], c["E"]), seed, 4).mul_(0.01) if c["dscores"] else None
    elif kind == "quant":
        x = _randn((c["batch"], c["rows"], c["cols"]), seed, 5)
        s["x"] = (x if c["axis"] == 1 else x.mul_(c["rows"] ** -0.5)).to(dtype)
    elif kind == "layer":
        T, d, f, E, k = c["T"], c["d"], c["f"], c["E"], c["k"]
        x = _randn((T, d), seed, 6)
        s["x"] = (x * x.square().mean(1, keepdim=True).rsqrt()).to(dtype)
        s["residual"] = _randn((T, d), seed, 7).to(dtype) if c["residual"] else None
        s["W1"], s["W3"], s["W2"] = _experts(E, d, f, seed, 100), _experts(E, d, f, seed, 300), _experts(E, f, d, seed, 500)
        logits = _randn((T, E), seed, 8).mul_(1.28)
        top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
        counts, offsets, perm, inv = _group(idx[:, :k].contiguous(), E)
        s["routing"] = SimpleNamespace(topk_idx=idx[:, :k].int().contiguous(), gates=torch.softmax(top[:, :k], 1).contiguous(), counts=counts,
                                       offsets=offsets, perm=perm, inv_pos=inv)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """Outputs and workspaces that a program keeps between its calls."""
    from paper_2403_07816_amd import binding as B
    c, lib = s["case"], B.load_library()
    if c["kind"] == "route":
        s["out"] = B.alloc_group_routing(c["T"], c["E"], c["k"], "cuda")
        bytes_ = lib.btx_moe_group_route_workspace_bytes(c["T"], c["E"], c["k"])
    elif c["kind"] == "route_bwd":
        s["out"] = torch.empty_like(s["logits"])
        s["routing"] = SimpleNamespace(topk_idx=s["topk_idx"], gates=s["gates"])
        return
    elif c["kind"] == "quant":
        s["out"] = B.alloc_mx4(s["x"].shape, c["axis"] - 2, "cuda")
        s["back"] = torch.empty_like(s["x"])
        return
    else:
        s["out"] = torch.empty_like(s["x"])
        for name, K in (("W1", c["d"]), ("W3", c["d"]), ("W2", c["f"])):
            s[name] = B.Mx4(*s[name], K)
        bytes_ = lib.btx_moe_ff_forward_mx4_workspace_bytes(c["T"], c["d"], c["f"], c["E"], c["k"])
    s["ws"] = torch.empty(max(bytes_, 256), dtype=torch.uint8, device="cuda")


# ---- the plain form ------------------------------------------------------------------------------------------


def _scores(logits, score):
    l = logits.double()
    return torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1)


def _plain_route(s):
    c = s["case"]
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    scores = _scores(s["logits"], c["score"])
    v = scores + s["bias"].double() if s["bias"] is not None else scores
    if G > 1:
        best = torch.sort(v.reshape(T, G, E // G), dim=2, descending=True).values
        value = best[:, :, :2].sum(2) if c["gscore"] == "top2" else best[:, :, 0]
        kept = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :c["keep"]]
        inside = torch.zeros((T, G), dtype=torch.bool, device=v.device).scatter_(1, kept, True)
        v = torch.where(inside.repeat_interleave(E // G, dim=1), v, -math.inf)
    idx = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k].contiguous()
    w = scores.gather(1, idx)
    gates = c["scale"] * (w / (w.sum(1, keepdim=True) + TINY) if c["renorm"] else w)
    counts, offsets, perm, inv = _group(idx, E)
    return dict(topk_idx=idx.int(), gates=gates.float(), scores=scores.float(), counts=counts, offsets=offsets, perm=perm, inv_pos=inv)


def _plain_route_bwd(s):
    c = s["case"]
    scores, idx = _scores(s["logits"], c["score"]), s["topk_idx"].long()
    w, dg = scores.gather(1, idx), s["dgates"].double()
    if c["renorm"]:
        total = w.sum(1, keepdim=True) + TINY
        dw = c["scale"] * (dg - (dg * w).sum(1, keepdim=True) / total) / total
    else:
        dw = c["scale"] * dg
    ds = s["dscores"].double() if s["dscores"] is not None else torch.zeros_like(scores)
    ds = ds.scatter_add(1, idx, dw)
    if c["score"] == "sigmoid":
        dl = ds * scores * torch.sigmoid(-s["logits"].double())
    else:
        dl = scores * (ds - (ds * scores).sum(1, keepdim=True))
    return dl.to(s["logits"].dtype)


def _decode(codes, byte):
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    v = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).reshape(*codes.shape[:-1], -1, BLOCK)
    scale = (byte.int() << 23).view(torch.float32)                       # 2^(byte - 127), from its bits: exact
    return (v * torch.where(byte > 0, scale, 2.0 ** -127).unsqueeze(-1)).flatten(-2)


def _plain_quant(s):
    x = s["x"] if s["case"]["axis"] == 1 else s["x"].transpose(1, 2)
    v = torch.stack([_decode(*_encode(part)).to(x.dtype) for part in x])
    return v if s["case"]["axis"] == 1 else v.transpose(1, 2).contiguous()


def _weights(W, e):
    """Expert e's matrix [N, K]."""
    codes, scales = W
    return _decode(codes[e], scales[e][:, :codes.shape[2] * 2 // BLOCK])


def _plain_layer(s):
    c, r = s["case"], s["routing"]
    xq = _decode(*_encode(s["x"]))
    out = s["residual"].float() if s["residual"] is not None else torch.zeros_like(xq)
    for e in range(c["E"]):
        token, slot = (r.topk_idx == e).nonzero(as_tuple=True)
        if token.numel() == 0:
            continue
        xs = xq[token]
        h1, h3 = xs @ _weights(s["W1"], e).T, xs @ _weights(s["W3"], e).T
        act = _decode(*_encode(h1 * (1.0 / (1.0 + torch.exp(-h1))) * h3))
        out[token] += r.gates[token, slot].unsqueeze(1) * (act @ _weights(s["W2"], e).T)
    return out.to(s["x"].dtype)


# ---- one pass ------------------------------------------------------------------------------------------------


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"route": _plain_route, "route_bwd": _plain_route_bwd, "quant": _plain_quant, "layer": _plain_layer}[c["kind"]](s)
    from paper_2403_07816_amd import binding as B
    if c["kind"] in ("route", "route_bwd"):
        opts = dict(score_fn=B.BTX_SCORE_SIGMOID if c["score"] == "sigmoid" else B.BTX_SCORE_SOFTMAX, renorm=c["renorm"], scale=c["scale"])
        if c["kind"] == "route":
            r = B.btx_moe_group_route(s["logits"], c["k"], bias=s["bias"], n_groups=c["groups"], topk_groups=c["keep"],
                                      group_score=B.BTX_GROUP_TOP2 if c["gscore"] == "top2" else B.BTX_GROUP_MAX, out=s["out"],
                                      workspace=s["ws"], **opts)
            return dict(topk_idx=r.topk_idx, gates=r.gates, scores=r.scores, counts=r.counts, offsets=r.offsets, perm=r.perm,
                        inv_pos=r.inv_pos)
        return B.btx_moe_group_route_backward(s["logits"], s["routing"], s["dgates"], dscores=s["dscores"], out=s["out"], **opts)
    if c["kind"] == "quant":
        q = B.btx_mx4_quantize(s["x"], axis=c["axis"] - 2, out=s["out"])
        return B.btx_mx4_dequantize(q, s["x"].dtype, axis=c["axis"] - 2, out=s["back"])
    return B.btx_moe_ff_forward_mx4(s["x"], s["W1"], s["W3"], s["W2"], s["routing"], out=s["out"], workspace=s["ws"],
                                    residual=s["residual"])


# ---- what a pass cannot do without ---------------------------------------------------------------------------


def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] in ("route", "route_bwd"):
        T, E, k = c["T"], c["E"], c["k"]
        if c["kind"] == "route":     # logits in; scores, indices, gates, perm, inv_pos out
            return {"bytes": T * E * (size + 4) + 16 * T * k + 4 * E * (3 if c["bias"] else 2), "flops": 8 * T * E}
        # logits, indices and the gates' gradient in (and the scores'); the logits' gradient out
        return {"bytes": T * E * (2 * size + (4 if c["dscores"] else 0)) + 8 * T * k, "flops": 8 * T * E}
    if c["kind"] == "quant":         # in and out in the tensor's type, 17 bytes for 32 elements in between, out and in
        n = c["batch"] * c["rows"] * c["cols"]
        return {"bytes": 2 * n * size + 2 * n * 17 // 32, "flops": 4 * n}
    T, d, f, E, k = c["T"], c["d"], c["f"], c["E"], c["k"]
    busy = E * (1.0 - (1.0 - k / E) ** T)                # experts with a row, if all are equally likely
    return {"bytes": int(3 * busy * d * f * 17 / 32) + T * d * size * (3 if c["residual"] else 2) + 16 * T * k, "flops": 6 * T * k * d * f}


# ---- the definition in 64 bits, written apart from the plain form ---------------------------------------------


def _exact_pick(v, n):
    """The n largest of every row one after another, the first of equal ones; [rows, n] indices."""
    v, picked = v.clone(), []
    for _ in range(n):
        top = v.max(1, keepdim=True).values
        first = torch.where(v == top, torch.arange(v.shape[1], device=v.device), v.shape[1]).min(1, keepdim=True).values
        picked.append(first)
        v.scatter_(1, first, -math.inf)
    return torch.cat(picked, 1)


def _exact_scores(l, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    z = torch.exp(l - l.max(1, keepdim=True).values)
    return z / z.sum(1, keepdim=True)


def _exact_route(s):
    c = s["case"]
    G, per = c["groups"], c["E"] // c["groups"]
    p = _exact_scores(s["logits"].double(), c["score"])
    v = p if s["bias"] is None else p + s["bias"].double()
    if G > 1:
        in_group = v.reshape(-1, G, per)
        value = in_group.max(2).values
        if c["gscore"] == "top2" and per > 1:
            first = in_group.argmax(2, keepdim=True)
            value = value + in_group.scatter(2, first, -math.inf).max(2).values
        kept = _exact_pick(value, c["keep"])
        allowed = (torch.arange(c["E"], device=v.device) // per).reshape(1, -1, 1) == kept.unsqueeze(1)
        v = v.masked_fill(~allowed.any(2), -math.inf)
    idx = _exact_pick(v, c["k"])
    w = torch.stack([p[torch.arange(c["T"], device=p.device), idx[:, j]] for j in range(c["k"])], 1)
    gates = w * c["scale"]
    if c["renorm"]:
        gates = gates / (w.sum(1, keepdim=True) + TINY)
    # order the pairs by (expert, pair number)
    pair = torch.arange(idx.numel(), device=idx.device)
    perm = torch.argsort(idx.reshape(-1) * idx.numel() + pair)
    counts = torch.bincount(idx.reshape(-1), minlength=c["E"])
    offsets = torch.zeros(c["E"] + 1, dtype=torch.long, device=idx.device)
    offsets[1:] = torch.cumsum(counts, 0)
    inv = torch.argsort(perm).reshape(idx.shape)
    return dict(topk_idx=idx.int(), gates=gates, scores=p, counts=counts.int(), offsets=offsets.int(), perm=perm.int(), inv_pos=inv.int())


def _exact_route_bwd(s):
    """Differentiated by torch, in 64 bits."""
    c = s["case"]
    l = s["logits"].double().requires_grad_(True)
    p = _exact_scores(l, c["score"])
    w = torch.take_along_dim(p, s["topk_idx"].long(), 1)
    gates = c["scale"] * w / (w.sum(1, keepdim=True) + TINY) if c["renorm"] else c["scale"] * w
    loss = (gates * s["dgates"].double()).sum()
    if s["dscores"] is not None:
        loss = loss + (p * s["dscores"].double()).sum()
    return torch.autograd.grad(loss, l)[0]


def _power_of_two(exponent):
    """2^exponent in 64 bits, from its bits: library powers of two are an ulp off now and then."""
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _exact_round(x):
    """The nearest MXFP4 value of every element of [..., K], in 64 bits: of two equally near ones the one with an even code."""
    v = x.double().unflatten(-1, (-1, BLOCK))
    exponent = torch.frexp(v.abs().amax(-1, keepdim=True)).exponent - 3
    exponent = torch.where(v.abs().amax(-1, keepdim=True) > 0, exponent, -127).clamp(min=-127)
    unit = _power_of_two(exponent)
    a = (v / unit).abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return (torch.round(a / step) * step * unit * torch.sign(v)).flatten(-2)


def _exact_matrix(W, e):
    codes, scales = W
    n, K = codes.shape[1], codes.shape[2] * 2
    nibble = torch.stack([codes[e] % 16, codes[e] // 16], 2).reshape(n, K).long()
    mag, sign = nibble % 8, 1.0 - 2.0 * (nibble // 8)
    value = torch.where(mag < 2, mag * 0.5, (1.0 + 0.5 * (mag % 2)) * _power_of_two(mag // 2 - 1))
    return sign * value * _power_of_two(scales[e][:, :K // BLOCK].long() - 127).repeat_interleave(BLOCK, 1)


def _exact_layer(s):
    c, r = s["case"], s["routing"]
    x = _exact_round(s["x"])
    total = torch.zeros_like(x) if s["residual"] is None else s["residual"].double()
    for e in range(c["E"]):
        rows = (r.topk_idx == e).any(1).nonzero().squeeze(1)
        if rows.numel() == 0:
            continue
        gate = (r.gates[rows] * (r.topk_idx[rows] == e)).sum(1, keepdim=True).double()
        up, lin = torch.mm(x[rows], _exact_matrix(s["W1"], e).t()), torch.mm(x[rows], _exact_matrix(s["W3"], e).t())
        total.index_add_(0, rows, gate * torch.mm(_exact_round(up / (1.0 + torch.exp(-up)) * lin), _exact_matrix(s["W2"], e).t()))
    return total


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind == "route":
        return _exact_route(s)
    if kind == "route_bwd":
        return _exact_route_bwd(s)
    if kind == "quant":
        return _exact_round(s["x"]) if case["axis"] == 1 else _exact_round(s["x"].transpose(1, 2)).transpose(1, 2)
    return _exact_layer(s)
