"""The operators of a mixture-of-experts block around weight-only layers with group scales, as they are timed.

  product       `sq_w4a16_gemm_gs`: fp16 tokens times 4-bit weights with one scale (and offset) per group of input channels
  experts       `sq_w4a16_gemm_gs_grouped`: the same for every expert of a layer, on rows that the router sorted on the device
  route         `sq_route`: the experts of every token, their gates, the rows sorted by expert, per-expert counts, balance loss
  route_back    `sq_route_backward`: the gradient of gates and balance loss with respect to the router's logits
  combine       `sq_combine`: the experts' rows of a token, added up with their gates
  combine_back  `sq_combine_backward`: the gradient with respect to the experts' rows and the gates

`run` computes them in elementary torch operations in 32 bits, or, where `own` is true, through the library.  Weights are random
codes with scales that make them about N(0, 0.02); tokens are N(0, 1), which is what a rotation leaves of activations.
"""
import math

import torch

own = False

_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
_CODES = {"fp16": 0, "bf16": 1, "fp32": 2}          # SQ_F16, SQ_BF16, SQ_F32
_BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}
# Within eight channels, the nibble position that holds channel c (positions count from a 32-bit word's low end).
_POSITION = [0, 4, 1, 5, 2, 6, 3, 7]


def _product(rows, K, N, group, offset):
    return {"kind": "product", "rows": rows, "K": K, "N": N, "group": group, "offset": offset}


def _experts(tokens, experts, k, K, N, group, offset):
    return {"kind": "experts", "tokens": tokens, "experts": experts, "k": k, "K": K, "N": N, "group": group, "offset": offset}


def _route(kind, tokens, experts, k, dtype, renorm, padded):
    return {"kind": kind, "tokens": tokens, "experts": experts, "k": k, "dtype": dtype, "renorm": renorm, "padded": padded}


def _combine(kind, tokens, experts, k, N):
    return {"kind": kind, "tokens": tokens, "experts": experts, "k": k, "N": N}


def listed():
    return [
        # One user decoding: the up projection of a block, one token.
        dict(_product(1, 4096, 14336, 128, False), name="product_m1_up"),
        # A few users decoding through the long-row projection, small groups with offsets (an asymmetric checkpoint).
        dict(_product(5, 14336, 4096, 64, True), name="product_m5_down"),
        # A ragged decode batch through the largest projection that the benchmark has.
        dict(_product(50, 8192, 28672, 128, False), name="product_m50_70b"),
        # A prompt of odd length.
        dict(_product(777, 4096, 11008, 128, True), name="product_m777"),
        # Sixteen users decoding through a sparse block: two of eight experts each, four rows an expert on average.
        dict(_experts(16, 8, 2, 4096, 14336, 128, False), name="experts_t16_e8"),
        # Many small experts, eight of sixty-four for each of 61 users.
        dict(_experts(61, 64, 8, 2048, 1408, 32, True), name="experts_t61_e64"),
        # A long prompt through the sparse block: the largest call.
        dict(_experts(2048, 8, 2, 4096, 14336, 128, False), name="experts_t2048_e8"),
        # The router of a decoding step: the smallest call, latency is all there is.
        dict(_route("route", 16, 8, 2, "fp16", True, False), name="route_t16_e8"),
        # The router over a padded training batch with many experts.
        dict(_route("route", 16384, 256, 8, "bf16", False, True), name="route_t16384_e256"),
        # Tuning the router behind frozen 4-bit experts: its gradient.
        dict(_route("route_back", 8191, 64, 2, "fp32", True, True), name="route_back_t8191_e64"),
        # Back to token order, a prompt.
        dict(_combine("combine", 2048, 8, 2, 4096), name="combine_t2048"),
        # The gradient of that, with an odd number of tokens and more experts for each.
        dict(_combine("combine_back", 1021, 64, 6, 4096), name="combine_back_t1021"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above: from one token to a long prompt, any number of channels in steps of 2 (outputs) and 64
    (inputs), from two experts to 256."""
    kind = rng.choice(["product", "product", "experts", "experts", "route", "route_back", "combine", "combine_back"])
    if kind == "product":
        K = 64 * _log_int(rng, 8, 448)
        N = 2 * _log_int(rng, 128, min(14336, 100_000_000 // K))
        rows = _log_int(rng, 1, 2048) if rng.random() < 0.5 else rng.randint(1, 32)
        return _product(rows, K, N, rng.choice([32, 64, 128]), rng.random() < 0.5)
    if kind == "experts":
        E = rng.choice([2, 4, 8, 16, 32, 60, 64, 128])
        K = 64 * _log_int(rng, 8, 112)
        N = 2 * _log_int(rng, 128, max(128, min(7168, 200_000_000 // (K * E))))
        k = min(E, rng.choice([1, 2, 4, 6, 8]))
        tokens = _log_int(rng, 1, max(1, min(2048, 2048 * 16 // E, 240_000_000_000 // (k * K * N))))
        return _experts(tokens, E, k, K, N, rng.choice([32, 64, 128]), rng.random() < 0.5)
    if kind in ("route", "route_back"):
        E = rng.randint(2, 16) if rng.random() < 0.4 else _log_int(rng, 17, 256)
        k = rng.randint(1, min(E, 8))
        return _route(kind, _log_int(rng, 1, 16384), E, k, rng.choice(["fp16", "bf16", "fp32"] if kind == "route" else ["bf16", "fp32"]),
                      rng.random() < 0.5, rng.random() < 0.5)
    E = rng.choice([4, 8, 16, 60, 64])
    return _combine(kind, _log_int(rng, 1, 4096), E, min(E, rng.choice([1, 2, 4, 6, 8])), 8 * _log_int(rng, 32, 1024))


# -- inputs ---------------------------------------------------------------------------------------------------------------


def _random(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _weights(g, experts, N, K, group, offset):
    """Packed codes [experts, N, K/2], scales and offsets [experts, K/group, N]."""
    G = -(-K // group)
    Wq = torch.randint(0, 256, (experts, N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    sg = ((0.5 + torch.rand(experts, G, N, device="cuda", generator=g)) * 0.0043).half()
    bg = ((torch.rand(experts, G, N, device="cuda", generator=g) - 0.5) * 0.02).half() if offset else None
    return Wq, sg, bg


def _sorted_rows(g, T, E, k):
    """A routing of T tokens: (row_token [T k], offsets [E + 1], pos [T, k]).  Some experts are liked more than others."""
    logits = torch.randn(T, E, device="cuda", generator=g) + 0.7 * torch.randn(E, device="cuda", generator=g)
    ids = logits.topk(k, dim=1).indices.reshape(-1)
    order = torch.sort(ids, stable=True).indices
    pos = torch.empty(T * k, dtype=torch.int32, device="cuda")
    pos[order] = torch.arange(T * k, dtype=torch.int32, device="cuda")
    counts = torch.bincount(ids, minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    return (order // k).int(), offsets, pos.reshape(T, k)


def prepare(case, seed):
    g = _random(seed)
    c = dict(case)
    kind = c["kind"]
    if kind == "product":
        c["X"] = torch.randn(c["rows"], c["K"], device="cuda", generator=g).half()
        Wq, sg, bg = _weights(g, 1, c["N"], c["K"], c["group"], c["offset"])
        c["Wq"], c["sg"], c["bg"] = Wq[0], sg[0], None if bg is None else bg[0]
        c["Y"] = torch.zeros(c["rows"], c["N"], dtype=torch.float16, device="cuda")
    elif kind == "experts":
        T, E, k = c["tokens"], c["experts"], c["k"]
        c["X"] = torch.randn(T, c["K"], device="cuda", generator=g).half()
        c["Wq"], c["sg"], c["bg"] = _weights(g, E, c["N"], c["K"], c["group"], c["offset"])
        c["row_token"], c["offsets"], _ = _sorted_rows(g, T, E, k)
        c["Y"] = torch.zeros(T * k, c["N"], dtype=torch.float16, device="cuda")
        c["workspace"] = torch.empty(T * k * c["K"] * 2 + 256, dtype=torch.uint8, device="cuda")
    elif kind in ("route", "route_back"):
        T, E, k = c["tokens"], c["experts"], c["k"]
        like = 0.7 * torch.randn(E, device="cuda", generator=g)
        c["logits"] = (1.5 * torch.randn(T, E, device="cuda", generator=g) + like).to(_DTYPES[c["dtype"]])
        c["mask"] = None
        if c["padded"]:                       # the last tokens of the batch's four sequences are padding
            length = -(-T // 4)
            lens = torch.randint(max(1, length // 2), length + 1, (4,), device="cuda", generator=g)
            t = torch.arange(T, device="cuda")
            c["mask"] = (t % length < lens[t // length]).to(torch.uint8)
        if kind == "route":
            c["ids"] = torch.zeros(T, k, dtype=torch.int32, device="cuda")
            c["gates"] = torch.zeros(T, k, device="cuda")
            c["counts"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
            c["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
            c["row_token"] = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
            c["pos"] = torch.zeros(T, k, dtype=torch.int32, device="cuda")
            c["loss"] = torch.zeros(1, device="cuda")
            c["workspace"] = torch.empty(4 << 20, dtype=torch.uint8, device="cuda")
        else:
            r = _route_plain(c)
            c["ids"], c["gates"], c["counts"] = r["ids"], r["gates"], r["counts"]
            c["dgates"] = 0.01 * torch.randn(T, k, device="cuda", generator=g)
            c["dloss"] = 0.5 + torch.rand(1, device="cuda", generator=g)
            c["dlogits"] = torch.zeros_like(c["logits"])
    else:
        T, E, k, N = c["tokens"], c["experts"], c["k"], c["N"]
        _, _, c["pos"] = _sorted_rows(g, T, E, k)
        c["Y"] = torch.randn(T * k, N, device="cuda", generator=g).half()
        c["gates"] = torch.softmax(torch.randn(T, k, device="cuda", generator=g), 1)
        if kind == "combine":
            c["out"] = torch.zeros(T, N, dtype=torch.float16, device="cuda")
        else:
            c["dout"] = torch.randn(T, N, device="cuda", generator=g).half()
            c["dY"] = torch.zeros(T * k, N, dtype=torch.float16, device="cuda")
            c["dgates"] = torch.zeros(T, k, device="cuda")
    return c


# -- plain forms ----------------------------------------------------------------------------------------------------------


def _dequantised(Wq, sg, bg, group):
    """The weights [..., N, K] in 32 bits."""
    nibbles = torch.stack([Wq & 15, Wq >> 4], -1).reshape(*Wq.shape[:-1], -1, 8)[..., _POSITION]
    codes = ((nibbles ^ 8).to(torch.float32) - 8).flatten(-2)
    group_of = torch.arange(codes.shape[-1], device=codes.device) // group
    w = codes * sg.float()[..., group_of, :].transpose(-1, -2)
    return w if bg is None else w + bg.float()[..., group_of, :].transpose(-1, -2)


def _product_plain(s):
    return (s["X"].float() @ _dequantised(s["Wq"], s["sg"], s["bg"], s["group"]).t()).half()


def _experts_plain(s):
    """Every token times every expert, of which the rows that were asked for are kept: no size depends on the routing."""
    w = _dequantised(s["Wq"], s["sg"], s["bg"], s["group"])
    every = s["X"].float() @ w.transpose(1, 2)                       # [experts, tokens, N]
    rows = torch.arange(s["row_token"].shape[0], device=w.device)
    expert = torch.searchsorted(s["offsets"][1:].long(), rows, right=True)
    return every[expert, s["row_token"].long()].half()


def _live(s):
    T = s["logits"].shape[0]
    return torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0


def _softmax(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _route_plain(s):
    T, E = s["logits"].shape
    k, live = s["k"], _live(s)
    x = s["logits"].float()
    best = torch.sort(x, dim=1, descending=True, stable=True)        # equal logits: the lower index first
    p = _softmax(x)
    sel = best.values[:, :k]
    gates = _softmax(sel) if s["renorm"] else p.gather(1, best.indices[:, :k])
    gates = torch.where(live[:, None], gates, torch.zeros_like(gates))
    ids = torch.where(live[:, None], best.indices[:, :k], -torch.ones_like(best.indices[:, :k]))
    flat = torch.where(ids >= 0, ids, torch.full_like(ids, E)).reshape(-1)                      # padding behind all experts
    slots = torch.arange(T * k, device="cuda")
    counts = torch.zeros(E + 1, dtype=torch.long, device="cuda").scatter_add(0, flat, torch.ones_like(flat))[:E]
    ends = counts.cumsum(0)
    order = torch.sort(flat, stable=True).indices                    # rows of an expert in the tokens' order
    pos = torch.empty_like(flat).scatter(0, order, slots)
    pos = torch.where(flat < E, pos, -torch.ones_like(pos))
    row_token = torch.where(slots < ends[-1], order // k, -torch.ones_like(order))
    first = torch.cat([ends.new_zeros(1), ends])
    n = live.sum()
    share = counts.double() / (k * n).clamp(min=1)
    mean = (p.double() * live[:, None]).sum(0) / n.clamp(min=1)
    return {"ids": ids.int(), "gates": gates, "counts": torch.cat([counts, n.reshape(1)]).int(), "offsets": first.int(),
            "row_token": row_token.int(), "pos": pos.int().reshape(T, k),
            "loss": (E * (share * mean).sum()).float().reshape(1)}


def _route_back_plain(s):
    E, k, live = s["experts"], s["k"], _live(s)
    p = _softmax(s["logits"].float())
    n = s["counts"][E].double().clamp(min=1)
    dp = (s["dloss"].double() * E * s["counts"][:E].double() / (k * n) / n).float().expand_as(p)
    ids = s["ids"].long().clamp(min=0)
    dg = torch.where(s["ids"] >= 0, s["dgates"], torch.zeros_like(s["dgates"]))
    if s["renorm"]:
        dx = p * (dp - (p * dp).sum(1, keepdim=True))
        dsel = s["gates"] * (dg - (s["gates"] * dg).sum(1, keepdim=True))
        dx = dx.scatter_add(1, ids, dsel)
    else:
        dp = dp.scatter_add(1, ids, dg)
        dx = p * (dp - (p * dp).sum(1, keepdim=True))
    return torch.where(live[:, None], dx, torch.zeros_like(dx)).to(s["logits"].dtype)


def _combine_plain(s):
    return (s["Y"].float()[s["pos"].long()] * s["gates"][..., None]).sum(1).half()


def _combine_back_plain(s):
    dout, pos = s["dout"].float(), s["pos"].long()
    dY = torch.zeros_like(s["Y"])
    dY[pos.reshape(-1)] = (dout[:, None] * s["gates"][..., None]).half().flatten(0, 1)
    return {"dY": dY, "dgates": (s["Y"].float()[pos] * dout[:, None]).sum(-1)}


_PLAIN = {"product": _product_plain, "experts": _experts_plain, "route": _route_plain, "route_back": _route_back_plain,
          "combine": _combine_plain, "combine_back": _combine_back_plain}


# -- the library ----------------------------------------------------------------------------------------------------------


def _product_own(s):
    from paper_2511_22316_b200 import binding as sq
    sq.sq_w4a16_gemm_gs(s["X"], s["Wq"], s["sg"], s["bg"], s["rows"], s["N"], s["K"], s["group"], s["Y"])
    return s["Y"]


def _experts_own(s):
    from paper_2511_22316_b200 import binding as sq
    ws = s["workspace"]
    sq.sq_w4a16_gemm_gs_grouped(s["X"], s["tokens"], s["row_token"], s["offsets"], s["experts"], s["Wq"], s["sg"], s["bg"],
                                s["tokens"] * s["k"], s["N"], s["K"], s["group"], ws, ws.numel(), s["Y"])
    return s["Y"]


def _route_own(s):
    from paper_2511_22316_b200 import binding as sq
    ws, E = s["workspace"], s["experts"]
    sq.sq_route(s["logits"], _CODES[s["dtype"]], s["tokens"], E, E, s["k"], sq.SQ_ROUTE_RENORM if s["renorm"] else 0, s["mask"],
                s["ids"], s["gates"], s["counts"], s["offsets"], s["row_token"], s["pos"], s["loss"], ws, ws.numel())
    return {f: s[f] for f in ("ids", "gates", "counts", "offsets", "row_token", "pos", "loss")}


def _route_back_own(s):
    from paper_2511_22316_b200 import binding as sq
    E = s["experts"]
    sq.sq_route_backward(s["logits"], _CODES[s["dtype"]], s["tokens"], E, E, s["k"], sq.SQ_ROUTE_RENORM if s["renorm"] else 0, s["mask"],
                         s["ids"], s["gates"], s["counts"], s["dgates"], s["dloss"], s["dlogits"], E)
    return s["dlogits"]


def _combine_own(s):
    from paper_2511_22316_b200 import binding as sq
    sq.sq_combine(s["Y"], s["Y"].shape[0], s["pos"], s["gates"], s["tokens"], s["k"], s["N"], s["out"])
    return s["out"]


def _combine_back_own(s):
    from paper_2511_22316_b200 import binding as sq
    sq.sq_combine_backward(s["dout"], s["Y"], s["Y"].shape[0], s["pos"], s["gates"], s["tokens"], s["k"], s["N"], s["dY"], s["dgates"])
    return {"dY": s["dY"], "dgates": s["dgates"]}


_OWN = {"product": _product_own, "experts": _experts_own, "route": _route_own, "route_back": _route_back_own,
        "combine": _combine_own, "combine_back": _combine_back_own}


def run(state):
    if own:
        return _OWN[state["kind"]](state)
    return _PLAIN[state["kind"]](state)


# -- what a pass cannot do without ----------------------------------------------------------------------------------------


def work(case):
    c = case
    if c["kind"] in ("product", "experts"):
        K, N = c["K"], c["N"]
        weights = N * K / 2 + 2 * (-(-K // c["group"])) * N * (2 if c["offset"] else 1)
        if c["kind"] == "product":
            return {"bytes": weights + 2 * c["rows"] * (K + N), "flops": 2.0 * c["rows"] * K * N}
        T, E, k = c["tokens"], c["experts"], c["k"]
        active = E * (1.0 - (1.0 - k / E) ** T)                      # experts that any token takes, if all were liked alike
        return {"bytes": active * weights + 2 * T * K + T * k * (2 * N + 4), "flops": 2.0 * T * k * K * N}
    T, E, k = c["tokens"], c["experts"], c["k"]
    if c["kind"] == "route":
        return {"bytes": T * E * _BYTES[c["dtype"]] + T * k * 16 + (T if c["padded"] else 0) + 8 * (E + 1) + 4, "flops": 3.0 * T * E}
    if c["kind"] == "route_back":
        return {"bytes": 2 * T * E * _BYTES[c["dtype"]] + T * k * 12 + (T if c["padded"] else 0) + 4 * (E + 2), "flops": 6.0 * T * E}
    N = c["N"]
    if c["kind"] == "combine":
        return {"bytes": 2 * T * (k + 1) * N + 8 * T * k, "flops": 2.0 * T * k * N}
    return {"bytes": 2 * T * (2 * k + 1) * N + 12 * T * k, "flops": 3.0 * T * k * N}


# -- the definitions in 64 bits -------------------------------------------------------------------------------------------


def exact(case, seed):
    def weight(Wq, sg, bg, group):
        """Expert by expert: [N, K] in 64 bits, from the words' bits."""
        N, half = Wq.shape
        words = Wq.view(torch.int32).long() & 0xFFFFFFFF                 # [N, K / 8], little-endian
        w = torch.empty(N, 2 * half, dtype=torch.float64, device=Wq.device)
        for position, channel in enumerate((0, 2, 4, 6, 1, 3, 5, 7)):
            nibble = (words >> (4 * position)) & 15
            w[:, channel::8] = (nibble - 16 * (nibble >= 8).long()).double()
        for i in range(sg.shape[0]):
            part = w[:, i * group:(i + 1) * group]
            part *= sg[i].double()[:, None]
            if bg is not None:
                part += bg[i].double()[:, None]
        return w

    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "product":
        return s["X"].double() @ weight(s["Wq"], s["sg"], s["bg"], s["group"]).T
    if kind == "experts":
        Y = torch.zeros(s["Y"].shape, dtype=torch.float64, device="cuda")
        ends = s["offsets"].tolist()
        for e in range(s["experts"]):
            if ends[e + 1] > ends[e]:
                W = weight(s["Wq"][e], s["sg"][e], None if s["bg"] is None else s["bg"][e], s["group"])
                Y[ends[e]:ends[e + 1]] = s["X"][s["row_token"][ends[e]:ends[e + 1]].long()].double() @ W.T
        return Y
    if kind in ("route", "route_back"):
        x = s["logits"].double()
        T, E = x.shape
        k = s["k"]
        alive = torch.ones(T, device="cuda", dtype=torch.float64) if s["mask"] is None else s["mask"].double()
        p = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
        taken = torch.zeros_like(x)                                  # 1 where an expert is the token's
        left, gates = x.clone(), []
        for _ in range(k):
            best = left.max(1, keepdim=True).values
            first = (left == best).double().cumsum(1).eq(1) & (left == best)
            taken += first.double()
            gates.append(p[first])
            left[first] = -math.inf
        gates = torch.stack(gates, 1)
        if s["renorm"]:
            gates = gates / gates.sum(1, keepdim=True)
        taken *= alive[:, None]
        n = max(1.0, float(alive.sum()))
        share = taken.sum(0) / (k * n)
        if kind == "route":
            loss = E * (share * (p * alive[:, None]).sum(0) / n).sum()
            return {"ids": None, "gates": gates * alive[:, None], "counts": None, "offsets": None, "row_token": None, "pos": None,
                    "loss": loss.reshape(1)}
        x.requires_grad_(True)
        with torch.enable_grad():
            p = torch.softmax(x, 1)
            q = p.gather(1, s["ids"].long().clamp(min=0))
            if s["renorm"]:
                q = q / q.sum(1, keepdim=True)
            loss = E * (share * (p * alive[:, None]).sum(0) / n).sum()
            total = loss * s["dloss"].double().sum() + (q * s["dgates"].double() * alive[:, None]).sum()
        return torch.autograd.grad(total, x)[0]
    pos, gates, Y = s["pos"].long(), s["gates"].double(), s["Y"].double()
    if kind == "combine":
        return torch.einsum("tkn,tk->tn", Y[pos], gates)
    dout = s["dout"].double()
    dY = torch.zeros_like(Y).index_add_(0, pos.reshape(-1), torch.einsum("tn,tk->tkn", dout, gates).flatten(0, 1))
    return {"dY": dY, "dgates": torch.einsum("tkn,tn->tk", Y[pos], dout)}
