"""A block's MLP of experts, as timed passes: the router that sends each token to a few of many experts, the products with the
experts' quantized weights, and the weighted way back to one row a token.

A case is one pass through one operator.

kinds
  route    router logits -> the chosen experts and their weights, and the rows (token, choice) sorted by expert
  gemm     one linear layer of all experts: rows sorted by expert, ragged groups, each times its own expert's packed weights
  combine  the weighted sum of each token's rows, added to what the block has so far

tokens go to `top` of `experts` each.
route: `bits` 16 or 32 of the logits; `sigmoid`: scores are sigmoids with a bias that steers the choice, and some tokens are padding (every
expert masked), else a softmax.
gemm: p-bit weights [experts, N, K], q-bit activation codes of K; `gather`: the rows are the tokens' own (up projections), else they
have been through the experts already (down projections: one row a choice).
combine: rows of N.
"""
import torch

own = False


def _route(tokens, experts, top, bits=16, sigmoid=False, name=None):
    c = {"kind": "route", "tokens": tokens, "experts": experts, "top": top, "bits": bits, "sigmoid": sigmoid}
    return c if name is None else {"name": name, **c}


def _gemm(p, q, tokens, experts, top, N, K, gather, name=None):
    c = {"kind": "gemm", "p": p, "q": q, "tokens": tokens, "experts": experts, "top": top, "N": N, "K": K, "gather": gather}
    return c if name is None else {"name": name, **c}


def _combine(tokens, top, N, name=None):
    c = {"kind": "combine", "tokens": tokens, "top": top, "N": N}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one token of one request: all latency
        _route(1, 8, 2, name="route_m1_8"),
        # a decoding step of 64 requests, many small experts, logits in binary32
        _route(64, 128, 8, 32, name="route_m64_128"),
        # prompts of odd lengths in a padded batch, sigmoid scores with a bias that balances the load
        _route(4099, 64, 6, 32, True, name="route_padded_4099_64"),
        # a large batch of prompts
        _route(32768, 128, 8, name="route_prompts_32k_128"),
        # one token, up projection of two of eight experts of a 7B model's MLP size
        _gemm(4, 8, 1, 8, 2, 11008, 4096, True, name="gemm_w4a8_m1_8x11008"),
        # a decoding step of 32 requests over many small experts
        _gemm(4, 8, 32, 64, 8, 1408, 2048, True, name="gemm_w4a8_m32_64x1408"),
        # a decoding step of 32 requests over eight large experts, down projection, narrow weights
        _gemm(2, 8, 32, 8, 2, 4096, 11008, False, name="gemm_w2a8_m32_8x4096_down"),
        # a chunk of 333 tokens, six bits
        _gemm(6, 6, 333, 8, 2, 11008, 4096, True, name="gemm_w6a6_m333_8x11008"),
        # prompts of 2048 tokens, down projection of many small experts, eight bits
        _gemm(8, 8, 2048, 64, 6, 2048, 1408, False, name="gemm_w8a8_m2048_64x2048_down"),
        # prompts of 2048 tokens, up projection of eight large experts: the largest
        _gemm(4, 4, 2048, 8, 2, 11008, 4096, True, name="gemm_w4a4_m2048_8x11008"),
        # one token's two rows: all latency
        _combine(1, 2, 4096, name="combine_m1"),
        # prompts of 4099 tokens, eight rows each
        _combine(4099, 8, 5120, name="combine_4099x8"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(lo * (hi / lo) ** rng.random()))
    return max(lo, v // step * step)


def draw(rng):
    while True:
        kind = rng.choice(["route", "gemm", "gemm", "gemm", "combine"])
        experts = rng.choice([4, 8, 8, 16, 32, 60, 64, 128, 160, 256])
        top = min(rng.choice([1, 2, 2, 4, 6, 8]), experts)
        if kind == "route":
            c = _route(_log(rng, 1, 32768), experts, top, rng.choice([16, 32]), rng.random() < 0.4)
            if work(c)["bytes"] <= work(_route(32768, 128, 8))["bytes"]:
                return c
        elif kind == "combine":
            c = _combine(_log(rng, 1, 8192), top, _log(rng, 256, 8192))
            if work(c)["bytes"] <= work(_combine(4099, 8, 5120))["bytes"]:
                return c
        else:
            odd = rng.random() < 0.25   # sizes that are no multiple of anything
            c = _gemm(rng.choice([1, 2, 3, 4, 4, 4, 5, 6, 7, 8]), rng.choice([1, 2, 4, 4, 6, 8, 8, 8]), _log(rng, 1, 2048), experts, top,
                      _log(rng, 256, 13824, 1 if odd else 64), _log(rng, 256, 13824, 1 if odd else 64), rng.random() < 0.5)
            if c["K"] * (2 ** c["p"] - 1) * (2 ** c["q"] - 1) < 2**31 and experts * c["N"] * c["K"] < 4e8 and work(c)["flops"] < 3.7e11 and c["tokens"] * top < 16384:
                return c


# ---- inputs -------------------------------------------------------------------------------------
def _uniform(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _codes(gen, bits, *shape):
    return torch.randint(0, 1 << bits, shape, generator=gen, device="cuda", dtype=torch.uint8)


def _logits(gen, tokens, experts):
    """A router's logits: some experts are more popular than others."""
    return torch.randn((tokens, experts), generator=gen, device="cuda") * 1.5 + torch.randn(experts, generator=gen, device="cuda") * 0.5


def _sorted_by_expert(ids, experts):
    """Rows (token, choice) sorted by expert, those of one expert in their own order: first row of each expert, the row of each place."""
    flat = ids.flatten().long()
    starts = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    starts[1:] = (flat[:, None] == torch.arange(experts, device="cuda")).sum(0).cumsum(0)
    return starts, torch.sort(flat, stable=True)[1].to(torch.int32)


def _inputs(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    T, top = c["tokens"], c["top"]
    if c["kind"] == "combine":
        rows = T * top
        return {"case": c, "y": torch.randn((rows, c["N"]), generator=gen, device="cuda").to(torch.float16),
                "places": torch.randperm(rows, generator=gen, device="cuda").to(torch.int32).view(T, top),
                "weights": torch.softmax(torch.randn((T, top), generator=gen, device="cuda"), 1),
                "add": torch.randn((T, c["N"]), generator=gen, device="cuda").to(torch.float16)}
    E = c["experts"]
    logits = _logits(gen, T, E)
    if c["kind"] == "route":
        s = {"case": c, "bias": None, "scale": 1.0}
        if c["sigmoid"]:
            if T > 1:
                logits[torch.rand(T, generator=gen, device="cuda") < 0.06] = float("-inf")
            s["bias"], s["scale"] = _uniform(gen, (E,), -0.2, 0.2), 2.5
        s["logits"] = logits.to(torch.float16 if c["bits"] == 16 else torch.float32)
        return s
    p, q, N, K = c["p"], c["q"], c["N"], c["K"]
    starts, order = _sorted_by_expert(torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :top], E)
    M = T if c["gather"] else T * top
    return {"case": c, "starts": starts, "order": order,
            "a": (_codes(gen, q, M, K), _uniform(gen, (M,), 0.5, 1.0) * (4.0 / 2**q), torch.randint(0, 1 << q, (M,), generator=gen, device="cuda", dtype=torch.int32)),
            "w": (_codes(gen, p, E, N, K), _uniform(gen, (E, N), 0.5, 1.0) * (2.0 / (K ** 0.5 * 2**p)),
                  torch.randint(0, 1 << p, (E, N), generator=gen, device="cuda", dtype=torch.int32))}


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] == "gemm":
        from paper_2408_08554_amd import binding as abq
        s["w"] = abq.abq_pack_experts(case["p"], *s["w"])
    return s


# ---- one pass -----------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"route": _route_plain, "gemm": _gemm_plain, "combine": _combine_plain}[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2408_08554_amd import binding as abq
    c = s["case"]
    if c["kind"] == "route":
        return abq.abq_moe_route(s["logits"], c["top"], bias=s["bias"], sigmoid=c["sigmoid"], scale=s["scale"])
    if c["kind"] == "combine":
        return abq.abq_moe_combine(s["y"], s["places"], s["weights"], add=s["add"])
    if c["gather"]:
        return abq.abq_moe_gemm(c["p"], c["q"], c["N"], *s["a"], s["w"], s["starts"], order=s["order"], top=c["top"])
    return abq.abq_moe_gemm(c["p"], c["q"], c["N"], *s["a"], s["w"], s["starts"])


def _route_plain(s):
    c, x = s["case"], s["logits"].float()
    E, top = c["experts"], c["top"]
    there = x > float("-inf")
    key = x.double()   # (what decides a choice is compared in 64 bits)
    if c["sigmoid"]:
        key = torch.where(there, 1 / (1 + torch.exp(-key)) + s["bias"].double(), float("-inf"))
    ids = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :top]
    chosen = there.gather(1, ids)
    if c["sigmoid"]:
        w = 1 / (1 + torch.exp(-x.gather(1, ids)))
    else:
        w = torch.exp(x.gather(1, ids) - x.gather(1, ids).amax(1, keepdim=True))
    w = torch.where(chosen, w / w.sum(1, keepdim=True) * s["scale"], 0.0)
    ids = torch.where(chosen, ids, -1)
    # rows sorted by expert; choices that name none come last and have no place
    flat = torch.where(ids < 0, E, ids).flatten()
    sorted_, order = torch.sort(flat, stable=True)
    starts = torch.searchsorted(sorted_, torch.arange(E + 1, device="cuda"))
    places = torch.empty_like(order)
    places[order] = torch.arange(len(order), device="cuda")
    order = torch.where(sorted_ < E, order, -1)
    places = torch.where(flat < E, places, -1)
    return ids.to(torch.int32), w, starts.to(torch.int32), order.to(torch.int32), places.to(torch.int32).view(-1, top)


def _gemm_plain(s):
    c = s["case"]
    codes, scale, zero = s["a"]
    a = codes.float() - zero[:, None]
    if c["gather"]:
        token = s["order"].long() // c["top"]
        a, scale = a[token], scale[token]
    y = torch.empty((len(a), c["N"]), dtype=torch.float16, device="cuda")
    starts = s["starts"].tolist()
    for e, (w, w_scale, w_zero) in enumerate(zip(*s["w"])):
        rows = slice(starts[e], starts[e + 1])
        if starts[e] < starts[e + 1]:
            y[rows] = (a[rows] @ (w.float() - w_zero[:, None]).T * scale[rows, None] * w_scale).to(torch.float16)
    return y


def _combine_plain(s):
    y = s["y"].float()[s["places"].long()]
    return ((y * s["weights"][..., None]).sum(1) + s["add"].float()).to(torch.float16)


# ---- floor --------------------------------------------------------------------------------------
def work(case):
    c = case
    T, top = c["tokens"], c["top"]
    if c["kind"] == "combine":
        return {"bytes": 2.0 * T * c["N"] * (top + 2) + 8.0 * T * top, "flops": 2.0 * T * top * c["N"]}
    E = c["experts"]
    if c["kind"] == "route":
        return {"bytes": T * (E * c["bits"] / 8 + 16.0 * top) + 4.0 * (E + 1), "flops": 1.0 * T * E}
    N, K, rows = c["N"], c["K"], T * top
    read = E * (1 - (1 - top / E) ** T)   # experts that have rows: their expected number, all being alike
    return {"bytes": read * (c["p"] * N * K / 8 + 12.0 * N) + (T if c["gather"] else rows) * (K + 8.0) + 2.0 * rows * N + 4.0 * (rows * c["gather"] + E + 1), "flops": 2.0 * rows * N * K}


# ---- the definition, in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"route": _route_exact, "gemm": _gemm_exact, "combine": _combine_exact}[case["kind"]](s)


def _route_exact(s):
    c = s["case"]
    E, top = c["experts"], c["top"]
    x = s["logits"].double()
    there = ~torch.isinf(x)
    score = torch.sigmoid(x) if c["sigmoid"] else torch.softmax(x, 1)
    key = score + s["bias"].double() if c["sigmoid"] else x
    ids, weights = [], []
    left = there.clone()
    for _ in range(top):   # the largest that is left, the first of equals, one after the other
        k = torch.where(left, key, float("-inf"))
        best = (k == k.amax(1, keepdim=True)).to(torch.uint8).argmax(1, keepdim=True)
        some = left.any(1, keepdim=True)
        ids.append(torch.where(some, best, -1))
        weights.append(torch.where(some, score.gather(1, best), 0.0))
        left.scatter_(1, best, False)
    ids, weights = torch.cat(ids, 1), torch.cat(weights, 1)
    weights = weights * (s["scale"] / weights.sum(1, keepdim=True).clamp(min=1e-300))
    flat = ids.flatten()
    order = torch.cat([(flat == e).nonzero()[:, 0] for e in range(E)])
    places = torch.full_like(flat, -1)
    places[order] = torch.arange(len(order), device="cuda")
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.stack([(flat == e).sum() for e in range(E)]).cumsum(0)])
    order = torch.cat([order, torch.full((len(flat) - len(order),), -1, device="cuda")])
    return ids.to(torch.int32), weights, starts.to(torch.int32), order.to(torch.int32), places.view(-1, top).to(torch.int32)


def _gemm_exact(s):
    c = s["case"]
    (a, a_scale, a_zero), (w, w_scale, w_zero) = s["a"], s["w"]
    y = torch.empty((len(s["order"]), c["N"]), dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        at = torch.arange(int(s["starts"][e]), int(s["starts"][e + 1]), device="cuda")
        if len(at):
            row = s["order"][at].long() // c["top"] if c["gather"] else at
            x = (a[row].double() - a_zero[row].double().unsqueeze(1)) * a_scale[row].double().unsqueeze(1)
            y[at] = x @ ((w[e].double() - w_zero[e].double().unsqueeze(1)) * w_scale[e].double().unsqueeze(1)).T.contiguous()
    return y


def _combine_exact(s):
    out = s["add"].double()
    for j in range(s["case"]["top"]):
        out += s["weights"][:, j].double().unsqueeze(1) * s["y"][s["places"][:, j].long()].double()
    return out
