"""The attention half of a decoder block served to many requests, as timed passes: what happens between the quantized
q / k / v projections and the output projection, and the requests' own adapters beside those projections.

A case is one pass through one operator, on binary16 tensors as the projections write them.

kinds
  append  new tokens' keys and values, rotated to their positions, go into a paged cache; the queries are rotated too
  attn    the new tokens' queries over everything the paged cache holds of their sequences (causal, grouped heads)
  lora    low-rank adapters, one of many for each row, added to a shared projection's output

append and attn: `seqs` sequences with up to `new` new tokens each (`mixed`: only the first, one token for the others)
after up to `past` cached ones; hq / hkv query and key heads of `dim`; pages of `page` tokens; `bits` 16 (binary16) or 8
(codes with a scale and a zero-point per vector).
lora: x [M,K], y [M,N]; `adapters` pairs of matrices of rank `rank`; rows of one adapter adjacent (`runs`) or not.
"""
import torch

own = False

_PHI = 2654435761   # spreads lengths over a range, the same ones for a case whatever the seed


def _paged(kind, bits, seqs, new, past, hq, hkv, dim, page, mixed=False, name=None):
    c = {"kind": kind, "bits": bits, "seqs": seqs, "new": new, "past": past, "hq": hq, "hkv": hkv, "dim": dim, "page": page, "mixed": mixed}
    return c if name is None else {"name": name, **c}


def _adapted(M, N, K, rank, adapters, runs, name=None):
    c = {"kind": "lora", "M": M, "N": N, "K": K, "rank": rank, "adapters": adapters, "runs": runs}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one token of one request of a 7B model: all latency
        _paged("append", 16, 1, 1, 512, 32, 32, 128, 16, name="append_m1"),
        # a decoding step of 64 requests with the cache in 8 bits, and the new vectors read back
        _paged("append", 8, 64, 1, 1024, 32, 8, 128, 16, name="append_codes_m64"),
        # prompts of a 13B model, 1024..2048 tokens each, into empty caches
        _paged("append", 16, 2, 2048, 0, 40, 40, 128, 64, name="append_prompts_2x2048"),
        # one token of one request over a short context: all latency
        _paged("attn", 16, 1, 1, 512, 32, 32, 128, 16, name="attn_m1_ctx513"),
        # a decoding step of 32 requests of a 7B model with 1..2 thousand tokens each
        _paged("attn", 16, 32, 1, 2047, 32, 32, 128, 16, name="attn_decode_32x2k"),
        # a decoding step over long contexts, grouped heads, cache in 8 bits
        _paged("attn", 8, 4, 1, 32767, 32, 8, 128, 64, name="attn_decode_codes_4x32k"),
        # a prompt's odd chunk beside eight decoding requests
        _paged("attn", 16, 9, 333, 1000, 32, 8, 128, 16, mixed=True, name="attn_mixed_333_and_8"),
        # a whole prompt of a 7B model
        _paged("attn", 16, 1, 2048, 0, 32, 32, 128, 16, name="attn_prompt_2048"),
        # a chunk of 1024 tokens over a long prompt's earlier ones, grouped heads, cache in 8 bits: the largest
        _paged("attn", 8, 1, 1024, 15360, 32, 8, 128, 64, name="attn_chunk_codes_1k_16k"),
        # one token's adapter beside an attention projection of a 7B model
        _adapted(1, 4096, 4096, 16, 8, False, name="lora_m1_r16"),
        # 64 decoding requests with 32 adapters in any order, up projection of a 7B model
        _adapted(64, 11008, 4096, 16, 32, False, name="lora_m64_r16"),
        # prompts of four requests, one adapter each, up projection of a 13B model
        _adapted(2048, 13824, 5120, 64, 4, True, name="lora_prompts_2048_r64"),
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(lo * (hi / lo) ** rng.random()))
    return max(lo, v // step * step)


def draw(rng):
    while True:
        kind = rng.choice(["append", "attn", "attn", "attn", "lora"])
        if kind == "lora":
            c = _adapted(_log(rng, 1, 2048), _log(rng, 256, 13824, 8), _log(rng, 256, 13824, 8), rng.choice([8, 16, 16, 24, 32, 64, 128]), _log(rng, 1, 48), rng.random() < 0.5)
            if 3 * c["adapters"] * c["rank"] * c["M"] <= 2048 * 2048 and work(c)["bytes"] < 180e6:
                return c
            continue
        hq, hkv = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (12, 12), (28, 4), (16, 1)])
        dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
        new = _log(rng, 2, 2048) if rng.random() < 0.5 else 1
        c = _paged(kind, rng.choice([16, 16, 8]), _log(rng, 1, 48), new, rng.randint(0, 3) if rng.random() < 0.15 else _log(rng, 4, 32768), hq, hkv, dim,
                   rng.choice([16, 16, 32, 64, 128]), new > 1 and rng.random() < 0.4)
        w = work(c)
        longest = c["new"] + c["past"]
        padded = c["seqs"] * longest * max(4 * c["hkv"] * dim, c["hq"] * c["new"])
        if padded < 1 << 30 and w["bytes"] < 8e8 and w["flops"] < 2.4e11 and sum(_news(c)) <= 4096:
            return c


# ---- lengths ------------------------------------------------------------------------------------
def _news(c):
    """New tokens of each sequence: `new` for the first; for the others as many to half as many, or one."""
    return [c["new"] if s == 0 else 1 if c["mixed"] else c["new"] - (s * _PHI % 2**32 * (c["new"] // 2) >> 32) for s in range(c["seqs"])]


def _lens(c):
    """Tokens of each sequence, the new ones among them."""
    return [n + c["past"] - (s * _PHI % 2**32 * (c["past"] // 2) >> 32) for s, n in enumerate(_news(c))]


# ---- inputs -------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)


def _quantize(x):
    """Codes 0..255, scale and zero-point of each vector (last axis) of binary16 values."""
    x = x.float()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    scale = torch.where(hi > lo, (hi - lo) / 255.0, torch.ones_like(hi))
    zero = torch.round(-lo / scale).clamp_(0, 255)
    codes = (torch.round(x / scale[..., None]) + zero[..., None]).clamp_(0, 255)
    return codes.to(torch.uint8), scale, zero.to(torch.uint8)


def _cache(gen, c, pages):
    """A cache of [pages, heads, page, dim] whose every vector holds something: (k, v) or, in 8 bits, (k, v, k_scale, k_zero, v_scale, v_zero)."""
    k, v = _normal(gen, pages, c["hkv"], c["page"], c["dim"]), _normal(gen, pages, c["hkv"], c["page"], c["dim"])
    k[..., 3] *= 4.0   # (keys have channels of large magnitude)
    if c["bits"] == 16:
        return k, v
    k, ks, kz = _quantize(k)
    v, vs, vz = _quantize(v)
    return k, v, ks, kz, vs, vz


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if c["kind"] == "lora":
        M, N, K, r, n = c["M"], c["N"], c["K"], c["rank"], c["adapters"]
        if c["runs"]:
            ids = torch.arange(M, device="cuda") * n // M
        else:   # every eighth row on average has no adapter
            ids = torch.randint(0, n, (M,), generator=gen, device="cuda")
            ids[torch.rand(M, generator=gen, device="cuda") < (0.125 if M > 1 else 0.0)] = -1
        return {"case": c, "x": _normal(gen, M, K), "y": _normal(gen, M, N), "ids": ids.to(torch.int32),
                "a": _normal(gen, n, r, K) / K ** 0.5, "b": _normal(gen, n, N, r) / r ** 0.5,
                "scale": torch.rand(n, generator=gen, device="cuda") + 0.5}
    news, lens = _news(c), _lens(c)
    rows, most = sum(news), -(-max(lens) // c["page"])
    used = [-(-n // c["page"]) for n in lens]
    pages = sum(used) + 4
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)[: sum(used)]
    table = torch.full((c["seqs"], most), -1, dtype=torch.int32)
    filled = torch.arange(most)[None, :] < torch.tensor(used)[:, None]
    table = table.cuda()
    table[filled.cuda()] = order
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(news).cumsum(0)]).to(torch.int32).cuda()
    state = {"case": c, "cache": _cache(gen, c, pages), "batch": (starts, torch.tensor(lens, dtype=torch.int32).cuda(), table),
             "max_new": max(news), "max_len": max(lens)}
    width = (c["hq"] + 2 * c["hkv"]) * c["dim"]
    qkv = _normal(gen, rows, width)   # a fused projection's output: q, k and v are column ranges of it
    q, k, v = qkv.split([c["hq"] * c["dim"], c["hkv"] * c["dim"], c["hkv"] * c["dim"]], dim=1)
    if c["kind"] == "attn":
        return {**state, "q": (q * 1.5).contiguous()}
    seq = torch.repeat_interleave(torch.arange(c["seqs"]), torch.tensor(news))
    at = torch.arange(rows) - starts.cpu()[seq] + (torch.tensor(lens) - torch.tensor(news))[seq]
    slots = table.cpu()[seq, at // c["page"]] * c["page"] + (at % c["page"]).to(torch.int32)
    freq = 10000.0 ** (-torch.arange(0, c["dim"], 2, device="cuda", dtype=torch.float64) / c["dim"])
    return {**state, "q": q, "k": k, "v": v, "inv_freq": freq.float(), "slots": slots.cuda()}


# ---- one pass -----------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"append": _append_plain, "attn": _attn_plain, "lora": _lora_plain}[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2408_08554_amd import binding as abq
    c = s["case"]
    if c["kind"] == "lora":
        return abq.abq_lora_add(s["x"], s["ids"], s["a"], s["b"], s["scale"], s["y"])
    if c["kind"] == "attn":
        return abq.abq_attn_paged(s["cache"], s["batch"], s["q"], c["dim"] ** -0.5, max_new=s["max_new"], max_len=s["max_len"])
    q = abq.abq_kv_append(s["cache"], s["batch"], s["k"], s["v"], q=s["q"], inv_freq=s["inv_freq"])
    if c["bits"] == 16:
        return q, s["cache"][0], s["cache"][1]
    return (q, *abq.abq_kv_read(s["cache"], s["slots"]))


def _rows(s):
    """Sequence and position of each row of the batch."""
    starts, lens, _ = s["batch"]
    rows = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(starts[1:].contiguous(), rows, right=True)
    return seq, lens[seq] - starts[seq + 1] + rows


def _rotated(x, cos, sin, dim):
    x = x.float().unflatten(1, (-1, dim))
    lo, hi = x[..., : dim // 2], x[..., dim // 2:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.float16)


def _append_plain(s):
    c, cache = s["case"], s["cache"]
    seq, at = _rows(s)
    angle = at.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q, k = _rotated(s["q"], cos, sin, c["dim"]), _rotated(s["k"], cos, sin, c["dim"])
    v = s["v"].unflatten(1, (-1, c["dim"]))
    page, off = s["batch"][2][seq, at // c["page"]].long(), at % c["page"]
    if c["bits"] == 16:
        cache[0][page, :, off], cache[1][page, :, off] = k, v
        return q.flatten(1), cache[0], cache[1]
    for t, x in zip((cache[0], cache[2], cache[3], cache[1], cache[4], cache[5]), (*_quantize(k), *_quantize(v))):
        t[page, :, off] = x
    page, off = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
    read = [((codes[page, :, off].float() - zero[page, :, off, None].float()) * scale[page, :, off, None]).to(torch.float16).flatten(1)
            for codes, scale, zero in ((cache[0], cache[2], cache[3]), (cache[1], cache[4], cache[5]))]
    return q.flatten(1), *read


def _values(cache, which, pages):
    """Keys (0) or values (1) of the pages, in 32 bits: [..., heads, page, dim]."""
    x = cache[which][pages].float()
    if len(cache) == 2:
        return x
    return (x - cache[3 + 2 * which][pages].float()[..., None]) * cache[2 + 2 * which][pages][..., None]


def _attn_plain(s):
    c = s["case"]
    starts, lens, table = s["batch"]
    S, D, G = c["seqs"], c["dim"], c["hq"] // c["hkv"]
    seq, at = _rows(s)
    rows = torch.arange(len(seq), device="cuda")
    place = rows - starts[seq]
    # the batch padded to its longest sequence: queries [S, heads, group * new, D], keys and values [S, heads, length, D]
    q = torch.zeros(S, s["max_new"], c["hkv"], G, D, device="cuda")
    q[seq, place] = s["q"].float().reshape(-1, c["hkv"], G, D) * D ** -0.5
    q = q.permute(0, 2, 3, 1, 4).reshape(S, c["hkv"], -1, D)
    pages = table.clamp(min=0).long()
    k, v = (_values(s["cache"], i, pages).transpose(1, 2).flatten(2, 3) for i in (0, 1))
    last = (lens - starts[1:] + starts[:-1])[:, None] + torch.arange(s["max_new"], device="cuda")   # position of each padded row
    hidden = torch.arange(k.shape[2], device="cuda") > last[..., None]
    hidden |= (torch.arange(k.shape[2], device="cuda") >= lens[:, None])[:, None]
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).unflatten(2, (G, -1))
    p.masked_fill_(hidden[:, None, None], float("-inf"))
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, -1)) / total
    return o.permute(0, 3, 1, 2, 4)[seq, place].flatten(1).to(torch.float16)


def _lora_plain(s):
    c = s["case"]
    u = (s["x"].float() @ s["a"].float().flatten(0, 1).T).unflatten(1, (c["adapters"], -1))
    mine = s["ids"][:, None] == torch.arange(c["adapters"], device="cuda")
    u *= (mine * s["scale"])[..., None]
    return (s["y"].float() + u.flatten(1) @ s["b"].float().permute(0, 2, 1).flatten(0, 1)).to(torch.float16)


# ---- floor --------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "lora":
        M, N, K, r = c["M"], c["N"], c["K"], c["rank"]
        pairs = min(c["adapters"], M)
        return {"bytes": 2.0 * (M * K + 2 * M * N + pairs * r * (K + N)), "flops": 2.0 * M * r * (K + N)}
    rows, vector = sum(_news(c)), c["dim"] * 2 if c["bits"] == 16 else c["dim"] + 5
    q_bytes = 2.0 * rows * c["hq"] * c["dim"]
    if c["kind"] == "append":
        kv = 2.0 * rows * c["hkv"]
        back = 0.0 if c["bits"] == 16 else kv * (vector + 2 * c["dim"])   # the new vectors are read back as binary16
        return {"bytes": 2 * q_bytes + kv * (2 * c["dim"] + vector) + back, "flops": 3.0 * rows * (c["hq"] + c["hkv"]) * c["dim"]}
    seen = sum(n * (2 * t - n + 1) // 2 for n, t in zip(_news(c), _lens(c)))
    return {"bytes": 2 * q_bytes + 2.0 * sum(_lens(c)) * c["hkv"] * vector, "flops": 4.0 * seen * c["hq"] * c["dim"]}


# ---- the definition, in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _append_exact, "attn": _attn_exact, "lora": _lora_exact}[case["kind"]](s)


def _lora_exact(s):
    y = s["y"].double()
    for i, id_ in enumerate(s["ids"].unique().tolist()):
        if id_ >= 0:
            at = (s["ids"] == id_).nonzero()[:, 0]
            y[at] += s["scale"][id_].double() * ((s["x"][at].double() @ s["a"][id_].double().T.contiguous()) @ s["b"][id_].double().T.contiguous())
    return y


def _sequence(s, i):
    """Rows of a sequence, their positions, and the cache's place of each of its tokens."""
    starts, lens, table = s["batch"]
    page, n, first, end = s["case"]["page"], int(lens[i]), int(starts[i]), int(starts[i + 1])
    t = torch.arange(n, device="cuda")
    return slice(first, end), t[n - (end - first):], table[i][t // page].long(), t % page


def _held(cache, which, page, off):
    """What the cache holds of all heads at some tokens: [tokens, heads, dim]."""
    x = cache[which][page, :, off].double()
    if len(cache) == 6:
        x = (x - cache[3 if which == 0 else 5][page, :, off].double().unsqueeze(2)) * cache[2 if which == 0 else 4][page, :, off].double().unsqueeze(2)
    return x


def _attn_exact(s):
    c, D = s["case"], s["case"]["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for i in range(c["seqs"]):
        rows, at, page, off = _sequence(s, i)
        k, v = _held(s["cache"], 0, page, off), _held(s["cache"], 1, page, off)
        for h in range(c["hq"]):
            kv = h * c["hkv"] // c["hq"]
            score = s["q"][rows, h * D:(h + 1) * D].double() @ k[:, kv].T.contiguous() / D ** 0.5
            score = torch.where(torch.arange(len(page), device="cuda") <= at[:, None], score, float("-inf"))
            out[rows, h * D:(h + 1) * D] = torch.softmax(score, 1) @ v[:, kv].contiguous()
    return out


def _turned(x, at, freq):
    """Each head's vectors turned by their positions' angles: coordinate j with coordinate j + dim / 2, as complex numbers."""
    n = len(freq)
    z = torch.complex(*x.double().reshape(len(x), -1, 2, n).unbind(2))
    z = z * torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), at.double().outer(freq.double())).unsqueeze(1)
    return torch.cat([z.real, z.imag], 2)


def _append_exact(s):
    c, cache = s["case"], s["cache"]
    q, back = [], []
    held = [t.double() for t in cache[:2]] if c["bits"] == 16 else None
    for i in range(c["seqs"]):
        rows, at, page, off = _sequence(s, i)
        page, off = page[at], off[at]
        k, v = _turned(s["k"][rows], at, s["inv_freq"]), s["v"][rows].double().reshape(len(at), -1, c["dim"])
        q.append(_turned(s["q"][rows], at, s["inv_freq"]).flatten(1))
        if held:
            held[0][page, :, off], held[1][page, :, off] = k, v
            continue
        pair = []
        for x in (k.to(torch.float16).double(), v):   # (what is quantized is the binary16 vector)
            lo, hi = x.amin(2, keepdim=True).clamp(max=0), x.amax(2, keepdim=True).clamp(min=0)
            step = ((hi - lo) / 255).to(torch.float32).double()
            step[step == 0] = 1
            z = (-lo / step).round().clamp(0, 255)
            pair.append((((x / step).round() + z).clamp(0, 255) - z).mul(step).flatten(1))
        back.append(pair)
    if held:
        return torch.cat(q), held[0], held[1]
    return torch.cat(q), torch.cat([b[0] for b in back]), torch.cat([b[1] for b in back])
