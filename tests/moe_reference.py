"""A layer of experts from its formulas, in 64 bits on the CPU (torch tensors of codes, scales, logits in; float64 out)."""
import torch

INF = float("inf")


def scores(logits, sigmoid):
    """float64 [tokens, experts]; 0 for experts that are not there (minus infinity, NaN)."""
    x = logits.double()
    there = x > -INF
    x = torch.where(there, x, -INF)
    if sigmoid:
        s = torch.sigmoid(x)
    else:
        top = x.amax(1, keepdim=True)
        e = torch.where(there, torch.exp(x - torch.where(top > -INF, top, 0.0)), 0.0)
        s = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    return torch.where(there, s, 0.0), there


def routed(logits, top, bias=None, sigmoid=False, renormalize=True, scale=1.0):
    """(ids, weights float64, starts, order, places, bound of a weight's error)."""
    T, E = logits.shape
    s, there = scores(logits, sigmoid)
    key = logits.double() if bias is None else s + bias.double()
    there = there & (key > -INF)
    ids = torch.full((T, top), -1, dtype=torch.int64)
    for t in range(T):
        ok = there[t].nonzero()[:, 0].tolist()
        ok.sort(key=lambda e: (-float(key[t, e]), e))
        ids[t, : min(top, len(ok))] = torch.tensor(ok[:top], dtype=torch.int64)
    chosen = ids >= 0
    at = ids.clamp(min=0)
    x = torch.where(chosen, logits.double().gather(1, at), -INF)
    if renormalize and not sigmoid:   # (from the logits: scores may all underflow)
        m = x.amax(1, keepdim=True)
        w = torch.where(chosen, torch.exp(x - torch.where(m > -INF, m, 0.0)), 0.0)
    elif renormalize:                 # (the largest logit taken out where all are far below 0)
        m = x.amax(1, keepdim=True).clamp(max=0.0)
        m = torch.where(m > -INF, m, 0.0)
        w = torch.where(chosen, torch.where(x > 0, 1 / (1 + torch.exp(-x)), torch.exp(x - m) / (1 + torch.exp(x))), 0.0)
    else:
        w = torch.where(chosen, s.gather(1, at), 0.0)
    if renormalize:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    w = w * scale
    flat = ids.flatten()
    order = torch.cat([(flat == e).nonzero()[:, 0] for e in range(E)])
    places = torch.full_like(flat, -1)
    places[order] = torch.arange(len(order))
    starts = torch.tensor([0] + [int((flat == e).sum()) for e in range(E)]).cumsum(0)
    order = torch.cat([order, torch.full((T * top - len(order),), -1)])
    # Half steps of binary32: the difference from the largest logit (its rounding is |difference| / 2^24 of the exponential), an exponential
    # within two steps of its value in numerator and denominator (8), a sum of up to 16 and 6 levels (22), whose terms' own differences weigh
    # at most ln(1024) < 7, quotient, complement and scale (3).  What underflows is off by less than 2^-126.
    best = torch.where(there, logits.double(), -INF).amax(1, keepdim=True)
    d = torch.where(chosen & (best > -INF), (x - best).abs(), 0.0)
    bound = (d + 40) * 2.0**-24 * w.abs() + 2.0**-126 * max(1.0, abs(scale))
    return ids, w, starts, order, places.view(T, top), bound


def gemm(codes, a_scale, a_zero, w_codes, w_scale, w_zero, p, q, starts, order, top, rows):
    """Rows of Y as binary16 (the integer sum exact, two binary32 products, one rounding), NaN where no expert has the row."""
    y = torch.full((rows, w_codes.shape[1]), float("nan"), dtype=torch.float16)
    a = (codes & (2**q - 1)).double() - a_zero.double()[:, None]
    w = (w_codes & (2**p - 1)).double() - w_zero.double()[..., None]
    for e in range(len(starts) - 1):
        r = torch.arange(int(starts[e]), int(starts[e + 1]))
        if len(r):
            src = r if order is None else order[r].long() // top
            acc = (a[src] @ w[e].T).long()   # (a whole number: no -0)
            y[r] = (acc.float() * a_scale[src][:, None] * w_scale[e]).to(torch.float16)
    return y


def combined(y, places, weights, add=None):
    """(out float64, bound of its error): a chain of `top` binary32 operations over the terms, and the rounding to binary16."""
    T, top = places.shape
    out = torch.zeros((T, y.shape[1]), dtype=torch.float64) if add is None else add.double()
    size = out.abs()
    for j in range(top):
        there = ((places[:, j] >= 0) & (places[:, j] < len(y)))[:, None]
        term = weights[:, j, None].double() * y[places[:, j].clamp(0, len(y) - 1).long()].double()
        out = out + torch.where(there, term, 0.0)
        size = size + torch.where(there, term.abs(), 0.0)
    chain = size * top * 2.0**-24
    return out, chain + (out.abs() + chain) * 2.0**-11 + 2.0**-25


def groups(counts):
    """Row starts of experts with so many rows each."""
    return torch.tensor([0, *counts]).cumsum(0).to(torch.int32)


