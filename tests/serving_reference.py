"""Plain 64-bit forms of the paged cache, the attention over it and the adapters, on host tensors, and the inputs of their tests."""
import torch

F64 = torch.float64


class Paged:
    """A cache and a batch on the host: seqs given as (new, past) pairs, pages handed out in a random order with holes between."""

    def __init__(self, seqs, heads_q, heads, dim, page, bits=16, seed=0, extra_rows=0, extra_pages=3):
        g = torch.Generator().manual_seed(seed)
        self.gen, self.bits, self.page, self.heads_q, self.heads, self.dim = g, bits, page, heads_q, heads, dim
        self.news = [n for n, _ in seqs]
        self.lens = torch.tensor([max(0, n + past) for n, past in seqs], dtype=torch.int32)
        self.row_start = torch.tensor([0] + self.news).cumsum(0).to(torch.int32)
        self.rows = max(1, int(self.row_start[-1]) + extra_rows)
        used = [-(-int(n) // page) for n in self.lens]
        total = sum(used) + extra_pages
        order = torch.randperm(total, generator=g)[: sum(used)].to(torch.int32)
        self.pages = torch.full((len(seqs), max(1, max(used))), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(used):
            self.pages[s, :n] = order[at:at + n]
            at += n
        shape = (total, heads, page, dim)
        if bits == 16:
            self.cache = [self.normal(*shape), self.normal(*shape)]
        else:
            self.cache = [torch.randint(0, 256, shape, generator=g, dtype=torch.uint8), torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)]
            for _ in range(2):
                self.cache += [torch.rand(shape[:3], generator=g) * 0.03 + 0.002, torch.randint(96, 160, shape[:3], generator=g, dtype=torch.uint8)]
        self.q = self.normal(self.rows, heads_q * dim)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen).to(torch.float16)

    def device(self):
        """(cache, batch, q) on the device."""
        return tuple(t.cuda() for t in self.cache), (self.row_start.cuda(), self.lens.cuda(), self.pages.cuda()), self.q.cuda()

    def held(self, which, s, t):
        """What the cache holds for token t of sequence s: [heads, dim], or None where there is no page."""
        at = t // self.page
        if at >= self.pages.shape[1]:
            return None
        page = int(self.pages[s, at])
        if not 0 <= page < self.cache[0].shape[0]:
            return None
        x = self.cache[which][page, :, t % self.page].to(F64)
        if self.bits == 8:
            x = (x - self.cache[3 + 2 * which][page, :, t % self.page].to(F64)[:, None]) * self.cache[2 + 2 * which][page, :, t % self.page].to(F64)[:, None]
        return x

    def attention(self, scale, causal=True, max_new=None, max_len=None):
        """(y, bound) [rows, heads_q, dim] in 64 bits, NaN for rows that are left as they were; bound: how far a result in
        binary16 may be off.  With eps = 2^-24 a score's dot product of d terms and its scaling are off by (d + 4) eps sum |q k|
        scale, which changes a weight by that much relatively (twice that in the quotient, whose denominator has the same
        error), exponential and logarithm (of a scale of codes, up to 2^5 in size) by 2^-18 together, and each weight - of codes: times
        its scale - by half a step of binary16, 2^-11, or 2^-24 of the largest where it falls below the normal range; n sums
        add n eps; the result is rounded by half a step."""
        y = torch.full((self.rows, self.heads_q, self.dim), float("nan"), dtype=F64)
        bound = torch.zeros_like(y)
        group = self.heads_q // self.heads
        for s, n in enumerate(self.news):
            length = int(self.lens[s]) if max_len is None else min(int(self.lens[s]), max_len)
            held = [(t, self.held(0, s, t), self.held(1, s, t)) for t in range(length)]
            held = [h for h in held if h[1] is not None]
            step = torch.ones(self.heads, 1, len(held), dtype=F64)   # what a value's weight is multiplied by ahead of the product
            if self.bits == 8:
                for j, h in enumerate(held):
                    step[:, 0, j] = self.cache[4][int(self.pages[s, h[0] // self.page]), :, h[0] % self.page].to(F64)
            times = torch.tensor([h[0] for h in held])
            if held:
                k, v = torch.stack([h[1] for h in held]), torch.stack([h[2] for h in held])   # [tokens, heads, dim]
            for i in range(n if max_new is None else min(n, max_new)):
                row, pos = int(self.row_start[s]) + i, int(self.lens[s]) - n + i
                y[row] = 0
                see = (times <= pos) if causal else torch.ones(len(held), dtype=torch.bool)
                if not len(held) or not see.any():
                    continue
                q = self.q[row].to(F64).view(self.heads, group, self.dim)
                kk, vv = k[see].permute(1, 0, 2), v[see].permute(1, 0, 2)
                score = q @ kk.transpose(1, 2) * scale
                w = torch.softmax(score, -1)
                y[row] = (w @ vv).reshape(self.heads_q, self.dim)
                size = (q.abs() @ kk.abs().transpose(1, 2) * abs(scale)).amax(-1, keepdim=True)
                off = 2 * (self.dim + 4) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -11 + int(see.sum()) * 2.0 ** -24
                st = step[..., see]
                mean = w @ vv.abs() * off + 2.0 ** -24 * (w * st).amax(-1, keepdim=True) * (vv.abs() / st.transpose(1, 2)).sum(1, keepdim=True)
                bound[row] = mean.reshape(self.heads_q, self.dim) + 2.0 ** -11 * y[row].abs() + 2.0 ** -25
        return y, bound


def rotated(x, positions, inv_freq, interleaved=False):
    """x [rows, heads, dim] turned by position * inv_freq, in 64 bits; (values, sizes of the two products)."""
    x, r = x.to(F64), 2 * len(inv_freq)
    a = positions.to(F64)[:, None, None] * inv_freq.to(F64)
    y, size = x.clone(), x.abs()
    i0 = torch.arange(r // 2) * 2 if interleaved else torch.arange(r // 2)
    i1 = i0 + 1 if interleaved else i0 + r // 2
    y[..., i0], y[..., i1] = x[..., i0] * a.cos() - x[..., i1] * a.sin(), x[..., i1] * a.cos() + x[..., i0] * a.sin()
    size[..., i0] = size[..., i1] = x[..., i0].abs() + x[..., i1].abs()
    return y, size


def rotated_bound(y, size):
    """Sine and cosine within 2^-23, a product rounded in binary32, one rounding of the sum, then half a step of binary16."""
    return size * 2.0 ** -22 + (y.abs() + size * 2.0 ** -22) * 2.0 ** -11 + 2.0 ** -25


def adapted(x, ids, a, b, scale, y):
    """(out, bound) of the adapters in 64 bits.  K products summed in binary32, A x kept to 2^-21 of its largest element, rank products
    summed in binary32, times scale, plus y, half a step of binary16."""
    out, bound = y.to(F64).clone(), torch.zeros(y.shape, dtype=F64)
    K, r = x.shape[1], a.shape[1]
    for m, i in enumerate(ids.tolist()):
        if 0 <= i < a.shape[0]:
            A, B, s = a[i].to(F64), b[i].to(F64), float(scale[i])
            u = A @ x[m].to(F64)
            off = (K + 2) * 2.0 ** -24 * (A.abs() @ x[m].to(F64).abs()) + 2.0 ** -21 * u.abs().max()
            out[m] += s * (B @ u)
            bound[m] = abs(s) * (B.abs() @ (off + (r + 4) * 2.0 ** -24 * u.abs())) + 2.0 ** -23 * out[m].abs()
    return out, torch.where(bound > 0, bound + 2.0 ** -11 * (out.abs() + bound) + 2.0 ** -25, bound)
