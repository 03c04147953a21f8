"""abq_attn_paged where scores, weights or hidden tokens are out of the ordinary: infinite keys, scores of any size, tokens that a row does
not see, and every token of a long context for itself."""
import pytest
import torch

from serving_reference import Paged

pytestmark = pytest.mark.gpu


def run(abq, p, scale=None, **kw):
    cache, batch, q = p.device()
    return abq.abq_attn_paged(cache, batch, q, p.dim ** -0.5 if scale is None else scale, **kw).cpu().view(p.rows, p.heads_q, p.dim)


def place(p, s, t):
    """Page and offset of token t of sequence s."""
    return int(p.pages[s, t // p.page]), t % p.page


class Without(Paged):
    """Tokens whose weight is zero: the 64-bit form leaves them out."""
    out = ()

    def held(self, which, s, t):
        return None if (s, t) in self.out else super().held(which, s, t)


# ---- infinite keys ---------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [1, 3, 40, 90])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 144, 160, 256])
def test_a_key_whose_score_is_minus_infinity_has_no_weight(abq, dim, n):
    """In any column, the first eight (which stand in for the columns behind narrower heads) among them."""
    for column in (0, 7, 8, dim - 1):
        p = Without([(n, 70), (2, 11)], 4, 2, dim, 16, seed=dim + column)
        p.q.view(p.rows, 4, dim)[..., column] = 1.0 + torch.arange(p.rows)[:, None] % 3
        p.out = [(0, 0), (0, 5), (0, 40), (1, 3)]
        for s, t in p.out:
            page, o = place(p, s, t)
            p.cache[0][page, :, o, column] = -float("inf")
        y = run(abq, p)
        want, bound = p.attention(dim ** -0.5)
        assert ((y.double() - want).abs() <= bound).all(), column


@pytest.mark.parametrize("n", [1, 3, 40, 90])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_a_key_whose_score_is_infinite_makes_its_row_nan(abq, dim, n):
    p = Paged([(n, 70)], 4, 2, dim, 16, seed=dim)
    p.q.view(p.rows, 4, dim)[..., 1] = 1.0
    page, o = place(p, 0, 70 + n - 1)
    p.cache[0][page, 0, o, 1] = float("inf")
    y = run(abq, p)
    assert y[n - 1, :2].isnan().all() and y[n - 1, 2:].isfinite().all() and y[:n - 1].isfinite().all()


# ---- weights in more bits than binary16 has ----------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("hq,beside", [(4, 0), (40, 0), (4, 100)])
def test_weights_of_few_rows_are_not_rounded_to_binary16(abq, hq, beside, dim, bits):
    """Two, four or six tokens of nearly the same weight whose values, of size 1, cancel but for 2^-7.  With 21 bits of a weight, 2^-21 for its
    exponential and, of codes, 2^-18 for the logarithm of a scale: a result is off by 2^-17 at most, and by half a step of its own."""
    p = Paged([(1, 1 + 2 * (s % 3)) for s in range(24)] + ([(beside, 0)] if beside else []), hq, 2, dim, 16, bits, seed=dim + hq)
    p.q.zero_()
    p.q.view(p.rows, hq, dim)[..., 5] = 1.0
    sign = torch.where(torch.rand(p.cache[1].shape, generator=p.gen) < 0.5, 1.0, -1.0)
    sign[:, :, 1::2] = -sign[:, :, ::2]
    if bits == 16:
        p.cache[0].copy_(torch.rand(p.cache[0].shape, generator=p.gen) * 2.0 ** -6)
        p.cache[1].copy_(sign)
    else:
        p.cache[2].fill_(2.0 ** -13), p.cache[3].fill_(128)
        level = torch.randint(1, 120, p.cache[4].shape, generator=p.gen)   # one value's codes and scale, of size 1 together
        p.cache[1].copy_((128 + sign * level[..., None]).to(torch.uint8))
        p.cache[4].copy_(1.0 / level.float()), p.cache[5].fill_(128)
    y = run(abq, p, 1.0).double()[:24]
    want = p.attention(1.0)[0][:24]
    assert want.abs().max() < 2.0 ** -5
    assert ((y - want).abs() <= 2.0 ** -17 + 2.0 ** -11 * want.abs() + 2.0 ** -25).all()
    assert not torch.equal(y, torch.zeros_like(y))


# ---- tokens that a row does not see ----------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("n,hq,past", [(4, 4, 300), (3, 10, 330), (5, 10, 350), (100, 2, 700), (60, 4, 400), (70, 4, 1500)])
def test_hidden_tokens_do_not_reach_the_bits(abq, n, hq, past, dim, bits):
    """Other keys and values in the last new tokens: the rows before them keep every bit, whatever the later rows' scores do."""
    p = Paged([(n, past), (1, 20)], hq, 2, dim, 16, bits, seed=n + dim)
    first = run(abq, p)
    for t in range(past + n - 2, past + n):
        page, o = place(p, 0, t)
        aim = p.q[n - 1].view(2, hq // 2, dim)[:, 0].float().sign()
        if bits == 16:
            p.cache[0][page, :, o] = (aim * 8).half()
            p.cache[1][page, :, o] = 3.0
        else:
            p.cache[0][page, :, o] = (128 + 127 * aim).to(torch.uint8)
            p.cache[2][page, :, o], p.cache[3][page, :, o] = 0.06, 128
            p.cache[4][page, :, o] = 0.5
    then = run(abq, p)
    assert torch.equal(first[:n - 2], then[:n - 2]) and torch.equal(first[n:], then[n:])
    assert not torch.equal(first[n - 1], then[n - 1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 0.0, -float("inf")])
@pytest.mark.parametrize("dim", [64, 80, 256])
@pytest.mark.parametrize("n", [1, 20, 90])
def test_scales_of_codes_in_hidden_places_stay_there(abq, n, dim, bad):
    """The rest of the last page, pages of no sequence (the first one stands in where a page is missing), and later tokens."""
    p = Paged([(n, 50), (2, 11), (40, 300)], 4, 2, dim, 16, bits=8, seed=n)
    p.pages[2, 3], p.pages[0, 1] = -1, 1 << 30
    used = torch.zeros(p.cache[0].shape[0], 16, dtype=torch.bool)
    for s, length in enumerate(p.lens.tolist()):
        for t in range(length):
            if 0 <= int(p.pages[s, t // 16]) < len(used):
                used[int(p.pages[s, t // 16]), t % 16] = True
    for i in (2, 4):
        p.cache[i].permute(0, 2, 1)[~used] = bad
    for causal in (True, False):
        y = run(abq, p, causal=causal)
        want, bound = p.attention(dim ** -0.5, causal)
        assert ((y.double() - want).abs() <= bound).all()
    before = run(abq, p)
    for s, t in ((0, 50 + n - 1), (2, 339)):
        page, o = place(p, s, t)
        p.cache[2][page, :, o] = p.cache[4][page, :, o] = bad
    after = run(abq, p)
    mine = [n - 1, p.rows - 1]
    keep = torch.tensor([r for r in range(p.rows) if r not in mine])
    assert torch.equal(before[keep], after[keep])


# ---- scores of any size ----------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("past", [30, 1500])
@pytest.mark.parametrize("n", [1, 5, 90])
@pytest.mark.parametrize("ahead", ["last", "first"])
@pytest.mark.parametrize("scale", [0.125, -0.3, 1e12, 1e28])
def test_large_scores(abq, n, past, bits, ahead, scale):
    """Scores of 2^17 to 2^124, whole multiples of their difference: the token that is ahead, a row's own or the first, has all the weight, and
    its value comes out as it is."""
    p = Paged([(n, past)], 4, 2, 64, 16, bits, seed=n)
    sign = torch.where(torch.randn(64, generator=p.gen) < 0, -1.0, 1.0)
    p.q[:] = (sign * (8192.0 if (scale > 0) == (ahead == "last") else -8192.0)).half().repeat(4)
    for t in range(past + n):
        page, o = place(p, 0, t)
        if bits == 16:
            p.cache[0][page, :, o] = ((t + 1) * 2.0 * sign).half()
        else:
            p.cache[0][page, :, o] = (128 + sign * 100).to(torch.uint8)
            p.cache[2][page, :, o], p.cache[3][page, :, o] = (t + 1) / 64, 128
    y = run(abq, p, scale)
    for i in range(n):
        want = p.held(1, 0, past + i if ahead == "last" else 0)[:, None]
        assert ((y[i].double().view(2, 2, 64) - want).abs() <= (2.0 ** -11 + 2.0 ** -20) * want.abs()).all(), i


# ---- rows without a weight -------------------------------------------------------------------------
@pytest.mark.parametrize("past", [20, 1500])
@pytest.mark.parametrize("n", [1, 3, 40, 90])
@pytest.mark.parametrize("dim", [64, 80, 256])
def test_rows_whose_scores_are_all_minus_infinity(abq, dim, n, past):
    """0 / 0 there, as by the formula; zeros where a row sees no token."""
    p = Paged([(n, past), (n, -n), (2, 11)], 4, 2, dim, 16, seed=dim + n)
    p.q.view(p.rows, 4, dim)[..., 2] = 1.0
    for t in range(past + n):
        page, o = place(p, 0, t)
        p.cache[0][page, 1, o, 2] = -float("inf")
    y = run(abq, p)
    assert y[:n, 2:].isnan().all() and y[:n, :2].isfinite().all()
    assert (y[n:2 * n] == 0).all() and y[2 * n:].isfinite().all()
    p.pages[0] = -1
    assert (run(abq, p)[:2 * n] == 0).all()


# ---- every token for itself ------------------------------------------------------------------------
LONG = [([(1, 5000)], 2, 2), ([(1, 2049)], 8, 1), ([(3, 3000), (2, 700)], 16, 2), ([(1, 2600), (1, 90)], 24, 1), ([(90, 1500)], 2, 2), ([(40, 5000), (1, 900), (0, 3)], 4, 2),
        ([(33, 4000)] + [(33, 0)] * 63 + [(1, 3000)], 4, 4), ([(2, 1200), (20, 600)], 20, 1), ([(1, 1700)] * 3 + [(300, 40)], 32, 1)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 112, 128, 256])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_every_token_counts_once(abq, case, dim, bits):
    """Equal weights (scale 0), and column d of head h one for the tokens t with t % (heads dim) = h dim + d: a row's result is how many
    of those it sees over how many it sees in all, so that a token lost or taken twice shows.  The weights, their sums and products are
    exact, the quotient takes a rounding of binary32, the result one of binary16."""
    seqs, hq, h = LONG[case]
    page = 64 if case % 2 else 16
    p = Paged(seqs, hq, h, dim, page, bits, seed=case)
    every = h * dim
    p.cache[1].zero_()
    if bits == 8:
        p.cache[4].fill_(1.0), p.cache[5].zero_()
    for s, length in enumerate(p.lens.tolist()):
        t = torch.arange(length)
        at = t % every
        p.cache[1][p.pages[s, t // page].long(), at // dim, t % page, at % dim] = 1
    y = run(abq, p, 0.0).double()
    cls = torch.arange(every).view(h, dim)
    for s, n in enumerate(p.news):
        for i in range(n):
            seen = int(p.lens[s]) - n + i + 1
            count = ((seen - 1 - cls) // every + 1).clamp(min=0)
            want = (count / seen)[:, None].expand(h, hq // h, dim).reshape(hq, dim)
            assert ((y[int(p.row_start[s]) + i] - want).abs() <= want * (2.0 ** -11 + 2.0 ** -22) + 2.0 ** -25).all(), (s, i)


EDGES = [0, 1, 15, 16, 31, 32, 33, 63, 64, 127, 128, 255, 256, 257, 511, 512, 513, 767, 768, 895, 896, 1023, 1024, 1025, 1791, 1792, 2048]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 112, 128, 256])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_every_key_is_its_tokens(abq, case, dim, bits):
    """Each row and head points at one token's key, those at edges of steps, parts and pages from either end among them, with a score of 80; the
    others', products with random vectors at up to 13 a standard deviation, stay below 60, and 6000 of them have 2^-16 of the weight."""
    seqs, hq, h = LONG[case]
    page, g = 16 if case % 2 else 64, hq // h
    p = Paged(seqs, hq, h, dim, page, bits, seed=case + 1)
    if bits == 8:
        p.cache[2].fill_(0.01)
    want = torch.empty(p.rows, h, g, dim, dtype=torch.float64)
    q = p.q.view(p.rows, h, g, dim)
    head = torch.arange(h)[None, :, None]
    for s, n in enumerate(p.news):
        row = int(p.row_start[s]) + torch.arange(n)
        seen = (int(p.lens[s]) - n + torch.arange(n) + 1)[:, None, None]
        r = (row[:, None, None] * 31 + head * 7 + torch.arange(g)) % (3 * len(EDGES))
        edge = torch.tensor(EDGES)[r % len(EDGES)]
        t = torch.where(r < len(EDGES), edge, torch.where(r < 2 * len(EDGES), seen - 1 - edge, -1))
        t = torch.where((t < 0) | (t >= seen), (torch.rand(t.shape, generator=p.gen) * seen).long(), t)
        pg, o = p.pages[s][t // page].long(), t % page
        key, value = (p.cache[i][pg, head, o].double() for i in (0, 1))
        if bits == 8:
            key = (key - p.cache[3][pg, head, o, None].double()) * 0.01
            value = (value - p.cache[5][pg, head, o, None].double()) * p.cache[4][pg, head, o, None].double()
        q[row] = (key * (80.0 * dim ** 0.5 / (key * key).sum(-1, keepdim=True))).half()
        want[row] = value
    y = run(abq, p).double().view(want.shape)
    own = torch.arange(p.rows) < int(p.row_start[-1])
    assert ((y - want).abs() <= 2.0 ** -10 * want.abs() + 2.0 ** -13)[own].all()


# ---- two tiles of few rows -------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_two_tiles_of_few_rows(abq, dim, bits):
    """17 to 32 rows of a sequence and key head: over long contexts in parts, and beside sequences with more."""
    for p, kw in ((Paged([(3, 3000), (2, 700)], 16, 2, dim, 16, bits, seed=dim), dict(max_new=3)), (Paged([(1, 2600), (1, 90), (0, 5)], 20, 1, dim, 64, bits, seed=dim + 1), dict(max_new=1)),
                  (Paged([(1, 2600), (1, 90), (40, 500)], 20, 1, dim, 16, bits, seed=dim + 2), {}), (Paged([(1, 1000), (5, 30), (1, 0), (9, 1500)], 32, 1, dim, 16, bits, seed=dim + 3, extra_rows=2), {})):
        y = run(abq, p, **kw)
        want, bound = p.attention(dim ** -0.5)
        left = want.isnan().all(-1).all(-1)
        assert ((y.double() - want).abs() <= bound)[~left].all()


# ---- the longest sequences -------------------------------------------------------------------------
@pytest.mark.parametrize("n", [1, 40])
def test_a_sequence_of_more_than_2_to_the_30_tokens(abq, n):
    """2^31 - 1 tokens in a table that names one page over and over: the first 2^30 are seen, as if it were the one page."""
    p = Paged([(n, 4096 - n)], 1, 1, 16, 4096, seed=n)
    (k, v), (starts, lens, pages), q = p.device()
    many = torch.full((1, 1 << 19), int(p.pages[0, 0]), dtype=torch.int32, device="cuda")
    lens.fill_((1 << 31) - 1)
    y = abq.abq_attn_paged((k, v), (starts, lens, many), q, 0.25).cpu().view(n, 1, 16).double()
    want, bound = p.attention(0.25, causal=False)
    # (sums: 2^15 to 2^20 additions of about the same in binary32 each, off by as many times 2^-24 at most)
    assert ((y - want).abs() <= bound + 2.0 ** -4 * want.abs() + 2.0 ** -6).all()


def test_none_is_the_default_mask(abq):
    p = Paged([(5, 20), (40, 3)], 4, 2, 64, 16, seed=1)
    y = run(abq, p, causal=None)
    assert torch.equal(y, run(abq, p, causal=True)) and torch.equal(y, run(abq, p)) and not torch.equal(y, run(abq, p, causal=False))


@pytest.mark.parametrize("n", [1, 60])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_missing_pages_cost_nothing_more_where_the_first_page_is_not_finite(abq, n, dim):
    """A sequence whose pages are gone but for the last (a window over a long context): the cache's first page, which stands in for them,
    may hold anything; results and time are as if it held numbers."""
    p = Paged([(n, 8000), (1, 3)], 8, 2, dim, 16, seed=dim)
    p.pages[0, :480] = -1
    p.pages[0, 480:], p.pages[1, 0] = 1 + torch.arange(p.pages.shape[1] - 480), 100   # (none of them the first)
    cache, batch, q = p.device()
    want, bound = p.attention(dim ** -0.5)

    def timed():
        best = 1e9
        for _ in range(3):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            for _ in range(4):
                y = abq.abq_attn_paged(cache, batch, q, dim ** -0.5)
            e[1].record()
            torch.cuda.synchronize()
            best = min(best, e[0].elapsed_time(e[1]))
        assert ((y.cpu().view(want.shape).double() - want).abs() <= bound).all()
        return best

    timed()
    before = timed()
    cache[0][0], cache[1][0] = float("nan"), float("inf")
    assert timed() < 4 * before
