"""abq_attn_paged against its 64-bit form: lengths, masks, heads, pages, types."""
import pytest
import torch

from serving_reference import Paged

pytestmark = pytest.mark.gpu


def check(abq, p, causal=True, scale=None, strided=False, **bounds):
    scale = p.dim ** -0.5 if scale is None else scale
    cache, batch, q = p.device()
    if strided:
        q = torch.cat([q, q, q], 1)[:, p.q.shape[1]:2 * p.q.shape[1]]
    y = torch.full((p.rows, p.heads_q * p.dim), 7.0, dtype=torch.float16, device="cuda")
    assert abq.abq_attn_paged(cache, batch, q, scale, causal=causal, y=y, **bounds) is y
    want, bound = p.attention(scale, causal, bounds.get("max_new"), bounds.get("max_len"))
    got = y.cpu().view(want.shape)
    left = want.isnan().all(-1).all(-1)
    assert (got[left] == 7.0).all(), "rows of no sequence were written"
    off = (got.double() - want).abs()
    ok = (off <= bound) | (want.isnan() & got.isnan()) | (got.double() == want)   # (the last: infinities)
    assert ok[~left].all(), f"{int((~ok[~left]).sum())} of {ok[~left].numel()} off, up to {(off / bound)[~left].nan_to_num(9e9).max():.3g} x the bound, rows {sorted(set((~ok).nonzero()[:, 0].tolist()))[:8]}"
    return y


ONE = [(1, 0), (1, 1), (1, 14), (1, 15), (1, 16), (1, 62), (1, 63), (1, 64), (1, 300)]
MIXED = [(1, 0), (3, 0), (17, 5), (1, 200), (0, 40), (70, 33), (2, 127), (130, 0)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hq,h", [(4, 4), (8, 1), (6, 2), (20, 1), (40, 1)])
def test_one_token_each(abq, bits, hq, h):
    check(abq, Paged(ONE, hq, h, 128, 16, bits, seed=hq), max_new=1)
    check(abq, Paged(ONE, hq, h, 128, 64, bits, seed=hq + 1))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 160, 256])
def test_head_sizes(abq, bits, dim):
    check(abq, Paged(ONE, 4, 2, dim, 16, bits, seed=dim), max_new=1)
    check(abq, Paged(MIXED, 4, 2, dim, 32, bits, seed=dim + 1, extra_rows=2))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hq,h", [(3, 3), (8, 2), (7, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks(abq, bits, hq, h, causal):
    check(abq, Paged(MIXED, hq, h, 128, 16, bits, seed=hq, extra_rows=1), causal, strided=True)


@pytest.mark.parametrize("n", [1, 2, 4, 5, 8, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200])
def test_lengths_of_a_chunk(abq, n):
    check(abq, Paged([(n, 0), (n, 40)], 2, 1, 64, 16, seed=n))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("past", [500, 1023, 2049, 5000])
def test_long_contexts(abq, bits, past):
    check(abq, Paged([(1, past)], 2, 2, 128, 16, bits, seed=past), max_new=1)
    check(abq, Paged([(2, past), (1, 7)], 8, 2, 64, 64, bits, seed=past + 1))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 128, 144])
def test_chunks_over_long_contexts(abq, bits, dim):
    check(abq, Paged([(70, 1500)], 2, 2, dim, 16, bits, seed=dim))      # in three parts, in ten
    check(abq, Paged([(40, 5000), (1, 900), (0, 3)], 4, 2, dim, 32, bits, seed=dim + 1))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim", [64, 128, 144])
def test_long_contexts_in_one_part(abq, bits, dim):
    """So many workgroups that nothing is shared out: each goes over more pages than it holds the numbers of."""
    check(abq, Paged([(33, 4000)] + [(33, 0)] * 63 + [(1, 9000)], 4, 4, dim, 16, bits, seed=dim, extra_rows=1))
    check(abq, Paged([(1, 5000)] + [(1, 3)] * 63, 16, 16, dim if dim > 128 else dim // 4, 16, bits, seed=dim + 1))


@pytest.mark.parametrize("page", [16, 32, 256, 4096])
def test_page_sizes(abq, page):
    check(abq, Paged([(40, 90), (1, 30)], 2, 2, 64, page, seed=page))


def test_rows_that_see_nothing(abq):
    p = Paged([(4, -4), (6, -3), (1, 20)], 4, 2, 64, 16, seed=1)   # no token at all; three tokens for six rows
    y = check(abq, p)
    assert (y[:7] == 0).all() and (y[10] != 0).any()
    p = Paged([(1, 40), (70, 0)], 4, 2, 64, 16, seed=2)
    p.pages[0], p.pages[1, 0] = -1, p.cache[0].shape[0]   # a sequence without a page, and one whose first is missing
    assert (check(abq, p)[:17] == 0).all()
    p.lens[0] = -5
    check(abq, p)


@pytest.mark.parametrize("n", [1, 3, 40])
def test_missing_pages_are_not_seen(abq, n):
    p = Paged([(n, 200)], 4, 2, 64, 16, seed=n)
    p.pages[0, 0], p.pages[0, 3], p.pages[0, 7] = -1, 1 << 30, -(1 << 31)
    check(abq, p)


def test_bounds_that_cut(abq):
    p = Paged([(40, 200), (1, 30)], 4, 2, 64, 16, seed=3)
    check(abq, p, max_len=100)
    check(abq, p, max_len=100, causal=False)
    check(abq, p, max_new=7)
    check(abq, p, max_new=1, max_len=1)
    p.lens[0] = 5000   # more than the table has
    check(abq, p)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 65504.0])
@pytest.mark.parametrize("n", [1, 20, 90])
def test_what_lies_in_masked_places_stays_there(abq, bad, n):
    """The rest of the last page, other pages, and (causal) the values and keys of later tokens."""
    p = Paged([(n, 50), (2, 11)], 4, 2, 64, 16, seed=n)
    clean, _ = p.attention(0.125)
    used = torch.zeros(p.cache[0].shape[0], 16, dtype=torch.bool)
    for s, length in enumerate(p.lens.tolist()):
        for t in range(length):
            used[int(p.pages[s, t // 16]), t % 16] = True
    for t in p.cache:
        t.permute(0, 2, 1, 3)[~used] = bad
    check(abq, p)
    if n > 1:   # the last new token: seen by its own row alone
        last = 50 + n - 1
        page = int(p.pages[0, last // 16])
        p.cache[1][page, :, last % 16, 3] = bad
        y = check(abq, p).cpu().view(p.rows, 4, 64).double()
        assert y[: n - 1].isfinite().all() and (bad == 65504.0 or not y[n - 1, :, 3].isfinite().any())
        assert y[n - 1, :, :3].isfinite().all()
        p.cache[0][page, :, last % 16] = bad
        y = abq.abq_attn_paged(*p.device()[:2], p.q.cuda(), 0.125).cpu().view(p.rows, 4, 64).double()
        want, bound = p.attention(0.125)
        assert ((y - want).abs() <= bound)[: n - 1].all()


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.5, 3.0])
def test_scales(abq, scale):
    """Uniform weights, weights on one token, the other sign."""
    check(abq, Paged([(1, 700), (33, 100)], 4, 2, 64, 16, seed=5), scale=scale)
    check(abq, Paged([(1, 700), (33, 100)], 4, 2, 64, 16, bits=8, seed=5), scale=scale)


def test_scores_that_grow_and_values_of_any_size(abq):
    """Keys that grow along the sequence (the running maximum moves all the way), and values at both ends of binary16."""
    for n in (1, 70):
        p = Paged([(n, 900)], 4, 2, 64, 16, seed=6)
        for t in range(900 + n):
            page, o = int(p.pages[0, t // 16]), t % 16
            p.cache[0][page, :, o] = (p.cache[0][page, :, o].float().abs() * (t / 300)).half()
            p.cache[1][page, :, o] *= 60000.0 / 5 if t % 7 == 0 else 2.0 ** -20
        p.q = p.q.abs()
        check(abq, p)


def test_scales_of_codes_of_any_size(abq):
    for n in (1, 70):
        p = Paged([(n, 300)], 4, 2, 64, 16, bits=8, seed=7)
        for i in (2, 4):
            p.cache[i] *= 2.0 ** torch.randint(-12, 8 if i == 4 else 1, p.cache[i].shape, generator=p.gen)
        check(abq, p)
        p.cache[4] *= 2.0 ** -10
        check(abq, p)


def test_many_sequences(abq):
    p = Paged([(1, i * 7 % 90) for i in range(150)] + [(5, 3)] * 30, 4, 2, 64, 16, seed=8)
    check(abq, p)


def test_offsets_beyond_32_bits(abq):
    pages, heads, page, dim = 70000, 8, 32, 128
    k, v = (torch.zeros(pages, heads, page, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    k[-1], v[-1] = torch.randn(heads, page, dim, device="cuda").half(), torch.randn(heads, page, dim, device="cuda").half()
    q = torch.randn(40, heads * dim, device="cuda").half()
    for n in (1, 20):
        far = abq.abq_attn_paged((k, v), (i32(0, n), i32(30), i32(pages - 1)[None]), q[:n], 0.1)
        near = abq.abq_attn_paged((k[-1:].clone(), v[-1:].clone()), (i32(0, n), i32(30), i32(0)[None]), q[:n], 0.1)
        assert torch.equal(far, near) and (far != 0).any()


def test_same_inputs_give_the_same_bits(abq):
    p = Paged([(1, 3000), (50, 700)], 8, 2, 128, 16, seed=9)
    cache, batch, q = p.device()
    first = abq.abq_attn_paged(cache, batch, q, 0.1)
    for _ in range(3):
        assert torch.equal(abq.abq_attn_paged(cache, batch, q, 0.1), first)


def test_captured_and_replayed(abq):
    """A graph of append and attention replayed on new inputs, with eager work between; and two graphs at once on two streams."""
    p = Paged([(1, 3000), (60, 100)], 8, 2, 128, 16, seed=10)
    cache, batch, q = p.device()
    k, v = p.normal(p.rows, 256).cuda(), p.normal(p.rows, 256).cuda()
    freq = (10000.0 ** (-torch.arange(0, 128, 2).double() / 128)).float().cuda()
    step = lambda: abq.abq_attn_paged(cache, batch, abq.abq_kv_append(cache, batch, k, v, q=q, inv_freq=freq), 0.09, max_len=3100)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=s):
            y = step()
        graphs.append((g, s, y))
    for turn in range(4):
        q.copy_(p.normal(*q.shape)), k.copy_(p.normal(*k.shape)), v.copy_(p.normal(*v.shape))
        want = step()
        torch.cuda.synchronize()
        for g, s, y in graphs:
            y.zero_()
        torch.cuda.synchronize()
        for g, s, y in graphs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for _, _, y in graphs), turn


def test_two_streams(abq):
    ps = [Paged([(1, 2500 + i), (40, 90)], 8, 2, 128, 16, seed=11 + i) for i in range(2)]
    on = [p.device() for p in ps]
    want = [abq.abq_attn_paged(*d, 0.09) for d in on]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in ps], []
    for _ in range(5):
        for s, d in zip(streams, on):
            with torch.cuda.stream(s):
                got.append(abq.abq_attn_paged(*d, 0.09))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))
