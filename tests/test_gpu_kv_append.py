"""abq_kv_append and abq_kv_read against their 64-bit forms: rotation, positions, pages, codes."""
import numpy as np
import pytest
import torch

import oracle
from serving_reference import Paged, rotated, rotated_bound

pytestmark = pytest.mark.gpu


def frequencies(r, base=10000.0):
    return (base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float()


def rows_of(p):
    """(row, sequence, position) of every row that belongs to a sequence."""
    return [(int(p.row_start[s]) + i, s, int(p.lens[s]) - n + i) for s, n in enumerate(p.news) for i in range(n)]


def check(abq, p, r, interleaved=False, with_q=True, strided=False, base=10000.0):
    freq = frequencies(r, base) if r else None
    k, v = p.normal(p.rows, p.heads * p.dim), p.normal(p.rows, p.heads * p.dim)
    cache, batch, q = p.device()
    before = [t.clone() for t in cache]
    if strided:
        wide = torch.cat([p.q, k, v], 1).cuda()
        q, kd, vd = wide.split([p.q.shape[1], k.shape[1], v.shape[1]], 1)
    else:
        kd, vd = k.cuda(), v.cuda()
    q_out = torch.full((p.rows, p.q.shape[1]), 7.0, dtype=torch.float16, device="cuda") if with_q else None
    got = abq.abq_kv_append(cache, batch, kd, vd, q=q if with_q else None, inv_freq=None if freq is None else freq.cuda(), interleaved=interleaved, q_out=q_out)
    assert got is q_out
    torch.cuda.synchronize()
    rows = rows_of(p)
    at = torch.zeros(p.rows, dtype=torch.int64)
    for row, _, pos in rows:
        at[row] = pos
    turn = lambda x: rotated(x.view(p.rows, -1, p.dim), at, freq if r else torch.zeros(0), interleaved)
    owned = torch.zeros(p.rows, dtype=torch.bool)
    owned[[row for row, _, _ in rows]] = True
    if with_q:
        want, size = turn(p.q)
        off = (got.cpu().view(want.shape).double() - want).abs()
        assert (off <= rotated_bound(want, size))[owned].all(), off[owned].max()
        if r < p.dim:
            assert torch.equal(got.cpu().view(want.shape)[owned][..., r:], p.q.view(want.shape)[owned][..., r:])
        assert (got.cpu()[~owned] == 7.0).all()
    want, size = turn(k)
    after = [t.cpu() for t in cache]
    expect = [t.cpu().clone() for t in before]
    for row, s, pos in rows:
        page = int(p.pages[s, pos // p.page]) if 0 <= pos < p.page * p.pages.shape[1] else -1
        if not 0 <= page < after[0].shape[0]:
            continue
        o = pos % p.page
        if p.bits == 16:
            assert ((after[0][page, :, o].double() - want[row]).abs() <= rotated_bound(want[row], size[row])).all()
            expect[0][page, :, o] = after[0][page, :, o]
            expect[1][page, :, o] = v[row].view(p.heads, p.dim)
        else:
            codes, scale, zero = oracle.quant_act(v[row].view(p.heads, p.dim).numpy(), 8)
            expect[1][page, :, o], expect[4][page, :, o], expect[5][page, :, o] = torch.from_numpy(codes), torch.from_numpy(scale), torch.from_numpy(zero).to(torch.uint8)
            # the keys: what they stand for is within half a step of the codes of the rotated vector (and its own rounding)
            step = after[2][page, :, o].double()[:, None]
            value = (after[0][page, :, o].double() - after[3][page, :, o].double()[:, None]) * step
            assert ((value - want[row]).abs() <= step * 0.501 + 2 * rotated_bound(want[row], size[row])).all()
            for i in (0, 2, 3):
                expect[i][page, :, o] = after[i][page, :, o]
    for e, a in zip(expect, after):   # and nothing else has changed
        assert torch.equal(e.view(torch.uint8), a.view(torch.uint8))
    return cache


HEADS = [(32, 8), (4, 4), (3, 1)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim,r", [(128, 128), (64, 64), (80, 80), (256, 64), (96, 0), (16, 16), (112, 32)])
def test_rows_go_to_their_places(abq, bits, dim, r):
    for i, (hq, h) in enumerate(HEADS):
        p = Paged([(1, 0), (5, 30), (17, 0), (1, 100), (0, 12)], hq, h, dim, 16, bits, seed=dim + r + i, extra_rows=3)
        check(abq, p, r, interleaved=i == 1, with_q=i != 2, strided=i == 0)


def test_one_row(abq):
    check(abq, Paged([(1, 0)], 1, 1, 128, 16, seed=3), 128)


def test_prompt_over_many_pages_and_sequences(abq):
    check(abq, Paged([(700, 3), (1, 4000), (33, 0)] + [(1, i) for i in range(80)], 8, 2, 128, 64, seed=4), 128)
    check(abq, Paged([(300, 3)], 8, 2, 64, 4096, bits=8, seed=5), 64)


def test_codes_are_the_quantizers_of_the_binary16_vector(abq):
    """The same rows into both kinds of cache: the codes are those of the vectors that the binary16 cache holds, to the bit."""
    a, b = (Paged([(40, 9), (3, 77)], 4, 4, 128, 16, bits, seed=6) for bits in (16, 8))
    b.q, b.gen = a.q, a.gen
    k, v = (a.normal(a.rows, 512).cuda() for _ in range(2))
    freq = frequencies(128).cuda()
    (ca, ba, _), (cb, bb, _) = a.device(), b.device()
    bb = (bb[0], bb[1], ba[2])
    v[5] = 0
    abq.abq_kv_append(ca, ba, k, v, inv_freq=freq)
    abq.abq_kv_append(cb, bb, k, v, inv_freq=freq)
    for row, s, pos in rows_of(a):
        page, o = int(a.pages[s, pos // 16]), pos % 16
        for which in (0, 1):
            codes, scale, zero = oracle.quant_act(ca[which][page, :, o].cpu().numpy(), 8)
            assert np.array_equal(cb[which][page, :, o].cpu().numpy(), codes)
            scale[(codes == zero[:, None]).all(1)] = 2.0 ** -32   # zeros
            assert np.array_equal(cb[2 + 2 * which][page, :, o].cpu().numpy(), scale) and np.array_equal(cb[3 + 2 * which][page, :, o].cpu().numpy(), zero)


def test_far_positions(abq):
    """Angles at positions where binary32 would have lost them; the tokens before are on pages that are not there."""
    for past in (131071, 1 << 20, (1 << 24) + 1, 2000000001):
        p = Paged([(2, 30)], 2, 1, 64, 4096, seed=past % 97)
        p.lens[0] = past + 2
        k = p.normal(2, 64)
        freq = frequencies(64)
        cache, batch, q = p.device()
        got = abq.abq_kv_append(cache, batch, k.cuda(), k.cuda(), q=q, inv_freq=freq.cuda()).cpu().view(2, 2, 64).double()
        want, size = rotated(p.q.view(2, 2, 64), torch.tensor([past, past + 1]), freq)
        assert ((got - want).abs() <= rotated_bound(want, size)).all()
        assert torch.equal(cache[0].cpu(), p.cache[0])   # (no page there)


def test_bad_pages_and_positions_are_skipped(abq):
    p = Paged([(20, 5), (8, -5), (4, 40)], 4, 2, 64, 16, seed=8)   # the second has fewer tokens than rows
    p.pages[0, 1] = -1
    p.pages[2, 2] = p.cache[0].shape[0]
    check(abq, p, 64)
    p = Paged([(20, 5), (4, 40)], 4, 2, 64, 16, bits=8, seed=9)
    p.pages[0, 0], p.pages[1, 2] = 1 << 30, -(1 << 31)
    check(abq, p, 64)
    p = Paged([(4, 12)], 4, 2, 64, 16, seed=10)
    p.lens[0] = 1000   # positions beyond the table
    check(abq, p, 64)


def test_queries_in_place(abq):
    p = Paged([(9, 50)], 4, 2, 128, 16, seed=11)
    k, freq = p.normal(9, 256).cuda(), frequencies(128).cuda()
    cache, batch, q = p.device()
    want = abq.abq_kv_append(cache, batch, k, k, q=q, inv_freq=freq)
    assert abq.abq_kv_append(cache, batch, k, k, q=q, inv_freq=freq, q_out=q) is q
    assert torch.equal(q, want)


@pytest.mark.parametrize("bits", [16, 8])
def test_read_back(abq, bits):
    p = Paged([(3, 100)], 4, 4, 80, 32, bits, seed=12)
    cache, _, _ = p.device()
    slots = torch.tensor([0, 5, 33, 96, 127, -1, p.cache[0].shape[0] * 32, 1 << 30, -(1 << 31), 33], dtype=torch.int32)
    k, v = abq.abq_kv_read(cache, slots.cuda())
    for i, s in enumerate(slots.tolist()):
        for which, got in ((0, k), (1, v)):
            want = torch.zeros(4, 80, dtype=torch.float16)
            if 0 <= s < p.cache[0].shape[0] * 32:
                x = p.cache[which][s // 32, :, s % 32]
                want = x if bits == 16 else ((x.float() - p.cache[3 + 2 * which][s // 32, :, s % 32].float()[:, None]) * p.cache[2 + 2 * which][s // 32, :, s % 32][:, None]).half()
            assert torch.equal(got[i].cpu().view(4, 80), want)


def test_offsets_beyond_32_bits(abq):
    """The last page of a cache of more than 2^31 elements."""
    pages, heads, page, dim = 70000, 8, 32, 128
    k, v = (torch.zeros(pages, heads, page, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    new = torch.randn(1, heads * dim, device="cuda").half()
    abq.abq_kv_append((k, v), (i32(0, 1), i32(32), i32(pages - 1)[None]), new, 2 * new)
    assert torch.equal(k[-1, :, 31].flatten(), new[0]) and torch.equal(v[-1, :, 31].flatten(), 2 * new[0])
    kr, vr = abq.abq_kv_read((k, v), i32(pages * page - 1))
    assert torch.equal(kr, new) and torch.equal(vr, 2 * new)
    assert int(k.count_nonzero()) == int(new.count_nonzero())


def test_sine_and_cosine_of_far_positions(abq):
    """Each within 2^-23 of the exact angle's, up to the last position: pairs of (1, 0) come out as them, after one rounding to binary16.  The
    exact angle is reduced in whole numbers of 2^-180 by pi / 2; sine and cosine of what is left are off by 2^-52."""
    half_pi = 2407238366421696601854996748563021104914972029442149625   # pi / 2 in those
    g = torch.Generator().manual_seed(5)
    rows = 2000
    at = torch.randint(1 << 30, (1 << 31) - 2, (rows,), generator=g)
    at[:4] = torch.tensor([(1 << 31) - 2, (1 << 31) - 3, 1 << 30, 5])
    freq = 1.0 - torch.rand(32, generator=g) / 8
    freq[0], freq[1] = 1.0, 0.5
    x = torch.cat([torch.ones(rows, 32), torch.zeros(rows, 32)], 1).half().cuda()
    cache = tuple(torch.zeros(1, 1, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    batch = (torch.arange(rows + 1, dtype=torch.int32).cuda(), (at + 1).to(torch.int32).cuda(), torch.full((rows, 1), -1, dtype=torch.int32).cuda())
    y = abq.abq_kv_append(cache, batch, x, x, q=x, inv_freq=freq.cuda()).cpu().double()
    mant = [int(f * 2.0 ** 40) for f in freq.double()]
    rest = np.empty((rows, 32, 2))
    for i, p in enumerate(at.tolist()):
        for j, m in enumerate(mant):
            a = p * m << 140
            turns = (a + half_pi // 2) // half_pi
            rest[i, j] = (a - turns * half_pi) / 2 ** 180, turns % 4
    sine, cosine, quadrant = np.sin(rest[..., 0]), np.cos(rest[..., 0]), rest[..., 1]
    want = [np.select([quadrant == i for i in range(4)], c) for c in ((cosine, -sine, -cosine, sine), (sine, cosine, -sine, -cosine))]
    want = torch.from_numpy(np.concatenate(want, 1))
    assert ((y - want).abs() <= 2.0 ** -23 + 2.0 ** -11 * want.abs() + 2.0 ** -25).all()
