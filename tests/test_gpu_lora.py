"""abq_lora_add against its 64-bit form."""
import pytest
import torch

from serving_reference import adapted

pytestmark = pytest.mark.gpu


def make(M, N, K, rank, adapters, seed=0, ids=None):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g)
    x, y = normal(M, K).half(), normal(M, N).half()
    a, b = (normal(adapters, rank, K) / K ** 0.5).half(), (normal(adapters, N, rank) / rank ** 0.5).half()
    if ids is None:
        ids = torch.randint(-1, adapters, (M,), generator=g)
    return [x, ids.to(torch.int32), a, b, torch.rand(adapters, generator=g) * 2 - 0.5, y]


def check(abq, t, **kw):
    got = abq.abq_lora_add(*(v.cuda() for v in t), **kw).cpu()
    want, bound = adapted(*t)
    off = (got.double() - want).abs()
    assert (off <= bound).all(), f"{int((off > bound).sum())} of {off.numel()}, rows {sorted(set((off > bound).nonzero()[:, 0].tolist()))[:8]}"
    return got


@pytest.mark.parametrize("rank", [1, 4, 8, 16, 24, 32, 64, 100, 128, 256])
def test_ranks(abq, rank):
    for M in (1, 21):
        check(abq, make(M, 200, 264, rank, 5, seed=rank))


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 130, 300])
def test_rows(abq, M):
    check(abq, make(M, 136, 512, 16, 7, seed=M))
    check(abq, make(M, 136, 512, 16, 3, seed=M, ids=torch.arange(M) * 3 // M))


@pytest.mark.parametrize("N,K", [(1, 1), (7, 3), (15, 513), (17, 100), (1003, 33), (64, 4091), (129, 31), (4096, 8), (16, 11008), (301, 4096)])
def test_sizes_that_divide_nothing(abq, N, K):
    check(abq, make(5, N, K, 8, 3, seed=N))
    check(abq, make(40, N, K, 20, 3, seed=K))


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 100, 128, 136, 256])
@pytest.mark.parametrize("M,adapters", [(1, 3), (20, 9), (270, 3), (333, 40)])
def test_whole_blocks_of_columns(abq, rank, M, adapters):
    """Columns in whole blocks of 64, for few and many rows, with the adapters in any order; and runs of rows."""
    check(abq, make(M, 192, 160, rank, adapters, seed=rank + M))
    if M > 100:
        check(abq, make(M, 320, 1056, rank, adapters, seed=rank, ids=torch.arange(M) * adapters // M - 1))


def test_many_rows_and_columns(abq):
    check(abq, make(1100, 2048, 300, 16, 5, seed=1, ids=torch.arange(1100) * 5 // 1100))
    check(abq, make(700, 4100, 64, 8, 3, seed=2))


def test_every_row_its_own_adapter_and_all_rows_one(abq):
    check(abq, make(50, 96, 256, 16, 50, ids=torch.randperm(50)))
    check(abq, make(50, 96, 256, 16, 50, ids=torch.full((50,), 49)))


def test_rows_without_an_adapter_are_copied(abq):
    ids = torch.tensor([-1, 3, 0, 1 << 30, -(1 << 31), 2, 3])
    t = make(7, 77, 64, 8, 3, ids=ids)
    t[5][0, 5], t[5][1, 6], t[5][3, 7] = float("nan"), float("inf"), -0.0
    got = abq.abq_lora_add(*(v.cuda() for v in t)).cpu()
    for m in (0, 1, 3, 4, 6):
        assert torch.equal(got[m].view(torch.int16), t[5][m].view(torch.int16))
    t = make(20, 77, 64, 8, 3, ids=torch.full((20,), -1))
    assert torch.equal(check(abq, t), t[5])


def test_other_rows_do_not_matter(abq):
    """Infinities and NaN in one adapter, in another row's input: a row with others comes out as it does alone, to the bit."""
    t = make(40, 200, 512, 16, 6, seed=3)
    t[1] = torch.arange(40, dtype=torch.int32) % 6
    want = abq.abq_lora_add(*(v.cuda() for v in t)).cpu()
    bad = [v.clone() for v in t]
    bad[2][2], bad[3][4, 50:] = float("nan"), float("inf")
    bad[0][7] = float("inf")
    got = abq.abq_lora_add(*(v.cuda() for v in bad)).cpu()
    rows = torch.tensor([m for m in range(40) if m % 6 not in (2, 4) and m != 7])
    assert torch.equal(got[rows], want[rows])
    assert torch.equal(got[4::6, :50], want[4::6, :50])


def test_in_place_and_strided(abq):
    t = make(33, 96, 128, 16, 4, seed=4)
    want, bound = adapted(*t)
    wide = torch.full((33, 300), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 104:200] = t[5].cuda()
    x = torch.cat([t[0], t[0]], 1).cuda()[:, 128:]
    y = wide[:, 104:200]
    d = [v.cuda() for v in t]
    assert abq.abq_lora_add(x, *d[1:5], y, out=y) is y
    assert ((y.cpu().double() - want).abs() <= bound).all()
    assert (wide[:, :104] == 7).all() and (wide[:, 200:] == 7).all()
    odd = torch.zeros(33, 101, dtype=torch.float16, device="cuda")   # rows off 16-byte boundaries
    odd[:, :96] = d[5]
    x = torch.zeros(33, 131, dtype=torch.float16, device="cuda")
    x[:, :128] = d[0]
    got = abq.abq_lora_add(x[:, :128], *d[1:5], odd[:, :96], out=odd[:, :96])
    assert ((got.cpu().double() - want).abs() <= bound).all() and (odd[:, 96:] == 0).all()


def test_large_and_small_inner_products(abq):
    """A x beyond binary16's range and far below it: only the result has to fit."""
    t = make(6, 64, 4096, 16, 2, seed=5)
    t[2] *= 1000.0
    t[2] = t[2].abs()
    t[0] = t[0].abs() * 50
    t[3] *= 2.0 ** -14
    check(abq, t)
    t = make(6, 64, 256, 16, 2, seed=6)
    t[2] *= 2.0 ** -12
    t[0] *= 2.0 ** -10
    t[5] *= 2.0 ** -20
    check(abq, t)


def test_same_inputs_same_bits_and_replays(abq):
    t = [v.cuda() for v in make(70, 1000, 2048, 16, 9, seed=7)]
    want = abq.abq_lora_add(*t)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = abq.abq_lora_add(*t)
    for i in range(4):
        t[0].mul_(-1.0)
        want = abq.abq_lora_add(*t)
        y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("M,N,K,rank", [(300, 192, 160, 16), (300, 200, 161, 24), (290, 128, 264, 100), (290, 136, 264, 128), (270, 192, 96, 200), (700, 1000, 96, 8)])
def test_in_place_and_strided_many_rows(abq, M, N, K, rank):
    """The shapes of many rows (tiles of 64, 32 and 16), in place and on rows off 16-byte boundaries."""
    t = make(M, N, K, rank, 5, seed=M + rank)
    d = [v.cuda() for v in t]
    want = check(abq, t).cuda()
    x = torch.zeros(M, K + 9, dtype=torch.float16, device="cuda")
    x[:, :K] = d[0]
    wide = torch.full((M, N + 13), 7.0, dtype=torch.float16, device="cuda")
    wide[:, 8:8 + N] = d[5]
    y = wide[:, 8:8 + N]
    assert abq.abq_lora_add(x[:, :K], *d[1:5], y, out=y) is y
    assert torch.equal(y, want) and (wide[:, :8] == 7).all() and (wide[:, 8 + N:] == 7).all()
    assert abq.abq_lora_add(*d, out=d[5]) is d[5]
    assert torch.equal(d[5], want)


@pytest.mark.parametrize("M,rank", [(300, 16), (300, 64), (290, 128), (270, 200), (1100, 8)])
def test_other_rows_do_not_matter_many_rows(abq, M, rank):
    t = make(M, 192, 200, rank, 6, seed=rank)
    t[1] = torch.randperm(M, generator=torch.Generator().manual_seed(M)).to(torch.int32) % 7 - 1
    want = abq.abq_lora_add(*(v.cuda() for v in t)).cpu()
    bad = [v.clone() for v in t]
    bad[2][2], bad[3][4, 50:], bad[4][1] = float("nan"), float("inf"), float("nan")
    bad[0][7] = float("inf")
    got = abq.abq_lora_add(*(v.cuda() for v in bad)).cpu()
    rows = torch.tensor([m for m in range(M) if int(t[1][m]) not in (1, 2, 4) and m != 7])
    assert torch.equal(got[rows].view(torch.int16), want[rows].view(torch.int16))
    four = torch.tensor([m for m in range(M) if int(t[1][m]) == 4 and m != 7])
    assert torch.equal(got[four][:, :50], want[four][:, :50])


@pytest.mark.parametrize("N", [8256, 8250])
@pytest.mark.parametrize("rank", [8, 20, 64])
def test_two_blocks_a_wave(abq, N, rank):
    """Rows and columns enough for two blocks of columns a wave, the last waves with one or none; adapters in runs and in any order."""
    for ids in (None, torch.arange(2048) * 5 // 2048 - 1):
        t = make(2048, N, 64, rank, 4, seed=N + rank, ids=ids)
        d = [v.cuda() for v in t]
        got = abq.abq_lora_add(*d)
        u = torch.zeros(2048, N, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(u)
        for i in range(4):
            at = (d[1] == i).nonzero()[:, 0]
            A, B, s = d[2][i].double(), d[3][i].double(), float(d[4][i])
            x = d[0][at].double()
            a = x @ A.T.contiguous()
            u[at] = s * (a @ B.T.contiguous())
            off = (64 + 2) * 2.0 ** -24 * (x.abs() @ A.abs().T.contiguous()) + 2.0 ** -21 * a.abs().amax(1, keepdim=True)
            size[at] = abs(s) * ((off + (rank + 4) * 2.0 ** -24 * a.abs()) @ B.abs().T.contiguous())
        want = d[5].double() + u
        bound = size + 2.0 ** -23 * want.abs()
        bound = bound + 2.0 ** -11 * (want.abs() + bound) + 2.0 ** -25
        assert ((got.double() - want).abs() <= bound).all()
        none = d[1] < 0
        assert torch.equal(got[none], d[5][none])
        assert abq.abq_lora_add(*d, out=d[5]) is d[5]
        assert torch.equal(d[5], got)
