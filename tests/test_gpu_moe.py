"""A layer of experts on the GPU against its 64-bit form: router, products with the experts' weights, weighted sum, and all of it in a run."""
import pytest
import torch

from moe_reference import INF, combined, gemm, groups, routed

pytestmark = pytest.mark.gpu


# ---- router ----------------------------------------------------------------------------------------
def check_route(abq, logits, top, **kw):
    on = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    got = [t.cpu() for t in abq.abq_moe_route(logits.cuda(), top, **on)]
    want = routed(logits, top, **kw)
    for name, g, w in zip(("ids", "starts", "order", "places"), (got[0], got[2], got[3], got[4]), (want[0], want[2], want[3], want[4])):
        assert torch.equal(g.long(), w), f"{name}: {int((g.long() != w).sum())} of {g.numel()} differ"
    off = (got[1].double() - want[1]).abs()
    assert (off <= want[5]).all(), f"weights: off by {float((off / want[5]).nan_to_num().max()):.2f} bounds"
    return got


def some_logits(T, E, half, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, E, generator=g) * 2
    return x.half() if half else x


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("E", [1, 2, 7, 8, 16, 17, 33, 60, 64, 100, 128, 160, 256, 257, 512, 513, 1000, 1024])
def test_experts(abq, E, half):
    g = torch.Generator().manual_seed(E)
    for T in (1, 37):
        x = some_logits(T, E, half, E + T)
        for top in sorted({1, min(E, 3), min(E, 8), min(E, 16)}):
            check_route(abq, x, top)
        check_route(abq, x, min(E, 5), bias=torch.rand(E, generator=g) - 0.5, sigmoid=True, scale=2.5)
        check_route(abq, x, min(E, 5), bias=(torch.rand(E, generator=g) - 0.5) * 0.1)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 63, 64, 65, 255, 256, 257, 300, 1000, 4099, 16385])
def test_tokens(abq, T):
    """One launch and two, chunks of 64 and more, whole and with a rest."""
    check_route(abq, some_logits(T, 16, T % 2 == 0, T), 2)
    if T < 5000:
        check_route(abq, some_logits(T, 130, T % 2 == 1, T), 7, renormalize=False)


@pytest.mark.parametrize("T,E,top", [(512, 16, 16), (513, 16, 16), (512, 1, 1), (513, 1, 1), (64, 128, 16), (65, 128, 16), (32, 256, 16), (33, 256, 16), (8, 1024, 16), (9, 1024, 16), (31, 257, 16), (128, 16, 8), (129, 16, 8), (64, 60, 16), (436, 8, 6), (700, 8, 2), (2000, 4, 4)])
def test_at_the_border_of_one_launch(abq, T, E, top):
    for half in (True, False):
        check_route(abq, some_logits(T, E, half, T), top)
    check_route(abq, some_logits(T, E, False, T + 1), top, bias=torch.linspace(-0.2, 0.2, E), sigmoid=True)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("half", [False, True])
def test_scores(abq, sigmoid, renormalize, biased, half):
    x = some_logits(70, 48, half, 5)
    x[3], x[4], x[5, ::2] = x[3] * 20, x[4] - 200, x[5, ::2] - 60000   # sharp rows; rows whose sigmoids underflow
    bias = torch.rand(48, generator=torch.Generator().manual_seed(1)) - 0.5 if biased else None
    check_route(abq, x, 6, bias=bias, sigmoid=sigmoid, renormalize=renormalize, scale=1.75)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("kw", [{}, dict(sigmoid=True), dict(sigmoid=True, bias=torch.zeros(64)), dict(bias=torch.zeros(64))])
def test_ties_go_to_the_lowest_expert(abq, half, kw):
    x = torch.randint(-2, 3, (300, 64), generator=torch.Generator().manual_seed(3)).float()
    x[7], x[8, ::2] = 0.0, -0.0
    x[9] = -0.0
    check_route(abq, x.half() if half else x, 8, **kw)


@pytest.mark.parametrize("T", [40, 500])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("kw", [{}, dict(renormalize=False), dict(sigmoid=True, bias=torch.linspace(-0.3, 0.3, 24)), dict(bias=torch.linspace(-0.3, 0.3, 24), renormalize=False)])
def test_experts_that_are_not_there(abq, T, half, kw):
    """Padding rows, rows with fewer experts than choices, NaN among the logits; the lowest value of the type is a value."""
    x = some_logits(T, 24, half, 9)
    x[::5] = -INF
    x[1, 2:], x[2, 1:], x[3, :20] = -INF, -INF, -INF
    x[4, ::3] = float("nan")
    x[6] = float("nan")
    x[7, :] = torch.finfo(x.dtype).min
    x[8, 3:] = torch.finfo(x.dtype).min
    got = check_route(abq, x, 4, **kw)
    assert int((got[0][0] == -1).sum()) == 4 and (got[1][0] == 0).all() and int((got[0][2] >= 0).sum()) == 1
    check_route(abq, torch.full((T, 24), -INF, dtype=x.dtype), 3, **kw)


@pytest.mark.parametrize("half", [False, True])
def test_logits_at_the_ends_of_their_type(abq, half):
    """The smallest values beside zeros of both signs, the largest of both signs: all different, or ties."""
    t = torch.float16 if half else torch.float32
    f = torch.finfo(t)
    values = [0.0, -0.0, f.smallest_normal, -f.smallest_normal, f.max, f.min, 1.0, -1.0, 1 + f.eps, -1 - f.eps] + [k * f.smallest_normal * f.eps for k in (1, 2, 3, -1, -2, -3)]
    g = torch.Generator().manual_seed(2)
    x = torch.tensor(values, dtype=torch.float64)[torch.randint(0, len(values), (200, 40), generator=g)].to(t)
    assert ((x != 0) & (x.abs() < f.smallest_normal)).any()
    got = check_route(abq, x, 8)
    assert (got[0] >= 0).all()
    x[:, 7] = INF   # the choice; what becomes of the weights is not said
    ids = abq.abq_moe_route(x.cuda(), 3)[0].cpu()
    assert (ids[:, 0] == 7).all() and torch.equal(ids[:, 1:].long(), routed(torch.cat([x[:, :7], x[:, 8:]], 1), 2)[0] + (routed(torch.cat([x[:, :7], x[:, 8:]], 1), 2)[0] >= 7).long())


def test_a_bias_takes_experts_out(abq):
    bias = torch.zeros(12)
    bias[::2] = -INF
    got = check_route(abq, some_logits(50, 12, True), 3, bias=bias, sigmoid=True)
    assert (got[0] % 2 == 1).all()


def test_strides_and_given_outputs(abq):
    wide = torch.randn(90, 77, generator=torch.Generator().manual_seed(1)).cuda()
    for x in (wide[:, :33], wide.half()[:, 40:73]):
        if x.data_ptr() % 16:
            x = x.clone()
        want = abq.abq_moe_route(x.contiguous(), 4)
        out = tuple(torch.full_like(t, -7) for t in want)
        assert abq.abq_moe_route(x, 4, out=out) is out
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("experts,top,most", [(128, 8, 16385), (16, 2, 8704), (640, 4, 9000)])
def test_one_workspace_of_the_largest_batch(abq, experts, top, most):
    """It serves every smaller batch, and nothing behind its end is written."""
    need = abq.abq_moe_route_workspace_bytes(most, experts, top)
    around = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    x = torch.randn(most, experts, generator=torch.Generator().manual_seed(top)).half().cuda()
    for T in (most, 8192, 8193, 700, 5, 4097):
        want = abq.abq_moe_route(x[:T], top)
        got = abq.abq_moe_route(x[:T], top, workspace=around[:need])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f"{T} tokens"
        assert (around[need:] == 0x5A).all()


def test_every_token_to_the_same_experts(abq):
    x = torch.zeros(3000, 32)
    x[:, 5], x[:, 30] = 2.0, 1.0
    got = check_route(abq, x, 2)
    assert got[2].tolist() == [0] * 6 + [3000] * 25 + [6000] * 2


# ---- products --------------------------------------------------------------------------------------
def layer(p, q, E, N, K, T, seed=0):
    g = torch.Generator().manual_seed(seed)
    u = lambda *s: torch.rand(s, generator=g)
    i = lambda top, *s: torch.randint(0, top, s, generator=g)
    return {"a": (i(256, T, K).to(torch.uint8), (u(T) + 0.5) * (4.0 / 2**q), i(2**q, T).to(torch.int32)),   # (bits above q are dropped)
            "w": (i(2**p, E, N, K).to(torch.uint8), (u(E, N) + 0.5) * (2.0 / (K**0.5 * 2**p)), i(2**p, E, N).to(torch.int32))}


POISON = 0x7E2A   # (a NaN's bits)


def check_gemm(abq, p, q, counts, N, K, top=0, T=0, seed=0, behind=0, layout=0):
    """counts: rows of each expert; top 0: without order.  Every bit of every row, and the rows behind the last one as they were."""
    used = sum(counts)
    rows, E = used + behind, len(counts)
    g = torch.Generator().manual_seed(seed + 1)
    if top:
        T = T or -(-rows // top)
        order = torch.cat([torch.randint(0, T * top, (used,), generator=g), torch.full((behind,), -1)]).to(torch.int32)
    else:
        T, order = rows, None
    s = layer(p, q, E, N, K, T, seed)
    starts = groups(counts)
    w = abq.abq_pack_experts(p, *(t.cuda() for t in s["w"]), layout=layout)
    y = torch.full((rows, N), POISON, dtype=torch.int16, device="cuda").view(torch.float16)
    abq.abq_moe_gemm(p, q, N, *(t.cuda() for t in s["a"]), w, starts.cuda(), order=None if order is None else order.cuda(), top=max(top, 1), w_layout=layout, y=y)
    got, want = y.cpu().view(torch.int16), gemm(*s["a"], *s["w"], p, q, starts, order, max(top, 1), rows)
    want = torch.where(torch.arange(rows)[:, None] < used, want.view(torch.int16), torch.tensor(POISON, dtype=torch.int16))
    bad = (got != want).nonzero()
    assert not len(bad), f"{len(bad)} of {got.numel()} differ, rows {sorted(set(bad[:, 0].tolist()))[:8]}, columns {sorted(set(bad[:, 1].tolist()))[:8]}"


@pytest.mark.parametrize("q", [1, 4, 7, 8])
@pytest.mark.parametrize("p", range(1, 9))
def test_widths(abq, p, q):
    """Every weight width on every kernel: few rows (one and two tiles of rows, one to four super-chunks a wave), 64, 128 and 256 rows a workgroup."""
    check_gemm(abq, p, q, [1, 0, 5, 16, 2], 80, 1024, top=2, seed=p)
    check_gemm(abq, p, q, [1, 0, 5, 16, 2], 48, 8704, seed=p)
    check_gemm(abq, p, q, [3, 1], 32, 14336, top=2, seed=p)
    check_gemm(abq, p, q, [20, 32, 17], 96, 512, top=3, seed=p)
    check_gemm(abq, p, q, [20, 32, 17], 64, 6656, seed=p)
    check_gemm(abq, p, q, [70, 33, 64, 0], 144, 640, top=2, seed=p)
    check_gemm(abq, p, q, [140, 0, 128, 97], 272, 512, seed=p)
    check_gemm(abq, p, q, [300, 256], 528, 1024, top=2, seed=p)


@pytest.mark.parametrize("q", [3, 8])
@pytest.mark.parametrize("p", range(1, 9))
def test_widths_of_64_rows(abq, p, q):
    """Enough channels for tiles of 64 rows: whole and ragged ones, with and without order."""
    check_gemm(abq, p, q, [70, 33, 64, 0, 1], 4400 + 8 * p, 640, top=2, seed=p, behind=4)
    check_gemm(abq, p, q, [20, 32, 17], 8193, 130, seed=p)
    check_gemm(abq, p, q, [65] + [16] * 40, 523, 257, top=3, seed=p)


@pytest.mark.parametrize("K", [1, 7, 15, 16, 17, 31, 63, 64, 65, 100, 127, 500, 511, 512, 513, 1000, 1408, 2047, 4095, 5121, 8193, 12289, 16383])
@pytest.mark.parametrize("top", [0, 3])
def test_lengths_that_divide_nothing(abq, K, top):
    for p, q in ((4, 8), (3, 5), (8, 8)):
        check_gemm(abq, p, q, [2, 0, 1, 9], 40, K, top=top, seed=K)
        check_gemm(abq, p, q, [40, 60], 40, K, top=top, seed=K)
    check_gemm(abq, 4, 8, [1], 16, K, top=top)


@pytest.mark.parametrize("T,K", [(1, 16), (1, 79), (1, 65), (1, 127), (1, 143), (1, 527), (1, 4111), (2, 79), (3, 1039)])
def test_codes_that_end_with_their_allocation(abq, T, K):
    """The last slice of the last row, also where it is the only row's and less than sixteen codes are left for it: the vectors that hold it are moved back
    into the tensor, which ends with a 32 MiB allocation but for its alignment."""
    s = layer(4, 8, 2, 40, K, T, K)
    w = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    whole = torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")
    at = (len(whole) - T * K) // 16 * 16
    codes = whole[at:at + T * K].view(T, K)
    codes.copy_(s["a"][0])
    starts = groups([T - 1, 1])
    y = abq.abq_moe_gemm(4, 8, 40, codes, s["a"][1].cuda(), s["a"][2].cuda(), w, starts.cuda())
    assert torch.equal(y.cpu().view(torch.int16), gemm(*s["a"], *s["w"], 4, 8, starts, None, 1, T).view(torch.int16))


@pytest.mark.parametrize("N", [1, 2, 7, 15, 16, 17, 33, 127, 129, 255, 257, 1003])
def test_columns_that_divide_nothing(abq, N):
    for counts in ([1], [3, 0, 12], [40, 25], [100, 150], [500, 230]):
        check_gemm(abq, 4, 8, counts, N, 320, top=2, seed=N)
        check_gemm(abq, 6, 6, counts, N, 200, seed=N, behind=3)
    for counts in ([40, 25, 0, 60], [100] * 3):   # (wide enough for blocks)
        check_gemm(abq, 4, 8, counts, 6144 + N, 320, top=2, seed=N)


@pytest.mark.parametrize("counts", [[0, 0, 0, 5], [5, 0, 0, 0], [0] * 70 + [3] + [0] * 60 + [1, 2], [1] * 64, [1] * 65, [17] + [1] * 40, [100] + [1] * 12, [1000] + [0] * 40 + [1] * 3,
                                    [1] * 300, [0] * 1023 + [4], [2] * 1024, [16] * 9, [65, 0, 64, 63], [128, 129, 1], [257, 255, 0, 256], [600] + [0] * 100 + [8]])
def test_ragged_groups(abq, counts):
    check_gemm(abq, 4, 8, counts, 48, 192, top=2, seed=len(counts), behind=5)
    check_gemm(abq, 2, 8, counts, 272 if len(counts) < 200 else 16, 64, seed=len(counts))


@pytest.mark.parametrize("p", range(1, 9))
def test_heights_of_the_last_block(abq, p):
    """Enough tiles for 256 rows each: last blocks of an expert with every height of tile, at its borders and inside."""
    counts = [129, 1, 256, 192, 0, 193, 128, 64, 257, 384, 385, 255, 448, 449, 0, 512, 17, 320, 130, 200, 100, 191, 250, 127]
    check_gemm(abq, p, 8, counts, 2048 + 8 * p, 130, top=2, seed=p, behind=7)
    check_gemm(abq, p, 5, counts[::-1], 1031 + 1024, 700, seed=p)
    check_gemm(abq, p, 8, [97, 96, 128, 129, 0, 225, 1, 95, 224, 90], 4099, 640, top=2, seed=p, behind=3)   # (128 rows a tile, and 96)


@pytest.mark.parametrize("p", [2, 3, 4, 7, 8])
@pytest.mark.parametrize("K", [64, 128, 192, 256, 400, 512, 640, 768])
def test_k_that_ends_inside_a_super_chunk(abq, p, K):
    """Every number of steps modulo the super-chunk's four, on every height of tile."""
    check_gemm(abq, p, 8, [1, 33, 64, 40], 144, K, top=2, seed=K)
    check_gemm(abq, p, 8, [1, 33, 64, 40], 4400, K, top=2, seed=K)
    if K % 256 == 0 or p in (2, 7):
        check_gemm(abq, p, 8, [140, 128, 150], 11008, K, seed=K)
        check_gemm(abq, p, 8, [300, 128, 180, 200], 11008, K, top=2, seed=K)


def test_no_rows_at_all(abq):
    check_gemm(abq, 4, 8, [0] * 8, 64, 256, top=2, behind=16)
    check_gemm(abq, 4, 8, [0] * 8, 64, 256, top=2, behind=700)


@pytest.mark.parametrize("p,E,N,K", [(1, 3, 17, 65), (3, 1, 16, 512), (4, 5, 33, 1001), (6, 2, 1, 1), (7, 4, 100, 640), (8, 70, 40, 300)])
def test_packed_together_as_one_by_one(abq, p, E, N, K):
    w = [t.cuda() for t in layer(p, 8, E, N, K, 1, seed=p)["w"]]
    for layout in (0, abq.ABQ_LAYOUT_PLANES, abq.ABQ_LAYOUT_BOTH):
        got = abq.abq_pack_experts(p, *w, layout=layout, out=torch.zeros((E, abq.abq_packed_weight_bytes(p, N, K, layout)), dtype=torch.uint8, device="cuda"))
        for e in range(E):
            one = torch.zeros_like(got[e])
            abq.abq_pack_weights(p, *(t[e].clone() for t in w), layout=layout, out=one)
            assert torch.equal(got[e], one), f"expert {e}"


def test_blobs_that_hold_planes_too(abq):
    check_gemm(abq, 4, 8, [3, 5], 64, 512, top=2, layout=abq.ABQ_LAYOUT_BOTH)
    check_gemm(abq, 5, 8, [90, 50], 64, 512, top=2, layout=abq.ABQ_LAYOUT_BOTH)


@pytest.mark.parametrize("p,q,counts,N,K", [(4, 8, [1, 1], 11008, 4096), (2, 8, [3, 9, 0, 1], 4096, 11008), (8, 8, [30, 22], 2048, 1408), (6, 6, [90, 75], 1003, 4096), (4, 4, [500, 612], 2048, 4096)])
def test_same_bits_as_the_products_of_one_expert(abq, p, q, counts, N, K):
    E, rows = len(counts), sum(counts)
    s = {k: [t.cuda() for t in v] for k, v in layer(p, q, E, N, K, rows).items()}
    s["a"][0] &= 2**q - 1
    w = abq.abq_pack_experts(p, *s["w"])
    got = abq.abq_moe_gemm(p, q, N, *s["a"], w, groups(counts).cuda())
    at = 0
    for e, n in enumerate(counts):
        if n:
            one = abq.abq_gemm_act_codes(p, q, n, N, K, *(t[at:at + n].clone() for t in s["a"]), w[e], 0)[0]
            assert torch.equal(got[at:at + n].view(torch.int16), one.view(torch.int16))
        at += n


def test_arrays_that_name_nothing_touch_nothing_else(abq):
    """Starts that do not ascend or point outside, order entries that name no row: rows without an expert, and what lies around Y, stay."""
    N, K, T, E = 64, 256, 24, 6
    s = layer(4, 8, E, N, K, T)
    w = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    a = [t.cuda() for t in s["a"]]
    for rows in (48, 640):
        for starts in ([0, 5, -3, 1 << 30, 7, 40, 9], [-5, -4, -3, -2, -1, 0, 0], [1 << 30] * 7, [40, 30, 20, 10, 5, 2, 1], [0, rows, 0, rows, 0, rows, 0]):
            around = torch.full((rows + 32, N), POISON, dtype=torch.int16, device="cuda")
            y = around[16:16 + rows].view(torch.float16)
            order = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), dtype=torch.int64).to(torch.int32).cuda()
            abq.abq_moe_gemm(4, 8, N, *a, w, torch.tensor(starts, dtype=torch.int32).cuda(), order=order, top=2, y=y)
            assert (around[:16] == POISON).all() and (around[16 + rows:] == POISON).all()
            mine = torch.zeros(rows, dtype=torch.bool)
            for lo, hi in zip(starts, starts[1:]):
                mine[min(max(lo, 0), rows):min(max(hi, 0), rows)] = True
            assert (y.view(torch.int16).cpu()[~mine] == POISON).all()


def kernel_of(abq, p, q, counts, N, K, top=0, behind=0):
    """Whether the product packs its codes for the block kernel, or takes them as they are in the few-rows kernel."""
    rows = sum(counts) + behind
    return "block" if abq.abq_moe_gemm_workspace_bytes(p, q, rows, N, K, -(-rows // top) if top else rows, len(counts)) else "few rows"


# Means of 110, and of 220 rows an expert, with tiles for every unit: 128 and 256 rows a workgroup (192 channels there for p = 7).
@pytest.mark.parametrize("p,E,rows,N", [(4, 10, 1100, 4100), (7, 10, 1100, 4100), (4, 24, 5300, 2050), (7, 24, 5300, 2050), (8, 70, 16100, 600), (2, 130, 14300, 300)])
def test_arrays_that_name_nothing_on_tall_tiles(abq, p, E, rows, N):
    """Starts that name more tiles than there can be, fewer, or rows outside: what no expert has stays, and what lies around Y. The same launch serves
    starts that ascend right after."""
    K, T = 130, 64
    assert kernel_of(abq, p, 8, [rows // E] * (E - 1) + [rows - rows // E * (E - 1)], N, K) == "block"
    s = layer(p, 8, E, N, K, T, seed=E)
    w = abq.abq_pack_experts(p, *(t.cuda() for t in s["w"]))
    a = [t.cuda() for t in s["a"]]
    g = torch.Generator().manual_seed(rows)
    for starts in (([0, 5, -3, 1 << 30, 7, 40, 9] * E)[:E] + [rows // 2], list(range(-E, 1)), [1 << 30] * (E + 1), [rows - rows * i // E for i in range(E + 1)],
                   [0 if i % 2 == 0 else rows for i in range(E + 1)], [rows // 3 if i % 2 == 0 else rows - rows // 7 for i in range(E + 1)], [i * ((1 << 30) // E) for i in range(E + 1)]):
        around = torch.full((rows + 32, N), POISON, dtype=torch.int16, device="cuda")
        y = around[16:16 + rows].view(torch.float16)
        order = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), generator=g).to(torch.int32).cuda()
        abq.abq_moe_gemm(p, 8, N, *a, w, torch.tensor(starts, dtype=torch.int32).cuda(), order=order, top=2, y=y)
        assert (around[:16] == POISON).all() and (around[16 + rows:] == POISON).all()
        mine = torch.zeros(rows, dtype=torch.bool)
        for lo, hi in zip(starts, starts[1:]):
            mine[min(max(lo, 0), rows):min(max(hi, 0), rows)] = True
        assert (y.view(torch.int16).cpu()[~mine] == POISON).all()
    starts = torch.tensor([rows * i // E for i in range(E + 1)], dtype=torch.int32)
    order = torch.randint(0, 2 * T, (rows,), generator=g).to(torch.int32)
    y = abq.abq_moe_gemm(p, 8, N, *a, w, starts.cuda(), order=order.cuda(), top=2)
    assert torch.equal(y.cpu().view(torch.int16), gemm(*s["a"], *s["w"], p, 8, starts, order, 2, rows).view(torch.int16))


# Rows of each expert that the rule sends to the block kernel, with as many channels as each shape of its tiles wants: means of 117, 110 and 207 rows an
# expert; too few tiles for anything but 64 rows a workgroup, enough for 128 and its shorter ones of 96, enough for 256, 192 and 128.
TILES_OF_64 = [120, 101, 130]
TILES_OF_128 = [97, 96, 128, 129, 0, 225, 1, 95, 224, 105]
TILES_OF_256 = [129, 1, 256, 192, 0, 193, 128, 64, 257, 384, 385, 255, 448, 449, 0, 512, 17, 320, 130, 200, 100, 191, 250, 127]


def check_block(abq, p, q, counts, N, K, top=0, behind=0, **kw):
    assert kernel_of(abq, p, q, counts, N, K, top, behind) == "block"
    check_gemm(abq, p, q, counts, N, K, top=top, behind=behind, **kw)


@pytest.mark.parametrize("q", [1, 4, 7, 8])
@pytest.mark.parametrize("p", range(1, 9))
def test_widths_on_every_tile(abq, p, q):
    """Every pair of widths on tiles of 64, 128 and 256 rows and their shorter ones, and on the few-rows kernel with one to four super-chunks a wave."""
    check_block(abq, p, q, TILES_OF_64, 80 + p, 640, top=2, seed=p)
    check_block(abq, p, q, TILES_OF_128, 4096 + 4 * p, 192, seed=p, behind=3)
    check_block(abq, p, q, TILES_OF_256, 2048 + 8 * p, 200, top=3, seed=q)
    for K in (1024, 8704, 12288) + ((14336, 16384) if p <= 4 else ()):
        assert kernel_of(abq, p, q, [2, 0, 7], 40, K, 2) == "few rows"
        check_gemm(abq, p, q, [2, 0, 7], 40, K, top=2, seed=p)


@pytest.mark.parametrize("K", [1, 7, 15, 16, 17, 31, 63, 64, 65, 100, 127, 500, 511, 512, 513, 1000, 1408, 2047, 4095, 5121, 8193, 12289, 16385])
@pytest.mark.parametrize("top", [0, 3])
def test_lengths_that_divide_nothing_on_blocks(abq, K, top):
    for p, q in ((4, 8), (3, 5), (8, 8)):
        check_block(abq, p, q, [140, 0, 160, 1, 199], 40, K, top=top, seed=K)


@pytest.mark.parametrize("N", [1, 2, 7, 15, 17, 33, 127, 129, 191, 193, 255])
def test_columns_that_divide_nothing_on_blocks(abq, N):
    check_block(abq, 4, 8, TILES_OF_64, N, 320, top=2, seed=N)
    check_block(abq, 4, 8, TILES_OF_128, 4096 + N, 96, top=2, seed=N)
    check_block(abq, 6, 6, TILES_OF_256, 2048 + N, 96, seed=N, behind=2)
    check_block(abq, 8, 8, TILES_OF_256, 2048 + N, 96, seed=N)


# Row sums of 2^23 and more, up to the longest K: the epilogue's 32-bit multiplies.
@pytest.mark.parametrize("p,q,K", [(8, 8, 33000), (4, 8, 40000), (1, 8, 131072)])
@pytest.mark.parametrize("counts,N", [([4, 5], 40), ([129, 91], 14200), ([260, 180], 19800)])
def test_sums_of_more_than_24_bits(abq, p, q, K, counts, N):
    """64, 128 and 256 rows a workgroup; columns at either end and in the middle."""
    rows = sum(counts)
    assert kernel_of(abq, p, q, counts, N, K) == "block" and K * (2**max(p, q) - 1) >= 1 << 23
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.randint(0, 2**p, (2, N, K), generator=g, device="cuda", dtype=torch.uint8)
    scale, zero = (torch.rand(2, N, generator=g, device="cuda") + 0.5) / (K**0.5 * 2**p), torch.randint(0, 2**p, (2, N), generator=g, device="cuda", dtype=torch.int32)
    a, starts = layer(p, q, 1, 1, K, rows)["a"], groups(counts)
    got = abq.abq_moe_gemm(p, q, N, *(t.cuda() for t in a), abq.abq_pack_experts(p, codes, scale, zero), starts.cuda())
    for at in (0, N // 2, N - 17):
        at = slice(at, at + 17)
        want = gemm(*a, codes[:, at].cpu(), scale[:, at].cpu(), zero[:, at].cpu(), p, q, starts, None, 1, rows)
        assert torch.equal(got[:, at].cpu().view(torch.int16), want.view(torch.int16)), f"columns from {at.start}"


def test_blobs_that_hold_planes_too_on_blocks(abq):
    check_block(abq, 5, 8, TILES_OF_64, 64, 512, top=2, layout=abq.ABQ_LAYOUT_BOTH)
    check_block(abq, 3, 8, TILES_OF_128, 4100, 130, layout=abq.ABQ_LAYOUT_BOTH)


@pytest.mark.parametrize("p,q,counts,N,K", [(8, 8, [130, 122], 2048, 1408), (6, 6, [190, 175], 1003, 4096), (4, 8, [130, 99, 120], 12000, 1024), (4, 4, [500, 612], 16384, 512)])
def test_same_bits_as_the_products_of_one_expert_on_blocks(abq, p, q, counts, N, K):
    assert kernel_of(abq, p, q, counts, N, K) == "block"
    test_same_bits_as_the_products_of_one_expert(abq, p, q, counts, N, K)


@pytest.mark.parametrize("counts,N", [([130, 97, 200], 48), ([190, 0, 140], 16500), ([600, 500, 700], 6200)])
def test_offsets_beyond_32_bits_on_blocks(abq, counts, N):
    """The second and third expert's weights 2.5 and 5 GiB from the first, on tiles of 64, 128 and 256 rows."""
    K, n = 512, sum(counts)
    assert kernel_of(abq, 4, 8, counts, N, K) == "block"
    s = layer(4, 8, 3, N, K, n)
    packed = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    stride = 5 << 29
    far = torch.empty(2 * stride + packed.shape[1], dtype=torch.uint8, device="cuda").as_strided((3, packed.shape[1]), (stride, 1))
    far.copy_(packed)
    a, starts = [t.cuda() for t in s["a"]], groups(counts).cuda()
    assert torch.equal(abq.abq_moe_gemm(4, 8, N, *a, far, starts), abq.abq_moe_gemm(4, 8, N, *a, packed, starts))


def test_graphs_serve_whatever_the_arrays_hold_later(abq):
    """Router, products and sum captured once; replayed for other logits, other codes."""
    T, E, top, N, K = 40, 16, 3, 96, 512
    s = layer(4, 8, E, N, K, T)
    w = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    a = [t.cuda() for t in s["a"]]
    x = some_logits(T, E, True).cuda()

    def step():
        ids, weights, starts, order, places = abq.abq_moe_route(x, top)
        y = abq.abq_moe_gemm(4, 8, N, *a, w, starts, order=order, top=top)
        return abq.abq_moe_combine(y, places, weights)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        x.copy_(some_logits(T, E, True, seed + 10))
        if seed == 2:
            x[:, 1:] = -INF   # every token to one expert, the other choices none
        a[0].copy_(layer(4, 8, 1, 16, K, T, seed)["a"][0])
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, step())


def test_graphs_with_workspaces(abq):
    """The same through the router's two launches and the block kernel, whose counts and packed codes lie in workspaces of the graph: every replay against the
    64-bit form, with other eager work of the same calls in between."""
    T, E, top, N, K = 900, 8, 2, 136, 320
    assert abq.abq_moe_route_workspace_bytes(T, E, top) > 0 and abq.abq_moe_gemm_workspace_bytes(4, 8, T * top, N, K, T, E) > 0
    s = layer(4, 8, E, N, K, T)
    w = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    a = [t.cuda() for t in s["a"]]
    x = some_logits(T, E, False).cuda()

    def step(x, a):
        routed_to = abq.abq_moe_route(x, top)
        y = abq.abq_moe_gemm(4, 8, N, *a, w, routed_to[2], order=routed_to[3], top=top)
        return (*routed_to, y, abq.abq_moe_combine(y, routed_to[4], routed_to[1]))

    step(x, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, a)
    for seed in range(5):
        logits, codes = some_logits(T, E, False, seed + 20), layer(4, 8, 1, 1, K, T, seed + 1)["a"]
        if seed == 1:
            logits[:, 1:] = -INF          # every token to one expert, the other choices none
        if seed == 3:
            logits[::3] = -INF            # padding
            logits[:, 2] = 50.0
            logits[::3, 2] = -INF
        x.copy_(logits)
        for t, new in zip(a, codes):
            t.copy_(new)
        graph.replay()
        ids, weights, starts, order, places, y, total = [t.cpu() for t in out]
        want = routed(logits, top)
        for name, g, r in zip(("ids", "starts", "order", "places"), (ids, starts, order, places), (want[0], want[2], want[3], want[4])):
            assert torch.equal(g.long(), r), f"{name}, replay {seed}"
        assert ((weights.double() - want[1]).abs() <= want[5]).all()
        used = int(starts[-1])
        assert torch.equal(y[:used].view(torch.int16), gemm(*codes, *s["w"], 4, 8, starts, order, top, T * top)[:used].view(torch.int16)), f"replay {seed}"
        full, bound = combined(torch.where(torch.arange(T * top)[:, None] < used, y, 0), places, weights)
        assert ((total.double() - full).abs() <= bound).all(), f"replay {seed}"
        step(some_logits(T, E, False, seed + 40).cuda(), a)
        torch.cuda.synchronize()


def test_offsets_beyond_32_bits(abq):
    """Experts' weights, and rows that the sum reads, more than 4 GiB from the first."""
    s = layer(4, 8, 3, 48, 512, 40)
    packed = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    stride = 5 << 29   # 2.5 GiB
    far = torch.empty(2 * stride + packed.shape[1], dtype=torch.uint8, device="cuda").as_strided((3, packed.shape[1]), (stride, 1))
    far.copy_(packed)
    for counts in ([2, 3, 1], [13, 14, 13]):
        n = sum(counts)
        a, starts = [t[:n].clone().cuda() for t in s["a"]], groups(counts).cuda()
        assert torch.equal(abq.abq_moe_gemm(4, 8, 48, *a, far, starts), abq.abq_moe_gemm(4, 8, 48, *a, packed, starts))
    del far
    rows = (1 << 32) // 8192 + 9
    y = torch.empty((rows, 8192), dtype=torch.float16, device="cuda")
    y[-7:] = torch.arange(7, device="cuda")[:, None].half()
    places = torch.tensor([[rows - 1, rows - 7, rows - 3]], dtype=torch.int32, device="cuda")
    out = abq.abq_moe_combine(y, places, torch.tensor([[1.0, 5.0, 0.5]], device="cuda"))
    assert (out == 8).all()


@pytest.mark.parametrize("N,K,few", [((1 << 19) + 4099, 4096, True), ((1 << 17) + 67, 16512, False)])
def test_experts_of_more_than_2_gib(abq, N, K, few):
    """One expert's weights beyond 2 GiB of codes and of blob, on both kernels: columns at either end and around the 2 GiB."""
    n = 3
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.randint(0, 256, (2, N, K), generator=g, device="cuda", dtype=torch.uint8)
    s = layer(8, 8, 2, 1, K, 2 * n)
    scale, zero = torch.rand(2, N, generator=g, device="cuda") / 2**14, torch.randint(0, 256, (2, N), generator=g, device="cuda", dtype=torch.int32)
    assert (abq.abq_moe_gemm_workspace_bytes(8, 8, 2 * n, N, K, 2 * n, 2) == 0) == few
    w = abq.abq_pack_experts(8, codes, scale, zero)
    assert w.shape[1] > 1 << 31
    starts = groups([n, n])
    got = abq.abq_moe_gemm(8, 8, N, *(t.cuda() for t in s["a"]), w, starts.cuda())
    for at in (0, (1 << 31) // K - 16, N - 32):
        at = slice(at, at + 32)
        want = gemm(*s["a"], codes[:, at].cpu(), scale[:, at].cpu(), zero[:, at].cpu(), 8, 8, starts, None, 1, 2 * n)
        assert torch.equal(got[:, at].cpu().view(torch.int16), want.view(torch.int16)), f"columns from {at.start}"


@pytest.mark.parametrize("T,E,top,half", [(1 << 22, 8, 1, False), (1 << 18, 1024, 16, True), ((1 << 19) - 5, 513, 8, False), (700001, 64, 5, True), ((1 << 22) - 3, 520, 1, True)])
def test_the_routers_largest_batches(abq, T, E, top, half):
    """The most rows there can be, the longest chunks, logits past 4 GiB. (Choices compared on the device, in pieces.)"""
    g = torch.Generator(device="cuda").manual_seed(E)
    x = torch.empty((T, E), dtype=torch.float16 if half else torch.float32, device="cuda").normal_(generator=g)
    x[::7] = -INF
    ids, weights, starts, order, places = abq.abq_moe_route(x, top)
    for at in range(0, T, 1 << 16):
        piece = x[at:at + (1 << 16)].float()
        for j in range(top):   # the largest that is left, the first of equals
            best = torch.where(piece == piece.amax(1, keepdim=True), torch.arange(E, device="cuda"), E).amin(1)
            best = torch.where(piece.amax(1) > -INF, best, -1)
            assert torch.equal(ids[at:at + (1 << 16), j].long(), best), f"tokens from {at}, choice {j}"
            piece.scatter_(1, best.clamp(min=0)[:, None], -INF)
    there = ids >= 0
    assert ((weights.sum(1) - there.any(1).float()).abs() < 1e-5).all()
    flat = torch.where(there, ids, E).flatten()
    by_expert, slots = torch.sort(flat, stable=True)
    assert torch.equal(starts.long(), torch.searchsorted(by_expert, torch.arange(E + 1, device="cuda")))
    assert torch.equal(order.long(), torch.where(by_expert < E, slots, -1))
    want = torch.empty_like(slots)
    want[slots] = torch.arange(len(slots), device="cuda")
    assert torch.equal(places.flatten().long(), torch.where(flat < E, want, -1))


def check_far_rows(abq, p, q, N, K, T, counts, order, look):
    """Rows `look` of Y, of codes that are made on the device."""
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.empty((T, K), dtype=torch.uint8, device="cuda").random_(0, 256, generator=g)
    scale, zero = torch.rand(T, generator=g, device="cuda") / 64, torch.randint(0, 2**q, (T,), generator=g, device="cuda", dtype=torch.int32)
    w, starts = layer(p, q, len(counts), N, K, 1)["w"], groups(counts)
    y = abq.abq_moe_gemm(p, q, N, codes, scale, zero, abq.abq_pack_experts(p, *(t.cuda() for t in w)), starts.cuda(), order=order)
    src = look if order is None else order.cpu()[look].long()
    expert = torch.searchsorted(starts.long(), look, right=True) - 1
    for e in range(len(counts)):
        mine = look[expert == e]
        if len(mine):
            at = src[expert == e].cuda()
            want = gemm(codes[at].cpu(), scale[at].cpu(), zero[at].cpu(), *w, p, q, groups([0] * e + [len(mine)] + [0] * (len(counts) - e - 1)), None, 1, len(mine))
            assert torch.equal(y[mine.cuda()].cpu().view(torch.int16), want.view(torch.int16)), f"expert {e}"


def test_the_products_largest_batches(abq):
    """The most rows there can be, codes and outputs of more than 4 GiB, on both kernels."""
    T = (1 << 22) - 1
    ends = lambda n: torch.cat([torch.arange(0, 300), torch.arange(n // 3 - 150, n // 3 + 150), torch.arange(n // 2 - 150, n // 2 + 150), torch.arange(n - 300, n)])
    check_far_rows(abq, 4, 8, 24, 1000, T, [T // 3, T // 2 - T // 3, T - T // 2], None, ends(T))
    check_far_rows(abq, 4, 8, 24, 1000, T, [3, 0, 5], torch.tensor([T - 1, 0, T - 2, T // 2, T - 1, 7, T - 600, T // 2 + 1], dtype=torch.int32, device="cuda"), torch.arange(8))
    n = 1 << 18
    check_far_rows(abq, 8, 8, 16400, 16, n, [n // 3, n // 2 - n // 3, n - n // 2], None, ends(n))
    check_far_rows(abq, 2, 8, 1 << 20, 16, 2100, [700, 700, 700], None, torch.tensor([0, 699, 700, 2098, 2099]))


def test_new_outputs_are_tensors_of_their_own(abq):
    """They are made in one allocation; each has its shape and type, and nothing written to one shows in another."""
    x = some_logits(37, 24, True).cuda()
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            got = abq.abq_moe_route(x, 3)
            assert [(t.shape, t.dtype, t.is_contiguous()) for t in got] == [((37, 3), torch.int32, True), ((37, 3), torch.float32, True), ((25,), torch.int32, True),
                                                                            ((111,), torch.int32, True), ((37, 3), torch.int32, True)]
            kept = [t.clone() for t in got]
            for i, t in enumerate(got):
                t.fill_(-9)
                assert all(torch.equal(g, k) for g, k in list(zip(got, kept))[i + 1:]) and (t == -9).all()
    a = torch.nn.Parameter(torch.ones(3, device="cuda"))
    weights = abq.abq_moe_route(x, 3)[1]
    (weights * a).sum().backward()
    assert torch.allclose(a.grad, weights.sum(0), rtol=1e-5)


def test_refused_sizes_take_no_memory(abq):
    """Outputs of a size that the library refuses are not made first."""
    routes = [(torch.zeros((1 << 18) + 1, 16, dtype=torch.float16, device="cuda"), 16), (torch.zeros(1000, 1025, device="cuda"), 16)]
    rows = (1 << 22) + 1
    a = torch.zeros((1, 16), dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    w = torch.zeros((2, abq.abq_packed_weight_bytes(4, 256, 16)), dtype=torch.uint8, device="cuda")
    starts, order = groups([3, 4]).cuda(), torch.zeros(rows, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    for call in [lambda x=x, top=top: abq.abq_moe_route(x, top) for x, top in routes] + [lambda: abq.abq_moe_gemm(4, 8, 256, *a, w, starts, order=order)]:
        with pytest.raises(abq.AbqError) as e:
            call()
        assert e.value.status == abq.ABQ_ERR_SHAPE
    assert torch.cuda.max_memory_allocated() == before


def test_two_streams_at_once(abq):
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    s = layer(4, 8, 8, 256, 1024, 300)
    w = abq.abq_pack_experts(4, *(t.cuda() for t in s["w"]))
    a = [t.cuda() for t in s["a"]]
    x = some_logits(300, 8, False).cuda()

    def step():
        ids, weights, starts, order, places = abq.abq_moe_route(x, 2)
        return abq.abq_moe_combine(abq.abq_moe_gemm(4, 8, 256, *a, w, starts, order=order, top=2), places, weights)

    want = step()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for stream in (one, two):
            with torch.cuda.stream(stream):
                got.append(step())
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_two_streams_with_work_of_their_own(abq):
    """Each stream its own logits, codes and results, through the calls that take workspaces (the router's counts, the packed codes): nothing is shared between them."""
    T, E, top, N, K = 1700, 8, 2, 256, 512
    assert abq.abq_moe_route_workspace_bytes(T, E, top) > 0 and abq.abq_moe_gemm_workspace_bytes(4, 8, T * top, N, K, T, E) > 0
    w = abq.abq_pack_experts(4, *(t.cuda() for t in layer(4, 8, E, N, K, 1)["w"]))

    def step(x, a):
        ids, weights, starts, order, places = abq.abq_moe_route(x, top)
        y = abq.abq_moe_gemm(4, 8, N, *a, w, starts, order=order, top=top)
        return ids, starts, order, y, abq.abq_moe_combine(y, places, weights)

    work = [(torch.cuda.Stream(), some_logits(T, E, False, seed).cuda(), [t.cuda() for t in layer(4, 8, 1, 1, K, T, seed)["a"]]) for seed in (1, 2)]
    want = [step(x, a) for _, x, a in work]
    assert not any(torch.equal(one, two) for one, two in zip(*want))
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        for i, (stream, x, a) in enumerate(work):
            with torch.cuda.stream(stream):
                got.append((i, step(x, a)))
    torch.cuda.synchronize()
    for n, (i, outs) in enumerate(got):
        assert all(torch.equal(g, w) for g, w in zip(outs, want[i])), f"call {n}"


# ---- weighted sum ----------------------------------------------------------------------------------
def check_combine(abq, T, top, N, rows, seed=0, add=True, missing=0.1):
    g = torch.Generator().manual_seed(seed)
    y = torch.randn(rows, N, generator=g).half()
    places = torch.randint(0, rows, (T, top), generator=g).to(torch.int32)
    places[torch.rand(T, top, generator=g) < missing] = -1
    weights = torch.rand(T, top, generator=g)
    base = torch.randn(T, N, generator=g).half() if add else None
    got = abq.abq_moe_combine(y.cuda(), places.cuda(), weights.cuda(), add=base.cuda() if add else None).cpu()
    want, bound = combined(y, places, weights, base)
    off = (got.double() - want).abs()
    assert (off <= bound).all(), f"{int((off > bound).sum())} of {off.numel()} off"


@pytest.mark.parametrize("N", [1, 2, 7, 8, 9, 64, 100, 2047, 2048, 2049, 4096, 5121])
@pytest.mark.parametrize("top", [1, 2, 3, 6, 8, 16, 33])
def test_sums(abq, N, top):
    for T in (1, 5):
        check_combine(abq, T, top, N, 3 * T + 1, seed=N, add=bool(top % 2))
    check_combine(abq, 130, top, N, 64, seed=top)


def test_choices_that_are_none(abq):
    y = torch.full((4, 40), float("nan"), dtype=torch.float16).cuda()
    y[2] = 1.5
    places = torch.tensor([[-1, -1], [2, -1], [4, 2], [-(1 << 31), (1 << 31) - 1]], dtype=torch.int32).cuda()
    weights = torch.full((4, 2), 2.0).cuda()
    weights[0] = float("nan")
    assert abq.abq_moe_combine(y, places, weights).cpu()[:, 7].tolist() == [0.0, 3.0, 3.0, 0.0]
    add = torch.full((4, 40), -0.5, dtype=torch.float16).cuda()
    assert abq.abq_moe_combine(y, places, weights, add=add).cpu()[:, 39].tolist() == [-0.5, 2.5, 2.5, -0.5]
    y[2, 3], y[2, 4] = INF, 60000.0
    out = abq.abq_moe_combine(y, places, weights).cpu()
    assert out[1, 3] == INF and out[1, 4] == INF and out[0, 3] == 0


def test_sums_in_place_and_in_columns(abq):
    g = torch.Generator().manual_seed(4)
    y, places, weights = torch.randn(50, 100, generator=g).half().cuda(), torch.randint(0, 50, (20, 4), generator=g).to(torch.int32).cuda(), torch.rand(20, 4, generator=g).cuda()
    add = torch.randn(20, 100, generator=g).half().cuda()
    want = abq.abq_moe_combine(y, places, weights, add=add)
    wide = torch.zeros(50, 333, dtype=torch.float16, device="cuda")
    wide[:, 8:108], wide[:20, 128:228] = y, add
    out = torch.full((20, 211), 7.0, dtype=torch.float16, device="cuda")
    abq.abq_moe_combine(wide[:, 8:108], places, weights, add=wide[:20, 128:228], out=out[:, 16:116])
    assert torch.equal(out[:, 16:116], want) and (out[:, :16] == 7).all() and (out[:, 116:] == 7).all()
    assert abq.abq_moe_combine(y, places, weights, add=add, out=add) is add and torch.equal(add, want)


# ---- a run of them ---------------------------------------------------------------------------------
@pytest.mark.parametrize("T,E,top,D,F,p,q", [(1, 8, 2, 512, 1024, 4, 8), (7, 16, 4, 520, 264, 2, 8), (33, 8, 2, 1024, 512, 6, 6), (300, 12, 3, 256, 384, 8, 8), (700, 4, 2, 512, 768, 4, 4)])
def test_a_layer_of_experts(abq, T, E, top, D, F, p, q):
    """Norm with its quantizer, router, gate and up, SiLU with its quantizer, down, weighted sum on the residual; every step against its own
    64-bit form on what the steps before it gave, some of the tokens padding."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, D, generator=g).half()
    gamma = torch.ones(D).half()
    logits = torch.randn(T, E, generator=g).half()
    if T > 5:
        logits[::4] = -INF
    up, gate, down = layer(p, q, E, F, D, 1, 1)["w"], layer(p, q, E, F, D, 1, 2)["w"], layer(p, q, E, D, F, 1, 3)["w"]
    w = [abq.abq_pack_experts(p, *(t.cuda() for t in m)) for m in (gate, up, down)]
    codes, scale, zero, _ = abq.abq_rmsnorm_quant_act(q, x.cuda(), gamma.cuda(), 1e-5)
    ids, weights, starts, order, places = abq.abq_moe_route(logits.cuda(), top)
    gu = [abq.abq_moe_gemm(p, q, F, codes, scale, zero, m, starts, order=order, top=top) for m in w[:2]]
    used = int(starts[-1])
    for m, got in zip((gate, up), gu):
        want = gemm(codes.cpu(), scale.cpu(), zero.cpu(), *m, p, q, starts.cpu(), order.cpu(), top, T * top)
        assert torch.equal(got.cpu()[:used].view(torch.int16), want[:used].view(torch.int16))
    hc, hs, hz, _ = abq.abq_silu_mul_quant_act(q, *gu)
    y = abq.abq_moe_gemm(p, q, D, hc, hs, hz, w[2], starts)
    want = gemm(hc.cpu(), hs.cpu(), hz.cpu(), *down, p, q, starts.cpu(), None, 1, T * top)
    assert torch.equal(y.cpu()[:used].view(torch.int16), want[:used].view(torch.int16))
    out = abq.abq_moe_combine(y, places, weights, add=x.cuda()).cpu()
    full, bound = combined(y.cpu(), places.cpu(), weights.cpu(), x)
    assert ((out.double() - full).abs() <= bound).all()
    if T > 5:
        assert torch.equal(out[::4], x[::4])   # padding: the residual
    assert int((ids >= 0).sum()) == used
