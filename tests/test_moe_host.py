"""What the calls of a layer of experts refuse, on a host without a GPU: nothing here reaches a launch."""
import pytest
import torch

from paper_2408_08554_amd import binding as B

A16 = 0x1000   # any 16-byte aligned address; refused before it is read
NULL, BITS, SHAPE, ALIGN, SIZE, LAYOUT = B.ABQ_ERR_NULL, B.ABQ_ERR_BITS, B.ABQ_ERR_SHAPE, B.ABQ_ERR_ALIGN, B.ABQ_ERR_SIZE, B.ABQ_ERR_LAYOUT


def route(T=300, E=64, top=8, logits=A16, bits=16, ld=64, bias=A16, scale=1.0, ids=A16, weights=A16, starts=A16, order=A16, places=A16, ws=A16, wsb=1 << 30):
    return B.load().abq_moe_route(T, E, top, logits, bits, ld, bias, 0, 1, scale, ids, weights, starts, order, places, ws, wsb, None)


@pytest.mark.parametrize("kw,want", [({n: None}, NULL) for n in ("logits", "ids", "weights", "starts", "order", "places", "ws")] +
                         [({n: A16 + 4}, ALIGN) for n in ("logits", "bias", "ids", "weights", "starts", "order", "places", "ws")] +
                         [(dict(bits=8), BITS), (dict(bits=0), BITS), (dict(T=0), SHAPE), (dict(T=-1), SHAPE), (dict(E=0, ld=1), SHAPE), (dict(E=1025, ld=1025), SHAPE), (dict(top=0), SHAPE),
                          (dict(top=17), SHAPE), (dict(E=7, top=8), SHAPE), (dict(T=1 << 20), SHAPE), (dict(T=2**31 - 1, top=1), SHAPE), (dict(ld=63), SHAPE), (dict(ld=-64), SHAPE), (dict(wsb=16), SIZE)])
def test_route_refuses(kw, want):
    assert route(**kw) == want


def gemm(p=4, q=8, rows=32, N=128, K=256, T=16, E=4, top=2, a=A16, s=A16, z=A16, w=A16, stride=1 << 20, layout=0, starts=A16, order=A16, y=A16, ws=A16, wsb=1 << 40):
    return B.load().abq_moe_gemm(p, q, rows, N, K, T, E, top, a, s, z, w, stride, layout, starts, order, y, ws, wsb, None)


BAD_GEMM = [({n: None}, NULL) for n in ("a", "s", "z", "w", "starts", "y")] + [({n: A16 + 8}, ALIGN) for n in ("a", "s", "z", "w", "starts", "order", "y", "ws")]
BAD_GEMM += [(dict(p=0), BITS), (dict(p=9), BITS), (dict(q=0), BITS), (dict(q=9), BITS), (dict(rows=0), SHAPE), (dict(rows=(1 << 22) + 1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE),
             (dict(K=B.ABQ_MAX_K + 1), SHAPE), (dict(T=0), SHAPE), (dict(T=(1 << 22) + 1), SHAPE), (dict(E=0), SHAPE), (dict(E=1025), SHAPE), (dict(top=0), SHAPE), (dict(order=None), SHAPE),
             (dict(p=8, q=8, K=65536), SHAPE), (dict(T=1 << 22, K=1000), SHAPE), (dict(rows=1 << 22, N=1 << 16), SHAPE), (dict(N=2**31 - 1), SHAPE), (dict(rows=1, T=1, E=1, top=1, N=(1 << 27) + 1), SHAPE), (dict(stride=(1 << 20) + 8), ALIGN), (dict(stride=16384), SIZE), (dict(stride=0), SIZE)]
BAD_GEMM += [(dict(layout=v), LAYOUT) for v in (B.ABQ_LAYOUT_PLANES, B.ABQ_LAYOUT_FIELDS_G128, B.ABQ_LAYOUT_FIELDS | B.ABQ_USE_FIELDS, 77, -1)]
BAD_GEMM += [(dict(rows=4096, T=2048, ws=None), NULL), (dict(rows=4096, T=2048, wsb=1024), SIZE)]


@pytest.mark.parametrize("kw,want", BAD_GEMM)
def test_gemm_refuses(kw, want):
    assert gemm(**kw) == want


def combine(T=16, N=128, rows=32, top=2, y=A16, ldy=128, places=A16, weights=A16, add=A16, ldadd=128, out=A16 * 2, ldout=128):
    return B.load().abq_moe_combine(T, N, rows, top, y, ldy, places, weights, add, ldadd, out, ldout, None)


@pytest.mark.parametrize("kw,want", [({n: None}, NULL) for n in ("y", "places", "weights", "out")] + [({n: A16 + 2}, ALIGN) for n in ("y", "places", "weights", "add", "out")] +
                         [({n: v}, SHAPE) for n in ("T", "N", "rows", "top") for v in (0, -1, 2**31 - 1)] +
                         [(dict(ldy=127), SHAPE), (dict(ldout=127), SHAPE), (dict(ldadd=127), SHAPE), (dict(add=A16 * 2, ldadd=256), SHAPE), (dict(T=1 << 22, N=8193, ldy=8193, ldadd=8193, ldout=8193), SHAPE)])
def test_combine_refuses(kw, want):
    assert combine(**kw) == want


def pack(p=4, E=4, N=128, K=256, w=A16, s=A16, z=A16, layout=0, out=A16, stride=1 << 20):
    return B.load().abq_pack_experts(p, E, N, K, w, s, z, layout, out, stride, None)


@pytest.mark.parametrize("kw,want", [({n: None}, NULL) for n in ("w", "s", "z", "out")] + [({n: A16 + 8}, ALIGN) for n in ("w", "s", "z", "out")] +
                         [(dict(p=0), BITS), (dict(p=9), BITS), (dict(E=0), SHAPE), (dict(E=1025), SHAPE), (dict(E=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=B.ABQ_MAX_K + 1), SHAPE),
                          (dict(stride=(1 << 20) + 8), ALIGN), (dict(stride=16384), SIZE), (dict(stride=0), SIZE), (dict(layout=B.ABQ_LAYOUT_FIELDS_G128), LAYOUT), (dict(layout=77), LAYOUT)])
def test_pack_refuses(kw, want):
    assert pack(**kw) == want


def test_workspace_queries():
    """Zero for what the call refuses, and where the calls need none."""
    assert B.abq_moe_route_workspace_bytes(1, 8, 2) == 0 and B.abq_moe_route_workspace_bytes(0, 8, 2) == 0 and B.abq_moe_route_workspace_bytes(300, 8, 9) == 0
    assert B.abq_moe_route_workspace_bytes(100000, 64, 8) >= 64 * 4
    assert B.abq_moe_gemm_workspace_bytes(4, 8, 16, 128, 256, 8, 4) == 0 and B.abq_moe_gemm_workspace_bytes(9, 8, 4096, 128, 256, 2048, 4) == 0
    assert B.abq_moe_gemm_workspace_bytes(4, 8, 4096, 128, 256, 2048, 4) >= 2048 * 512


@pytest.mark.parametrize("experts,top", [(1, 1), (8, 2), (64, 6), (128, 8), (256, 16), (512, 16), (513, 16), (1024, 1)])
def test_the_routers_workspace_never_falls_as_tokens_grow(experts, top):
    """So that one of the largest batch serves every smaller one."""
    most = (1 << 22) // top
    tokens = sorted({t for t in [*range(1, 20000), *(c * 512 + d for c in range(1, most // 512, 97) for d in (-1, 0, 1)), *range(most - 600, most + 1)] if 1 <= t <= most})
    sizes = [B.abq_moe_route_workspace_bytes(t, experts, top) for t in tokens]
    falls = [(a, b) for a, b, x, y in zip(tokens, tokens[1:], sizes, sizes[1:]) if y < x]
    assert not falls, f"{len(falls)} times, first from {falls[0][0]} to {falls[0][1]} tokens"
    assert sizes[-1] > 0


@pytest.mark.parametrize("p,experts,top,N,K", [(4, 8, 2, 512, 4096), (8, 64, 6, 320, 448), (2, 128, 8, 1408, 2048), (1, 1, 1, 64, 8), (5, 8, 2, 4096, 14336)])
def test_the_products_workspace_never_falls_as_tokens_grow(p, experts, top, N, K):
    for gather in (True, False):   # (down projections: as many rows of codes as rows)
        sizes = [B.abq_moe_gemm_workspace_bytes(p, 8, t * top, N, K, t if gather else t * top, experts) for t in range(1, 3000)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[-1] > 0


def test_operands_on_the_host_are_refused():
    """Every operand is a device tensor; the binding says so before anything is launched."""
    x = torch.zeros(4, 8)
    with pytest.raises(AssertionError):
        B.abq_moe_route(x, 2)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(AssertionError):
        B.abq_moe_gemm(4, 8, 16, torch.zeros(4, 16, dtype=torch.uint8), x[:, 0], i(4), torch.zeros(2, 4096, dtype=torch.uint8), i(3))
    with pytest.raises(AssertionError):
        B.abq_moe_combine(x.half(), i(2, 2), torch.zeros(2, 2))
    with pytest.raises(AssertionError):
        B.abq_pack_experts(4, torch.zeros(2, 16, 16, dtype=torch.uint8), torch.zeros(2, 16), i(2, 16))


def test_arguments_are_checked():
    with pytest.raises(TypeError):
        B.abq_moe_route(torch.zeros(4, 8), 2, none=1)
    with pytest.raises(TypeError):
        B.abq_moe_combine(1, 2, 3)
    with pytest.raises(ValueError):
        B.abq_moe_route(torch.zeros(8), 2)
