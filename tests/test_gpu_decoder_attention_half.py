"""The attention half of a decoder block as a server runs it, one operator behind the other: add + RMSNorm + quantizer, quantized q / k / v
projections, the requests' adapters beside them, append with rotation, attention, quantizer, output projection with adapters.  Every
operator's result is checked against its own 64-bit form on the inputs that it got, over steps that fill the cache."""
import numpy as np
import pytest
import torch

import oracle
from helpers import y_tolerance
from paper_2408_08554_amd import synth
from serving_reference import Paged, adapted, rotated, rotated_bound

pytestmark = pytest.mark.gpu

HIDDEN, HQ, H, D, PAGE = 512, 8, 2, 64, 16
P, Q = 4, 8


class Layer:
    def __init__(self, abq, seed):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.abq, self.w = abq, {}
        for name, (n, k) in dict(q=(HQ * D, HIDDEN), k=(H * D, HIDDEN), v=(H * D, HIDDEN), o=(HIDDEN, HQ * D)).items():
            codes, scale = rng.integers(0, 16, (n, k), dtype=np.uint8), (rng.uniform(0.5, 1.0, n) * 2 / (16 * k ** 0.5)).astype(np.float32)
            zero = rng.integers(6, 10, n).astype(np.int32)
            dev = [torch.from_numpy(x).cuda() for x in (codes, scale, zero)]
            self.w[name] = (codes, scale, zero, abq.abq_pack_weights(P, *dev))
        g = torch.Generator().manual_seed(seed)
        self.adapters = {name: ((torch.randn(3, 8, k, generator=g) / k ** 0.5).half(), (torch.randn(3, n, 8, generator=g) * 0.3).half(), torch.rand(3, generator=g) + 0.5)
                         for name, (n, k) in dict(q=(HQ * D, HIDDEN), v=(H * D, HIDDEN), o=(HIDDEN, HQ * D)).items()}
        self.gamma = torch.from_numpy(synth.act_fp16(seed, 1, HIDDEN, outliers=False)[0]).abs() + 0.5

    def linear(self, name, codes, scale, zero, M):
        wc, ws, wz, packed = self.w[name]
        N, K = wc.shape
        y, _ = self.abq.abq_gemm_act_codes(P, Q, M, N, K, codes, scale, zero, packed, self.abq.ABQ_LAYOUT_FIELDS)
        want, _ = oracle.dequant(oracle.acc_centered(codes.cpu().numpy(), wc, zero.cpu().numpy(), wz), scale.cpu().numpy(), ws)
        assert (np.abs(y.cpu().numpy().astype(np.float64) - want) <= y_tolerance(want)).all()
        return y

    def adapt(self, name, x, ids, y):
        a, b, s = self.adapters[name]
        out = self.abq.abq_lora_add(x, ids, a.cuda(), b.cuda(), s.cuda(), y)
        want, bound = adapted(x.cpu(), ids.cpu(), a, b, s, y.cpu())
        assert ((out.cpu().double() - want).abs() <= bound).all()
        return out


@pytest.mark.parametrize("bits", [16, 8])
def test_steps_of_a_layer(abq, bits):
    layer = Layer(abq, 31)
    freq = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float()
    tokens = [0, 0, 0]   # of three requests so far
    whole = Paged([(0, 200)] * 3, HQ, H, D, PAGE, bits, seed=5)   # room for 200 tokens each; the cache lives on the device
    cache = tuple(t.cuda() for t in whole.cache)
    ids_of = torch.tensor([1, -1, 2])
    residual = None
    for news in ([37, 5, 1], [1, 1, 1], [1, 70, 0], [1, 1, 1]):   # prompts, a step, a chunk beside a step, a step
        rows = sum(news)
        tokens = [t + n for t, n in zip(tokens, news)]
        start = torch.tensor([0] + news).cumsum(0).to(torch.int32)
        seq = torch.repeat_interleave(torch.arange(3), torch.tensor(news))
        ids = ids_of[seq].to(torch.int32).cuda()
        batch = (start.cuda(), torch.tensor(tokens, dtype=torch.int32).cuda(), whole.pages.cuda())
        x = torch.from_numpy(synth.act_fp16(rows, rows, HIDDEN)).cuda()
        residual = torch.from_numpy(synth.act_fp16(rows + 1, rows, HIDDEN)).cuda()
        codes, scale, zero, h, normed = abq.abq_add_rmsnorm_quant_act(Q, x, residual, layer.gamma.cuda(), 1e-5, want_y=True)
        q = layer.adapt("q", normed, ids, layer.linear("q", codes, scale, zero, rows))
        k = layer.linear("k", codes, scale, zero, rows)
        v = layer.adapt("v", normed, ids, layer.linear("v", codes, scale, zero, rows))
        turned = abq.abq_kv_append(cache, batch, k, v, q=q, inv_freq=freq.cuda())
        at = torch.arange(rows) - start[:-1][seq] + torch.tensor(tokens)[seq] - torch.tensor(news)[seq]
        want, size = rotated(q.cpu().view(rows, HQ, D), at, freq)
        assert ((turned.cpu().view(rows, HQ, D).double() - want).abs() <= rotated_bound(want, size)).all()
        slots = whole.pages[seq, at // PAGE] * PAGE + (at % PAGE).to(torch.int32)
        k_back, v_back = abq.abq_kv_read(cache, slots.cuda())
        step = lambda x: (x.amax(-1).clamp(min=0) - x.amin(-1).clamp(max=0))[..., None] / 255 * 0.501 if bits == 8 else 0.0   # half a step of the codes
        want, size = rotated(k.cpu().view(rows, H, D), at, freq)
        assert ((k_back.cpu().view(rows, H, D).double() - want).abs() <= step(want) + 3 * rotated_bound(want, size)).all()
        v3 = v.cpu().view(rows, H, D).double()
        assert ((v_back.cpu().view(rows, H, D).double() - v3).abs() <= step(v3) + (2.0 ** -10 * v3.abs() + 2.0 ** -24 if bits == 8 else 0.0)).all()
        y = abq.abq_attn_paged(cache, batch, turned, D ** -0.5, max_new=max(news), max_len=max(tokens))
        now = Paged([(n, t - n) for n, t in zip(news, tokens)], HQ, H, D, PAGE, bits, seed=6)
        now.pages, now.cache, now.q = whole.pages, [t.cpu() for t in cache], turned.cpu()
        want, bound = now.attention(D ** -0.5)
        assert ((y.cpu().view(want.shape).double() - want).abs() <= bound).all()
        blob = abq.abq_quant_pack_act(Q, y)
        codes, scale, zero, _ = abq.abq_unpack_act(Q, rows, HQ * D, abq.ABQ_LAYOUT_AUTO, blob, abq.ABQ_LAYOUT_FIELDS)
        out = layer.adapt("o", y, ids, layer.linear("o", codes, scale, zero, rows))
        assert out.shape == (rows, HIDDEN) and out.isfinite().all()


def test_a_decoding_step_as_a_graph(abq):
    """The same chain for single tokens, captured once and replayed while the cache fills: lengths, pages and inputs change under it."""
    layer = Layer(abq, 32)
    freq = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().cuda()
    whole = Paged([(0, 400)] * 2, HQ, H, D, PAGE, seed=7)
    caches = [tuple(t.cuda() for t in whole.cache) for _ in range(2)]
    start, pages = torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), whole.pages.cuda()
    lens = torch.tensor([130, 17], dtype=torch.int32).cuda()
    x, ids = torch.zeros(2, HIDDEN, dtype=torch.float16, device="cuda"), torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    packed = {n: w[3] for n, w in layer.w.items()}
    adapters = {n: tuple(t.cuda() for t in a) for n, a in layer.adapters.items()}
    gamma = layer.gamma.cuda()

    def step(cache):
        codes, scale, zero, normed = abq.abq_rmsnorm_quant_act(Q, x, gamma, 1e-5, want_y=True)
        lin = lambda n: abq.abq_gemm_act_codes(P, Q, 2, layer.w[n][0].shape[0], HIDDEN, codes, scale, zero, packed[n], abq.ABQ_LAYOUT_FIELDS)[0]
        q = abq.abq_lora_add(normed, ids, *adapters["q"], lin("q"))
        v = lin("v")
        abq.abq_lora_add(normed, ids, *adapters["v"], v, out=v)
        q = abq.abq_kv_append(cache, (start, lens, pages), lin("k"), v, q=q, inv_freq=freq, q_out=q)
        return abq.abq_attn_paged(cache, (start, lens, pages), q, D ** -0.5, max_new=1)

    step(caches[0])
    torch.cuda.synchronize()
    for a, b in zip(*caches):
        b.copy_(a)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step(caches[0])
    for i in range(6):
        x.copy_(torch.from_numpy(synth.act_fp16(100 + i, 2, HIDDEN)))
        lens += 40 if i == 3 else 1
        want = step(caches[1])
        torch.cuda.synchronize()
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        assert all(torch.equal(a, b) for a, b in zip(*caches)), i


@pytest.mark.parametrize("n", [1, 40])
def test_codes_of_a_token_whose_values_are_zero(abq, n):
    """Such a token, looked at most of all, leaves the others' small values their digits: it is held with the smallest scale."""
    p = Paged([(200, 0)], 4, 2, 64, 16, bits=8, seed=n)
    cache, (starts, lens, pages), _ = p.device()
    k, v = p.normal(200, 128), p.normal(200, 128) * 0.01
    q = p.normal(200, 256)
    k[7], v[7] = q[199, :64].repeat(2) * 0.5, 0.0
    abq.abq_kv_append(cache, (starts, lens, pages), k.cuda(), v.cuda())
    p.cache = [t.cpu() for t in cache]
    assert (p.cache[4][int(p.pages[0, 0]), :, 7] == 2.0 ** -32).all() and (p.cache[1][int(p.pages[0, 0]), :, 7] == 0).all()
    p.news, p.rows, p.row_start, p.q = [n], n, torch.tensor([0, n], dtype=torch.int32), q[200 - n:]
    y = abq.abq_attn_paged(cache, (p.row_start.cuda(), lens, pages), p.q.cuda(), 0.125).cpu().view(n, 4, 64).double()
    want, bound = p.attention(0.125)
    assert ((y - want).abs() <= bound).all() and bound.max() < 2.0 ** -10   # (values of up to 2^-4)


def test_a_step_of_prompts_over_codes_as_graphs(abq):
    """Adapters of many rows, append to a cache of codes, reading back and attention of prompts beside single tokens, in parts: two graphs of their
    own workspaces, replayed at once on two streams, with eager work between, on inputs and lengths that change."""
    p = Paged([(300, 900), (1, 3000), (2, 40)], HQ, H, 128, PAGE, bits=8, seed=8, extra_rows=2)
    g = torch.Generator().manual_seed(8)
    start, pages = p.row_start.cuda(), p.pages.cuda()
    lens = p.lens.cuda()
    x, ids = torch.zeros(p.rows, 256, dtype=torch.float16, device="cuda"), torch.randint(-1, 3, (p.rows,), generator=g).to(torch.int32).cuda()
    a, b = (torch.randn(3, 8, 256, generator=g) / 16).half().cuda(), (torch.randn(3, HQ * 128, 8, generator=g) * 0.3).half().cuda()
    scale, freq = torch.ones(3, device="cuda"), (10000.0 ** (-torch.arange(0, 128, 2).double() / 128)).float().cuda()
    k, v, base = (p.normal(p.rows, n * 128).cuda() for n in (H, H, HQ))
    slots = torch.arange(0, 200, 7, dtype=torch.int32).cuda()

    def step(cache):
        q = abq.abq_lora_add(x, ids, a, b, scale, base)
        q = abq.abq_kv_append(cache, (start, lens, pages), k, v, q=q, inv_freq=freq, q_out=torch.zeros_like(q))
        return abq.abq_attn_paged(cache, (start, lens, pages), q, 128 ** -0.5, y=torch.zeros_like(q)), *abq.abq_kv_read(cache, slots)

    caches = [tuple(t.cuda() for t in p.cache) for _ in range(3)]
    step(caches[0])
    torch.cuda.synchronize()
    for c in caches[1:]:
        for to, t in zip(c, caches[0]):
            to.copy_(t)
    graphs = []
    for c in caches[1:]:
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            out = step(c)
        graphs.append((graph, stream, out))
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=g).half())
        k.copy_(p.normal(*k.shape)), v.copy_(p.normal(*v.shape))
        lens -= i
        want = step(caches[0])
        torch.cuda.synchronize()
        for graph, stream, _ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (_, _, out), c in zip(graphs, caches[1:]):
            assert all(torch.equal(y, w) for y, w in zip(out, want)), i
            assert all(torch.equal(t, w) for t, w in zip(c, caches[0])), i
