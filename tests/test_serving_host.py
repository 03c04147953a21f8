"""What the calls of the paged cache, the attention over it and the adapters refuse, on a host without a GPU: nothing here
reaches a launch."""
import ctypes

import pytest
import torch

from paper_2408_08554_amd import binding as B

A16 = 0x1000   # any 16-byte aligned address; refused before it is read


def cache(**kw):
    d = dict(kv_bits=16, num_pages=4, page_size=16, heads=2, head_dim=64, k=A16, v=A16)
    d.update(kw)
    return B.AbqKvCache(**d)


def batch(**kw):
    d = dict(rows=8, seqs=3, max_pages=5, max_new=8, max_len=80, row_start=A16, lens=A16, pages=A16)
    d.update(kw)
    return B.AbqBatch(**d)


CODES = dict(kv_bits=8, k_scale=A16, k_zero=A16, v_scale=A16, v_zero=A16)
BAD_CACHES = [(dict(k=0), B.ABQ_ERR_NULL), (dict(v=0), B.ABQ_ERR_NULL), (dict(kv_bits=4), B.ABQ_ERR_BITS), (dict(kv_bits=0), B.ABQ_ERR_BITS), (dict(kv_bits=8), B.ABQ_ERR_NULL),
              (dict(num_pages=0), B.ABQ_ERR_SHAPE), (dict(page_size=8), B.ABQ_ERR_SHAPE), (dict(page_size=48), B.ABQ_ERR_SHAPE), (dict(page_size=8192), B.ABQ_ERR_SHAPE),
              (dict(heads=0), B.ABQ_ERR_SHAPE), (dict(head_dim=8), B.ABQ_ERR_SHAPE), (dict(head_dim=72), B.ABQ_ERR_SHAPE), (dict(head_dim=272), B.ABQ_ERR_SHAPE),
              (dict(heads=1 << 30), B.ABQ_ERR_SHAPE), (dict(page_size=-16), B.ABQ_ERR_SHAPE), (dict(k=A16 + 8), B.ABQ_ERR_ALIGN), (dict(v=A16 + 2), B.ABQ_ERR_ALIGN)]
BAD_CACHES += [(dict(CODES, **{n: 0}), B.ABQ_ERR_NULL) for n in ("k_scale", "k_zero", "v_scale", "v_zero")]
BAD_CACHES += [(dict(CODES, **{n: A16 + 4}), B.ABQ_ERR_ALIGN) for n in ("k_scale", "k_zero", "v_scale", "v_zero")]
BAD_BATCHES = [({n: 0}, B.ABQ_ERR_NULL) for n in ("row_start", "lens", "pages")] + [({n: A16 + 4}, B.ABQ_ERR_ALIGN) for n in ("row_start", "lens", "pages")]
BAD_BATCHES += [({n: v}, B.ABQ_ERR_SHAPE) for n in ("rows", "seqs", "max_pages", "max_new", "max_len") for v in (0, -1)] + [(dict(max_new=9), B.ABQ_ERR_SHAPE), (dict(seqs=65536), B.ABQ_ERR_SHAPE)]


def append(c, b, heads_q=4, r=64, inter=0, freq=A16, q=A16, ldq=256, k=A16, ldk=128, v=A16, ldv=128, out=A16):
    at = lambda s: None if s is None else ctypes.addressof(s)
    return B.load().abq_kv_append(at(c), at(b), heads_q, r, inter, freq, q, ldq, k, ldk, v, ldv, out, None)


def attend(c, b, heads_q=4, q=A16, ldq=256, y=A16, ws=A16, wsb=1 << 30):
    at = lambda s: None if s is None else ctypes.addressof(s)
    return B.load().abq_attn_paged(at(c), at(b), heads_q, q, ldq, 0.1, 1, y, ws, wsb, None)


def read(c, count=3, slots=A16, k=A16, v=A16):
    return B.load().abq_kv_read(None if c is None else ctypes.addressof(c), count, slots, k, v, None)


@pytest.mark.parametrize("bad,want", BAD_CACHES)
def test_caches(bad, want):
    c = cache(**bad)
    assert append(c, batch(), heads_q=4 * max(1, c.heads // 2) if c.heads > 0 else 4) == want
    assert attend(c, batch()) == want and read(c) == want
    assert B.abq_attn_paged_workspace_bytes(c, batch(), 4) == 0


@pytest.mark.parametrize("bad,want", BAD_BATCHES)
def test_batches(bad, want):
    assert append(cache(), batch(**bad)) == want and attend(cache(), batch(**bad)) == want
    assert B.abq_attn_paged_workspace_bytes(cache(), batch(**bad), 4) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(c=None), B.ABQ_ERR_NULL), (dict(b=None), B.ABQ_ERR_NULL), (dict(k=None), B.ABQ_ERR_NULL), (dict(v=None), B.ABQ_ERR_NULL), (dict(out=None), B.ABQ_ERR_NULL),
    (dict(freq=None), B.ABQ_ERR_NULL), (dict(heads_q=3), B.ABQ_ERR_SHAPE), (dict(heads_q=0), B.ABQ_ERR_SHAPE), (dict(r=80), B.ABQ_ERR_SHAPE), (dict(r=24), B.ABQ_ERR_SHAPE),
    (dict(r=-16), B.ABQ_ERR_SHAPE), (dict(ldq=248), B.ABQ_ERR_SHAPE), (dict(ldk=120), B.ABQ_ERR_SHAPE), (dict(ldv=0), B.ABQ_ERR_SHAPE), (dict(ldq=260), B.ABQ_ERR_ALIGN),
    (dict(ldk=132), B.ABQ_ERR_ALIGN), (dict(q=A16 + 2), B.ABQ_ERR_ALIGN), (dict(k=A16 + 8), B.ABQ_ERR_ALIGN), (dict(v=A16 + 8), B.ABQ_ERR_ALIGN), (dict(out=A16 + 8), B.ABQ_ERR_ALIGN),
    (dict(freq=A16 + 4), B.ABQ_ERR_ALIGN)])
def test_append_refuses(kw, want):
    assert append(**{"c": cache(), "b": batch(), **kw}) == want


@pytest.mark.parametrize("kw,want", [
    (dict(c=None), B.ABQ_ERR_NULL), (dict(b=None), B.ABQ_ERR_NULL), (dict(q=None), B.ABQ_ERR_NULL), (dict(y=None), B.ABQ_ERR_NULL), (dict(heads_q=5), B.ABQ_ERR_SHAPE),
    (dict(ldq=128), B.ABQ_ERR_SHAPE), (dict(ldq=257), B.ABQ_ERR_ALIGN), (dict(q=A16 + 2), B.ABQ_ERR_ALIGN), (dict(y=A16 + 2), B.ABQ_ERR_ALIGN), (dict(ws=A16 + 2), B.ABQ_ERR_ALIGN)])
def test_attention_refuses(kw, want):
    assert attend(**{"c": cache(), "b": batch(), **kw}) == want


@pytest.mark.parametrize("kw,want", [(dict(c=None), B.ABQ_ERR_NULL), (dict(slots=None), B.ABQ_ERR_NULL), (dict(k=None), B.ABQ_ERR_NULL), (dict(v=None), B.ABQ_ERR_NULL),
                                     (dict(count=0), B.ABQ_ERR_SHAPE), (dict(slots=A16 + 4), B.ABQ_ERR_ALIGN), (dict(k=A16 + 4), B.ABQ_ERR_ALIGN)])
def test_read_refuses(kw, want):
    assert read(**{"c": cache(), **kw}) == want


GOOD = dict(M=4, N=100, K=60, rank=8, adapters=3, x=A16, ldx=60, ids=A16, a=A16, b=A16, scale=A16, y=A16, ldy=100, out=A16 * 2, ldout=100, ws=A16, wsb=1 << 30)


@pytest.mark.parametrize("kw,want", [({n: None}, B.ABQ_ERR_NULL) for n in ("x", "ids", "a", "b", "scale", "y", "out", "ws")] + [
    ({n: 0}, B.ABQ_ERR_SHAPE) for n in ("M", "N", "K", "rank", "adapters")] + [({n: A16 + 2}, B.ABQ_ERR_ALIGN) for n in ("x", "ids", "a", "b", "scale", "y", "out", "ws")] + [
    (dict(K=B.ABQ_MAX_K + 1, ldx=1 << 20), B.ABQ_ERR_SHAPE), (dict(rank=257), B.ABQ_ERR_SHAPE), (dict(ldx=59), B.ABQ_ERR_SHAPE), (dict(ldy=99), B.ABQ_ERR_SHAPE), (dict(ldout=99), B.ABQ_ERR_SHAPE),
    (dict(out=A16, ldout=104), B.ABQ_ERR_SHAPE), (dict(wsb=16), B.ABQ_ERR_SIZE)])
def test_adapters_refuse(kw, want):
    d = {**GOOD, **kw}
    assert B.load().abq_lora_add(*d.values(), None) == want


def test_workspace_queries():
    assert B.abq_lora_add_workspace_bytes(4, 100, 60, 8) > 0
    for bad in ((0, 100, 60, 8), (4, 0, 60, 8), (4, 100, 0, 8), (4, 100, B.ABQ_MAX_K + 1, 8), (4, 100, 60, 0), (4, 100, 60, 257)):
        assert B.abq_lora_add_workspace_bytes(*bad) == 0
    assert B.abq_attn_paged_workspace_bytes(cache(), batch(), 3) == 0


def half(*s):
    return torch.zeros(s, dtype=torch.float16)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_the_module_refuses_what_is_no_operand():
    """Types, tuples and dimensions; tensors that are not on a device."""
    c, b = (half(4, 2, 16, 64), half(4, 2, 16, 64)), (i32(4), i32(3), i32(3, 5))
    for bad in (list(c), c[:1], c * 2, c[0], None):
        with pytest.raises(TypeError, match="tuple"):
            B.abq_attn_paged(bad, b, half(8, 128), 0.1)
    with pytest.raises(ValueError, match="head_dim"):
        B.abq_kv_read((half(4, 2, 64), half(4, 2, 64)), i32(3))
    with pytest.raises(AssertionError, match="keys: expected a device tensor"):
        B.abq_attn_paged(c, b, half(8, 128), 0.1)
    with pytest.raises(AssertionError, match="x: expected a device tensor"):
        B.abq_lora_add(half(4, 8), i32(4), half(2, 8, 8), half(2, 8, 8), torch.zeros(2), half(4, 8))
    with pytest.raises(TypeError, match="expected a tensor"):
        B.abq_lora_add(7, i32(4), half(2, 8, 8), half(2, 8, 8), torch.zeros(2), half(4, 8))
    with pytest.raises(ValueError, match="two dimensions"):
        B.abq_lora_add(half(8), i32(4), half(2, 8, 8), half(2, 8, 8), torch.zeros(2), half(4, 8))
    with pytest.raises(TypeError, match="missing required argument: 'batch'"):
        B.abq_kv_append(c)
    for call in (lambda **k: B.abq_attn_paged(c, b, half(8, 128), 0.1, **k),):
        for name in ("max_new", "max_len"):
            with pytest.raises(OverflowError):
                call(**{name: 1 << 31})
    with pytest.raises(OverflowError):
        B.abq_lora_add(half(1).expand(1, (1 << 32) + 16), i32(4), half(2, 8, 8), half(2, 8, 8), torch.zeros(2), half(4, 8))


def test_launches_that_no_grid_can_have():
    """Sizes that a tensor could still have, but whose threads would pass 2^32 in one launch."""
    wide, most = dict(heads=1 << 15, head_dim=16), dict(rows=1 << 22, max_new=1)
    assert append(cache(), batch(rows=(1 << 22) + 1)) == attend(cache(), batch(rows=(1 << 22) + 1)) == B.ABQ_ERR_SHAPE
    assert append(cache(**wide), batch(**most), heads_q=1 << 15, ldq=1 << 19, ldk=1 << 19, ldv=1 << 19) == B.ABQ_ERR_SHAPE
    assert attend(cache(**wide), batch(**most), heads_q=1 << 15, ldq=1 << 19) == B.ABQ_ERR_SHAPE
    assert attend(cache(**wide), batch(rows=100, seqs=65), heads_q=1 << 15, ldq=1 << 19) == B.ABQ_ERR_SHAPE
    assert read(cache(), count=(1 << 22) + 1) == B.ABQ_ERR_SHAPE
    assert B.load().abq_lora_add(*{**GOOD, "N": (1 << 28) + 1, "ldy": 1 << 29, "ldout": 1 << 29}.values(), None) == B.ABQ_ERR_SHAPE
    assert B.abq_lora_add_workspace_bytes(4, (1 << 28) + 1, 60, 8) == 0


@pytest.mark.gpu
def test_the_module_refuses_operands_that_do_not_fit(abq):
    """Types, shapes, layouts on the device: refused before anything is launched."""
    dev = lambda t: t.cuda()
    k = dev(half(4, 2, 16, 64))
    c, b, q, kv = (k, k.clone()), tuple(dev(t) for t in (i32(4), i32(3), i32(3, 5))), dev(half(8, 256)), dev(half(8, 128))
    wrong = [((k, k[:3].clone()), b, q), ((k, k.float()), b, q), ((k, k.transpose(1, 2)), b, q), ((k, k.cpu()), b, q), (c, (b[0][:3].contiguous(), *b[1:]), q),
             (c, (b[0], b[1].long(), b[2]), q), (c, (*b[:2], b[2].T), q), (c, b, q.float()), (c, b, q.T), (c, b, q[:, :100].contiguous()),
             ((k, k, dev(torch.zeros(4, 2, 16)), dev(torch.zeros(4, 2, 16)), dev(torch.zeros(4, 2, 16)), dev(torch.zeros(4, 2, 16))), b, q)]
    for args in wrong:
        with pytest.raises((AssertionError, ValueError)):
            abq.abq_attn_paged(*args, 0.1)
    with pytest.raises(AssertionError):
        abq.abq_attn_paged(c, b, q, 0.1, y=dev(half(256, 8)).T)
    with pytest.raises(ValueError):
        abq.abq_attn_paged(c, b, q, 0.1, y=dev(half(8, 128)))
    with pytest.raises(AssertionError):
        abq.abq_attn_paged(c, b, q, 0.1, workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    for args in ((kv, kv[:7]), (kv, q), (q, q)):
        with pytest.raises(ValueError):
            abq.abq_kv_append(c, b, *args)
    with pytest.raises(ValueError, match="q_out"):
        abq.abq_kv_append(c, b, kv, kv, q_out=q)
    with pytest.raises(abq.AbqError) as e:
        abq.abq_kv_append(c, b, kv, kv, inv_freq=torch.zeros(40, device="cuda"))
    assert e.value.status == abq.ABQ_ERR_SHAPE
    with pytest.raises(abq.AbqError) as e:   # rows that overlap each other
        abq.abq_attn_paged(c, b, q[:1].expand(8, 256), 0.1)
    assert e.value.status == abq.ABQ_ERR_SHAPE
    with pytest.raises(abq.AbqError) as e:   # rows off 16-byte boundaries
        abq.abq_attn_paged(c, b, dev(half(8, 260))[:, :256], 0.1)
    assert e.value.status == abq.ABQ_ERR_ALIGN
    with pytest.raises(abq.AbqError) as e:
        abq.abq_attn_paged(c, b, q, 0.1, max_new=9)
    assert e.value.status == abq.ABQ_ERR_SHAPE
    x, ids, a, bb, s, y = dev(half(4, 64)), dev(i32(4)), dev(half(2, 8, 64)), dev(half(2, 96, 8)), dev(torch.zeros(2)), dev(half(4, 96))
    for args in ((x, ids[:3], a, bb, s, y), (x, ids, a[:, :, :32].contiguous(), bb, s, y), (x, ids, a, bb[:, :, :4].contiguous(), s, y), (x, ids, a, bb, s[:1], y),
                 (x, ids, a, bb, s, y[:3]), (x, ids.long(), a, bb, s, y), (x, ids, a.transpose(1, 2), bb, s, y), (x.cpu(), ids, a, bb, s, y)):
        with pytest.raises((AssertionError, ValueError)):
            abq.abq_lora_add(*args)
    with pytest.raises(ValueError):
        abq.abq_lora_add(x, ids, a, bb, s, y, out=dev(half(4, 95)))
