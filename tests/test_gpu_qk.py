"""Norm and rotation of queries and keys, alone (sq_qk_rope) and into the slots
of reserved or drafted tokens (sq_qkv_store), against float64.

Tolerance of a computed value y, a rotated pair (a, b) scaled by r w and mscale:
the angle is exact to 2^-25 of a turn after its reduction in 64 bits and cosine
and sine to 2^-22, the norm's factor and the products take five roundings of
2^-24, all relative to the pair's magnitude, together below 2^-20 of it; then
one rounding to bf16 (2^-8 of y) or to an E4M3 code (2^-4 of y, or 2^-10 of a
step's unit below the smallest normal code)."""

import numpy as np
import pytest

from oracle import draft as odr
from oracle import fp8 as ofp8
from paper_2602_22603_amd import workload as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_22603_amd import sq as sqmod
    sqmod.lib()
    return sqmod


def _inputs(n, hq, hkv, d, seed, gap=0):
    """Views of one projection's rows, `gap` elements between tokens."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (hq + 2 * hkv) * d
    x = torch.randn(n, width + gap, generator=g, device="cuda").to(torch.bfloat16)
    x[:, ::37] *= 8.0
    x = x[:, :width].view(n, hq + 2 * hkv, d) if gap == 0 else x[:, :width].unflatten(1, (hq + 2 * hkv, d))
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _opts(d, rot, interleaved, norm, seed, mscale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    o = dict(interleaved=interleaved, mscale=mscale, eps=1e-6)
    if rot:
        o["inv_freq"] = (1e6 ** (-2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot)).float()
    if "q" in norm:
        o["q_weight"] = 1.0 + 0.25 * torch.randn(d, generator=g, device="cuda")
    if "k" in norm:
        o["k_weight"] = 1.0 + 0.25 * torch.randn(d, generator=g, device="cuda")
    return o


def _want(x, pos, o, which):
    """(value, magnitude its fp32 errors are relative to) in float64."""
    x = x.double().cpu().numpy()
    w = o.get(which + "_weight")
    f = o.get("inv_freq")
    kw = dict(inv_freq=None if f is None else f.cpu().numpy(), weight=None if w is None else w.cpu().numpy(),
              eps=o["eps"], interleaved=o["interleaved"], mscale=o["mscale"])
    y = odr.norm_rotate(x, pos, **kw)
    kw["inv_freq"] = None
    flat = np.abs(odr.norm_rotate(x, pos, **kw))
    mag = flat.copy()
    if f is not None:
        n = len(f)
        i = np.arange(n)
        a, b = (2 * i, 2 * i + 1) if o["interleaved"] else (i, i + n)
        mag[..., a] = mag[..., b] = (flat[..., a] + flat[..., b]) * abs(o["mscale"])
    return y, mag


def _close(got, want, mag, half=2.0 ** -8):
    tol = half * np.abs(want) + (1 + half) * 2.0 ** -20 * mag
    worst = np.abs(got - want) - tol
    assert np.isfinite(got).all() and (worst <= 0).all(), float(worst.max())


CASES = [  # hq, hkv, d, n, rot, interleaved, norm, gap
    (32, 8, 128, 16, 128, False, "qk", 0), (32, 8, 128, 1, 128, False, "qk", 0),
    (64, 8, 64, 37, 32, True, "", 8), (8, 8, 64, 17, 64, False, "k", 0), (16, 2, 128, 130, 64, False, "q", 24),
    (3, 1, 64, 5, 16, False, "qk", 0), (5, 3, 64, 33, 64, True, "qk", 0), (1, 1, 128, 2, 8, True, "qk", 0),
    (7, 5, 128, 15, 0, False, "qk", 16), (4, 4, 64, 300, 40, False, "", 0), (32, 8, 128, 1000, 128, True, "qk", 0)]


@pytest.mark.parametrize("hq,hkv,d,n,rot,interleaved,norm,gap", CASES)
def test_rope_matches_float64(sq, hq, hkv, d, n, rot, interleaved, norm, gap):
    import torch
    q, k, _ = _inputs(n, hq, hkv, d, 7 * n + d, gap)
    o = _opts(d, rot, interleaved, norm, n, mscale=1.25 if n % 2 else 1.0)
    g = torch.Generator().manual_seed(n)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, dtype=torch.int32)
    pos[0] = 0 if n == 1 else (1 << 27) - 1
    qo, ko = sq.qk_rope(q, k, pos.cuda(), **o)
    for got, x, which in ((qo, q, "q"), (ko, k, "k")):
        _close(got.double().cpu().numpy(), *_want(x, pos.numpy(), o, which))


def test_rope_without_options_copies(sq):
    import torch
    q, k, _ = _inputs(21, 8, 2, 64, 3, gap=8)
    pos = torch.arange(21, dtype=torch.int32, device="cuda")
    qo, ko = sq.qk_rope(q, k, pos)
    assert torch.equal(qo, q) and torch.equal(ko, k)


def test_rope_in_place_zero_heads_and_no_tokens(sq):
    """Packed inputs may be the outputs; a head of zeros stays zero; no tokens
    is no work; a token's result does not depend on its neighbours."""
    import torch
    q, k, _ = _inputs(19, 4, 2, 128, 11)
    q, k = q.contiguous(), k.contiguous()
    q[3, 1] = 0
    o = _opts(128, 128, False, "qk", 5)
    pos = (torch.arange(19, dtype=torch.int32, device="cuda") * 999)
    want = sq.qk_rope(q, k, pos, **o)
    assert (want[0][3, 1] == 0).all()
    one = sq.qk_rope(q[7:8], k[7:8], pos[7:8], **o)
    assert torch.equal(one[0][0], want[0][7]) and torch.equal(one[1][0], want[1][7])
    got = sq.qk_rope(q, k, pos, q_out=q, k_out=k, **o)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0] is q
    none = sq.qk_rope(q[:0], k[:0], pos[:0], **o)
    assert none[0].shape == (0, 4, 128)


def test_rope_binding_refusals(sq):
    import torch
    q, k, _ = _inputs(4, 8, 2, 64, 1)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    f = torch.ones(32, device="cuda")
    for bad in (dict(q=q.float()), dict(q=q.transpose(1, 2)), dict(q=q[..., :32]), dict(k=k[:3]), dict(k=k.cpu()),
                dict(positions=pos.long()), dict(positions=pos[:3]), dict(positions=pos.cpu()),
                dict(inv_freq=f.double()), dict(inv_freq=torch.ones(33, device="cuda")), dict(inv_freq=f[:6]),
                dict(inv_freq=f[None]), dict(q_weight=torch.ones(32, device="cuda")), dict(q_out=q),
                dict(k_out=torch.empty(4, 2, 64, device="cuda")), dict(eps=-1.0, inv_freq=f)):
        with pytest.raises(sq.SqError):
            sq.qk_rope(**dict(dict(q=q, k=k, positions=pos), **bad))


def _store(sq, layers, hq, hkv, d, pages, kv8=False, maxp=None):
    return sq.Store(layers, hq, hkv, d, num_pages=pages, max_seqs=8, max_pages_per_seq=maxp or pages,
                    kv_scales=[(0.11, 0.07)] * layers if kv8 else None)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (5, 5, 64), (16, 2, 128), (3, 3, 128)])
def test_store_without_options_is_an_append(sq, hq, hkv, d, kv8):
    """K, V and positions land as sq_append puts them, bit for bit, from
    projections that lie apart, for three sequences at once that start at
    every kind of slot; other slots keep what they held."""
    import torch
    a, b = (_store(sq, 2, hq, hkv, d, 60, kv8) for _ in range(2))
    for s in (a, b):  # the same content in every slot that nobody writes
        s.k_pool.copy_((torch.arange(s.k_pool.numel(), device="cuda") % 97).view(s.k_pool.shape))
        s.v_pool.copy_((torch.arange(s.v_pool.numel(), device="cuda") % 89).view(s.v_pool.shape))
    g = torch.Generator(device="cuda").manual_seed(d)
    for bases, counts in (((0, 5, 31), (40, 11, 1)), ((3, 2, 7), (1, 30, 17)), ((0, 1, 15), (64, 15, 33))):
        seqs = [s.seq_create() for s in (a, b) for _ in range(3)][:3]
        for h, n in zip(seqs, bases):
            kv = torch.randn(2, n, hkv, d, generator=g, device="cuda").to(torch.bfloat16)
            for s in (a, b):
                if n:
                    s.append(h, kv, kv)
        total = sum(counts)
        qs, ks, vs = zip(*[_inputs(total, hq, hkv, d, 10 * i + total, gap=8) for i in range(2)])
        a.reserve(seqs, counts)
        at = 0
        for h, n in zip(seqs, counts):
            b.append(h, torch.stack([k[at:at + n] for k in ks]), torch.stack([v[at:at + n] for v in vs]))
            at += n
        for layer in (1, 0):
            assert torch.equal(a.qkv_store(layer, qs[layer], ks[layer], vs[layer]), qs[layer])
        assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool)
        assert torch.equal(a.pos_pool, b.pos_pool)
        for h in seqs:
            assert a.positions(h).tolist() == b.positions(h).tolist() and a.page_table(h) == b.page_table(h)
            a.release(h), b.release(h)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv,d,base,n,rot,interleaved,norm", [
    (32, 8, 128, 37, 100, 128, False, "qk"), (64, 8, 64, 16, 16, 32, True, "k"), (8, 8, 64, 5, 1, 64, False, "qk"),
    (16, 2, 128, 0, 777, 64, False, "q"), (4, 1, 64, 15, 34, 48, True, "qk")])
def test_store_matches_float64(sq, hq, hkv, d, base, n, rot, interleaved, norm, kv8):
    import torch
    s = _store(sq, 1, hq, hkv, d, 64, kv8)
    h = s.seq_create()
    if base:
        s.append(h, *[wl.device_normal_bf16((1, base, hkv, d), i, "cuda") for i in (1, 2)])
    q, k, v = _inputs(n, hq, hkv, d, n + d)
    o = _opts(d, rot, interleaved, norm, n)
    s.reserve([h], [n])
    qo = s.qkv_store(0, q, k, v, **o)
    pos = base + np.arange(n)
    _close(qo.double().cpu().numpy(), *_want(q, pos, o, "q"))
    table = torch.tensor(s.page_table(h), device="cuda")
    at = torch.arange(base, base + n, device="cuda")
    kp = s.k_pool[0][:, table[at // 16], at % 16].transpose(0, 1)
    vp = s.v_pool[0][:, table[at // 16], :, at % 16]
    assert s.pos_pool[table[at // 16], at % 16].tolist() == pos.tolist()
    want, mag = _want(k, pos, o, "k")
    if not kv8:
        _close(kp.double().cpu().numpy(), want, mag)
        assert torch.equal(vp, v)
        return
    got = ofp8.decode(kp.cpu().numpy())
    inv = np.float64(ofp8.inv_scale(0.11))
    want, mag = np.clip(want * inv, -448, 448), mag * inv
    tol = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + (1 + 2.0 ** -4) * 2.0 ** -20 * mag
    assert (np.abs(got - want) <= tol).all()
    assert (ofp8.quantize(v.float().cpu().numpy(), 0.07) == vp.cpu().numpy()).all()


def test_store_replays_from_a_capture(sq):
    """One capture of a layer's call replays for later chunks of the same
    counts, whatever slots they start at, each checked against an eager call
    in another store."""
    import torch
    a, b = (_store(sq, 1, 8, 2, 128, 80) for _ in range(2))
    seqs = [a.seq_create(), a.seq_create()]
    assert [b.seq_create(), b.seq_create()] == seqs
    counts = [19, 3]
    q, k, v = (x.contiguous() for x in _inputs(22, 8, 2, 128, 2))
    o = _opts(128, 128, False, "qk", 2)
    qo = torch.empty_like(q)
    a.reserve(seqs, counts)
    a.qkv_store(0, q, k, v, q_out=qo, **o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.qkv_store(0, q, k, v, q_out=qo, **o)
    b.reserve(seqs, counts)
    b.qkv_store(0, q, k, v, **o)
    for i in range(4):
        for x, y in zip((q, k, v), _inputs(22, 8, 2, 128, 50 + i)):
            x.copy_(y)
        for s in (a, b):
            s.reserve(seqs, counts)
        graph.replay()
        want = b.qkv_store(0, q, k, v, **o)
        torch.cuda.synchronize()
        assert torch.equal(qo, want)
        assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool)
        assert torch.equal(a.pos_pool, b.pos_pool)


def test_store_refusals(sq):
    import torch
    s = _store(sq, 1, 8, 2, 64, 16)
    h = s.seq_create()
    q, k, v = _inputs(4, 8, 2, 64, 1)
    with pytest.raises(sq.SqError):
        s.qkv_store(0, q, k, v)
    s.reserve([h], [4])
    for bad in (dict(layer=1), dict(layer=-1), dict(q=q[:3]), dict(k=k[:, :1]), dict(v=v.float()),
                dict(q_out=torch.empty(4, 8, 64, device="cuda")), dict(q=q.cpu())):
        with pytest.raises(sq.SqError):
            s.qkv_store(**dict(dict(layer=0, q=q, k=k, v=v), **bad))
    s.qkv_store(0, q, k, v)
    s.qkv_store(0, q, k, v)  # again is fine
    s.append(h, k[None].contiguous(), v[None].contiguous())
    with pytest.raises(sq.SqError):  # the store changed since
        s.qkv_store(0, q, k, v)
