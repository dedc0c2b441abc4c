"""A window with the sequence's first tokens visible beside it
(sq_attn_opts.first) in decode (every mode), decode steps and extend (every
tile, split and not), against float64.  Tolerance 5e-4, as for every attention
output from N(0, 1) inputs."""

import math

import pytest

from paper_2602_22603_amd import workload as wl

pytestmark = pytest.mark.gpu
TOL = 5e-4


@pytest.fixture(scope="module")
def sq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_22603_amd import sq as sqmod
    sqmod.lib()
    return sqmod


def _attend(q, k, v, base, window, first, sinks):
    """Row j of q at index base + j, in float64."""
    import torch
    n, hq, d = q.shape
    here = base + torch.arange(n, device="cuda")[:, None]
    t = torch.arange(k.shape[0], device="cuda")[None]
    mask = (t <= here) & ((t > here - window) | (t < first))
    out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    for h in range(hq):
        g = h // (hq // k.shape[1])
        s = (q[:, h].double() @ k[:, g].double().T.contiguous()) / math.sqrt(d)
        s = s.masked_fill(~mask, -math.inf)
        if sinks is not None:
            s = torch.cat([s, sinks[h].double().expand(n, 1)], 1)
        out[:, h] = torch.softmax(s, 1)[:, :k.shape[0]] @ v[:, g].double().contiguous()
    return out


def _sinks(hq):
    import torch
    return torch.randn(hq, generator=torch.Generator().manual_seed(hq)).cuda()


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 2, 64), (64, 8, 64), (4, 4, 128)])
@pytest.mark.parametrize("window,first", [(1, 1), (5, 4), (16, 16), (17, 3), (100, 64), (100, 131), (40, 650),
                                          (5000, 4), (30, 10 ** 6)])
def test_decode(sq, hq, hkv, d, window, first):
    """Caches shorter than the first tokens, first tokens that meet the window,
    ends inside and at the edges of pages, an empty sequence, every mode."""
    import torch
    s = sq.Store(1, hq, hkv, d, num_pages=220, max_seqs=8, max_pages_per_seq=60)
    seqs, kv, lengths = [], [], [700, 47, 1, 0, 641, 144]
    for i, n in enumerate(lengths):
        h = s.seq_create()
        k, v = (wl.device_normal_bf16((1, n, hkv, d), 10 * i + j + hq, "cuda") for j in (0, 1))
        if n:
            s.append(h, k, v)
        seqs.append(h), kv.append((k, v))
    q = wl.device_normal_bf16((len(seqs), hq, d), 77, "cuda")
    for mode in (sq.ATTN_AUTO, sq.ATTN_STREAM, sq.ATTN_SHARED_PREFIX, sq.ATTN_MFMA):
        for sinks in (None, _sinks(hq)):
            got = s.decode(0, seqs, q, mode=mode, window=window, first=first, sinks=sinks)
            for i, n in enumerate(lengths):
                want = _attend(q[i:i + 1], kv[i][0][0], kv[i][1][0], n - 1, window, first, sinks) if n else 0
                assert (got[i].double() - want).abs().max() <= TOL, (mode, i)


def test_decode_batch_of_many_on_an_8bit_store(sq):
    """64 entries of two segments each, the most a call may have."""
    from oracle import fp8 as ofp8
    import torch
    s = sq.Store(1, 8, 2, 128, num_pages=64 * 20, max_seqs=64, max_pages_per_seq=20, kv_scales=[(0.11, 0.07)])
    seqs, kv = [], []
    for i in range(64):
        h = s.seq_create()
        k, v = (wl.device_normal_bf16((1, 100 + 3 * i, 2, 128), 2 * i + j, "cuda") for j in (0, 1))
        s.append(h, k, v)
        seqs.append(h)
        kv.append([torch.from_numpy(ofp8.roundtrip(x[0].float().cpu().numpy(), sc)).cuda() for x, sc in ((k, 0.11), (v, 0.07))])
    q = wl.device_normal_bf16((64, 8, 128), 5, "cuda")
    got = s.decode(0, seqs, q, window=33, first=20)
    for i in range(64):
        want = _attend(q[i:i + 1], *kv[i], 99 + 3 * i, 33, 20, None)
        assert (got[i].double() - want).abs().max() <= TOL


@pytest.mark.parametrize("window,first", [(1, 1), (8, 4), (64, 64), (33, 500)])
def test_steps(sq, window, first):
    """Windowed and full layers of one step, eager and replayed; then a step
    without a window, whose plan must not keep the windowed one."""
    import torch
    hq, hkv, d = 16, 4, 64
    s = sq.Store(2, hq, hkv, d, num_pages=80, max_seqs=3, max_pages_per_seq=40)
    seqs, kv = [], []
    for i, n in enumerate((300, 15, 0)):
        h = s.seq_create()
        k, v = (wl.device_normal_bf16((2, n, hkv, d), 10 * i + j, "cuda") for j in (0, 1))
        if n:
            s.append(h, k, v)
        seqs.append(h), kv.append([k, v])
    kn, vn = (torch.empty(2, 3, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.empty(2, 3, hq, d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(2, 3, hq, d, device="cuda")
    sinks = _sinks(hq)

    def layers():
        s.step_attn(0, kn[0], vn[0], q[0], out=out[0], window=window, first=first, sinks=sinks)
        s.step_attn(1, kn[1], vn[1], q[1], out=out[1])

    graph = None
    for turn in range(6):
        for x, seed in ((kn, 1), (vn, 2), (q, 3)):
            x.copy_(wl.device_normal_bf16(tuple(x.shape), 100 * turn + seed, "cuda"))
        s.step_begin(seqs, window=window, first=first)
        if graph is None:
            layers()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                layers()
            out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i in range(3):
            for j, new in enumerate((kn, vn)):
                kv[i][j] = torch.cat([kv[i][j], new[:, i:i + 1]], 1)
            n = kv[i][0].shape[1]
            for layer, (w, f, sk) in enumerate(((window, first, sinks), (10 ** 6, 0, None))):
                want = _attend(q[layer, i:i + 1], kv[i][0][layer], kv[i][1][layer], n - 1, w, f, sk)
                assert (out[layer, i].double() - want).abs().max() <= TOL, (turn, i, layer)
    s.step_begin(seqs, window=window, first=first)
    with pytest.raises(sq.SqError):
        s.step_attn(0, kn[0], vn[0], q[0], window=window, first=first + 1)
    with pytest.raises(sq.SqError):
        s.step_attn(0, kn[0], vn[0], q[0], window=window + 1, first=first)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv,d,base,n", [
    (32, 8, 128, 2000, 300), (32, 8, 128, 3000, 9), (8, 8, 64, 500, 700), (64, 8, 64, 1500, 33), (16, 8, 128, 0, 400),
    (4, 4, 128, 777, 1), (8, 1, 128, 900, 64)])
@pytest.mark.parametrize("window,first", [(1, 1), (64, 4), (100, 64), (129, 131), (700, 65), (10 ** 6, 4), (20, 10 ** 6)])
def test_extend(sq, hq, hkv, d, base, n, window, first, kv8):
    import torch
    s = sq.Store(1, hq, hkv, d, num_pages=240, max_seqs=1, max_pages_per_seq=240,
                 kv_scales=[(0.11, 0.07)] if kv8 else None)
    h = s.seq_create()
    k, v = (wl.device_normal_bf16((1, base + n, hkv, d), j + hq + n, "cuda") for j in (0, 1))
    s.append(h, k, v)
    if kv8:
        from oracle import fp8 as ofp8
        k, v = (torch.from_numpy(ofp8.roundtrip(x.float().cpu().numpy(), sc)).cuda() for x, sc in ((k, 0.11), (v, 0.07)))
    q = wl.device_normal_bf16((n, hq, d), 9, "cuda")
    for sinks in (None, _sinks(hq)):
        got = s.extend(0, h, q, window=window, first=first, sinks=sinks)
        want = _attend(q, k[0], v[0], base, window, first, sinks)
        assert (got.double() - want).abs().max() <= TOL


def test_extend_split_over_a_long_cache(sq):
    """Few rows over a wide window and many first tokens: the list of key blocks
    is split, over the gap too."""
    s = sq.Store(1, 32, 8, 128, num_pages=1300, max_seqs=1, max_pages_per_seq=1300)
    h = s.seq_create()
    k, v = (wl.device_normal_bf16((1, 20005, 8, 128), j, "cuda") for j in (0, 1))
    s.append(h, k, v)
    for n, window, first in ((5, 8000, 3001), (77, 5000, 4), (200, 300, 9000)):
        q = wl.device_normal_bf16((n, 32, 128), n, "cuda")
        got = s.extend(0, h, q, window=window, first=first)
        assert (got.double() - _attend(q, k[0], v[0], 20005 - n, window, first, None)).abs().max() <= TOL


def test_refusals(sq):
    s = sq.Store(1, 8, 2, 64, num_pages=8, max_seqs=2, max_pages_per_seq=4)
    h = s.seq_create()
    k = wl.device_normal_bf16((1, 20, 2, 64), 1, "cuda")
    s.append(h, k, k)
    q = wl.device_normal_bf16((1, 8, 64), 2, "cuda")
    for f in (lambda: s.decode(0, [h], q, window=4, first=-1), lambda: s.extend(0, h, q, window=4, first=-1),
              lambda: s.step_begin([h], window=4, first=-2)):
        with pytest.raises(sq.SqError):
            f()
    s.span_mark(h, 0, 2, 5)
    s.evict(h, [0], deferred=True)
    with pytest.raises(sq.SqError):
        s.decode(0, [h], q, window=4, first=1)
