"""Drafted trees (sq_draft_begin, sq_draft_attn, sq_draft_accept) against
float64: every head shape, trees of 1 to 64 nodes over caches of no token to
100 thousand, windows with first tokens, sinks, 8-bit stores, masked slots,
branches; the accepted path's K, V and positions bit for bit; whole
verification steps; captures.

Tolerances, for values v of at most V in magnitude: a weight is held to 2^-17
(two bf16 halves), its exponent to the error of a score, whose D products of
bf16 pairs are exact and summed in fp32, below 2 D 2^-24 sum |q_i k_i| scale;
with N(0, 1) inputs the sum is below 1.5 sqrt(D) / scale, so one output is
within V (2^-16 + 3 D^1.5 2^-24): 3e-4 V at D = 128, and a row's errors, which
are of either sign, within 1e-5 of the output in the 2-norm (weights alone:
2^-18 rms)."""

import math
import random

import numpy as np
import pytest

from oracle import draft as odr
from oracle import fp8 as ofp8
from paper_2602_22603_amd import workload as wl

pytestmark = pytest.mark.gpu
SCALES = (0.11, 0.07)


@pytest.fixture(scope="module")
def sq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_22603_amd import sq as sqmod
    sqmod.lib()
    return sqmod


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    import gc
    import torch
    gc.collect()
    torch.cuda.empty_cache()


def _tree(rng, n, back=6):
    return [-1] + [rng.randrange(max(-1, i - back), i) for i in range(1, n)]


def _held(x, kv8, which):
    """What a store holds of bf16 x, in float64 on the device."""
    import torch
    if not kv8:
        return x.double()
    y = torch.from_numpy(ofp8.roundtrip(x.float().cpu().numpy(), SCALES[which]))
    return y.to(x.device)


def _attend(q, k, v, parents, window=0, first=0, sinks=None, keep=None):
    """The definition in float64 on the device: q [n, Hq, D], k, v [L + n, Hkv, D]."""
    import torch
    n, hq, d = q.shape
    length, hkv = k.shape[0] - n, k.shape[1]
    mask = torch.zeros(n, length + n, dtype=torch.bool, device=q.device)
    here = torch.tensor(odr.depths(parents), device=q.device) + length
    t = torch.arange(length, device=q.device)
    seen = torch.ones(n, length, dtype=torch.bool, device=q.device)
    if window:
        seen = (t[None] > here[:, None] - window) | (t[None] < first)
    if keep is not None:
        seen = seen & keep[None]
    mask[:, :length] = seen
    for i in range(n):
        for depth, node in enumerate(odr.path_to(parents, i)):
            index = length + depth
            mask[i, length + node] = not window or index > int(here[i]) - window or index < first
    out = torch.empty(n, hq, d, dtype=torch.float64, device=q.device)
    for h in range(hq):
        g = h // (hq // hkv)
        s = (q[:, h].double() @ k[:, g].T.contiguous()) / math.sqrt(d)
        s = s.masked_fill(~mask, -math.inf)
        if sinks is not None:
            s = torch.cat([s, sinks[h].double().expand(n, 1)], 1)
        out[:, h] = torch.softmax(s, 1)[:, :length + n] @ v[:, g].contiguous()
    return out


def _check(got, want, vmax, d):
    import torch
    err = (got.double() - want).abs().max().item()
    rel = (torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want)).item()
    assert torch.isfinite(got).all()
    assert err <= vmax * (2.0 ** -16 + 3 * d ** 1.5 * 2.0 ** -24), err
    assert rel <= 1e-5, rel


class Batch:
    """Sequences of given lengths with a tree behind each, one or more layers."""

    def __init__(self, sq, hq, hkv, d, lengths, sizes, kv8=False, layers=1, seed=0, poison=False, extra=4):
        import torch
        self.sq, self.kv8, self.d, self.hkv, self.layers = sq, kv8, d, hkv, layers
        rng = random.Random(seed)
        pages = sum(-(-(a + b) // 16) for a, b in zip(lengths, sizes)) + extra
        self.s = sq.Store(layers, hq, hkv, d, num_pages=pages, max_seqs=len(lengths) + 4,
                          max_pages_per_seq=-(-(max(lengths) + 64) // 16) + 2,
                          kv_scales=[SCALES] * layers if kv8 else None)
        if poison:  # slots that hold no token hold NaN
            self.s.k_pool.fill_(0x7F if kv8 else math.nan)
            self.s.v_pool.fill_(0x7F if kv8 else math.nan)
        self.trees = [_tree(rng, n) for n in sizes]
        self.seqs, self.k, self.v = [], [], []
        for i, (a, n) in enumerate(zip(lengths, sizes)):
            h = self.s.seq_create()
            k, v = (wl.device_normal_bf16((layers, a + n, hkv, d), 1000 * seed + 2 * i + j, "cuda") for j in (0, 1))
            if a:
                self.s.append(h, k[:, :a].contiguous(), v[:, :a].contiguous())
            self.seqs.append(h), self.k.append(k), self.v.append(v)
        self.lengths, self.sizes = lengths, sizes
        self.q = wl.device_normal_bf16((layers, sum(sizes), hq, d), 1000 * seed + 999, "cuda")
        self.sinks = torch.randn(hq, generator=torch.Generator().manual_seed(seed)).cuda()

    def nodes(self, x, layer):
        import torch
        return torch.cat([t[layer, a:] for t, a in zip(x, self.lengths)])

    def begin(self, **kw):
        self.s.draft_begin(self.seqs, self.trees, **kw)
        for layer in range(self.layers):
            self.s.qkv_store(layer, self.q[layer], self.nodes(self.k, layer), self.nodes(self.v, layer))

    def want(self, layer=0, window=0, first=0, sinks=None, keeps=None):
        import torch
        out, at = [], 0
        for b, n in enumerate(self.sizes):
            out.append(_attend(self.q[layer, at:at + n], _held(self.k[b][layer], self.kv8, 0),
                               _held(self.v[b][layer], self.kv8, 1), self.trees[b], window, first, sinks,
                               None if keeps is None else keeps[b]))
            at += n
        return torch.cat(out)

    def check(self, layer=0, window=0, first=0, sinks=False, keeps=None):
        s = self.sinks if sinks else None
        got = self.s.draft_attn(layer, self.q[layer], window=window, first=first, sinks=s)
        vmax = max(x.abs().max().item() for x in self.v)
        _check(got, self.want(layer, window, first, s, keeps), vmax, self.d)
        return got


HEADS = [(32, 8, 128), (8, 8, 64), (64, 8, 64), (8, 1, 128), (4, 2, 64), (5, 5, 128)]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_trees_over_ragged_caches(sq, hq, hkv, d, kv8):
    """Caches that end at every kind of slot, none among them, trees of 1 to 64
    nodes whose rows need every tile, NaN in the slots that hold nothing."""
    lengths = [0, 1, 15, 16, 63, 64, 65, 200, 1000, 130]
    for most in (64, 16, 7):
        sizes = [min(most, n) for n in (64, 1, 2, 33, 16, 17, 64, 5, 63, 31)]
        b = Batch(sq, hq, hkv, d, lengths, sizes, kv8, seed=most, poison=True)
        b.begin()
        b.check()
        b.check(sinks=True)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("sizes", [[40, 33, 48, 36], [64, 60, 64, 56], [33, 64, 34, 35]])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (16, 2, 64)])
def test_trees_of_more_rows_than_a_tile(sq, hq, hkv, d, sizes, kv8):
    """Every tree needs more than 128 rows, its last tile full, half full or
    nearly empty."""
    b = Batch(sq, hq, hkv, d, [0, 1111, 64, 5003], sizes, kv8, seed=sum(sizes), poison=True)
    b.begin(window=700, first=70)
    b.check(sinks=True)
    b.check(window=700, first=70)


@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (5, 0), (5, 4), (64, 1), (64, 64), (100, 131), (300, 4),
                                          (5000, 4), (16, 3000)])
@pytest.mark.parametrize("hq,hkv,d,kv8", [(32, 8, 128, False), (64, 8, 64, True), (4, 4, 64, False)])
def test_windows_and_first_tokens(sq, hq, hkv, d, kv8, window, first):
    """A window counts along each node's own path; windowed and full layers of
    one draft."""
    lengths, sizes = [0, 3, 64, 200, 777, 1500], [64, 20, 33, 64, 7, 18]
    b = Batch(sq, hq, hkv, d, lengths, sizes, kv8, seed=window + first, poison=True)
    b.begin(window=window, first=first)
    got = b.check(window=window, first=first, sinks=True)
    b.check(window=window, first=first)
    b.check()
    if window == 1 and first == 0 and not kv8:  # each node sees itself alone
        v = b.nodes(b.v, 0).double().repeat_interleave(hq // hkv, 1)
        s = b.sinks[None, :, None].double()
        k = b.nodes(b.k, 0).double().repeat_interleave(hq // hkv, 1)
        dot = (b.q[0].double() * k).sum(-1, keepdim=True) / math.sqrt(d)
        assert ((got.double() - v * (1 / (1 + (s - dot).exp()))).abs().max() < 1e-5)


@pytest.mark.parametrize("hq,hkv,d,kv8,lengths,sizes", [
    (32, 8, 128, False, [100003], [64]), (32, 8, 128, True, [50001, 33, 7000], [3, 64, 40]),
    (8, 1, 128, False, [70001], [5]), (64, 8, 64, False, [20011, 20011], [24, 64]), (8, 8, 64, False, [30000], [1])])
def test_long_caches_are_split_and_joined(sq, hq, hkv, d, kv8, lengths, sizes):
    b = Batch(sq, hq, hkv, d, lengths, sizes, kv8, seed=3)
    b.begin(window=4000, first=100)
    b.check(sinks=True)
    b.check(window=4000, first=100)


def test_large_scores_raise_the_reference(sq):
    """Keys 64 times as large late in the cache: weights overflow the reference
    that the early keys set."""
    import torch
    b = Batch(sq, 8, 2, 128, [0], [64], seed=9)
    k = wl.device_normal_bf16((1, 700, 2, 128), 1, "cuda")
    k[:, 300:] *= 64
    v = wl.device_normal_bf16((1, 700, 2, 128), 2, "cuda")
    s = sq.Store(1, 8, 2, 128, num_pages=60, max_seqs=2, max_pages_per_seq=60)
    h = s.seq_create()
    s.append(h, k[:, :636].contiguous(), v[:, :636].contiguous())
    s.draft_begin([h], b.trees)
    s.qkv_store(0, b.q[0], k[0, 636:], v[0, 636:])
    got = s.draft_attn(0, b.q[0])
    want = _attend(b.q[0], k[0].double(), v[0].double(), b.trees[0])
    # scores up to a few thousand: fp32 holds them to 2^-13
    assert torch.isfinite(got).all() and (got.double() - want).abs().max() < 2.0 ** -10 * v.abs().max()


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64)])
def test_a_chain_is_an_appended_chunk(sq, hq, hkv, d):
    """A draft without branches sees what extend's chunk sees."""
    import torch
    b = Batch(sq, hq, hkv, d, [333, 40], [50, 64], seed=4)
    b.trees = [[-1] + list(range(n - 1)) for n in b.sizes]
    b.begin()
    got = b.check()
    s = sq.Store(1, hq, hkv, d, num_pages=64, max_seqs=2, max_pages_per_seq=40)
    at = 0
    for k, v, n in zip(b.k, b.v, b.sizes):
        h = s.seq_create()
        s.append(h, k, v)
        want = s.extend(0, h, b.q[0, at:at + n].contiguous())
        assert torch.linalg.vector_norm(got[at:at + n] - want) <= 2e-5 * torch.linalg.vector_norm(want)
        at += n


@pytest.mark.parametrize("kv8", [False, True])
def test_masked_slots_evictions_and_branches(sq, kv8):
    """Slots that deferred evictions masked are skipped; after a compaction, and
    on a branch beside its parent, the trees see what is left."""
    import torch
    b = Batch(sq, 16, 2, 128, [500, 333], [33, 64], kv8, seed=8, extra=90)
    s = b.s
    keeps = [torch.ones(n, dtype=torch.bool, device="cuda") for n in b.lengths]
    for i, (lo, hi) in enumerate([(3, 40), (64, 192), (450, 490)]):
        s.span_mark(b.seqs[0], i, lo, hi)
        keeps[0][lo:hi] = False
    s.evict(b.seqs[0], [0, 1, 2], deferred=True)
    b.begin()
    b.check(keeps=keeps, sinks=True)
    s.draft_accept([[], []])
    s.compact(b.seqs[0])
    n, m = int(keeps[0].sum()), b.lengths[0]
    for x in (b.k, b.v):
        x[0] = torch.cat([x[0][:, :m][:, keeps[0]], x[0][:, m:]], 1)
    b.lengths[0] = n
    child = s.fork(b.seqs[1], 111)
    b.seqs.append(child), b.trees.append([-1, 0, 0]), b.lengths.append(111), b.sizes.append(3)
    for x, seed in ((b.k, 71), (b.v, 72)):
        x.append(torch.cat([x[1][:, :111], wl.device_normal_bf16((1, 3, 2, 128), seed, "cuda")], 1))
    b.q = torch.cat([b.q, wl.device_normal_bf16((1, 3, 16, 128), 73, "cuda")], 1)
    b.begin(window=99, first=5)
    b.check()
    b.check(window=99, first=5)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hkv,d,layers", [(2, 128, 3), (3, 64, 2)])
def test_accept_moves_the_path_bit_for_bit(sq, hkv, d, layers, kv8):
    """K, V and positions of random paths (none, all of a chain, a root, deep
    ones) equal those of the same tokens appended; nothing else of the pools
    changes; pages come back; twice in a row."""
    import torch
    rng = random.Random(d)
    lengths, sizes = [0, 5, 16, 30, 61, 100, 7], [64, 1, 40, 64, 17, 33, 64]
    b = Batch(sq, hkv, hkv, d, lengths, sizes, kv8, layers, seed=d)
    b.trees[3] = [-1] + list(range(63))
    b.trees[5] = _tree(rng, 33, back=2)
    s = b.s
    for turn in range(2):
        b.begin()
        paths = [odr.path_to(t, rng.randrange(len(t) // 2, len(t))) for t in b.trees]
        if turn == 0:
            paths[1], paths[2], paths[3] = [], [0], list(range(64))
        before = s.k_pool.clone(), s.v_pool.clone(), s.pos_pool.clone()
        tables = [s.page_table(h) for h in b.seqs]
        s.draft_accept(paths)
        for i, (h, p) in enumerate(zip(b.seqs, paths)):
            base, table = b.lengths[i], torch.tensor(tables[i], device="cuda")
            assert s.positions(h).tolist() == list(range(base + len(p)))
            assert s.page_table(h) == tables[i][:-(-(base + len(p)) // 16)]
            src = base + torch.tensor(p, device="cuda", dtype=torch.long)
            dst = base + torch.arange(len(p), device="cuda")
            sp, ss, dp, ds = table[src // 16], src % 16, table[dst // 16], dst % 16
            old = before[0].clone(), before[1].clone()
            before[0][:, :, dp, ds] = old[0][:, :, sp, ss]
            before[1][:, :, dp, :, ds] = old[1][:, :, sp, :, ss]
            before[2][dp, ds] = dst.to(torch.int32)
            for x in (b.k, b.v):
                x[i] = torch.cat([x[i][:, :base], x[i][:, src], wl.device_normal_bf16(
                    (layers, b.sizes[i], hkv, d), 31 * turn + i + (7 if x is b.v else 0), "cuda")], 1)
            b.lengths[i] = base + len(p)
        assert torch.equal(s.k_pool, before[0]) and torch.equal(s.v_pool, before[1])
        assert torch.equal(s.pos_pool, before[2])
        need = sum(-(-n // 16) for n in b.lengths)
        assert s.stats()["live_pages"] == need
        room = sum(-(-(n + m) // 16) for n, m in zip(b.lengths, b.sizes))
        if room > s.num_pages:
            break
    for layer in range(layers):  # what is cached now attends as the tokens do
        for i, h in enumerate(b.seqs):
            if b.lengths[i]:
                q = wl.device_normal_bf16((1, hkv, d), i, "cuda")
                n = b.lengths[i]
                k, v = (_held(x[i][layer, :n], kv8, w) for w, x in enumerate((b.k, b.v)))
                want = _attend(q, k, v, [-1])  # (the last token is the query's own)
                _check(s.decode(layer, [h], q), want, v.abs().max().item(), d)


def test_verification_steps_as_a_model_runs_them(sq):
    """Three turns of two layers: a chunk reserved, stored and attended; a draft
    begun, stored with norm and rotation, attended, a path kept; a decode step
    on top - each checked against float64 over the tokens kept so far."""
    import torch
    hq, hkv, d, layers = 16, 4, 128, 2
    s = sq.Store(layers, hq, hkv, d, num_pages=120, max_seqs=3, max_pages_per_seq=60)
    seqs = [s.seq_create(), s.seq_create()]
    freq = (1e4 ** (-torch.arange(64, device="cuda", dtype=torch.float64) / 64)).float()
    opts = [dict(inv_freq=freq, q_weight=1 + 0.1 * torch.randn(d, device="cuda"),
                 k_weight=1 + 0.1 * torch.randn(d, device="cuda")) for _ in range(layers)]
    kept = [[(torch.zeros(0, hkv, d, device="cuda", dtype=torch.float64),) * 2 for _ in seqs] for _ in range(layers)]
    rng = random.Random(1)

    def project(n, seed):
        x = wl.device_normal_bf16((layers, n, hq + 2 * hkv, d), seed, "cuda")
        return [x[i].split([hq, hkv, hkv], 1) for i in range(layers)]

    def rotated(layer, k, pos):
        one = torch.zeros(k.shape[0], 1, d, dtype=torch.bfloat16, device="cuda")
        return sq.qk_rope(one, k, pos, **opts[layer])[1]

    for turn in range(3):
        ns = [5 + 11 * turn, 1]
        s.reserve(seqs, ns)
        for layer, (q, k, v) in enumerate(project(sum(ns), turn)):
            qr = s.qkv_store(layer, q, k, v, **opts[layer])
            at = 0
            for i, (h, n) in enumerate(zip(seqs, ns)):
                pos = torch.arange(len(kept[layer][i][0]), len(kept[layer][i][0]) + n, device="cuda", dtype=torch.int32)
                kk = torch.cat([kept[layer][i][0], rotated(layer, k[at:at + n], pos).double()])
                vv = torch.cat([kept[layer][i][1], v[at:at + n].double()])
                kept[layer][i] = (kk, vv)
                got = s.extend(layer, h, qr[at:at + n].contiguous())
                _check(got, _attend(qr[at:at + n], kk, vv, [-1] + list(range(n - 1))), 6.0, d)
                at += n
        trees = [_tree(rng, 20 + turn), _tree(rng, 3)]
        s.draft_begin(seqs, trees)
        paths = [odr.path_to(t, len(t) - 1) for t in trees]
        for layer, (q, k, v) in enumerate(project(sum(map(len, trees)), 100 + turn)):
            qr = s.qkv_store(layer, q, k, v, **opts[layer])
            got = s.draft_attn(layer, qr)
            at = 0
            for i, t in enumerate(trees):
                n, base = len(t), len(kept[layer][i][0])
                pos = torch.tensor([base + x for x in odr.depths(t)], device="cuda", dtype=torch.int32)
                kn = rotated(layer, k[at:at + n], pos).double()
                vn = v[at:at + n].double()
                _check(got[at:at + n], _attend(qr[at:at + n], torch.cat([kept[layer][i][0], kn]),
                                               torch.cat([kept[layer][i][1], vn]), t), 6.0, d)
                kept[layer][i] = (torch.cat([kept[layer][i][0], kn[paths[i]]]),
                                  torch.cat([kept[layer][i][1], vn[paths[i]]]))
                at += n
        s.draft_accept(paths)
        s.step_begin(seqs)
        for layer, (q, k, v) in enumerate(project(2, 200 + turn)):
            pos = torch.tensor([len(kept[layer][i][0]) for i in range(2)], device="cuda", dtype=torch.int32)
            qr, kr = sq.qk_rope(q, k, pos, **opts[layer])
            got = s.step_attn(layer, kr, v.contiguous(), qr)
            for i in range(2):
                kept[layer][i] = (torch.cat([kept[layer][i][0], kr[i:i + 1].double()]),
                                  torch.cat([kept[layer][i][1], v[i:i + 1].double()]))
                _check(got[i:i + 1], _attend(qr[i:i + 1], *kept[layer][i], [-1]), 6.0, d)
    for i, h in enumerate(seqs):
        assert s.positions(h).tolist() == list(range(len(kept[0][i][0])))


def test_captured_layer_replays_for_later_drafts(sq):
    """One capture of a layer (windowed and full attention) replays for later
    drafts of the same counts over caches that have grown, with eager work
    between, each replay equal to the eager calls."""
    import torch
    counts = [20, 7]
    b = Batch(sq, 16, 4, 128, [100, 1900], counts, seed=5, extra=40)
    s = b.s
    kn, vn = b.nodes(b.k, 0).contiguous(), b.nodes(b.v, 0).contiguous()
    q = b.q[0].clone()
    out, outw = (torch.zeros(27, 16, 128, device="cuda") for _ in range(2))

    def layer(stored, full, windowed):
        s.qkv_store(0, q, kn, vn, q_out=stored)
        s.draft_attn(0, stored, out=full)
        s.draft_attn(0, stored, out=windowed, window=50, first=3, sinks=b.sinks)

    stored = torch.empty_like(q)
    s.draft_begin(b.seqs, b.trees, window=50, first=3)
    layer(stored, out, outw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(stored, out, outw)
    rng = random.Random(2)
    for i in range(4):
        s.draft_accept([odr.path_to(t, len(t) - 1) for t in b.trees] if i % 2 else [[], []])
        if i == 2:
            s.append(b.seqs[0], *[wl.device_normal_bf16((1, 300, 4, 128), 60 + j, "cuda") for j in (0, 1)])
        b.trees = [_tree(rng, n) for n in counts]
        s.draft_begin(b.seqs, b.trees, window=50, first=3)
        for x, y in ((q, 1), (kn, 2), (vn, 3)):
            x.copy_(wl.device_normal_bf16(tuple(x.shape), 10 * i + y, "cuda"))
        out.zero_(), outw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, wantw = torch.empty_like(out), torch.empty_like(outw)
        layer(torch.empty_like(q), want, wantw)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(outw, wantw) and out.abs().sum() > 0


def test_a_capture_takes_no_call_that_moves_slots(sq):
    """reserve, draft_begin, draft_accept and truncate are refused in a capture,
    changing nothing and leaving the capture whole."""
    import torch
    b = Batch(sq, 8, 2, 64, [50], [5], seed=1)
    s, h = b.s, b.seqs[0]
    x = torch.zeros(4, device="cuda")
    for call in (lambda: s.reserve([h], [3]), lambda: s.draft_begin([h], [[-1]]), lambda: s.truncate(h, 20),
                 lambda: s.draft_accept([[0]])):
        if call.__code__.co_names[0] == "draft_accept":
            b.begin()
        before, graph = s.seq_info(h), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.add_(1)
            with pytest.raises(sq.SqError):
                call()
        assert s.seq_info(h) == before
        graph.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [4.0] * 4
    b.check()
    s.draft_accept([[0]])
    s.truncate(h, 20)
    assert s.seq_info(h)["length"] == 20


@pytest.mark.parametrize("kv8", [False, True])
def test_a_replay_for_a_larger_draft_stays_in_its_buffers(sq, kv8):
    """A capture is for drafts of its own counts.  Replayed with a larger one
    open, it writes nothing behind the rows it was captured with."""
    import torch
    b = Batch(sq, 16, 4, 128, [700], [64], kv8, seed=9)
    s, h = b.s, b.seqs[0]
    q, kn, vn = (torch.zeros(64, n, 128, device="cuda", dtype=torch.bfloat16) for n in (16, 4, 4))
    stored, out = torch.zeros_like(q), torch.zeros(64, 16, 128, device="cuda")
    for n in (5, 12, 33):
        s.draft_begin([h], [b.trees[0][:n]])
        s.qkv_store(0, q[:n], kn[:n], vn[:n], q_out=stored[:n])
        s.draft_attn(0, stored[:n], out=out[:n])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.qkv_store(0, q[:n], kn[:n], vn[:n], q_out=stored[:n])
            s.draft_attn(0, stored[:n], out=out[:n])
        s.draft_accept([[]])
        stored.fill_(7), out.fill_(7)
        s.draft_begin([h], b.trees)
        graph.replay()
        torch.cuda.synchronize()
        assert (stored[n:] == 7).all() and (out[n:] == 7).all()
        s.draft_accept([[]])
    b.begin()
    b.check()


def test_same_inputs_give_the_same_bits_on_any_stream(sq):
    import torch
    b = Batch(sq, 32, 8, 128, [5000, 3000], [30, 64], seed=6)
    b.begin()
    first = b.s.draft_attn(0, b.q[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = b.s.draft_attn(0, b.q[0])
    by_handle = b.s.draft_attn(0, b.q[0], stream=side)
    side.synchronize()
    assert torch.equal(first, again) and torch.equal(first, by_handle)


def test_device_refusals(sq):
    import torch
    b = Batch(sq, 8, 2, 64, [50], [5], seed=1)
    with pytest.raises(sq.SqError):
        b.s.draft_attn(0, b.q[0])
    b.begin(window=8, first=2)
    q = b.q[0]
    for bad in (dict(layer=1), dict(q=q[:4]), dict(q=q.float()), dict(out=torch.empty(5, 8, 64)), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=math.inf), dict(window=7, first=2), dict(window=8, first=1), dict(window=-1),
                dict(sinks=torch.zeros(7, device="cuda"))):
        with pytest.raises(sq.SqError):
            b.s.draft_attn(**dict(dict(layer=0, q=q), **bad))
    h = b.seqs[0]
    with pytest.raises(sq.SqError):
        b.s.decode(0, [h], q[:1].contiguous())
    with pytest.raises(sq.SqError):
        b.s.extend(0, h, q)
    b.check(window=8, first=2)
    b.s.draft_accept([[0]])
    with pytest.raises(sq.SqError):
        b.s.draft_attn(0, q)
    big = sq.Store(1, 128, 128, 64, num_pages=80, max_seqs=64, max_pages_per_seq=2)
    many = [big.seq_create() for _ in range(33)]
    with pytest.raises(sq.SqError):  # 33 x 128 rows of work
        big.draft_begin(many, [[-1]] * 33)
    big.draft_begin(many[:32], [[-1]] * 32)
    big.draft_accept([[]] * 32)


def test_stats_and_profile(sq):
    b = Batch(sq, 8, 2, 64, [50, 200], [5, 9], seed=1)
    b.s.profile_enable()
    b.begin()
    b.s.draft_attn(0, b.q[0])
    pr, st = b.s.profile_read(), b.s.stats()
    assert pr["qkv_launches"] == 1 and pr["draft_launches"] == 1 and pr["draft_ms"] > 0
    assert (st["draft_calls"], st["draft_tokens"], st["draft_kv_bytes"]) == (1, 14, 264 * 2 * 64 * 4)
    assert st["append_tokens"] == 250
    b.s.draft_accept([[0], []])
    assert b.s.stats()["append_tokens"] == 251
