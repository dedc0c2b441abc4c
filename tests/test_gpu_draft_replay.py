"""A layer captured for one draft and replayed while another is open: with other
numbers of nodes, tiles or windows it writes no output at all, and the open
draft's own results are as without it."""

import pytest

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


def _chain(n):
    return [-1] + list(range(n - 1))


@pytest.mark.parametrize("hq,hkv,d,kv8,length,captured,opened", [
    (8, 1, 64, False, 150000, [64], [5]),    # wide tiles captured, narrow ones in many pieces open
    (8, 1, 64, False, 150000, [5], [64]),
    (4, 1, 64, False, 150000, [64], [3]),
    (16, 2, 128, True, 3000, [2] * 8, [16]), # as many nodes, other tiles
    (16, 2, 128, True, 3000, [16], [2] * 8),
    (32, 8, 128, False, 9000, [16, 3], [16]),
    (32, 8, 128, True, 9000, [1], [40, 64, 7]),
    (64, 8, 64, True, 2000, [64] * 4, [33])])
def test_for_another_draft_nothing_is_written(sq, hq, hkv, d, kv8, length, captured, opened):
    import torch
    n_seqs = max(len(captured), len(opened))
    pages = -(-(length + 64) // 16) + 1
    s = sq.Store(1, hq, hkv, d, num_pages=pages * n_seqs, max_seqs=n_seqs, max_pages_per_seq=pages,
                 kv_scales=[(0.11, 0.07)] if kv8 else None)
    seqs = [s.seq_create() for _ in range(n_seqs)]
    for i, h in enumerate(seqs):
        s.append(h, *(wl.device_normal_bf16((1, length, hkv, d), 2 * i + j, "cuda") for j in (0, 1)))
    most = max(sum(captured), sum(opened))
    q, k, v = (wl.device_normal_bf16((most, n, d), 90 + n, "cuda") for n in (hq, hkv, hkv))
    out = torch.empty(most, hq, d, device="cuda")
    n, m = sum(captured), sum(opened)

    def begin(sizes, **kw):
        s.draft_begin(seqs[:len(sizes)], [_chain(c) for c in sizes], **kw)
        s.qkv_store(0, q[:sum(sizes)], k[:sum(sizes)], v[:sum(sizes)])

    begin(opened)
    want = s.draft_attn(0, q[:m])
    s.draft_accept([[]] * len(opened))
    begin(captured, window=100, first=4)
    graphs = []
    for kw in (dict(), dict(window=100, first=4)):
        s.draft_attn(0, q[:n], out=out[:n], **kw)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.draft_attn(0, q[:n], out=out[:n], **kw)
    own = [s.draft_attn(0, q[:n], **kw) for kw in (dict(), dict(window=100, first=4))]
    s.draft_accept([[]] * len(captured))
    for kw in (dict(window=100, first=4), dict()):
        out.fill_(7)
        begin(opened, **kw)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert (out == 7).all()
        assert torch.equal(s.draft_attn(0, q[:m]), want)
        s.draft_accept([[]] * len(opened))
    begin(captured)  # (no window: that layer's replay has nothing to do)
    graphs[0].replay()
    assert torch.equal(out[:n], own[0])
    out.fill_(7)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert (out == 7).all()
    s.draft_accept([[]] * len(captured))
    begin(captured, window=100, first=4)
    for g, w in zip(graphs, own):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:n], w)
    s.draft_accept([[]] * len(captured))
