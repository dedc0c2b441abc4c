"""Host side of reserved tokens, drafts and truncation on a metadata-only store
(CPU): lengths, pages, refcounts and positions against a list-of-tokens model
over random call sequences, and every refusal changing nothing."""

import os
import random

import numpy as np
import pytest

from oracle import draft as odr

PAGES, P, SEQS, MAXP = 60, 4, 6, 16


@pytest.fixture(scope="module")
def sq():
    from paper_2602_22603_amd import build_lib, sq as sqmod
    if not os.path.exists(sqmod.LIB_PATH):
        build_lib.build()
    sqmod.lib()
    return sqmod


def _store(sq, pages=PAGES, page=P, maxp=MAXP):
    return sq.Store(2, 4, 2, 8, num_pages=pages, max_seqs=SEQS, max_pages_per_seq=maxp, page_size=page,
                    metadata_only=True)


def _tree(rng, n):
    return [-1] + [rng.randrange(-1, i) for i in range(1, n)]


def _state(s):
    out = {"ref": s.refcounts().tolist(), "stats": s.stats()}
    for h in range(SEQS):
        try:
            out[h] = (s.seq_info(h), s.page_table(h), s.positions(h).tolist(), s.spans(h))
        except Exception:  # noqa: BLE001 - not live
            out[h] = None
    return out


def _refused(s, code, fn, *args, **kw):
    before = _state(s)
    with pytest.raises(Exception) as e:
        fn(*args, **kw)
    assert e.value.code == code, str(e.value)
    assert _state(s) == before


@pytest.mark.parametrize("seed", range(12))
def test_random_calls_match_a_list_of_tokens(sq, seed):
    """Appends, reservations, forks, truncations, drafts accepted whole, in
    part or not at all, releases: the positions are the model's, each sequence
    has the pages its length needs and every page the references it has."""
    rng = random.Random(seed)
    s = _store(sq)
    pos, nxt = {}, {}
    for _ in range(250):
        op = rng.choice(["create", "append", "reserve", "fork", "truncate", "draft", "draft", "release"])
        live = sorted(pos)
        try:
            if op == "create":
                h = s.seq_create()
                pos[h], nxt[h] = [], 0
            elif not live:
                continue
            elif op == "append":
                h, n = rng.choice(live), rng.randrange(0, 9)
                s.append(h, n=n)
                pos[h] += range(nxt[h], nxt[h] + n)
                nxt[h] += n
            elif op == "reserve":
                hs = rng.sample(live, rng.randrange(1, len(live) + 1))
                ns = [rng.randrange(1, 7) for _ in hs]
                s.reserve(hs, ns)
                for h, n in zip(hs, ns):
                    pos[h] += range(nxt[h], nxt[h] + n)
                    nxt[h] += n
            elif op == "fork":
                h = rng.choice(live)
                n = rng.randrange(0, len(pos[h]) + 1)
                c = s.fork(h, n)
                pos[c] = pos[h][:n]
                nxt[c] = nxt[h] if n == len(pos[h]) else pos[h][n]
            elif op == "truncate":
                h = rng.choice(live)
                n = rng.randrange(0, len(pos[h]) + 1)
                s.truncate(h, n)
                if n < len(pos[h]):
                    nxt[h] = pos[h][n]
                pos[h] = pos[h][:n]
            elif op == "release":
                h = rng.choice(live)
                s.release(h)
                del pos[h], nxt[h]
            else:
                hs = rng.sample(live, rng.randrange(1, len(live) + 1))
                trees = [_tree(rng, rng.randrange(1, 10)) for _ in hs]
                s.draft_begin(hs, trees)
                for h, t in zip(hs, trees):  # a node's position: the next one, plus its depth
                    assert s.positions(h).tolist() == pos[h] + [nxt[h] + d for d in odr.depths(t)]
                    assert s.seq_info(h)["length"] == len(pos[h]) + len(t)
                paths = [odr.path_to(t, rng.randrange(-1, len(t))) for t in trees]
                s.draft_accept(paths)
                for h, p in zip(hs, paths):
                    pos[h] += range(nxt[h], nxt[h] + len(p))
                    nxt[h] += len(p)
        except sq.SqError as e:
            assert e.code in (sq.ERR_NO_PAGES, sq.ERR_INVALID), str(e)
        refs = np.zeros(PAGES, dtype=np.int64)
        for h in pos:
            info = s.seq_info(h)
            assert s.positions(h).tolist() == pos[h]
            assert (info["length"], info["next_pos"]) == (len(pos[h]), nxt[h])
            table = s.page_table(h)
            assert len(table) == -(-len(pos[h]) // P)
            refs[table] += 1
            if len(pos[h]) % P:  # the page appended to next is the sequence's own
                assert s.refcounts()[table[-1]] == 1
        assert s.refcounts().tolist() == refs.tolist()
    s.close()


def test_reserve_refusals(sq):
    s = _store(sq)
    a, b = s.seq_create(), s.seq_create()
    s.append(a, n=5)
    _refused(s, sq.ERR_INVALID, s.reserve, [], [])
    _refused(s, sq.ERR_INVALID, s.reserve, [a, a], [1, 1])
    _refused(s, sq.ERR_INVALID, s.reserve, [a, b], [1, 0])
    _refused(s, sq.ERR_INVALID, s.reserve, [a], [-2])
    _refused(s, sq.ERR_INVALID, s.reserve, [a], [MAXP * P])
    _refused(s, sq.ERR_INVALID, s.reserve, [a], [sq.MAX_RESERVE + 1])
    _refused(s, sq.ERR_UNKNOWN_SEQ, s.reserve, [a, 5], [1, 1])
    _refused(s, sq.ERR_INVALID, s.reserve, [a] * 65, [1] * 65)
    with pytest.raises(sq.SqError):
        s.reserve([a, b], [1])
    c = s.seq_create()
    d = s.seq_create()
    for h in (b, c, d):
        s.append(h, n=MAXP * P)
    s.append(a, n=6 * P - 5)
    _refused(s, sq.ERR_NO_PAGES, s.reserve, [a], [6 * P + 1])
    s.reserve([a], [6 * P])
    with pytest.raises(sq.SqError):  # no pools: nothing to store
        s.qkv_store(0, None, None, None)
    assert sq.lib().sq_qkv_store(s._handle, 0, 16, 64, 16, 64, 16, 64, None, 16, None) == sq.ERR_INVALID
    assert sq.lib().sq_reserve(None, None, None, 1, None) == sq.ERR_INVALID
    s.close()


def test_draft_refusals(sq):
    """Bad trees, batches and paths; and an open draft's sequences refuse every
    other call, while others go on."""
    s = _store(sq)
    a, b, c = s.seq_create(), s.seq_create(), s.seq_create()
    s.append(a, n=6)
    s.append(c, n=3)
    _refused(s, sq.ERR_INVALID, s.draft_begin, [], [])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[]])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[0]])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1, 2, 0]])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-2]])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a, a], [[-1], [-1]])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1] * (sq.MAX_DRAFT + 1)])
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1]], window=-1)
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1]], window=4, first=-1)
    _refused(s, sq.ERR_UNKNOWN_SEQ, s.draft_begin, [a, 5], [[-1], [-1]])
    with pytest.raises(sq.SqError):
        s.draft_accept([[0]])
    assert sq.lib().sq_draft_accept(s._handle, sq._i32_array([1]), sq._i32_array([0]), None) == sq.ERR_INVALID
    s.draft_begin([a, b], [[-1, 0, 0, 1], [-1, -1]])
    for fn, args in ((s.append, (a, None, None, 2)), (s.append_batch, ([c, a],)), (s.fork, (a, 2)),
                     (s.release, (a,)), (s.evict, (a, [])), (s.compact, (b,)), (s.truncate, (a, 1)),
                     (s.span_mark, (a, 1, 0, 2)), (s.step_begin, ([a],)), (s.reserve, ([c], [1])),
                     (s.reserve, ([a], [1])), (s.draft_begin, ([c], [[-1]])), (s.draft_begin, ([a], [[-1]])),
                     (s.draft_accept, ([[0, 2, 3], []],)), (s.draft_accept, ([[1], []],)),
                     (s.draft_accept, ([[0, 4], []],)), (s.draft_accept, ([[0], [0, 1]],)),
                     (s.draft_accept, ([[0, 0], []],)), (s.draft_accept, ([[0, -1], []],))):
        _refused(s, sq.ERR_INVALID, fn, *args)
    with pytest.raises(sq.SqError):
        s.draft_accept([[0]])
    s.append(c, n=4)  # another sequence
    d = s.fork(c, 2)
    s.release(d)
    s.draft_accept([[0, 1, 3], [1]])
    assert s.positions(a).tolist() == list(range(9)) and s.positions(b).tolist() == [0]
    assert s.seq_info(a)["next_pos"] == 9
    s.draft_begin([c], [[-1, 0]])
    s.draft_accept([[]])  # abandoned
    assert s.seq_info(c)["length"] == 7 and s.seq_info(c)["next_pos"] == 7
    s.reserve([c], [1])
    s.close()


def test_draft_pages_and_capacity(sq):
    s = _store(sq, pages=5)
    a, b = s.seq_create(), s.seq_create()
    s.append(a, n=7)
    s.append(b, n=8)
    _refused(s, sq.ERR_NO_PAGES, s.draft_begin, [a], [[-1] * 6])
    s.draft_begin([a, b], [[-1], [-1] * 4])  # the last page
    _refused(s, sq.ERR_INVALID, s.append, b, None, None, 1)
    s.draft_accept([[0], []])
    assert s.stats()["free_pages"] == 1
    s.close()
    s = _store(sq, maxp=2)
    a = s.seq_create()
    s.append(a, n=7)
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1, 0]])
    s.draft_begin([a], [[-1]])
    s.draft_accept([[0]])
    s.close()


def test_truncate_spans_masks_and_shared_pages(sq):
    """A span past the new end refuses; masked slots behind it are forgotten;
    a part-full last page that a branch shares becomes the sequence's own."""
    s = _store(sq)
    a = s.seq_create()
    s.append(a, n=16)
    s.span_mark(a, 0, 2, 5)
    s.span_mark(a, 1, 9, 13)
    _refused(s, sq.ERR_SPAN, s.truncate, a, 12)
    _refused(s, sq.ERR_INVALID, s.truncate, a, 17)
    _refused(s, sq.ERR_INVALID, s.truncate, a, -1)
    _refused(s, sq.ERR_UNKNOWN_SEQ, s.truncate, 4, 0)
    s.evict(a, [0, 1], deferred=True)
    assert s.seq_info(a)["n_masked"] == 7
    b = s.fork(a, 16)
    s.truncate(b, 10)
    assert s.seq_info(b)["n_masked"] == 4 and s.keep_flags(b).tolist() == [1, 1, 0, 0, 0, 1, 1, 1, 1, 0]
    assert s.page_table(b)[:2] == s.page_table(a)[:2] and s.page_table(b)[2] != s.page_table(a)[2]
    s.append(b, n=3)
    assert s.keep_flags(b).tolist() == [1, 1, 0, 0, 0, 1, 1, 1, 1, 0, 1, 1, 1]
    assert s.seq_info(a)["n_masked"] == 7 and s.positions(b).tolist() == list(range(13))
    s.truncate(b, 2)
    assert s.seq_info(b)["n_masked"] == 0 and s.seq_info(b)["next_pos"] == 2
    s.compact(a)
    assert s.positions(a).tolist() == [0, 1, 5, 6, 7, 8, 13, 14, 15]
    s.truncate(a, 3)
    assert s.seq_info(a)["next_pos"] == 6  # the first dropped token's
    s.truncate(a, 3)
    s.truncate(a, 0)
    assert s.seq_info(a)["next_pos"] == 0 and s.page_table(a) == []
    s.close()
    s = _store(sq, pages=4)
    a = s.seq_create()
    s.append(a, n=16)
    b = s.fork(a, 16)
    _refused(s, sq.ERR_NO_PAGES, s.truncate, b, 14)
    s.truncate(b, 12)
    s.close()


def test_a_draft_over_masked_slots_takes_no_window(sq):
    s = _store(sq)
    a = s.seq_create()
    s.append(a, n=16)
    s.span_mark(a, 0, 2, 5)
    s.evict(a, [0], deferred=True)
    _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [[-1]], window=4)
    s.draft_begin([a], [[-1, 0]])
    s.draft_accept([[0]])
    assert s.seq_info(a)["n_masked"] == 3 and s.seq_info(a)["length"] == 17
    s.close()


def test_qk_rope_refusals(sq):
    """Checked before anything is launched, so no GPU is needed."""
    import ctypes as C
    f = sq.lib().sq_qk_rope
    good = dict(q=16, qs=512, k=32, ks=128, pos=4, n=3, hq=4, hkv=1, d=128, qo=48, ko=64)

    def call(opts=None, **kw):
        a = dict(good, **kw)
        return f(a["q"], a["qs"], a["k"], a["ks"], a["pos"], a["n"], a["hq"], a["hkv"], a["d"],
                 None if opts is None else C.byref(opts), a["qo"], a["ko"], None)

    for bad in (dict(n=-1), dict(hq=0), dict(hkv=0), dict(d=96), dict(q=0), dict(q=8), dict(k=24), dict(qo=None),
                dict(ko=40), dict(pos=None), dict(pos=6), dict(qs=504), dict(qs=515), dict(ks=120), dict(ks=-128)):
        assert call(**bad) == sq.ERR_INVALID, bad
    for o in (dict(inv_freq=4, rot_dim=0), dict(inv_freq=4, rot_dim=12), dict(inv_freq=4, rot_dim=136),
              dict(inv_freq=6, rot_dim=64), dict(q_weight=2), dict(k_weight=1), dict(eps=-1.0), dict(eps=float("nan")),
              dict(inv_freq=4, rot_dim=64, interleaved=2), dict(inv_freq=4, rot_dim=64, mscale=float("inf"))):
        assert call(opts=sq.QkOpts(**o)) == sq.ERR_INVALID, o
    assert call(n=0, q=0) == sq.OK


def test_qk_rope_refuses_sizes_past_its_grid(sq):
    def call(n, hq, hkv):
        return sq.lib().sq_qk_rope(16, 1 << 24, 32, 1 << 24, 4, n, hq, hkv, 128, None, 48, 64, None)

    for bad in (((1 << 24) + 1, 1, 1), (2**31 - 1, 1, 1), (1, 65537, 1), (1, 1, 65537)):
        assert call(*bad) == sq.ERR_INVALID, bad


def test_trees_and_paths_are_integers(sq):
    """Nodes that are no 32-bit integers are refused before the library sees them."""
    s = _store(sq)
    a = s.seq_create()
    for bad in ([-1, 0.5], [-1, 1 << 31], [None], ["0"]):
        _refused(s, sq.ERR_INVALID, s.draft_begin, [a], [bad])
    s.draft_begin([a], [(-1, 0)])
    _refused(s, sq.ERR_INVALID, s.draft_accept, [[0.0]])
    s.draft_accept([(0, 1)])
    assert s.seq_info(a)["length"] == 2
    s.close()


def test_first_tokens_of_a_window_are_checked(sq):
    """A metadata-only store checks step options before it opens the step."""
    import ctypes as C
    s = _store(sq)
    a = s.seq_create()
    s.append(a, n=9)
    _refused(s, sq.ERR_INVALID, s.step_begin, [a], window=4, first=-1)
    o = sq.AttnOpts()
    o.window, o.reserved2 = 4, 1
    assert sq.lib().sq_step_begin_opts(s._handle, sq._i32_array([a]), 1, 0, C.byref(o), None) == sq.ERR_INVALID
    s.step_begin([a], window=4, first=2)
    assert s.seq_info(a)["length"] == 10
    s.close()
