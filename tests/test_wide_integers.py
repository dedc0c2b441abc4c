"""The binding refuses integers that the library's arguments cannot hold, where
they would wrap to another value (metadata-only store, CPU)."""

import os

import pytest

P, MAXP = 4, 16
WRAPS = 1 << 32


@pytest.fixture(scope="module")
def sq():
    from paper_2602_22603_amd import build_lib, sq as sqmod
    if not os.path.exists(sqmod.LIB_PATH):
        build_lib.build()
    sqmod.lib()
    return sqmod


@pytest.fixture
def store(sq):
    s = sq.Store(2, 4, 2, 8, num_pages=40, max_seqs=3, max_pages_per_seq=MAXP, page_size=P, metadata_only=True)
    h = s.seq_create()
    s.append(h, n=9)
    yield s, h
    s.close()


def _refused(sq, s, h, fn):
    before = (s.seq_info(h), s.page_table(h), s.positions(h).tolist(), s.refcounts().tolist())
    with pytest.raises(sq.SqError) as e:
        fn()
    assert e.value.code == sq.ERR_INVALID
    assert (s.seq_info(h), s.page_table(h), s.positions(h).tolist(), s.refcounts().tolist()) == before


@pytest.mark.parametrize("kw", [dict(window=WRAPS), dict(window=WRAPS + 4), dict(window=4, first=WRAPS + 4),
                                dict(window=WRAPS + 4, first=2), dict(window=1 << 31), dict(window=4, first=1 << 31),
                                dict(window=4 - WRAPS), dict(first=WRAPS)])
def test_windows_and_first_tokens(sq, store, kw):
    """(_opts is what decode, step_attn, extend and draft_attn build theirs with.)"""
    s, h = store
    for fn in (lambda: s.step_begin([h], **kw), lambda: s.draft_begin([h], [[-1]], **kw),
               lambda: s._opts(kw.get("window", 0), None, kw.get("first", 0))):
        _refused(sq, s, h, fn)


def test_lengths_counts_and_handles(sq, store):
    s, h = store
    for fn in (lambda: s.truncate(h, 1 << 64), lambda: s.truncate(h, (1 << 64) + 3), lambda: s.truncate(h + WRAPS, 3),
               lambda: s.truncate(h, -(1 << 64)), lambda: s.reserve([h], [WRAPS + 1]), lambda: s.reserve([h + WRAPS], [1]),
               lambda: s.draft_begin([h + WRAPS], [[-1]]), lambda: s.step_begin([h + WRAPS])):
        _refused(sq, s, h, fn)
    s.reserve([h], [3])
    s.truncate(h, 9)
    assert s.positions(h).tolist() == list(range(9))


def test_handles_and_layers_are_whole(sq, store):
    """As ctypes has it for every other call: no number is cut to an integer."""
    s, h = store
    for handle in (h + 0.5, "0", None):
        with pytest.raises(TypeError):
            s.truncate(handle, 3)
    assert s.seq_info(h)["length"] == 9


def test_integers_that_fit_stay_as_they_were(sq, store):
    import numpy as np
    s, h = store
    s.step_begin([np.int64(h)], window=np.int32(4), first=2 ** 31 - 1)
    s.draft_begin([h], [[-1, 0]], window=2 ** 31 - 1, first=np.int64(3))
    s.draft_accept([[0]])
    s.truncate(np.int64(h), np.int64(2))
    assert s.seq_info(h)["length"] == 2
