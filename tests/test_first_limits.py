"""How many (range, KV head) pairs a decode step's windowed plan has room for,
first tokens beside the window being a range of their own (metadata-only store,
CPU)."""

import os

import pytest


@pytest.fixture(scope="module")
def sq():
    from paper_2602_22603_amd import build_lib, sq as sqmod
    if not os.path.exists(sqmod.LIB_PATH):
        build_lib.build()
    sqmod.lib()
    return sqmod


@pytest.mark.parametrize("batch,kw,fits", [
    (64, dict(window=4), True), (64, dict(window=4, first=2), False), (63, dict(window=4, first=2), True),
    (64, dict(window=30, first=39), True),  # (they meet: one range)
    (64, dict(window=100, first=2), True), (64, dict(first=2), True)])
def test_ranges_of_a_step(sq, batch, kw, fits):
    s = sq.Store(1, 64, 64, 8, num_pages=200, max_seqs=64, max_pages_per_seq=4, metadata_only=True)
    seqs = [s.seq_create() for _ in range(batch)]
    for h in seqs:
        s.append(h, n=40)
    if fits:
        s.step_begin(seqs, **kw)
        assert all(s.seq_info(h)["length"] == 41 for h in seqs)
    else:
        with pytest.raises(sq.SqError) as e:
            s.step_begin(seqs, **kw)
        assert e.value.code == sq.ERR_INVALID and all(s.seq_info(h)["length"] == 40 for h in seqs)
    s.close()
