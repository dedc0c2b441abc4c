"""draft_begin and draft_accept take any iterables (metadata-only store, CPU)."""

import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def sq():
    from paper_2602_22603_amd import build_lib, sq as sqmod
    if not os.path.exists(sqmod.LIB_PATH):
        build_lib.build()
    sqmod.lib()
    return sqmod


TREES = [[-1, 0, 0, 1], [-1, -1]]
FORMS = [lambda t: t, lambda t: (x for x in t), lambda t: map(list, t), lambda t: [iter(x) for x in t],
         lambda t: [np.array(x) for x in t], lambda t: tuple(map(tuple, t)), lambda t: (iter(x) for x in t)]


@pytest.mark.parametrize("form", FORMS)
def test_trees_and_paths(sq, form):
    s = sq.Store(1, 4, 2, 8, num_pages=20, max_seqs=3, max_pages_per_seq=10, page_size=4, metadata_only=True)
    a, b = s.seq_create(), s.seq_create()
    s.append(a, n=6)
    s.draft_begin(iter([a, b]), form(TREES))
    assert s.positions(a).tolist() == list(range(6)) + [6, 7, 7, 8] and s.positions(b).tolist() == [0, 0]
    s.draft_accept(form([[0, 1, 3], [1]]))
    assert s.positions(a).tolist() == list(range(9)) and s.positions(b).tolist() == [0]
    s.close()
